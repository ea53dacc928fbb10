// The pass over the bank as a matrix product of tiles, for large bf16 batches
// (gfx950, wave64).
#pragma once

#include "attend_scan.hpp"

namespace rb {

namespace {

constexpr int AG_ROWS = 256, AG_REQS = 256;   // of a workgroup's tile
constexpr int AG_RT = 8, AG_NG = 4;           // 16-row tiles and request groups of a wave
constexpr int AG_K = 64;                      // elements of a stage
constexpr int AG_SLOT = (AG_ROWS + AG_REQS) * AG_K * 2;   // bytes of a stage in LDS

// A lane number that the compiler takes for new: what is computed from it is
// computed again each time, where kept through the products it would take the
// registers of their fragments.
__device__ __forceinline__ int fresh(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// What a tile brings beside its rows: their norms, the mask bytes (from an
// aligned word on, mask_shift bytes before the first), and up to 64 pieces of 64
// label words, as the kernel wants them.
struct TileSide {
    float norms[AG_ROWS];
    uint32_t mask[128];
    float spare[WAVE];
};

// 4 bytes per lane from the lane's own address to dst + 4 * lane.
__device__ __forceinline__ void dma4(const void *src, void *dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                     (__attribute__((address_space(3))) void *)dst, 4, 0, 0);
}

// A workgroup of 8 waves (two per SIMD) takes tiles of 256 bank rows against
// its 256 requests, wave w the 128 rows 128 * (w/4) .. and the 64 requests 64 *
// (w%4) ..: 32 accumulators of 16 x 16. A stage brings 128 bytes of each of the
// 512 rows and requests into one of two LDS slots, whole lines (8 rows a load;
// row ri of load f keeps its 16-byte chunk c at 8*ri + (c ^ x), x one of 0, 1, 4,
// 5 by row pair, ^ 2 in odd loads, so that a fragment read meets every bank
// once). A stage is two k-steps of 32; of each a wave reads 12 fragments for 32
// MFMAs, every one while the products before it run, the first of a stage in the
// stage before. The one barrier of a stage sits where its last fragments are
// read: behind it the slot just read takes the stage after next and the next
// stage's fragments come in.
// (Stages of 32 elements in four slots, half lines two and a half stages ahead:
// 256 x 1,000,000 x 768 535 us for 494, 1,024 x 250,000 x 768 475 for 432; with the
// barrier between stages and all waves' fragments read behind it 571 and more.)
// The accumulators have the layout of scan_slabs, so that what takes them is
// alike.
// In a tile's first stage its side data is sent for, LAB pieces of labels by
// every wave: label(row, piece, lane) is a lane's address in piece `piece`, and they
// land at labels + 64 * piece; end(tile, acc), behind the last stage, reads
// them. nst: stages of a tile, at least 2.
template <bool BANK_COLS, int LAB, typename Label, typename End>
__device__ __forceinline__ void gemm_tiles(const AttendBank &A, int nst, uint8_t *ring,
                                           TileSide *side, float *labels, int q0, long tile0,
                                           int n_tiles, int wave, int lane, Label &&label,
                                           End &&end)
{
    const uint32_t rowb = (uint32_t)A.d * 2;
    constexpr int RT = AG_RT, LOADS = 8, STEPS = 2 * RT;
    const int wr = wave >> 2, wq = wave & 3;
    const int col = lane & 15, jg = lane >> 4;
    const int nq = min(A.B - q0, AG_REQS);
    const __amdgpu_buffer_rsrc_t rqr =
        make_rsrc(A.queries + (size_t)q0 * rowb, (uint32_t)nq * rowb);
    auto turn = [](int ri) { return ((ri >> 1) & 1) | ((ri >> 2) << 2); };   // 0, 1, 4, 5
    // load f = wave + 8*j brings rows (or requests) 8*f .., lane l row l/8 of
    // them, chunk (l % 8) ^ x
    const int ri = lane >> 3, chunk = (lane & 7) ^ turn(ri) ^ ((wave & 1) << 1);
    const uint32_t lo = (uint32_t)(8 * wave + ri) * rowb + (uint32_t)chunk * 16;
    int it = 0, ik = 0;   // the stage to send for: tile, part of K
    auto issue = [&](uint32_t slot) {
        const long row0 = (tile0 + it) * AG_ROWS;
        const bool in = it < n_tiles;
        const int rows = in ? (int)min((long)AG_ROWS, A.N - row0) : 0;
        const __amdgpu_buffer_rsrc_t rbk =
            make_rsrc(A.rows + (size_t)(in ? row0 : 0) * rowb, (uint32_t)rows * rowb);
        const uint32_t at = lo + (uint32_t)ik * (AG_K * 2);
        const bool some = (uint32_t)(ik * (AG_K * 2) + chunk * 16) < rowb && in;
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
            dma16(j < 4 ? rbk : rqr, (i32x4 *)(ring + slot) + (wave + 8 * j) * WAVE,
                  some ? at + (uint32_t)((j & 3) * 64) * rowb : OFF_NONE);
        if (++ik == nst) {
            ik = 0;
            ++it;
        }
    };
    // fragment addresses of k-step 0: row tile i of a wave's lies 2 KB behind the
    // one before; k-step 1 differs in bit 6
    auto place = [&](int r) {
        const int g = r >> 3, x = turn(r & 7) ^ ((g & 1) << 1);
        return (uint32_t)(g * 1024 + (r & 7) * 128 + ((jg ^ x) * 16));
    };
    const uint32_t pa = place(16 * RT * wr + col),
                   pb = (uint32_t)(AG_ROWS * AG_K * 2) + place(64 * wq + col);
    // waves 0 to 3 bring 64 norms each, 4 and 5 the mask's words (each word holds
    // a byte of the mask), the others a word that nothing reads
    const uint32_t *const mask4 = (const uint32_t *)((uintptr_t)A.mask & ~(uintptr_t)3);
    const long mask_last = ((long)A.N - 1 + ((uintptr_t)A.mask & 3)) / 4;
    auto side_loads = [&](int tile) {
        const long row0 = (tile0 + tile) * AG_ROWS;
        const void *src = A.norms;
        void *dst = side->spare;
        if (wave < 4) {
            src = A.norms + min(row0 + wave * 64 + lane, (long)A.N - 1);
            dst = side->norms + wave * 64;
        } else if (A.mask && wave < 6) {
            src = mask4 + min(row0 / 4 + (wave - 4) * 64 + lane, mask_last);
            dst = side->mask + (wave - 4) * 64;
        }
        dma4(src, dst);
        const int l = fresh(lane);
#pragma unroll
        for (int j = 0; j < LAB; ++j)
            dma4(label(row0, wave * LAB + j, l), labels + (wave * LAB + j) * WAVE);
    };
    f32x4 acc[RT][AG_NG];
    const int n_stg = n_tiles * nst;
    i32x4 a[4], b[AG_NG];   // fragments: a wave's row tiles in turn, its requests
    auto read_a = [&](uint32_t slot, uint32_t s, int i) {
        return *(const i32x4 *)(ring + slot + (pa ^ s) + i * 2048);
    };
    auto read_b = [&](uint32_t slot, uint32_t s, int g) {
        return *(const i32x4 *)(ring + slot + (pb ^ s) + g * 2048);
    };
    // a stage's first fragments
    auto open = [&](uint32_t slot) {
#pragma unroll
        for (int g = 0; g < AG_NG; ++g)
            b[g] = read_b(slot, 0, g);
        a[0] = read_a(slot, 0, 0);
        a[1] = read_a(slot, 0, 1);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int g = 0; g < AG_NG; ++g)
                acc[i][g] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    issue(0);
    issue(AG_SLOT);
    wait_vmcnt<LOADS>();
    stream_barrier();
    uint32_t slot = 0;
    open(slot);
    for (int z = 0, tile = 0, kc = 0; z < n_stg; ++z) {
        const uint32_t next = AG_SLOT - slot;
        // the products of step n (row tile n % RT of k-step n / RT), and the reads
        // of the step after the next, behind the last of the next stage's
        auto products = [&](auto I) {
            constexpr int n = decltype(I)::value, i = n % RT, m = (n + 2) % STEPS;
#pragma unroll
            for (int g = 0; g < AG_NG; ++g) {
                acc[i][g] = BANK_COLS ? mfma_step<1>(b[g], a[n % 4], acc[i][g])
                                      : mfma_step<1>(a[n % 4], b[g], acc[i][g]);
                if constexpr (i == RT - 1)
                    b[g] = n == RT - 1 ? read_b(slot, 64, g) : read_b(next, 0, g);
            }
            a[m % 4] = n + 2 < STEPS ? read_a(slot, m < RT ? 0u : 64u, m % RT)
                                     : read_a(next, 0, m);
        };
        auto order = [&](auto I) {   // as written
            constexpr int i = decltype(I)::value % RT;
            if constexpr (i == RT - 1) {
                static_for<0, AG_NG>([&](auto) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                });
            } else {
                __builtin_amdgcn_sched_group_barrier(0x008, AG_NG, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        };
        constexpr int LAST = STEPS - 2;   // steps whose fragments this slot holds
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, LAST>(products);
        static_for<0, LAST>(order);
        __builtin_amdgcn_sched_barrier(0);
        // the next stage has landed and this one is read, behind the barrier by
        // every wave
        wait_vmcnt<0>();
        stream_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (kc == 0)
            side_loads(tile);
        issue(slot);
        __builtin_amdgcn_sched_barrier(0);
        static_for<LAST, STEPS>(products);
        static_for<LAST, STEPS>(order);
        __builtin_amdgcn_sched_barrier(0);
        slot = next;
        if (++kc == nst) {
            kc = 0;
            end(tile, acc);
            ++tile;
            open(slot);
        }
    }
    wait_vmcnt<0>();   // (no global-to-LDS load in flight when the workgroup ends)
}

// x and y rounded to two bf16 values (x in the low half); what that leaves of
// them in their places.
__device__ __forceinline__ int split_bf16(float &x, float &y)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const int w = __builtin_bit_cast(int, bf16x2{(__bf16)x, (__bf16)y});
    x -= __int_as_float(w << 16);
    y -= __int_as_float(w & (int)0xffff0000);
    return w;
}

// -|x|^2/2 of rows r .. r+3 of a tile with `left` rows of the bank (the others
// lie past it), -inf for rows masked or past it.
__device__ __forceinline__ f32x4 tile_norms(const AttendBank &A, const TileSide *side, int left,
                                            int r)
{
    const f32x4 n = *(const f32x4 *)(side->norms + r);
    uint32_t four = ~0u;
    if (A.mask)
        four = __builtin_amdgcn_alignbyte(side->mask[r / 4 + 1], side->mask[r / 4],
                                          (uint32_t)((uintptr_t)A.mask & 3));
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        h[e] = r + e < left && (four >> (8 * e) & 0xffu) != 0 ? -0.5f * n[e] : -INFINITY;
    return h;
}

// The same of one row, for kernels with the bank's rows over the lanes.
__device__ __forceinline__ float tile_norm(const AttendBank &A, const TileSide *side, int left,
                                           int r)
{
    const uint32_t at = (uint32_t)r + (uint32_t)((uintptr_t)A.mask & 3);
    const bool ok = r < left && (!A.mask || ((const uint8_t *)side->mask)[at] != 0);
    return ok ? -0.5f * side->norms[r] : -INFINITY;
}

// A resource for a region that is the same for the whole wave, by scalar registers
// (one whose address the compiler computes in vector registers becomes a loop
// over the lanes at every use).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t wave_rsrc(const void *base, uint32_t bytes)
{
    const uint64_t p = (uint64_t)base;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p),
                   hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
    return make_rsrc((const void *)((uint64_t)hi << 32 | lo),
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes));
}

// 4 bytes to a lane's place in a resource (nothing past it).
__device__ __forceinline__ void buffer_store4(__amdgpu_buffer_rsrc_t r, uint32_t at, float v)
{
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, (int)at, 0, 0);
}

}  // namespace

}  // namespace rb
