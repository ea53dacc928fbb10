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
static_assert(AG_SLOT == 1 << 16, "a slot is one address bit");

// A workgroup of 8 waves (two per SIMD) takes tiles of 256 bank rows against
// its 256 requests, wave w the 128 rows 128 * (w/4) .. and the 64 requests 64 *
// (w%4) ..: 32 accumulators of 16 x 16. A stage brings 128 bytes of each of the
// 512 rows and requests into one of two LDS slots, whole 128-byte lines (8 rows
// a load; row ri of load f keeps its 16-byte chunk c at 8*ri + (c ^ x), x one
// of 0, 1, 4, 5 by row pair, ^ 2 in odd loads, so that a fragment read meets
// every bank once); its loads go out while the stage before is computed. Per
// k-step of 32 a wave reads 12 fragments for 32 MFMAs. The accumulators have the
// layout of scan_slabs, so that what takes them is alike.
// first(tile) and then(tile) run in a tile's first and second stage (what the
// first sends for has landed by the second; then may write LDS that end reads),
// end(tile, acc) behind its last. nst: stages of a tile, at least 2.
template <bool BANK_COLS, typename First, typename Then, typename End>
__device__ __forceinline__ void gemm_tiles(const AttendBank &A, int nst, uint8_t *ring, int q0,
                                           long tile0, int n_tiles, int wave, int lane,
                                           First &&first, Then &&then, End &&end)
{
    const uint32_t rowb = (uint32_t)A.d * 2;
    const int wr = wave >> 2, wq = wave & 3;
    const int col = lane & 15, jg = lane >> 4;
    auto turn = [](int ri) { return ((ri >> 1) & 1) | ((ri >> 2) << 2); };   // 0, 1, 4, 5
    const int nq = min(A.B - q0, AG_REQS);
    const __amdgpu_buffer_rsrc_t rqr =
        make_rsrc(A.queries + (size_t)q0 * rowb, (uint32_t)nq * rowb);
    // load f = wave + 8*j brings rows (or requests) 8*f .., lane l row l/8 of
    // them, chunk (l % 8) ^ x
    const int ri = lane >> 3, chunk = (lane & 7) ^ turn(ri) ^ ((wave & 1) << 1);
    const uint32_t lo = (uint32_t)(8 * wave + ri) * rowb + (uint32_t)chunk * 16;
    int it = 0, ik = 0;   // the stage to send for: tile, part of K
    auto issue = [&](int slot) {
        const long row0 = (tile0 + it) * AG_ROWS;
        const bool in = it < n_tiles;
        const int rows = in ? (int)min((long)AG_ROWS, A.N - row0) : 0;
        const __amdgpu_buffer_rsrc_t rbk =
            make_rsrc(A.rows + (size_t)(in ? row0 : 0) * rowb, (uint32_t)rows * rowb);
        const uint32_t at = lo + (uint32_t)ik * (AG_K * 2);
        const bool some = (uint32_t)(ik * (AG_K * 2) + chunk * 16) < rowb && in;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            dma16(j < 4 ? rbk : rqr,
                  (i32x4 *)(ring + slot * AG_SLOT) + (wave + 8 * j) * WAVE,
                  some ? at + (uint32_t)((j & 3) * 64) * rowb : OFF_NONE);
        if (++ik == nst) {
            ik = 0;
            ++it;
        }
    };
    // fragment addresses of k-step 0: tile i of a wave's rows lies 2 KB behind
    // the one before; k-step 1 differs in bit 6
    auto place = [&](int r) {
        const int g = r >> 3, x = turn(r & 7) ^ ((g & 1) << 1);
        return (uint32_t)(g * 1024 + (r & 7) * 128 + ((jg ^ x) * 16));
    };
    const uint32_t pa = place(128 * wr + col), pb = (uint32_t)(AG_SLOT / 2) + place(64 * wq + col);
    f32x4 acc[AG_RT][AG_NG];
    issue(0);
    const int n_stg = n_tiles * nst;
    for (int z = 0, tile = 0, kc = 0; z < n_stg; ++z) {
        __builtin_amdgcn_sched_barrier(0);
        // the stage has landed for every wave, and the other slot is read
        wait_vmcnt<0>();
        stream_barrier();
        issue((z + 1) & 1);
        if (kc == 0) {
            first(tile);
#pragma unroll
            for (int i = 0; i < AG_RT; ++i)
#pragma unroll
                for (int g = 0; g < AG_NG; ++g)
                    acc[i][g] = f32x4{0.f, 0.f, 0.f, 0.f};
        } else if (kc == 1) {
            then(tile);
        }
        __builtin_amdgcn_sched_barrier(0);
        const uint8_t *slot = ring + (z & 1) * AG_SLOT;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint8_t *ra = slot + (pa ^ (64u * s)), *rb = slot + (pb ^ (64u * s));
            i32x4 b[AG_NG];
#pragma unroll
            for (int g = 0; g < AG_NG; ++g)
                b[g] = *(const i32x4 *)(rb + g * 2048);
#pragma unroll
            for (int i = 0; i < AG_RT; ++i) {
                const i32x4 a = *(const i32x4 *)(ra + i * 2048);
#pragma unroll
                for (int g = 0; g < AG_NG; ++g)
                    acc[i][g] = BANK_COLS ? mfma_step<1>(b[g], a, acc[i][g])
                                          : mfma_step<1>(a, b[g], acc[i][g]);
            }
        }
        // the order of a stage: a fragment or two ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, AG_NG + 2, 0);
        static_for<0, 2 * AG_RT>([&](auto I) {
            constexpr int i = decltype(I)::value;
            __builtin_amdgcn_sched_group_barrier(0x008, AG_NG, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, i == AG_RT - 3 ? 1 + AG_NG : 1, 0);
        });
        __builtin_amdgcn_sched_barrier(0);
        if (++kc == nst) {
            kc = 0;
            end(tile, acc);
            ++tile;
        }
    }
    wait_vmcnt<0>();   // (no global-to-LDS load in flight when the workgroup ends)
}

}  // namespace

}  // namespace rb
