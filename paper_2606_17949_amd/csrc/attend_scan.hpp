// The pass over the bank that the attention kernels share (gfx950, wave64).
#pragma once

#include "attend.hpp"
#include "knn_common.hpp"

namespace rb {

namespace {

constexpr int AT_RT = 2;                 // 16-row tiles of a fragment of ds
constexpr int AT_SLAB = 16 * AT_RT;
constexpr float LOG2E = 1.442695040888963407f;

// What 16 bytes of a bank row per lane are (a k-step: 64 bytes of each of 16
// rows), and how many request fragments of 16 bytes per lane meet them.
template <int DT> struct AtElem;
template <> struct AtElem<AT_F32> { static constexpr int KS = 16, SUB = 1, QSZ = 4; };
template <> struct AtElem<AT_BF16> { static constexpr int KS = 32, SUB = 1, QSZ = 2; };
template <> struct AtElem<AT_Q4> { static constexpr int KS = 128, SUB = 4, QSZ = 2; };

inline __host__ __device__ int at_ks(int dtype)
{
    return dtype == AT_F32 ? 16 : dtype == AT_BF16 ? 32 : 128;
}
inline __host__ __device__ uint32_t at_row_bytes(int dtype, int d)
{
    return (uint32_t)(dtype == AT_F32 ? d * 4 : dtype == AT_BF16 ? d * 2 : d / 2);
}
inline __host__ __device__ uint32_t at_query_bytes(int dtype, int d)
{
    return (uint32_t)(dtype == AT_F32 ? d * 4 : d * 2);
}

// 16-row tiles of a slab: 64 requests read each fragment of theirs from LDS for
// 64 rows; with 32, LDS reads alone take as long as the products.
constexpr int at_rt(int dt, int ng) { return dt != AT_F32 && ng == 4 ? 4 : 2; }
// k-steps of bank rows in flight (4-bit rows: 128 elements each; 64 requests over
// 1,000,000 x 768 of them 133 us a call with one, 134 with two and spilled registers)
constexpr int at_ring(int dt, int rt) { return dt == AT_Q4 ? (rt == 4 ? 1 : 3) : rt == 4 ? 2 : 4; }

// Shares of a bank whose waves' parts stay under 1 GB (32-bit offsets).
inline long at_least_shares(long rows, int dtype, int d)
{
    return (rows * at_row_bytes(dtype, d) >> 30) / AT_WAVES + 1;
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Sum over the wave in 64 bits, in the order of wave_reduce.
__device__ __forceinline__ double wave_sum64(double v)
{
    auto plus = [](double x, auto move) {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        return x + __builtin_bit_cast(double, (uint64_t)move((uint32_t)(b >> 32)) << 32 |
                                                  move((uint32_t)b));
    };
    v = plus(v, [](uint32_t w) { return dpp<0xb1>(w); });
    v = plus(v, [](uint32_t w) { return dpp<0x4e>(w); });
    v = plus(v, [](uint32_t w) { return dpp<0x141>(w); });
    v = plus(v, [](uint32_t w) { return dpp<0x140>(w); });
    v = plus(v, [](uint32_t w) { return dpp<0x142, 0xa>(w); });
    v = plus(v, [](uint32_t w) { return dpp<0x143, 0xc>(w); });
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(
        double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63) << 32 |
                    (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63));
}

// The request tile (NG groups of 16 from request q0 on, every k-step) into LDS:
// qs[(k-step * SUB + sub) * NG + group][lane], lane (request lane % 16, K part
// lane / 16). Zero past the batch and past the row.
template <int DT, int NG>
__device__ __forceinline__ void load_requests(const AttendBank &A, int nks, int q0, i32x4 *qs,
                                              int wave, int n_waves, int lane)
{
    using E = AtElem<DT>;
    const uint32_t rowb = at_query_bytes(DT, A.d);
    const int col = lane & 15, jg = lane >> 4;
    // (a resource of this tile alone: a batch may pass 4 GB)
    const int nq = min(A.B - q0, NG * 16);
    const __amdgpu_buffer_rsrc_t rq =
        make_rsrc(A.queries + (size_t)q0 * rowb, (uint32_t)nq * rowb);
    for (int f = wave; f < nks * E::SUB * NG; f += n_waves) {
        const int ks = f / (E::SUB * NG), rest = f - ks * E::SUB * NG;
        const int sub = rest / NG, q = (rest - sub * NG) * 16 + col;
        // the lane's first element: bank elements of the same lane and place
        const int el = ks * E::KS + jg * (E::KS / 4) + sub * 8;
        dma16(rq, qs + f * WAVE,
              q < nq && el < A.d ? (uint32_t)q * rowb + (uint32_t)el * E::QSZ : OFF_NONE);
    }
}

// A lane's 32 elements of 4 bits (codes of 0, 0.5, 1, 1.5, 2, 3, 4, 6, bit 3
// the sign) times their scale, as four bf16 fragments: exact, every product is
// a bf16 value.
__device__ __forceinline__ i32x4 widen4(uint32_t codes, float scale)
{
    i32x4 r;
    r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return r;
}

// One wave's pass over slabs [s0, s1) (of 16 * RT rows) of the bank against the
// request tile in LDS. Bank rows come from HBM straight into MFMA operand
// registers, R k-steps (a block) ahead across slab ends, and no wave waits for
// another once the request tile, sent for before the call, has landed; ready()
// is called then, in every wave. side(slab) sends for what end(slab, acc) reads
// beside the products.
// A slab's first block stands apart from the others: there the compiler knows
// that side's loads came after the block's own, so that waiting for the block
// does not wait for them. (In one loop over all blocks every slab emptied the
// ring: one request over 14,919 x 384 fp32 took 13.5 us for 9.6, over 100,000 x
// 768 in 4 bits 23.2 for 14.7.)
// BANK_COLS false: acc[r][g][e] is <q, x> of row 16*r + 4*(lane/16) + e and
// request 16*g + lane%16; true: of row 16*r + lane%16 and request
// 16*g + 4*(lane/16) + e.
template <int DT, int NG, int RT, int R, bool BANK_COLS, typename Ready, typename Side,
          typename End>
__device__ __forceinline__ void scan_slabs(const AttendBank &A, int nks, const i32x4 *qs, long s0,
                                           long s1, int lane, Ready &&ready, Side &&side,
                                           End &&end)
{
    using E = AtElem<DT>;
    constexpr int MDT = DT == AT_F32 ? 0 : 1;
    constexpr int SLAB = 16 * RT;
    const int col = lane & 15, jg = lane >> 4;
    const uint32_t rowb = at_row_bytes(DT, A.d);
    const int n_slabs = (int)(s1 - s0);
    if (n_slabs <= 0) {   // (every wave meets at the barrier)
        wait_vmcnt<0>();
        stream_barrier();
        ready();
        return;
    }
    const long row0 = s0 * SLAB;
    const int nrows = (int)min((long)n_slabs * SLAB, A.N - row0);
    const __amdgpu_buffer_rsrc_t rbk =
        make_rsrc(A.rows + (size_t)row0 * rowb, (uint32_t)nrows * rowb);
    const int nsc = A.d / 32;   // scales of a row
    const __amdgpu_buffer_rsrc_t rsc =
        DT == AT_Q4 ? make_rsrc(A.scales + (size_t)row0 * nsc, (uint32_t)nrows * nsc) : rbk;
    const int n_blk = (nks + R - 1) / R;
    i32x4 ring[R][RT];
    uint8_t rsca[DT == AT_Q4 ? R : 1][RT];
    // k-step u of block (slab ls, block lb) into ring[u]; k-steps past the row
    // load zeros, as do rows past the share
    int ls = 0, lb = 0;
    auto issue = [&](auto U) {
        constexpr int u = decltype(U)::value;
        const int ks = lb * R + u;
        const bool none = ks * E::KS + jg * (E::KS / 4) >= A.d;
        const uint32_t at = (uint32_t)(ls * SLAB + col);
        const uint32_t vo = at * rowb + (uint32_t)(ks * KSTEP_BYTES + jg * 16);
        const uint32_t so = at * nsc + (uint32_t)(ks * 4 + jg);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            ring[u][r] = buffer_load16(rbk, none ? OFF_NONE : vo + (uint32_t)r * 16 * rowb);
            if constexpr (DT == AT_Q4)
                rsca[u][r] = __builtin_amdgcn_raw_buffer_load_b8(
                    rsc, (int)(none ? OFF_NONE : so + (uint32_t)(r * 16 * nsc)), 0, 0);
        }
    };
    auto advance = [&] {
        if (++lb == n_blk) {
            lb = 0;
            ++ls;
        }
    };
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, R>([&](auto U) { issue(U); });
    advance();
    // the request tile has landed once at most the loads after it are
    // outstanding, and after the barrier in every wave
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<R * RT * (DT == AT_Q4 ? 2 : 1)>();
    stream_barrier();
    __builtin_amdgcn_sched_barrier(0);
    ready();

    // A block's products are summed by themselves: a score is then a sum of few
    // partial sums, and off by what those few additions round away. (One chain of
    // 256 products of four fp32 elements: 12 requests over 1,473 x 1,024 at beta 21
    // had gradients off by 2e-5 in their weights, now 3e-6. Tiles of 64 requests over
    // bf16 or 4-bit rows have no registers for it: one chain over the row.)
    constexpr bool PARTS = RT == 2;
    f32x4 acc[RT][NG], sum[PARTS ? RT : 1][PARTS ? NG : 1];
    auto clear = [&](auto &x) {
#pragma unroll
        for (auto &row : x)
#pragma unroll
            for (auto &v : row)
                v = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    // the products of block b, and the loads of the block after it
    auto block = [&](int b) {
        if constexpr (PARTS)
            clear(acc);
        static_for<0, R>([&](auto U) {
            constexpr int u = decltype(U)::value;
            __builtin_amdgcn_sched_barrier(0);
            const int ks = b * R + u;
            // (a k-step past the row: its bank elements are zeros)
            const i32x4 *fk = qs + (ks < nks ? ks : 0) * E::SUB * NG * WAVE + lane;
            static_for<0, E::SUB>([&](auto T) {
                constexpr int t = decltype(T)::value;
                i32x4 a[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if constexpr (DT == AT_Q4)
                        a[r] = widen4((uint32_t)ring[u][r][t],
                                      __uint_as_float((uint32_t)rsca[u][r] << 23));
                    else
                        a[r] = ring[u][r];
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const i32x4 q = fk[(t * NG + g) * WAVE];
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        acc[r][g] = BANK_COLS ? mfma_step<MDT>(q, a[r], acc[r][g])
                                              : mfma_step<MDT>(a[r], q, acc[r][g]);
                }
            });
            issue(U);
        });
        if constexpr (PARTS)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    sum[r][g] = b == 0 ? acc[r][g] : sum[r][g] + acc[r][g];
        advance();
    };
    for (int slab = 0; slab < n_slabs; ++slab) {
        side(slab);
        if constexpr (!PARTS)
            clear(acc);
        block(0);
        __builtin_amdgcn_sched_barrier(0);
        for (int b = 1; b < n_blk; ++b)
            block(b);
        if constexpr (PARTS)
            end(slab, sum);
        else
            end(slab, acc);
    }
}

}  // namespace

}  // namespace rb
