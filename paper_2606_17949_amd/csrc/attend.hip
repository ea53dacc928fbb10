// Attention of requests over the labelled bank: the forward pass.
#include "attend_gemm.hpp"

#include <math.h>

namespace rb {

namespace {

// A running maximum is raised when a score passes it by this many powers of
// two: weights stay below 2^16 and few slabs rescale what went before.
// The maximum is kept in units of the scores and subtracted before c multiplies: the
// largest weight is then 1 (2^AT_SLACK at most) for any c. (Subtracted from rounded
// products c*u, it left up to half a step of them in the exponent: from c*u = 2^31 on
// weights of 0 or infinity.)
constexpr float AT_SLACK = 16.f;

// The maximum of no scores: below any, and a number, so that differences are none
// that is not. What has only masked rows keeps it, with sums of 0, and so does what
// has only rows whose scores are no numbers, with sums that are none and show
// whatever weight they are joined with.
constexpr float AT_NO_MAX = -3.402823466e38f;

// What the sums of a part of the rows, relative to its maximum, count for beside
// the whole's maximum m.
__device__ __forceinline__ float part_weight(float c, float part, float m)
{
    return __builtin_amdgcn_exp2f(c * (part - m));
}

struct AttendArgs {
    AttendBank b;
    const float *qual, *len;
    int M, nks, n_chunks, n_qt;
    long slabs;
    float *ml;   // [n_chunks][B][2] maximum (of u) and sum of the weights
    float *o;    // [n_chunks][n_lt][B][ct * 16] sums of weighted labels
};

// One workgroup per (share of the bank, tile of NG * 16 requests, tile of CT *
// 16 label columns); each wave has its own part of the share, its own running
// maximum and sums, and the waves' are joined in LDS at the end.
//   scores   u = <q, x> - |x|^2/2 (MFMA; |q|^2 changes no weight; the join adds it
//            to lse)
//   maximum  of u, raised now and then, the sums rescaled when it is
//   weights  p = 2^(c * (u - maximum)), their sum, and sum of p * label as a second
//            MFMA (fp32, 16 label columns x 16 requests, 4 rows): its operand
//            p[row 4*(lane/16) + e][request lane%16] is register e of the
//            scores as it stands.
// Bound by the bank's way to the compute units (64 requests over 100,000 x 768 bf16
// 35 us, 4.4 TB/s, called again and again, so that the last-level cache serves part of
// it; over 1,000,000 x 768 in 4 bits 133 us a call, 3.3 TB/s, where the products and the
// widening of the codes take as long), small banks by latency (one request over
// 14,919 x 384 fp32 9.4 us, and 4.2 the join). A second product of fp32 keeps the
// weights' 24 bits.
template <int DT, int NG, int RT, int CT>
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void attend_kernel(const AttendArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    i32x4 *qs = (i32x4 *)smem;
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int n_waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int q0 = t * NG * 16, lt = blockIdx.y;
    const long gw = (long)ch * n_waves + wave, n_gw = (long)A.n_chunks * n_waves;
    const long s0 = gw * A.slabs / n_gw, s1 = (gw + 1) * A.slabs / n_gw;
    const int N = A.b.N;
    const float c = A.b.c;

    load_requests<DT, NG>(A.b, A.nks, q0, qs, wave, n_waves, lane);
    // this lane's label columns
    const float *lab[CT];
    bool lab_ok[CT];
#pragma unroll
    for (int k = 0; k < CT; ++k) {
        const int cc = (lt * CT + k) * 16 + col;
        lab_ok[k] = cc < 2 * A.M;
        lab[k] = cc < A.M ? A.qual + cc : lab_ok[k] ? A.len + (cc - A.M) : A.qual;
    }
    float ref[NG], l[NG];
    f32x4 o[NG][CT];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        ref[g] = AT_NO_MAX;   // the maximum that the sums are relative to
        l[g] = 0.f;
#pragma unroll
        for (int k = 0; k < CT; ++k)
            o[g][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // norms, mask and labels of a slab: this lane's rows 16*r + 4*jg + e (the
    // last row again for those past the bank)
    float nrm[RT][4], v[RT][4][CT];
    // four rows' mask bytes lie in one or two aligned words
    uint32_t mk[RT][2];
    const bool masked = A.b.mask != nullptr;
    const uint32_t *const mask4 = (const uint32_t *)((uintptr_t)A.b.mask & ~(uintptr_t)3);
    const uint32_t mask_sh = (uint32_t)((uintptr_t)A.b.mask & 3);
    const size_t mask_last = ((size_t)N - 1 + mask_sh) / 4;
    auto side = [&](int slab) {
        const long r0 = (s0 + slab) * (16 * RT) + jg * 4;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const size_t at = (size_t)min(r0 + r * 16 + e, (long)N - 1);
                nrm[r][e] = A.b.norms[at];
#pragma unroll
                for (int k = 0; k < CT; ++k)
                    v[r][e][k] = lab[k][at * A.M];
            }
        if (masked)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const size_t w = (size_t)(r0 + r * 16) / 4;
                mk[r][0] = mask4[min(w, mask_last)];
                mk[r][1] = mask4[min(w + 1, mask_last)];
            }
    };
    auto end = [&](int slab, f32x4(&acc)[RT][NG]) {
        const long r0 = (s0 + slab) * (16 * RT) + jg * 4;
        __builtin_amdgcn_sched_barrier(0);
        // scores: -inf for rows masked or past the bank, whatever they hold
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const uint32_t four =
                masked ? __builtin_amdgcn_alignbyte(mk[r][1], mk[r][0], mask_sh) : ~0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool ok = r0 + r * 16 + e < N && (four >> (8 * e) & 0xffu) != 0;
                const float nh = -0.5f * nrm[r][e];
#pragma unroll
                for (int k = 0; k < CT; ++k)
                    v[r][e][k] = ok && lab_ok[k] ? v[r][e][k] : 0.f;
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    acc[r][g][e] = ok ? acc[r][g][e] + nh : -INFINITY;
            }
        }
        bool raise = false;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float m = -INFINITY;
#pragma unroll
            for (int r = 0; r < RT; ++r)
                m = fmaxf(m, max4(acc[r][g]));
            raise |= c * (m - ref[g]) > AT_SLACK;
        }
        if (ballot(raise)) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float m = -INFINITY;
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    m = fmaxf(m, max4(acc[r][g]));
                m = rows_reduce(m, [](float x, float y) { return fmaxf(x, y); });
                const float up = fmaxf(ref[g], m);
                const float f = part_weight(c, ref[g], up);
                ref[g] = up;
                l[g] *= f;
#pragma unroll
                for (int k = 0; k < CT; ++k)
                    o[g][k] *= f;
            }
        }
        // (no instruction moves across a row's bounds, which keeps few weights live)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float p = __builtin_amdgcn_exp2f(c * (acc[r][g][e] - ref[g]));
                    l[g] += p;
#pragma unroll
                    for (int k = 0; k < CT; ++k)
                        o[g][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][e][k], p, o[g][k], 0,
                                                                      0, 0);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    scan_slabs<DT, NG, RT, at_ring(DT, RT), false>(A.b, A.nks, qs, s0, s1, lane, [] {}, side, end);

    // ---- the waves' sums, joined (the request tile's LDS is free now)
    constexpr int W = 2 + 16 * CT;
    float *jn = (float *)smem;   // [n_waves][NG * 16][W]
    stream_barrier();
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        const float ls = rows_reduce(l[g], [](float x, float y) { return x + y; });
        float *at = jn + (wave * NG * 16 + g * 16 + col) * W;
        if (jg == 0) {
            at[0] = ref[g];
            at[1] = ls;
        }
#pragma unroll
        for (int k = 0; k < CT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                at[2 + k * 16 + jg * 4 + e] = o[g][k][e];
    }
    stream_barrier();
    for (int i = tid; i < NG * 16 * (W - 1); i += blockDim.x) {
        const int q = i / (W - 1), x = i - q * (W - 1);   // x 0: the sum, else a column
        if (q0 + q >= A.b.B)
            continue;
        float m = AT_NO_MAX, sum = 0.f;
        for (int w = 0; w < n_waves; ++w)
            m = fmaxf(m, jn[(w * NG * 16 + q) * W]);
        for (int w = 0; w < n_waves; ++w) {
            const float *at = jn + (w * NG * 16 + q) * W;
            sum = fmaf(part_weight(c, at[0], m), at[1 + x], sum);
        }
        if (x > 0) {
            A.o[(((size_t)ch * gridDim.y + lt) * A.b.B + q0 + q) * (16 * CT) + x - 1] = sum;
        } else if (lt == 0) {
            float *ml = A.ml + ((size_t)ch * A.b.B + q0 + q) * 2;
            ml[0] = m;
            ml[1] = sum;
        }
    }
}

// The same as a matrix product of tiles (attend_gemm.hpp), for large bf16
// batches and 16 label columns. The weighted labels are products of bf16
// MFMA too: p as two bf16 values (hi + lo = p to 2^-17), a label as three
// (exact), five products of 16 columns x 16 requests x 32 rows in place of
// eight fp32 ones that take twice as long each. The sum of the weights is that
// of hi + lo, a column of ones: it stands behind the labels (ONES false: at
// column 2 M), or, where they fill all 16 columns, is two products more.
// 256 requests over 1,000,000 x 768: 495 us, 795 TFLOP/s (the product alone 400, the
// rest powers of two and splits that its waves do all at one time).
constexpr int ONE2 = 0x3f803f80;   // two bf16 ones

template <bool ONES>
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void attend_gemm_kernel(const AttendArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    uint8_t *ring = smem;
    float *labels = (float *)(smem + 2 * AG_SLOT);   // [64][64]
    TileSide *side = (TileSide *)(labels + 64 * WAVE);
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    __builtin_assume(tid < AT_WAVES * WAVE);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int wr = wave >> 2, wq = wave & 3;
    const int q0 = t * AG_REQS, lt = blockIdx.y;
    const long t0 = (long)ch * A.slabs / A.n_chunks, t1 = (long)(ch + 1) * A.slabs / A.n_chunks;
    const int N = A.b.N, M = A.M;
    const float c = A.b.c;
    // the lane's label column (16 to a tile; behind the last, the first again)
    const int cc = lt * 16 + col;
    const float *lab = cc < M ? A.qual + cc : cc < 2 * M ? A.len + (cc - M) : A.qual;
    const bool one = !ONES && lt == 0 && cc == 2 * M;
    // piece 8*b + 4*h + e: rows 32*b + 16*h + 4*(lane/16) + e
    auto label = [&](long row0, int f, int l) {
        const long row = row0 + (f >> 3) * 32 + ((f >> 2) & 1) * 16 + 4 * (l >> 4) + (f & 3);
        return lab + (size_t)min(row, (long)N - 1) * M;
    };

    float ref[AG_NG];
    // of the lane's label column, the sum of the labels that are no numbers: every
    // weight is above 0, so a request's average is that sum whatever its weights
    float beyond = 0.f;
    f32x4 o[AG_NG], ol[ONES ? AG_NG : 1];
#pragma unroll
    for (int g = 0; g < AG_NG; ++g) {
        ref[g] = AT_NO_MAX;
        o[g] = f32x4{0.f, 0.f, 0.f, 0.f};
        ol[ONES ? g : 0] = o[g];
    }
    const bool masked = A.b.mask != nullptr;
    auto end = [&](int tile, f32x4(&acc)[AG_RT][AG_NG]) {
        const int left = (int)min((long)AG_ROWS, N - (t0 + tile) * AG_ROWS);
        bool raise = false;
        float top[AG_NG];
#pragma unroll
        for (int g = 0; g < AG_NG; ++g)
            top[g] = -INFINITY;
#pragma unroll
        for (int r = 0; r < AG_RT; ++r) {
            __builtin_amdgcn_sched_barrier(0);
            const f32x4 n4 = tile_norms(A.b, side, left, 128 * wr + 16 * r + 4 * jg);
#pragma unroll
            for (int g = 0; g < AG_NG; ++g) {
                f32x4 u = acc[r][g] + n4;
                if (masked)   // (a masked row may hold anything)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        u[e] = n4[e] == -INFINITY ? -INFINITY : u[e];
                acc[r][g] = u;
                top[g] = fmaxf(top[g], max4(u));
            }
        }
#pragma unroll
        for (int g = 0; g < AG_NG; ++g)
            raise |= c * (top[g] - ref[g]) > AT_SLACK;
        if (ballot(raise)) {
#pragma unroll
            for (int g = 0; g < AG_NG; ++g) {
                const float m =
                    rows_reduce(top[g], [](float x, float y) { return fmaxf(x, y); });
                const float up = fmaxf(ref[g], m);
                const float f = part_weight(c, ref[g], up);
                ref[g] = up;
                o[g] *= f;
                if constexpr (ONES)
                    ol[g] *= f;
            }
        }
        uint32_t odd = 0;   // the largest of the labels' magnitudes, doubled
        const i32x4 ones = i32x4{ONE2, ONE2, ONE2, ONE2};
#pragma unroll
        for (int r = 0; r < AG_RT; r += 2) {
            __builtin_amdgcn_sched_barrier(0);
            // the labels of these 32 rows as three bf16 values each, made finite (those
            // of rows without weight may hold anything)
            i32x4 vh, vm, vl;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float y = labels[(8 * (4 * wr + r / 2) + 2 * j + i) * WAVE + lane];
                    x[i] = one ? 1.f : __builtin_amdgcn_fmed3f(y, -3e38f, 3e38f);
                    odd = max(odd, __float_as_uint(y) << 1);
                }
                vh[j] = split_bf16(x[0], x[1]);
                vm[j] = split_bf16(x[0], x[1]);
                vl[j] = split_bf16(x[0], x[1]);
            }
            i32x4 ph[AG_NG], pl[AG_NG];
#pragma unroll
            for (int g = 0; g < AG_NG; ++g) {
                if (g == 2)
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4 &u = acc[r + (j >> 1)][g];
                    float x = __builtin_amdgcn_exp2f(c * (u[2 * (j & 1)] - ref[g]));
                    float y = __builtin_amdgcn_exp2f(c * (u[2 * (j & 1) + 1] - ref[g]));
                    ph[g][j] = split_bf16(x, y);
                    pl[g][j] = split_bf16(x, y);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            // (product by product over the groups: no product waits for the one before)
            auto weigh = [&](const i32x4 &v, const i32x4(&p)[AG_NG], f32x4(&to)[AG_NG]) {
#pragma unroll
                for (int g = 0; g < AG_NG; ++g)
                    to[g] = mfma_step<1>(v, p[g], to[g]);
            };
            weigh(vh, ph, o);
            weigh(vm, ph, o);
            weigh(vl, ph, o);
            weigh(vh, pl, o);
            weigh(vm, pl, o);
            if constexpr (ONES) {
#pragma unroll
                for (int g = 0; g < AG_NG; ++g) {
                    ol[g] = mfma_step<1>(ones, ph[g], ol[g]);
                    ol[g] = mfma_step<1>(ones, pl[g], ol[g]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // labels that are no numbers, in rows that are not masked
        if (ballot(odd >= 0xff000000u))
#pragma unroll 1
            for (int k = 0; k < 32; ++k) {
                const float y = labels[(32 * wr + k) * WAVE + lane];
                const int at = 128 * wr + 32 * (k >> 3) + 16 * (k >> 2 & 1) + 4 * jg + (k & 3);
                if (!__builtin_isfinite(y) && tile_norm(A.b, side, left, at) != -INFINITY)
                    beyond += y;
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    gemm_tiles<false, 8>(A.b, A.nks, ring, side, labels, q0, t0, (int)(t1 - t0), wave, lane,
                             label, end);

    // ---- the two halves of the rows joined: maximum, then 16 columns (and the
    // sum of the weights, where it is none of them)
    constexpr int W = 18;
    float *jn = (float *)smem;            // [2][256][W]
    float *far = jn + 2 * AG_REQS * W;    // [2][16]
    stream_barrier();
    beyond = rows_reduce(cc < 2 * M ? beyond : 0.f, [](float x, float y) { return x + y; });
    if (wq == 0 && jg == 0)
        far[16 * wr + col] = beyond;
#pragma unroll
    for (int g = 0; g < AG_NG; ++g) {
        float *at = jn + (wr * AG_REQS + 64 * wq + 16 * g + col) * W;
        if (jg == 0) {
            at[0] = ref[g];
            if constexpr (ONES)
                at[1] = ol[g][0];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            at[2 + 4 * jg + e] = o[g][e];
            if (!ONES && 4 * jg + e == 2 * M)
                at[1] = o[g][e];
        }
    }
    stream_barrier();
    for (int i = tid; i < AG_REQS * (W - 1); i += AT_WAVES * WAVE) {
        const int q = i / (W - 1), x = i - q * (W - 1);
        if (q0 + q >= A.b.B)
            continue;
        const float *a = jn + q * W, *b = a + AG_REQS * W;
        const float m = fmaxf(a[0], b[0]);
        const float sum =
            fmaf(part_weight(c, b[0], m), b[1 + x], part_weight(c, a[0], m) * a[1 + x]);
        if (x > 0) {
            A.o[(((size_t)ch * gridDim.y + lt) * A.b.B + q0 + q) * 16 + x - 1] =
                sum + (far[x - 1] + far[15 + x]);
        } else if (lt == 0) {
            float *ml = A.ml + ((size_t)ch * A.b.B + q0 + q) * 2;
            ml[0] = m;
            ml[1] = sum;
        }
    }
}

// The shares' sums joined: one workgroup of 256 threads per request, 256 shares
// at a time. What bounds it is latency: a share's maximum and sum, and the
// columns (16 at a time, 16 shares side by side), are all sent for before the
// first is used.
__global__ __launch_bounds__(256) void attend_join_kernel(const float *ml, const float *o,
                                                          int n_chunks, int n_lt, int width, int B,
                                                          int M, const uint8_t *queries, int qbytes,
                                                          bool bf16, float c, double c_exact,
                                                          float *q_hat, float *l_hat, float *lse)
{
    __shared__ float red[256], wts[256], part[2][4];
    const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
    __shared__ double squares[4];
    const int col = tid & 15, row = tid >> 4;
    // the block's maximum or sum of one value a thread
    auto over = [&](int which, float v, auto op, float none) {
        v = wave_reduce(v, op);
        if ((tid & 63) == 0)
            part[which][wave] = v;
        __syncthreads();
        v = none;
        for (int w = 0; w < 4; ++w)
            v = op(v, part[which][w]);
        return v;
    };
    auto pair = [&](int ch) {
        return ch < n_chunks ? *(const f32x2 *)(ml + ((size_t)ch * B + b) * 2)
                             : f32x2{AT_NO_MAX, 0.f};
    };
    // column cc of 16 of the 256 shares from k0 on
    auto columns = [&](int c0, int k0, float(&x)[16]) {
        const int cc = c0 + col, tile = cc / width;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int ch = k0 + k * 16 + row;
            x[k] = cc < 2 * M && ch < n_chunks
                       ? o[(((size_t)ch * n_lt + tile) * B + b) * width + cc - tile * width]
                       : 0.f;
        }
    };
    float x[16];
    float q2 = 0.f;
    if (lse)
        for (int at = tid * 16; at < qbytes; at += 256 * 16) {
            const i32x4 q = load16(queries + (size_t)b * qbytes + at);
            q2 = bf16 ? sumsq16<1>(q, q2) : sumsq16<0>(q, q2);
        }
    f32x2 mine = pair(tid);
    columns(0, 0, x);
    float m = mine[0];
    for (int ch = tid + 256; ch < n_chunks; ch += 256)
        m = fmaxf(m, pair(ch)[0]);
    m = over(0, m, [](float u, float v) { return fmaxf(u, v); }, AT_NO_MAX);
    auto weight = [&](float v) { return part_weight(c, v, m); };
    float sum = weight(mine[0]) * mine[1];
    wts[tid] = weight(mine[0]);
    for (int ch = tid + 256; ch < n_chunks; ch += 256) {
        const f32x2 p = pair(ch);
        sum = fmaf(weight(p[0]), p[1], sum);
    }
    const float total = over(1, sum, [](float u, float v) { return u + v; }, 0.f);
    if (lse) {
        // the maximum and |q|^2/2 nearly cancel: in 64 bits, with c unrounded
        const double w2 = wave_sum64(q2);
        if ((tid & 63) == 0)
            squares[wave] = w2;
        __syncthreads();
        if (tid == 0) {
            const double s2 = (squares[0] + squares[1]) + (squares[2] + squares[3]);
            lse[b] = (float)(((m - 0.5 * s2) * c_exact + __builtin_amdgcn_logf(total)) *
                             0.6931471805599453);
        }
    }
    for (int c0 = 0; c0 < 2 * M; c0 += 16) {
        float s = 0.f;
        for (int k0 = 0; k0 < n_chunks; k0 += 256) {
            if (n_chunks > 256) {
                __syncthreads();
                wts[tid] = weight(pair(k0 + tid)[0]);
                __syncthreads();
            }
            if (c0 > 0 || k0 > 0)
                columns(c0, k0, x);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const float w = wts[k * 16 + row];
                s = w != 0.f ? fmaf(w, x[k], s) : s;
            }
        }
        __syncthreads();
        red[tid] = s;
        __syncthreads();
        const int cc = c0 + col;
        if (tid < 16 && cc < 2 * M) {
            s = 0.f;
            for (int k = 0; k < 16; ++k)
                s += red[k * 16 + col];
            s /= total;
            if (cc < M)
                q_hat[(size_t)b * M + cc] = s;
            else
                l_hat[(size_t)b * M + cc - M] = s;
        }
    }
}

template <int DT, int NG, int RT, int CT>
hipError_t launch_one(const AttendPlan &p, const AttendArgs &a, hipStream_t s)
{
    auto kern = attend_kernel<DT, NG, RT, CT>;
    const hipError_t e = hipFuncSetAttribute(
        (const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds_bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(p.n_chunks * p.n_qt, p.n_lt), dim3(p.waves * WAVE), p.lds_bytes,
                       s, a);
    return hipGetLastError();
}

template <int DT, int CT>
hipError_t launch_ng(const AttendPlan &p, const AttendArgs &a, hipStream_t s)
{
    switch (p.ng) {
    case 1: return launch_one<DT, 1, 2, CT>(p, a, s);
    case 2: return launch_one<DT, 2, 2, CT>(p, a, s);
    case 4: return launch_one<DT, 4, at_rt(DT, 4), CT>(p, a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_gemm(const AttendPlan &p, const AttendArgs &a, hipStream_t s)
{
    auto kern = 2 * a.M < 16 ? attend_gemm_kernel<false> : attend_gemm_kernel<true>;
    const hipError_t e = hipFuncSetAttribute(
        (const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds_bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(p.n_chunks * p.n_qt, p.n_lt), dim3(AT_WAVES * WAVE), p.lds_bytes,
                       s, a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_dt(const AttendPlan &p, const AttendArgs &a, hipStream_t s)
{
    return p.ct == 1 ? launch_ng<DT, 1>(p, a, s) : launch_ng<DT, 2>(p, a, s);
}

}  // namespace

bool plan_attend(int B, int N, int d, int dtype, int M, int n_cu, AttendPlan *p)
{
    const int ks = at_ks(dtype);
    p->dtype = dtype;
    p->nks = (d + ks - 1) / ks;
    p->gemm = at_gemm(dtype, B, N, d, M, n_cu);
    if (p->gemm) {
        p->nks = (d + AG_K - 1) / AG_K;
        p->ct = 1;
        p->n_lt = (2 * M + 15) / 16;
        p->n_qt = (B + AG_REQS - 1) / AG_REQS;
        p->slabs = (int)(((long)N + AG_ROWS - 1) / AG_ROWS);
        const int most = n_cu / (p->n_qt * p->n_lt);
        p->n_chunks = most < 1 ? 1 : most < p->slabs ? most : p->slabs;
        p->waves = AT_WAVES;
        p->lds_bytes = 2 * AG_SLOT + 64 * WAVE * 4 + sizeof(TileSide);
        p->off_ml = 0;
        p->off_o = up256((size_t)p->n_chunks * B * 2 * 4);
        p->bytes = p->off_o + up256((size_t)p->n_chunks * p->n_lt * B * 16 * 4);
        return true;
    }
    p->ct = 2 * M <= 16 ? 1 : 2;
    p->n_lt = (2 * M + 16 * p->ct - 1) / (16 * p->ct);
    const size_t group = (size_t)p->nks * ks * (dtype == AT_F32 ? 4 : 2) * 16;
    const int ng = at_groups(B, N, group, n_cu, 1, [&](int g) { return 16 * at_rt(dtype, g); });
    if (ng == 0)
        return false;
    p->ng = ng;
    const int slab = 16 * at_rt(dtype, ng);
    p->slabs = (int)(((long)N + slab - 1) / slab);
    p->n_qt = (B + ng * 16 - 1) / (ng * 16);
    // one workgroup per compute unit, as far as there are slabs for its waves;
    // a wave's part of the bank stays under 1 GB (32-bit offsets)
    const long tiles = (long)p->n_qt * p->n_lt;
    long chunks = n_cu / tiles;
    const long by_size = at_least_shares((long)p->slabs * slab, dtype, d);
    if (chunks < by_size)
        chunks = by_size;
    if (chunks > p->slabs)
        chunks = p->slabs;
    if (chunks < 1)
        chunks = 1;
    p->n_chunks = (int)chunks;
    const long per = (p->slabs + chunks - 1) / chunks;
    p->waves = per < AT_WAVES ? (int)per : AT_WAVES;
    const size_t join = (size_t)p->waves * ng * 16 * (2 + 16 * p->ct) * 4;
    p->lds_bytes = group * ng > join ? group * ng : join;
    p->off_ml = 0;
    p->off_o = up256((size_t)chunks * B * 2 * 4);
    p->bytes = p->off_o + up256((size_t)chunks * p->n_lt * B * 16 * p->ct * 4);
    return true;
}

hipError_t launch_attend(const AttendPlan &p, const AttendBank &b, const float *qual,
                         const float *len, int M, float *q_hat, float *l_hat, float *lse, void *ws,
                         hipStream_t s)
{
    AttendArgs a;
    a.b = b;
    a.qual = qual;
    a.len = len;
    a.M = M;
    a.nks = p.nks;
    a.n_chunks = p.n_chunks;
    a.n_qt = p.n_qt;
    a.slabs = p.slabs;
    a.ml = (float *)((uint8_t *)ws + p.off_ml);
    a.o = (float *)((uint8_t *)ws + p.off_o);
    const hipError_t e = p.gemm               ? launch_gemm(p, a, s)
                         : p.dtype == AT_F32  ? launch_dt<AT_F32>(p, a, s)
                         : p.dtype == AT_BF16 ? launch_dt<AT_BF16>(p, a, s)
                                              : launch_dt<AT_Q4>(p, a, s);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(attend_join_kernel, dim3(b.B), dim3(256), 0, s, a.ml, a.o, p.n_chunks,
                       p.n_lt, 16 * p.ct, b.B, M, b.queries, (int)at_query_bytes(p.dtype, b.d),
                       p.dtype != AT_F32, b.c, b.c_exact(), q_hat, l_hat, lse);
    return hipGetLastError();
}

}  // namespace rb
