// Attention of requests over the labelled bank: the passes that recompute its
// probabilities, the rows' accumulated weight and the gradients.
#include "attend_scan.hpp"

#include <math.h>

namespace rb {

namespace {

// k-steps of bank rows in flight (4-bit rows: 128 elements each)
constexpr int at_ring(int dt, int rt) { return dt == AT_Q4 || rt == 4 ? 2 : 4; }
// 16-row tiles of a slab: 64 requests read each fragment of theirs from LDS for
// 64 rows; with 32, LDS reads alone take as long as the products.
constexpr int at_rt(int dt, int ng) { return dt != AT_F32 && ng == 4 ? 4 : 2; }
constexpr size_t PART_BYTES = 128u << 20;   // ds of a part of the bank

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Per request: -|q|^2/2, lse in powers of two, and what is subtracted from the
// weights' gradient, sum of the outputs' gradients times the outputs less the
// gradient of lse. A request without a row (lse = -inf) gets lse2 = inf, so
// that its weights are 2^(-inf) = 0, as do the places past the batch.
struct Side {
    float hq, lse2, shift, none;
};

template <int QDT>
__global__ __launch_bounds__(256) void side_kernel(const uint8_t *queries, int B, int d, int M,
                                                   const float *lse, const float *q_hat,
                                                   const float *l_hat, const float *dq,
                                                   const float *dl, const float *dlse,
                                                   float *dout, int pitch, Side *side)
{
    const int lane = threadIdx.x & 63;
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= B)
        return;
    const int n16 = d * Elem<QDT>::ESZ / 16;
    const uint8_t *q = queries + (size_t)b * d * Elem<QDT>::ESZ;
    float s = 0.f;
    for (int i = lane; i < n16; i += WAVE)
        s = sumsq16<QDT>(load16(q + (size_t)i * 16), s);
    s = wave_sum(s);
    const bool alive = lse[b] != -INFINITY;
    float dot = 0.f;
    if (dout) {
        // (a dead request's outputs are no numbers, and its gradients may be none)
        for (int c = lane; c < pitch; c += WAVE) {
            float g = 0.f, o = 0.f;
            if (alive && c < 2 * M) {
                const size_t at = (size_t)b * M + (c < M ? c : c - M);
                g = c < M ? dq[at] : dl[at];
                o = c < M ? q_hat[at] : l_hat[at];
            }
            dot = fmaf(g, o, dot);
            dout[(size_t)b * pitch + c] = g;
        }
        dot = wave_sum(dot);
        if (alive && dlse)
            dot -= dlse[b];
    }
    if (lane == 0)
        side[b] = Side{-0.5f * s, alive ? lse[b] * LOG2E : INFINITY, dot, 0.f};
}

struct UsageArgs {
    AttendBank b;
    const Side *side;
    int nks, n_chunks, n_qt;
    long slabs;
    float decay;
    float *usage, *part;   // part [n_qt][N], null where one tile holds the batch
};

// Weights of the bank's rows: as the forward pass, with the bank's rows over
// the lanes, so that a row's sum over the requests is a sum over registers and
// four lanes. There is no running maximum: lse is known.
template <int DT, int NG, int RT>
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void usage_kernel(const UsageArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    i32x4 *qs = (i32x4 *)smem;
    Side *sd = (Side *)(qs + (size_t)A.nks * AtElem<DT>::SUB * NG * WAVE);   // [NG * 16]
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int n_waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int q0 = t * NG * 16;
    const long gw = (long)ch * n_waves + wave, n_gw = (long)A.n_chunks * n_waves;
    const long s0 = gw * A.slabs / n_gw, s1 = (gw + 1) * A.slabs / n_gw;
    const int N = A.b.N;
    const float c = A.b.c;
    load_requests<DT, NG>(A.b, A.nks, q0, qs, wave, n_waves, lane);
    for (int i = tid; i < NG * 16; i += blockDim.x)
        sd[i] = q0 + i < A.b.B ? A.side[q0 + i] : Side{0.f, INFINITY, 0.f, 0.f};
    wait_vmcnt<0>();
    stream_barrier();

    float hq[NG][4], lse2[NG][4];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Side &x = sd[g * 16 + 4 * jg + e];
            hq[g][e] = x.hq;
            lse2[g][e] = x.lse2;
        }
    float nrm[RT];
    uint8_t mk[RT];
    const bool masked = A.b.mask != nullptr;
    const uint8_t *const mask = masked ? A.b.mask : (const uint8_t *)A.b.norms;
    auto side = [&](int slab) {
        const long r0 = (s0 + slab) * (16 * RT) + col;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const size_t at = (size_t)min(r0 + r * 16, (long)N - 1);
            nrm[r] = A.b.norms[at];
            mk[r] = mask[at];
        }
    };
    auto end = [&](int slab, f32x4(&acc)[RT][NG]) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            __builtin_amdgcn_sched_barrier(0);
            const long row = (s0 + slab) * (16 * RT) + r * 16 + col;
            const float nh = -0.5f * nrm[r];
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += __builtin_amdgcn_exp2f(
                        fmaf(c, acc[r][g][e] + (nh + hq[g][e]), -lse2[g][e]));
            sum = rows_reduce(sum, [](float x, float y) { return x + y; });
            if (masked && mk[r] == 0)
                sum = 0.f;
            if (jg == 0 && row < N) {
                if (A.part)
                    A.part[(size_t)t * N + row] = sum;
                else
                    A.usage[row] = fmaf(A.decay, A.usage[row], sum);
            }
        }
    };
    scan_slabs<DT, NG, RT, at_ring(DT, RT), true>(A.b, A.nks, qs, s0, s1, lane, side, end);
}

__global__ __launch_bounds__(256) void usage_join_kernel(const float *part, int n_qt, int N,
                                                         float decay, float *usage)
{
    const long n = (long)blockIdx.x * 256 + threadIdx.x;
    if (n >= N)
        return;
    float s = 0.f;
    for (int t = 0; t < n_qt; ++t)
        s += part[(size_t)t * N + n];
    usage[n] = fmaf(decay, usage[n], s);
}

__global__ __launch_bounds__(256) void decay_kernel(float *usage, int N, float decay)
{
    const long n = (long)blockIdx.x * 256 + threadIdx.x;
    if (n < N)
        usage[n] *= decay;
}

__global__ __launch_bounds__(256) void zero_kernel(uint32_t *p, size_t words)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256)
        p[i] = 0;
}

struct DsArgs {
    AttendBank b;
    const float *qual, *len;
    int M;
    const Side *side;
    const float *dout;      // [B][pitch]
    int pitch;
    int nks, n_chunks, n_qt, n_blk;
    long slab0, slabs;      // this part
    i32x4 *ds;              // of this part, null if neither product is wanted
    float *rowsum;          // [n_qt][rows of a part]
    long part_rows;
    float *d_qual, *d_len;  // [n_qt][N][M] each, or the results where n_qt is 1; null: not wanted
    float *req;             // [n_chunks][B][2] sums of ds and of -ds * distance
    bool first;             // the first part sets req, the others add
};

// Where lane l (bank row l % 16, requests 4*(l/16) ..) of a fragment of ds has
// its 16 bytes: rows turned by 4 for each four requests, so that reading it
// across (four rows, 16 requests) meets every bank once.
__device__ __forceinline__ int ds_place(int lane)
{
    return (lane & 48) | ((lane & 15) ^ ((lane >> 4) << 2));
}

// ds of a part: p from the recomputed scores, dp = dout . labels by fp32 MFMA,
// ds = p * (dp - shift). It goes out as MFMA fragments of the products that
// follow: bf16 banks as two bf16 values, hi + lo = ds to 2^-17 (one value
// alone, 2^-9, would add as much error to the gradients as their own rounding
// does); fp32 banks as it is. With the bank's rows over the lanes, p is also
// the operand of the labels' gradient p^T . dout as it stands.
template <int DT, int NG, bool TAB>
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void ds_kernel(const DsArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    i32x4 *qs = (i32x4 *)smem;
    float *sd = (float *)(qs + (size_t)A.nks * NG * WAVE);   // [3][NG * 16] hq, lse2, shift
    float *tab = sd + 4 * NG * 16;                           // [NG * 16][pitch]
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int n_waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int q0 = t * NG * 16;
    const long gw = (long)ch * n_waves + wave, n_gw = (long)A.n_chunks * n_waves;
    const long s0 = A.slab0 + gw * A.slabs / n_gw, s1 = A.slab0 + (gw + 1) * A.slabs / n_gw;
    const int N = A.b.N, M = A.M;
    const float c = A.b.c;
    load_requests<DT, NG>(A.b, A.nks, q0, qs, wave, n_waves, lane);
    for (int i = tid; i < NG * 16; i += blockDim.x) {
        const Side x = q0 + i < A.b.B ? A.side[q0 + i] : Side{0.f, INFINITY, 0.f, 0.f};
        sd[i] = x.hq;
        sd[NG * 16 + i] = x.lse2;
        sd[2 * NG * 16 + i] = x.shift;
    }
    // of this lane's four requests of group g
    auto side4 = [&](int which, int g) {
        return *(const f32x4 *)(sd + which * NG * 16 + g * 16 + 4 * jg);
    };
    if constexpr (TAB)
        for (int i = tid; i < NG * 16 * A.pitch; i += blockDim.x)
            tab[i] = q0 + i / A.pitch < A.b.B ? A.dout[(size_t)q0 * A.pitch + i] : 0.f;
    wait_vmcnt<0>();
    stream_barrier();
    // label gradient column cc of request q of the tile
    auto dout = [&](int q, int cc) -> float {
        if constexpr (TAB)
            return tab[q * A.pitch + cc];
        else
            return A.dout[(size_t)min(q0 + q, A.b.B - 1) * A.pitch + cc];
    };
    float sum_ds[NG][4], sum_db[NG][4];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum_ds[g][e] = sum_db[g][e] = 0.f;
    float nrm[AT_RT], vr[AT_RT][4];   // norms, mask, the first 16 label columns
    uint8_t mk[AT_RT];
    const bool masked = A.b.mask != nullptr;
    const uint8_t *const mask = masked ? A.b.mask : (const uint8_t *)A.b.norms;
    const float *lab[4];   // label column 4*j + jg
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int cc = 4 * j + jg;
        lab[j] = cc < M ? A.qual + cc : cc < 2 * M ? A.len + (cc - M) : A.qual;
    }
    auto side = [&](int slab) {
        const long r0 = (s0 + slab) * AT_SLAB + col;
#pragma unroll
        for (int r = 0; r < AT_RT; ++r) {
            const size_t at = (size_t)min(r0 + r * 16, (long)N - 1);
            nrm[r] = A.b.norms[at];
            mk[r] = mask[at];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                vr[r][j] = lab[j][at * M];
        }
    };
    const int n_ct = (2 * M + 15) / 16;
    auto end = [&](int slab, f32x4(&acc)[AT_RT][NG]) {
        const long row0 = (s0 + slab) * AT_SLAB + col;
        float nh[AT_RT];   // -inf for rows masked or past the bank
#pragma unroll
        for (int r = 0; r < AT_RT; ++r)
            nh[r] = row0 + r * 16 < N && !(masked && mk[r] == 0) ? -0.5f * nrm[r] : -INFINITY;
        // ---- dp: 4 label columns a step, request groups x row tiles
        f32x4 dp[AT_RT][NG];
#pragma unroll
        for (int r = 0; r < AT_RT; ++r)
#pragma unroll
            for (int g = 0; g < NG; ++g)
                dp[r][g] = -side4(2, g);
        // (a masked row's labels may be no numbers)
        auto dp_step = [&](int c0, float(&x)[AT_RT]) {
            const int cc = c0 + jg;
#pragma unroll
            for (int r = 0; r < AT_RT; ++r)
                x[r] = nh[r] != -INFINITY && cc < 2 * M ? x[r] : 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float a = dout(g * 16 + col, cc);
#pragma unroll
                for (int r = 0; r < AT_RT; ++r)
                    dp[r][g] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, x[r], dp[r][g], 0, 0, 0);
            }
        };
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * j < 2 * M) {
                float x[AT_RT];
#pragma unroll
                for (int r = 0; r < AT_RT; ++r)
                    x[r] = vr[r][j];
                dp_step(4 * j, x);
            }
        for (int c0 = 16; c0 < 2 * M; c0 += 4) {
            const int cc = c0 + jg;
            float x[AT_RT];
#pragma unroll
            for (int r = 0; r < AT_RT; ++r) {
                const size_t at = (size_t)min(row0 + r * 16, (long)N - 1) * M;
                x[r] = cc < M ? A.qual[at + cc] : cc < 2 * M ? A.len[at + cc - M] : 0.f;
            }
            dp_step(c0, x);
        }
        // ---- p in place of the scores, ds in place of dp
        float rs[AT_RT];
#pragma unroll
        for (int r = 0; r < AT_RT; ++r) {
            rs[r] = 0.f;
            const bool live = nh[r] != -INFINITY;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                __builtin_amdgcn_sched_barrier(0);
                const f32x4 hq = side4(0, g), lse2 = side4(1, g);
                float hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = live ? acc[r][g][e] + (nh[r] + hq[e]) : 0.f;
                    const float p =
                        live ? __builtin_amdgcn_exp2f(fmaf(c, a, -lse2[e])) : 0.f;
                    const float ds = p * dp[r][g][e];
                    acc[r][g][e] = p;
                    sum_db[g][e] = fmaf(2.f * a, ds, sum_db[g][e]);   // -distance = 2 a
                    float held = ds;
                    if constexpr (DT == AT_BF16) {
                        hi[e] = (float)(__bf16)ds;
                        lo[e] = (float)(__bf16)(ds - hi[e]);
                        held = hi[e] + lo[e];
                    }
                    dp[r][g][e] = ds;
                    sum_ds[g][e] += held;
                    rs[r] += held;
                }
                if constexpr (DT == AT_BF16) {
                    // two bf16 to a register: hi in dp's first two, lo in its last two
                    auto two = [](float x, float y) {
                        return __uint_as_float((__float_as_uint(y) & 0xffff0000u) |
                                               (__float_as_uint(x) >> 16));
                    };
                    dp[r][g] = f32x4{two(hi[0], hi[1]), two(hi[2], hi[3]), two(lo[0], lo[1]),
                                     two(lo[2], lo[3])};
                }
            }
        }
        // ---- fragments of ds: [row tile][block of requests][hi, lo][64]
        if (A.ds) {
            const long tile0 = (s0 + slab - A.slab0) * AT_RT;
            const int place = ds_place(lane);
#pragma unroll
            for (int r = 0; r < AT_RT; ++r) {
                if constexpr (DT == AT_BF16) {
#pragma unroll
                    for (int g = 0; g < NG; g += 2) {
                        const int blk = (q0 >> 5) + (g >> 1);
                        if (blk >= A.n_blk)
                            break;
                        const f32x4 x = dp[r][g];
                        f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
                        if (g + 1 < NG)
                            y = dp[r][g + 1 < NG ? g + 1 : g];
                        i32x4 *at = A.ds + ((tile0 + r) * A.n_blk + blk) * 2 * WAVE + place;
                        at[0] = __builtin_bit_cast(i32x4, f32x4{x[0], x[1], y[0], y[1]});
                        at[WAVE] = __builtin_bit_cast(i32x4, f32x4{x[2], x[3], y[2], y[3]});
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const int blk = (q0 >> 4) + g;
                        if (blk < A.n_blk)
                            A.ds[((tile0 + r) * A.n_blk + blk) * WAVE + place] =
                                __builtin_bit_cast(i32x4, dp[r][g]);
                    }
                }
                const float sum = rows_reduce(rs[r], [](float x, float y) { return x + y; });
                if (jg == 0)
                    A.rowsum[(size_t)t * A.part_rows + (tile0 + r) * 16 + col] = sum;
            }
        }
        // ---- the labels' gradient: 16 columns x 16 rows, 4 requests a step
        if (A.d_qual || A.d_len) {
            for (int k = 0; k < n_ct; ++k) {
                f32x4 dv[AT_RT];
#pragma unroll
                for (int r = 0; r < AT_RT; ++r)
                    dv[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = dout(g * 16 + 4 * jg + e, k * 16 + col);
#pragma unroll
                        for (int r = 0; r < AT_RT; ++r)
                            dv[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, acc[r][g][e], dv[r],
                                                                         0, 0, 0);
                    }
#pragma unroll
                for (int r = 0; r < AT_RT; ++r) {
                    const long row = row0 + r * 16;
                    if (row < N)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int cc = k * 16 + 4 * jg + e;
                            const size_t at = ((size_t)t * N + row) * M;
                            if (cc < M) {
                                if (A.d_qual)
                                    A.d_qual[at + cc] = dv[r][e];
                            } else if (cc < 2 * M && A.d_len)
                                A.d_len[at + cc - M] = dv[r][e];
                        }
                }
            }
        }
    };
    scan_slabs<DT, NG, AT_RT, at_ring(DT, AT_RT), true>(A.b, A.nks, qs, s0, s1, lane, side, end);

    // ---- the requests' sums, joined over the waves
    float *jn = (float *)smem;   // [n_waves][NG * 16][2]
    stream_barrier();
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            auto add = [](float x, float y) { return x + y; };
            const float x = row16_reduce(sum_ds[g][e], add), y = row16_reduce(sum_db[g][e], add);
            if (col == 0) {
                float *at = jn + (wave * NG * 16 + g * 16 + 4 * jg + e) * 2;
                at[0] = x;
                at[1] = y;
            }
        }
    stream_barrier();
    for (int i = tid; i < NG * 32; i += blockDim.x) {
        if (q0 + i / 2 >= A.b.B)
            continue;
        float s = 0.f;
        for (int w = 0; w < n_waves; ++w)
            s += jn[w * NG * 32 + i];
        float *at = A.req + ((size_t)ch * A.b.B + q0) * 2 + i;
        *at = A.first ? s : *at + s;
    }
}

// Fragments of the requests for d_bank: [block of requests][16 columns][64]
// lanes, lane (column l % 16, requests 4*(l/16) .. of a group; bf16: of two).
template <int QDT>
__global__ __launch_bounds__(256) void qpack_kernel(const uint8_t *queries, int B, int d, int n_blk,
                                                    int n_dt, i32x4 *out)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long)n_blk * n_dt * WAVE)
        return;
    const int lane = (int)(i % WAVE), dt = (int)(i / WAVE % n_dt), blk = (int)(i / WAVE / n_dt);
    const int colm = dt * 16 + (lane & 15), jg = lane >> 4;
    i32x4 r = i32x4{0, 0, 0, 0};
    if (colm < d) {
        if constexpr (QDT == 1) {
            const uint16_t *q = (const uint16_t *)queries;
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = blk * 32 + (j >> 2) * 16 + 4 * jg + (j & 3);
                v[j] = b < B ? q[(size_t)b * d + colm] : 0u;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                r[j] = (int)(v[2 * j] | (v[2 * j + 1] << 16));
        } else {
            const int *q = (const int *)queries;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = blk * 16 + 4 * jg + j;
                r[j] = b < B ? q[(size_t)b * d + colm] : 0;
            }
        }
    }
    out[i] = r;
}

// Four elements of a gradient, rounded once.
template <int DT>
__device__ __forceinline__ void store4(uint8_t *base, size_t at, const f32x4 &v)
{
    if constexpr (DT == AT_F32) {
        *(f32x4 *)(base + at * 4) = v;
    } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *(bf16x4 *)(base + at * 2) =
            bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    }
}

template <int DT>
__device__ __forceinline__ f32x4 load4(const uint8_t *base, size_t at)
{
    if constexpr (DT == AT_F32) {
        return *(const f32x4 *)(base + at * 4);
    } else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 w = *(const u32x2 *)(base + at * 2);
        return f32x4{bf16lo(w[0]), bf16hi(w[0]), bf16lo(w[1]), bf16hi(w[1])};
    }
}

struct DxArgs {
    const i32x4 *ds, *qpack;
    const float *rowsum;
    const uint8_t *rows, *mask;
    uint8_t *d_bank;
    int n_blk, n_dt, n_qt, d;
    long part_rows, row0, nrows;   // rows of this part
    float scale;                   // 2 * beta
};

constexpr int DX_COLS = 8;   // 16-column tiles of a wave

// d_bank of a part: 2 beta (ds^T . q - x * sum of ds). A wave has 32 rows x 128
// columns, D[column 4*(lane/16) + e][row lane % 16].
template <int DT>
__global__ __launch_bounds__(256) void dx_kernel(const DxArgs A)
{
    constexpr int H = DT == AT_BF16 ? 2 : 1;   // values of ds
    constexpr int MDT = DT == AT_F32 ? 0 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, jg = lane >> 4;
    const long r0 = ((long)blockIdx.x * 4 + wave) * AT_SLAB;
    if (r0 >= A.nrows)
        return;
    const int dt0 = blockIdx.y * DX_COLS;
    const int place = ds_place(lane);
    f32x4 acc[AT_RT][DX_COLS];
#pragma unroll
    for (int r = 0; r < AT_RT; ++r)
#pragma unroll
        for (int k = 0; k < DX_COLS; ++k)
            acc[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    const i32x4 *ds = A.ds + (r0 / 16) * A.n_blk * H * WAVE + place;
    for (int blk = 0; blk < A.n_blk; ++blk) {
        i32x4 s[AT_RT][H];
#pragma unroll
        for (int r = 0; r < AT_RT; ++r)
#pragma unroll
            for (int h = 0; h < H; ++h)
                s[r][h] = ds[((size_t)r * A.n_blk + blk) * H * WAVE + h * WAVE];
        const i32x4 *qp = A.qpack + ((size_t)blk * A.n_dt + dt0) * WAVE + lane;
#pragma unroll
        for (int k = 0; k < DX_COLS; ++k) {
            const i32x4 q = qp[(dt0 + k < A.n_dt ? k : 0) * WAVE];
#pragma unroll
            for (int r = 0; r < AT_RT; ++r)
#pragma unroll
                for (int h = 0; h < H; ++h)
                    acc[r][k] = mfma_step<MDT>(q, s[r][h], acc[r][k]);
        }
    }
#pragma unroll
    for (int r = 0; r < AT_RT; ++r) {
        const long lr = r0 + r * 16 + col;
        if (lr >= A.nrows)
            continue;
        float sum = 0.f;
        for (int t = 0; t < A.n_qt; ++t)
            sum += A.rowsum[(size_t)t * A.part_rows + lr];
        const size_t row = (size_t)(A.row0 + lr);
        const bool live = !A.mask || A.mask[row] != 0;
#pragma unroll
        for (int k = 0; k < DX_COLS; ++k) {
            const int c0 = (dt0 + k) * 16 + 4 * jg;
            if (c0 >= A.d)
                continue;
            const f32x4 x = load4<DT>(A.rows, row * A.d + c0);
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = live ? A.scale * (acc[r][k][e] - x[e] * sum) : 0.f;
            store4<DT>(A.d_bank, row * A.d + c0, v);
        }
    }
}

struct DqArgs {
    const i32x4 *ds;
    const uint8_t *rows, *mask;
    int B, d, n_blk, n_chunks;
    long row0, nrows, slabs;   // rows and slabs of this part
    float *part;               // [n_chunks][B][d]
    bool first;                // the first part sets part, the others add
};

constexpr int DQ_COLS = 256, DQ_GROUPS = 8;   // columns and request groups of a workgroup

// Partial d_queries of a share of a part: sum over its rows of ds * row. A
// workgroup of 8 waves has 256 columns x 128 requests, a wave 64 x 64; 32 rows
// at a time go through LDS, read across (ds_read_b64_tr_b16: four rows of 16
// columns become a column's four rows per lane) for the product over rows:
// D[column 4*(lane/16) + e][request lane % 16].
template <int DT>
__global__ __launch_bounds__(512, 1) void dq_kernel(const DqArgs A)
{
    constexpr int H = DT == AT_BF16 ? 2 : 1;
    constexpr int ESZ = DT == AT_F32 ? 4 : 2;
    constexpr int ROWB = DQ_COLS * ESZ;               // bytes of a row in LDS
    constexpr int XB = AT_SLAB * ROWB;                // a slab's rows
    // ds of a slab: bf16 [2 row tiles][4 blocks][2][64], fp32 [2][8][64] of 16 bytes
    constexpr int NB = DT == AT_BF16 ? DQ_GROUPS / 2 : DQ_GROUPS;
    constexpr int SB = AT_RT * NB * H * WAVE * 16;
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int wd = wave & 3, wq = wave >> 2;   // 64 columns, 4 groups of this wave
    const int c0 = blockIdx.y * DQ_COLS, b0 = blockIdx.z * NB;
    const long z0 = (long)blockIdx.x * A.slabs / A.n_chunks,
               z1 = (long)(blockIdx.x + 1) * A.slabs / A.n_chunks;
    const uint32_t rowb = (uint32_t)A.d * ESZ;

    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            acc[i][g] = f32x4{0.f, 0.f, 0.f, 0.f};

    // slab z into buffer (z - z0) & 1
    constexpr int XL = XB / 1024, SL = SB / 1024;   // loads of 64 x 16 bytes
    auto issue = [&](long z) {
        uint8_t *buf = smem + ((z - z0) & 1) * (XB + SB);
        const long r0 = z * AT_SLAB;
        const int rows = (int)max(0L, min((long)AT_SLAB, A.nrows - r0));
        const __amdgpu_buffer_rsrc_t rx = make_rsrc(A.rows + (size_t)(A.row0 + r0) * rowb,
                                                    z < z1 ? (uint32_t)rows * rowb : 0u);
#pragma unroll
        for (int j = 0; j < XL / 8; ++j) {
            const int f = wave * (XL / 8) + j;
            const int pos = f * 64 + lane;              // 16-byte places, row by row
            const int row = pos / (ROWB / 16), at = pos % (ROWB / 16);
            const int swz = DT == AT_BF16 ? (row & 3) * 2 : ((row >> 2) & 3) * 4;
            const uint32_t byte = (uint32_t)c0 * ESZ + (uint32_t)(at ^ swz) * 16;
            dma16(rx, (i32x4 *)(buf + f * 1024),
                  byte < rowb ? (uint32_t)row * rowb + byte : OFF_NONE);
        }
        const __amdgpu_buffer_rsrc_t rs =
            make_rsrc(A.ds + (size_t)z * AT_RT * A.n_blk * H * WAVE,
                      z < z1 ? (uint32_t)(AT_RT * A.n_blk * H * WAVE * 16) : 0u);
#pragma unroll
        for (int j = 0; j < SL / 8; ++j) {
            const int f = wave * (SL / 8) + j;
            const int r = f / (NB * H), rest = f % (NB * H);
            const int blk = b0 + rest / H, h = rest % H;
            dma16(rs, (i32x4 *)(buf + XB + f * 1024),
                  blk < A.n_blk ? (uint32_t)((((r * A.n_blk + blk) * H + h) * WAVE + lane) * 16)
                                : OFF_NONE);
        }
    };
    constexpr int LOADS = XL / 8 + SL / 8;
    issue(z0);
    for (long z = z0; z < z1; ++z) {
        issue(z + 1);
        wait_vmcnt<LOADS>();
        stream_barrier();
        const uint8_t *xb = smem + ((z - z0) & 1) * (XB + SB), *sb = xb + XB;
        if constexpr (DT == AT_BF16) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 *lds4;
            // rows that are masked hold anything: 0 in their places
            uint32_t keep[4] = {~0u, ~0u, ~0u, ~0u};
            if (A.mask) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long row = z * AT_SLAB + (j >> 2) * 16 + 4 * jg + (j & 3);
                    const bool ok = row < A.nrows && A.mask[A.row0 + row] != 0;
                    if (!ok)
                        keep[j >> 1] &= (j & 1) ? 0x0000ffffu : 0xffff0000u;
                }
            }
            i32x4 a[4];
            const int ti = lane & 15;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = r * 16 + 4 * jg + (ti >> 2);
                    const int el = wd * 64 + i * 16 + 4 * (ti & 3);
                    const uint8_t *p =
                        xb + row * ROWB + ((el >> 3) ^ ((row & 3) * 2)) * 16 + (el & 7) * 2;
                    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p);
                    typedef int i32x2 __attribute__((ext_vector_type(2)));
                    const i32x2 w = __builtin_bit_cast(i32x2, v);
                    a[i][2 * r] = (int)((uint32_t)w[0] & keep[2 * r]);
                    a[i][2 * r + 1] = (int)((uint32_t)w[1] & keep[2 * r + 1]);
                }
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // group wq*4 + g: half g & 1 of block wq*2 + g/2
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    i32x4 s;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int src = (ti & 3) * 16 + 4 * jg + (ti >> 2);   // the lane that wrote it
                        const uint8_t *p = sb +
                                           (size_t)((r * NB + wq * 2 + (g >> 1)) * 2 + h) * 1024 +
                                           ds_place(src) * 16 + (g & 1) * 8;
                        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p);
                        typedef int i32x2 __attribute__((ext_vector_type(2)));
                        const i32x2 w = __builtin_bit_cast(i32x2, v);
                        s[2 * r] = w[0];
                        s[2 * r + 1] = w[1];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[i][g] = mfma_step<1>(a[i], s, acc[i][g]);
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < AT_RT; ++r) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = r * 16 + 4 * jg + e;
                    bool ok = true;
                    if (A.mask) {
                        const long at = z * AT_SLAB + row;
                        ok = at < A.nrows && A.mask[A.row0 + at] != 0;
                    }
                    float x[4], s[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int el = wd * 64 + i * 16 + col;
                        const float y = *(const float *)(xb + row * ROWB +
                                                         ((el >> 2) ^ (jg * 4)) * 16 + (el & 3) * 4);
                        x[i] = ok ? y : 0.f;
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int src = (col >> 2) * 16 + 4 * jg + e;
                        s[g] = *(const float *)(sb + (size_t)(r * NB + wq * 4 + g) * 1024 +
                                                ds_place(src) * 16 + (col & 3) * 4);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            acc[i][g] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], s[g], acc[i][g],
                                                                             0, 0, 0);
                }
            }
        }
        stream_barrier();   // (the slab after next comes into this buffer)
    }
    wait_vmcnt<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int cc = c0 + wd * 64 + i * 16 + 4 * jg;
            const int b = (DT == AT_BF16 ? b0 * 32 : b0 * 16) + (wq * 4 + g) * 16 + col;
            if (cc < A.d && b < A.B) {
                f32x4 *at = (f32x4 *)(A.part + ((size_t)blockIdx.x * A.B + b) * A.d + cc);
                *at = A.first ? acc[i][g] : *at + acc[i][g];
            }
        }
}

// d_queries and d_beta: the shares' sums, 2 beta (sum - q * sum of ds).
template <int DT>
__global__ __launch_bounds__(256) void dq_join_kernel(const float *part, int n_part,
                                                      const float *req, int n_req,
                                                      const uint8_t *queries, int B, int d,
                                                      float scale, uint8_t *d_queries,
                                                      float *d_beta)
{
    __shared__ float red[2][256];
    const int b = blockIdx.x, tid = threadIdx.x;
    float s0 = 0.f, s1 = 0.f;
    for (int k = tid; k < n_req; k += 256) {
        const float *at = req + ((size_t)k * B + b) * 2;
        s0 += at[0];
        s1 += at[1];
    }
    red[0][tid] = s0;
    red[1][tid] = s1;
    __syncthreads();
    for (int k = 128; k > 0; k >>= 1) {
        if (tid < k) {
            red[0][tid] += red[0][tid + k];
            red[1][tid] += red[1][tid + k];
        }
        __syncthreads();
    }
    const float sum = red[0][0];
    if (tid == 0 && d_beta)
        d_beta[b] = red[1][0];
    if (!d_queries)
        return;
    for (int c0 = tid * 4; c0 < d; c0 += 1024) {
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < n_part; ++k)
            v += *(const f32x4 *)(part + ((size_t)k * B + b) * d + c0);
        const f32x4 q = load4<DT>(queries, (size_t)b * d + c0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = scale * (v[e] - q[e] * sum);
        store4<DT>(d_queries, (size_t)b * d + c0, v);
    }
}

// The request tiles' label gradients, added in order.
__global__ __launch_bounds__(256) void label_join_kernel(const float *part, int n_qt, size_t n,
                                                         float *out)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n)
        return;
    float s = 0.f;
    for (int t = 0; t < n_qt; ++t)
        s += part[(size_t)t * n + i];
    out[i] = s;
}

template <typename K>
hipError_t allow_lds(K kern, size_t bytes)
{
    return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize,
                               (int)bytes);
}

template <int DT, int NG, int RT>
hipError_t usage_one(const UsagePlan &p, const UsageArgs &a, hipStream_t s)
{
    auto kern = usage_kernel<DT, NG, RT>;
    const hipError_t e = allow_lds(kern, p.lds_bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(p.n_chunks * p.n_qt), dim3(p.waves * WAVE), p.lds_bytes, s, a);
    return hipGetLastError();
}

template <int DT>
hipError_t usage_dt(const UsagePlan &p, const UsageArgs &a, hipStream_t s)
{
    switch (p.ng) {
    case 1: return usage_one<DT, 1, 2>(p, a, s);
    case 2: return usage_one<DT, 2, 2>(p, a, s);
    case 4: return usage_one<DT, 4, at_rt(DT, 4)>(p, a, s);
    }
    return hipErrorInvalidValue;
}

template <int DT, int NG, bool TAB>
hipError_t ds_one(const GradPlan &p, const DsArgs &a, hipStream_t s)
{
    auto kern = ds_kernel<DT, NG, TAB>;
    const hipError_t e = allow_lds(kern, p.lds_bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(p.n_chunks * p.n_qt), dim3(p.waves * WAVE), p.lds_bytes, s, a);
    return hipGetLastError();
}

template <int DT>
hipError_t ds_dt(const GradPlan &p, const DsArgs &a, hipStream_t s)
{
    switch (p.ng) {
    case 1: return p.tab ? ds_one<DT, 1, true>(p, a, s) : ds_one<DT, 1, false>(p, a, s);
    case 2: return p.tab ? ds_one<DT, 2, true>(p, a, s) : ds_one<DT, 2, false>(p, a, s);
    case 4: return p.tab ? ds_one<DT, 4, true>(p, a, s) : ds_one<DT, 4, false>(p, a, s);
    }
    return hipErrorInvalidValue;
}

// Shares of `slabs` slabs for n_qt request tiles: about one workgroup per
// compute unit, a wave's part of the bank under 1 GB.
void shares(int slabs, int slab, int dtype, int d, int n_qt, int n_cu, int *n_chunks, int *waves)
{
    long chunks = n_cu / n_qt;
    const long by_size = ((long)slabs * slab * at_row_bytes(dtype, d) >> 30) / AT_WAVES + 1;
    if (chunks < by_size)
        chunks = by_size;
    if (chunks > slabs)
        chunks = slabs;
    if (chunks < 1)
        chunks = 1;
    const long per = (slabs + chunks - 1) / chunks;
    *n_chunks = (int)chunks;
    *waves = per < AT_WAVES ? (int)per : AT_WAVES;
}

template <int QDT>
hipError_t run_side(const AttendBank &b, int M, const float *lse, const GradArgs *g, float *dout,
                    int pitch, Side *side, hipStream_t s)
{
    hipLaunchKernelGGL(side_kernel<QDT>, dim3((b.B + 3) / 4), dim3(256), 0, s, b.queries, b.B, b.d,
                       M, lse, g ? g->q_hat : nullptr, g ? g->l_hat : nullptr,
                       g ? g->dq_hat : nullptr, g ? g->dl_hat : nullptr, g ? g->dlse : nullptr,
                       dout, pitch, side);
    return hipGetLastError();
}

template <int DT>
hipError_t run_grad(const GradPlan &p, const AttendBank &b, const GradArgs &g, uint8_t *wb,
                    hipStream_t s)
{
    constexpr int QDT = DT == AT_F32 ? 0 : 1;
    constexpr int H = DT == AT_BF16 ? 2 : 1;
    Side *side = (Side *)(wb + p.off_side);
    float *dout = (float *)(wb + p.off_dout);
    i32x4 *qpack = (i32x4 *)(wb + p.off_qpack);
    hipError_t e = run_side<QDT>(b, g.M, g.lse, &g, dout, p.pitch, side, s);
    if (e != hipSuccess)
        return e;
    const int n_dt = (b.d + 15) / 16;
    if (g.d_bank) {
        const long n = (long)p.n_blk * n_dt * WAVE;
        hipLaunchKernelGGL(qpack_kernel<QDT>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s,
                           b.queries, b.B, b.d, p.n_blk, n_dt, qpack);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
    }
    DsArgs a;
    a.b = b;
    a.qual = g.qual;
    a.len = g.len;
    a.M = g.M;
    a.side = side;
    a.dout = dout;
    a.pitch = p.pitch;
    a.nks = p.nks;
    a.n_chunks = p.n_chunks;
    a.n_qt = p.n_qt;
    a.n_blk = p.n_blk;
    a.ds = g.d_queries || g.d_bank ? (i32x4 *)(wb + p.off_ds) : nullptr;
    a.rowsum = (float *)(wb + p.off_rowsum);
    a.part_rows = (long)p.part_slabs * AT_SLAB;
    float *lab = (float *)(wb + p.off_lab);
    const size_t n_lab = (size_t)b.N * g.M;
    a.d_qual = g.d_qual && p.n_qt > 1 ? lab : g.d_qual;
    a.d_len = g.d_len && p.n_qt > 1 ? lab + n_lab * p.n_qt : g.d_len;
    a.req = (float *)(wb + p.off_req);
    float *dq = (float *)(wb + p.off_dq);
    const float scale = 2.f * g.beta;
    for (int z0 = 0; z0 < p.slabs; z0 += p.part_slabs) {
        const int slabs = p.slabs - z0 < p.part_slabs ? p.slabs - z0 : p.part_slabs;
        const long row0 = (long)z0 * AT_SLAB;
        const long nrows = b.N - row0 < (long)slabs * AT_SLAB ? b.N - row0 : (long)slabs * AT_SLAB;
        a.slab0 = z0;
        a.slabs = slabs;
        a.first = z0 == 0;
        if ((e = ds_dt<DT>(p, a, s)) != hipSuccess)
            return e;
        if (g.d_queries) {
            DqArgs q{a.ds, b.rows, b.mask, b.B, b.d, p.n_blk, p.q_chunks, row0, nrows, slabs, dq,
                     z0 == 0};
            constexpr int NB = DT == AT_BF16 ? DQ_GROUPS / 2 : DQ_GROUPS;
            const size_t lds = 2 * (size_t)(AT_SLAB * DQ_COLS * (DT == AT_F32 ? 4 : 2) +
                                            AT_RT * NB * H * WAVE * 16);
            if ((e = allow_lds(dq_kernel<DT>, lds)) != hipSuccess)
                return e;
            hipLaunchKernelGGL(dq_kernel<DT>,
                               dim3(p.q_chunks, (b.d + DQ_COLS - 1) / DQ_COLS,
                                    (p.n_blk + NB - 1) / NB),
                               dim3(512), lds, s, q);
            if ((e = hipGetLastError()) != hipSuccess)
                return e;
        }
        if (g.d_bank) {
            DxArgs x{a.ds, qpack, a.rowsum, b.rows, b.mask, (uint8_t *)g.d_bank, p.n_blk, n_dt,
                     p.n_qt, b.d, a.part_rows, row0, nrows, scale};
            hipLaunchKernelGGL(dx_kernel<DT>,
                               dim3((unsigned)((nrows + 4 * AT_SLAB - 1) / (4 * AT_SLAB)),
                                    (n_dt + DX_COLS - 1) / DX_COLS),
                               dim3(256), 0, s, x);
            if ((e = hipGetLastError()) != hipSuccess)
                return e;
        }
    }
    if (g.d_queries || g.d_beta) {
        hipLaunchKernelGGL(dq_join_kernel<DT>, dim3(b.B), dim3(256), 0, s, dq, p.q_chunks, a.req,
                           p.n_chunks, b.queries, b.B, b.d, scale, (uint8_t *)g.d_queries,
                           g.d_beta);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
    }
    if (p.n_qt > 1) {
        const unsigned blocks = (unsigned)((n_lab + 255) / 256);
        if (g.d_qual)
            hipLaunchKernelGGL(label_join_kernel, dim3(blocks), dim3(256), 0, s, a.d_qual, p.n_qt,
                               n_lab, g.d_qual);
        if (g.d_len)
            hipLaunchKernelGGL(label_join_kernel, dim3(blocks), dim3(256), 0, s, a.d_len, p.n_qt,
                               n_lab, g.d_len);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

bool plan_usage(int B, int N, int d, int dtype, int n_cu, UsagePlan *p)
{
    const int ks = at_ks(dtype);
    p->dtype = dtype;
    p->nks = (d + ks - 1) / ks;
    const size_t group = (size_t)p->nks * ks * (dtype == AT_F32 ? 4 : 2) * 16 + 16 * sizeof(Side);
    int ng = B <= 16 ? 1 : B <= 32 ? 2 : 4;
    while (ng > 1 && group * ng > (size_t)AT_LDS)
        ng /= 2;
    if (group * ng > (size_t)AT_LDS)
        return false;
    p->ng = ng;
    const int slab = 16 * at_rt(dtype, ng);
    p->slabs = (int)(((long)N + slab - 1) / slab);
    p->n_qt = (B + ng * 16 - 1) / (ng * 16);
    shares(p->slabs, slab, dtype, d, p->n_qt, n_cu, &p->n_chunks, &p->waves);
    p->lds_bytes = group * ng;
    p->off_side = 0;
    p->off_part = up256((size_t)B * sizeof(Side));
    p->bytes = p->off_part + (p->n_qt > 1 ? up256((size_t)p->n_qt * N * 4) : 0);
    return true;
}

hipError_t launch_usage(const UsagePlan &p, const AttendBank &b, const float *lse, float decay,
                        float *usage, void *ws, hipStream_t s)
{
    Side *side = (Side *)((uint8_t *)ws + p.off_side);
    hipError_t e = p.dtype == AT_F32 ? run_side<0>(b, 0, lse, nullptr, nullptr, 0, side, s)
                                     : run_side<1>(b, 0, lse, nullptr, nullptr, 0, side, s);
    if (e != hipSuccess)
        return e;
    UsageArgs a;
    a.b = b;
    a.side = side;
    a.nks = p.nks;
    a.n_chunks = p.n_chunks;
    a.n_qt = p.n_qt;
    a.slabs = p.slabs;
    a.decay = decay;
    a.usage = usage;
    a.part = p.n_qt > 1 ? (float *)((uint8_t *)ws + p.off_part) : nullptr;
    e = p.dtype == AT_F32    ? usage_dt<AT_F32>(p, a, s)
        : p.dtype == AT_BF16 ? usage_dt<AT_BF16>(p, a, s)
                             : usage_dt<AT_Q4>(p, a, s);
    if (e != hipSuccess || p.n_qt == 1)
        return e;
    hipLaunchKernelGGL(usage_join_kernel, dim3((unsigned)(((long)b.N + 255) / 256)), dim3(256), 0, s, a.part, p.n_qt,
                       b.N, decay, usage);
    return hipGetLastError();
}

hipError_t launch_decay(float *usage, int N, float decay, hipStream_t s)
{
    hipLaunchKernelGGL(decay_kernel, dim3((unsigned)(((long)N + 255) / 256)), dim3(256), 0, s,
                       usage, N, decay);
    return hipGetLastError();
}

hipError_t launch_zero(void *p, size_t bytes, hipStream_t s)
{
    const size_t words = bytes / 4, blocks = (words + 255) / 256;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0,
                       s, (uint32_t *)p, words);
    return hipGetLastError();
}

bool plan_grad(int B, int N, int d, int dtype, int M, int n_cu, GradPlan *p)
{
    if (dtype != AT_F32 && dtype != AT_BF16)
        return false;
    const int ks = at_ks(dtype);
    p->dtype = dtype;
    p->nks = (d + ks - 1) / ks;
    p->slabs = (int)(((long)N + AT_SLAB - 1) / AT_SLAB);
    p->pitch = (2 * M + 15) / 16 * 16 + 4;
    const size_t group = (size_t)p->nks * ks * (dtype == AT_F32 ? 4 : 2) * 16 + 16 * sizeof(Side);
    const size_t tab = (size_t)p->pitch * 4 * 16;
    int ng = B <= 16 ? 1 : B <= 32 ? 2 : 4;
    while (ng > 1 && group * ng > (size_t)AT_LDS)
        ng /= 2;
    if (group * ng > (size_t)AT_LDS)
        return false;
    p->tab = (group + tab) * ng <= (size_t)AT_LDS;
    p->ng = ng;
    p->n_qt = (B + ng * 16 - 1) / (ng * 16);
    const int per = dtype == AT_BF16 ? 32 : 16;   // requests of a fragment of ds
    p->n_blk = (B + per - 1) / per;
    // (a fragment of 64 x 16 bytes for 16 rows; bf16: hi and lo)
    const size_t slab_ds = (size_t)AT_RT * p->n_blk * (dtype == AT_BF16 ? 2 : 1) * WAVE * 16;
    long part = (long)(PART_BYTES / slab_ds);
    if (part < 1)
        part = 1;
    if (part > p->slabs)
        part = p->slabs;
    const int n_parts = (int)((p->slabs + part - 1) / part);
    part = (p->slabs + n_parts - 1) / n_parts;
    p->part_slabs = (int)part;
    shares((int)part, AT_SLAB, dtype, d, p->n_qt, n_cu, &p->n_chunks, &p->waves);
    const long tiles = (long)((d + DQ_COLS - 1) / DQ_COLS) *
                       ((B + DQ_GROUPS * 16 - 1) / (DQ_GROUPS * 16));
    long qc = n_cu / tiles;
    qc = qc < 1 ? 1 : qc;
    p->q_chunks = (int)(qc > part ? part : qc);
    const size_t lds = (group + (p->tab ? tab : 0)) * ng;
    const size_t join = (size_t)p->waves * ng * 16 * 2 * 4;
    p->lds_bytes = lds > join ? lds : join;
    const int n_dt = (d + 15) / 16;
    size_t o = 0;
    p->off_side = o;
    o += up256((size_t)B * sizeof(Side));
    p->off_dout = o;
    o += up256((size_t)B * p->pitch * 4);
    p->off_qpack = o;
    o += up256((size_t)p->n_blk * n_dt * WAVE * 16);
    p->off_ds = o;
    o += up256((size_t)part * slab_ds);
    p->off_rowsum = o;
    o += up256((size_t)p->n_qt * part * AT_SLAB * 4);
    p->off_lab = o;
    o += p->n_qt > 1 ? up256((size_t)p->n_qt * N * M * 8) : 0;
    p->off_req = o;
    o += up256((size_t)p->n_chunks * B * 2 * 4);
    p->off_dq = o;
    o += up256((size_t)p->q_chunks * B * d * 4);
    p->bytes = o;
    return true;
}

hipError_t launch_grad(const GradPlan &p, const AttendBank &b, const GradArgs &g, void *ws,
                       hipStream_t s)
{
    return p.dtype == AT_F32 ? run_grad<AT_F32>(p, b, g, (uint8_t *)ws, s)
                             : run_grad<AT_BF16>(p, b, g, (uint8_t *)ws, s);
}

}  // namespace rb
