// Attention of requests over the labelled bank: the passes that recompute its
// probabilities, the rows' accumulated weight and the gradients.
#include "attend_gemm.hpp"

#include <math.h>

namespace rb {

namespace {

constexpr size_t PART_BYTES = 128u << 20;   // ds of a part of the bank

// Per request: -|q|^2/2, lse in powers of two, and what is subtracted from the
// weights' gradient, sum of the outputs' gradients times the outputs less the
// gradient of lse. A request without a row (lse = -inf) gets lse2 = inf, so
// that its weights are 2^(-inf) = 0, as do the places past the batch.
struct Side {
    float hq, lse2, shift, none;
};

struct PrepArgs {
    const uint8_t *queries;
    int B, d, M, n_j;
    int places;      // requests of whole tiles: what follows the batch is zeros
    const float *lse, *q_hat, *l_hat, *dq, *dl, *dlse;
    float *dout;     // label gradients as fragments (dout_place); null: not wanted
    Side *side;
    int n_blk, n_dt; // fragments of the requests, [n_blk][n_dt][64]
    i32x4 *qpack;
    double c, more;  // the passes' c, and what it lacks, over c
};

// The label gradients as MFMA fragments, [group of 16 requests][n_j][64]: column
// c of request b, lane (request % 16, column % 4) of piece c/4. n_j: pieces, a
// multiple of four; columns past the labels and requests past the batch hold 0.
__device__ __forceinline__ size_t dout_place(int b, int c, int n_j)
{
    return ((size_t)(b >> 4) * n_j + (c >> 2)) * WAVE + (c & 3) * 16 + (b & 15);
}

// What rounding lse2 and c takes from the exponent of a row near the request (c * a
// about lse2), of a request's weights as a whole: up to 2^-23 of lse2.
__device__ __forceinline__ double lost_to_rounding(float lse, float lse2, double more)
{
    return lse == -INFINITY
               ? 0.0
               : more * (double)lse2 - ((double)lse * 1.4426950408889634 - (double)lse2);
}

// A weight from its logarithm, c * a - lse2: 1 at most, also where the roundings of a
// and lse (at most 2^-23 of c * a, each) pass 1 and the difference is of no more use.
// NaN stays NaN.
__device__ __forceinline__ float weight_of(float log2w)
{
    return __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(log2w, 0.f));
}

template <int QDT>
__device__ __forceinline__ void make_side(const PrepArgs &A, int b, int lane)
{
    if (b >= A.B) {
        if (A.dout && b < A.places)
            for (int c = lane; c < 4 * A.n_j; c += WAVE)
                A.dout[dout_place(b, c, A.n_j)] = 0.f;
        return;
    }
    const int n16 = A.d * Elem<QDT>::ESZ / 16;
    const uint8_t *q = A.queries + (size_t)b * A.d * Elem<QDT>::ESZ;
    float s = 0.f;
    for (int i = lane; i < n16; i += WAVE)
        s = sumsq16<QDT>(load16(q + (size_t)i * 16), s);
    const double s2 = wave_sum64(s);
    const float lse = A.lse[b];
    const bool alive = lse != -INFINITY;
    const float lse2 = alive ? lse * LOG2E : INFINITY;
    // (the gradients are linear in the weights, and get what rounding lost with the
    // outputs' ones, by a factor of 2 at most: past that all roundings are as large;
    // for the usage it goes into hq)
    const double lost = lost_to_rounding(lse, lse2, A.more);
    const float f = __builtin_amdgcn_exp2f(__builtin_amdgcn_fmed3f((float)lost, -1.f, 1.f));
    double dot = 0.0;
    if (A.dout) {
        // (a dead request's outputs are no numbers, and its gradients may be none)
        for (int c = lane; c < 4 * A.n_j; c += WAVE) {
            float g = 0.f, o = 0.f;
            if (alive && c < 2 * A.M) {
                const size_t at = (size_t)b * A.M + (c < A.M ? c : c - A.M);
                g = f * (c < A.M ? A.dq[at] : A.dl[at]);
                o = c < A.M ? A.q_hat[at] : A.l_hat[at];
            }
            dot += (double)g * (double)o;
            A.dout[dout_place(b, c, A.n_j)] = g;
        }
        // (one rounding of it, which every row's gradient of this request shares)
        dot = wave_sum64(dot);
        if (alive && A.dlse)
            dot -= (double)f * (double)A.dlse[b];
    }
    if (lane == 0)
        A.side[b] =
            Side{(float)((A.dout ? 0.0 : lost / A.c) - 0.5 * s2), lse2, (float)dot, 0.f};
}

// Fragments of the requests for d_bank: [block of requests][16 columns][64]
// lanes, lane (column m = l % 16, requests 4*(l/16) .. of a group; bf16: of
// two). Columns are dealt to pairs of fragments so that a lane's results of a
// pair, m = 4*(l/16) + e of each, are eight that lie side by side.
__device__ __forceinline__ int dealt_column(int dt, int m)
{
    return (dt >> 1) * 32 + (m >> 2) * 8 + (dt & 1) * 4 + (m & 3);
}

template <int QDT>
__device__ __forceinline__ void make_qpack(const PrepArgs &A, long i)
{
    if (i >= (long)A.n_blk * A.n_dt * WAVE)
        return;
    const int lane = (int)(i % WAVE), dt = (int)(i / WAVE % A.n_dt),
              blk = (int)(i / WAVE / A.n_dt);
    const int cc = dealt_column(dt, lane & 15), jg = lane >> 4;
    i32x4 r = i32x4{0, 0, 0, 0};
    if (cc < A.d) {
        if constexpr (QDT == 1) {
            const uint16_t *q = (const uint16_t *)A.queries;
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = blk * 32 + (j >> 2) * 16 + 4 * jg + (j & 3);
                v[j] = b < A.B ? q[(size_t)b * A.d + cc] : 0u;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                r[j] = (int)(v[2 * j] | (v[2 * j + 1] << 16));
        } else {
            const int *q = (const int *)A.queries;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = blk * 16 + 4 * jg + j;
                r[j] = b < A.B ? q[(size_t)b * A.d + cc] : 0;
            }
        }
    }
    A.qpack[i] = r;
}

// What the other passes want of the requests, in one launch: four waves of one
// request each, then blocks of fragments.
template <int QDT>
__global__ __launch_bounds__(256) void prep_kernel(const PrepArgs A, int side_blocks)
{
    if ((int)blockIdx.x < side_blocks) {
        make_side<QDT>(A, blockIdx.x * 4 + (threadIdx.x >> 6), threadIdx.x & 63);
    } else {
        make_qpack<QDT>(A, (long)(blockIdx.x - side_blocks) * 256 + threadIdx.x);
    }
}

struct UsageArgs {
    AttendBank b;
    const float *lse;
    double more;           // what c lacks, over c
    const Side *side;      // of the pass by tiles
    int nks, n_chunks, n_qt;
    long slabs;
    float decay;
    float *usage, *part;   // part [n_qt][N], null where one tile holds the batch
};

// Weights of the bank's rows: as the forward pass, with the bank's rows over
// the lanes, so that a row's sum over the requests is a sum over registers and
// four lanes. There is no running maximum: lse is known. The requests' norms come
// from their tile in LDS (a launch before for them took 4.6 us). Bound as that one: 64
// requests over 100,000 x 768 bf16 32 us, 4.8 TB/s.
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
    for (int i = tid; i < NG * 16; i += blockDim.x) {
        const float lse = q0 + i < A.b.B ? A.lse[q0 + i] : -INFINITY;
        const float lse2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
        sd[i] = Side{(float)(lost_to_rounding(lse, lse2, A.more) / c), lse2, 0.f, 0.f};
    }
    float hq[NG][4], lse2[NG][4];
    auto ready = [&] {
        for (int g = wave; g < NG; g += n_waves) {
            double s = 0.0;
#pragma unroll 4
            for (int f = 0; f < A.nks * AtElem<DT>::SUB; ++f)
                s += sumsq16<DT == AT_F32 ? 0 : 1>(qs[(f * NG + g) * WAVE + lane], 0.f);
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (jg == 0)
                sd[g * 16 + col].hq = (float)((double)sd[g * 16 + col].hq - 0.5 * s);
        }
        stream_barrier();
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Side &x = sd[g * 16 + 4 * jg + e];
                hq[g][e] = x.hq;
                lse2[g][e] = x.lse2;
            }
    };
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
                    sum += weight_of(fmaf(c, (acc[r][g][e] + nh) + hq[g][e], -lse2[g][e]));
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
    scan_slabs<DT, NG, RT, at_ring(DT, RT), true>(A.b, A.nks, qs, s0, s1, lane, ready, side, end);
}

// The same as a matrix product of tiles, for large bf16 batches; part [4 *
// n_qt][N], one of the waves of each 64 requests. 256 requests over 1,000,000 x 768:
// 445 us, 885 TFLOP/s.
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void usage_gemm_kernel(const UsageArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    TileSide *side = (TileSide *)(smem + 2 * AG_SLOT);
    float *sd = (float *)(side + 1);   // [2][256] hq, lse2
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    __builtin_assume(tid < AT_WAVES * WAVE);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int wr = wave >> 2, wq = wave & 3;
    const int q0 = t * AG_REQS;
    const long t0 = (long)ch * A.slabs / A.n_chunks, t1 = (long)(ch + 1) * A.slabs / A.n_chunks;
    const int N = A.b.N;
    const float c = A.b.c;
    if (tid < AG_REQS) {
        const Side x = q0 + tid < A.b.B ? A.side[q0 + tid] : Side{0.f, INFINITY, 0.f, 0.f};
        sd[tid] = x.hq;
        sd[AG_REQS + tid] = x.lse2;
    }
    const bool any = q0 + 64 * wq < A.b.B;
    float *const part = A.part + (size_t)(any ? t * 4 + wq : 0) * N;
    auto end = [&](int tile, f32x4(&acc)[AG_RT][AG_NG]) {
        const long row0 = (t0 + tile) * AG_ROWS;
        const int left = (int)min((long)AG_ROWS, N - row0);
        const __amdgpu_buffer_rsrc_t to = make_rsrc(part + row0, any ? (uint32_t)left * 4u : 0u);
        float sum[AG_RT];
#pragma unroll
        for (int r = 0; r < AG_RT; ++r)
            sum[r] = 0.f;
#pragma unroll
        for (int g = 0; g < AG_NG; ++g) {
            const float *at = sd + 64 * wq + 16 * g + 4 * jg;
            const f32x4 hq = *(const f32x4 *)at, lse2 = *(const f32x4 *)(at + AG_REQS);
#pragma unroll
            for (int r = 0; r < AG_RT; ++r) {
                if (r % 2 == 0)
                    __builtin_amdgcn_sched_barrier(0);
                const float nh = -0.5f * side->norms[128 * wr + 16 * r + col];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum[r] += weight_of(fmaf(c, (acc[r][g][e] + nh) + hq[e], -lse2[e]));
            }
        }
#pragma unroll
        for (int r = 0; r < AG_RT; ++r) {
            float s = rows_reduce(sum[r], [](float x, float y) { return x + y; });
            const int at = 128 * wr + 16 * r + col;
            // (a masked row may hold anything)
            s = tile_norm(A.b, side, left, at) == -INFINITY ? 0.f : s;
            buffer_store4(to, jg == 0 ? (uint32_t)at * 4u : OFF_NONE, s);
        }
    };
    gemm_tiles<true, 0>(A.b, A.nks, smem, side, nullptr, q0, t0, (int)(t1 - t0), wave, lane,
                        [&](long, int, int) { return A.b.norms; }, end);
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
    const float *dout;      // fragments of whole tiles, n_j pieces a group
    int n_j;
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
// across (four rows, 16 requests) meets every bank once. The two halves of a
// bf16 fragment (four requests of one group and of the next) change places in
// rows 4-7 and 12-15, for the sake of reading eight rows at a time.
__device__ __forceinline__ int ds_place(int lane)
{
    return (lane & 48) | ((lane & 15) ^ ((lane >> 4) << 2));
}

// A wave's 16 rows of the bank in the passes below; the same for all its lanes.
struct RowTile {
    long row0, tile16;   // first row, number among the part's row tiles
    int rows;            // rows of the bank in it
    int t, q0;           // request tile (of rowsum and the labels' gradients), its first request
};

// ds of 16 rows and NG groups of requests: p from the recomputed scores, dp =
// dout . labels by fp32 MFMA, ds = p * (dp - shift). It goes out as MFMA fragments
// of the products that follow: bf16 banks as two bf16 values, hi + lo = ds to
// 2^-17 (one value alone, 2^-9, would add as much error to the gradients as their
// own rounding does); fp32 banks as it is. With the bank's rows over the lanes, p
// is also the operand of the labels' gradient p^T . dout as it stands.
//   sd     [3][stride] in LDS: hq, lse2, shift of these requests
//   tab    label gradients of these requests, fragments of n_j pieces
//   sc     <q, x> of row l%16 and requests 16*g + 4*(l/16) + e
//   lab(c) the lane's label, of column c + l/16 in row l%16
template <int DT, int NG, typename Lab>
__device__ __forceinline__ void ds_row_tile(const DsArgs &A, const RowTile &T, const float *sd,
                                            int stride, const float *tab, int l, float nh,
                                            f32x4 (&sc)[NG], Lab &&lab, float (&sum_ds)[NG][4],
                                            float (&sum_db)[NG][4])
{
    const int col = l & 15, jg = l >> 4, M = A.M;
    const float c = A.b.c;
    const bool live = nh != -INFINITY;
    auto side4 = [&](int which, int g) {
        return *(const f32x4 *)(sd + which * stride + 16 * g + 4 * jg);
    };
    // (what the requests have in LDS is read again for every row tile: kept in
    // registers it would not leave room for the scores)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    f32x4 dp[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g)
        dp[g] = -side4(2, g);
    auto dp_step = [&](int j) {
        // (a masked row's labels may be no numbers)
        const float x = live && 4 * j + jg < 2 * M ? lab(j) : 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g)
            dp[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(tab[(g * A.n_j + j) * WAVE + l], x, dp[g],
                                                         0, 0, 0);
    };
    static_for<0, 4>([&](auto J) {
        if (4 * decltype(J)::value < 2 * M)
            dp_step(decltype(J)::value);
    });
    for (int j = 4; 4 * j < 2 * M; ++j)
        dp_step(j);
    // ---- p in place of the scores, ds in place of dp
    float rs = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        __builtin_amdgcn_sched_barrier(0);
        const f32x4 hq = side4(0, g), lse2 = side4(1, g);
        float ds[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = live ? (sc[g][e] + nh) + hq[e] : 0.f;
            const float p = live ? weight_of(fmaf(c, a, -lse2[e])) : 0.f;
            ds[e] = p * dp[g][e];
            sc[g][e] = p;
            sum_db[g][e] = fmaf(2.f * a, ds[e], sum_db[g][e]);   // -distance = 2 a
        }
        if constexpr (DT == AT_BF16) {
            int h[2], w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float y0 = ds[2 * i], y1 = ds[2 * i + 1];
                h[i] = split_bf16(y0, y1);
                w[i] = split_bf16(y0, y1);
                ds[2 * i] -= y0;       // what the two values hold
                ds[2 * i + 1] -= y1;
            }
            dp[g] = __builtin_bit_cast(f32x4, i32x4{h[0], h[1], w[0], w[1]});
        } else {
            dp[g] = f32x4{ds[0], ds[1], ds[2], ds[3]};
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum_ds[g][e] += ds[e];
            rs += ds[e];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    // ---- fragments of ds: [row tile][block of requests][hi, lo][64]
    if (A.ds) {
        constexpr int H = DT == AT_BF16 ? 2 : 1;   // values, and groups of a block
        const uint32_t place = (uint32_t)ds_place(l) * 16;
#pragma unroll
        for (int g = 0; g < NG; g += H) {
            const int blk = T.q0 / (16 * H) + g / H;
            const __amdgpu_buffer_rsrc_t to =
                wave_rsrc(A.ds + (T.tile16 * A.n_blk + min(blk, A.n_blk - 1)) * H * WAVE,
                          blk < A.n_blk ? H * WAVE * 16u : 0u);
            if constexpr (H == 2) {
                const f32x4 none = f32x4{0.f, 0.f, 0.f, 0.f};
                const f32x4 x = dp[g], y = g + 1 < NG ? dp[g + 1 < NG ? g + 1 : g] : none;
                const bool turned = col & 4;
                const f32x4 u = turned ? y : x, w = turned ? x : y;
                __builtin_amdgcn_raw_buffer_store_b128(
                    __builtin_bit_cast(i32x4, f32x4{u[0], u[1], w[0], w[1]}), to, (int)place, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(
                    __builtin_bit_cast(i32x4, f32x4{u[2], u[3], w[2], w[3]}), to,
                    (int)(place + WAVE * 16), 0, 0);
            } else {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, dp[g]), to,
                                                       (int)place, 0, 0);
            }
        }
        rs = rows_reduce(rs, [](float x, float y) { return x + y; });
        buffer_store4(wave_rsrc(A.rowsum + (size_t)T.t * A.part_rows + T.tile16 * 16, 64u),
                      jg == 0 ? (uint32_t)col * 4u : OFF_NONE, rs);
    }
    // ---- the labels' gradient: 16 columns x 16 rows, 4 requests a step
    if (A.d_qual || A.d_len) {
        const size_t at = ((size_t)T.t * A.b.N + T.row0) * M;
        const uint32_t bytes = (uint32_t)(T.rows * M) * 4u;
        const __amdgpu_buffer_rsrc_t to_q =
            wave_rsrc((A.d_qual ? A.d_qual : A.d_len) + at, A.d_qual ? bytes : 0u);
        const __amdgpu_buffer_rsrc_t to_l =
            wave_rsrc((A.d_len ? A.d_len : A.d_qual) + at, A.d_len ? bytes : 0u);
        for (int k = 0; 16 * k < 2 * M; ++k) {
            f32x4 dv = f32x4{0.f, 0.f, 0.f, 0.f};
            const int cl = 16 * k + col;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                // of label column cl, this lane's four requests
                const f32x4 d4 = *(const f32x4 *)(tab + (g * A.n_j + (cl >> 2)) * WAVE +
                                                  (cl & 3) * 16 + 4 * jg);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    dv = __builtin_amdgcn_mfma_f32_16x16x4f32(d4[e], sc[g][e], dv, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int cc = 16 * k + 4 * jg + e;
                const uint32_t to = (uint32_t)(col * M + cc) * 4u;
                buffer_store4(to_q, cc < M ? to : OFF_NONE, dv[e]);
                buffer_store4(to_l, cc >= M && cc < 2 * M ? to - 4u * M : OFF_NONE, dv[e]);
            }
        }
    }
}

// A wave's sums over its rows, [NG][4] of the lane, to places at[request][2].
template <int NG>
__device__ __forceinline__ void put_sums(const float (&sum_ds)[NG][4],
                                         const float (&sum_db)[NG][4], float *at, int lane)
{
    auto add = [](float x, float y) { return x + y; };
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = row16_reduce(sum_ds[g][e], add), y = row16_reduce(sum_db[g][e], add);
            if ((lane & 15) == 0) {
                float *to = at + (16 * g + 4 * (lane >> 4) + e) * 2;
                to[0] = x;
                to[1] = y;
            }
        }
}

// The side data of n requests from q0 on into LDS, [3][n].
__device__ __forceinline__ void load_side(const DsArgs &A, int q0, int n, float *sd)
{
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const Side x = q0 + i < A.b.B ? A.side[q0 + i] : Side{0.f, INFINITY, 0.f, 0.f};
        sd[i] = x.hq;
        sd[n + i] = x.lse2;
        sd[2 * n + i] = x.shift;
    }
}

// The label gradients of a tile of n requests from q0 on into LDS.
__device__ __forceinline__ void load_dout(const DsArgs &A, int q0, int n, float *tab)
{
    const int per = A.n_j * WAVE;
    for (int i = threadIdx.x; i < n / 16 * per; i += blockDim.x)
        tab[i] = A.dout[(size_t)(q0 / 16) * per + i];
}

// The pass by tiles of NG * 16 requests, as the forward one. TAB: their label
// gradients are in LDS. 64 requests over 100,000 x 768 bf16 take 43 us, near the
// bank's way from memory; 256 take 126, of which builds without the step in question
// lay 45 to loading a row again for every 64 requests (16 rows x 64 bytes an
// instruction, 22 bytes a clock and compute unit, whatever is in flight), 38 to what
// follows the scores and 20 to storing ds. (Tiles of 256 x 256 through LDS, as in the
// pass above, were no faster: nothing runs beside their longer ends.)
template <int DT, int NG, bool TAB>
__global__ __launch_bounds__(AT_WAVES * WAVE, 1) void ds_kernel(const DsArgs A)
{
    extern __shared__ __align__(16) uint8_t smem[];
    i32x4 *qs = (i32x4 *)smem;
    float *sd = (float *)(qs + (size_t)A.nks * NG * WAVE);   // [3][NG * 16] hq, lse2, shift
    float *tab = sd + 4 * NG * 16;                           // [NG][n_j][64]
    int t, ch;
    chunk_and_tile(A.n_chunks, A.n_qt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int n_waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q0 = t * NG * 16;
    const long gw = (long)ch * n_waves + wave, n_gw = (long)A.n_chunks * n_waves;
    const long s0 = A.slab0 + gw * A.slabs / n_gw, s1 = A.slab0 + (gw + 1) * A.slabs / n_gw;
    const int N = A.b.N, M = A.M;
    load_requests<DT, NG>(A.b, A.nks, q0, qs, wave, n_waves, lane);
    load_side(A, q0, NG * 16, sd);
    if constexpr (TAB)
        load_dout(A, q0, NG * 16, tab);
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
    auto column = [&](int l, int j, size_t row) {   // label 4*j + l/16 of a row, or another
        const int cc = 4 * j + (l >> 4);
        return (cc < M || cc >= 2 * M ? A.qual : A.len) + row * M +
               (cc < M ? cc : cc < 2 * M ? cc - M : 0);
    };
    auto side = [&](int slab) {
        const int l = fresh(lane);
        const long r0 = (s0 + slab) * AT_SLAB + (l & 15);
#pragma unroll
        for (int r = 0; r < AT_RT; ++r) {
            const size_t at = (size_t)min(r0 + r * 16, (long)N - 1);
            nrm[r] = A.b.norms[at];
            mk[r] = mask[at];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                vr[r][j] = *column(l, j, at);
        }
    };
    auto end = [&](int slab, f32x4(&acc)[AT_RT][NG]) {
        const int l = fresh(lane);
#pragma unroll
        for (int r = 0; r < AT_RT; ++r) {
            const long row0 = (s0 + slab) * AT_SLAB + r * 16, row = row0 + (l & 15);
            const float nh = row < N && !(masked && mk[r] == 0) ? -0.5f * nrm[r] : -INFINITY;
            const RowTile T{row0, (s0 + slab - A.slab0) * AT_RT + r,
                            (int)max(0L, min(16L, N - row0)), t, q0};
            auto lab = [&](int j) {
                return j < 4 ? (j == 0   ? vr[r][0]
                                : j == 1 ? vr[r][1]
                                : j == 2 ? vr[r][2]
                                         : vr[r][3])
                             : *column(l, j, (size_t)min(row, (long)N - 1));
            };
            const float *const douts = TAB ? tab : A.dout + (size_t)(q0 >> 4) * A.n_j * WAVE;
            ds_row_tile<DT, NG>(A, T, sd, NG * 16, douts, l, nh, acc[r], lab, sum_ds, sum_db);
        }
    };
    scan_slabs<DT, NG, AT_RT, at_ring(DT, AT_RT), true>(A.b, A.nks, qs, s0, s1, lane, [] {}, side,
                                                        end);
    // ---- the requests' sums, joined over the waves
    float *jn = (float *)smem;   // [n_waves][NG * 16][2]
    stream_barrier();
    put_sums<NG>(sum_ds, sum_db, jn + wave * NG * 32, lane);
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
    int n_row_blocks;              // of 256
    float scale;                   // 2 * beta
};

constexpr int DX_SLOTS = 4, DX_TILES = 8;   // slots of request fragments, of them in one

// d_bank of a part: 2 beta (ds^T . q - x * sum of ds). A workgroup of 8 waves
// has 256 rows x 128 columns, a wave 32 rows of all the columns; the requests'
// fragments of a block (8 KB) go through LDS, three blocks ahead, and a wave's
// fragments of ds straight into registers, two ahead. A stage is 32 MFMAs a wave
// (bf16), its LDS reads half of what the LDS gives in that time. Few requests are
// bound by the bank's way in and d_bank's out (16 over 100,000 x 768 bf16 60 us, 5.1
// TB/s); 256, at 115 us, have 31 us of MFMAs, 65 of memory and, six times, ds from
// L2. (With each row's loads waited for by themselves at the end they took 134.)
template <int DT>
__global__ __launch_bounds__(512, 1) void dx_kernel(const DxArgs A)
{
    constexpr int H = DT == AT_BF16 ? 2 : 1;   // values of ds
    constexpr int MDT = DT == AT_F32 ? 0 : 1, ESZ = DT == AT_F32 ? 4 : 2;
    constexpr int NC = DX_TILES;               // one fragment of a block to fetch a wave
    constexpr int SLOT = NC * WAVE;            // 16-byte places
    __shared__ __align__(16) i32x4 ring[DX_SLOTS * SLOT];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, jg = lane >> 4;
    // (the columns of a block of rows run on one XCD: ds comes from memory once)
    int ct, rb_;
    chunk_and_tile(A.n_row_blocks, (A.n_dt + NC - 1) / NC, &rb_, &ct);
    if (rb_ >= A.n_row_blocks)
        return;
    const long r0 = ((long)rb_ * 8 + wave) * AT_SLAB;
    const bool any = r0 < A.nrows;
    const int dt0 = ct * NC;
    const __amdgpu_buffer_rsrc_t rq =
        make_rsrc(A.qpack, (uint32_t)((size_t)A.n_blk * A.n_dt * WAVE * 16));
    const __amdgpu_buffer_rsrc_t rs =
        make_rsrc(A.ds + (any ? (r0 / 16) * A.n_blk * H * WAVE : 0),
                  any ? (uint32_t)(AT_RT * A.n_blk * H * WAVE * 16) : 0u);
    const uint32_t place = (uint32_t)ds_place(lane) * 16;
    auto fetch = [&](int blk) {   // a fragment of block blk by this wave
        dma16(rq, ring + (blk % DX_SLOTS) * SLOT + wave * WAVE,
              blk < A.n_blk && dt0 + wave < A.n_dt
                  ? (uint32_t)(((blk * A.n_dt + dt0 + wave) * WAVE + lane) * 16)
                  : OFF_NONE);
    };
    i32x4 s[2][AT_RT][H];
    auto load_ds = [&](int blk, i32x4(&to)[AT_RT][H]) {
#pragma unroll
        for (int r = 0; r < AT_RT; ++r)
#pragma unroll
            for (int h = 0; h < H; ++h)
                to[r][h] = buffer_load16(
                    rs, blk < A.n_blk
                            ? (uint32_t)(((r * A.n_blk + blk) * H + h) * WAVE * 16) + place
                            : OFF_NONE);
    };
    f32x4 acc[AT_RT][NC];
#pragma unroll
    for (int r = 0; r < AT_RT; ++r)
#pragma unroll
        for (int k = 0; k < NC; ++k)
            acc[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_sched_barrier(0);
    fetch(0);
    fetch(1);
    load_ds(0, s[0]);
    fetch(2);
    load_ds(1, s[1]);
    for (int b0 = 0; b0 < A.n_blk; b0 += 2) {
        static_for<0, 2>([&](auto U) {
            constexpr int u = decltype(U)::value;
            const int blk = b0 + u;
            __builtin_amdgcn_sched_barrier(0);
            // this wave's part of the block and its ds are there once only what
            // was sent after them is outstanding; after the barrier every wave's
            // part is, and no wave reads the slot of the block before any more
            wait_vmcnt<1 + AT_RT * H>();
            stream_barrier();
            fetch(blk + 3);
            __builtin_amdgcn_sched_barrier(0);
            const i32x4 *slot = ring + (blk % DX_SLOTS) * SLOT + lane;
            if constexpr (DT == AT_BF16) {   // (halves in their places again)
                const bool turned = col & 4;
#pragma unroll
                for (int r = 0; r < AT_RT; ++r)
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        const i32x4 x = s[u][r][h];
                        s[u][r][h] = turned ? i32x4{x[2], x[3], x[0], x[1]} : x;
                    }
            }
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const i32x4 q = slot[k * WAVE];
#pragma unroll
                for (int r = 0; r < AT_RT; ++r)
#pragma unroll
                    for (int h = 0; h < H; ++h)
                        acc[r][k] = mfma_step<MDT>(q, s[u][r][h], acc[r][k]);
            }
            __builtin_amdgcn_sched_barrier(0);
            load_ds(blk + 2, s[u]);
        });
    }
    // (all of a wave's rows are sent for before the first is used; rows and columns
    // past the end load zeros and are not stored)
    const uint32_t rowb = (uint32_t)A.d * ESZ;
    const int left = any ? (int)min((long)AT_SLAB, A.nrows - r0) : 0;
    const size_t first = (size_t)(A.row0 + (any ? r0 : 0)) * rowb;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(A.rows + first, (uint32_t)left * rowb);
    const __amdgpu_buffer_rsrc_t to = make_rsrc(A.d_bank + first, (uint32_t)left * rowb);
    auto byte = [&](int r, int k, int h) {
        const int c0 = dealt_column(dt0 + k, 4 * jg) + 4 * h;
        return c0 < A.d ? (uint32_t)(r * 16 + col) * rowb + (uint32_t)c0 * ESZ : OFF_NONE;
    };
    constexpr int HX = DT == AT_F32 ? 2 : 1;   // 16-byte pieces of eight columns
    i32x4 x[AT_RT][NC / 2][HX];
#pragma unroll
    for (int r = 0; r < AT_RT; ++r)
#pragma unroll
        for (int k = 0; k < NC; k += 2)
#pragma unroll
            for (int h = 0; h < HX; ++h)
                x[r][k / 2][h] = buffer_load16(rx, byte(r, k, h));
    float sum[AT_RT];
    bool live[AT_RT];
#pragma unroll
    for (int r = 0; r < AT_RT; ++r) {
        const long lr = min(r0 + r * 16 + col, A.nrows - 1);
        live[r] = !A.mask || A.mask[A.row0 + lr] != 0;
        sum[r] = 0.f;
        // (a lane row every fourth tile, four in flight)
#pragma unroll 4
        for (int t = jg; t < A.n_qt; t += 4)
            sum[r] += A.rowsum[(size_t)t * A.part_rows + lr];
    }
#pragma unroll
    for (int r = 0; r < AT_RT; ++r)
        sum[r] = rows_reduce(sum[r], [](float u, float v) { return u + v; });
    wait_vmcnt<0>();   // (no global-to-LDS load in flight when the workgroup ends)
    // eight columns a lane: 16 rows x 64 bytes an instruction of bf16 (four at a
    // time took 160 us for 131 at 256 x 100,000 x 768)
#pragma unroll
    for (int r = 0; r < AT_RT; ++r)
#pragma unroll
        for (int k = 0; k < NC; k += 2) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int w = x[r][k / 2][DT == AT_F32 ? e / 4 : 0][DT == AT_F32 ? e % 4 : e / 2];
                const float v = DT == AT_F32 ? __int_as_float(w)
                                : e % 2      ? bf16hi((uint32_t)w)
                                             : bf16lo((uint32_t)w);
                y[e] = live[r] ? A.scale * (acc[r][k + e / 4][e % 4] - v * sum[r]) : 0.f;
            }
            if constexpr (DT == AT_BF16) {
                bf16x8 z;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    z[e] = (__bf16)y[e];
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, z), to,
                                                       (int)byte(r, k, 0), 0, 0);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    __builtin_amdgcn_raw_buffer_store_b128(
                        __builtin_bit_cast(i32x4, f32x4{y[4 * h], y[4 * h + 1], y[4 * h + 2],
                                                        y[4 * h + 3]}),
                        to, (int)byte(r, k, h), 0, 0);
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

constexpr int DQ_COLS = 256;     // columns of a workgroup
constexpr int DQ_MASKS = 1024;   // most slabs of a share

// NI: 16-column tiles of a wave; G: groups of 16 requests of it. Its accumulators
// are 4 * NI * G, and a workgroup's eight waves have 256 columns and NI * G / 2
// groups.
template <int DT, int NI, int G> struct DqLayout {
    static constexpr int H = DT == AT_BF16 ? 2 : 1;
    static constexpr int ESZ = DT == AT_F32 ? 4 : 2;
    static constexpr int WD = 16 / NI, WQ = 8 / WD;          // waves over columns, requests
    static constexpr int REQS = WQ * G * 16;
    static constexpr int NB = REQS / (DT == AT_BF16 ? 32 : 16);   // blocks of requests
    static constexpr int ROWB = DQ_COLS * ESZ;               // bytes of a row in LDS
    static constexpr int XB = AT_SLAB * ROWB;                // of a slab's rows
    static constexpr int SB = AT_RT * NB * H * WAVE * 16;    // of its ds, [2][NB][H][64]
    static constexpr int SLOTS = XB + SB <= 32 * 1024 ? 4 : 3;
    static constexpr size_t BYTES = (size_t)SLOTS * (XB + SB) + DQ_MASKS * 4;
};

// Partial d_queries of a share of a part: sum over its rows of ds * row. A
// workgroup of 8 waves has 256 columns x 32 to 256 requests, a wave 16 * NI
// columns x 16 * G; slabs of 32 rows go through LDS, two or three ahead, and are
// read across (ds_read_b64_tr_b16: four rows of 16 columns become a column's four
// rows per lane) for the product over rows: D[column 4*(lane/16) + e][request
// lane % 16]. With many requests these reads bound it: a slab takes NI + 2 * G of 1
// KB a wave for 2 * G * NI MFMAs; with few, the rows' way from memory. (256 x 100,000 x
// 768 with NI = 4 107 us, with 8 87, and 7 more for the join of twice the shares.)
// Masked rows hold anything and are not fetched: zeros.
template <int DT, int NI, int G>
__global__ __launch_bounds__(512, 1) void dq_kernel(const DqArgs A)
{
    using L = DqLayout<DT, NI, G>;
    constexpr int H = L::H, ESZ = L::ESZ, ROWB = L::ROWB, XB = L::XB, SB = L::SB, NB = L::NB;
    constexpr int SLOTS = L::SLOTS;
    extern __shared__ __align__(16) uint8_t smem[];
    uint32_t *keep = (uint32_t *)(smem + SLOTS * (XB + SB));   // [slab of the share] a bit a row
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, jg = lane >> 4;
    const int wd = wave % L::WD, wq = wave / L::WD;   // columns, requests of this wave
    // (a share's tiles run on one XCD: its rows and its ds come from memory once)
    const int n_ct = (A.d + DQ_COLS - 1) / DQ_COLS, n_bt = (A.n_blk + NB - 1) / NB;
    int ch, t;
    chunk_and_tile(A.n_chunks, n_ct * n_bt, &ch, &t);
    if (ch >= A.n_chunks)
        return;
    const int c0 = t % n_ct * DQ_COLS, b0 = t / n_ct * NB;
    const long z0 = (long)ch * A.slabs / A.n_chunks, z1 = (long)(ch + 1) * A.slabs / A.n_chunks;
    const uint32_t rowb = (uint32_t)A.d * ESZ;

    if (A.mask) {
        for (long z = z0 + wave; z < z1; z += 8) {
            const long row = z * AT_SLAB + (lane & 31);
            const uint64_t b = ballot(row < A.nrows && A.mask[A.row0 + row] != 0);
            if (lane == 0)
                keep[z - z0] = (uint32_t)b;
        }
        __syncthreads();
    }
    f32x4 acc[NI][G];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g)
            acc[i][g] = f32x4{0.f, 0.f, 0.f, 0.f};

    // loads of 64 x 16 bytes: the rows', ds's, and how many of these a wave sends for
    // (all waves as many: of four pieces each goes out twice, to one place)
    constexpr int XL = XB / 1024, SL = SB / 1024, SW = (SL + 7) / 8;
    auto issue = [&](long z) {
        uint8_t *buf = smem + ((z - z0) % SLOTS) * (XB + SB);
        const long r0 = z * AT_SLAB;
        const bool in = z < z1;
        const int rows = in ? (int)min((long)AT_SLAB, A.nrows - r0) : 0;
        const __amdgpu_buffer_rsrc_t rx = make_rsrc(
            A.rows + (size_t)(A.row0 + (in ? r0 : 0)) * rowb, (uint32_t)rows * rowb);
        const uint32_t live = A.mask && in ? keep[z - z0] : ~0u;
#pragma unroll
        for (int j = 0; j < XL / 8; ++j) {
            const int f = wave * (XL / 8) + j;
            const int pos = f * 64 + lane;              // 16-byte places, row by row
            const int row = pos / (ROWB / 16), at = pos % (ROWB / 16);
            const int swz = DT == AT_BF16 ? (row & 7) * 2 : ((row >> 2) & 3) * 4;
            const uint32_t byte = (uint32_t)c0 * ESZ + (uint32_t)(at ^ swz) * 16;
            dma16(rx, (i32x4 *)(buf + f * 1024),
                  byte < rowb && (live >> row & 1) ? (uint32_t)row * rowb + byte : OFF_NONE);
        }
        const __amdgpu_buffer_rsrc_t rs =
            make_rsrc(A.ds + (size_t)(in ? z : 0) * AT_RT * A.n_blk * H * WAVE,
                      in ? (uint32_t)(AT_RT * A.n_blk * H * WAVE * 16) : 0u);
#pragma unroll
        for (int j = 0; j < SW; ++j) {
            const int f = (wave * SW + j) % SL;
            const int r = f / (NB * H), rest = f % (NB * H);
            const int blk = b0 + rest / H, h = rest % H;
            dma16(rs, (i32x4 *)(buf + XB + f * 1024),
                  blk < A.n_blk ? (uint32_t)((((r * A.n_blk + blk) * H + h) * WAVE + lane) * 16)
                                : OFF_NONE);
        }
    };
    constexpr int LOADS = XL / 8 + SW;
    for (int k = 0; k < SLOTS - 1; ++k)
        issue(z0 + k);
    if constexpr (DT == AT_BF16) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) s16x4 *lds4;
        auto across = [&](uint32_t at) {
            return __builtin_bit_cast(
                i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(smem + at)));
        };
        // 16 columns of the rows: four of 32 of them to a lane row, twice
        const int ti = lane & 15, xrow = 4 * jg + (ti >> 2);
        const uint32_t xat = (uint32_t)(xrow * ROWB + (ti & 1) * 8), xsw = (uint32_t)(xrow & 7) * 2;
        auto read_x = [&](uint32_t slot, int i) {
            i32x4 x;
#pragma unroll
            for (int r = 0; r < 2; ++r) {   // (16 rows on, the same turn)
                const uint32_t c16 = (uint32_t)(wd * NI * 2 + i * 2) + ((ti >> 1) & 1);
                const i32x2 w = across(slot + xat + r * 16 * ROWB + (c16 ^ xsw) * 16);
                x[2 * r] = w[0];
                x[2 * r + 1] = w[1];
            }
            return x;
        };
        // step n: value n % 2 (hi, lo) of group wq*G + n/2, which is half n/2 % 2 of
        // block wq*G/2 + n/4; the lane that wrote the four values this one reads
        const uint32_t src = (uint32_t)ds_place((ti & 3) * 16 + 4 * jg + (ti >> 2)) * 16;
        auto read_s = [&](uint32_t slot, int n) {
            i32x4 s;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const i32x2 w =
                    across(slot + XB + ((r * NB + wq * (G / 2) + n / 4) * 2 + n % 2) * 1024 + src +
                           (uint32_t)(((n / 2) ^ jg) & 1) * 8);
                s[2 * r] = w[0];
                s[2 * r + 1] = w[1];
            }
            return s;
        };
        // A slab's 2 * G steps of NI MFMAs, each step's fragment read two steps
        // ahead, the rows' as the last step lets go of those before: the barrier,
        // half way, finds fragments in registers.
        constexpr int NS = 2 * G;
        i32x4 x[NI], s[4];
        wait_vmcnt<(SLOTS - 2) * LOADS>();
        stream_barrier();
        __builtin_amdgcn_sched_barrier(0);
        uint32_t slot = 0;
#pragma unroll
        for (int i = 0; i < NI; ++i)
            x[i] = read_x(slot, i);
        s[0] = read_s(slot, 0);
        s[1] = read_s(slot, 1);
        for (long z = z0; z < z1; ++z) {
            const uint32_t next =
                slot == (uint32_t)(SLOTS - 1) * (XB + SB) ? 0u : slot + (XB + SB);
            auto step = [&](auto I) {
                constexpr int n = decltype(I)::value;
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    acc[i][n / 2] = mfma_step<1>(x[i], s[n % 4], acc[i][n / 2]);
                    if constexpr (n == NS - 1)
                        x[i] = read_x(next, i);
                }
                s[(n + 2) % 4] =
                    n < NS - 2 ? read_s(slot, n + 2) : read_s(next, n + 2 - NS);
                if constexpr (n == NS - 1)
                    static_for<0, NI>([&](auto) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    });
                else
                    __builtin_amdgcn_sched_group_barrier(0x008, NI, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            };
            __builtin_amdgcn_sched_barrier(0);
            static_for<0, NS / 2>(step);
            __builtin_amdgcn_sched_barrier(0);
            // the next slab has landed for every wave, and the one before is read
            wait_vmcnt<(SLOTS - 3) * LOADS>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            issue(z + SLOTS - 1);
            __builtin_amdgcn_sched_barrier(0);
            static_for<NS / 2, NS>(step);
            __builtin_amdgcn_sched_barrier(0);
            slot = next;
        }
    } else {
        for (long z = z0; z < z1; ++z) {
            __builtin_amdgcn_sched_barrier(0);
            // slab z has landed for every wave, and slab z - 1 is read
            wait_vmcnt<(SLOTS - 2) * LOADS>();
            stream_barrier();
            issue(z + SLOTS - 1);
            __builtin_amdgcn_sched_barrier(0);
            const uint8_t *xb = smem + ((z - z0) % SLOTS) * (XB + SB), *sb = xb + XB;
#pragma unroll
            for (int r = 0; r < AT_RT; ++r) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = r * 16 + 4 * jg + e;
                    float x[NI], s[G];
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const int el = wd * NI * 16 + i * 16 + col;
                        x[i] = *(const float *)(xb + row * ROWB + ((el >> 2) ^ (jg * 4)) * 16 +
                                                (el & 3) * 4);
                    }
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const int src = (col >> 2) * 16 + 4 * jg + e;
                        s[g] = *(const float *)(sb + (r * NB + wq * G + g) * 1024 +
                                                ds_place(src) * 16 + (col & 3) * 4);
                    }
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int g = 0; g < G; ++g)
                            acc[i][g] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], s[g], acc[i][g],
                                                                             0, 0, 0);
                }
            }
        }
    }
    wait_vmcnt<0>();
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int cc = c0 + (wd * NI + i) * 16 + 4 * jg;
            const int b = (DT == AT_BF16 ? b0 * 32 : b0 * 16) + (wq * G + g) * 16 + col;
            if (cc < A.d && b < A.B) {
                f32x4 *at = (f32x4 *)(A.part + ((size_t)ch * A.B + b) * A.d + cc);
                *at = A.first ? acc[i][g] : *at + acc[i][g];
            }
        }
}

struct JoinArgs {
    // d_queries and d_beta (null: not wanted)
    const float *part, *req;
    int n_part, n_req, B, d;
    const uint8_t *queries;
    float scale;
    uint8_t *d_queries;
    float *d_beta;
    int n_dq, n_col;             // workgroups of these, for the columns of a request
    // the label gradients of several request tiles, [n_qt][n] each
    const float *lab[2];
    float *out[2];               // null: not wanted
    int n_qt;
    size_t n;
};

// The request tiles' label gradients, added in order.
__device__ __forceinline__ void join_labels(const JoinArgs &A, int block, int blocks)
{
    for (int h = 0; h < 2; ++h) {
        if (!A.out[h])
            continue;
        for (size_t i = (size_t)block * 256 + threadIdx.x; i < A.n; i += (size_t)blocks * 256) {
            float s = 0.f;
#pragma unroll 4
            for (int t = 0; t < A.n_qt; ++t)
                s += A.lab[h][(size_t)t * A.n + i];
            A.out[h][i] = s;
        }
    }
}

// What shares and request tiles left, joined. d_queries and d_beta: the shares'
// sums, 2 beta (sum - q * sum of ds); a workgroup per request and 256 columns, a
// wave every fourth share. The label gradients: the workgroups behind them.
template <int DT>
__global__ __launch_bounds__(256) void grad_join_kernel(const JoinArgs A)
{
    __shared__ float red[2][4];
    __shared__ f32x4 sums[3][WAVE];
    if ((int)blockIdx.x >= A.n_dq) {
        join_labels(A, blockIdx.x - A.n_dq, gridDim.x - A.n_dq);
        return;
    }
    const int b = blockIdx.x / A.n_col, y = blockIdx.x % A.n_col;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c0 = y * 256 + lane * 4;
    const bool in = A.d_queries && c0 < A.d;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    if (in) {
        const float *at = A.part + (size_t)b * A.d + c0;
        const size_t step = (size_t)A.B * A.d;
#pragma unroll 8
        for (int k = wave; k < A.n_part; k += 4)
            v += *(const f32x4 *)(at + k * step);
    }
    float s0 = 0.f, s1 = 0.f;
    for (int k = tid; k < A.n_req; k += 256) {
        const float *at = A.req + ((size_t)k * A.B + b) * 2;
        s0 += at[0];
        s1 += at[1];
    }
    s0 = wave_sum(s0);
    s1 = wave_sum(s1);
    if (lane == 0) {
        red[0][wave] = s0;
        red[1][wave] = s1;
    }
    if (wave > 0)
        sums[wave - 1][lane] = v;
    __syncthreads();
    if (tid == 0 && y == 0 && A.d_beta)
        A.d_beta[b] = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    if (wave > 0 || !in)
        return;
    const float sum = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
    for (int w = 0; w < 3; ++w)
        v += sums[w][lane];
    const f32x4 q = load4<DT>(A.queries, (size_t)b * A.d + c0);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = A.scale * (v[e] - q[e] * sum);
    store4<DT>(A.d_queries, (size_t)b * A.d + c0, v);
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

hipError_t usage_gemm(const UsagePlan &p, const UsageArgs &a, hipStream_t s)
{
    const hipError_t e = allow_lds(usage_gemm_kernel, p.lds_bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(usage_gemm_kernel, dim3(p.n_chunks * p.n_qt), dim3(AT_WAVES * WAVE),
                       p.lds_bytes, s, a);
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
    const long by_size = at_least_shares((long)slabs * slab, dtype, d);
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
hipError_t run_prep(const PrepArgs &a, hipStream_t s)
{
    const int side_blocks = (a.places + 3) / 4;
    const long frags = a.qpack ? (long)a.n_blk * a.n_dt * WAVE : 0;
    hipLaunchKernelGGL(prep_kernel<QDT>, dim3((unsigned)(side_blocks + (frags + 255) / 256)),
                       dim3(256), 0, s, a, side_blocks);
    return hipGetLastError();
}

template <int DT>
hipError_t dx_one(const DxArgs &x, hipStream_t s)
{
    hipLaunchKernelGGL(dx_kernel<DT>,
                       dim3(x.n_row_blocks * ((x.n_dt + DX_TILES - 1) / DX_TILES)), dim3(512), 0,
                       s, x);
    return hipGetLastError();
}

template <int DT, int NI, int G>
hipError_t dq_one(const DqArgs &q, hipStream_t s)
{
    using L = DqLayout<DT, NI, G>;
    const hipError_t e = allow_lds(dq_kernel<DT, NI, G>, L::BYTES);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((dq_kernel<DT, NI, G>),
                       dim3(q.n_chunks * ((q.d + DQ_COLS - 1) / DQ_COLS) *
                            ((q.n_blk + L::NB - 1) / L::NB)),
                       dim3(512), L::BYTES, s, q);
    return hipGetLastError();
}

template <int DT>
hipError_t run_grad(const GradPlan &p, const AttendBank &b, const GradArgs &g, uint8_t *wb,
                    hipStream_t s)
{
    constexpr int QDT = DT == AT_F32 ? 0 : 1;
    Side *side = (Side *)(wb + p.off_side);
    float *dout = (float *)(wb + p.off_dout);
    i32x4 *qpack = (i32x4 *)(wb + p.off_qpack);
    const int n_dt = p.n_dt;
    hipError_t e = run_prep<QDT>({b.queries, b.B, b.d, g.M, p.n_j, p.n_qt * p.ng * 16, g.lse,
                                  g.q_hat, g.l_hat, g.dq_hat, g.dl_hat, g.dlse, dout, side,
                                  p.n_blk, n_dt, g.d_bank ? qpack : nullptr, b.c,
                                  b.c_exact() / b.c - 1.0},
                                 s);
    if (e != hipSuccess)
        return e;
    DsArgs a;
    a.b = b;
    a.qual = g.qual;
    a.len = g.len;
    a.M = g.M;
    a.side = side;
    a.dout = dout;
    a.n_j = p.n_j;
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
    const float scale = 2.f * b.beta;
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
            if constexpr (DT == AT_BF16)
                e = p.dq_reqs == 256   ? dq_one<DT, 8, 4>(q, s)
                    : p.dq_reqs == 128 ? dq_one<DT, 4, 4>(q, s)
                    : p.dq_reqs == 64  ? dq_one<DT, 2, 4>(q, s)
                                       : dq_one<DT, 2, 2>(q, s);
            else
                e = p.dq_reqs == 128  ? dq_one<DT, 4, 4>(q, s)
                    : p.dq_reqs == 64 ? dq_one<DT, 2, 4>(q, s)
                                      : dq_one<DT, 2, 2>(q, s);
            if (e != hipSuccess)
                return e;
        }
        if (g.d_bank) {
            DxArgs x{a.ds, qpack, a.rowsum, b.rows, b.mask, (uint8_t *)g.d_bank, p.n_blk, n_dt,
                     p.n_qt, b.d, a.part_rows, row0, nrows,
                     (int)((nrows + 8 * AT_SLAB - 1) / (8 * AT_SLAB)), scale};
            if ((e = dx_one<DT>(x, s)) != hipSuccess)
                return e;
        }
    }
    JoinArgs w{};
    w.part = dq;
    w.req = a.req;
    w.n_part = p.q_chunks;
    w.n_req = p.n_chunks;
    w.B = b.B;
    w.d = b.d;
    w.queries = b.queries;
    w.scale = scale;
    w.d_queries = (uint8_t *)g.d_queries;
    w.d_beta = g.d_beta;
    w.n_col = g.d_queries ? (b.d + 255) / 256 : 1;
    w.n_dq = g.d_queries || g.d_beta ? b.B * w.n_col : 0;
    size_t blocks = 0;
    if (p.n_qt > 1) {
        w.lab[0] = a.d_qual;
        w.lab[1] = a.d_len;
        w.out[0] = g.d_qual;
        w.out[1] = g.d_len;
        w.n_qt = p.n_qt;
        w.n = n_lab;
        if (g.d_qual || g.d_len)
            blocks = (n_lab + 255) / 256 < 8192 ? (n_lab + 255) / 256 : 8192;
    }
    if (w.n_dq + blocks == 0)
        return hipSuccess;
    hipLaunchKernelGGL(grad_join_kernel<DT>, dim3((unsigned)(w.n_dq + blocks)), dim3(256), 0, s, w);
    return hipGetLastError();
}

}  // namespace

bool plan_usage(int B, int N, int d, int dtype, int n_cu, UsagePlan *p)
{
    const int ks = at_ks(dtype);
    p->dtype = dtype;
    p->nks = (d + ks - 1) / ks;
    p->gemm = at_gemm(dtype, B, N, d, 0, n_cu);
    p->off_side = 0;
    p->off_part = p->gemm ? up256((size_t)B * sizeof(Side)) : 0;
    const size_t group = (size_t)p->nks * ks * (dtype == AT_F32 ? 4 : 2) * 16 + 16 * sizeof(Side);
    if (p->gemm) {
        p->nks = (d + AG_K - 1) / AG_K;
        p->n_qt = (B + AG_REQS - 1) / AG_REQS;
        p->n_part = (B + 63) / 64;
        p->slabs = (int)(((long)N + AG_ROWS - 1) / AG_ROWS);
        const int most = n_cu / p->n_qt;
        p->n_chunks = most < 1 ? 1 : most < p->slabs ? most : p->slabs;
        p->lds_bytes = 2 * AG_SLOT + sizeof(TileSide) + 2 * AG_REQS * 4;
        p->bytes = p->off_part + up256((size_t)p->n_part * N * 4);
        return true;
    }
    const int ng = at_groups(B, N, group, n_cu, 1, [&](int g) { return 16 * at_rt(dtype, g); });
    if (ng == 0)
        return false;
    p->ng = ng;
    const int slab = 16 * at_rt(dtype, ng);
    p->slabs = (int)(((long)N + slab - 1) / slab);
    p->n_qt = (B + ng * 16 - 1) / (ng * 16);
    shares(p->slabs, slab, dtype, d, p->n_qt, n_cu, &p->n_chunks, &p->waves);
    p->lds_bytes = group * ng;
    p->n_part = p->n_qt;
    // (256 bytes where nothing is needed: a workspace is asked for all the same)
    p->bytes = p->off_part + (p->n_qt > 1 ? up256((size_t)p->n_qt * N * 4) : 256);
    return true;
}

hipError_t launch_usage(const UsagePlan &p, const AttendBank &b, const float *lse, float decay,
                        float *usage, void *ws, hipStream_t s)
{
    Side *side = (Side *)((uint8_t *)ws + p.off_side);
    const double more = b.c_exact() / b.c - 1.0;
    hipError_t e = hipSuccess;
    if (p.gemm) {
        PrepArgs pa{};
        pa.queries = b.queries;
        pa.B = pa.places = b.B;
        pa.d = b.d;
        pa.lse = lse;
        pa.side = side;
        pa.c = b.c;
        pa.more = more;
        if ((e = run_prep<1>(pa, s)) != hipSuccess)
            return e;
    }
    UsageArgs a;
    a.b = b;
    a.lse = lse;
    a.more = more;
    a.side = side;
    a.nks = p.nks;
    a.n_chunks = p.n_chunks;
    a.n_qt = p.n_qt;
    a.slabs = p.slabs;
    a.decay = decay;
    a.usage = usage;
    a.part = p.gemm || p.n_part > 1 ? (float *)((uint8_t *)ws + p.off_part) : nullptr;
    e = p.gemm               ? usage_gemm(p, a, s)
        : p.dtype == AT_F32  ? usage_dt<AT_F32>(p, a, s)
        : p.dtype == AT_BF16 ? usage_dt<AT_BF16>(p, a, s)
                             : usage_dt<AT_Q4>(p, a, s);
    if (e != hipSuccess || !a.part)
        return e;
    hipLaunchKernelGGL(usage_join_kernel, dim3((unsigned)(((long)b.N + 255) / 256)), dim3(256), 0,
                       s, a.part, p.n_part, b.N, decay, usage);
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
    p->n_j = (2 * M + 15) / 16 * 4;
    const size_t group = (size_t)p->nks * ks * (dtype == AT_F32 ? 4 : 2) * 16 + 16 * sizeof(Side);
    const size_t tab = (size_t)p->n_j * WAVE * 4;
    // (a bf16 fragment of ds is of two groups, which one tile has to hold where
    // there are two)
    const int least = dtype == AT_BF16 && B > 16 ? 2 : 1;
    const int ng = at_groups(B, N, group, n_cu, least, [](int) { return AT_SLAB; });
    if (ng < least)
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
    // (the requests of a tile that the batch does not have cost what the others do:
    // tiles of 128 for 1 to 32 requests took 21 us for 10 over 14,919 x 384 fp32, 46
    // for 33 over 100,000 x 768 bf16, and for 64 of these 51 for 43)
    p->dq_reqs = B <= 32 ? 32 : B <= 64 ? 64 : B <= 128 || dtype == AT_F32 ? 128 : 256;
    const int dq_reqs = p->dq_reqs;
    const long tiles = (long)((d + DQ_COLS - 1) / DQ_COLS) * ((B + dq_reqs - 1) / dq_reqs);
    long qc = n_cu / tiles;
    qc = qc < 1 ? 1 : qc;
    // (a share's masks are kept in LDS)
    const long fewest = (part + DQ_MASKS - 1) / DQ_MASKS;
    qc = qc < fewest ? fewest : qc;
    p->q_chunks = (int)(qc > part ? part : qc);
    const size_t lds = (group + (p->tab ? tab : 0)) * ng;
    const size_t join = (size_t)p->waves * ng * 16 * 2 * 4;
    p->lds_bytes = lds > join ? lds : join;
    const int n_dt = (d + 31) / 32 * 2;
    p->n_dt = n_dt;
    // (32-bit offsets into the requests' fragments and into a slab's ds)
    if ((size_t)p->n_blk * (n_dt > 4 ? n_dt : 4) * WAVE * 16 >= (size_t)1 << 31)
        return false;
    size_t o = 0;
    p->off_side = o;
    o += up256((size_t)B * sizeof(Side));
    p->off_dout = o;
    o += up256((size_t)p->n_qt * ng * tab);
    p->off_qpack = o;
    o += up256((size_t)p->n_blk * n_dt * WAVE * 16);
    p->off_ds = o;
    // (a part as large as any, so that the size grows with B: a slab has at least
    // 2048 bytes of ds for 16 requests, and 128 of sums for a request tile)
    const size_t n16 = ((size_t)B + 15) / 16, all = (size_t)p->slabs;
    const size_t room = PART_BYTES > slab_ds ? PART_BYTES : slab_ds;
    o += up256(all * slab_ds < room ? all * slab_ds : room);
    p->off_rowsum = o;
    o += up256(all * n16 * 128 < room / 16 ? all * n16 * 128 : room / 16);
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
