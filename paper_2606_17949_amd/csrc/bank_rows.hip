// Rows of the labelled bank: written in place (in their own type, or held in 4
// bits), and chosen to make room.
#include "attend_scan.hpp"

namespace rb {

namespace {

// Code of |y| <= 6 among 0, 0.5, 1, 1.5, 2, 3, 4, 6: the nearest, of two as
// near the even code.
__device__ __forceinline__ uint32_t code4(float y)
{
    const float a = fabsf(y);
    const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) +
                       (a >= 3.5f) + (a > 5.f);
    return c | (__float_as_uint(y) >> 31 << 3);
}

// One wave per row. A row of the bank's own type is copied 16 bytes a lane and
// its norm summed as rb_bank_norms sums it. A row held in 4 bits goes by 512
// elements at a time, 8 a lane: four lanes find their 32 elements' largest
// magnitude, its scale is the least power of two (2^-126 at least) under which
// it is at most 6, and the norm is that of the values held.
template <int SDT, int DT>
__global__ __launch_bounds__(256) void write_rows_kernel(const RowsArgs A)
{
    constexpr int ESZ = Elem<SDT>::ESZ;
    const int lane = threadIdx.x & 63;
    const long n_waves = (long)gridDim.x * 4;
    for (long j = (long)blockIdx.x * 4 + (threadIdx.x >> 6); j < A.n; j += n_waves) {
        const long row = A.at ? A.at[j] : j;
        if (row < 0 || row >= A.N)
            continue;
        const uint8_t *src = A.src + (size_t)j * A.d * ESZ;
        float s = 0.f;
        if constexpr (DT == AT_Q4) {
            uint8_t *const out = A.rows + (size_t)row * (A.d / 2);
            uint8_t *const sc = A.scales + (size_t)row * (A.d / 32);
            for (int at = lane * 8; at - lane * 8 < A.d; at += 512) {
                const bool in = at < A.d;
                float x[8];
                if constexpr (SDT == 1) {
                    const i32x4 w = in ? load16(src + (size_t)at * 2) : i32x4{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[2 * e] = bf16lo((uint32_t)w[e]);
                        x[2 * e + 1] = bf16hi((uint32_t)w[e]);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const i32x4 w =
                            in ? load16(src + (size_t)at * 4 + h * 16) : i32x4{0, 0, 0, 0};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[4 * h + e] = __int_as_float(w[e]);
                    }
                }
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    top = fmaxf(top, fabsf(x[e]));
                top = fmaxf(top, dpp<0xb1>(top));   // quad_perm [1,0,3,2]
                top = fmaxf(top, dpp<0x4e>(top));   // quad_perm [2,3,0,1]
                // top = 1.m * 2^k is at most 6 * 2^e for e = k - 2 if 1.m <= 1.5
                const uint32_t bits = __float_as_uint(top);
                int e8 = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x400000u);
                e8 = max(e8, 1);
                const float up = __uint_as_float((uint32_t)(254 - e8) << 23);
                const float scale = __uint_as_float((uint32_t)e8 << 23);
                uint32_t codes = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    codes |= code4(x[e] * up) << (4 * e);
                const i32x4 v = widen4(codes, scale);
                s = sumsq16<1>(v, s);
                if (in) {
                    *(uint32_t *)(out + at / 2) = codes;
                    if ((lane & 3) == 0)
                        sc[at / 32] = (uint8_t)e8;
                }
            }
        } else {
            uint8_t *const out = A.rows + (size_t)row * A.d * ESZ;
            const int row_bytes = A.d * ESZ;
            for (int off = lane * 16; off < row_bytes; off += WAVE * 16) {
                const i32x4 v = load16(src + off);
                *(i32x4 *)(out + off) = v;
                s = sumsq16<SDT>(v, s);
            }
        }
        s = wave_sum(s);
        if (lane == 0) {
            A.norms[row] = s;
            if (A.usage)
                A.usage[row] = A.usage0;
        }
        if (A.qual)
            for (int m = lane; m < A.M; m += WAVE) {
                A.qual[(size_t)row * A.M + m] = A.new_qual[(size_t)j * A.M + m];
                A.len[(size_t)row * A.M + m] = A.new_len[(size_t)j * A.M + m];
            }
    }
}

// ---- the n least of N, by three histograms of the ordered bits of the keys
// (11, 11 and 10 of them), which leave the n-th least key T and how many of
// those equal to it are taken; then every block writes its rows below T, and its
// share of those at T, behind those of the blocks before it. What bounds it is
// latency: four passes over 4 bytes a row, each a launch. Usage falls into few of
// the first histogram's bins (of one exponent and two bits of mantissa), so
// blocks add to one of EV_COPIES histograms, and the n-th key's bin is found by
// every block of the next pass for itself (found by the last block of a pass to
// arrive, with a counter and fences between, a pass over 4,000,000 rows took 42
// us). With few blocks each has a first histogram of its own, which nothing has to
// clear before (64 of 40,000 rows 20.4 us for 22.9, of 130,000 23.1 for 23.4; 61
// blocks with one each 28.4 for 22.6); the first pass clears the other two. The
// third leaves, block by block, how many rows come before each of its bins: the
// last pass needs no pass before it that counts them (with one, 10 of 10,000 took
// 22.0 us for 19.1, 50,000 of 4,000,000 35.5 for 34.0).
constexpr int EV_BINS = 2048, EV_THREADS = 1024, EV_COPIES = 8;
constexpr int EV_TILE = EV_THREADS * 4;   // rows a block takes at a time, four a thread
constexpr int EV_BLOCKS = 256;            // most blocks
constexpr int EV_OWN = 32;                // most blocks with a first histogram each
constexpr int EV_LAST = 1024, EV_CUM = EV_LAST + 1;   // bins of the last histogram

// Workspace in 32-bit words: the states, the histograms of the second and third
// pass, those of the first (one each or EV_COPIES), [blocks][EV_CUM] rows before
// the third's bins.
constexpr int EV_HIST = EV_COPIES * EV_BINS;
constexpr int EV_AT_HIST = 64, EV_AT_FIRST = EV_AT_HIST + 2 * EV_HIST;
constexpr int EV_AT_CUM = EV_AT_FIRST + EV_OWN * EV_BINS;
static_assert(EV_OWN >= EV_COPIES, "room of the first histograms");

// Where the search stands behind each histogram: the bits of T found so far,
// the rows to take among those with these bits, and whether there are fewer
// rows than asked for and all are taken.
struct EvictState {
    uint32_t prefix, remain, all, none;
};

// Ordered bits of a usage: -0 is 0, and every NaN, of either sign, the greatest key
// (f2key orders numbers only: a NaN with the sign bit set comes below -inf there).
__device__ __forceinline__ uint32_t usage_key(float u)
{
    return u != u ? KEY_NONE : f2key(u + 0.f);
}

// Rows i .. i+3: their keys, and which of them may go (none past the end).
struct Four {
    uint32_t key[4];
    bool in[4];
};

__device__ __forceinline__ Four load_four(const float *usage, const uint8_t *may_go, long i, int N)
{
    typedef uint32_t u32_any __attribute__((aligned(1)));
    Four f;
    if (i + 4 <= N) {
        const f32x4 u = *(const f32x4_any *)(usage + i);
        const uint32_t go = may_go ? *(const u32_any *)(may_go + i) : ~0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f.key[e] = usage_key(u[e]);
            f.in[e] = (go >> (8 * e) & 0xffu) != 0;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool at = i + e < N;
            f.key[e] = at ? usage_key(usage[i + e]) : 0u;
            f.in[e] = at && (!may_go || may_go[i + e] != 0);
        }
    }
    return f;
}

__global__ __launch_bounds__(EV_THREADS) void evict_clear_kernel(uint32_t *ws)
{
    ws[EV_AT_FIRST + blockIdx.x * EV_THREADS + threadIdx.x] = 0;
}

constexpr int ev_bits(int level) { return level == 2 ? 10 : 11; }
constexpr int ev_shift(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }

// The state behind histogram L, from the one before it (L 0: n rows to take).
// Every thread of the block gets it.
template <int L>
__device__ __forceinline__ EvictState evict_pick(const uint32_t *ws, EvictState st)
{
    constexpr int PER = EV_BINS / EV_THREADS, NW = EV_THREADS / WAVE;
    static_assert(PER == 2, "the loads below");
    __shared__ uint32_t sums[NW];
    __shared__ EvictState found;
    if (L > 0 && st.all)
        return st;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 *hist =
        (const u32x2 *)(ws + (L == 0 ? EV_AT_FIRST : EV_AT_HIST + (L - 1) * EV_HIST));
    u32x2 own = u32x2{0, 0};
    const int copies = L == 0 && gridDim.x <= EV_OWN ? gridDim.x : EV_COPIES;
#pragma unroll 8
    for (int k = 0; k < copies; ++k)
        own += hist[k * (EV_BINS / 2) + tid];
    // rows in the bins of the threads before
    const uint32_t total = own[0] + own[1];
    uint32_t upto = total;
    for (int k = 1; k < WAVE; k <<= 1) {
        const uint32_t x = (uint32_t)__shfl_up((int)upto, k);
        upto += lane >= k ? x : 0;
    }
    __syncthreads();   // (of an earlier call: read)
    if (lane == WAVE - 1)
        sums[wave] = upto;
    __syncthreads();
    uint32_t before = upto - total, rows_in = 0;
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? sums[w] : 0;
        rows_in += sums[w];
    }
    if (rows_in < st.remain)   // (the first histogram only)
        return EvictState{0, 0, 1, 0};
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (before < st.remain && st.remain <= before + own[j])
            found = EvictState{(st.prefix << ev_bits(L)) | (uint32_t)(tid * PER + j),
                               st.remain - before, 0, 0};
        before += own[j];
    }
    __syncthreads();
    return found;
}

// Histogram L, of the keys that share the bits found so far. states[L - 1] is
// found and left for the passes behind the next one.
template <int L>
__global__ __launch_bounds__(EV_THREADS) void evict_hist_kernel(const float *usage,
                                                                const uint8_t *may_go, int N, int n,
                                                                int rows, uint32_t *ws)
{
    constexpr int SHIFT = ev_shift(L), BITS = ev_bits(L);
    constexpr uint32_t MASK = (1u << BITS) - 1;
    __shared__ uint32_t bins[EV_BINS], sums[EV_THREADS / WAVE], under;
    EvictState *const states = (EvictState *)ws;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < EV_BINS; i += EV_THREADS)
        bins[i] = 0;
    if (tid == 0)
        under = 0;
    if constexpr (L == 0)
        for (int i = blockIdx.x * EV_THREADS + tid; i < 2 * EV_HIST; i += gridDim.x * EV_THREADS)
            ws[EV_AT_HIST + i] = 0;
    EvictState st{0, (uint32_t)n, 0, 0};
    if constexpr (L > 0) {
        if constexpr (L > 1)
            st = states[L - 2];
        st = evict_pick<L - 1>(ws, st);
        if (blockIdx.x == 0 && tid == 0)
            states[L - 1] = st;
        if (L < 2 && st.all)
            return;
    }
    __syncthreads();
    const long r0 = (long)blockIdx.x * rows;
    uint32_t less = 0;   // the last histogram's: rows below all of its bins
#pragma unroll 4
    for (int z = 0; z < rows; z += EV_TILE) {
        const Four f = load_four(usage, may_go, r0 + z + tid * 4, N);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t high = L == 0 ? 0 : f.key[e] >> (SHIFT + BITS);
            less += L == 2 && f.in[e] && (st.all || high < st.prefix);
            if (f.in[e] && (L == 0 || (high == st.prefix && !st.all)))
                atomicAdd(&bins[(f.key[e] >> SHIFT) & MASK], 1u);
        }
    }
    if constexpr (L == 2) {
        less = wave_reduce(less, [](uint32_t x, uint32_t y) { return x + y; });
        if (lane == 0 && less)
            atomicAdd(&under, less);
    }
    __syncthreads();
    if (L == 0 && gridDim.x <= EV_OWN) {
        for (int i = tid; i < EV_BINS; i += EV_THREADS)
            ws[EV_AT_FIRST + blockIdx.x * EV_BINS + i] = bins[i];
        return;
    }
    uint32_t *mine = ws + (L == 0 ? EV_AT_FIRST : EV_AT_HIST + (L - 1) * EV_HIST) +
                     blockIdx.x % EV_COPIES * EV_BINS;
    for (int i = tid; i < EV_BINS; i += EV_THREADS)
        if (bins[i])
            atomicAdd(&mine[i], bins[i]);
    if constexpr (L == 2) {
        static_assert(EV_LAST == EV_THREADS && MASK + 1 == EV_LAST, "a bin a thread");
        uint32_t upto = bins[tid];
        for (int k = 1; k < WAVE; k <<= 1) {
            const uint32_t x = (uint32_t)__shfl_up((int)upto, k);
            upto += lane >= k ? x : 0;
        }
        if (lane == WAVE - 1)
            sums[wave] = upto;
        __syncthreads();
        upto += under;
        for (int w = 0; w < wave; ++w)
            upto += sums[w];
        uint32_t *cum = ws + EV_AT_CUM + (size_t)blockIdx.x * EV_CUM;
        cum[tid + 1] = upto;
        if (tid == 0)
            cum[0] = under;
    }
}

// A block's rows below T and at T.
__device__ __forceinline__ void below_and_at(const Four &f, uint32_t T, bool all, bool (&lt)[4],
                                             bool (&eq)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lt[e] = f.in[e] && (all || f.key[e] < T);
        eq[e] = f.in[e] && !all && f.key[e] == T;
    }
}

// Both sums over the block, for every thread.
__device__ __forceinline__ void block_sums(uint32_t &x, uint32_t &y,
                                           uint32_t (&red)[2][EV_THREADS / WAVE])
{
    auto add = [](uint32_t a, uint32_t b) { return a + b; };
    x = wave_reduce(x, add);
    y = wave_reduce(y, add);
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        red[0][wave] = x;
        red[1][wave] = y;
    }
    __syncthreads();
    x = y = 0;
    for (int w = 0; w < EV_THREADS / WAVE; ++w) {
        x += red[0][w];
        y += red[1][w];
    }
}

__global__ __launch_bounds__(EV_THREADS) void evict_write_kernel(const float *usage,
                                                                 const uint8_t *may_go, int N,
                                                                 int rows, int n,
                                                                 const uint32_t *ws,
                                                                 int32_t *victims)
{
    constexpr int NW = EV_THREADS / WAVE;
    __shared__ uint32_t red[2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EvictState st = evict_pick<2>(ws, ((const EvictState *)ws)[1]);
    const uint32_t T = st.prefix;
    const bool all = st.all != 0;
    const uint32_t remain = all ? 0u : st.remain;
    // rows below T and at T, of a block
    auto counts = [&](int k, uint32_t &b, uint32_t &a) {
        const uint32_t *cum = ws + EV_AT_CUM + (size_t)k * EV_CUM + (all ? 0 : T & (EV_LAST - 1));
        b = cum[0];
        a = all ? 0u : cum[1] - cum[0];
    };
    uint32_t below = 0, at = 0, own_below, own_at;
    if (tid < (int)blockIdx.x)
        counts(tid, below, at);   // (of the blocks before)
    counts(blockIdx.x, own_below, own_at);
    block_sums(below, at, red);
    const bool none = own_below == 0 && (own_at == 0 || at >= remain);
    const long r0 = (long)blockIdx.x * rows;
    if (!none) {
        const uint64_t under = (1ull << lane) - 1;
        for (int z = 0; z < rows; z += EV_TILE) {
            const long i = r0 + z + tid * 4;
            const Four f = load_four(usage, may_go, i, N);
            bool lt[4], eq[4];
            below_and_at(f, T, all, lt, eq);
            // of the wave, and of its lanes before this one
            uint32_t wl = 0, we = 0, pl = 0, pe = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t bl = ballot(lt[e]), be = ballot(eq[e]);
                wl += __popcll(bl);
                we += __popcll(be);
                pl += __popcll(bl & under);
                pe += __popcll(be & under);
            }
            __syncthreads();
            if (lane == 0) {
                red[0][wave] = wl;
                red[1][wave] = we;
            }
            __syncthreads();
            pl += below;
            pe += at;
            for (int w = 0; w < NW; ++w) {
                if (w < wave) {
                    pl += red[0][w];
                    pe += red[1][w];
                }
                below += red[0][w];
                at += red[1][w];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (lt[e] || (eq[e] && pe < remain)) {
                    const uint32_t pos = pl + min(pe, remain);
                    if (pos < (uint32_t)n)
                        victims[pos] = (int32_t)(i + e);
                }
                pl += lt[e];
                pe += eq[e];
            }
        }
    }
    // fewer rows than asked for: no row behind them
    if (all && blockIdx.x == gridDim.x - 1) {
        for (long k = (long)below + tid; k < n; k += EV_THREADS)
            victims[k] = -1;
    }
}

// Rows of a block: whole tiles, at most EV_BLOCKS blocks.
int evict_rows(int N)
{
    const long per = ((long)N + EV_BLOCKS - 1) / EV_BLOCKS;
    return (int)((per + EV_TILE - 1) / EV_TILE * EV_TILE);   // (under 2^24)
}

template <int SDT>
hipError_t write_rows(int dtype, const RowsArgs &a, int grid, hipStream_t s)
{
    if (dtype == AT_Q4)
        hipLaunchKernelGGL((write_rows_kernel<SDT, AT_Q4>), dim3(grid), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((write_rows_kernel<SDT, SDT>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_write_rows(int src_dtype, int dtype, const RowsArgs &a, hipStream_t s)
{
    long grid = ((long)a.n + 3) / 4;
    if (grid > 65536)
        grid = 65536;
    return src_dtype == AT_F32 ? write_rows<0>(dtype, a, (int)grid, s)
                               : write_rows<1>(dtype, a, (int)grid, s);
}

size_t evict_bytes(int N)
{
    const int rows = evict_rows(N);
    return ((size_t)EV_AT_CUM + ((size_t)N + rows - 1) / rows * EV_CUM) * 4;
}

hipError_t launch_evict(const float *usage, const uint8_t *may_go, int N, int n, int32_t *victims,
                        void *ws_, hipStream_t s)
{
    uint32_t *ws = (uint32_t *)ws_;
    const int rows = evict_rows(N);
    const int blocks = (int)(((long)N + rows - 1) / rows);
    const dim3 grid((unsigned)blocks), block(EV_THREADS);
    static_assert(EV_BLOCKS <= EV_THREADS, "a thread for each block before");
    static_assert(EV_HIST % EV_THREADS == 0, "the clearing grid");
    if (blocks > EV_OWN)
        hipLaunchKernelGGL(evict_clear_kernel, dim3(EV_HIST / EV_THREADS), block, 0, s, ws);
    hipLaunchKernelGGL(evict_hist_kernel<0>, grid, block, 0, s, usage, may_go, N, n, rows, ws);
    hipLaunchKernelGGL(evict_hist_kernel<1>, grid, block, 0, s, usage, may_go, N, n, rows, ws);
    hipLaunchKernelGGL(evict_hist_kernel<2>, grid, block, 0, s, usage, may_go, N, n, rows, ws);
    hipLaunchKernelGGL(evict_write_kernel, grid, block, 0, s, usage, may_go, N, rows, n, ws,
                       victims);
    return hipGetLastError();
}

}  // namespace rb
