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
// those equal to it are taken; then every block counts its rows below T and at
// T, and writes its own behind those of the blocks before it.
constexpr int EV_BINS = 2048, EV_THREADS = 256, EV_ROWS = 8192;

struct EvictState {
    uint32_t ticket[3];
    uint32_t prefix;   // the bits of T found so far
    uint32_t remain;   // rows to take among those with these bits
    uint32_t all;      // fewer rows than asked for: every one is taken
};

__device__ __forceinline__ uint32_t usage_key(float u) { return f2key(u + 0.f); }   // -0 is 0

__global__ __launch_bounds__(EV_THREADS) void evict_clear_kernel(uint32_t *hist, EvictState *st,
                                                                 uint32_t n)
{
    const int i = blockIdx.x * EV_THREADS + threadIdx.x;
    if (i < 3 * EV_BINS)
        hist[i] = 0;
    if (i == 0) {
        st->ticket[0] = st->ticket[1] = st->ticket[2] = 0;
        st->prefix = 0;
        st->remain = n;
        st->all = 0;
    }
}

template <int L>
__global__ __launch_bounds__(EV_THREADS) void evict_hist_kernel(const float *usage,
                                                                const uint8_t *may_go, int N,
                                                                uint32_t *hist_all, EvictState *st)
{
    constexpr int SHIFT = L == 0 ? 21 : L == 1 ? 10 : 0;
    constexpr int BITS = L == 2 ? 10 : 11;
    constexpr uint32_t MASK = (1u << BITS) - 1;
    __shared__ uint32_t bins[EV_BINS];
    __shared__ uint32_t sums[EV_THREADS];
    __shared__ bool last;
    const int tid = threadIdx.x;
    uint32_t *hist = hist_all + L * EV_BINS;
    if (L > 0 && st->all)
        return;
    for (int i = tid; i < EV_BINS; i += EV_THREADS)
        bins[i] = 0;
    __syncthreads();
    const uint32_t prefix = L > 0 ? st->prefix : 0;
    for (long i = (long)blockIdx.x * EV_THREADS + tid; i < N; i += (long)gridDim.x * EV_THREADS) {
        const uint32_t key = usage_key(usage[i]);
        const bool in = (!may_go || may_go[i] != 0) &&
                        (L == 0 || (key >> (SHIFT + BITS)) == prefix);
        if (in)
            atomicAdd(&bins[(key >> SHIFT) & MASK], 1u);
    }
    __syncthreads();
    for (int i = tid; i < EV_BINS; i += EV_THREADS)
        if (bins[i])
            atomicAdd(&hist[i], bins[i]);
    // the last block to get here finds the bin
    __threadfence();
    __syncthreads();
    if (tid == 0)
        last = atomicAdd(&st->ticket[L], 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last)
        return;
    __threadfence();
    constexpr int PER = EV_BINS / EV_THREADS;
    uint32_t own[PER], total = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        own[j] = __hip_atomic_load(&hist[tid * PER + j], __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        total += own[j];
    }
    sums[tid] = total;
    __syncthreads();
    for (int k = 1; k < EV_THREADS; k <<= 1) {
        const uint32_t x = tid >= k ? sums[tid - k] : 0;
        __syncthreads();
        sums[tid] += x;
        __syncthreads();
    }
    const uint32_t remain = st->remain;
    uint32_t before = sums[tid] - total;
    __syncthreads();
    if (L == 0 && sums[EV_THREADS - 1] < remain) {
        if (tid == 0)
            st->all = 1;
        return;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (before < remain && remain <= before + own[j]) {
            st->prefix = (prefix << BITS) | (uint32_t)(tid * PER + j);
            st->remain = remain - before;
        }
        before += own[j];
    }
}

__global__ __launch_bounds__(EV_THREADS) void evict_count_kernel(const float *usage,
                                                                 const uint8_t *may_go, int N,
                                                                 const EvictState *st,
                                                                 uint32_t *counts)
{
    __shared__ uint32_t red[2][EV_THREADS / WAVE];
    const uint32_t T = st->prefix;
    const bool all = st->all != 0;
    uint32_t below = 0, at = 0;
    const long r0 = (long)blockIdx.x * EV_ROWS;
    for (long i = r0 + threadIdx.x; i < min(r0 + EV_ROWS, (long)N); i += EV_THREADS) {
        const uint32_t key = usage_key(usage[i]);
        const bool in = !may_go || may_go[i] != 0;
        below += in && (all || key < T);
        at += in && !all && key == T;
    }
    auto add = [](uint32_t x, uint32_t y) { return x + y; };
    below = wave_reduce(below, add);
    at = wave_reduce(at, add);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        red[0][wave] = below;
        red[1][wave] = at;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        uint32_t s = 0;
        for (int w = 0; w < EV_THREADS / WAVE; ++w)
            s += red[threadIdx.x][w];
        counts[blockIdx.x * 2 + threadIdx.x] = s;
    }
}

__global__ __launch_bounds__(EV_THREADS) void evict_write_kernel(const float *usage,
                                                                 const uint8_t *may_go, int N,
                                                                 int n, const EvictState *st,
                                                                 const uint32_t *counts,
                                                                 int32_t *victims)
{
    constexpr int NW = EV_THREADS / WAVE;
    __shared__ uint32_t red[2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t T = st->prefix, remain = st->remain;
    const bool all = st->all != 0;
    auto add = [](uint32_t x, uint32_t y) { return x + y; };
    // rows below T and at T in the blocks before
    uint32_t below = 0, at = 0;
    for (int k = tid; k < (int)blockIdx.x; k += EV_THREADS) {
        below += counts[2 * k];
        at += counts[2 * k + 1];
    }
    below = wave_reduce(below, add);
    at = wave_reduce(at, add);
    if (lane == 0) {
        red[0][wave] = below;
        red[1][wave] = at;
    }
    __syncthreads();
    below = at = 0;
    for (int w = 0; w < NW; ++w) {
        below += red[0][w];
        at += red[1][w];
    }
    __syncthreads();
    const long r0 = (long)blockIdx.x * EV_ROWS;
    for (long i0 = r0; i0 < min(r0 + EV_ROWS, (long)N); i0 += EV_THREADS) {
        const long i = i0 + tid;
        const bool in = i < N && (!may_go || may_go[i] != 0);
        const uint32_t key = in ? usage_key(usage[i]) : 0;
        const bool lt = in && (all || key < T), eq = in && !all && key == T;
        const uint64_t bl = ballot(lt), be = ballot(eq), under = (1ull << lane) - 1;
        if (lane == 0) {
            red[0][wave] = __popcll(bl);
            red[1][wave] = __popcll(be);
        }
        __syncthreads();
        uint32_t l0 = below, e0 = at;
        for (int w = 0; w < NW; ++w) {
            if (w < wave) {
                l0 += red[0][w];
                e0 += red[1][w];
            }
            below += red[0][w];
            at += red[1][w];
        }
        l0 += __popcll(bl & under);
        e0 += __popcll(be & under);
        if (lt || (eq && e0 < remain)) {
            const uint32_t pos = l0 + min(e0, all ? 0u : remain);
            if (pos < (uint32_t)n)
                victims[pos] = (int32_t)i;
        }
        __syncthreads();
    }
    // fewer rows than asked for: no row behind them
    if (all && blockIdx.x == gridDim.x - 1)
        for (long k = (long)below + tid; k < n; k += EV_THREADS)
            victims[k] = -1;
}

int evict_blocks(int N) { return (int)(((long)N + EV_ROWS - 1) / EV_ROWS); }

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
    const size_t b = 256 + 3 * EV_BINS * 4 + (size_t)evict_blocks(N) * 8;
    return (b + 255) & ~(size_t)255;
}

hipError_t launch_evict(const float *usage, const uint8_t *may_go, int N, int n, int32_t *victims,
                        void *ws, hipStream_t s)
{
    EvictState *st = (EvictState *)ws;
    uint32_t *hist = (uint32_t *)((uint8_t *)ws + 256);
    uint32_t *counts = hist + 3 * EV_BINS;
    const int blocks = evict_blocks(N), wide = blocks < 512 ? blocks : 512;
    hipLaunchKernelGGL(evict_clear_kernel, dim3((3 * EV_BINS + EV_THREADS - 1) / EV_THREADS),
                       dim3(EV_THREADS), 0, s, hist, st, (uint32_t)n);
    hipLaunchKernelGGL(evict_hist_kernel<0>, dim3(wide), dim3(EV_THREADS), 0, s, usage, may_go, N,
                       hist, st);
    hipLaunchKernelGGL(evict_hist_kernel<1>, dim3(wide), dim3(EV_THREADS), 0, s, usage, may_go, N,
                       hist, st);
    hipLaunchKernelGGL(evict_hist_kernel<2>, dim3(wide), dim3(EV_THREADS), 0, s, usage, may_go, N,
                       hist, st);
    hipLaunchKernelGGL(evict_count_kernel, dim3(blocks), dim3(EV_THREADS), 0, s, usage, may_go, N,
                       st, counts);
    hipLaunchKernelGGL(evict_write_kernel, dim3(blocks), dim3(EV_THREADS), 0, s, usage, may_go, N,
                       n, st, counts, victims);
    return hipGetLastError();
}

}  // namespace rb
