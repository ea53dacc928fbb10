// Attention of requests over the labelled bank: argument blocks, host plan and
// launchers (attend.hip the forward pass, attend_grad.hip the passes that
// recompute its probabilities, bank_rows.hip the rows of the bank themselves).
//
// Request b weighs bank row n by p[b][n] = exp(-beta*|q_b - x_n|^2) / Z_b, Z_b
// the sum over the rows whose mask is not 0. All kernels work with
//   a[b][n] = <q, x> - |q|^2/2 - |x|^2/2 = -|q - x|^2/2,
// the accumulators of a matrix product that starts from the norms, and with
// powers of two: p = 2^(c*a - lse*log2(e)), c = 2*beta*log2(e).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rb {

constexpr int AT_F32 = 0, AT_BF16 = 1, AT_Q4 = 2;   // rb_dtype of a bank
constexpr int AT_WAVES = 8;                         // most waves of a workgroup
constexpr int AT_LDS = 160 * 1024;                  // bytes of LDS of a compute unit

struct AttendBank {
    const uint8_t *queries, *rows, *scales;   // scales: 4-bit banks only
    const float *norms;
    const uint8_t *mask;                      // [N] or null
    int B, N, d;
    float beta, c;                            // c: 2 * beta * log2(e), rounded
    double c_exact() const { return 2.0 * (double)beta * 1.4426950408889634; }
};

struct AttendPlan {
    bool gemm;             // as a matrix product of tiles
    int dtype, ng;         // request tile: ng groups of 16
    int n_qt, n_chunks;    // request tiles, shares of the bank
    int waves, nks;        // waves of a workgroup, k-steps of a row
    int n_lt;              // tiles of label columns
    int ct;                //   of ct * 16 columns each
    int slabs;             // pieces of the bank: slabs, or tiles of 256 rows
    size_t lds_bytes;
    size_t off_ml, off_o, bytes;   // workspace: partial maxima and sums, partial averages
};

// Whether a batch goes by as a matrix product of tiles (attend_gemm.hpp) of 256
// rows and 256 requests: more than half a tile of bf16 requests, for which the
// scan by tiles of 64 would read the bank three times or more, and tiles for half
// the compute units. Forward, scan / tiles: 256 x 100,000 x 768 97 / 67 us, 512 x
// 100,000 x 384 95 / 83, but 128 x 100,000 x 768 59 / 67 and 150 x 15,000 x 768 30 /
// 40.
// With labels of M models (0: none are averaged) each product of tiles takes 16 of
// the 2 M label columns, each scan 32: not where that makes twice as many products,
// unless LDS holds fewer than 64 requests of a scan. 256 x 100,000 x 768, M = 8 90 /
// 65, 9 107 / 115, 16 102 / 115, 17 180 / 146, 32 176 / 191; 256 x 1,000,000 x 768, M = 8
// 829 / 507, 9 924 / 887, 16 887 / 891, 32 1,584 / 1,701; 300 x 200,000 x 2,048, M = 16
// 938 / 717, 32 1,896 / 1,348.
inline bool at_gemm(int dtype, int B, int N, int d, int M, int n_cu)
{
    const long tiles = ((long)N + 255) / 256 * ((B + 255) / 256);
    const bool held = (size_t)((d + 31) / 32) * 64 * 64 <= (size_t)AT_LDS;
    const int products = (2 * M + 15) / 16, scans = (2 * M + 31) / 32;
    return dtype == AT_BF16 && d >= 128 && B > 128 && 2 * tiles >= n_cu &&
           (products < 2 * scans || !held || M == 0);
}

// Groups of 16 requests of a scan's tile: four where LDS holds them, fewer for a
// smaller batch, and fewer for a small bank, so that two waves a compute unit
// have something to do (64 x 1,000 x 768: 31 us by one tile of 64, 19 by four of
// 16), but at least `least`. `group`: bytes of LDS of 16 requests; slab(ng): rows
// of a slab. 0: none fits.
template <typename Slab>
int at_groups(int B, int N, size_t group, int n_cu, int least, Slab slab)
{
    int ng = B <= 16 ? 1 : B <= 32 ? 2 : 4;
    while (ng > 1 && group * ng > (size_t)AT_LDS)
        ng /= 2;
    if (group * ng > (size_t)AT_LDS)
        return 0;
    while (ng > least && ((long)N + slab(ng) - 1) / slab(ng) * ((B + 16L * ng - 1) / (16 * ng)) <
                         2L * n_cu)
        ng /= 2;
    return ng;
}

// The forward pass on a device of n_cu compute units; false if no layout fits.
bool plan_attend(int B, int N, int d, int dtype, int M, int n_cu, AttendPlan *p);

hipError_t launch_attend(const AttendPlan &p, const AttendBank &a, const float *qual,
                         const float *len, int M, float *q_hat, float *l_hat, float *lse, void *ws,
                         hipStream_t s);

// The accumulated weight of the bank's rows: usage = decay * usage + sum over
// the batch of p.
struct UsagePlan {
    bool gemm;            // as a matrix product of tiles
    int dtype, ng, n_qt, n_chunks, waves, nks, slabs;
    int n_part;           // partial sums of a row
    size_t lds_bytes;
    size_t off_side, off_part, bytes;   // per request; partial sums per request tile
};

bool plan_usage(int B, int N, int d, int dtype, int n_cu, UsagePlan *p);

hipError_t launch_usage(const UsagePlan &p, const AttendBank &a, const float *lse, float decay,
                        float *usage, void *ws, hipStream_t s);

// usage *= decay, and zeros, for batches of no requests.
hipError_t launch_decay(float *usage, int N, float decay, hipStream_t s);
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s);   // bytes a multiple of 4

// The gradients. The bank goes by in parts, each in three passes: the scores'
// gradient ds (and what needs no further product), then d_queries += ds * rows,
// then d_bank = ds^T * queries.
struct GradPlan {
    int dtype, ng, n_qt, n_chunks, waves, nks, slabs;
    bool tab;             // the label gradients of a request tile fit LDS
    int n_blk;            // blocks of requests of one fragment of ds (32, fp32 16)
    int n_dt;             // fragments of 16 columns of a block of requests
    int n_j;              // pieces of 4 label columns, a multiple of four
    int part_slabs;       // slabs of a part
    int q_chunks;         // shares of a part in the d_queries pass
    int dq_reqs;          // requests of its tiles: 32, 64, 128 or 256
    size_t lds_bytes;
    size_t off_side, off_dout, off_qpack, off_ds, off_rowsum, off_lab, off_req, off_dq, bytes;
};

struct GradArgs {
    const float *qual, *len;
    int M;
    const float *q_hat, *l_hat, *lse, *dq_hat, *dl_hat, *dlse;   // dlse may be null
    void *d_queries, *d_bank;                                    // may be null
    float *d_qual, *d_len, *d_beta;                              // may be null
};

bool plan_grad(int B, int N, int d, int dtype, int M, int n_cu, GradPlan *p);

hipError_t launch_grad(const GradPlan &p, const AttendBank &a, const GradArgs &g, void *ws,
                       hipStream_t s);

// Rows of the bank (bank_rows.hip). Row j of src (fp32 or bf16) becomes row
// at[j] (j, if at is null) of the bank, with its norm; rows outside [0, N) are
// left out. Labels and usage where their pointers are not null.
struct RowsArgs {
    const uint8_t *src;
    const int32_t *at;
    int n, N, d, M;
    uint8_t *rows, *scales;
    float *norms;
    const float *new_qual, *new_len;
    float *qual, *len, *usage;
    float usage0;
};

hipError_t launch_write_rows(int src_dtype, int dtype, const RowsArgs &a, hipStream_t s);

// The n rows of least usage (equal usage: the lower row first) of those whose
// may_go is not 0, ascending; -1 behind them where there are fewer.
size_t evict_bytes(int N);

hipError_t launch_evict(const float *usage, const uint8_t *may_go, int N, int n, int32_t *victims,
                        void *ws, hipStream_t s);

}  // namespace rb
