// Dense matrix products on CTA pairs (tcgen05, cta_group::2) with fused epilogues: the products of modse_linear, its
// gradients, modse_orthogonalize and modse_cross_entropy.
#pragma once

#include <cuda.h>

#include "modse_internal.h"

namespace modse {

// What happens to an accumulator on its way out.
enum DenseMode : int {
    DenseLinear = 0,   // y = act(acc * sx * sw + bias) + residual, z beside it
    DensePlain = 1,    // out = acc (bf16)
    DenseGram = 2,     // out = alpha acc (fp16), symmetric
    DensePoly = 3,     // out = alpha acc + beta in0 + scale I (fp16), symmetric
    DenseStep = 4,     // x = alpha acc + beta in0: its two fp16 halves, or the final bf16 result times scale
    DenseLse = 5,      // rows of logits: largest and sum of exponentials of each run of 128 columns, the label's logit
    DenseSoftmax = 6,  // logits to their gradient: factor (exp(acc - lse) - [column is the label]) (bf16)
    DenseSum = 7       // out = acc + in0: a running fp32 sum (kDenseAdd, kDenseKeep) whose last part leaves as bf16
};
enum DenseType : int { DenseBf16 = 0, DenseF16 = 1, DenseE4m3 = 2 };
enum : int {
    kDenseAMn = 1,     // the row operand lies with its rows along the contiguous axis ([K, M]), not [M, K]
    kDenseBMn = 2,     // same for the column operand ([K, N], not [N, K])
    kDenseSym = 4,     // out is symmetric: tiles below the diagonal are not computed but mirrored
    kDenseLast = 8,    // DenseStep: write the final result
    kDenseAdd = 32,    // DenseSum: in0 is added
    kDenseKeep = 64,   // DenseSum: the sum goes to out1 in fp32, not to out0
    kDenseTmaOut = 16  // set by the launch: the final result's rows are aligned for TMA and whole 16-byte pieces long
};

// One product out[M, N] = sum_k A[m, k] B[n, k] of a launch.
struct DenseProblem {
    int M, N, nk;            // output extents, k-blocks (128 bytes of the contraction axis each)
    int mt, nt;              // row and column tiles
    int tile0;               // this problem's first tile in the launch's list
    int flags;
    float alpha, beta, scale;
    const void *in0;
    void *out0, *out1;
    long long ld_in, ld_out; // elements
    const float *gain;       // DenseSum: what leaves as bf16 is multiplied by this number (null: 1)
};

struct LinearEpilogue {
    const float *sx, *sw;
    const __nv_bfloat16 *bias, *residual;
    __nv_bfloat16 *z, *y;
    int act;
};

// Token ids as the caller holds them; read from L2, where everything the stream held before the call has arrived.
struct TokenIds {
    const void *p;
    int wide;          // 64-bit
#ifdef __CUDACC__
    __device__ __forceinline__ long long at(long long i) const
    {
        return wide ? __ldcg(static_cast<const long long *>(p) + i) : (long long)__ldcg(static_cast<const int *>(p) + i);
    }
#endif
};

// The rows of DenseLse and DenseSoftmax.  DenseLse writes, for run c of 128 columns and row t, part[c * rows + t] =
// (M, sum over the run of exp(z - M)), M the run's largest logit held to finite numbers.  Both subtract before they multiply
// by log2(e): a difference from the largest logit is exact where it is small, however large the logits are, while the
// product's rounding grows with them (1e5 log2(e) is off by up to 2^-8).
struct LossEpilogue {
    TokenIds labels;
    long long first;       // vocabulary index of column 0
    long long rows;
    float2 *part;
    float *picked;         // [rows] the label's logit
    int *counter;          // cleared by DenseLse for the kernel behind it
    const float *lse, *factor, *factor_scale;      // [rows] lse, factor; and a number that all factors are multiplied by
};
constexpr int kDenseLseCols = 128;
// A running sum of DenseSum: blocks of 32 rows x 32 columns, row by row of blocks, block element (r, c) at
// (c / 4) * 128 + r * 4 + c % 4, so that a warp that holds a row a lane moves 512 contiguous bytes at a time.
inline size_t dense_sum_bytes(long long rows, long long cols) { return (size_t)((rows + 31) / 32) * (size_t)((cols + 31) / 32) * 4096; }

// out[c] = sum over r of part[r][c], in order, done beside the products of a DensePlain launch (cols 0: none).
struct DenseColumnSum {
    const float *part;
    float *out;
    int rows, cols;
};

constexpr int kDenseMaxProblems = 16, kDenseMaxSums = 9;      // of a launch; of one in the mode DenseSum
// An operand as it lies in memory: rows x cols elements, ld elements from row to row (a multiple of 16 bytes).
struct DenseOperand {
    const void *base;
    long long rows, cols, ld;
};
struct DenseItem {
    DenseOperand a, b;
    DenseProblem p;          // mt, nt, nk, tile0 are filled in by the launch
    long long k;             // length of the contraction in elements
};

// Workspace of a call that launches dense products: the status word, the arrival counters of cut tiles, then the fp32
// pieces of cut tiles.  A launch leaves the counters zero.  Before the first launch of a call the head is either zeroed
// by another kernel of the call (kDenseHeadZero) or raw (kDenseHeadRaw): the launch then clears the status word itself
// and zeroes the counters if it uses them.
enum : int { kDenseHeadZero = 0, kDenseHeadRaw = 1 };
constexpr int kDenseSms = 148;                         // workspace sizes are asked for without a device
constexpr int kDenseMaxSplitItems = 128;               // pieces of one launch: at most one for each CTA pair
constexpr size_t kDenseCounterOffset = 64;
constexpr size_t kDenseZeroBytes = kDenseCounterOffset + (size_t)kDenseMaxSplitItems * 16 * 4;
constexpr size_t kDenseHead = (kDenseZeroBytes + 255) / 256 * 256;

// Bytes behind the head that a launch of these products (extents and flags of p, k) can use for pieces.
size_t dense_partial_bytes(DenseType type, const DenseItem *items, int n);
// Bytes that hold the pieces of these products and of any set with smaller extents or contractions: it never falls when an
// extent grows, as the exact figure does (2048 -> 5632: 14.7 MB for 2048 tokens, none for 8192).
size_t dense_partial_bound(DenseType type, const DenseItem *items, int n);

// Launches n products of one mode and type as one kernel on a workspace whose head is `ws`.
cudaError_t dense_launch(DenseMode mode, DenseType type, const DenseItem *list, int n, const LinearEpilogue *lin,
                         const DenseColumnSum *sum, void *ws, size_t partial_capacity, int head, cudaStream_t s);
// ... of DenseLse and DenseSoftmax: one product
cudaError_t dense_launch_loss(DenseMode mode, const DenseItem &item, const LossEpilogue &loss, void *ws, size_t partial_capacity,
                              int head, cudaStream_t s);

}  // namespace modse
