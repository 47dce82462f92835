// Dense matrix products on CTA pairs (tcgen05, cta_group::2) with fused epilogues: the products of modse_linear, its
// gradients and modse_orthogonalize.
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
    DenseStep = 4      // x = alpha acc + beta in0: its two fp16 halves, or the final bf16 result times scale
};
enum DenseType : int { DenseBf16 = 0, DenseF16 = 1, DenseE4m3 = 2 };
enum : int {
    kDenseAMn = 1,     // the row operand lies with its rows along the contiguous axis ([K, M]), not [M, K]
    kDenseBMn = 2,     // same for the column operand ([K, N], not [N, K])
    kDenseSym = 4,     // out is symmetric: tiles below the diagonal are not computed but mirrored
    kDenseLast = 8,    // DenseStep: write the final result
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
};

struct LinearEpilogue {
    const float *sx, *sw;
    const __nv_bfloat16 *bias, *residual;
    __nv_bfloat16 *z, *y;
    int act;
};

// out[c] = sum over r of part[r][c], in order, done beside the products of a DensePlain launch (cols 0: none).
struct DenseColumnSum {
    const float *part;
    float *out;
    int rows, cols;
};

constexpr int kDenseMaxProblems = 16;
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

}  // namespace modse
