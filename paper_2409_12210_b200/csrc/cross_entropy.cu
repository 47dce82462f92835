// Softmax cross entropy over a vocabulary straight from hidden rows, and its gradient, without logits in memory.
//
//   z = x w^T;  lse_t = log sum_v exp z_tv;  loss_t = lse_t - z_t,label
//   dz_t = f_t (exp(z_t - lse_t) - [v = label]);  dx = dz w;  dw = dz^T x
//
// Forward: the product's epilogue turns every run of 128 logits of a row into their largest and the sum of exponentials
// over it (DenseLse), 8 bytes for 256; a second kernel joins the runs of a row.  What bounds it is the product.
// Gradient: the logits are formed again, a piece of the vocabulary at a time, and leave the product as dz in bf16
// (DenseSoftmax); dx and dw of the piece follow as one launch, dx on top of the sum of the pieces before (DenseSum).  That
// is 8 T d V operations with the forward's 2, against 6 of a form that keeps T x V logits.
#include <algorithm>

#include "dense_gemm.h"
#include "launch.h"

namespace modse {
namespace {

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

constexpr float kLog2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

// ---- the runs of a row joined ----
struct RowsArgs {
    TokenIds labels;
    const float2 *part;
    const float *picked;
    float *loss, *lse, *total;
    double2 *sums;           // of each block: losses, tokens counted
    int *counter, *status;
    int n, runs, vocabulary;
};

// 32 rows a block, one a lane; warp w joins an even share of their runs, the first warp the 32 shares.
__global__ void __launch_bounds__(1024) loss_rows_kernel(const RowsArgs p)
{
    __shared__ float2 share[32][33];
    __shared__ double2 sum[32];
    __shared__ int last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long t = (long long)blockIdx.x * 32 + lane;
    wait_for_earlier_kernels();
    allow_next_kernel();
    // largest first, then the sums brought to it: 2^(m - M) is 0 for a run of nothing and must not meet an infinite sum
    auto join = [](float2 a, float2 b) {
        const float m = fmaxf(a.x, b.x);
        auto to = [m](float2 v) { return v.y == INFINITY ? v.y : v.y * exp2f(v.x - m); };
        return make_float2(m, to(a) + to(b));
    };
    const int lo = (int)((long long)p.runs * warp / 32), hi = (int)((long long)p.runs * (warp + 1) / 32);
    float2 v = make_float2(-3.402823466e38f, 0.f);
    if (t < p.n) {
        for (int c0 = lo; c0 < hi; c0 += 8) {
            float2 r[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) r[u] = c0 + u < hi ? __ldcg(p.part + (long long)(c0 + u) * p.n + t) : make_float2(-3.402823466e38f, 0.f);
#pragma unroll
            for (int u = 0; u < 8; ++u) v = join(v, r[u]);
        }
    }
    share[warp][lane] = v;
    __syncthreads();
    if (warp == 0) {
        float loss = 0.f;
        bool counted = false;
        if (t < p.n) {
            for (int w = 1; w < 32; ++w) v = join(v, share[w][lane]);
            const float lse = (v.x + log2f(v.y)) * kLog2;
            const long long label = p.labels.at(t);
            counted = label >= 0 && label < p.vocabulary;
            if (label >= p.vocabulary) atomicMax(p.status, kDevBounds);
            if (counted) loss = lse - __ldcg(p.picked + t);
            p.loss[t] = loss;
            p.lse[t] = lse;
        }
        double s = loss, k = counted ? 1.0 : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            k += __shfl_xor_sync(0xFFFFFFFFu, k, o);
        }
        if (lane == 0 && p.total != nullptr) {
            __stcg(p.sums + blockIdx.x, make_double2(s, k));
            __threadfence();
            last = atomicAdd(p.counter, 1) == (int)gridDim.x - 1;
        }
    }
    if (p.total == nullptr) return;
    __syncthreads();
    if (!last) return;
    // whichever block is last, the order of the additions is the same
    __threadfence();
    double s = 0.0, k = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 1024) {
        const double2 b = __ldcg(p.sums + i);
        s += b.x;
        k += b.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        k += __shfl_xor_sync(0xFFFFFFFFu, k, o);
    }
    if (lane == 0) sum[warp] = make_double2(s, k);
    __syncthreads();
    if (threadIdx.x == 0) {
        s = k = 0.0;
        for (int w = 0; w < 32; ++w) {
            s += sum[w].x;
            k += sum[w].y;
        }
        p.total[0] = (float)s;
        p.total[1] = (float)k;
    }
}

// ---- what a row of the gradient is multiplied by ----
struct FactorArgs {
    TokenIds labels;
    const float *lse, *dloss, *total;
    float *lse2, *factor;
    int *head;               // status word and counters of the products that follow
    float scale;
    int n, vocabulary;
};

constexpr int kFactorThreads = 1024;
__global__ void __launch_bounds__(kFactorThreads) loss_factor_kernel(const FactorArgs p)
{
    __shared__ int bad;
    if (threadIdx.x == 0) bad = 0;
    wait_for_earlier_kernels();
    allow_next_kernel();
    const long long t = (long long)blockIdx.x * kFactorThreads + threadIdx.x;
    if (t < p.n) {
        const long long label = p.labels.at(t);
        float f = 0.f;
        if (label >= 0 && label < p.vocabulary) {
            f = p.scale;
            if (p.dloss) f *= __ldcg(p.dloss + t);
            if (p.total) f /= __ldcg(p.total + 1);
        }
        p.factor[t] = f;
        p.lse2[t] = __ldcg(p.lse + t) * kLog2e;
    }
    if (blockIdx.x != 0) return;
    // the first block clears the head and, having looked at all labels, says whether one lies past the vocabulary
    for (int i = threadIdx.x; i < (int)(kDenseZeroBytes / 4); i += kFactorThreads) p.head[i] = 0;
    __syncthreads();
    for (long long t0 = threadIdx.x; t0 < p.n; t0 += 8 * kFactorThreads) {
        bool past = false;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const long long i = t0 + u * kFactorThreads;
            past |= (i < p.n ? p.labels.at(i) : -1) >= p.vocabulary;
        }
        if (past) bad = 1;
    }
    __syncthreads();
    if (threadIdx.x == 0 && bad) p.head[0] = kDevBounds;
}

// ---- host ----
// Limits of the products' 32-bit indexes.
bool shape_ok(int n, int d, int vocabulary)
{
    return n >= 0 && n <= (1 << 28) && d >= 8 && d % 8 == 0 && d <= (1 << 20) && vocabulary >= 1 && vocabulary <= (1 << 28) &&
           (((long long)n + 255) / 256) * (((long long)vocabulary + 127) / 128) < (1ll << 30) &&
           (((long long)std::max(n, vocabulary) + 255) / 256) * ((d + 127) / 128) < (1ll << 30);
}
bool id_bytes_ok(int b) { return b == 4 || b == 8; }

DenseItem logits_item(int n, int d, int vocabulary, const void *x, const void *w)
{
    DenseItem it{};
    it.a = {x, n, d, d};
    it.b = {w, vocabulary, d, d};
    it.p.M = n;
    it.p.N = vocabulary;
    it.k = d;
    return it;
}

struct ForwardLayout { size_t counter, partials, partial_bytes, picked, part, sums, total; int runs; };
ForwardLayout forward_layout(int n, int d, int vocabulary)
{
    ForwardLayout L;
    const DenseItem it = logits_item(n, d, vocabulary, nullptr, nullptr);
    L.runs = (vocabulary + kDenseLseCols - 1) / kDenseLseCols;
    // twice the bound of 128-column tiles holds that of the 256-column ones this product takes
    L.partial_bytes = 2 * dense_partial_bound(DenseBf16, &it, 1);
    L.counter = up256(kDenseHead + L.partial_bytes);
    L.picked = L.counter + 256;
    L.part = up256(L.picked + (size_t)n * 4);
    L.sums = up256(L.part + (size_t)L.runs * n * 8);
    L.total = up256(L.sums + ((size_t)n + 31) / 32 * 16);
    return L;
}

// dx = dz w and dw = dz^T x of a piece of the vocabulary
DenseItem dx_item(int n, int d, int cols, int ld, const void *dz, const void *w, void *dx, float *sum, bool add, bool keep)
{
    DenseItem it{};
    it.a = {dz, n, cols, ld};
    it.b = {w, cols, d, d};
    it.p.M = n;
    it.p.N = d;
    it.p.flags = kDenseBMn | (add ? kDenseAdd : 0) | (keep ? kDenseKeep : 0);
    it.p.in0 = sum;
    it.p.out0 = dx;
    it.p.out1 = sum;
    it.p.ld_out = d;
    it.k = cols;
    return it;
}
DenseItem dw_item(int n, int d, int cols, int ld, const void *dz, const void *x, void *dw)
{
    DenseItem it{};
    it.a = {dz, n, cols, ld};
    it.b = {x, n, d, d};
    it.p.M = cols;
    it.p.N = d;
    it.p.flags = kDenseAMn | kDenseBMn;
    it.p.out0 = dw;
    it.p.ld_out = d;
    it.k = n;
    return it;
}

// Columns of a piece: dz of a piece is at most 2^26 elements (128 MB, about what L2 holds) or 2048 columns, whichever is more, the pieces
// evenly long and whole tiles wide.
int piece_cols(int n, int vocabulary)
{
    const long long most = std::max<long long>(2048, (1ll << 26) / std::max(n, 1));
    if (vocabulary <= most) return vocabulary;
    const long long pieces = (vocabulary + most - 1) / most;
    return (int)(((vocabulary + pieces - 1) / pieces + 255) / 256 * 256);
}
int up64(int v) { return (v + 63) / 64 * 64; }

// One launch for both products unless dx's few long tiles would outlast all the others: then dx is cut along the vocabulary
// in a launch of its own.
bool together(int n, int d, int cols)
{
    const long long tn = (n + 255) / 256, td = (d + 255) / 256, tv = (cols + 255) / 256, kn = (n + 63) / 64, kv = (cols + 63) / 64;
    return kv * (kDenseSms / 2) <= tn * td * kv + tv * td * kn;
}

struct BackwardLayout { size_t partials, partial_bytes, lse2, factor, dz, sum, total; int cols; };
BackwardLayout backward_layout(int n, int d, int vocabulary)
{
    BackwardLayout L;
    L.cols = piece_cols(n, vocabulary);
    size_t need = 0;
    auto more = [&](const DenseItem *items, int c) { need = std::max(need, dense_partial_bound(DenseBf16, items, c)); };
    // the last piece may be narrower, and the bound does not fall with an extent
    const DenseItem z = logits_item(n, d, L.cols, nullptr, nullptr);
    more(&z, 1);
    const DenseItem both[2] = {dx_item(n, d, L.cols, up64(L.cols), nullptr, nullptr, nullptr, nullptr, false, false),
                               dw_item(n, d, L.cols, up64(L.cols), nullptr, nullptr, nullptr)};
    more(both, 2);
    more(both, 1);
    more(both + 1, 1);
    L.partials = kDenseHead;
    L.partial_bytes = need;
    L.lse2 = up256(L.partials + need);
    L.factor = up256(L.lse2 + (size_t)n * 4);
    L.dz = up256(L.factor + (size_t)n * 4);
    L.sum = up256(L.dz + (size_t)n * up64(L.cols) * 2);
    L.total = L.sum + (L.cols < vocabulary ? dense_sum_bytes(n, d) : 0);
    return L;
}

}  // namespace
}  // namespace modse

using namespace modse;

#define MODSE_CUDA(expr)                                \
    do {                                                \
        if ((expr) != cudaSuccess) return MODSE_ERR_CUDA; \
    } while (0)

extern "C" {

size_t modse_cross_entropy_workspace_bytes(int n_tokens, int d_model, int vocabulary)
{
    return shape_ok(n_tokens, d_model, vocabulary) ? forward_layout(n_tokens, d_model, vocabulary).total : 0;
}

modse_status_t modse_cross_entropy(int n_tokens, int d_model, int vocabulary, const modse_cross_entropy_t *args, void *workspace,
                                   size_t workspace_bytes, void *cuda_stream)
{
    if (args == nullptr || !shape_ok(n_tokens, d_model, vocabulary) || !id_bytes_ok(args->label_bytes) || !aligned(args->total, 4))
        return MODSE_ERR_INVALID_ARG;
    const modse_cross_entropy_t &a = *args;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, s);
        if (a.total) MODSE_CUDA(cudaMemsetAsync(a.total, 0, 8, s));
        return MODSE_OK;
    }
    if (a.x == nullptr || a.w == nullptr || a.labels == nullptr || a.loss == nullptr || a.lse == nullptr || !aligned(a.x, 16) ||
        !aligned(a.w, 16) || !aligned(a.labels, a.label_bytes) || !aligned(a.loss, 4) || !aligned(a.lse, 4) ||
        workspace == nullptr || !aligned(workspace, 256))
        return MODSE_ERR_INVALID_ARG;
    const ForwardLayout L = forward_layout(n_tokens, d_model, vocabulary);
    if (workspace_bytes < L.total) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    unsigned char *ws = (unsigned char *)workspace;
    const TokenIds labels{a.labels, a.label_bytes == 8};
    LossEpilogue loss{};
    loss.labels = labels;
    loss.rows = n_tokens;
    loss.part = (float2 *)(ws + L.part);
    loss.picked = (float *)(ws + L.picked);
    loss.counter = (int *)(ws + L.counter);
    MODSE_CUDA(dense_launch_loss(DenseLse, logits_item(n_tokens, d_model, vocabulary, a.x, a.w), loss, ws, L.partial_bytes,
                                 kDenseHeadRaw, s));
    const RowsArgs r{labels, loss.part, loss.picked, a.loss, a.lse, a.total, (double2 *)(ws + L.sums), loss.counter, (int *)ws,
                     n_tokens, L.runs, vocabulary};
    MODSE_CUDA(launch_overlapped(loss_rows_kernel, (unsigned)((n_tokens + 31) / 32), 1024, 0, s, r));
    return MODSE_OK;
}

size_t modse_cross_entropy_backward_workspace_bytes(int n_tokens, int d_model, int vocabulary)
{
    return shape_ok(n_tokens, d_model, vocabulary) ? backward_layout(n_tokens, d_model, vocabulary).total : 0;
}

modse_status_t modse_cross_entropy_backward(int n_tokens, int d_model, int vocabulary, const modse_cross_entropy_grads_t *args,
                                            void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (args == nullptr || !shape_ok(n_tokens, d_model, vocabulary) || !id_bytes_ok(args->label_bytes)) return MODSE_ERR_INVALID_ARG;
    const modse_cross_entropy_grads_t &a = *args;
    if (!aligned(a.dw, 16) || !aligned(a.dx, 16)) return MODSE_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, s);
        if (a.dw) MODSE_CUDA(cudaMemsetAsync(a.dw, 0, (size_t)vocabulary * d_model * 2, s));
        return MODSE_OK;
    }
    if (a.x == nullptr || a.w == nullptr || a.labels == nullptr || a.lse == nullptr || (a.dx == nullptr && a.dw == nullptr) ||
        !aligned(a.x, 16) || !aligned(a.w, 16) || !aligned(a.labels, a.label_bytes) || !aligned(a.lse, 4) || !aligned(a.dloss, 4) ||
        !aligned(a.total, 4) || workspace == nullptr || !aligned(workspace, 256))
        return MODSE_ERR_INVALID_ARG;
    const BackwardLayout L = backward_layout(n_tokens, d_model, vocabulary);
    if (workspace_bytes < L.total) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    unsigned char *ws = (unsigned char *)workspace;
    const TokenIds labels{a.labels, a.label_bytes == 8};
    LossEpilogue loss{};
    loss.labels = labels;
    loss.rows = n_tokens;
    loss.lse2 = (float *)(ws + L.lse2);
    loss.factor = (float *)(ws + L.factor);
    const FactorArgs f{labels, a.lse, a.dloss, a.total, (float *)(ws + L.lse2), (float *)(ws + L.factor), (int *)ws, a.scale,
                       n_tokens, vocabulary};
    MODSE_CUDA(launch_overlapped(loss_factor_kernel, (unsigned)((n_tokens + kFactorThreads - 1) / kFactorThreads), kFactorThreads, 0, s, f));
    float *sum = (float *)(ws + L.sum);
    void *dz = ws + L.dz;
    for (int first = 0; first < vocabulary; first += L.cols) {
        const int cols = std::min(L.cols, vocabulary - first), ld = up64(cols);
        const size_t at = (size_t)first * d_model * 2;
        const void *w = (const unsigned char *)a.w + at;
        DenseItem z = logits_item(n_tokens, d_model, cols, a.x, w);
        z.p.out0 = dz;
        z.p.ld_out = ld;
        loss.first = first;
        MODSE_CUDA(dense_launch_loss(DenseSoftmax, z, loss, ws, L.partial_bytes, kDenseHeadZero, s));
        DenseItem items[2];
        int c = 0;
        if (a.dx) items[c++] = dx_item(n_tokens, d_model, cols, ld, dz, w, a.dx, sum, first > 0, first + cols < vocabulary);
        if (a.dw) items[c++] = dw_item(n_tokens, d_model, cols, ld, dz, a.x, (unsigned char *)a.dw + at);
        const bool one = c < 2 || together(n_tokens, d_model, cols);
        MODSE_CUDA(dense_launch(DenseSum, DenseBf16, items, one ? c : 1, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s));
        if (!one) MODSE_CUDA(dense_launch(DenseSum, DenseBf16, items + 1, 1, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s));
    }
    return MODSE_OK;
}

}  // extern "C"
