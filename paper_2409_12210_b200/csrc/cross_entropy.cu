// Softmax cross entropy over a vocabulary straight from hidden rows, and its gradient, without logits in memory.
//
//   z = x w^T;  lse_t = log sum_v exp z_tv;  loss_t = lse_t - z_t,label
//   dz_t = f_t (exp(z_t - lse_t) - [v = label]);  dx = dz w;  dw = dz^T x
//
// Forward: the product's epilogue turns every run of 128 logits of a row into their largest and the sum of exponentials
// over it (DenseLse), 8 bytes for 256; a second kernel joins the runs of a row.  What bounds it is the product (16384 x 2048
// over 32000: 1.42 to 1.49 ms, 1.44 to 1.51 PFLOP/s, by itself; 1.58 to 1.70 in a long row of calls, which the power limit holds down).  Rows of
// 64 or 256 columns are bound by the epilogue (5000 x 64 over 9000: 37 us).  Up to 32 rows, which are bound by
// reading w, go through the kernel in cross_entropy_few.cu instead.
// Gradient: the logits are formed again, a piece of the vocabulary at a time, and leave the product as dz in bf16
// (DenseSoftmax); dx and dw of the piece follow as one launch, dx on top of the sum of the pieces before (DenseSum).  That
// is 8 T d V operations with the forward's 2, against 6 of a form that keeps T x V logits.  8192 x 2048 over 32000: 2.11 to 2.24 ms,
// 1.44 to 1.53 PFLOP/s, by itself, 2.38 to 2.60 in a long row; 2051 x 1536 over 100003: 1.49 to 1.58 ms, 1.20 to 1.27, and 1.71
// to 1.81.
//
// dz is rounded to bf16 once, because the products read 16-bit operands.  A factor that all rows share - the 1 / count of a
// mean - would be rounded with it, by the same amount everywhere (0.0033 off in norm where the count was 7372, 0.0023 without), so
// rows enter with their weight over the largest one and the rest multiplies the sums in fp32.
#include <algorithm>

#include "cross_entropy.h"
#include "launch.h"

namespace modse {
namespace {

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

constexpr float kLog2e = 1.4426950408889634f;

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

// 32 rows a block.  First warp w joins an even share of the runs of all rows, one a lane; then the 32 shares of row w, one a lane.
__global__ void __launch_bounds__(1024) loss_rows_kernel(const RowsArgs p)
{
    __shared__ float2 share[32][33];
    __shared__ double2 sum[32];
    __shared__ int last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row0 = (long long)blockIdx.x * 32;
    wait_for_earlier_kernels();
    allow_next_kernel();
    // a sum brought to another largest number: exp(m - M) is 0 for a run of nothing and must not meet an infinite sum
    auto to = [](float2 v, float m) { return v.y == INFINITY ? v.y : v.y * exp2f((v.x - m) * kLog2e); };
    const int lo = (int)((long long)p.runs * warp / 32), hi = (int)((long long)p.runs * (warp + 1) / 32);
    const float2 none = make_float2(-3.402823466e38f, 0.f);
    float2 v = none;
    if (row0 + lane < p.n) {
        for (int c0 = lo; c0 < hi; c0 += 8) {
            float2 r[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) r[u] = c0 + u < hi ? __ldcg(p.part + (long long)(c0 + u) * p.n + row0 + lane) : none;
            float m = v.x;
#pragma unroll
            for (int u = 0; u < 8; ++u) m = fmaxf(m, r[u].x);
            float s = to(v, m);
#pragma unroll
            for (int u = 0; u < 8; ++u) s += to(r[u], m);
            v = make_float2(m, s);
        }
    }
    share[warp][lane] = v;
    __syncthreads();
    v = share[lane][warp];
    float m = v.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float s = to(v, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) {
        const long long t = row0 + warp;
        float loss = 0.f;
        bool counted = false;
        if (t < p.n) {
            const float lse = m + logf(s);
            const long long label = p.labels.at(t);
            counted = label >= 0 && label < p.vocabulary;
            if (label >= p.vocabulary) atomicMax(p.status, kDevBounds);
            if (counted) loss = lse - __ldcg(p.picked + t);
            p.loss[t] = loss;
            p.lse[t] = lse;
        }
        sum[warp] = make_double2(loss, counted ? 1.0 : 0.0);
    }
    if (p.total == nullptr) return;
    __syncthreads();
    if (warp == 0) {
        double a = sum[lane].x, k = sum[lane].y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
            k += __shfl_xor_sync(0xFFFFFFFFu, k, o);
        }
        if (lane == 0) {
            if (gridDim.x == 1) {
                p.total[0] = (float)a;
                p.total[1] = (float)k;
                last = 0;
            } else {
                __stcg(p.sums + blockIdx.x, make_double2(a, k));
                __threadfence();
                last = atomicAdd(p.counter, 1) == (int)gridDim.x - 1;
            }
        }
    }
    __syncthreads();
    if (!last) return;
    // whichever block is last, the order of the additions is the same
    __threadfence();
    double a = 0.0, k = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 1024) {
        const double2 b = __ldcg(p.sums + i);
        a += b.x;
        k += b.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        k += __shfl_xor_sync(0xFFFFFFFFu, k, o);
    }
    if (lane == 0) sum[warp] = make_double2(a, k);
    __syncthreads();
    if (threadIdx.x == 0) {
        a = k = 0.0;
        for (int w = 0; w < 32; ++w) {
            a += sum[w].x;
            k += sum[w].y;
        }
        p.total[0] = (float)a;
        p.total[1] = (float)k;
    }
}

// ---- what a row of the gradient is multiplied by ----
struct FactorArgs {
    TokenIds labels;
    const float *dloss, *total;
    float *factor;
    float *scalars;          // 1 / the largest factor, and what the sums are multiplied by: scale / total[1] times the largest factor
    int *head;               // status word and counters of the products that follow
    float scale;
    int n, vocabulary;
};

constexpr int kFactorThreads = 1024;
__global__ void __launch_bounds__(kFactorThreads) loss_factor_kernel(const FactorArgs p)
{
    __shared__ int bad, wild;
    __shared__ float most[32];
    if (threadIdx.x == 0) bad = wild = 0;
    wait_for_earlier_kernels();
    allow_next_kernel();
    auto factor_of = [&](long long label, long long t) {
        return label >= 0 && label < p.vocabulary ? (p.dloss ? __ldcg(p.dloss + t) : 1.f) : 0.f;
    };
    const long long t = (long long)blockIdx.x * kFactorThreads + threadIdx.x;
    if (t < p.n) p.factor[t] = factor_of(p.labels.at(t), t);
    if (blockIdx.x != 0) return;
    // the first block clears the head and, having looked at all rows, says whether a label lies past the vocabulary and how
    // large the largest factor is
    for (int i = threadIdx.x; i < (int)(kDenseZeroBytes / 4); i += kFactorThreads) p.head[i] = 0;
    __syncthreads();
    float m = 0.f;
    for (long long t0 = threadIdx.x; t0 < p.n; t0 += 8 * kFactorThreads) {
        long long label[8];
        bool past = false;
#pragma unroll
        for (int u = 0; u < 8; ++u) label[u] = t0 + u * kFactorThreads < p.n ? p.labels.at(t0 + u * kFactorThreads) : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            past |= label[u] >= p.vocabulary;
            const float f = fabsf(factor_of(label[u], t0 + u * kFactorThreads));
            if (f < INFINITY) m = fmaxf(m, f);           // an infinity or a NaN is no measure for the others
            else wild = 1;
        }
        if (past) bad = 1;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; ++w) m = fmaxf(m, most[w]);
        if (bad) p.head[0] = kDevBounds;
        // (below 2^-126 the quotient would be infinite; without a row that counts nothing is multiplied, by no count either, unless
        // an infinity or a NaN is to be seen)
        const bool some = m >= 1.17549435e-38f;
        const float rest = p.total ? p.scale / __ldcg(p.total + 1) : p.scale;
        const float gain = some ? rest * m : m == 0.f && !wild ? 0.f : rest;
        p.scalars[0] = gain == 0.f ? 0.f : some ? 1.f / m : 1.f;      // (where the gain is 0 no row counts, whatever its logits are)
        p.scalars[1] = gain;
    }
}

// dx = gain times the sum of `parts` running sums (see dense_sum_bytes), where dx was summed up in parts.
__global__ void __launch_bounds__(256) loss_join_kernel(const float *sums, long long part_floats, int parts, const float *gain, __nv_bfloat16 *dx,
                                                        int n, int d)
{
    wait_for_earlier_kernels();
    allow_next_kernel();
    const int lane = threadIdx.x & 31, across = (d + 31) / 32;
    const long long block = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (block >= (long long)((n + 31) / 32) * across) return;
    const float g = __ldcg(gain);
    const int r = (int)(block / across) * 32 + lane, c0 = (int)(block % across) * 32;
    float4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q = 0; q < parts; ++q) {
        const float4 *at = reinterpret_cast<const float4 *>(sums + q * part_floats + block * 1024) + lane;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 u = __ldcg(at + 32 * j);
            v[j].x += u.x; v[j].y += u.y; v[j].z += u.z; v[j].w += u.w;
        }
    }
    if (r >= n) return;
    auto pack = [g](float a, float b) {
        __nv_bfloat162 t = __floats2bfloat162_rn(a * g, b * g);
        return *reinterpret_cast<uint32_t *>(&t);
    };
#pragma unroll
    for (int j = 0; j < 8; j += 2)
        if (c0 + 4 * j < d)                              // (d is a multiple of 8)
            *reinterpret_cast<uint4 *>(dx + (size_t)r * d + c0 + 4 * j) =
                make_uint4(pack(v[j].x, v[j].y), pack(v[j].z, v[j].w), pack(v[j + 1].x, v[j + 1].y), pack(v[j + 1].z, v[j + 1].w));
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
    const int wide = (vocabulary + kDenseLseCols - 1) / kDenseLseCols, few = few_tiles(vocabulary).count;
    L.runs = few_takes(n, d, vocabulary) ? few : wide;
    // twice the bound of 128-column tiles holds that of the 256-column ones this product takes
    L.partial_bytes = 2 * dense_partial_bound(DenseBf16, &it, 1);
    L.counter = up256(kDenseHead + L.partial_bytes);
    L.picked = L.counter + 256;
    L.part = up256(L.picked + (size_t)n * 4);
    // (what holds more rows holds fewer)
    L.sums = up256(L.part + std::max((size_t)few * std::min(n, kFewRows), (size_t)wide * n) * 8);
    L.total = up256(L.sums + ((size_t)n + 31) / 32 * 16);
    return L;
}

// dx = dz w of a piece of the vocabulary (or of a part of its columns), on top of `sum` or into it, and dw = dz^T x
DenseItem dx_item(int n, int d, int cols, int ld, const void *dz, const void *w, void *dx, float *sum, bool add, bool keep, const float *gain)
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
    it.p.gain = gain;
    it.k = cols;
    return it;
}
DenseItem dw_item(int n, int d, int cols, int ld, const void *dz, const void *x, void *dw, const float *gain)
{
    DenseItem it{};
    it.a = {dz, n, cols, ld};
    it.b = {x, n, d, d};
    it.p.M = cols;
    it.p.N = d;
    it.p.flags = kDenseAMn | kDenseBMn;
    it.p.out0 = dw;
    it.p.ld_out = d;
    it.p.gain = gain;
    it.k = n;
    return it;
}

// Columns of a piece: dz of a piece is about 2^26 elements (128 MB, about what L2 holds) or 2048 columns, whichever is more, the pieces
// evenly long and whole tiles wide, which makes them at most 255 columns wider than that.
int piece_cols(int n, int vocabulary)
{
    const long long most = std::max<long long>(2048, (1ll << 26) / std::max(n, 1));
    if (vocabulary <= most) return vocabulary;
    const long long pieces = (vocabulary + most - 1) / most;
    return (int)(((vocabulary + pieces - 1) / pieces + 255) / 256 * 256);
}
int up64(int v) { return (v + 63) / 64 * 64; }

// Parts into which dx's contraction over a piece's columns is cut, each with a running sum of its own: as many as keep one of its
// tiles below a quarter of what a CTA pair has to do in all (2051 x 1536 over pieces of 25088: 54 tiles of 392 k-blocks beside 588 of
// 33; the whole gradient over four pieces takes 1862 us in one part, 1551 in four), but not below 24 k-blocks.
int parts_of(int n, int d, int cols)
{
    const long long tn = (n + 255) / 256, td = (d + 255) / 256, tv = (cols + 255) / 256, kn = (n + 63) / 64, kv = (cols + 63) / 64;
    const long long each = (tn * td * kv + tv * td * kn) / (kDenseSms / 2);
    int parts = 1;
    while (2 * parts < kDenseMaxSums && kv * 4 > each * parts && kv >= 48 * parts) parts *= 2;
    return parts;
}
int part_cols(int cols, int parts) { return up64((cols + parts - 1) / parts); }

// The products of one piece; *n_dx is how many of them are parts of dx.
int piece_items(DenseItem *items, int n, int d, int cols, int ld, int parts, unsigned char *dz, const unsigned char *w, const void *x, void *dx,
                void *dw, float *sums, size_t part_floats, bool add, bool keep, const float *gain, int *n_dx)
{
    int c = 0;
    if (dx) {
        const int each = part_cols(cols, parts);
        for (int at = 0; at < cols; at += each, ++c)
            items[c] = dx_item(n, d, std::min(each, cols - at), ld, dz + (size_t)at * 2, w + (size_t)at * d * 2, dx, sums + c * part_floats, add, keep, gain);
    }
    *n_dx = c;
    if (dw) items[c++] = dw_item(n, d, cols, ld, dz, x, dw, gain);
    return c;
}

// What the products of pieces of `cols` columns, dx in `parts`, can use for tiles that they cut.
size_t partials_of(int n, int d, int cols, int parts)
{
    size_t need = 0;
    auto more = [&](const DenseItem *items, int c) { need = std::max(need, dense_partial_bound(DenseBf16, items, c)); };
    // the last piece may be narrower, and the bound does not fall with an extent
    const DenseItem z = logits_item(n, d, cols, nullptr, nullptr);
    more(&z, 1);
    unsigned char *const some = reinterpret_cast<unsigned char *>(16);
    DenseItem items[kDenseMaxSums];
    int n_dx;
    const int c = piece_items(items, n, d, cols, up64(cols), parts, some, some, some, some, some, nullptr, 0, false, false, nullptr, &n_dx);
    more(items, c);
    more(items, n_dx);
    more(items + n_dx, 1);
    return need;
}

// More rows are worked off in narrower pieces and fewer parts, so that what a call needs may fall as n grows (2048 columns,
// 32000 words: 222.7 MB for 2097 rows, 156.3 for 2098).  A workspace for many rows is to serve fewer, so room is made for
// bounds that do not fall:
// dz: n rows of the whole vocabulary, or of the widest piece that n makes;
// sums: parts_of doubles from p to 2 p only where kv 4 > each p, and each >= tn td kv / 74, so 2 p < 592 / (tn td); a sum is at
// most tn td tiles of 256 KB;
// pieces of cut tiles: those of products as long as the vocabulary, a sum as many as there can be.
constexpr size_t kMostSums = (size_t)8 * (kDenseSms / 2) * 256 * 256 * 4;
struct BackwardLayout { size_t partials, partial_bytes, scalars, factor, dz, sum, total; int cols, parts; };
BackwardLayout backward_layout(int n, int d, int vocabulary)
{
    BackwardLayout L;
    L.cols = piece_cols(n, vocabulary);
    L.parts = parts_of(n, d, L.cols);
    int most_parts = 1;
    while (2 * most_parts < kDenseMaxSums && (vocabulary + 63) / 64 >= 48 * most_parts) most_parts *= 2;
    const size_t widest = std::max((size_t)n * 2048, ((size_t)1 << 26) + (size_t)n * 255), one = dense_sum_bytes(n, d);
    const size_t dz = std::min((size_t)n * up64(vocabulary), widest);
    const size_t sums = L.cols == vocabulary && most_parts == 1 ? 0 : std::max(one, std::min(most_parts * one, kMostSums));
    DenseItem items[kDenseMaxSums];
    for (int i = 0; i < most_parts; ++i) items[i] = dx_item(n, d, vocabulary, up64(vocabulary), nullptr, nullptr, nullptr, nullptr, false, false, nullptr);
    items[most_parts] = dw_item(n, d, vocabulary, up64(vocabulary), nullptr, nullptr, nullptr, nullptr);
    const size_t partials = std::max({partials_of(n, d, vocabulary, 1), dense_partial_bound(DenseBf16, items, most_parts),
                                      dense_partial_bound(DenseBf16, items, most_parts + 1)});
    L.partial_bytes = partials_of(n, d, L.cols, L.parts);
    L.partials = kDenseHead;
    L.scalars = up256(L.partials + partials);
    L.factor = L.scalars + 256;
    L.dz = up256(L.factor + (size_t)n * 4);
    L.sum = up256(L.dz + dz * 2);
    L.total = L.sum + sums;
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
    if (few_takes(n_tokens, d_model, vocabulary)) MODSE_CUDA(launch_loss_few(n_tokens, d_model, vocabulary, a.x, a.w, loss, (int *)ws, s));
    else MODSE_CUDA(dense_launch_loss(DenseLse, logits_item(n_tokens, d_model, vocabulary, a.x, a.w), loss, ws, L.partial_bytes, kDenseHeadRaw, s));
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
    loss.lse = a.lse;
    loss.factor = (float *)(ws + L.factor);
    loss.factor_scale = (float *)(ws + L.scalars);
    const float *gain = loss.factor_scale + 1;
    const FactorArgs f{labels, a.dloss, a.total, (float *)(ws + L.factor), (float *)(ws + L.scalars), (int *)ws, a.scale, n_tokens, vocabulary};
    MODSE_CUDA(launch_overlapped(loss_factor_kernel, (unsigned)((n_tokens + kFactorThreads - 1) / kFactorThreads), kFactorThreads, 0, s, f));
    float *sum = (float *)(ws + L.sum);
    unsigned char *dz = ws + L.dz;
    const size_t part_floats = dense_sum_bytes(n_tokens, d_model) / 4;
    for (int first = 0; first < vocabulary; first += L.cols) {
        const int cols = std::min(L.cols, vocabulary - first), ld = up64(cols);
        const size_t at = (size_t)first * d_model * 2;
        const unsigned char *w = (const unsigned char *)a.w + at;
        DenseItem z = logits_item(n_tokens, d_model, cols, a.x, w);
        z.p.out0 = dz;
        z.p.ld_out = ld;
        loss.first = first;
        MODSE_CUDA(dense_launch_loss(DenseSoftmax, z, loss, ws, L.partial_bytes, kDenseHeadZero, s));
        DenseItem items[kDenseMaxSums];
        int n_dx;
        const bool keep = L.parts > 1 || first + cols < vocabulary;
        const int c = piece_items(items, n_tokens, d_model, cols, ld, L.parts, dz, w, a.x, a.dx, a.dw ? (unsigned char *)a.dw + at : nullptr, sum,
                                  part_floats, first > 0, keep, gain, &n_dx);
        MODSE_CUDA(dense_launch(DenseSum, DenseBf16, items, c, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s));
    }
    if (a.dx && L.parts > 1) {
        const int parts = (L.cols + part_cols(L.cols, L.parts) - 1) / part_cols(L.cols, L.parts);
        const long long blocks = (long long)((n_tokens + 31) / 32) * ((d_model + 31) / 32);
        MODSE_CUDA(launch_overlapped(loss_join_kernel, (unsigned)((blocks + 7) / 8), 256, 0, s, (const float *)sum, (long long)part_floats, parts, gain,
                                     (__nv_bfloat16 *)a.dx, n_tokens, d_model));
    }
    return MODSE_OK;
}

}  // extern "C"
