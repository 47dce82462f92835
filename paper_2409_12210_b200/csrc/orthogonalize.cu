// modse_orthogonalize: Newton-Schulz iteration on a set of matrices of diverse sizes.
//
//   X0 = G / (|G|_F + eps);  repeat: A = X X^T (the shorter side),  B = a I + b A + c A^2,  X <- B X;  update = scale X
//
// Three grouped products an iteration over all matrices of a call (dense_gemm.cu): A and B are symmetric, so only tiles
// on and above the diagonal are computed; a tall matrix is not transposed, its products read X along the other axis.
//
// Numbers.  The products read fp16 factors (11 bits, against 8 of bf16: the error of the result is an eighth) and
// accumulate in fp32.  X itself is carried as the sum hi + lo of two fp16 numbers (22 bits) and the step is
// B hi + a lo: the iteration multiplies small singular values by a at every step, so a rounding of the X that is carried
// on is amplified by a^steps (485 for Muon's five steps) and swamps them; a rounding of B only scales what is there, and
// lo's share of (b A + c A^2) X is below the roundings of the product.  On 64-bit models of the iteration (Gaussian,
// low-rank and decaying spectra, shorter side 256-1024) the relative error of the result is 0.10-0.17 % this way (a
// bf16 rounding alone is 0.17 %), against 0.1-6.6 % with X carried in fp16 and 1-50 % in bf16.
// Factors are stored scaled by powers of two (X by 2^12, A and B by 2^10) to stay clear of fp16's subnormals; the call
// checks on the host that the coefficients keep every singular value inside the range this leaves.
#include <cuda_fp16.h>

#include <cmath>

#include "dense_gemm.h"
#include "launch.h"
#include "orthogonalize_small.h"

namespace modse {
namespace {

constexpr int kGroup = kDenseMaxProblems;     // matrices of one launch
constexpr int kNormParts = 128;               // partial sums of squares of a matrix
constexpr float kScaleX = kOrthScaleX, kScaleA = kOrthScaleA, kScaleB = kOrthScaleB;
constexpr double kMaxSigma = 7.5, kMaxB = 60.0;     // 7.5 * 2^12 and 60 * 2^10 are below fp16's 65504

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
long long up8(long long v) { return (v + 7) / 8 * 8; }

struct PrepMatrix {
    const void *g;
    __half *hi, *lo;
    long long ld;         // of g
    int rows, cols;
};
struct PrepArgs {
    PrepMatrix m[kGroup];
    double *parts;        // [group][kNormParts]
    int *head;            // of the workspace, to be zeroed (null: zeroed already)
    float eps;
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, bool wide, int valid, float (&f)[8])
{
    if (wide) {
        if constexpr (sizeof(T) == 2) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
            f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < valid ? (float)p[i] : 0.f;
    }
}

// Row of the i-th vector of a matrix of `vecs` vectors a row; 32-bit division where the count allows it (a 64-bit one costs
// more than the eight elements it leads to).
__device__ __forceinline__ int row_of(long long i, int vecs, long long total)
{
    return total <= 0x7FFFFFFF ? (int)((unsigned)i / (unsigned)vecs) : (int)(i / vecs);
}

// 8 elements of a row a thread: 16-byte loads where the matrix allows them for all of its rows.
template <typename T>
__device__ __forceinline__ bool wide_rows(const PrepMatrix &m)
{
    return (reinterpret_cast<uintptr_t>(m.g) & 15) == 0 && m.ld * sizeof(T) % 16 == 0;
}

template <typename T>
__global__ void __launch_bounds__(256) square_sums_kernel(const __grid_constant__ PrepArgs a)
{
    __shared__ double sh[8];
    const PrepMatrix &m = a.m[blockIdx.y];
    const int vecs = (m.cols + 7) / 8;
    const long long total = (long long)m.rows * vecs;
    const bool wide = wide_rows<T>(m);
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (a.head && blockIdx.x == 0 && blockIdx.y == 0)      // status word and counters of the products that follow
        for (int i = threadIdx.x; i < (int)(kDenseZeroBytes / 4); i += 256) a.head[i] = 0;
    // Squares of fp32 numbers leave fp32's range long before the numbers do: eight are summed in fp32 where the sum is well
    // inside it (what underflows beside it does not count), in fp64 otherwise, and all sums are fp64.
    double acc = 0.0;
    constexpr int kAt = 4;                    // vectors in flight
    const bool whole = wide && m.cols % 8 == 0 && total <= 0x7FFFFFFF;
    const long long step = (long long)gridDim.x * 256;
    for (long long i0 = (long long)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += kAt * step) {
        float f[kAt][8];
        if (whole && i0 + (kAt - 1) * step < total) {
            // no branch between the loads: it would make each wait for the one before (88 us against 39 for 185 MB)
            const T *at[kAt];
#pragma unroll
            for (int k = 0; k < kAt; ++k) {
                const unsigned i = (unsigned)(i0 + k * step);
                at[k] = (const T *)m.g + (m.ld == m.cols ? 8ll * i : (long long)(i / (unsigned)vecs) * m.ld + 8 * (i % (unsigned)vecs));
            }
#pragma unroll
            for (int k = 0; k < kAt; ++k) load8(at[k], true, 8, f[k]);
        } else {
#pragma unroll
            for (int k = 0; k < kAt; ++k) {
                const long long i = i0 + k * step;
                if (i < total) {
                    const int r = (int)(i / vecs), c = 8 * (int)(i - (long long)r * vecs);
                    load8((const T *)m.g + r * m.ld + c, wide && c + 8 <= m.cols, m.cols - c, f[k]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[k][j] = 0.f;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kAt; ++k) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fmaf(f[k][j], f[k][j], s);
            if (s >= 1e-30f && s <= 1e30f) {
                acc += (double)s;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc = fma((double)f[k][j], (double)f[k][j], acc);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int i = 0; i < 8; ++i) t += sh[i];
        a.parts[blockIdx.y * kNormParts + blockIdx.x] = t;
    }
}

// X0 = G / (|G| + eps) as hi + lo, rows padded with zeros to a multiple of 8
template <typename T>
__global__ void __launch_bounds__(256) normalise_kernel(const __grid_constant__ PrepArgs a)
{
    __shared__ StartScale start_sh;
    const PrepMatrix &m = a.m[blockIdx.y];
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (threadIdx.x < 32) {
        const double *p = a.parts + blockIdx.y * kNormParts;
        double t = 0.0;
#pragma unroll
        for (int i = 0; i < kNormParts / 32; ++i) t += p[threadIdx.x + 32 * i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
        if (threadIdx.x == 0) start_sh = start_scale(sqrt(t), a.eps);
    }
    __syncthreads();
    const StartScale start = start_sh;
    const int vecs = (m.cols + 7) / 8;
    const long long total = (long long)m.rows * vecs, ldx = 8ll * vecs;
    const bool wide = wide_rows<T>(m);
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const int r = row_of(i, vecs, total), c = 8 * (int)(i - (long long)r * vecs);
        float f[8];
        load8((const T *)m.g + r * m.ld + c, wide && c + 8 <= m.cols, m.cols - c, f);
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = f[2 * j] * start.pre * start.inv, y = f[2 * j + 1] * start.pre * start.inv;
            const __half2 hh = __floats2half2_rn(x, y);
            const float2 back = __half22float2(hh);
            const __half2 ll = __floats2half2_rn(x - back.x, y - back.y);
            h[j] = *reinterpret_cast<const uint32_t *>(&hh);
            l[j] = *reinterpret_cast<const uint32_t *>(&ll);
        }
        *reinterpret_cast<uint4 *>(m.hi + r * ldx + c) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4 *>(m.lo + r * ldx + c) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

struct MatrixSpace { size_t hi0, hi1, lo, a, b; };
struct GroupLayout { size_t partials, partial_bytes, parts, total; MatrixSpace m[kGroup]; };

bool matrix_ok(const modse_matrix_t &m)
{
    return m.rows >= 1 && m.cols >= 1 && m.rows <= (1 << 20) && m.cols <= (1 << 20) && m.ld_grad >= m.cols &&
           m.ld_update >= m.cols && m.ld_grad < (1ll << 40) && m.ld_update < (1ll << 40) &&
           (m.rows < m.cols ? m.rows : m.cols) <= (1 << 17);
}

// The three products of one matrix; buffers may be null when only extents are wanted.
void step_items(const modse_matrix_t &m, const __half *hi, __half *A, __half *B, DenseItem &gram, DenseItem &poly, DenseItem &step)
{
    const bool tall = m.rows > m.cols;
    const int n = tall ? m.cols : m.rows;
    const long long ldx = up8(m.cols), ldn = up8(n);
    const DenseOperand X{hi, m.rows, m.cols, ldx}, sa{A, n, n, ldn}, sb{B, n, n, ldn};
    gram = DenseItem{};
    gram.a = gram.b = X;
    gram.p.M = gram.p.N = n;
    gram.p.flags = kDenseSym | (tall ? kDenseAMn | kDenseBMn : 0);
    gram.p.alpha = kScaleA / (kScaleX * kScaleX);
    gram.p.out0 = A;
    gram.p.ld_out = ldn;
    gram.k = tall ? m.rows : m.cols;
    poly = DenseItem{};
    poly.a = poly.b = sa;
    poly.p.M = poly.p.N = n;
    poly.p.flags = kDenseSym;
    poly.p.in0 = A;
    poly.p.out0 = B;
    poly.p.ld_out = ldn;
    poly.k = n;
    step = DenseItem{};
    step.a = tall ? X : sb;
    step.b = tall ? sb : X;
    step.p.M = m.rows;
    step.p.N = m.cols;
    step.p.flags = tall ? 0 : kDenseBMn;
    step.p.ld_in = ldx;
    step.k = n;
}

void group_layout(const modse_matrix_t *m, int n, GroupLayout &L)
{
    DenseItem gram[kGroup], poly[kGroup], step[kGroup];
    for (int i = 0; i < n; ++i) step_items(m[i], nullptr, nullptr, nullptr, gram[i], poly[i], step[i]);
    size_t need = dense_partial_bytes(DenseF16, gram, n);
    const size_t p2 = dense_partial_bytes(DenseF16, poly, n), p3 = dense_partial_bytes(DenseF16, step, n);
    need = need > p2 ? need : p2;
    need = need > p3 ? need : p3;
    L.partials = kDenseHead;
    L.partial_bytes = need;
    L.parts = up256(kDenseHead + need);
    size_t at = up256(L.parts + (size_t)kGroup * kNormParts * sizeof(double));
    for (int i = 0; i < n; ++i) {
        const int s = m[i].rows < m[i].cols ? m[i].rows : m[i].cols;
        const size_t x = up256((size_t)m[i].rows * up8(m[i].cols) * 2), q = up256((size_t)s * up8(s) * 2);
        L.m[i].hi0 = at; at += x;
        L.m[i].hi1 = at; at += x;
        L.m[i].lo = at; at += x;
        L.m[i].a = at; at += q;
        L.m[i].b = at; at += q;
    }
    L.total = at;
}

// Whether the iteration stays inside the range of the scaled fp16 factors for every start (singular values in [0, 1]).
bool coefficients_ok(float a, float b, float c, int steps)
{
    double top = 1.0;
    for (int s = 0; s < steps; ++s) {
        double next = 0.0;
        for (int i = 0; i <= 1024; ++i) {
            const double x = top * i / 1024.0, x2 = x * x, q = (double)a + (double)b * x2 + (double)c * x2 * x2;
            if (!(std::fabs(q) <= kMaxB)) return false;
            const double y = std::fabs(x * q);
            next = y > next ? y : next;
        }
        if (!(next <= kMaxSigma)) return false;
        top = next;
    }
    return true;
}

cudaError_t run_group(modse_dtype_t dtype, const modse_matrix_t *m, int n, int steps, const float *k, float eps,
                      unsigned char *ws, bool first, cudaStream_t s)
{
    GroupLayout L;
    group_layout(m, n, L);
    PrepArgs prep{};
    prep.parts = (double *)(ws + L.parts);
    prep.head = first ? (int *)ws : nullptr;
    prep.eps = eps;
    long long most = 0;
    for (int i = 0; i < n; ++i) {
        prep.m[i] = {m[i].grad, (__half *)(ws + L.m[i].hi0), (__half *)(ws + L.m[i].lo), m[i].ld_grad, m[i].rows, m[i].cols};
        const long long v = (long long)m[i].rows * (up8(m[i].cols) / 8);
        most = most > v ? most : v;
    }
    const int blocks = (int)(most / 1024 < 1 ? 1 : most / 1024 > 1024 ? 1024 : most / 1024);
    const dim3 g1(kNormParts, n), g2(blocks, n);
    cudaError_t e = dtype == MODSE_F32 ? launch_overlapped(square_sums_kernel<float>, g1, 256, 0, s, prep)
                                       : launch_overlapped(square_sums_kernel<__nv_bfloat16>, g1, 256, 0, s, prep);
    if (e == cudaSuccess)
        e = dtype == MODSE_F32 ? launch_overlapped(normalise_kernel<float>, g2, 256, 0, s, prep)
                               : launch_overlapped(normalise_kernel<__nv_bfloat16>, g2, 256, 0, s, prep);
    DenseItem gram[kGroup], poly[kGroup], step[kGroup];
    for (int it = 0; e == cudaSuccess && it < steps; ++it) {
        const bool last = it + 1 == steps;
        for (int i = 0; i < n; ++i) {
            const MatrixSpace &sp = L.m[i];
            __half *cur = (__half *)(ws + ((it & 1) ? sp.hi1 : sp.hi0)), *next = (__half *)(ws + ((it & 1) ? sp.hi0 : sp.hi1));
            __half *lo = (__half *)(ws + sp.lo);
            step_items(m[i], cur, (__half *)(ws + sp.a), (__half *)(ws + sp.b), gram[i], poly[i], step[i]);
            poly[i].p.alpha = k[2] * kScaleB / (kScaleA * kScaleA);
            poly[i].p.beta = k[1] * kScaleB / kScaleA;
            poly[i].p.scale = k[0] * kScaleB;
            DenseProblem &p = step[i].p;
            p.in0 = lo;
            p.alpha = 1.f / kScaleB;
            p.beta = k[0];
            if (last) {
                p.flags |= kDenseLast;
                p.out0 = m[i].update;
                p.ld_out = m[i].ld_update;
                p.scale = m[i].scale / kScaleX;
            } else {
                p.out0 = next;
                p.out1 = lo;           // a tile's lo is read and written by the warp that owns its rows
            }
        }
        e = dense_launch(DenseGram, DenseF16, gram, n, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s);
        if (e == cudaSuccess) e = dense_launch(DensePoly, DenseF16, poly, n, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s);
        if (e == cudaSuccess) e = dense_launch(DenseStep, DenseF16, step, n, nullptr, nullptr, ws, L.partial_bytes, kDenseHeadZero, s);
    }
    return e;
}

// The layer's expert matrices, three a expert: gate [h, d], up [h, d], down [d, h] (a column block of [d, S]).
void layer_matrices(const modse_layer_t *layer, int e, modse_dtype_t dtype, const modse_wgrads_t *g, const modse_wgrads_t *u,
                    const float *scales, modse_matrix_t (&out)[3])
{
    int d, off, h, S;
    layer_expert(layer, e, &d, &S, &off, &h);
    const size_t esz = dtype == MODSE_F32 ? 4 : 2;
    const void *gs[3] = {g ? g->dw_gate : nullptr, g ? g->dw_up : nullptr, g ? g->dw_down : nullptr};
    void *us[3] = {u ? u->dw_gate : nullptr, u ? u->dw_up : nullptr, u ? u->dw_down : nullptr};
    for (int j = 0; j < 3; ++j) {
        const size_t at = j < 2 ? (size_t)off * d : (size_t)off;
        out[j].grad = gs[j] ? (const unsigned char *)gs[j] + at * esz : nullptr;
        out[j].update = us[j] ? (unsigned char *)us[j] + at * 2 : nullptr;
        out[j].rows = j < 2 ? h : d;
        out[j].cols = j < 2 ? d : h;
        out[j].ld_grad = out[j].ld_update = j < 2 ? d : S;
        out[j].scale = scales ? scales[3 * e + j] : 1.f;
    }
}

modse_status_t check_call(modse_dtype_t dtype, int steps, const float *k, float eps)
{
    if (dtype != MODSE_F32 && dtype != MODSE_BF16) return MODSE_ERR_INVALID_ARG;
    if (steps < 1 || steps > 64 || k == nullptr || !(eps >= 0.f) || eps > 3e38f) return MODSE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (!std::isfinite(k[i])) return MODSE_ERR_INVALID_ARG;
    return coefficients_ok(k[0], k[1], k[2], steps) ? MODSE_OK : MODSE_ERR_UNSUPPORTED;
}

// Which form a matrix of a set takes.  Short sides above 128 take the grouped one.  The others take the one-kernel form,
// unless the set needs grouped launches anyway and they all fit beside its matrices there: those launches wait more than
// they compute when matrices are small, and the two forms would run one after the other (86 x 717 with 1508 x 717: 257 us
// in both forms, 190 in one).
// Clusters of sixteen blocks are for sets of at most seven matrices, as many as run at the same time (3500 x 128: seven of
// them 102 us against 168 in the grouped form, eight 200 against 170); all matrices of a launch take the same cluster.
constexpr int kWideSet = 7;
struct SetPlan {
    bool small_form;      // whether the one-kernel form is used
    int most;             // blocks of a cluster there
};
bool fits_small(const modse_matrix_t &m, int most) { return orthogonalize_small_form(m.rows, m.cols, most).blocks > 0; }
SetPlan plan_set(const modse_matrix_t *m, int total)
{
    const int most = total <= kWideSet ? 16 : 8;
    int grouped = 0, small = 0;
    for (int i = 0; i < total; ++i) (fits_small(m[i], most) ? small : grouped) += 1;
    const int room = (kGroup - grouped % kGroup) % kGroup;
    return {grouped == 0 || small > room, most};
}
bool takes_small(const SetPlan &p, const modse_matrix_t &m) { return p.small_form && fits_small(m, p.most); }

// The next matrices from index i on, up to a launch's worth, that take the grouped form; i moves on.
int next_group(const SetPlan &p, const modse_matrix_t *m, int total, int &i, modse_matrix_t (&group)[kGroup])
{
    int n = 0;
    for (; i < total && n < kGroup; ++i)
        if (!takes_small(p, m[i])) group[n++] = m[i];
    return n;
}

bool pointers_ok(modse_dtype_t dtype, const modse_matrix_t &m)
{
    return m.grad != nullptr && m.update != nullptr && (reinterpret_cast<uintptr_t>(m.grad) & (dtype == MODSE_F32 ? 3 : 1)) == 0 &&
           (reinterpret_cast<uintptr_t>(m.update) & 1) == 0 && std::isfinite(m.scale);
}

}  // namespace
}  // namespace modse

using namespace modse;

extern "C" {

size_t modse_orthogonalize_workspace_bytes(int n_matrices, const modse_matrix_t *matrices)
{
    if (n_matrices < 0 || (n_matrices > 0 && matrices == nullptr)) return 0;
    for (int i = 0; i < n_matrices; ++i)
        if (!matrix_ok(matrices[i])) return 0;
    const SetPlan plan = plan_set(matrices, n_matrices);
    size_t most = kDenseHead;
    modse_matrix_t group[kGroup];
    for (int i = 0; i < n_matrices;) {
        const int n = next_group(plan, matrices, n_matrices, i, group);
        if (n == 0) break;
        GroupLayout L;
        group_layout(group, n, L);
        most = L.total > most ? L.total : most;
    }
    return most;
}

modse_status_t modse_orthogonalize(modse_dtype_t dtype, int n_matrices, const modse_matrix_t *matrices, int steps,
                                   const float *coefficients, float eps, void *workspace, size_t workspace_bytes,
                                   void *cuda_stream)
{
    const modse_status_t st = check_call(dtype, steps, coefficients, eps);
    if (st != MODSE_OK) return st;
    const size_t need = modse_orthogonalize_workspace_bytes(n_matrices, matrices);
    if (need == 0) return MODSE_ERR_INVALID_ARG;
    if (n_matrices == 0) {
        clear_workspace_status(workspace, workspace_bytes, (cudaStream_t)cuda_stream);
        return MODSE_OK;
    }
    for (int i = 0; i < n_matrices; ++i)
        if (!pointers_ok(dtype, matrices[i])) return MODSE_ERR_INVALID_ARG;
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MODSE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const SetPlan plan = plan_set(matrices, n_matrices);
    bool first = true;               // the call's first kernel zeroes the workspace head
    SmallArgs small{};
    for (int j = 0; j < 3; ++j) small.k[j] = coefficients[j];
    small.eps = eps;
    small.steps = steps;
    int n = 0;
    for (int i = 0; i <= n_matrices; ++i) {
        if (i < n_matrices && takes_small(plan, matrices[i])) {
            const modse_matrix_t &m = matrices[i];
            small.m[n++] = {m.grad, (__nv_bfloat16 *)m.update, m.ld_grad, m.ld_update, m.rows, m.cols, m.scale};
        }
        if (n == kOrthSmallBatch || (i == n_matrices && n > 0)) {
            small.head = first ? (int *)workspace : nullptr;
            small.head_ints = (int)(kDenseZeroBytes / 4);
            if (launch_orthogonalize_small(dtype == MODSE_F32, small, n, plan.most, s) != cudaSuccess) return MODSE_ERR_CUDA;
            first = false;
            n = 0;
        }
    }
    modse_matrix_t group[kGroup];
    for (int i = 0; i < n_matrices;) {
        const int c = next_group(plan, matrices, n_matrices, i, group);
        if (c == 0) break;
        if (run_group(dtype, group, c, steps, coefficients, eps, (unsigned char *)workspace, first, s) != cudaSuccess)
            return MODSE_ERR_CUDA;
        first = false;
    }
    return MODSE_OK;
}

size_t modse_orthogonalize_wgrads_workspace_bytes(const modse_layer_t *layer)
{
    if (layer == nullptr) return 0;
    modse_matrix_t list[3 * kMaxExperts];
    const int N = layer_experts(layer);
    for (int e = 0; e < N; ++e) {
        modse_matrix_t three[3];
        layer_matrices(layer, e, MODSE_BF16, nullptr, nullptr, nullptr, three);
        for (int j = 0; j < 3; ++j) list[j * N + e] = three[j];
    }
    return modse_orthogonalize_workspace_bytes(3 * N, list);
}

modse_status_t modse_orthogonalize_wgrads(const modse_layer_t *layer, modse_dtype_t dtype, const modse_wgrads_t *grads,
                                          const modse_wgrads_t *updates, const float *scales, int steps,
                                          const float *coefficients, float eps, void *workspace, size_t workspace_bytes,
                                          void *cuda_stream)
{
    if (layer == nullptr || grads == nullptr || updates == nullptr) return MODSE_ERR_INVALID_ARG;
    modse_matrix_t list[3 * kMaxExperts];
    const int N = layer_experts(layer);
    if (!grads->dw_gate || !grads->dw_up || !grads->dw_down || !updates->dw_gate || !updates->dw_up || !updates->dw_down)
        return MODSE_ERR_INVALID_ARG;
    for (int e = 0; e < N; ++e) {
        modse_matrix_t three[3];
        layer_matrices(layer, e, dtype, grads, updates, scales, three);
        for (int j = 0; j < 3; ++j) list[j * N + e] = three[j];
    }
    return modse_orthogonalize(dtype, 3 * N, list, steps, coefficients, eps, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
