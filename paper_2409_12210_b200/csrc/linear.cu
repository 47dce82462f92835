// modse_linear and its gradient: host side and the elementwise part of the gradient.
#include "activations.h"
#include "dense_gemm.h"
#include "launch.h"
#include "linear_rows.h"

namespace modse {
namespace {

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Limits of the kernels' 32-bit indexes: row, column and k extents below 2^30, column extents a multiple of 8.
bool extents_ok(int T, int k, int n, int k_step)
{
    return T >= 0 && T <= (1 << 30) && k >= k_step && k % k_step == 0 && k <= (1 << 26) && n >= 8 && n % 8 == 0 && n <= (1 << 26);
}
// tiles of 256 x 128 have to be countable in 31 bits
bool countable(long long m, long long n) { return ((m + 255) / 256) * ((n + 127) / 128) < (1ll << 30); }

DenseItem forward_item(int T, int k, int n, const void *x, const void *w)
{
    DenseItem it{};
    it.a = {x, T, k, k};
    it.b = {w, n, k, k};
    it.p.M = T;
    it.p.N = n;
    it.k = k;
    return it;
}

// dx = dz w and dw = dz^T x as one launch of up to two products
int backward_items(DenseItem *items, int T, int k, int n, const void *dz, const void *x, const void *w, void *dx, void *dw)
{
    int c = 0;
    if (dx) {
        DenseItem &it = items[c++];
        it = DenseItem{};
        it.a = {dz, T, n, n};
        it.b = {w, n, k, k};
        it.p.M = T;
        it.p.N = k;
        it.p.flags = kDenseBMn;
        it.p.out0 = dx;
        it.p.ld_out = k;
        it.k = n;
    }
    if (dw) {
        DenseItem &it = items[c++];
        it = DenseItem{};
        it.a = {dz, T, n, n};
        it.b = {x, T, k, k};
        it.p.M = n;
        it.p.N = k;
        it.p.flags = kDenseAMn | kDenseBMn;
        it.p.out0 = dw;
        it.p.ld_out = k;
        it.k = T;
    }
    return c;
}

// ---- dz = dy act'(z), and the columns' sums of the unrounded dz ----
constexpr int kDzRows = 64;          // rows of a block's strip
constexpr int kDzCols = 256;         // columns of a block's strip: 32 lanes of 8, eight warps share its rows

__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

template <int ACT>
__global__ void __launch_bounds__(256)
linear_dz_kernel(const __nv_bfloat16 *dy, const __nv_bfloat16 *z, __nv_bfloat16 *dz, float *part, int *head, int T, int n)
{
    __shared__ float sh[8][kDzCols];
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (blockIdx.x == 0 && blockIdx.y == 0)      // status word and counters of the products that follow
        for (int i = threadIdx.x; i < (int)(kDenseZeroBytes / 4); i += 256) head[i] = 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * kDzCols + lane * 8, row0 = blockIdx.y * kDzRows;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    if (c < n) {
        constexpr int kAt = 4;               // rows of a warp in flight
#pragma unroll
        for (int i0 = 0; i0 < kDzRows / 8; i0 += kAt) {
            uint4 gv[kAt], fv[kAt];
#pragma unroll
            for (int i = 0; i < kAt; ++i) {
                const int r = row0 + (i0 + i) * 8 + warp;
                const size_t at = (size_t)r * n + c;
                gv[i] = fv[i] = make_uint4(0, 0, 0, 0);
                if (r < T) {
                    gv[i] = *reinterpret_cast<const uint4 *>(dy + at);
                    if constexpr (ACT != MODSE_ACT_NONE) fv[i] = *reinterpret_cast<const uint4 *>(z + at);
                }
            }
#pragma unroll
            for (int i = 0; i < kAt; ++i) {
                const int r = row0 + (i0 + i) * 8 + warp;
                float g[8], f[8];
                unpack8(gv[i], g);
                if constexpr (ACT != MODSE_ACT_NONE) {
                    unpack8(fv[i], f);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) times_slope2<ACT>(g[j], g[j + 1], f[j], f[j + 1]);
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        __nv_bfloat162 t = __floats2bfloat162_rn(g[2 * j], g[2 * j + 1]);
                        w[j] = *reinterpret_cast<uint32_t *>(&t);
                    }
                    if (r < T) *reinterpret_cast<uint4 *>(dz + (size_t)r * n + c) = make_uint4(w[0], w[1], w[2], w[3]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += g[j];      // rows past the end hold zeros
            }
        }
    }
    if (part == nullptr) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sh[warp][lane * 8 + j] = sum[j];
    __syncthreads();
    const int col = blockIdx.x * kDzCols + threadIdx.x;
    if (col < n) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += sh[w][threadIdx.x];
        part[(size_t)blockIdx.y * n + col] = t;
    }
}

// Strips of 64 rows of the dz kernel, its second grid extent: at most 65535 of them, so at most 4194240 tokens a call.
int dz_strips(int T) { return (int)(((long long)T + kDzRows - 1) / kDzRows); }

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct BackwardLayout { size_t partials, partial_bytes, dz, part, total; };
BackwardLayout backward_layout(int T, int k, int n)
{
    BackwardLayout L{};
    DenseItem items[2];
    size_t need = 0;
    for (int which = 1; which <= 3; ++which) {        // dx alone, dw alone, both: the largest of the three
        const int c = backward_items(items, T, k, n, nullptr, nullptr, nullptr, (which & 1) ? (void *)1 : nullptr,
                                     (which & 2) ? (void *)1 : nullptr);
        const size_t b = dense_partial_bound(DenseBf16, items, c);
        need = b > need ? b : need;
    }
    L.partials = kDenseHead;
    L.partial_bytes = need;
    L.dz = up256(L.partials + need);
    L.part = up256(L.dz + (size_t)T * n * 2);
    L.total = up256(L.part + (size_t)dz_strips(T) * n * 4);
    return L;
}

cudaError_t launch_dz(int act, const void *dy, const void *z, void *dz, float *part, int *head, int T, int n, cudaStream_t s)
{
    const dim3 grid((n + kDzCols - 1) / kDzCols, dz_strips(T));
    const auto *g = (const __nv_bfloat16 *)dy, *f = (const __nv_bfloat16 *)z;
    auto *o = (__nv_bfloat16 *)dz;
    switch (act) {
    case MODSE_ACT_RELU: return launch_overlapped(linear_dz_kernel<MODSE_ACT_RELU>, grid, 256, 0, s, g, f, o, part, head, T, n);
    case MODSE_ACT_GELU: return launch_overlapped(linear_dz_kernel<MODSE_ACT_GELU>, grid, 256, 0, s, g, f, o, part, head, T, n);
    case MODSE_ACT_SILU: return launch_overlapped(linear_dz_kernel<MODSE_ACT_SILU>, grid, 256, 0, s, g, f, o, part, head, T, n);
    default: return launch_overlapped(linear_dz_kernel<MODSE_ACT_NONE>, grid, 256, 0, s, g, f, o, part, head, T, n);
    }
}

}  // namespace

void clear_workspace_status(void *workspace, size_t workspace_bytes, cudaStream_t s)
{
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < sizeof(int)) return;
    if (cudaMemsetAsync(workspace, 0, sizeof(int), s) != cudaSuccess) (void)cudaGetLastError();
}

}  // namespace modse

using namespace modse;

#define MODSE_CUDA(expr)                                \
    do {                                                \
        if ((expr) != cudaSuccess) return MODSE_ERR_CUDA; \
    } while (0)

extern "C" {

size_t modse_linear_workspace_bytes(modse_dtype_t dtype, int n_tokens, int d_in, int d_out)
{
    if ((dtype != MODSE_BF16 && dtype != MODSE_E4M3) || !extents_ok(n_tokens, d_in, d_out, dtype == MODSE_E4M3 ? 16 : 8) ||
        !countable(n_tokens, d_out))
        return 0;
    const DenseType type = dtype == MODSE_E4M3 ? DenseE4m3 : DenseBf16;
    if (n_tokens <= kLinearRowsMax) return kDenseHead;
    const DenseItem it = forward_item(n_tokens, d_in, d_out, nullptr, nullptr);
    return kDenseHead + up256(dense_partial_bound(type, &it, 1));
}

modse_status_t modse_linear(modse_dtype_t dtype, int n_tokens, int d_in, int d_out, modse_activation_t activation,
                            const modse_linear_t *args, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (dtype == MODSE_F32) return MODSE_ERR_UNSUPPORTED;
    if (args == nullptr || activation < MODSE_ACT_NONE || activation > MODSE_ACT_SILU) return MODSE_ERR_INVALID_ARG;
    const size_t need = modse_linear_workspace_bytes(dtype, n_tokens, d_in, d_out);
    if (need == 0) return MODSE_ERR_INVALID_ARG;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, (cudaStream_t)cuda_stream);
        return MODSE_OK;
    }
    const modse_linear_t &a = *args;
    if (a.x == nullptr || a.w == nullptr || a.y == nullptr || !aligned(a.x, 16) || !aligned(a.w, 16) || !aligned(a.bias, 16) ||
        !aligned(a.residual, 16) || !aligned(a.z, 16) || !aligned(a.y, 16))
        return MODSE_ERR_INVALID_ARG;
    const bool f8 = dtype == MODSE_E4M3;
    if (f8 != (a.x_scale != nullptr) || f8 != (a.w_scale != nullptr) || !aligned(a.x_scale, 4) || !aligned(a.w_scale, 16))
        return MODSE_ERR_INVALID_ARG;
    if (workspace == nullptr || !aligned(workspace, 256)) return MODSE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const DenseType type = f8 ? DenseE4m3 : DenseBf16;
    const LinearEpilogue lin{a.x_scale, a.w_scale, (const __nv_bfloat16 *)a.bias, (const __nv_bfloat16 *)a.residual,
                             (__nv_bfloat16 *)a.z, (__nv_bfloat16 *)a.y, (int)activation};
    if (n_tokens <= kLinearRowsMax) {
        MODSE_CUDA(launch_linear_rows(type, a.x, a.w, n_tokens, d_in, d_out, lin, (int *)workspace, s));
        return MODSE_OK;
    }
    const DenseItem it = forward_item(n_tokens, d_in, d_out, a.x, a.w);
    MODSE_CUDA(dense_launch(DenseLinear, type, &it, 1, &lin, nullptr, workspace, need - kDenseHead, kDenseHeadRaw, s));
    return MODSE_OK;
}

size_t modse_linear_backward_workspace_bytes(int n_tokens, int d_in, int d_out)
{
    if (!extents_ok(n_tokens, d_in, d_out, 8) || !countable(n_tokens, d_in) || !countable(d_out, d_in) ||
        dz_strips(n_tokens) > 65535)
        return 0;
    return backward_layout(n_tokens, d_in, d_out).total;
}

modse_status_t modse_linear_backward(int n_tokens, int d_in, int d_out, modse_activation_t activation,
                                     const modse_linear_grads_t *args, void *workspace, size_t workspace_bytes,
                                     void *cuda_stream)
{
    if (args == nullptr || activation < MODSE_ACT_NONE || activation > MODSE_ACT_SILU) return MODSE_ERR_INVALID_ARG;
    const size_t need = modse_linear_backward_workspace_bytes(n_tokens, d_in, d_out);
    if (need == 0) return MODSE_ERR_INVALID_ARG;
    const modse_linear_grads_t &a = *args;
    if (!aligned(a.dw, 16) || !aligned(a.dbias, 4)) return MODSE_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, s);
        if (a.dw) MODSE_CUDA(cudaMemsetAsync(a.dw, 0, (size_t)d_out * d_in * 2, s));
        if (a.dbias) MODSE_CUDA(cudaMemsetAsync(a.dbias, 0, (size_t)d_out * 4, s));
        return MODSE_OK;
    }
    if (a.dx == nullptr && a.dw == nullptr && a.dbias == nullptr) return MODSE_ERR_INVALID_ARG;
    if (a.dy == nullptr || !aligned(a.dy, 16) || !aligned(a.dx, 16)) return MODSE_ERR_INVALID_ARG;
    if (activation != MODSE_ACT_NONE && (a.z == nullptr || !aligned(a.z, 16))) return MODSE_ERR_INVALID_ARG;
    if ((a.dx && (a.w == nullptr || !aligned(a.w, 16))) || (a.dw && (a.x == nullptr || !aligned(a.x, 16))))
        return MODSE_ERR_INVALID_ARG;
    if (workspace == nullptr || !aligned(workspace, 256)) return MODSE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    const BackwardLayout L = backward_layout(n_tokens, d_in, d_out);
    unsigned char *ws = (unsigned char *)workspace;
    const void *dz = a.dy;
    float *part = a.dbias ? (float *)(ws + L.part) : nullptr;
    int head = kDenseHeadRaw;
    if (activation != MODSE_ACT_NONE || part) {
        MODSE_CUDA(launch_dz((int)activation, a.dy, a.z, ws + L.dz, part, (int *)ws, n_tokens, d_out, s));
        head = kDenseHeadZero;
        if (activation != MODSE_ACT_NONE) dz = ws + L.dz;
    }
    DenseItem items[2];
    const int c = backward_items(items, n_tokens, d_in, d_out, dz, a.x, a.w, a.dx, a.dw);
    const DenseColumnSum sum{part, a.dbias, dz_strips(n_tokens), d_out};
    if (c > 0)
        MODSE_CUDA(dense_launch(DensePlain, DenseBf16, items, c, nullptr, part ? &sum : nullptr, workspace, L.partial_bytes, head, s));
    else if (part)
        MODSE_CUDA(launch_column_sum(part, dz_strips(n_tokens), d_out, a.dbias, s));
    return MODSE_OK;
}

modse_status_t modse_check_workspace_status(const void *workspace, void *cuda_stream)
{
    if (workspace == nullptr) return MODSE_ERR_INVALID_ARG;
    int word = 0;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    MODSE_CUDA(cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, s));
    MODSE_CUDA(cudaStreamSynchronize(s));
    return word == kDevOk ? MODSE_OK : word == kDevTimeout ? MODSE_ERR_DEVICE_TIMEOUT : MODSE_ERR_DEVICE_BOUNDS;
}

}  // extern "C"
