// Residual addition with root-mean-square norm, forward (16/32-bit rows and 8-bit rows with a scale a row) and backward.
//
//   s = x + r;  rstd = 1 / sqrt(mean_c s_c^2 + eps);  y_c = s_c rstd w_c;  scale = max_c |y_c| / 448;  q_c = e4m3(y_c / scale)
//   backward, with u = dy w:  dx = rstd (u - s rstd^2 mean_c(u_c s_c)) + dsum;   dw_c = sum_t dy_tc s_tc rstd_t
//
// Both passes are bound by HBM: a row is read once, held in registers while its sums are formed, and written once.
// "Vector" below: 8 consecutive elements of a row (16 bytes of bf16, 32 of fp32).  A row belongs to TPR threads of a
// block, VPT vectors each; the choice of (TPR, VPT) is in pick_shape.  All sums are fp32 of fp32 terms.
#include <cuda_fp8.h>

#include "f32x2.h"
#include "launch.h"
#include "modse_internal.h"

namespace modse {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr int kNormBlock = 256;
constexpr int kNormMaxD = 32768;

template <typename T> struct Vec;                      // 8 elements as they lie in memory
template <> struct Vec<__nv_bfloat16> { uint4 a; };
template <> struct Vec<float> { float4 a, b; };

__device__ __forceinline__ void load_vec(Vec<__nv_bfloat16> &v, const __nv_bfloat16 *p) { v.a = *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void load_vec(Vec<float> &v, const float *p)
{
    v.a = *reinterpret_cast<const float4 *>(p);
    v.b = *reinterpret_cast<const float4 *>(p + 4);
}
__device__ __forceinline__ void zero_vec(Vec<__nv_bfloat16> &v) { v.a = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void zero_vec(Vec<float> &v) { v.a = v.b = make_float4(0, 0, 0, 0); }
__device__ __forceinline__ void unpack(const Vec<__nv_bfloat16> &v, float (&f)[8])
{
    const uint32_t w[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const Vec<float> &v, float (&f)[8])
{
    f[0] = v.a.x; f[1] = v.a.y; f[2] = v.a.z; f[3] = v.a.w;
    f[4] = v.b.x; f[5] = v.b.y; f[6] = v.b.z; f[7] = v.b.w;
}
__device__ __forceinline__ void store_vec(__nv_bfloat16 *p, const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&t);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_vec(float *p, const float (&f)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sums of two numbers over a warp with six exchanges instead of ten: the half-warps trade one number each, then every half
// sums its own.
__device__ __forceinline__ void warp_sum2(float &a, float &b)
{
    const bool upper = (threadIdx.x & 16) != 0;
    float v = (upper ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    const float other = __shfl_xor_sync(0xFFFFFFFFu, v, 16);
    a = upper ? other : v;
    b = upper ? v : other;
}

// Sum over the TPR threads of a row (every one of them gets it; fixed order).  `slot`: this row's TPR / 32 words.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *slot)
{
    v = warp_sum(v);
    if constexpr (TPR == 32) return v;
    constexpr int W = TPR / 32;
    const int w = (threadIdx.x % TPR) >> 5;
    if ((threadIdx.x & 31) == 0) slot[w] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) s += slot[i];
    return s;
}
template <int TPR>
__device__ __forceinline__ unsigned row_max(unsigned v, unsigned *slot)
{
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if constexpr (TPR == 32) return v;
    constexpr int W = TPR / 32;
    const int w = (threadIdx.x % TPR) >> 5;
    if ((threadIdx.x & 31) == 0) slot[w] = v;
    __syncthreads();
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) m = max(m, slot[i]);
    return m;
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    unsigned char *q;
    float *q_scale;
    int T, d;
    float eps;
};

template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR < kNormBlock ? kNormBlock : TPR)
add_rms_norm_kernel(const NormArgs a)
{
    constexpr int kThreads = TPR < kNormBlock ? kNormBlock : TPR;
    constexpr int kRows = kThreads / TPR;
    __shared__ float sums[kThreads / 32];
    __shared__ unsigned maxs[kThreads / 32];
    const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR;
    const int row = blockIdx.x * kRows + group;
    const bool live = row < a.T;                  // rows past the end take part in the barriers and touch no memory
    wait_for_earlier_kernels();
    allow_next_kernel();
    const int nv = a.d / 8;
    const size_t base = (size_t)(live ? row : 0) * a.d;
    Vec<T> xv[VPT], rv[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * TPR;
        if (live && v < nv) {
            load_vec(xv[i], (const T *)a.x + base + 8 * (size_t)v);
            if (a.residual) load_vec(rv[i], (const T *)a.residual + base + 8 * (size_t)v);
            else zero_vec(rv[i]);
        } else {
            zero_vec(xv[i]);
            zero_vec(rv[i]);
        }
    }
    float s[VPT][8];
    float acc = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float f[8];
        unpack(xv[i], s[i]);
        unpack(rv[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (a.residual) s[i][j] += f[j];      // (-0) + (+0) would lose the sign of a zero where there is no residual
            acc = fmaf(s[i][j], s[i][j], acc);
        }
        const int v = lane + i * TPR;
        if (a.sum && live && v < nv) store_vec((T *)a.sum + base + 8 * (size_t)v, s[i]);
    }
    if (a.y == nullptr && a.q == nullptr) return;
    const float total = row_sum<TPR>(acc, sums + group * (TPR / 32));
    const float rstd = 1.f / sqrtf(total / (float)a.d + a.eps);
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * TPR;
        if (v >= nv) continue;
        float w[8];
        Vec<T> wv;
        if (a.weight) load_vec(wv, (const T *)a.weight + 8 * v);
        if (a.weight) unpack(wv, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[i][j] = a.weight ? s[i][j] * rstd * w[j] : s[i][j] * rstd;
            top = max(top, __float_as_uint(s[i][j]) & 0x7FFFFFFFu);   // ordered like |y|, a NaN above all numbers
        }
        if (a.y && live) store_vec((T *)a.y + base + 8 * (size_t)v, s[i]);
    }
    if (a.q == nullptr) return;
    const float scale = __uint_as_float(row_max<TPR>(top, maxs + group * (TPR / 32))) / kE4m3Max;
    // one reciprocal a row; where it would overflow (a scale below the normal range) the division itself is used
    const bool tiny = scale < 1.17549435e-38f;
    const float inv = tiny ? 0.f : 1.f / scale;
    if (live && lane == 0) a.q_scale[row] = scale;
    if (tiny) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] = scale > 0.f ? s[i][j] / scale : 0.f;
    }
    const float by = tiny ? 1.f : inv;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * TPR;
        if (!live || v >= nv) continue;
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = s[i][4 * h + j] * by;
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(t[0], t[1]), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(t[2], t[3]), __NV_SATFINITE, __NV_E4M3);
            w[h] = lo | (hi << 16);
        }
        *reinterpret_cast<uint2 *>(a.q + base + 8 * (size_t)v) = make_uint2(w[0], w[1]);
    }
}

struct NormBwdArgs {
    const void *s, *weight, *dy, *dsum;
    void *dx;
    float *dw_part;          // [blocks][d]
    int T, d;
    float eps;
};

__device__ __forceinline__ void cp_async16(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The elements of a vector as four pairs, and back.
__device__ __forceinline__ void pairs(const Vec<__nv_bfloat16> &v, f32x2 (&f)[4])
{
    const uint32_t w[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void pairs(const Vec<float> &v, f32x2 (&f)[4])
{
    f[0] = pack2(v.a.x, v.a.y);
    f[1] = pack2(v.a.z, v.a.w);
    f[2] = pack2(v.b.x, v.b.y);
    f[3] = pack2(v.b.z, v.b.w);
}
template <typename T>
__device__ __forceinline__ void store_pairs(T *p, const f32x2 (&f)[4])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(f[i], v[2 * i], v[2 * i + 1]);
    store_vec(p, v);
}

// TPR threads of a 512-thread block share a row, VPT vectors each.  Every thread keeps a ring of two rows' pieces (s, dy,
// dsum) in shared memory, filled by cp.async one row ahead, so that HBM is busy while a row's two sums and its dx are
// formed; it reads back only the pieces it copied itself, so the only meeting is that of the row's warps over the sums (a
// named barrier; none where the row is one warp's).  dweight sums stay in registers (VPT * 8 <= 32) and meet in shared
// memory at the end, in the order of the row groups.
// Rows too long for the ring (1024 threads a row) are read from global memory twice instead, the second time
// from L2.
constexpr int kSlots = 2;
template <typename T, int TPR, int VPT, bool WEIGHT, bool SUM>
__global__ void __launch_bounds__(TPR == 1024 ? 1024 : 512, 1)
add_rms_norm_bwd_kernel(const NormBwdArgs a)
{
    constexpr bool RING = TPR != 1024;
    extern __shared__ unsigned char ring[];
    constexpr int kBwdThreads = RING ? 512 : 1024;
    constexpr int kGroups = kBwdThreads / TPR, W = TPR / 32, kPieces = sizeof(T) / 2;      // 16-byte pieces of a vector
    __shared__ float2 part[2][kBwdThreads / 32];
    const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR, warp = threadIdx.x >> 5, nv = a.d / 8;
    // ring: [slot][tensor][vector][piece] of 16 bytes a thread, neighbouring threads side by side
    unsigned char *mine = ring + threadIdx.x * 16;
    auto piece = [&](int slot, int tensor, int i, int h) -> unsigned char * {
        return mine + (size_t)(((slot * 3 + tensor) * VPT + i) * kPieces + h) * (kBwdThreads * 16);
    };
    int row = blockIdx.x * kGroups + group, slot = 0;
    auto fetch = [&](int slot, int tensor, int i, Vec<T> &v) {
        if constexpr (!RING) {
            const T *src = (const T *)(tensor == 0 ? a.s : tensor == 1 ? a.dy : a.dsum);
            load_vec(v, src + (size_t)row * a.d + 8 * (lane + TPR * i));
        } else if constexpr (kPieces == 1) {
            v.a = *reinterpret_cast<const uint4 *>(piece(slot, tensor, i, 0));
        } else {
            v.a = *reinterpret_cast<const float4 *>(piece(slot, tensor, i, 0));
            v.b = *reinterpret_cast<const float4 *>(piece(slot, tensor, i, 1));
        }
    };
    const int stride = gridDim.x * kGroups;
    auto issue = [&](int row, int slot) {
        if constexpr (!RING) return;
        if (row < a.T) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int v = lane + TPR * i;
                if (v < nv) {
                    const size_t at = ((size_t)row * a.d + 8 * (size_t)v) * sizeof(T);
#pragma unroll
                    for (int h = 0; h < kPieces; ++h) {
                        cp_async16(piece(slot, 0, i, h), (const unsigned char *)a.s + at + 16 * h);
                        cp_async16(piece(slot, 1, i, h), (const unsigned char *)a.dy + at + 16 * h);
                        if constexpr (SUM) cp_async16(piece(slot, 2, i, h), (const unsigned char *)a.dsum + at + 16 * h);
                    }
                }
            }
        }
        cp_async_commit();
    };
    f32x2 dw[VPT][4];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = 0;
    wait_for_earlier_kernels();
    allow_next_kernel();
    issue(row, 0);
    const float inv_d = 1.f / (float)a.d;
    for (; row < a.T; row += stride, slot ^= 1) {
        issue(row + stride, slot ^ 1);
        if constexpr (RING) cp_async_wait<1>();
        Vec<T> sv[VPT], yv[VPT];
        f32x2 ss2 = 0, us2 = 0;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = lane + TPR * i;
            if (v >= nv) continue;
            fetch(slot, 0, i, sv[i]);
            fetch(slot, 1, i, yv[i]);
            f32x2 f[4], g[4], w[4];
            pairs(sv[i], f);
            pairs(yv[i], g);
            if constexpr (WEIGHT) {
                Vec<T> wv;
                load_vec(wv, (const T *)a.weight + 8 * v);
                pairs(wv, w);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                ss2 = fma2(f[j], f[j], ss2);
                us2 = fma2(WEIGHT ? mul2(g[j], w[j]) : g[j], f[j], us2);
            }
        }
        float ss, us, t0, t1;
        unpack2(ss2, t0, t1);
        ss = t0 + t1;
        unpack2(us2, t0, t1);
        us = t0 + t1;
        warp_sum2(ss, us);
        if constexpr (W > 1) {
            // the buffers alternate: nobody writes one again before the group's next barrier
            if ((threadIdx.x & 31) == 0) part[slot][warp] = make_float2(ss, us);
            asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
            ss = us = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 p = part[slot][group * W + i];
                ss += p.x;
                us += p.y;
            }
        }
        const float rstd = rsqrtf(ss * inv_d + a.eps);       // within two units of the last place
        const f32x2 rstd2 = both(rstd), minus_c = both(-rstd * rstd * (us * inv_d));
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = lane + TPR * i;
            if (v >= nv) continue;
            f32x2 f[4], g[4], w[4], add[4], o[4];
            if constexpr (!RING) {
                fetch(slot, 0, i, sv[i]);
                fetch(slot, 1, i, yv[i]);
            }
            pairs(sv[i], f);
            pairs(yv[i], g);
            if constexpr (WEIGHT) {
                Vec<T> wv;
                load_vec(wv, (const T *)a.weight + 8 * v);
                pairs(wv, w);
            }
            if constexpr (SUM) {
                Vec<T> av;
                fetch(slot, 2, i, av);
                pairs(av, add);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 t = fma2(f[j], minus_c, WEIGHT ? mul2(g[j], w[j]) : g[j]);
                o[j] = SUM ? fma2(rstd2, t, add[j]) : mul2(rstd2, t);
                dw[i][j] = fma2(g[j], mul2(f[j], rstd2), dw[i][j]);
            }
            store_pairs((T *)a.dx + (size_t)row * a.d + 8 * (size_t)v, o);
        }
    }
    if (a.dw_part == nullptr) return;
    if constexpr (RING) cp_async_wait<0>();
    __syncthreads();
    float *out = a.dw_part + (size_t)blockIdx.x * a.d;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (lane + TPR * i < nv) store_pairs(out + 8 * (lane + TPR * i), dw[i]);
    } else {
        // the row groups' sums meet in the ring's memory and are added in group order
        float *acc = reinterpret_cast<float *>(ring);
        constexpr int kRow = TPR * VPT * 8;
#pragma unroll
        for (int i = 0; i < VPT; ++i) store_pairs(acc + group * kRow + 8 * (lane + TPR * i), dw[i]);
        __syncthreads();
        for (int c = 4 * threadIdx.x; c < a.d; c += 4 * kBwdThreads) {
            float4 t = *reinterpret_cast<const float4 *>(acc + c);
#pragma unroll
            for (int g = 1; g < kGroups; ++g) {
                const float4 f = *reinterpret_cast<const float4 *>(acc + g * kRow + c);
                t.x += f.x; t.y += f.y; t.z += f.z; t.w += f.w;
            }
            *reinterpret_cast<float4 *>(out + c) = t;
        }
    }
}

// out[c] = sum over the blocks' partial rows, in block order within 32 interleaved runs that are added in order.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float *part, int n_rows, int d, float *out)
{
    __shared__ float sh[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
    float acc = 0.f;
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (c < d)
#pragma unroll 8
        for (int r = run; r < n_rows; r += 32) acc += part[(size_t)r * d + c];
    sh[run][threadIdx.x & 31] = acc;
    __syncthreads();
    if (run == 0 && c < d) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sh[i][threadIdx.x];
        out[c] = t;
    }
}

template <typename T, int TPR, int VPT>
cudaError_t launch_norm(const NormArgs &a, cudaStream_t s)
{
    constexpr int threads = TPR < kNormBlock ? kNormBlock : TPR;
    constexpr int rows = threads / TPR;
    return launch_overlapped(add_rms_norm_kernel<T, TPR, VPT>, (a.T + rows - 1) / rows, threads, 0, s, a);
}

// Few rows: a row's latency counts, so it is spread over a block with one vector a thread where that holds it.
// Many rows: a warp a row as long as it fits in registers (no barrier in the row's sums).
template <typename T>
cudaError_t dispatch_norm(const NormArgs &a, int sms, cudaStream_t s)
{
    const int nv = a.d / 8;
    if (nv <= 32) return launch_norm<T, 32, 1>(a, s);
    if (a.T <= 2 * sms && nv <= 256) return launch_norm<T, 256, 1>(a, s);
    if (nv <= 64) return launch_norm<T, 32, 2>(a, s);
    if (nv <= 128) return launch_norm<T, 32, 4>(a, s);
    if (nv <= 256) return launch_norm<T, 32, 8>(a, s);
    if (nv <= 512) return launch_norm<T, 256, 2>(a, s);
    if (nv <= 1024) return launch_norm<T, 256, 4>(a, s);
    if (nv <= 2048) return launch_norm<T, 256, 8>(a, s);
    return launch_norm<T, 1024, 4>(a, s);
}

// Threads a row and vectors a thread of the backward kernel; its ring holds 2 x 3 x VPT vectors a thread.
constexpr int kBwdThreads = 512;
struct BwdShape { int tpr, vpt; };
BwdShape bwd_shape(int d, int esz)
{
    const int nv = d / 8, most = esz == 2 ? 4 : 2;      // vectors a thread that fit the ring
    int tpr = 32;
    while (tpr < kBwdThreads && tpr * most < nv) tpr *= 2;
    if (tpr * most < nv) return {1024, 4};              // no ring
    int vpt = 1;
    while (vpt * tpr < nv) vpt *= 2;
    return {tpr, vpt};
}
// Blocks for a batch: the partial dweight rows they write are part of the workspace, whose size is asked for without a
// device or a type, so the count goes by the batch and the longer of the types' rows alone (148 SMs).
int bwd_blocks(int T, int d)
{
    const int tpr = bwd_shape(d, 4).tpr;
    const long long groups = tpr < kBwdThreads ? kBwdThreads / tpr : 1, need = ((long long)T + groups - 1) / groups;
    return (int)(need < 148 ? need : 148);
}

template <typename T, int TPR, int VPT, bool WEIGHT, bool SUM>
cudaError_t launch_bwd_form(const NormBwdArgs &a, int blocks, cudaStream_t s)
{
    auto kern = add_rms_norm_bwd_kernel<T, TPR, VPT, WEIGHT, SUM>;
    constexpr int threads = TPR == 1024 ? 1024 : kBwdThreads;
    constexpr int smem = TPR == 1024 ? 0 : kBwdThreads * kSlots * 3 * VPT * 8 * (int)sizeof(T);
    static unsigned long long attr_done = 0;      // bit per device ordinal (devices beyond 63 set it every time)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (smem > 0 && (dev > 63 || !((attr_done >> dev) & 1ull))) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev <= 63) attr_done |= 1ull << dev;
    }
    return launch_overlapped(kern, blocks, threads, smem, s, a);
}
template <typename T, int TPR, int VPT>
cudaError_t launch_bwd(const NormBwdArgs &a, int blocks, cudaStream_t s)
{
    if (a.weight) return a.dsum ? launch_bwd_form<T, TPR, VPT, true, true>(a, blocks, s) : launch_bwd_form<T, TPR, VPT, true, false>(a, blocks, s);
    return a.dsum ? launch_bwd_form<T, TPR, VPT, false, true>(a, blocks, s) : launch_bwd_form<T, TPR, VPT, false, false>(a, blocks, s);
}
template <typename T>
cudaError_t dispatch_bwd(const NormBwdArgs &a, int blocks, cudaStream_t s)
{
    const BwdShape b = bwd_shape(a.d, (int)sizeof(T));
    if constexpr (sizeof(T) == 2) {
        switch (b.tpr * 8 + b.vpt) {
        case 32 * 8 + 1: return launch_bwd<T, 32, 1>(a, blocks, s);
        case 32 * 8 + 2: return launch_bwd<T, 32, 2>(a, blocks, s);
        case 32 * 8 + 4: return launch_bwd<T, 32, 4>(a, blocks, s);
        case 64 * 8 + 4: return launch_bwd<T, 64, 4>(a, blocks, s);
        case 128 * 8 + 4: return launch_bwd<T, 128, 4>(a, blocks, s);
        case 256 * 8 + 4: return launch_bwd<T, 256, 4>(a, blocks, s);
        case 512 * 8 + 4: return launch_bwd<T, 512, 4>(a, blocks, s);
        case 1024 * 8 + 4: return launch_bwd<T, 1024, 4>(a, blocks, s);
        }
    } else {
        switch (b.tpr * 8 + b.vpt) {
        case 32 * 8 + 1: return launch_bwd<T, 32, 1>(a, blocks, s);
        case 32 * 8 + 2: return launch_bwd<T, 32, 2>(a, blocks, s);
        case 64 * 8 + 2: return launch_bwd<T, 64, 2>(a, blocks, s);
        case 128 * 8 + 2: return launch_bwd<T, 128, 2>(a, blocks, s);
        case 256 * 8 + 2: return launch_bwd<T, 256, 2>(a, blocks, s);
        case 512 * 8 + 2: return launch_bwd<T, 512, 2>(a, blocks, s);
        case 1024 * 8 + 4: return launch_bwd<T, 1024, 4>(a, blocks, s);
        }
    }
    return cudaErrorInvalidValue;
}

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool norm_shape_ok(int T, int d) { return T >= 0 && T <= (1 << 30) && d >= 8 && d % 8 == 0; }

}  // namespace

int device_sms()
{
    static int cached[64];                         // by device ordinal; a lost race writes the same value
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (dev >= 0 && dev < 64 && cached[dev] > 0) return cached[dev];
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
    if (dev >= 0 && dev < 64) cached[dev] = n;
    return n;
}

cudaError_t launch_column_sum(const float *part, int n_rows, int d, float *out, cudaStream_t s)
{
    return launch_overlapped(column_sum_kernel, (d + 31) / 32, 1024, 0, s, part, n_rows, d, out);
}

}  // namespace modse

using namespace modse;

extern "C" {

modse_status_t modse_add_rms_norm(modse_dtype_t dtype, int n_tokens, int d_model, const void *x, const void *residual,
                                  const void *weight, float eps, void *sum, void *y, void *y_e4m3, float *y_scale,
                                  void *cuda_stream)
{
    if ((dtype != MODSE_F32 && dtype != MODSE_BF16) || !norm_shape_ok(n_tokens, d_model) || !(eps >= 0.f) || eps > 3e38f)
        return MODSE_ERR_INVALID_ARG;
    if (d_model > kNormMaxD) return MODSE_ERR_UNSUPPORTED;
    if (n_tokens == 0) return MODSE_OK;
    if (sum == nullptr && y == nullptr && y_e4m3 == nullptr) return MODSE_ERR_INVALID_ARG;
    if ((y_e4m3 == nullptr) != (y_scale == nullptr)) return MODSE_ERR_INVALID_ARG;
    if (x == nullptr || !aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16) || !aligned(sum, 16) ||
        !aligned(y, 16) || !aligned(y_e4m3, 16) || !aligned(y_scale, 4))
        return MODSE_ERR_INVALID_ARG;
    const NormArgs a{x, residual, weight, sum, y, (unsigned char *)y_e4m3, y_scale, n_tokens, d_model, eps};
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == MODSE_F32 ? dispatch_norm<float>(a, device_sms(), s)
                                             : dispatch_norm<__nv_bfloat16>(a, device_sms(), s);
    return e == cudaSuccess ? MODSE_OK : MODSE_ERR_CUDA;
}

size_t modse_add_rms_norm_backward_workspace_bytes(int n_tokens, int d_model)
{
    if (!norm_shape_ok(n_tokens, d_model) || d_model > kNormMaxD) return 0;
    return (size_t)bwd_blocks(n_tokens > 0 ? n_tokens : 1, d_model) * d_model * sizeof(float);
}

modse_status_t modse_add_rms_norm_backward(modse_dtype_t dtype, int n_tokens, int d_model, const void *sum,
                                           const void *weight, float eps, const void *dy, const void *dsum, void *dx,
                                           float *dweight, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if ((dtype != MODSE_F32 && dtype != MODSE_BF16) || !norm_shape_ok(n_tokens, d_model) || !(eps >= 0.f) || eps > 3e38f)
        return MODSE_ERR_INVALID_ARG;
    if (d_model > kNormMaxD) return MODSE_ERR_UNSUPPORTED;
    if (!aligned(dweight, 16)) return MODSE_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (n_tokens == 0) {
        if (dweight && cudaMemsetAsync(dweight, 0, (size_t)d_model * sizeof(float), s) != cudaSuccess) return MODSE_ERR_CUDA;
        return MODSE_OK;
    }
    if (sum == nullptr || dy == nullptr || dx == nullptr || !aligned(sum, 16) || !aligned(weight, 16) || !aligned(dy, 16) ||
        !aligned(dsum, 16) || !aligned(dx, 16))
        return MODSE_ERR_INVALID_ARG;
    if (dweight != nullptr) {
        if (workspace == nullptr || !aligned(workspace, 256)) return MODSE_ERR_INVALID_ARG;
        if (workspace_bytes < modse_add_rms_norm_backward_workspace_bytes(n_tokens, d_model))
            return MODSE_ERR_WORKSPACE_TOO_SMALL;
    }
    const int blocks = bwd_blocks(n_tokens, d_model);
    const NormBwdArgs a{sum, weight, dy, dsum, dx, dweight ? (float *)workspace : nullptr, n_tokens, d_model, eps};
    cudaError_t e = dtype == MODSE_F32 ? dispatch_bwd<float>(a, blocks, s) : dispatch_bwd<__nv_bfloat16>(a, blocks, s);
    if (e == cudaSuccess && dweight) e = launch_column_sum(a.dw_part, blocks, d_model, dweight, s);
    return e == cudaSuccess ? MODSE_OK : MODSE_ERR_CUDA;
}

}  // extern "C"
