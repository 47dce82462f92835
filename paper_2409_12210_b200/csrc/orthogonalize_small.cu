// Orthogonalised updates of matrices whose shorter side is at most 128: the whole iteration in one kernel.
//
// As grouped products such a matrix is seventeen launches that each last a few microseconds and compute for less than
// one.  Here a block - or a cluster of up to eight blocks that split the longer side - keeps X (hi and lo, fp16) in shared
// memory for all iterations and multiplies with mma.sync.  Per iteration:
//   A = X X^T    every block over its own columns; blocks of a cluster leave fp32 partial sums in their shared memory and
//                each adds up (in block order) and hands out its share of A through distributed shared memory;
//   B = aI + bA + cA^2  computed by every block for itself (a 128 x 128 product is cheaper than another meeting);
//   X <- B hi + a lo   every block on its own columns.
// The roundings are those of the grouped form (orthogonalize.cu): fp16 factors scaled by powers of two, X in 22 bits.
// A tall matrix is transposed on its way in and out.
#include <cuda_fp16.h>

#include "launch.h"
#include "orthogonalize_small.h"
#include "tc_device.h"

namespace modse {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr size_t kSmemMost = 227 * 1024 - 1024;       // dynamic; the static part stays below 1 KB

__host__ __device__ inline int up16(int v) { return (v + 15) / 16 * 16; }

// Shared memory of a block for n rows (a multiple of 16) and per columns: rows are padded by 16 bytes, so that eight
// consecutive rows of a matrix load fall into different banks.
struct SmallLayout {
    int xs, as;                         // row lengths in halves
    size_t hi0, hi1, lo, a, b, part, total;
};
__host__ __device__ inline SmallLayout small_layout(int n, int per, bool cluster)
{
    SmallLayout L;
    L.xs = per + 8;
    L.as = n + 8;
    const size_t x = (size_t)n * L.xs * 2, q = (size_t)n * L.as * 2;
    L.hi0 = 0;
    L.hi1 = x;
    L.lo = 2 * x;
    L.a = 3 * x;
    L.b = L.a + q;
    L.part = L.b + q;
    L.total = L.part + (cluster ? (size_t)n * n * 4 : 0);
    return L;
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 x 16 block (i0, j0) of P Q^T, P and Q row-major with row lengths ps, qs (halves), k a multiple of 16.
// acc[0]: columns j0 .. j0+7, acc[1]: the next eight.
__device__ __forceinline__ void block_nt(float (&acc)[2][4], uint32_t p, int ps, uint32_t q, int qs, int i0, int j0, int k, int lane)
{
    // matrices of a load: rows 0-7 / 8-15 at k 0-7, then the same rows at k 8-15
    const uint32_t pa = p + (uint32_t)((i0 + (lane & 15)) * ps + (lane >> 4) * 8) * 2;
    // for Q: rows 0-7 at k 0-7, rows 0-7 at k 8-15, rows 8-15 at k 0-7, rows 8-15 at k 8-15
    const uint32_t qa = q + (uint32_t)((j0 + (lane & 7) + ((lane >> 4) << 3)) * qs + ((lane >> 3) & 1) * 8) * 2;
#pragma unroll 4
    for (int kk = 0; kk < k; kk += 16) {
        uint32_t a[4], b[4];
        ldsm4(a, pa + kk * 2);
        ldsm4(b, qa + kk * 2);
        mma_f16(acc[0], a, b[0], b[1]);
        mma_f16(acc[1], a, b[2], b[3]);
    }
}
// 16 x 16 block (i0, j0) of P Q, Q [k][columns] row-major.
__device__ __forceinline__ void block_nn(float (&acc)[2][4], uint32_t p, int ps, uint32_t q, int qs, int i0, int j0, int k, int lane)
{
    const uint32_t pa = p + (uint32_t)((i0 + (lane & 15)) * ps + (lane >> 4) * 8) * 2;
    // transposed loads: k rows 0-7 / 8-15 at columns 0-7, then at columns 8-15
    const uint32_t qa = q + (uint32_t)((lane & 15) * qs + j0 + (lane >> 4) * 8) * 2;
#pragma unroll 4
    for (int kk = 0; kk < k; kk += 16) {
        uint32_t a[4], b[4];
        ldsm4(a, pa + kk * 2);
        ldsm4_t(b, qa + (uint32_t)(kk * qs) * 2);
        mma_f16(acc[0], a, b[0], b[1]);
        mma_f16(acc[1], a, b[2], b[3]);
    }
}

__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_u2(uint32_t addr, uint32_t a, uint32_t b)
{
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) orthogonalize_small_kernel(const __grid_constant__ SmallArgs args)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double warp_sums[kWarps];
    __shared__ double block_sums[8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int C = (int)cluster_size(), rank = (int)cluster_ctarank();
    const SmallMatrix m = args.m[blockIdx.x / C];
    const bool tall = m.rows > m.cols;
    const int n = tall ? m.cols : m.rows, len = tall ? m.rows : m.cols;
    const int np = up16(n), per = up16((len + C - 1) / C);
    const int c0 = rank * per, mine = max(0, min(per, len - c0));      // this block's columns of X
    const SmallLayout L = small_layout(np, per, C > 1);
    const uint32_t base = smem_u32(smem);
    __half *lo = reinterpret_cast<__half *>(smem + L.lo);
    if (C > 1) cluster_sync_all();      // every block of the cluster runs before its shared memory is written from outside
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (args.head && blockIdx.x == 0)
        for (int i = tid; i < args.head_ints; i += kThreads) args.head[i] = 0;

    // the elements (i, j) of this block's columns, threads along the contiguous axis of the matrix, eight loads in flight
    const T *g = (const T *)m.g + (tall ? (long long)c0 * m.ld_g : (long long)c0);
    auto each = [&](auto &&f) {
        constexpr int kAt = 8;
        const int outer = tall ? mine : n, inner = tall ? n : mine;
        for (int r0 = warp; r0 < outer; r0 += kAt * kWarps)
            for (int c = lane; c < inner; c += 32) {
                float v[kAt];
#pragma unroll
                for (int k = 0; k < kAt; ++k)
                    v[k] = r0 + k * kWarps < outer ? (float)g[(long long)(r0 + k * kWarps) * m.ld_g + c] : 0.f;
#pragma unroll
                for (int k = 0; k < kAt; ++k)
                    if (r0 + k * kWarps < outer) f(tall ? c : r0 + k * kWarps, tall ? r0 + k * kWarps : c, v[k]);
            }
    };
    double sq = 0.0;
    each([&](int, int, float v) { sq = fma((double)v, (double)v, sq); });
    // padding: zero rows and columns take part in the products
    for (int i = tid; i < (int)((3 * (size_t)np * L.xs) / 2); i += kThreads) reinterpret_cast<uint32_t *>(smem)[i] = 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
    if (lane == 0) warp_sums[warp] = sq;
    __syncthreads();
    if (tid == 0) {
        double t = 0.0;
        for (int w = 0; w < kWarps; ++w) t += warp_sums[w];
        for (int r = 0; r < C; ++r) {
            const uint32_t to = C > 1 ? map_to_cta(smem_u32(&block_sums[rank]), r) : smem_u32(&block_sums[0]);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(t) : "memory");
        }
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    double total = 0.0;
    for (int r = 0; r < C; ++r) total += block_sums[r];
    const float inv = (float)((double)kOrthScaleX / (sqrt(total) + (double)args.eps));
    {
        __half *hi = reinterpret_cast<__half *>(smem + L.hi0);
        each([&](int i, int j, float v) {
            const float x = v * inv;
            const __half h = __float2half_rn(x);
            hi[i * L.xs + j] = h;
            lo[i * L.xs + j] = __float2half_rn(x - __half2float(h));
        });
    }
    __syncthreads();

    const int nt = np / 16, pt = per / 16;
    const int fr = lane >> 2, fc = 2 * (lane & 3);          // a fragment's row (and row + 8) and columns (two of eight)
    const float beta = args.k[1] * kOrthScaleB / kOrthScaleA, alpha = args.k[2] * kOrthScaleB / (kOrthScaleA * kOrthScaleA);
    const float diagonal = args.k[0] * kOrthScaleB;
    constexpr float kGram = kOrthScaleA / (kOrthScaleX * kOrthScaleX);
    for (int it = 0; it < args.steps; ++it) {
        const size_t cur_off = (it & 1) ? L.hi1 : L.hi0, next_off = (it & 1) ? L.hi0 : L.hi1;
        const uint32_t cur = base + (uint32_t)cur_off;
        __half *A = reinterpret_cast<__half *>(smem + L.a), *B = reinterpret_cast<__half *>(smem + L.b);
        float *part = reinterpret_cast<float *>(smem + L.part);
        for (int t = warp; t < nt * nt; t += kWarps) {
            const int i0 = t / nt * 16, j0 = t % nt * 16;
            float acc[2][4] = {};
            block_nt(acc, cur, L.xs, cur, L.xs, i0, j0, per, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int i = i0 + fr + 8 * r, j = j0 + 8 * h + fc;
                    if (C == 1)
                        *reinterpret_cast<uint32_t *>(A + i * L.as + j) = half2_bits(acc[h][2 * r] * kGram, acc[h][2 * r + 1] * kGram);
                    else
                        *reinterpret_cast<float2 *>(part + i * np + j) = make_float2(acc[h][2 * r], acc[h][2 * r + 1]);
                }
        }
        if (C > 1) {
            cluster_sync_all();
            // four neighbouring elements a thread, shares of the blocks interleaved
            for (int q = rank * kThreads + tid; q < np * np / 4; q += C * kThreads) {
                float4 v = make_float4(0, 0, 0, 0);
                for (int r = 0; r < C; ++r) {
                    const float4 f = ld_cluster_f4(map_to_cta(base + (uint32_t)L.part + q * 16, r));
                    v.x += f.x; v.y += f.y; v.z += f.z; v.w += f.w;
                }
                const int i = 4 * q / np, j = 4 * q - i * np;
                const uint32_t w0 = half2_bits(v.x * kGram, v.y * kGram), w1 = half2_bits(v.z * kGram, v.w * kGram);
                for (int r = 0; r < C; ++r) st_cluster_u2(map_to_cta(base + (uint32_t)L.a + (i * L.as + j) * 2, r), w0, w1);
            }
            cluster_sync_all();
        } else {
            __syncthreads();
        }
        for (int t = warp; t < nt * nt; t += kWarps) {
            const int i0 = t / nt * 16, j0 = t % nt * 16;
            float acc[2][4] = {};
            block_nt(acc, base + (uint32_t)L.a, L.as, base + (uint32_t)L.a, L.as, i0, j0, np, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int at = (i0 + fr + 8 * r) * L.as + j0 + 8 * h + fc;
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(A + at));
                    const int off = (j0 + 8 * h + fc) - (i0 + fr + 8 * r);      // a I: this element's, or its neighbour's
                    *reinterpret_cast<uint32_t *>(B + at) =
                        half2_bits(fmaf(beta, f.x, alpha * acc[h][2 * r]) + (off == 0 ? diagonal : 0.f),
                                   fmaf(beta, f.y, alpha * acc[h][2 * r + 1]) + (off == -1 ? diagonal : 0.f));
                }
        }
        __syncthreads();
        const bool last = it + 1 == args.steps;
        __half *next = reinterpret_cast<__half *>(smem + next_off);
        for (int t = warp; t < nt * pt; t += kWarps) {
            const int i0 = t / pt * 16, j0 = t % pt * 16;
            float acc[2][4] = {};
            block_nn(acc, base + (uint32_t)L.b, L.as, cur, L.xs, i0, j0, np, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int at = (i0 + fr + 8 * r) * L.xs + j0 + 8 * h + fc;
                    const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(lo + at));
                    const float v0 = fmaf(args.k[0], y.x, acc[h][2 * r] * (1.f / kOrthScaleB));
                    const float v1 = fmaf(args.k[0], y.y, acc[h][2 * r + 1] * (1.f / kOrthScaleB));
                    if (last) {
                        const float s = m.scale / kOrthScaleX;
                        *reinterpret_cast<__nv_bfloat162 *>(next + at) = __floats2bfloat162_rn(v0 * s, v1 * s);
                    } else {
                        const __half2 hh = __floats2half2_rn(v0, v1);
                        const float2 back = __half22float2(hh);
                        *reinterpret_cast<__half2 *>(next + at) = hh;
                        *reinterpret_cast<uint32_t *>(lo + at) = half2_bits(v0 - back.x, v1 - back.y);
                    }
                }
        }
        __syncthreads();
    }
    // the result lies as bf16 in the buffer the last iteration wrote
    const __nv_bfloat16 *res = reinterpret_cast<const __nv_bfloat16 *>(smem + ((args.steps & 1) ? L.hi1 : L.hi0));
    if (!tall) {
        for (int i = warp; i < n; i += kWarps)
            for (int j = lane; j < mine; j += 32) m.out[(long long)i * m.ld_out + c0 + j] = res[i * L.xs + j];
    } else {
        for (int j = warp; j < mine; j += kWarps)
            for (int i = lane; i < n; i += 32) m.out[(long long)(c0 + j) * m.ld_out + i] = res[i * L.xs + j];
    }
    if (C > 1) cluster_sync_all();      // no block leaves while another may still read its shared memory
}

template <typename T>
cudaError_t launch(const SmallArgs &a, int n, int cluster, size_t smem, cudaStream_t s)
{
    auto kern = orthogonalize_small_kernel<T>;
    static unsigned long long attr_done = 0;      // bit per device ordinal (devices beyond 63 set it every time)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev > 63 || !((attr_done >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
        if (e != cudaSuccess) return e;
        if (dev <= 63) attr_done |= 1ull << dev;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(n * cluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

size_t smem_of(int rows, int cols, int cluster)
{
    const int n = rows < cols ? rows : cols, len = rows < cols ? cols : rows;
    return small_layout(up16(n), up16((len + cluster - 1) / cluster), cluster > 1).total;
}

}  // namespace

int orthogonalize_small_cluster(int rows, int cols)
{
    if ((rows < cols ? rows : cols) > kOrthSmallMax) return 0;
    for (int c = 1; c <= 8; c *= 2)
        if (smem_of(rows, cols, c) <= kSmemMost) return c;
    return 0;
}

cudaError_t launch_orthogonalize_small(bool f32, const SmallArgs &a, int n, cudaStream_t s)
{
    int cluster = 1;
    for (int i = 0; i < n; ++i) {
        const int c = orthogonalize_small_cluster(a.m[i].rows, a.m[i].cols);
        if (c == 0) return cudaErrorInvalidValue;
        cluster = c > cluster ? c : cluster;
    }
    size_t smem = 0;
    for (int i = 0; i < n; ++i) {
        const size_t b = smem_of(a.m[i].rows, a.m[i].cols, cluster);
        if (b > kSmemMost) return cudaErrorInvalidValue;
        smem = b > smem ? b : smem;
    }
    return f32 ? launch<float>(a, n, cluster, smem, s) : launch<__nv_bfloat16>(a, n, cluster, smem, s);
}

}  // namespace modse
