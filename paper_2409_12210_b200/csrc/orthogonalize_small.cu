// Orthogonalised updates of matrices whose shorter side is at most 128: the whole iteration in one kernel.
//
// As grouped products such a matrix is seventeen launches that each last a few microseconds and compute for less than
// one.  Here a block - or a cluster of up to sixteen blocks that split the longer side - keeps X (hi and lo, fp16) in shared
// memory for all iterations and multiplies with mma.sync.  Per iteration:
//   A = X X^T    every block over its own columns; blocks of a cluster leave fp32 partial sums in their shared memory and
//                each adds up (in block order) and hands out its share of A through distributed shared memory;
//   B = aI + bA + cA^2  computed by every block for itself (a 128 x 128 product is cheaper than another meeting);
//   X <- B hi + a lo   every block on its own columns.
// Of the longest matrices the step replaces hi in place instead of writing a second copy: a warp then takes all rows of
// sixteen columns.  Eight blocks hold 64 x 3968 to 128 x 896, sixteen 64 x 7936 to 128 x 1792 and in place 64 x 12544 to 128 x 3840
// (75 x 3499, 114 x 75 and 1345 x 75: 63 us against 175 as grouped products; 64 x 8448 97 against 141; 99 x 5000, near the
// end of the range, 115 against 133).
// The roundings are those of the grouped form (orthogonalize.cu): fp16 factors scaled by powers of two, X in 22 bits.
// A tall matrix is transposed on its way in and out.
#include <cuda_fp16.h>

#include "launch.h"
#include "orthogonalize_small.h"
#include "tc_device.h"

namespace modse {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMostBlocks = 16;                       // of a cluster (above eight only where a kernel is told so)
constexpr size_t kSmemMost = 227 * 1024 - 1024;       // dynamic; the static part stays below 1 KB

__host__ __device__ inline int up16(int v) { return (v + 15) / 16 * 16; }

// Shared memory of a block for n rows (a multiple of 16) and per columns: rows are padded by 16 bytes, so that eight
// consecutive rows of a matrix load fall into different banks.  In place: one copy of hi, and the partial sums of A lie
// where B is written after them.
struct SmallLayout {
    int xs, as;                         // row lengths in halves
    size_t hi0, hi1, lo, a, b, part, total;
};
__host__ __device__ inline SmallLayout small_layout(int n, int per, bool cluster, bool in_place)
{
    SmallLayout L;
    L.xs = per + 8;
    L.as = n + 8;
    const size_t x = (size_t)n * L.xs * 2, q = (size_t)n * L.as * 2;
    L.hi0 = 0;
    L.hi1 = in_place ? 0 : x;
    L.lo = L.hi1 + x;
    L.a = L.lo + x;
    L.b = L.a + q;
    L.part = in_place ? L.b : L.b + q;
    const size_t part = cluster ? (size_t)n * n * 4 : 0;
    L.total = L.b + (in_place ? (q > part ? q : part) : q + part);
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

// A warp's block of 16 MI x 16 NJ numbers of P Q^T (TRANS false: Q [columns][k]) or P Q (TRANS: Q [k][columns]) from (i0, j0)
// on, all row-major in shared memory with row lengths ps, qs (halves), k a multiple of 16.
template <bool TRANS, int MI, int NJ>
__device__ __forceinline__ void warp_block(float (&acc)[MI][NJ][2][4], uint32_t p, int ps, uint32_t q, int qs, int i0, int j0,
                                           int k, int lane)
{
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[i][j][e >> 2][e & 3] = 0.f;
    // matrices of a load of P: rows 0-7 / 8-15 at k 0-7, then the same rows at k 8-15
    const uint32_t pa = p + (uint32_t)((i0 + (lane & 15)) * ps + (lane >> 4) * 8) * 2;
    // of Q^T: rows 0-7 at k 0-7, rows 0-7 at k 8-15, rows 8-15 at k 0-7, rows 8-15 at k 8-15;
    // of Q, transposed on the way: k rows 0-7 / 8-15 at columns 0-7, then at columns 8-15
    const uint32_t qa = TRANS ? q + (uint32_t)((lane & 15) * qs + j0 + (lane >> 4) * 8) * 2
                              : q + (uint32_t)((j0 + (lane & 7) + ((lane >> 4) << 3)) * qs + ((lane >> 3) & 1) * 8) * 2;
#pragma unroll 2
    for (int kk = 0; kk < k; kk += 16) {
        uint32_t a[MI][4], b[NJ][4];
#pragma unroll
        for (int i = 0; i < MI; ++i) ldsm4(a[i], pa + (uint32_t)(16 * i * ps + kk) * 2);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            if constexpr (TRANS) ldsm4_t(b[j], qa + (uint32_t)(kk * qs + 16 * j) * 2);
            else ldsm4(b[j], qa + (uint32_t)(16 * j * qs + kk) * 2);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                mma_f16(acc[i][j][0], a[i], b[j][0], b[j][1]);
                mma_f16(acc[i][j][1], a[i], b[j][2], b[j][3]);
            }
    }
}
template <bool TRANS, int MI, int NJ, typename G, typename F>
__device__ __forceinline__ void warp_tile(uint32_t p, int ps, uint32_t q, int qs, int i0, int j0, int k, int lane, G &get, F &put)
{
    const int fr = lane >> 2, fc = 2 * (lane & 3);          // a fragment's row (and row + 8) and columns (two of eight)
    float acc[MI][NJ][2][4];
    uint32_t in[MI][NJ][2][2];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) in[i][j][h][r] = get(i0 + 16 * i + fr + 8 * r, j0 + 16 * j + 8 * h + fc);
    warp_block<TRANS, MI, NJ>(acc, p, ps, q, qs, i0, j0, k, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    put(i0 + 16 * i + fr + 8 * r, j0 + 16 * j + 8 * h + fc, acc[i][j][h][2 * r], acc[i][j][h][2 * r + 1], in[i][j][h][r]);
}
// All 16 MI x 16 NJ blocks of a rows x cols product (multiples of 16) shared out over the warps.  For every two
// neighbouring numbers of a row, get(row, column) reads what their epilogue needs before the products begin (after them
// every read would wait for the writes before it) and put(row, column, v0, v1, what get read) writes.  Reading the
// fragments costs as much as multiplying them in a 16 x 16 block, so a warp takes as large a block as leaves work for
// the others.
template <bool TRANS, int MI, int NJ, typename G, typename F>
__device__ __forceinline__ void warp_product(uint32_t p, int ps, uint32_t q, int qs, int rows, int cols, int k, int warp,
                                             int lane, G &&get, F &&put)
{
    const int tj = (cols + 16 * NJ - 1) / (16 * NJ), tiles = (rows + 16 * MI - 1) / (16 * MI) * tj;
    for (int t = warp; t < tiles; t += kWarps) {
        const int i0 = t / tj * 16 * MI, j0 = t % tj * 16 * NJ;
        if (i0 + 16 * MI <= rows && j0 + 16 * NJ <= cols) {
            warp_tile<TRANS, MI, NJ>(p, ps, q, qs, i0, j0, k, lane, get, put);
        } else {
            for (int i = i0; i < min(i0 + 16 * MI, rows); i += 16)
                for (int j = j0; j < min(j0 + 16 * NJ, cols); j += 16) warp_tile<TRANS, 1, 1>(p, ps, q, qs, i, j, k, lane, get, put);
        }
    }
}

// X <- P X in place (P n x n, X n x cols, multiples of 16): a warp takes all rows of sixteen columns, which no other warp
// reads.  get and put as above; get is called after the products, all of it before the first put.
template <typename G, typename F>
__device__ __forceinline__ void warp_columns(uint32_t p, int ps, uint32_t x, int xs, int n, int cols, int warp, int lane,
                                             G &&get, F &&put)
{
    constexpr int MI = kOrthSmallMax / 16;
    const int fr = lane >> 2, fc = 2 * (lane & 3);
    const uint32_t pa = p + (uint32_t)((lane & 15) * ps + (lane >> 4) * 8) * 2;
    for (int j0 = 16 * warp; j0 < cols; j0 += 16 * kWarps) {
        const uint32_t xa = x + (uint32_t)((lane & 15) * xs + j0 + (lane >> 4) * 8) * 2;
        float acc[MI][2][4];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[i][e >> 2][e & 3] = 0.f;
#pragma unroll 1
        for (int kk = 0; kk < n; kk += 16) {
            uint32_t b[4];
            ldsm4_t(b, xa + (uint32_t)(kk * xs) * 2);
#pragma unroll
            for (int i = 0; i < MI; ++i)
                if (16 * i < n) {
                    uint32_t a[4];
                    ldsm4(a, pa + (uint32_t)(16 * i * ps + kk) * 2);
                    mma_f16(acc[i][0], a, b[0], b[1]);
                    mma_f16(acc[i][1], a, b[2], b[3]);
                }
        }
        __syncwarp();                  // the columns are read
        uint32_t in[MI][2][2];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * i < n) in[i][e >> 1][e & 1] = get(16 * i + fr + 8 * (e & 1), j0 + 8 * (e >> 1) + fc);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * i < n)
                    put(16 * i + fr + 8 * (e & 1), j0 + 8 * (e >> 1) + fc, acc[i][e >> 1][2 * (e & 1)], acc[i][e >> 1][2 * (e & 1) + 1],
                        in[i][e >> 1][e & 1]);
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

template <typename T, bool IN_PLACE>
__global__ void __launch_bounds__(kThreads, 1) orthogonalize_small_kernel(const __grid_constant__ SmallArgs args)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double warp_sums[kWarps];
    __shared__ double block_sums[kMostBlocks];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int C = (int)cluster_size(), rank = (int)cluster_ctarank();
    const SmallMatrix m = args.m[blockIdx.x / C];
    const bool tall = m.rows > m.cols;
    const int n = tall ? m.cols : m.rows, len = tall ? m.rows : m.cols;
    const int np = up16(n), per = up16((len + C - 1) / C);
    const int c0 = rank * per, mine = max(0, min(per, len - c0));      // this block's columns of X
    const SmallLayout L = small_layout(np, per, C > 1, IN_PLACE);
    const uint32_t base = smem_u32(smem);
    __half *lo = reinterpret_cast<__half *>(smem + L.lo);
    if (C > 1) cluster_sync_all();      // every block of the cluster runs before its shared memory is written from outside
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (args.head && blockIdx.x == 0)
        for (int i = tid; i < args.head_ints; i += kThreads) args.head[i] = 0;

    // the elements (i, j) of this block's columns, threads along the contiguous axis of the matrix, two pieces of eight rows
    // in flight (zeros past the end)
    const T *g = (const T *)m.g + (tall ? (long long)c0 * m.ld_g : (long long)c0);
    constexpr int kAt = 8;
    const int outer = tall ? mine : n, inner = tall ? n : mine;
    auto each = [&](auto &&f) {
        for (int r0 = warp; r0 < outer; r0 += kAt * kWarps)
            for (int c = lane; c < inner; c += 64) {
                float v[2][kAt];
#pragma unroll
                for (int k = 0; k < kAt; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        v[h][k] = r0 + k * kWarps < outer && c + 32 * h < inner ? (float)g[(long long)(r0 + k * kWarps) * m.ld_g + c + 32 * h] : 0.f;
                f(r0, c, v[0]);
                if (c + 32 < inner) f(r0, c + 32, v[1]);
            }
    };
    double sq = 0.0;      // eight squares in fp32 where their sum is well inside its range, in fp64 otherwise
    each([&](int, int, const float (&v)[kAt]) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < kAt; ++k) t = fmaf(v[k], v[k], t);
        if (t >= 1e-30f && t <= 1e30f) {
            sq += (double)t;
        } else {
#pragma unroll
            for (int k = 0; k < kAt; ++k) sq = fma((double)v[k], (double)v[k], sq);
        }
    });
    // padding: zero rows and columns take part in the products
    for (int i = warp; i < np; i += kWarps)
        for (int j = (i < n ? mine : 0) + lane; j < L.xs; j += 32) {
            reinterpret_cast<__half *>(smem + L.hi0)[i * L.xs + j] = __ushort_as_half(0);
            if (!IN_PLACE) reinterpret_cast<__half *>(smem + L.hi1)[i * L.xs + j] = __ushort_as_half(0);
            lo[i * L.xs + j] = __ushort_as_half(0);
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
    if (lane == 0) warp_sums[warp] = sq;
    __syncthreads();
    if (warp == 0) {
        double t = lane < kWarps ? warp_sums[lane] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
        if (lane < C) {
            const uint32_t to = C > 1 ? map_to_cta(smem_u32(&block_sums[rank]), lane) : smem_u32(&block_sums[0]);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(t) : "memory");
        }
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    double total = 0.0;
    for (int r = 0; r < C; ++r) total += block_sums[r];
    const StartScale start = start_scale(sqrt(total), args.eps);
    {
        __half *hi = reinterpret_cast<__half *>(smem + L.hi0);
        const int step = kWarps * (tall ? 1 : L.xs);
        each([&](int r0, int c, const float (&v)[kAt]) {
            int at = tall ? c * L.xs + r0 : r0 * L.xs + c;
#pragma unroll
            for (int k = 0; k < kAt; ++k, at += step)
                if (r0 + k * kWarps < outer) {
                    const float x = v[k] * start.pre * start.inv;
                    const __half h = __float2half_rn(x);
                    hi[at] = h;
                    lo[at] = __float2half_rn(x - __half2float(h));
                }
        });
    }
    __syncthreads();

    const bool large = np == kOrthSmallMax;      // 32 x 32 a warp leaves none of the sixteen idle
    const float beta = args.k[1] * kOrthScaleB / kOrthScaleA, alpha = args.k[2] * kOrthScaleB / (kOrthScaleA * kOrthScaleA);
    const float diagonal = args.k[0] * kOrthScaleB;
    constexpr float kGram = kOrthScaleA / (kOrthScaleX * kOrthScaleX);
    for (int it = 0; it < args.steps; ++it) {
        const size_t cur_off = (it & 1) ? L.hi1 : L.hi0, next_off = (it & 1) ? L.hi0 : L.hi1;
        const uint32_t cur = base + (uint32_t)cur_off;
        __half *A = reinterpret_cast<__half *>(smem + L.a), *B = reinterpret_cast<__half *>(smem + L.b);
        float *part = reinterpret_cast<float *>(smem + L.part);
        auto get_none = [](int, int) { return 0u; };
        auto put_gram = [&](int i, int j, float v0, float v1, uint32_t) {
            if (C == 1) *reinterpret_cast<uint32_t *>(A + i * L.as + j) = half2_bits(v0 * kGram, v1 * kGram);
            else *reinterpret_cast<float2 *>(part + i * np + j) = make_float2(v0, v1);
        };
        if (large) warp_product<false, 2, 2>(cur, L.xs, cur, L.xs, np, np, per, warp, lane, get_none, put_gram);
        else warp_product<false, 1, 2>(cur, L.xs, cur, L.xs, np, np, per, warp, lane, get_none, put_gram);
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
        const uint32_t a_at = base + (uint32_t)L.a, b_at = base + (uint32_t)L.b;
        auto get_poly = [&](int i, int j) { return *reinterpret_cast<const uint32_t *>(A + i * L.as + j); };
        auto put_poly = [&](int i, int j, float v0, float v1, uint32_t in) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&in));
            *reinterpret_cast<uint32_t *>(B + i * L.as + j) = half2_bits(fmaf(beta, f.x, alpha * v0) + (i == j ? diagonal : 0.f),
                                                               fmaf(beta, f.y, alpha * v1) + (i == j + 1 ? diagonal : 0.f));
        };
        if (large) warp_product<false, 2, 2>(a_at, L.as, a_at, L.as, np, np, np, warp, lane, get_poly, put_poly);
        else warp_product<false, 1, 2>(a_at, L.as, a_at, L.as, np, np, np, warp, lane, get_poly, put_poly);
        __syncthreads();
        const bool last = it + 1 == args.steps;
        const float by = last ? m.scale / kOrthScaleX : 1.f;
        __half *next = reinterpret_cast<__half *>(smem + next_off);
        auto get_step = [&](int i, int j) { return *reinterpret_cast<const uint32_t *>(lo + i * L.xs + j); };
        auto put_step = [&](int i, int j, float v0, float v1, uint32_t in) {
            const int at = i * L.xs + j;
            const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&in));
            v0 = fmaf(args.k[0], y.x, v0 * (1.f / kOrthScaleB));
            v1 = fmaf(args.k[0], y.y, v1 * (1.f / kOrthScaleB));
            if (last) {
                *reinterpret_cast<__nv_bfloat162 *>(next + at) = __floats2bfloat162_rn(v0 * by, v1 * by);
            } else {
                const __half2 hh = __floats2half2_rn(v0, v1);
                const float2 back = __half22float2(hh);
                *reinterpret_cast<__half2 *>(next + at) = hh;
                *reinterpret_cast<uint32_t *>(lo + at) = half2_bits(v0 - back.x, v1 - back.y);
            }
        };
        if constexpr (IN_PLACE) warp_columns(b_at, L.as, cur, L.xs, np, per, warp, lane, get_step, put_step);
        else if (large) warp_product<true, 2, 2>(b_at, L.as, cur, L.xs, np, per, np, warp, lane, get_step, put_step);
        else warp_product<true, 1, 2>(b_at, L.as, cur, L.xs, np, per, np, warp, lane, get_step, put_step);
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

template <typename T, bool IN_PLACE>
cudaError_t launch(const SmallArgs &a, int n, int cluster, size_t smem, cudaStream_t s)
{
    auto kern = orthogonalize_small_kernel<T, IN_PLACE>;
    static DeviceFlags done;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!done.has(dev)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        done.set(dev);
    }
    return launch_clusters(kern, cluster, n * cluster, kThreads, smem, s, a);
}

size_t smem_of(int rows, int cols, const SmallForm &f)
{
    const int n = rows < cols ? rows : cols, len = rows < cols ? cols : rows;
    return small_layout(up16(n), up16((len + f.blocks - 1) / f.blocks), f.blocks > 1, f.in_place).total;
}

}  // namespace

SmallForm orthogonalize_small_form(int rows, int cols, int most)
{
    if ((rows < cols ? rows : cols) > kOrthSmallMax) return {0, false};
    for (int c = 1; c <= most; c *= 2)
        if (smem_of(rows, cols, {c, false}) <= kSmemMost) return {c, false};
    const SmallForm last{kMostBlocks, true};
    return most == kMostBlocks && smem_of(rows, cols, last) <= kSmemMost ? last : SmallForm{0, false};
}

cudaError_t launch_orthogonalize_small(bool f32, const SmallArgs &a, int n, int most, cudaStream_t s)
{
    SmallForm form{1, false};
    for (int i = 0; i < n; ++i) {
        const SmallForm f = orthogonalize_small_form(a.m[i].rows, a.m[i].cols, most);
        if (f.blocks == 0) return cudaErrorInvalidValue;
        form.blocks = f.blocks > form.blocks ? f.blocks : form.blocks;
        form.in_place |= f.in_place;
    }
    size_t smem = 0;
    for (int i = 0; i < n; ++i) {
        const size_t b = smem_of(a.m[i].rows, a.m[i].cols, form);
        if (b > kSmemMost) return cudaErrorInvalidValue;
        smem = b > smem ? b : smem;
    }
    if (form.in_place) return f32 ? launch<float, true>(a, n, form.blocks, smem, s) : launch<__nv_bfloat16, true>(a, n, form.blocks, smem, s);
    return f32 ? launch<float, false>(a, n, form.blocks, smem, s) : launch<__nv_bfloat16, false>(a, n, form.blocks, smem, s);
}

}  // namespace modse
