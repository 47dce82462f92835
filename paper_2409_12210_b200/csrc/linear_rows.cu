// modse_linear for a few tokens: the product streams the weights once.
//
// With T <= 32 rows the time is that of reading w [d_out, d_in] (8.4 MB for 2048 x 2048 in bf16: 1.3 us at the measured
// copy rate), so the kernel is built around loads in flight, not around the tensor cores' peak: a block of eight warps
// owns 16 rows of w, each warp takes every eighth 128-byte column block of them straight from global memory into
// mma.sync fragments, and the eight partial sums meet in shared memory in a fixed order.  A 128-row tcgen05 tile would
// spend its time on filling and draining itself.  Measured on rows of calls in a graph, each with weights of its own, so
// that they come from HBM (in brackets the weights' time at the measured copy rate): one token on 2048 x 5632 bf16 7.1 us
// (3.5), on 8448 x 8448 26.7 (21.8); 24 tokens on 2048 x 5632 e4m3 6.1 (1.8), 4.9 where the calls share weights that stay
// in L2.  A call by itself, cold and with all of its launch, takes 3 to 5 us more.  The tcgen05 form takes 12 to 46 us on these.
//
// Fragments without shared memory: a sum over k may be taken in any order as long as both operands agree on it.  Thread
// t of a group of four loads 16 contiguous bytes of its row of w and the same 16 bytes of its row of x; the k-th pair of
// 16-bit numbers in them plays the part of the fragment's columns 2t, 2t+1 (+8).  Four such loads of neighbouring threads
// cover 64 contiguous bytes of a row.  8-bit operands are widened to fp16 on the way (exact) and use the fp16 form.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "activations.h"
#include "dense_gemm.h"
#include "launch.h"
#include "linear_rows.h"

namespace modse {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool f16)
{
    if (f16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// four e4m3 bytes as two pairs of fp16
__device__ __forceinline__ void widen(uint32_t v, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(v));
}

// 16 bytes, or zeros where there are none.  volatile: the loads of a step stay ahead of its products.  Not the read-only
// path: the kernel ahead may still be writing x when this one starts, and that path promises nothing for such data, even
// where it is read after wait_for_earlier_kernels.
__device__ __forceinline__ uint4 load_stream(const unsigned char *p, bool in)
{
    uint4 v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
                 "mov.b32 %3, 0;\n\t@q ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)in));
    return v;
}
__device__ __forceinline__ uint4 load_shared_rows(const unsigned char *p, bool in)      // x: every block reads it, L1 may keep it
{
    uint4 v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
                 "mov.b32 %3, 0;\n\t@q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)in));
    return v;
}

__device__ __forceinline__ uint32_t word_at(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// products of 16 bytes of two rows of w (rows g and g + 8) with 16 bytes of NT rows of x
template <bool F8, int NT>
__device__ __forceinline__ void fragment_mma(float (&acc)[NT][4], const uint4 &w0, const uint4 &w1, const uint4 (&x)[NT])
{
    if constexpr (F8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[4];
            widen(word_at(w0, i), a[0], a[2]);
            widen(word_at(w1, i), a[1], a[3]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t b0, b1;
                widen(word_at(x[n], i), b0, b1);
                mma_16816(acc[n], a, b0, b1, true);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t a[4] = {word_at(w0, 2 * i), word_at(w1, 2 * i), word_at(w0, 2 * i + 1), word_at(w1, 2 * i + 1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16816(acc[n], a, word_at(x[n], 2 * i), word_at(x[n], 2 * i + 1), false);
        }
    }
}

struct RowsArgs {
    const unsigned char *x, *w;
    LinearEpilogue lin;
    int *status;
    int T, n;
    int row_bytes;         // of x and w, a multiple of 16
};

// MT x 16 rows of w a block, NT x 8 tokens, U units of 64 bytes a row in flight
template <bool F8, int MT, int NT, int U>
__global__ void __launch_bounds__(32 * kWarps)
linear_rows_kernel(const RowsArgs p)
{
    __shared__ float part[kWarps][NT * 8][MT * 16 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * (16 * MT);
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = kDevOk;
    // rows past the end read the last row; what they give is not stored
    const unsigned char *wr[2 * MT], *xr[NT];
#pragma unroll
    for (int m = 0; m < 2 * MT; ++m) wr[m] = p.w + (size_t)min(n0 + g + 8 * m, p.n - 1) * p.row_bytes + t * 16;
#pragma unroll
    for (int n = 0; n < NT; ++n) xr[n] = p.x + (size_t)min(8 * n + g, p.T - 1) * p.row_bytes + t * 16;
    float acc[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
    // a warp takes units 2 w, 2 w + 1 of every sixteen (16 bytes of a unit a thread)
    const int units = (p.row_bytes + 63) / 64;
    for (int u0 = 2 * warp; u0 < units; u0 += 8 * U) {
        uint4 w[U][2 * MT], x[U][NT];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int at = (u0 + (j >> 1) * 16 + (j & 1)) * 64;
            const bool in = at + t * 16 < p.row_bytes;
#pragma unroll
            for (int m = 0; m < 2 * MT; ++m) w[j][m] = load_stream(wr[m] + at, in);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[j][n] = load_shared_rows(xr[n] + at, in);
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int m = 0; m < MT; ++m) fragment_mma<F8, NT>(acc[m], w[j][2 * m], w[j][2 * m + 1], x[j]);
    }
    // accumulator (row, token): rows g, g + 8 of a 16-row block, tokens 8 n + 2 t, + 1
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][8 * n + 2 * t + (i & 1)][16 * m + g + 8 * (i >> 1)] = acc[m][n][i];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 8 * 8 * MT; i += 32 * kWarps) {
        const int tok = i / (8 * MT), c = 2 * (i % (8 * MT)), col = n0 + c;       // two neighbouring outputs a thread
        if (tok >= p.T || col >= p.n) continue;
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            v[0] += part[w][tok][c];
            v[1] += part[w][tok][c + 1];
        }
        const LinearEpilogue &lin = p.lin;
        const size_t at = (size_t)tok * p.n + col;
        if (F8) {
            const float s = lin.sx[tok];
            v[0] *= s * lin.sw[col];
            v[1] *= s * lin.sw[col + 1];
        }
        if (lin.bias) {
            v[0] += __bfloat162float(lin.bias[col]);
            v[1] += __bfloat162float(lin.bias[col + 1]);
        }
        if (lin.z) *reinterpret_cast<__nv_bfloat162 *>(lin.z + at) = __floats2bfloat162_rn(v[0], v[1]);
        switch (lin.act) {
        case MODSE_ACT_RELU: activate2<MODSE_ACT_RELU>(v[0], v[1]); break;
        case MODSE_ACT_GELU: activate2<MODSE_ACT_GELU>(v[0], v[1]); break;
        case MODSE_ACT_SILU: activate2<MODSE_ACT_SILU>(v[0], v[1]); break;
        default: break;
        }
        if (lin.residual) {
            const __nv_bfloat162 r = *reinterpret_cast<const __nv_bfloat162 *>(lin.residual + at);
            v[0] += __bfloat162float(r.x);
            v[1] += __bfloat162float(r.y);
        }
        *reinterpret_cast<__nv_bfloat162 *>(lin.y + at) = __floats2bfloat162_rn(v[0], v[1]);
    }
}

template <bool F8, int MT, int NT, int U>
cudaError_t launch_one(const RowsArgs &p, cudaStream_t s)
{
    return launch_overlapped(linear_rows_kernel<F8, MT, NT, U>, (p.n + 16 * MT - 1) / (16 * MT), 32 * kWarps, 0, s, p);
}

template <bool F8>
cudaError_t launch(const RowsArgs &p, cudaStream_t s)
{
    if (p.T <= 8) return launch_one<F8, 1, 1, 4>(p, s);
    if (p.T <= 16) return launch_one<F8, 1, 2, 4>(p, s);
    if constexpr (!F8) {
        // With more than 16 tokens a block reads more of x than of w: 32 rows of w a block halve that, where they still
        // leave a block for every SM (8448 x 8448, 32 tokens: 31 us against 50).  8-bit rows are half as long, and
        // widening them fills the registers (10.5 us against 7.5 at 2048 x 5632): 16 rows.
        if (p.n >= 32 * device_sms()) return p.T <= 24 ? launch_one<F8, 2, 3, 2>(p, s) : launch_one<F8, 2, 4, 2>(p, s);
    }
    return p.T <= 24 ? launch_one<F8, 1, 3, 4>(p, s) : launch_one<F8, 1, 4, 4>(p, s);
}

}  // namespace

cudaError_t launch_linear_rows(DenseType type, const void *x, const void *w, int T, int k, int n, const LinearEpilogue &lin,
                               int *status, cudaStream_t s)
{
    const RowsArgs p{(const unsigned char *)x, (const unsigned char *)w, lin, status, T, n, type == DenseE4m3 ? k : 2 * k};
    return type == DenseE4m3 ? launch<true>(p, s) : launch<false>(p, s);
}

}  // namespace modse
