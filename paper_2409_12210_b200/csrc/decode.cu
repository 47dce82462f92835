// modse_decode: the whole MoDSE layer for the few tokens of a generation step, in two kernels.
//
//   logits z = x W_g (+ the second term of Eq. 2), top-k, gates g (Eq. 2-3)
//   h_tj = g_tj silu(x_t W_gate^T) (x_t W_up^T) for the experts met,   y_t = sum_j h_tj W_down^T   (Eq. 4)
//
// What bounds it is reading the experts met once, 6 d h bytes each in bf16; tiles of 128 tokens, as the grouped products of
// modse_forward take them, would spend their time on filling and draining themselves.  So both kernels stream rows of
// weights into mma.sync fragments.
//
// First kernel: every block works out the routing of all tokens for itself (the router matrix is as large as sixteen rows of
// an expert and comes from L2; handing the result from block to block would cost a launch), then takes units of eight
// hidden columns: their eight rows of W_gate and of W_up fill the sixteen rows of a fragment, so a thread ends up with
// both factors of SwiGLU.  The eight warps of a block split the contraction; their sums meet in shared memory.
// Second kernel: sixteen rows of W_down a fragment, the contraction running over the hidden columns of all experts met.
// The whole of it, rows of fragments times contraction, is one line that is cut into even spans, one a block, wherever
// the cuts fall; a group of rows that several blocks share is added up in the blocks' order by the one that arrives last.
//
// The kernels in this file read fragments straight from global memory and take any layer, in bf16 and fp32; those in
// decode_tma.cu take the bf16 layers whose extents are multiples of 64.
#include <algorithm>

#include "decode.h"
#include "tc_gemm.h"

namespace modse {
namespace decode {
namespace {

constexpr int blocks_per_sm(int token_groups) { return token_groups == 1 ? 3 : 2; }
constexpr int kMaxBlocks = 3 * 148;        // workspace sizes are asked for without a device
constexpr int kLeastSpan = 32;             // units of the second kernel that are worth a block of their own: two steps of its warps

// The logits ahead of the first kernel, for layers of so many experts that every block forming them would cost more than a
// launch: a block sixteen experts.
template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads) decode_logits_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ float part[kWarps][NTM * 8][kRows + 1];
    wait_for_earlier_kernels();
    allow_next_kernel();
    router_tile<T, NTM>(p, blockIdx.x, p.logits, part);
}

template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NTM)) decode_up_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ float part[2][kWarps][NTM * 8][kRows + 1];     // two of them, so that one meeting a unit is enough
    __shared__ Routing r;
    __shared__ float z[NTM * 8 * kInBlockExperts];
    __shared__ __align__(16) int idx[kMaxPicks], scan[kMaxPicks];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int k = p.m.k, row = p.m.d * (int)sizeof(T), units = (row + kUnit - 1) / kUnit;
    fetch_router(p, row);
    wait_for_earlier_kernels();
    allow_next_kernel();
    route<T, NTM>(p, z, part[0], idx, scan, r);
    if (blockIdx.x == 0) publish(p, r, idx);
    int round = 0;
    for (UnitCursor at{(int)blockIdx.x, 0, 0, 0}; at.settle(r); at.u += gridDim.x, ++round) {
        const int count = r.first[at.s + 1] - r.first[at.s];
        const int *pick = r.pick + r.first[at.s];
        const size_t w = ((size_t)r.offset[at.s] + at.c0 + g) * row + t * 16;
        const unsigned char *x[NTM];
#pragma unroll
        for (int n = 0; n < NTM; ++n) x[n] = p.x + (size_t)(pick[min(8 * n + g, count - 1)] / k) * row + t * 16;
        auto &sums = part[round & 1];
        dot<T, NTM>(count, p.w_gate + w, p.w_up + w, x, 0, units, row, sums[warp]);
        __syncthreads();
        if (threadIdx.x < count * kUnitCols) {
            const int i = threadIdx.x / kUnitCols, c = threadIdx.x % kUnitCols;
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int v = 0; v < kWarps; ++v) {
                a += sums[v][i][c];
                b += sums[v][i][c + kUnitCols];
            }
            // one rounding of the gated hidden value, as in modse_forward
            const float h = gated(r.gate[pick[i]], a, b);
            T *out = reinterpret_cast<T *>(p.hidden + pick[i] * p.ld) + at.c0 + c;
            if constexpr (sizeof(T) == 2) *out = __float2bfloat16_rn(h);
            else *out = h;
        }
    }
}

template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NTM)) decode_down_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ float part[2][kWarps][NTM * 8][kRows + 1];
    __shared__ Routing r;
    __shared__ int upto[kMaxPicks + 1];          // units ahead of each expert met
    __shared__ __align__(16) float out[NTM * 8][kRows];
    __shared__ int last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, tid = threadIdx.x;
    const int k = p.m.k, d = p.m.d;
    constexpr int esz = sizeof(T);
    wait_for_earlier_kernels();
    allow_next_kernel();
    for (int i = tid; i < (int)(sizeof(Routing) / 4); i += kThreads) ((int *)&r)[i] = __ldcg((const int *)p.routing + i);
    __syncthreads();
    if (tid <= r.met) {
        int n = 0;
        for (int s = 0; s < tid; ++s) n += (r.width[s] * esz + kUnit - 1) / kUnit;
        upto[tid] = n;
    }
    __syncthreads();
    const Line line(upto[r.met], d, kRows, gridDim.x, kLeastSpan);
    if ((int)blockIdx.x >= line.blocks) return;
    const long long end = line.begin(blockIdx.x + 1);
    const size_t row = (size_t)p.m.S * esz;
    int round = 0;
    for (long long at = line.begin(blockIdx.x); at < end;) {
        const int group = (int)(at / line.per), lo = (int)(at - (long long)group * line.per), hi = (int)min((long long)line.per, lo + (end - at));
        at += hi - lo;
        __syncthreads();                         // `out` of the group before has been read
        for (int i = tid; i < p.T * kRows; i += kThreads) out[i / kRows][i % kRows] = 0.f;
        const int c0 = group * kRows;
        const unsigned char *w0 = p.w_down + (size_t)min(c0 + g, d - 1) * row, *w1 = p.w_down + (size_t)min(c0 + g + 8, d - 1) * row;
        int s = 0;
        while (upto[s + 1] <= lo) ++s;
        for (; s < r.met && upto[s] < hi; ++s, ++round) {
            const int off = r.offset[s], bytes = r.width[s] * esz;
            const int count = r.first[s + 1] - r.first[s];
            const int *pick = r.pick + r.first[s];
            const unsigned char *x[NTM];
#pragma unroll
            for (int n = 0; n < NTM; ++n) x[n] = p.hidden + pick[min(8 * n + g, count - 1)] * p.ld + t * 16;
            auto &sums = part[round & 1];
            const size_t col = (size_t)off * esz + t * 16;
            dot<T, NTM>(count, w0 + col, w1 + col, x, max(lo, upto[s]) - upto[s], min(hi, upto[s + 1]) - upto[s], bytes, sums[warp]);
            __syncthreads();
            for (int i = tid; i < count * kRows; i += kThreads) {
                const int q = i / kRows, c = i % kRows;
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) v += sums[w][q][c];
                out[pick[q] / k][c] += v;
            }
        }
        __syncthreads();
        // a block leaves its part of the group it begins in at place b, that of the one it ends in (part 0 there) behind all those
        const long long first = (long long)group * line.per;
        const int b0 = owner_of(first, line.length, line.blocks), b1 = owner_of(first + line.per - 1, line.length, line.blocks);
        leave_rows<kRows>(p, group, &out[0][0], blockIdx.x - b0, b1 - b0 + 1, b0, &last, esz == 4 || p.y_f32,
                          line.begin(b0) < first ? kMaxBlocks + b0 : -1);
    }
}

// ---- host ----
constexpr size_t kPartRows = std::max(2 * kMaxBlocks * kRows, kTmaBlocks * 128);      // rows of all parts
constexpr int kMaxExtent = 1 << 26;       // of d and the widths: offsets inside a row are 32 bits of bytes

struct DecodeLayout { size_t routing, arrivals, logits, hidden, part, total; long long ld; };
DecodeLayout decode_layout(const LayerMeta &m, int widest, int esz, int T)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    DecodeLayout L;
    L.routing = 256;                      // behind the status word
    L.ld = (long long)up((size_t)widest * esz);
    L.arrivals = up(L.routing + sizeof(Routing));
    L.logits = up(L.arrivals + (size_t)(m.d + kRows - 1) / kRows * 4);
    L.hidden = up(L.logits + (size_t)2 * T * m.N * 4);
    L.part = L.hidden + (size_t)T * m.k * L.ld;
    L.total = up(L.part + kPartRows * T * 4);
    return L;
}

template <typename T, int NTM>
cudaError_t launch(const DecodeArgs &a, bool tma, int sms, cudaStream_t s)
{
    if (a.logits) {
        const int tiles = (a.m.N + kRows - 1) / kRows * (a.w_noise ? 2 : 1);
        const cudaError_t e = launch_overlapped(decode_logits_kernel<T, NTM>, tiles, kThreads, 0, s, a);
        if (e != cudaSuccess) return e;
    }
    if (tma) return launch_tma(a, sms, s);
    // no more blocks than there is work for if all experts are met
    const int blocks = std::min(kMaxBlocks, blocks_per_sm(NTM) * sms);
    long long line = 0;
    for (int e = 0; e < a.m.N; ++e) line += ((long long)(a.m.hoff[e + 1] - a.m.hoff[e]) * (int)sizeof(T) + kUnit - 1) / kUnit;
    const int groups = (a.m.d + kRows - 1) / kRows;
    line = std::max<long long>(groups, line * groups / kLeastSpan);
    const cudaError_t e = launch_overlapped(decode_up_kernel<T, NTM>, std::min(blocks, a.m.S / kUnitCols), kThreads, 0, s, a);
    return e != cudaSuccess ? e : launch_overlapped(decode_down_kernel<T, NTM>, (int)std::min<long long>(blocks, line), kThreads, 0, s, a);
}
template <typename T>
cudaError_t launch_tokens(const DecodeArgs &a, bool tma, int sms, cudaStream_t s)
{
    if (a.T <= 8) return launch<T, 1>(a, tma, sms, s);
    return a.T <= 16 ? launch<T, 2>(a, tma, sms, s) : launch<T, 4>(a, tma, sms, s);
}

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int widest_of(const LayerMeta &m)
{
    int h = 0;
    for (int e = 0; e < m.N; ++e) h = std::max(h, m.hoff[e + 1] - m.hoff[e]);
    return h;
}

}  // namespace
}  // namespace decode
}  // namespace modse

using namespace modse;
using namespace modse::decode;

extern "C" {

size_t modse_decode_workspace_bytes(const modse_layer_t *layer, modse_dtype_t dtype, int n_tokens)
{
    if (layer == nullptr || (dtype != MODSE_F32 && dtype != MODSE_BF16) || n_tokens < 0 || n_tokens > kMaxTokens) return 0;
    const LayerMeta &m = *layer_meta(layer);
    if (m.d > kMaxExtent || widest_of(m) > kMaxExtent) return 0;
    return decode_layout(m, widest_of(m), dtype == MODSE_F32 ? 4 : 2, n_tokens).total;
}

modse_status_t modse_decode(const modse_layer_t *layer, modse_dtype_t dtype, const modse_weights_t *weights, const void *x,
                            int n_tokens, void *y, int *topk_idx, float *topk_gate, void *workspace, size_t workspace_bytes,
                            void *cuda_stream)
{
    if (layer == nullptr || weights == nullptr || (dtype != MODSE_F32 && dtype != MODSE_BF16) || n_tokens < 0)
        return MODSE_ERR_INVALID_ARG;
    if (n_tokens > kMaxTokens) return MODSE_ERR_UNSUPPORTED;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, (cudaStream_t)cuda_stream);
        return MODSE_OK;
    }
    const modse_weights_t &w = *weights;
    for (const void *q : {w.w_router, w.w_gate, w.w_up, w.w_down, x, (const void *)y})
        if (q == nullptr || !aligned(q, 16)) return MODSE_ERR_INVALID_ARG;
    if (!aligned(topk_idx, 4) || !aligned(topk_gate, 4) || workspace == nullptr || !aligned(workspace, 256)) return MODSE_ERR_INVALID_ARG;
    const LayerMeta &m = *layer_meta(layer);
    if (m.d > kMaxExtent || widest_of(m) > kMaxExtent) return MODSE_ERR_UNSUPPORTED;
    const DecodeLayout L = decode_layout(m, widest_of(m), dtype == MODSE_F32 ? 4 : 2, n_tokens);
    if (workspace_bytes < L.total) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    const NoiseGate &noise = *layer_noise(layer);
    unsigned char *ws = (unsigned char *)workspace;
    DecodeArgs a{};
    a.m = m;
    a.x = (const unsigned char *)x;
    a.w_router = (const unsigned char *)w.w_router;
    a.w_gate = (const unsigned char *)w.w_gate;
    a.w_up = (const unsigned char *)w.w_up;
    a.w_down = (const unsigned char *)w.w_down;
    a.w_noise = (const unsigned char *)noise.w_noise;
    a.gamma = noise.gamma;
    a.eps = noise.eps;
    const int rows = (m.N + kRows - 1) / kRows * kRows * (noise.w_noise ? 2 : 1);
    a.logits = rows > kInBlockExperts ? (float *)(ws + L.logits) : nullptr;
    a.hidden = ws + L.hidden;
    a.ld = L.ld;
    a.routing = (Routing *)(ws + L.routing);
    a.arrivals = (int *)(ws + L.arrivals);
    a.part = (float *)(ws + L.part);
    a.y = y;
    a.topk_idx = topk_idx;
    a.topk_gate = topk_gate;
    a.status = (int *)ws;
    a.wait_limit_ns = tc_wait_limit_ns();
    a.skip_block = tc_skip_tile(kTcDecode);
    a.T = n_tokens;
    a.y_f32 = layer_out_f32(layer);
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == MODSE_F32 ? launch_tokens<float>(a, false, device_sms(), s)
                                             : launch_tokens<__nv_bfloat16>(a, tma_takes(m), device_sms(), s);
    return e == cudaSuccess ? MODSE_OK : MODSE_ERR_CUDA;
}

}  // extern "C"
