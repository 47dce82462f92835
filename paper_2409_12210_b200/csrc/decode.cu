// modse_decode: the whole MoDSE layer for the few tokens of a generation step, in two kernels.
//
//   logits z = x W_g (+ the second term of Eq. 2), top-k, gates g (Eq. 2-3)
//   h_tj = g_tj silu(x_t W_gate^T) (x_t W_up^T) for the experts met,   y_t = sum_j h_tj W_down^T   (Eq. 4)
//
// What bounds it is reading the experts met once, 6 d h bytes each in bf16, so both kernels stream rows of weights straight
// from global memory into mma.sync fragments and keep as many loads in flight as registers hold; tiles of 128 tokens, as
// the grouped products of modse_forward take them, would spend their time on filling and draining themselves.
//
// First kernel: every block works out the routing of all tokens for itself (the router matrix is as large as sixteen rows of
// an expert and comes from L2; handing the result from block to block would cost a launch), then takes units of eight
// hidden columns: their eight rows of W_gate and of W_up fill the sixteen rows of a fragment, so a thread ends up with
// both factors of SwiGLU.  The eight warps of a block split the contraction; their sums meet in shared memory.
// Second kernel: sixteen rows of W_down a fragment, the contraction running over the hidden columns of all experts met.
// The whole of it, rows of fragments times contraction, is one line that is cut into even spans, one a block, wherever
// the cuts fall; a group of rows that several blocks share is added up in the blocks' order by the one that arrives last.
#include <algorithm>

#include "launch.h"
#include "rows_mma.h"

namespace modse {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kRows = 16, kMaxTokens = MODSE_DECODE_MAX_TOKENS, kMaxPicks = 2 * kMaxTokens;
constexpr int kUnit = 64;                 // bytes of a row that the four threads of a group load at a time
constexpr int kUnitCols = 8;              // hidden columns of a unit of the first kernel
constexpr int kInBlockExperts = 32;       // rows of router matrices that every block multiplies by itself
constexpr int blocks_per_sm(int token_groups) { return token_groups == 1 ? 3 : 2; }

// Which experts the tokens meet.  A pick is a token's slot: pick t * k + j.
struct Routing {
    int met;
    int expert[kMaxPicks];                // ascending
    int first[kMaxPicks + 1];             // of each expert's picks in `pick`
    int pick[kMaxPicks];                  // ascending within an expert
    float gate[kMaxPicks];                // by pick
};

struct DecodeArgs {
    LayerMeta m;
    const unsigned char *x, *w_router, *w_gate, *w_up, *w_down, *w_noise;
    float gamma, eps;
    float *logits;                        // [T][N], then x W_n [T][N], where a kernel ahead has formed them; else null
    unsigned char *hidden;                // [T * k][ld] gated hidden rows
    long long ld;                         // bytes
    Routing *routing;
    int *arrivals;                        // of each group of rows of the second kernel
    float *part;                          // [blocks][2][T][16]
    void *y;
    int *topk_idx;
    float *topk_gate;
    int T, y_f32;
};

// Sums over units [u0, u1) of 64 bytes of the products of sixteen rows of w with NT * 8 rows of x, this warp's share of
// them, into part[token][row].  w0, w1: the lane's rows g and g + 8; x: its rows 8 n + g; all from the lane's 16 bytes of
// the first unit on.  `row_bytes` cuts the last unit.
template <typename T> struct Dot;
template <> struct Dot<__nv_bfloat16> {
    template <int NT, int U, int NTM>
    static __device__ __forceinline__ void run(const unsigned char *w0, const unsigned char *w1, const unsigned char *const (&x)[NTM],
                                               int u0, int u1, int row_bytes, float (*part)[kRows + 1])
    {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
        // a warp takes units 2 w, 2 w + 1 of every sixteen
        for (int u = u0 + 2 * warp; u < u1; u += 8 * U) {
            uint4 a[U], b[U], v[U][NT];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int unit = u + (j >> 1) * 16 + (j & 1);
                const size_t at = (size_t)unit * kUnit;
                const bool in = unit < u1 && (int)at + t * 16 < row_bytes;
                a[j] = load_stream(w0 + at, in);
                b[j] = load_stream(w1 + at, in);
#pragma unroll
                for (int n = 0; n < NT; ++n) v[j][n] = load_shared_rows(x[n] + at, in);
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const uint32_t lo[4] = {a[j].x, b[j].x, a[j].y, b[j].y}, hi[4] = {a[j].z, b[j].z, a[j].w, b[j].w};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma_16816(acc[n], lo, v[j][n].x, v[j][n].y, false);
                    mma_16816(acc[n], hi, v[j][n].z, v[j][n].w, false);
                }
            }
        }
        // accumulator (row, token): rows g, g + 8, tokens 8 n + 2 t, + 1
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[8 * n + 2 * t + (i & 1)][g + 8 * (i >> 1)] = acc[n][i];
    }
};
// fp32: each of the four threads of a group adds up its quarter of the contraction for all tokens, whose rows x all of a
// warp reads (from L1)
template <> struct Dot<float> {
    template <int NT, int U, int NTM>
    static __device__ __forceinline__ void run(const unsigned char *w0, const unsigned char *w1, const unsigned char *const (&x)[NTM],
                                               int u0, int u1, int row_bytes, float (*part)[kRows + 1])
    {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float acc[NT * 8][2];
#pragma unroll
        for (int n = 0; n < NT * 8; ++n) acc[n][0] = acc[n][1] = 0.f;
        const uint4 none = make_uint4(0, 0, 0, 0);
        for (int u = u0 + 2 * warp; u < u1; u += 16) {
            uint4 a[2], b[2];
            bool in[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                in[j] = u + j < u1 && (u + j) * kUnit + t * 16 < row_bytes;
                a[j] = load_stream(w0 + (size_t)(u + j) * kUnit, in[j]);
                b[j] = load_stream(w1 + (size_t)(u + j) * kUnit, in[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 p = *reinterpret_cast<const float4 *>(&a[j]), q = *reinterpret_cast<const float4 *>(&b[j]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        // row 8 n + r of x: what lane 4 r + t calls its own
                        const unsigned long long at = __shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(x[n]), 4 * r + t);
                        const uint4 raw = in[j] ? *reinterpret_cast<const uint4 *>(at + (size_t)(u + j) * kUnit) : none;
                        const float4 v = *reinterpret_cast<const float4 *>(&raw);
                        float *s = acc[8 * n + r];
                        s[0] = fmaf(p.x, v.x, fmaf(p.y, v.y, fmaf(p.z, v.z, fmaf(p.w, v.w, s[0]))));
                        s[1] = fmaf(q.x, v.x, fmaf(q.y, v.y, fmaf(q.z, v.z, fmaf(q.w, v.w, s[1]))));
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < NT * 8; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float s = acc[n][i];
                s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
                s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
                if ((n & 3) == t) part[n][g + 8 * i] = s;
            }
    }
};

// ... with as many groups of eight tokens as there are
template <typename T, int NTM>
__device__ __forceinline__ void dot(int nt, const unsigned char *w0, const unsigned char *w1, const unsigned char *const (&x)[NTM],
                                    int u0, int u1, int row_bytes, float (*part)[kRows + 1])
{
    if constexpr (NTM >= 4) {
        if (nt == 4) return Dot<T>::template run<4, 2>(w0, w1, x, u0, u1, row_bytes, part);
        if (nt == 3) return Dot<T>::template run<3, 2>(w0, w1, x, u0, u1, row_bytes, part);
    }
    if constexpr (NTM >= 2)
        if (nt == 2) return Dot<T>::template run<2, 4>(w0, w1, x, u0, u1, row_bytes, part);
    Dot<T>::template run<1, 4>(w0, w1, x, u0, u1, row_bytes, part);
}

template <int NTM> using Part = float[2][kWarps][NTM * 8][kRows + 1];     // two of them, so that one meeting a unit is enough

__device__ __forceinline__ float softplus(float u) { return u > 0.f ? u + log1pf(expf(-u)) : log1pf(expf(u)); }
__device__ __forceinline__ float total(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sixteen rows of the router matrix (tile; those of W_n behind those of W_g) times all tokens: z[t * N + e].
template <typename T, int NTM>
__device__ __forceinline__ void router_tile(const DecodeArgs &p, int tile, float *z, Part<NTM> &part)
{
    const int tiles = (p.m.N + kRows - 1) / kRows, e0 = (tile % tiles) * kRows, last = p.m.N - 1, row = p.m.d * (int)sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned char *w = tile < tiles ? p.w_router : p.w_noise;
    const unsigned char *x[NTM];
#pragma unroll
    for (int n = 0; n < NTM; ++n) x[n] = p.x + (size_t)min(8 * n + g, p.T - 1) * row + t * 16;
    __syncthreads();
    dot<T, NTM>((p.T + 7) / 8, w + (size_t)min(e0 + g, last) * row + t * 16, w + (size_t)min(e0 + g + 8, last) * row + t * 16, x, 0,
                (row + kUnit - 1) / kUnit, row, part[0][warp]);
    __syncthreads();
    z += tile < tiles ? 0 : p.T * p.m.N;
    for (int i = threadIdx.x; i < p.T * kRows; i += kThreads) {
        const int tok = i / kRows, c = i % kRows;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < kWarps; ++v) s += part[0][v][tok][c];
        if (e0 + c < p.m.N) z[tok * p.m.N + e0 + c] = s;
    }
}

// Larger z first, then the lower index; a NaN counts as the least of all.
__device__ __forceinline__ void take_better(float v, int i, float &bv, int &bi)
{
    if (v > bv || (v == bv && i < bi)) {
        bv = v;
        bi = i;
    }
}
__device__ __forceinline__ void warp_best(float &bv, int &bi)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xFFFFFFFFu, bv, o);
        const int i = __shfl_xor_sync(0xFFFFFFFFu, bi, o);
        take_better(v, i, bv, bi);
    }
}

// Top-k and gates of every token from its logits, a warp a token, and the picks sorted by expert.
__device__ __forceinline__ void route(const DecodeArgs &p, const float *z, int *idx, int *scan, Routing &r)
{
    constexpr int kPer = kMaxExperts / 32;
    const int N = p.m.N, k = p.m.k, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    const float *u = z + p.T * N;
    for (int t = warp; t < p.T; t += kWarps) {
        float v[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = lane + 32 * i < N ? z[t * N + lane + 32 * i] : 0.f;
        if (p.w_noise) {
            float s[kPer], ss = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                s[i] = lane + 32 * i < N ? softplus(u[t * N + lane + 32 * i]) : 0.f;
                ss = fmaf(s[i], s[i], ss);
            }
            const float scale = p.gamma / sqrtf(total(ss) / (float)N + p.eps);
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] = fmaf(s[i], scale, v[i]);
        }
        float best[2];
        int at[2] = {-1, -1};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (j >= k) break;
            float bv = -INFINITY;
            int bi = 1 << 30;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = lane + 32 * i;
                if (e < N && e != at[0]) take_better(isnan(v[i]) ? -INFINITY : v[i], e, bv, bi);
            }
            warp_best(bv, bi);
            at[j] = bi;
            float mine = 0.f;             // the logit itself, NaN or not, from the lane that holds it
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i == (bi >> 5)) mine = v[i];
            best[j] = __shfl_sync(0xFFFFFFFFu, mine, bi & 31);
        }
        if (lane == 0) {
            if (k == 1) {
                idx[t] = at[0];
                r.gate[t] = 1.f;
            } else {
                const float e = expf(best[1] - best[0]), den = 1.f + e;
                idx[2 * t] = at[0];
                idx[2 * t + 1] = at[1];
                r.gate[2 * t] = 1.f / den;
                r.gate[2 * t + 1] = e / den;
            }
        }
    }
    __syncthreads();
    // thread e looks for expert e among the picks
    const int picks = p.T * k;
    int mine = 0, before = 0;
    for (int a = 0; a < picks; ++a) {
        mine += idx[a] == tid;
        before += idx[a] < tid;
    }
    const unsigned have = __ballot_sync(0xFFFFFFFFu, mine > 0);
    if (lane == 0) scan[warp] = __popc(have);
    __syncthreads();
    int place = __popc(have & ((1u << lane) - 1u)), met = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        place += w < warp ? scan[w] : 0;
        met += scan[w];
    }
    if (mine > 0) {
        r.expert[place] = tid;
        r.first[place] = before;
        for (int a = 0; a < picks; ++a)
            if (idx[a] == tid) r.pick[before++] = a;
    }
    if (tid == 0) {
        r.met = met;
        r.first[met] = picks;
    }
    __syncthreads();
}

// The logits ahead of the first kernel, for layers of so many experts that every block forming them would cost more than a
// launch: a block sixteen experts.
template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads) decode_logits_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ Part<NTM> part;
    wait_for_earlier_kernels();
    allow_next_kernel();
    router_tile<T, NTM>(p, blockIdx.x, p.logits, part);
}

template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NTM)) decode_up_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ Part<NTM> part;
    __shared__ Routing r;
    __shared__ float z[NTM * 8 * kInBlockExperts];
    __shared__ int idx[kMaxPicks], scan[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int k = p.m.k, row = p.m.d * (int)sizeof(T), units = (row + kUnit - 1) / kUnit;
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (p.logits == nullptr) {
        const int tiles = (p.m.N + kRows - 1) / kRows * (p.w_noise ? 2 : 1);
        for (int i = 0; i < tiles; ++i) router_tile<T, NTM>(p, i, z, part);
        __syncthreads();
    }
    route(p, p.logits ? p.logits : z, idx, scan, r);
    if (blockIdx.x == 0) {
        // for the second kernel and the caller
        for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += kThreads) ((int *)p.routing)[i] = ((const int *)&r)[i];
        for (int i = threadIdx.x; i < (p.m.d + kRows - 1) / kRows; i += kThreads) p.arrivals[i] = 0;
        if (threadIdx.x < p.T * k) {
            if (p.topk_idx) p.topk_idx[threadIdx.x] = idx[threadIdx.x];
            if (p.topk_gate) p.topk_gate[threadIdx.x] = r.gate[threadIdx.x];
        }
    }
    int s = 0, base = 0, round = 0;                          // expert of the unit, units ahead of it
    for (int u = blockIdx.x;; u += gridDim.x, ++round) {
        int width = 0;
        while (s < r.met) {
            width = p.m.hoff[r.expert[s] + 1] - p.m.hoff[r.expert[s]];
            if (u - base < width / kUnitCols) break;
            base += width / kUnitCols;
            ++s;
        }
        if (s >= r.met) break;
        const int count = r.first[s + 1] - r.first[s], c0 = (u - base) * kUnitCols;
        const int *pick = r.pick + r.first[s];
        const size_t at = ((size_t)p.m.hoff[r.expert[s]] + c0 + g) * row + t * 16;
        const unsigned char *x[NTM];
#pragma unroll
        for (int n = 0; n < NTM; ++n) x[n] = p.x + (size_t)(pick[min(8 * n + g, count - 1)] / k) * row + t * 16;
        auto &sums = part[round & 1];
        dot<T, NTM>((count + 7) / 8, p.w_gate + at, p.w_up + at, x, 0, units, row, sums[warp]);
        __syncthreads();
        if (threadIdx.x < count * kUnitCols) {
            const int i = threadIdx.x / kUnitCols, c = threadIdx.x % kUnitCols;
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                a += sums[w][i][c];
                b += sums[w][i][c + kUnitCols];
            }
            // one rounding of the gated hidden value, as in modse_forward
            const float h = r.gate[pick[i]] * (a / (1.f + expf(-a))) * b;
            T *out = reinterpret_cast<T *>(p.hidden + pick[i] * p.ld) + c0 + c;
            if constexpr (sizeof(T) == 2) *out = __float2bfloat16_rn(h);
            else *out = h;
        }
    }
}

// The block that position `at` of a line of `length` positions belongs to, when `blocks` share it evenly.
__device__ __forceinline__ int owner_of(long long at, long long length, int blocks) { return (int)(((at + 1) * blocks - 1) / length); }

template <typename T, int NTM>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NTM)) decode_down_kernel(const __grid_constant__ DecodeArgs p)
{
    __shared__ Part<NTM> part;
    __shared__ Routing r;
    __shared__ int upto[kMaxPicks + 1];          // units ahead of each expert met
    __shared__ float out[NTM * 8][kRows];
    __shared__ int last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, tid = threadIdx.x;
    const int k = p.m.k, d = p.m.d;
    constexpr int esz = sizeof(T);
    wait_for_earlier_kernels();
    allow_next_kernel();
    for (int i = tid; i < (int)(sizeof(Routing) / 4); i += kThreads) ((int *)&r)[i] = __ldcg((const int *)p.routing + i);
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int s = 0; s < r.met; ++s) {
            upto[s] = n;
            n += ((p.m.hoff[r.expert[s] + 1] - p.m.hoff[r.expert[s]]) * esz + kUnit - 1) / kUnit;
        }
        upto[r.met] = n;
    }
    __syncthreads();
    const int per = upto[r.met], groups = (d + kRows - 1) / kRows;
    const long long length = (long long)per * groups;
    const int blocks = (int)min((long long)gridDim.x, length);
    if ((int)blockIdx.x >= blocks) return;
    const long long begin = length * blockIdx.x / blocks, end = length * (blockIdx.x + 1) / blocks;
    int round = 0;
    for (long long at = begin; at < end;) {
        const int group = (int)(at / per), lo = (int)(at - (long long)group * per), hi = (int)min((long long)per, lo + (end - at));
        at += hi - lo;
        __syncthreads();                         // `out` of the group before has been read
        for (int i = tid; i < p.T * kRows; i += kThreads) out[i / kRows][i % kRows] = 0.f;
        const int c0 = group * kRows;
        const size_t line = (size_t)p.m.S * esz;
        const unsigned char *w0 = p.w_down + (size_t)min(c0 + g, d - 1) * line, *w1 = p.w_down + (size_t)min(c0 + g + 8, d - 1) * line;
        int s = 0;
        while (upto[s + 1] <= lo) ++s;
        for (; s < r.met && upto[s] < hi; ++s, ++round) {
            const int off = p.m.hoff[r.expert[s]], bytes = (p.m.hoff[r.expert[s] + 1] - off) * esz;
            const int count = r.first[s + 1] - r.first[s];
            const int *pick = r.pick + r.first[s];
            const unsigned char *x[NTM];
#pragma unroll
            for (int n = 0; n < NTM; ++n) x[n] = p.hidden + pick[min(8 * n + g, count - 1)] * p.ld + t * 16;
            auto &sums = part[round & 1];
            const size_t col = (size_t)off * esz + t * 16;
            dot<T, NTM>((count + 7) / 8, w0 + col, w1 + col, x, max(lo, upto[s]) - upto[s], min(hi, upto[s + 1]) - upto[s], bytes, sums[warp]);
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
        const long long first = (long long)group * per;
        const int b0 = owner_of(first, length, blocks), b1 = owner_of(first + per - 1, length, blocks);
        // a block leaves the part of the group it begins in first and that of the one it ends in second
        auto place = [&](int b) { return p.part + ((size_t)b * 2 + (b == b0 && length * b / blocks < first ? 1 : 0)) * p.T * kRows; };
        if (b0 != b1) {
            for (int i = tid; i < p.T * kRows; i += kThreads) __stcg(place(blockIdx.x) + i, out[i / kRows][i % kRows]);
            __threadfence();
            __syncthreads();
            if (tid == 0) last = atomicAdd(p.arrivals + group, 1) == b1 - b0;
            __syncthreads();
            if (!last) continue;
            __threadfence();
        }
        for (int i = tid; i < p.T * kRows; i += kThreads) {
            const int tok = i / kRows, c = i % kRows;
            if (c0 + c >= d) continue;
            float v = 0.f;
            if (b0 == b1) v = out[tok][c];
            else
                for (int b = b0; b <= b1; ++b) v += __ldcg(place(b) + i);
            const size_t to = (size_t)tok * d + c0 + c;
            if (esz == 4 || p.y_f32) static_cast<float *>(p.y)[to] = v;
            else static_cast<__nv_bfloat16 *>(p.y)[to] = __float2bfloat16_rn(v);
        }
    }
}

// ---- host ----
constexpr int kMaxBlocks = 3 * 148;       // workspace sizes are asked for without a device
constexpr int kMaxExtent = 1 << 26;       // of d and the widths: offsets inside a row are 32 bits of bytes

struct DecodeLayout { size_t arrivals, logits, hidden, part, total; long long ld; };
DecodeLayout decode_layout(const LayerMeta &m, int widest, int esz, int T)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    DecodeLayout L;
    L.ld = (long long)up((size_t)widest * esz);
    L.arrivals = up(sizeof(Routing));
    L.logits = up(L.arrivals + (size_t)(m.d + kRows - 1) / kRows * 4);
    L.hidden = up(L.logits + (size_t)2 * T * m.N * 4);
    L.part = L.hidden + (size_t)T * m.k * L.ld;
    L.total = up(L.part + (size_t)kMaxBlocks * 2 * T * kRows * 4);
    return L;
}

template <typename T, int NTM>
cudaError_t launch(DecodeArgs &a, int sms, cudaStream_t s)
{
    if (a.logits) {
        const int tiles = (a.m.N + kRows - 1) / kRows * (a.w_noise ? 2 : 1);
        const cudaError_t e = launch_overlapped(decode_logits_kernel<T, NTM>, tiles, kThreads, 0, s, a);
        if (e != cudaSuccess) return e;
    }
    const int blocks = std::min(kMaxBlocks, blocks_per_sm(NTM) * sms);
    const cudaError_t e = launch_overlapped(decode_up_kernel<T, NTM>, blocks, kThreads, 0, s, a);
    return e != cudaSuccess ? e : launch_overlapped(decode_down_kernel<T, NTM>, blocks, kThreads, 0, s, a);
}
template <typename T>
cudaError_t launch_tokens(DecodeArgs &a, int sms, cudaStream_t s)
{
    if (a.T <= 8) return launch<T, 1>(a, sms, s);
    return a.T <= 16 ? launch<T, 2>(a, sms, s) : launch<T, 4>(a, sms, s);
}

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int widest_of(const LayerMeta &m)
{
    int h = 0;
    for (int e = 0; e < m.N; ++e) h = std::max(h, m.hoff[e + 1] - m.hoff[e]);
    return h;
}

}  // namespace
}  // namespace modse

using namespace modse;

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
    if (n_tokens == 0) return MODSE_OK;
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
    a.routing = (Routing *)ws;
    a.arrivals = (int *)(ws + L.arrivals);
    a.part = (float *)(ws + L.part);
    a.y = y;
    a.topk_idx = topk_idx;
    a.topk_gate = topk_gate;
    a.T = n_tokens;
    a.y_f32 = layer_out_f32(layer);
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == MODSE_F32 ? launch_tokens<float>(a, device_sms(), s) : launch_tokens<__nv_bfloat16>(a, device_sms(), s);
    return e == cudaSuccess ? MODSE_OK : MODSE_ERR_CUDA;
}

}  // extern "C"
