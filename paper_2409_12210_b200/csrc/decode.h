// modse_decode: what its kernels share - the routing of a few tokens, which every block works out for itself, and the even
// cut of the second product.
#pragma once

#include "launch.h"
#include "rows_mma.h"

namespace modse {
namespace decode {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kRows = 16, kMaxTokens = MODSE_DECODE_MAX_TOKENS, kMaxPicks = 2 * kMaxTokens;
constexpr int kUnit = 64;                 // bytes of a row that the four threads of a group load at a time
constexpr int kUnitCols = 8;              // hidden columns of a unit of the first kernel
constexpr int kInBlockExperts = 32;       // rows of router matrices that every block multiplies by itself

// Which experts the tokens meet.  A pick is a token's slot: pick t * k + j.
struct Routing {
    int met;
    int offset[kMaxPicks], width[kMaxPicks];      // of the experts met, ascending
    int first[kMaxPicks + 1];             // of each expert's picks in `pick`
    int pick[kMaxPicks];                  // ascending within an expert
    float gate[kMaxPicks];                // by pick
};

struct DecodeArgs {
    LayerMeta m;
    const unsigned char *x, *w_router, *w_gate, *w_up, *w_down, *w_noise;
    float gamma, eps;
    float *logits;                        // [T][N], then x W_n [T][N], where a kernel ahead has formed them; else null
    unsigned char *hidden;                // [T * k][ld] gated hidden rows, by pick or (decode_tma.cu) by place in Routing::pick
    long long ld;                         // bytes
    Routing *routing;
    int *arrivals;                        // of each group of rows of the second kernel
    float *part;                          // [blocks][2][T][rows of a group]
    void *y;
    int *topk_idx;
    float *topk_gate;
    int *status;
    unsigned long long wait_limit_ns;
    int x_room;                           // bytes of shared memory for rows of x
    int up_blocks;                        // column blocks of a stage of decode_up_few
    int skip_block;                       // debugging: the block that stops loading weights (-1: none)
    int T, y_f32;
};

// Meeting of the first kThreads threads of a block.
__device__ __forceinline__ void team_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

// Sums over units [u0, u1) of 64 bytes of the products of sixteen rows of w with NT * 8 rows of x, this warp's share of
// them, into part[token][row].  w0, w1: the lane's rows g and g + 8; x: its rows 8 n + g; all from the lane's 16 bytes of
// the first unit on.  `row_bytes` cuts the last unit.
template <typename T> struct Dot;
template <> struct Dot<__nv_bfloat16> {
    template <int NT, int U, int NTM>
    static __device__ __forceinline__ void run(int tokens, const unsigned char *w0, const unsigned char *w1,
                                               const unsigned char *const (&x)[NTM], int u0, int u1, int row_bytes, float (*part)[kRows + 1])
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
    static __device__ __forceinline__ void run(int tokens, const unsigned char *w0, const unsigned char *w1,
                                               const unsigned char *const (&x)[NTM], int u0, int u1, int row_bytes, float (*part)[kRows + 1])
    {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float acc[NT * 8][2];
#pragma unroll
        for (int n = 0; n < NT * 8; ++n) acc[n][0] = acc[n][1] = 0.f;
        const uint4 none = make_uint4(0, 0, 0, 0);
        // a warp takes units 2 w, 2 w + 1 of every sixteen (four units in flight take longer: 8 tokens through eight experts of
        // 5632 x 2048 on average 243 us, with two 224)
        for (int u = u0 + 2 * warp; u < u1; u += 16) {
            uint4 a[2], b[2];
            bool in[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                in[j] = u + j < u1 && (u + j) * kUnit + t * 16 < row_bytes;
                a[j] = load_stream(w0 + (size_t)(u + j) * kUnit, in[j]);
                b[j] = load_stream(w1 + (size_t)(u + j) * kUnit, in[j]);
            }
            // token i's row of x: what lane 4 (i mod 8) + t calls its own
            auto row_of_token = [&](int i) { return __shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(x[i / 8]), 4 * (i % 8) + t); };
            auto add = [&](int j, int i, unsigned long long row) {
                const float4 p = *reinterpret_cast<const float4 *>(&a[j]), q = *reinterpret_cast<const float4 *>(&b[j]);
                const uint4 raw = in[j] ? *reinterpret_cast<const uint4 *>(row + (size_t)(u + j) * kUnit) : none;
                const float4 v = *reinterpret_cast<const float4 *>(&raw);
                acc[i][0] = fmaf(p.x, v.x, fmaf(p.y, v.y, fmaf(p.z, v.z, fmaf(p.w, v.w, acc[i][0]))));
                acc[i][1] = fmaf(q.x, v.x, fmaf(q.y, v.y, fmaf(q.z, v.z, fmaf(q.w, v.w, acc[i][1]))));
            };
            if constexpr (NT == 1) {
                // only the tokens that are there (1 token through that layer 110 -> 64 us; with more groups than one, skipping
                // costs more than it saves: 32 tokens of 1000 171 us against 136)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i >= tokens) break;
                    const unsigned long long row = row_of_token(i);
#pragma unroll
                    for (int j = 0; j < 2; ++j) add(j, i, row);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < NT * 8; ++i) add(j, i, row_of_token(i));
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

// ... with as many groups of eight tokens as there are, U1 units in flight with one of them.
template <typename T, int NTM, int U1 = 4>
__device__ __forceinline__ void dot(int tokens, const unsigned char *w0, const unsigned char *w1, const unsigned char *const (&x)[NTM],
                                    int u0, int u1, int row_bytes, float (*part)[kRows + 1])
{
    const int nt = (tokens + 7) / 8;
    if constexpr (NTM >= 4) {
        if (nt == 4) return Dot<T>::template run<4, 2>(tokens, w0, w1, x, u0, u1, row_bytes, part);
        if (nt == 3) return Dot<T>::template run<3, 2>(tokens, w0, w1, x, u0, u1, row_bytes, part);
    }
    if constexpr (NTM >= 2)
        if (nt == 2) return Dot<T>::template run<2, 4>(tokens, w0, w1, x, u0, u1, row_bytes, part);
    Dot<T>::template run<1, U1>(tokens, w0, w1, x, u0, u1, row_bytes, part);
}

__device__ __forceinline__ float softplus(float u) { return u > 0.f ? u + log1pf(expf(-u)) : log1pf(expf(u)); }
__device__ __forceinline__ float total(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sixteen rows of the router matrix (tile; those of W_n behind those of W_g) times all tokens: z[t * N + e].
template <typename T, int NTM>
__device__ __forceinline__ void router_tile(const DecodeArgs &p, int tile, float *z, float (&part)[kWarps][NTM * 8][kRows + 1])
{
    const int tiles = (p.m.N + kRows - 1) / kRows, e0 = (tile % tiles) * kRows, last = p.m.N - 1, row = p.m.d * (int)sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned char *w = tile < tiles ? p.w_router : p.w_noise;
    const unsigned char *x[NTM];
#pragma unroll
    for (int n = 0; n < NTM; ++n) x[n] = p.x + (size_t)min(8 * n + g, p.T - 1) * row + t * 16;
    team_sync();
    dot<T, NTM, 8>(p.T, w + (size_t)min(e0 + g, last) * row + t * 16, w + (size_t)min(e0 + g + 8, last) * row + t * 16, x, 0,
                (row + kUnit - 1) / kUnit, row, part[warp]);
    team_sync();
    z += tile < tiles ? 0 : p.T * p.m.N;
    for (int i = threadIdx.x; i < p.T * kRows; i += kThreads) {
        const int tok = i / kRows, c = i % kRows;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < kWarps; ++v) s += part[v][tok][c];
        if (e0 + c < p.m.N) z[tok * p.m.N + e0 + c] = s;
    }
}

// Integers in the order of logits: -0 and 0 are equal, and a NaN is larger than any number, so that it is kept and shows in the
// gates.  (As comparisons of floats, with the questions after a NaN in the chain of selections, 7 tokens through four experts
// took 45.0 us instead of 44.)
__device__ __forceinline__ int rank_of(float z)
{
    const int bits = __float_as_int(z + 0.f);
    return isnan(z) ? 0x7FFFFFFF : bits ^ ((bits >> 31) & 0x7FFFFFFF);
}
// Larger rank first, then the lower index.
__device__ __forceinline__ void take_better(int v, int i, int &bv, int &bi)
{
    if (v > bv || (v == bv && i < bi)) {
        bv = v;
        bi = i;
    }
}
__device__ __forceinline__ void warp_best(int &bv, int &bi)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const int v = __shfl_xor_sync(0xFFFFFFFFu, bv, o);
        const int i = __shfl_xor_sync(0xFFFFFFFFu, bi, o);
        take_better(v, i, bv, bi);
    }
}

// Top-k and gates of every token, a warp a token, and the picks sorted by expert.  mem: room for the logits.
template <typename T, int NTM>
__device__ __forceinline__ void route(const DecodeArgs &p, float *mem, float (&part)[kWarps][NTM * 8][kRows + 1], int *idx, int *scan, Routing &r)
{
    constexpr int kPer = kMaxExperts / 32;
    if (p.logits == nullptr) {
        const int tiles = (p.m.N + kRows - 1) / kRows * (p.w_noise ? 2 : 1);
        for (int i = 0; i < tiles; ++i) router_tile<T, NTM>(p, i, mem, part);
        team_sync();
    }
    const float *z = p.logits ? p.logits : mem;
    const int N = p.m.N, k = p.m.k, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    const float *u = z + p.T * N;
    auto gates = [&](int t, int e0, int e1, float z0, float z1) {
        if (k == 1) {
            idx[t] = e0;
            r.gate[t] = isnan(z0) ? z0 : 1.f;
        } else {
            const float e = expf(z1 - z0), den = 1.f + e;
            idx[2 * t] = e0;
            idx[2 * t + 1] = e1;
            r.gate[2 * t] = 1.f / den;
            r.gate[2 * t + 1] = e / den;
        }
    };
    if (N <= 32) {
        // few experts: a thread a token, which looks at one logit after the other
        if (tid < p.T) {
            const float *zt = z + tid * N, *ut = u + tid * N;
            float scale = 0.f;
            if (p.w_noise) {
                float ss = 0.f;
                for (int e = 0; e < N; ++e) {
                    const float s = softplus(ut[e]);
                    ss = fmaf(s, s, ss);
                }
                scale = p.gamma / sqrtf(ss / (float)N + p.eps);
            }
            int best[2] = {0, 0};
            float raw[2] = {0.f, 0.f};
            int at[2] = {-1, -1};
            for (int e0 = 0; e0 < N; e0 += 8) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = e0 + i < N ? zt[e0 + i] : 0.f;
                if (p.w_noise)
                    for (int i = 0; i < 8; ++i)
                        if (e0 + i < N) v[i] = fmaf(softplus(ut[e0 + i]), scale, v[i]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (e0 + i >= N) break;
                    const int c = rank_of(v[i]);
                    const bool top = at[0] < 0 || c > best[0], next = !top && (at[1] < 0 || c > best[1]);
                    best[1] = top ? best[0] : next ? c : best[1];
                    raw[1] = top ? raw[0] : next ? v[i] : raw[1];
                    at[1] = top ? at[0] : next ? e0 + i : at[1];
                    best[0] = top ? c : best[0];
                    raw[0] = top ? v[i] : raw[0];
                    at[0] = top ? e0 + i : at[0];
                }
            }
            gates(tid, at[0], at[1], raw[0], raw[1]);
        }
    } else {
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
            float best[2] = {0.f, 0.f};
            int at[2] = {-1, -1};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (j >= k) break;
                int bv = -0x7FFFFFFF - 1;
                int bi = 1 << 30;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int e = lane + 32 * i;
                    if (e < N && e != at[0]) take_better(rank_of(v[i]), e, bv, bi);
                }
                warp_best(bv, bi);
                at[j] = bi;
                float mine = 0.f;             // the logit itself, NaN or not, from the lane that holds it
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (i == (bi >> 5)) mine = v[i];
                best[j] = __shfl_sync(0xFFFFFFFFu, mine, bi & 31);
            }
            if (lane == 0) gates(t, at[0], at[1], best[0], best[1]);
        }
    }
    // The picks sorted by expert: a thread a pick, which compares it with all others (in fours; what is past the end is
    // larger than any expert).
    const int picks = p.T * k;
    if (tid >= picks && tid < kMaxPicks) idx[tid] = kMaxExperts;
    team_sync();
    int before = 0, mine = 0, e = kMaxExperts;
    const int4 *four = reinterpret_cast<const int4 *>(idx);
    if (tid < picks) {
        e = idx[tid];
        bool first = true;
        for (int i = 0; 4 * i < picks; ++i) {
            const int4 o = four[i];
            const int v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                before += v[c] < e;
                const bool same_ahead = v[c] == e && 4 * i + c < tid;
                mine += same_ahead;
                first = first && !same_ahead;
            }
        }
        r.pick[before + mine] = tid;
        scan[tid] = first ? e : kMaxExperts;      // an expert met, from the first token that meets it
    }
    if (tid >= picks && tid < kMaxPicks) scan[tid] = kMaxExperts;
    team_sync();
    int place = 0, met = 0;
    if (tid < picks) {
        four = reinterpret_cast<const int4 *>(scan);
        for (int i = 0; 4 * i < picks; ++i) {
            const int4 o = four[i];
            place += (o.x < e) + (o.y < e) + (o.z < e) + (o.w < e);
            met += (o.x < kMaxExperts) + (o.y < kMaxExperts) + (o.z < kMaxExperts) + (o.w < kMaxExperts);
        }
        if (mine == 0) {
            r.offset[place] = p.m.hoff[e];
            r.width[place] = p.m.hoff[e + 1] - p.m.hoff[e];
            r.first[place] = before;
        }
        if (tid == 0) {
            r.met = met;
            r.first[met] = picks;
        }
    }
    team_sync();
}

// Before the kernels ahead have ended: the router matrix on its way to L2, where every block reads it a moment later.
__device__ __forceinline__ void fetch_router(const DecodeArgs &p, int row_bytes)
{
    const size_t bytes = (size_t)p.m.N * row_bytes, at = ((size_t)blockIdx.x * blockDim.x + threadIdx.x) * 128;
    if (at < bytes) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.w_router + at));
}

// Block b's even share [begin, end) of n units.
__device__ __forceinline__ void share_of(int n, int &begin, int &end)
{
    const int b = blockIdx.x, each = n / (int)gridDim.x, more = n - each * (int)gridDim.x;
    begin = each * b + min(b, more);
    end = begin + each + (b < more);
}

// For the second kernel and the caller, by one block of the first.
__device__ __forceinline__ void publish(const DecodeArgs &p, const Routing &r, const int *idx)
{
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += kThreads) ((int *)p.routing)[i] = ((const int *)&r)[i];
    for (int i = threadIdx.x; i < (p.m.d + kRows - 1) / kRows; i += kThreads) p.arrivals[i] = 0;
    if (threadIdx.x < p.T * p.m.k) {
        if (p.topk_idx) p.topk_idx[threadIdx.x] = idx[threadIdx.x];
        if (p.topk_gate) p.topk_gate[threadIdx.x] = r.gate[threadIdx.x];
    }
    if (threadIdx.x == 0) *p.status = kDevOk;
}

// A unit of the first kernel: eight hidden columns of an expert met.
struct UnitCursor {
    int u, s, base, c0;                   // unit, its expert's place among those met, units ahead of that expert, first column
    __device__ __forceinline__ bool settle(const Routing &r)
    {
        while (s < r.met) {
            const int units = r.width[s] / kUnitCols;
            if (u - base < units) {
                c0 = (u - base) * kUnitCols;
                return true;
            }
            base += units;
            ++s;
        }
        return false;
    }
};

__device__ __forceinline__ float gated(float gate, float a, float b) { return gate * (a / (1.f + expf(-a))) * b; }

// The block that position `at` of a line of `length` positions belongs to, when `blocks` share it evenly.
__device__ __forceinline__ int owner_of(long long at, long long length, int blocks) { return (int)(((at + 1) * blocks - 1) / length); }

// The second kernel's line: for every group of rows of W_down (sixteen, or more) the units of the contraction over all experts met.  The
// blocks take even spans of it, wherever the cuts fall: a block a group at least, and more where there is more to do than a meeting costs.
struct Line {
    int per, blocks;                      // units of a group of rows
    long long length;
    __device__ __forceinline__ Line(int per_group, int d, int rows, int most_blocks, int least_span)
        : per(per_group), length((long long)per_group * ((d + rows - 1) / rows))
    {
        blocks = (int)min((long long)most_blocks, max((long long)((d + rows - 1) / rows), length / least_span));
    }
    __device__ __forceinline__ long long begin(int block) const { return length * block / blocks; }
};

// out[token][row], one of `share` blocks' part of the sums of a group of ROWS rows, to y; where there are several it goes to place
// slot + member of the workspace, and the block that arrives last adds the parts in order.  All threads of the team.
// first_slot: the place that part 0 takes instead (negative: none).
template <int ROWS>
__device__ __forceinline__ void leave_rows(const DecodeArgs &p, int group, const float *out, int member, int share, long long slot, int *last,
                                           bool f32, long long first_slot = -1)
{
    const int tid = threadIdx.x, d = p.m.d, c0 = group * ROWS;
    auto place = [&](int m) { return p.part + (m == 0 && first_slot >= 0 ? first_slot : slot + m) * (long long)(p.T * ROWS); };
    if (share > 1) {
        for (int i = 4 * tid; i < p.T * ROWS; i += 4 * kThreads)
            __stcg(reinterpret_cast<float4 *>(place(member) + i), *reinterpret_cast<const float4 *>(out + i));
        __threadfence();
        team_sync();
        if (tid == 0) *last = atomicAdd(p.arrivals + group, 1) == share - 1;
        team_sync();
        if (!*last) return;
        __threadfence();
    }
    // four neighbouring rows of a token a thread; many loads in flight
    for (int i = 4 * tid; i < p.T * ROWS; i += 4 * kThreads) {
        const int tok = i / ROWS, c = i % ROWS;
        if (c0 + c >= d) continue;               // (d is a multiple of 8)
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (share == 1) {
            v = *reinterpret_cast<const float4 *>(out + i);
        } else {
#pragma unroll 8
            for (int m = 0; m < share; ++m) {
                const float4 u = __ldcg(reinterpret_cast<const float4 *>(place(m) + i));
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
        }
        const size_t to = (size_t)tok * d + c0 + c;
        if (f32) {
            *reinterpret_cast<float4 *>(static_cast<float *>(p.y) + to) = v;
        } else {
            __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
            *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.y) + to) = make_uint2(*reinterpret_cast<uint32_t *>(&a), *reinterpret_cast<uint32_t *>(&b));
        }
    }
}

// The products with weights that TMA brings (decode_tma.cu): bf16, d and all widths multiples of 64.
bool tma_takes(const LayerMeta &m);
constexpr int kTmaBlocks = 148;           // workspace sizes are asked for without a device
cudaError_t launch_tma(const DecodeArgs &a, int sms, cudaStream_t s);

}  // namespace decode
}  // namespace modse
