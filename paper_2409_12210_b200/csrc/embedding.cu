// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   y_t = scale E[id_t];     dE_v = scale sum over t with id_t = v, ascending, of dy_t
//
// Both are bound by HBM: a row of the table or of dy is read once, a row of the result written once.  Lookup of 65536 rows of
// 2048 bf16 numbers out of 32000: 55 us, 7.3 TB/s, some of the table out of L2.
//
// Gradient, two kernels.  Atomic additions would make the result depend on the order of arrival, so the positions are
// sorted by token first (stable, least significant digit first): one cluster of eight blocks does all passes, each of its
// 256 warps owning a contiguous run of positions and a histogram of its own, so a pass is a count, a prefix over warps and
// blocks (through distributed shared memory) and a scatter, without tiles.  The second kernel has two kinds of blocks.  The
// first write zeros into the rows that no token names, which needs no sorted order, so they start beside the sort.  The
// others each take a chunk of sorted positions and a slab of columns and add up the rows of a token in order; sums of a
// token whose positions lie in several chunks meet in the workspace, where the block that arrives last adds them in the
// chunks' order.  16384 rows of dy of 2048 bf16 numbers into 32000 (fp32) rows: 70 us for 329 MB, 4.7 TB/s; the
// 14 us of the sort are hidden by the zeros.  Added to what is there, with no zeros to write, the sort stands in front: 57 us, of
// which the rows of dy and the 5836 rows that are touched (163 MB) take 25.
#include <algorithm>

#include "dense_gemm.h"
#include "launch.h"
#include "modse_internal.h"
#include "tc_device.h"

namespace modse {
namespace {

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename T> struct Piece;                    // 8 elements as they lie in memory
template <> struct Piece<__nv_bfloat16> { uint4 a; };
template <> struct Piece<float> { float4 a, b; };

// Plain loads: a kernel ahead that is still running when this one starts may have written what is read.
__device__ __forceinline__ void load_piece(Piece<__nv_bfloat16> &v, const __nv_bfloat16 *p) { v.a = *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void load_piece(Piece<float> &v, const float *p)
{
    v.a = *reinterpret_cast<const float4 *>(p);
    v.b = *reinterpret_cast<const float4 *>(p + 4);
}
__device__ __forceinline__ void unpack_piece(const Piece<__nv_bfloat16> &v, float (&f)[8])
{
    const uint32_t w[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack_piece(const Piece<float> &v, float (&f)[8])
{
    f[0] = v.a.x; f[1] = v.a.y; f[2] = v.a.z; f[3] = v.a.w;
    f[4] = v.b.x; f[5] = v.b.y; f[6] = v.b.z; f[7] = v.b.w;
}
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&t);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_piece(float *p, const float (&f)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

// ---- lookup ----
constexpr int kLookupThreads = 256, kLookupFlight = 4;

// A row belongs to `tpr` threads (a power of two); each has kLookupFlight pieces of 8 elements of it in flight.
template <typename T>
__global__ void __launch_bounds__(kLookupThreads)
embedding_kernel(const TokenIds ids, const T *table, float scale, T *y, int *status, int n, int d, int vocabulary, int tpr)
{
    wait_for_earlier_kernels();
    allow_next_kernel();
    const int per_block = kLookupThreads / tpr, at = threadIdx.x & (tpr - 1);
    const long long row = (long long)blockIdx.x * per_block + threadIdx.x / tpr;
    if (row >= n) return;
    const long long id = ids.at(row);
    const bool in = id >= 0 && id < vocabulary;
    if (id >= vocabulary && status != nullptr && at == 0) atomicMax(status, kDevBounds);
    const T *src = table + (in ? id : 0) * d;
    T *dst = y + row * d;
    const int pieces = d >> 3;
    for (int c0 = at; c0 < pieces; c0 += kLookupFlight * tpr) {
        Piece<T> v[kLookupFlight];
#pragma unroll
        for (int u = 0; u < kLookupFlight; ++u) {
            const int c = c0 + u * tpr;
            v[u] = Piece<T>{};
            if (in && c < pieces) load_piece(v[u], src + 8 * c);
        }
#pragma unroll
        for (int u = 0; u < kLookupFlight; ++u) {
            const int c = c0 + u * tpr;
            float f[8];
            unpack_piece(v[u], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = in ? f[i] * scale : 0.f;
            if (c < pieces) store_piece(dst + 8 * c, f);
        }
    }
}

template <typename T>
cudaError_t launch_lookup(const TokenIds &ids, const void *table, float scale, void *y, int *status, int n, int d, int vocabulary,
                          cudaStream_t s)
{
    int tpr = 8;       // threads of a row: as few as leave each of them at most kLookupFlight pieces
    while (tpr < kLookupThreads && tpr * kLookupFlight < d / 8) tpr *= 2;
    const int per_block = kLookupThreads / tpr;
    const unsigned grid = (unsigned)(((long long)n + per_block - 1) / per_block);
    return launch_overlapped(embedding_kernel<T>, grid, kLookupThreads, 0, s, ids, (const T *)table, scale, (T *)y, status, n, d,
                             vocabulary, tpr);
}

// ---- the positions sorted by token ----
constexpr int kSortBlocks = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortMaxBits = 10;

struct SortArgs {
    TokenIds ids;
    uint2 *a, *b;          // (token, position) pairs; pass p writes a where p is even, b where it is odd
    int *status, *counters;
    int n, vocabulary, bits, passes, n_counters;
};

// Positions whose id is not in 0 .. vocabulary-1 get the token `vocabulary`, which sorts last.
__global__ void __launch_bounds__(kSortThreads)
sort_kernel(const SortArgs p)
{
    extern __shared__ int sort_smem[];
    const int bins = 1 << p.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)cluster_ctarank();
    int *mine = sort_smem + warp * bins;            // this warp's histogram, then its first place of every digit
    int *total = sort_smem + kSortWarps * bins;     // this block's; read by the others
    int *base = total + bins;
    int *scan = base + bins;                        // [kSortWarps]
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (rank == 0 && tid == 0) *p.status = kDevOk;
    for (int i = rank * kSortThreads + tid; i < p.n_counters; i += kSortBlocks * kSortThreads) p.counters[i] = 0;
    const long long per = ((long long)p.n + kSortBlocks * kSortWarps - 1) / (kSortBlocks * kSortWarps);
    const long long lo = min((long long)p.n, per * (rank * kSortWarps + warp)), hi = min((long long)p.n, lo + per);
    bool bad = false;
    for (int pass = 0; pass < p.passes; ++pass) {
        const uint2 *src = (pass & 1) ? p.a : p.b;
        uint2 *dst = (pass & 1) ? p.b : p.a;
        const int shift = pass * p.bits;
        auto pair_at = [&](long long i) {
            if (pass > 0) return __ldcg(src + i);
            const long long id = p.ids.at(i);
            bad |= id >= p.vocabulary;
            return make_uint2((unsigned)(id >= 0 && id < p.vocabulary ? id : p.vocabulary), (unsigned)i);
        };
        for (int i = tid; i < kSortWarps * bins; i += kSortThreads) sort_smem[i] = 0;
        __syncthreads();
        for (long long i = lo + lane; i < hi; i += 32) atomicAdd(mine + ((pair_at(i).x >> shift) & (bins - 1)), 1);
        __syncthreads();
        if (tid < bins) {
            int s = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = sort_smem[w * bins + tid];
                sort_smem[w * bins + tid] = s;
                s += c;
            }
            total[tid] = s;
        }
        cluster_sync_all();
        int all = 0, before = 0;
        if (tid < bins) {
            const uint32_t at = smem_u32(total + tid);
#pragma unroll
            for (int r = 0; r < kSortBlocks; ++r) {
                int c;
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(c) : "r"(map_to_cta(at, r)));
                all += c;
                before += r < rank ? c : 0;
            }
        }
        int upto = all;                             // inclusive sums over the digits
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += t;
        }
        if (lane == 31) scan[warp] = upto;
        __syncthreads();
        if (warp == 0) {
            int t = scan[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xFFFFFFFFu, t, o);
                if (lane >= o) t += u;
            }
            scan[lane] = t;
        }
        __syncthreads();
        if (tid < bins) base[tid] = upto - all + (warp > 0 ? scan[warp - 1] : 0) + before;
        __syncthreads();
        for (long long i0 = lo; i0 < hi; i0 += 32) {
            const bool in = i0 + lane < hi;
            const uint2 v = in ? pair_at(i0 + lane) : make_uint2(0, 0);
            const int digit = in ? (int)((v.x >> shift) & (bins - 1)) : bins;
            const unsigned same = __match_any_sync(0xFFFFFFFFu, digit);
            const int ahead = __popc(same & ((1u << lane) - 1u));
            const int first = in ? mine[digit] : 0;
            __syncwarp();
            if (in) {
                dst[base[digit] + first + ahead] = v;
                if (ahead == 0) mine[digit] = first + __popc(same);
            }
            __syncwarp();
        }
        cluster_sync_all();                         // the pairs are written, and nobody reads `total` any more
    }
    if (bad) atomicMax(p.status, kDevBounds);
}

// ---- zeros and sums ----
constexpr int kSumThreads = 64, kSumCols = 8 * kSumThreads, kSumFlight = 8, kMaxChunk = 64, kJoinFlight = 8;
constexpr int kFillBits = 65536, kIdFlight = 16, kZeroBytes = 8192;

struct GradArgs {
    TokenIds ids;
    const uint2 *sorted;
    const void *dy;
    void *out;
    float *part;           // [chunks][2][d]: sums of the token that reaches in from the chunk before, and of the one that reaches out
    int *counters;         // [chunks][slabs] arrivals at the chunk where a token's sum begins
    float scale;
    int n, d, vocabulary, chunk, chunks, slabs, fill_blocks, accumulate;
};

// Zeros into the rows of a range of the vocabulary that no id names: bulk copies out of shared memory, which occupy a lane a
// warp (1000 positions into 32000 x 2048 in fp32, 46 us; by stores of all threads 51, a memset of the same bytes 67).
template <typename G>
__device__ void fill_rows(const GradArgs &p, int block, unsigned *named, uint4 *zero)
{
    for (int i = threadIdx.x; i < kZeroBytes / 16; i += blockDim.x) zero[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const int per = (p.vocabulary + p.fill_blocks - 1) / p.fill_blocks;
    const long long end = min((long long)p.vocabulary, (long long)per * (block + 1));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int bytes = p.d * (int)sizeof(G);
    for (long long v0 = (long long)per * block; v0 < end; v0 += kFillBits) {
        const int rows = (int)min((long long)kFillBits, end - v0);
        for (int i = threadIdx.x; i < (rows + 31) / 32; i += blockDim.x) named[i] = 0;
        __syncthreads();
        for (long long i0 = threadIdx.x; i0 < p.n; i0 += kIdFlight * blockDim.x) {
            long long id[kIdFlight];
#pragma unroll
            for (int u = 0; u < kIdFlight; ++u) {
                const long long i = i0 + u * blockDim.x;
                id[u] = i < p.n ? p.ids.at(i) : -1;
            }
#pragma unroll
            for (int u = 0; u < kIdFlight; ++u) {
                const unsigned long long r = (unsigned long long)(id[u] - v0);
                if (r < (unsigned long long)rows) atomicOr(named + (r >> 5), 1u << (r & 31));
            }
        }
        __syncthreads();
        // a warp's first lane asks for its rows, a copy of kZeroBytes zeros after the other
        if (lane == 0)
            for (int r = warp; r < rows; r += warps) {
                if ((named[r >> 5] >> (r & 31)) & 1u) continue;
                unsigned char *dst = reinterpret_cast<unsigned char *>(static_cast<G *>(p.out) + (v0 + r) * p.d);
                for (int at = 0; at < bytes; at += kZeroBytes)
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                                 ::"l"(dst + at), "r"(smem_u32(zero)), "r"(min(kZeroBytes, bytes - at)) : "memory");
            }
        __syncthreads();
    }
    if (lane == 0) {
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
}

template <typename G>
__device__ __forceinline__ void write_row(const GradArgs &p, unsigned token, int col, float (&f)[8])
{
    G *at = static_cast<G *>(p.out) + (size_t)token * p.d + col;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= p.scale;
    if (p.accumulate) {
        Piece<G> old;
        float o[8];
        load_piece(old, at);
        unpack_piece(old, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += o[i];
    }
    store_piece(at, f);
}

// How many chunks behind chunk c (step 1) or ahead of it (step -1) the token reaches: it does as long as the first position
// of the chunk behind, or the last one of the chunk ahead, holds it.  A warp looks at 32 borders at a time.
__device__ __forceinline__ int reach(const GradArgs &p, int c, int step, unsigned token)
{
    const int lane = threadIdx.x & 31;
    int steps = 0;
    while (true) {
        const int k = c + step * (steps + lane + (step > 0 ? 1 : 0));      // the border in front of chunk k
        const long long at = (long long)k * p.chunk - (step > 0 ? 0 : 1);
        const bool same = k > 0 && at < p.n && p.sorted[at].x == token;
        const unsigned other = ~__ballot_sync(0xFFFFFFFFu, same);
        if (other != 0) return steps + __ffs(other) - 1;
        steps += 32;
    }
}

__device__ __forceinline__ void group_sync(int group) { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(kSumThreads) : "memory"); }

struct SumShared {
    uint2 pair[kMaxChunk + 2];      // the chunk's, and those before and behind it
    int last;
};

// Adds up a chunk of sorted positions in a slab of columns: one group of kSumThreads threads, eight columns each.
template <typename T, typename G>
__device__ void sum_rows(const GradArgs &p, int chunk, int slab, int group, SumShared &sh)
{
    const int tid = threadIdx.x % kSumThreads, col = slab * kSumCols + 8 * tid;
    const bool active = col < p.d;
    const unsigned none = (unsigned)p.vocabulary;      // and above: no token
    const long long first = (long long)chunk * p.chunk;
    const int len = (int)min((long long)p.chunk, p.n - first);
    for (int i = tid; i < len + 2; i += kSumThreads) {
        const long long at = first - 1 + i;
        sh.pair[i] = at >= 0 && at < p.n ? p.sorted[at] : make_uint2(none + 1, 0);
    }
    group_sync(group);
    const uint2 *pair = sh.pair + 1;
    const T *dy = static_cast<const T *>(p.dy) + col;
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    // The sum of a token whose positions end in front of position `end` of the chunk and start at `start`: written, or
    // left in the workspace where the token reaches into another chunk.
    int start = 0;
    auto flush = [&](int end) {
        const unsigned token = pair[start].x;
        const bool in = start == 0 && pair[-1].x == token, out = end == len && pair[len].x == token;
        if (active) {
            if (!in && !out) {
                write_row<G>(p, token, col, acc);
            } else {
                float4 *at = reinterpret_cast<float4 *>(p.part + ((size_t)chunk * 2 + (in ? 0 : 1)) * p.d + col);
                __stcg(at, make_float4(acc[0], acc[1], acc[2], acc[3]));
                __stcg(at + 1, make_float4(acc[4], acc[5], acc[6], acc[7]));
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        start = end;
    };
    int valid = len;                                   // positions with a token; the others come last
    for (int i0 = 0; i0 < len; i0 += kSumFlight) {
        Piece<T> v[kSumFlight];
#pragma unroll
        for (int u = 0; u < kSumFlight; ++u) {
            v[u] = Piece<T>{};
            if (active && i0 + u < len && pair[i0 + u].x < none) load_piece(v[u], dy + (size_t)pair[i0 + u].y * p.d);
        }
#pragma unroll
        for (int u = 0; u < kSumFlight; ++u) {
            const int i = i0 + u;
            if (i >= valid) continue;
            if (pair[i].x >= none) { valid = i; continue; }
            if (pair[i].x != pair[start].x) flush(i);
            float f[8];
            unpack_piece(v[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += f[j];
        }
    }
    if (valid > 0) flush(valid);
    if (valid == 0) return;
    // What reaches across the chunk's borders: the group whose part arrives last adds the parts up in order.
    for (int side = 0; side < 2; ++side) {
        const unsigned token = pair[side ? valid - 1 : 0].x;
        const bool in = pair[-1].x == pair[0].x, through = pair[0].x == pair[valid - 1].x;
        const bool out = valid == len && pair[len].x == pair[len - 1].x;
        const bool mine = side == 0 ? in : out && !(in && through);
        if (!mine) continue;
        const bool goes_on = side == 1 || (through && out);
        __threadfence();
        group_sync(group);
        const int c0 = side == 0 ? chunk - reach(p, chunk, -1, token) : chunk;
        const int c1 = goes_on ? chunk + reach(p, chunk, 1, token) : chunk;
        if (tid == 0) sh.last = atomicAdd(p.counters + (size_t)c0 * p.slabs + slab, 1) == c1 - c0;
        group_sync(group);
        const bool last = sh.last != 0;
        if (!last || !active) continue;
        __threadfence();
        const float4 *at = reinterpret_cast<const float4 *>(p.part + ((size_t)c0 * 2 + 1) * p.d + col);
        float4 a = __ldcg(at), b = __ldcg(at + 1);
        float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        for (int c = c0 + 1; c <= c1; c += kJoinFlight) {
            float4 x[kJoinFlight], y[kJoinFlight];
#pragma unroll
            for (int u = 0; u < kJoinFlight; ++u) {
                x[u] = y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c + u <= c1) {
                    const float4 *q = reinterpret_cast<const float4 *>(p.part + (size_t)(c + u) * 2 * p.d + col);
                    x[u] = __ldcg(q);
                    y[u] = __ldcg(q + 1);
                }
            }
#pragma unroll
            for (int u = 0; u < kJoinFlight; ++u) {
                f[0] += x[u].x; f[1] += x[u].y; f[2] += x[u].z; f[3] += x[u].w;
                f[4] += y[u].x; f[5] += y[u].y; f[6] += y[u].z; f[7] += y[u].w;
            }
        }
        write_row<G>(p, token, col, f);
    }
}

constexpr int kGradThreads = 256, kGroups = kGradThreads / kSumThreads;

template <typename T, typename G>
__global__ void __launch_bounds__(kGradThreads, sizeof(T) == 2 ? 3 : 2)
embedding_grad_kernel(const GradArgs p)
{
    __shared__ union {
        struct { unsigned named[kFillBits / 32]; uint4 zero[kZeroBytes / 16]; } fill;
        SumShared sum[kGroups];
    } sh;
    // The blocks that write zeros wait for nothing: the sort lets this kernel start when all that came before the sort has
    // completed, and it writes neither the ids nor the result.
    if ((int)blockIdx.x < p.fill_blocks) {
        allow_next_kernel();
        fill_rows<G>(p, blockIdx.x, sh.fill.named, sh.fill.zero);
        return;
    }
    wait_for_earlier_kernels();
    allow_next_kernel();
    const int group = threadIdx.x / kSumThreads;
    const long long item = (long long)(blockIdx.x - p.fill_blocks) * kGroups + group;
    if (item >= (long long)p.chunks * p.slabs) return;
    sum_rows<T, G>(p, (int)(item / p.slabs), (int)(item % p.slabs), group, sh.sum[group]);
}

// ---- host ----
constexpr int kEmbeddingMaxD = 32768, kEmbeddingMaxTokens = 1 << 30, kEmbeddingMaxVocabulary = 1 << 30;

bool shape_ok(int n, int d, int vocabulary)
{
    return n >= 0 && n <= kEmbeddingMaxTokens && d >= 8 && d % 8 == 0 && vocabulary >= 1 && vocabulary <= kEmbeddingMaxVocabulary;
}
int slabs_of(int d) { return (d + kSumCols - 1) / kSumCols; }

// Positions of a chunk: short ones where there are few positions, so that every SM has rows to read, and at most 512
// chunks up to 32768 positions: that many parts are added up in a row where all positions hold one token (65536 rows of 2048:
// chunks of 64 132 us, of 128 142; if all hold one token, 65536 of 1024 take 220 and 138).
int chunk_of(int n)
{
    int c = 8;
    while (c < kMaxChunk && (n + c - 1) / c > 512) c *= 2;
    return c;
}
long long chunks_bound(int n) { return n <= 4096 ? (n + 7) / 8 : std::max(512, (n + kMaxChunk - 1) / kMaxChunk); }

struct GradLayout { size_t counters, a, b, part, total; };
GradLayout grad_layout(int n, int d)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t chunks = (size_t)chunks_bound(n);
    GradLayout L;
    L.counters = 256;                                   // behind the status word
    L.a = up(L.counters + chunks * slabs_of(d) * 4);
    L.b = up(L.a + (size_t)n * 8);
    L.part = up(L.b + (size_t)n * 8);
    L.total = up(L.part + chunks * 2 * d * 4);
    return L;
}

cudaError_t launch_sort(const SortArgs &a, cudaStream_t s)
{
    auto smem = [](int bits) { return (((kSortWarps + 2) << bits) + kSortWarps) * sizeof(int); };
    static DeviceFlags done;
    const cudaError_t e = allow_smem(sort_kernel, smem(kSortMaxBits), done);
    return e != cudaSuccess ? e : launch_clusters(sort_kernel, kSortBlocks, kSortBlocks, kSortThreads, smem(a.bits), s, a);
}

template <typename T, typename G>
cudaError_t launch_grad(const GradArgs &a, cudaStream_t s)
{
    const long long items = (long long)a.chunks * a.slabs;
    return launch_overlapped(embedding_grad_kernel<T, G>, (unsigned)(a.fill_blocks + (items + kGroups - 1) / kGroups),
                             kGradThreads, 0, s, a);
}

}  // namespace
}  // namespace modse

using namespace modse;

#define MODSE_CUDA(expr)                                \
    do {                                                \
        if ((expr) != cudaSuccess) return MODSE_ERR_CUDA; \
    } while (0)

extern "C" {

modse_status_t modse_embedding(modse_dtype_t dtype, int n_tokens, int d_model, int vocabulary, const void *ids, int id_bytes,
                               const void *table, float scale, void *y, int *status, void *cuda_stream)
{
    if ((dtype != MODSE_F32 && dtype != MODSE_BF16) || !shape_ok(n_tokens, d_model, vocabulary) ||
        (id_bytes != 4 && id_bytes != 8))
        return MODSE_ERR_INVALID_ARG;
    if (d_model > kEmbeddingMaxD) return MODSE_ERR_UNSUPPORTED;
    if (n_tokens == 0) return MODSE_OK;
    if (ids == nullptr || table == nullptr || y == nullptr || !aligned(ids, id_bytes) || !aligned(table, 16) ||
        !aligned(y, 16) || !aligned(status, 4))
        return MODSE_ERR_INVALID_ARG;
    const TokenIds in{ids, id_bytes == 8};
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (dtype == MODSE_F32) MODSE_CUDA(launch_lookup<float>(in, table, scale, y, status, n_tokens, d_model, vocabulary, s));
    else MODSE_CUDA(launch_lookup<__nv_bfloat16>(in, table, scale, y, status, n_tokens, d_model, vocabulary, s));
    return MODSE_OK;
}

size_t modse_embedding_backward_workspace_bytes(int n_tokens, int d_model, int vocabulary)
{
    if (!shape_ok(n_tokens, d_model, vocabulary) || d_model > kEmbeddingMaxD) return 0;
    return grad_layout(n_tokens, d_model).total;
}

modse_status_t modse_embedding_backward(modse_dtype_t dtype, int n_tokens, int d_model, int vocabulary, const void *ids,
                                        int id_bytes, const void *dy, float scale, modse_dtype_t grad_dtype, int accumulate,
                                        void *dtable, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if ((dtype != MODSE_F32 && dtype != MODSE_BF16) || (grad_dtype != MODSE_F32 && grad_dtype != MODSE_BF16) ||
        !shape_ok(n_tokens, d_model, vocabulary) || (id_bytes != 4 && id_bytes != 8))
        return MODSE_ERR_INVALID_ARG;
    if (d_model > kEmbeddingMaxD) return MODSE_ERR_UNSUPPORTED;
    if (dtable == nullptr || !aligned(dtable, 16)) return MODSE_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    if (n_tokens == 0) {
        clear_workspace_status(workspace, workspace_bytes, s);
        const size_t bytes = (size_t)vocabulary * d_model * (grad_dtype == MODSE_F32 ? 4 : 2);
        if (!accumulate) MODSE_CUDA(cudaMemsetAsync(dtable, 0, bytes, s));
        return MODSE_OK;
    }
    if (ids == nullptr || dy == nullptr || !aligned(ids, id_bytes) || !aligned(dy, 16) || workspace == nullptr ||
        !aligned(workspace, 256))
        return MODSE_ERR_INVALID_ARG;
    const GradLayout L = grad_layout(n_tokens, d_model);
    if (workspace_bytes < L.total) return MODSE_ERR_WORKSPACE_TOO_SMALL;
    unsigned char *ws = (unsigned char *)workspace;
    const TokenIds in{ids, id_bytes == 8};
    const int chunk = chunk_of(n_tokens), chunks = (n_tokens + chunk - 1) / chunk, slabs = slabs_of(d_model);
    int bits = 1;
    while (vocabulary >> bits) ++bits;
    const int passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
    const SortArgs sort{in, (uint2 *)(ws + L.a), (uint2 *)(ws + L.b), (int *)ws, (int *)(ws + L.counters), n_tokens, vocabulary,
                        (bits + passes - 1) / passes, passes, chunks * slabs};
    MODSE_CUDA(launch_sort(sort, s));
    // three blocks an SM write zeros, as many as fit while the positions are sorted, at least 16 rows each (5003 positions into
    // 100003 x 1536 in bf16: one an SM 79 us, two 64 to 71, three 61, four 64, six 65)
    const int fill = accumulate ? 0 : std::max(1, std::min(3 * device_sms(), vocabulary / 16));
    const GradArgs g{in, (passes & 1) ? sort.a : sort.b, dy, dtable, (float *)(ws + L.part), sort.counters, scale, n_tokens,
                     d_model, vocabulary, chunk, chunks, slabs, fill, accumulate != 0};
    const bool f32 = dtype == MODSE_F32;
    if (grad_dtype == MODSE_F32) MODSE_CUDA((f32 ? launch_grad<float, float>(g, s) : launch_grad<__nv_bfloat16, float>(g, s)));
    else MODSE_CUDA((f32 ? launch_grad<float, __nv_bfloat16>(g, s) : launch_grad<__nv_bfloat16, __nv_bfloat16>(g, s)));
    return MODSE_OK;
}

}  // extern "C"
