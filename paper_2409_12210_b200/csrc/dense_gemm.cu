// Dense products on Blackwell tensor cores: a persistent kernel in which a pair of CTAs on neighbouring SMs computes
// output tiles with tcgen05.mma.cta_group::2 (M = 256, up to 256 columns); operands are read K-major or MN-major straight
// from where they lie.  Each CTA of a pair stages its own rows of the row operand and half of the column operand by TMA.
//
// Two tile shapes, chosen by dense_plan:
//   512 x 256  each CTA holds two 128-row halves that share the column operand: 48 KB of shared memory to fill a k-block
//              of 1024 MMA clocks.  What bounds the smaller tile is that fill rate (32 KB in 512 clocks against about 56
//              bytes a clock and SM from L2), so this one runs the tensor cores faster; but both accumulators (all of
//              tensor memory) belong to one tile.  Its epilogue is hidden in part: the halves are drained one after
//              the other, and the next tile's first k-blocks are multiplied into the half that is free already.
//   256 x 256 / 256 x 128  one 128-row half a CTA; two accumulators in flight, the epilogue of one tile overlaps the
//              main loop of the next.  For outputs with too few tiles to fill the GPU.
//
// Tail.  The tiles left over after the last full round over the CTA pairs would leave most pairs idle for a whole tile.
// Of the tall shape they are handed out as their 256-row halves where those still fit one round.  Of the other they are
// cut along the contraction; every piece writes its fp32 accumulator to the workspace, and the epilogue warp that
// arrives last at a 32-row strip adds the pieces of that strip in order (so the sum does not depend on who was last)
// and runs the epilogue on it.
//
// Few tiles (at most 32).  Two or four pairs form a cluster that shares one tile: each multiplies its part of the
// contraction, hands the column chunks of its accumulator that another pair finishes to that pair through distributed
// shared memory (into what the 128-column tile leaves free of each stage), and adds up, in the pairs' order, and finishes
// its own.
//
// Every wait is bounded; one that expires records kDevTimeout in the status word and the CTAs drain and leave.
#include <cuda_fp16.h>

#include <algorithm>

#include "activations.h"
#include "dense_gemm.h"
#include "launch.h"
#include "tc_device.h"
#include "tc_gemm.h"

namespace modse {
namespace {

constexpr uint32_t kDenseRows = 16384;           // 128 rows of 128 bytes
constexpr int kDenseMaxStages = 6;
template <bool TALL> struct DenseShape {
    static constexpr int kStages = TALL ? 4 : 6;
    static constexpr int kStageBytes = TALL ? 49152 : 32768;      // one or two times 16 KB of rows, up to 16 KB of columns
    static constexpr int kTileRows = TALL ? 512 : 256;
};
constexpr int kDenseEpiWarps = 8;
constexpr int kDenseFirstEpi = 4;                // warps 0-1: TMA, MMA; 2-3 idle so that the epilogue starts on a warpgroup
constexpr int kDenseThreads = 32 * (kDenseFirstEpi + kDenseEpiWarps);
constexpr int kDenseAccCols = 256;
constexpr int kDenseTmemCols = 512;
constexpr int kDenseGroupRows = 8;               // row tiles whose column tiles are walked before the next group's

struct DenseTail {
    unsigned long long full[kDenseMaxStages], empty[kDenseMaxStages], tmem_full[2], tmem_empty[2];
    unsigned int tmem_base;
    int abort_flag;
};
constexpr int kDenseEpiBytes = 2 * kEpiBufBytes;    // two staging buffers an epilogue warp
constexpr size_t kDenseSmem = 1024 + (size_t)196608 + kDenseEpiWarps * kDenseEpiBytes + sizeof(DenseTail);
static_assert(kDenseSmem <= 232448, "shared memory per CTA");

template <int P> struct DenseParams {
    CUtensorMap a[P], b[P], o0[P], o1[P];     // operands; outputs as boxes of 32 rows x 64 bytes
    DenseProblem prob[P];
    LinearEpilogue lin;
    int n_prob, full_tiles, splits, items;   // tiles [0, full_tiles) are whole, the others cut into `splits` pieces
    int share;                               // CTA pairs of a cluster that share a tile (1: none)
    int *status, *counters;
    float *partial;
    unsigned long long wait_limit_ns;
    int clear_status;
    int skip_item;       // debugging: the producers that get this item stop without loading it (-1: none)
    DenseColumnSum sum;
};

struct DenseTile {
    int p, m0, n0, kb0, kb1;
    int tail;        // index among the tiles cut along the contraction, -1: a whole tile
    int split;
    bool two;        // the second 256-row half is computed too (tall tiles)
    bool skip;       // a half that lies outside the output
};

// The round-th item of a pair, -1: none.  The items of several products are sorted by decreasing length; every other round
// is dealt in the other direction, so that who got the longest item of one round gets the shortest of the next (1001
// tokens' dx and dw, 24 tiles of 44 k-blocks and 66 of 16: 34 -> 26 us).
template <int P>
__device__ __forceinline__ int dense_item(int round, int who, int n, int items)
{
    const int item = round * n + ((P > 1 && (round & 1)) ? n - 1 - who : who);
    return item < items ? item : -1;
}

template <int TN, bool TALL, int P>
__device__ __forceinline__ DenseTile dense_decode(const DenseParams<P> &prm, int item, int &cursor)
{
    DenseTile t;
    int tile = item, half = -1;
    t.tail = -1;
    t.split = 0;
    if (item >= prm.full_tiles && prm.splits > 1) {
        const int r = item - prm.full_tiles, c = r / prm.splits;
        tile = prm.full_tiles + c;
        if constexpr (TALL) {
            half = r - c * prm.splits;
        } else {
            t.tail = c;
            t.split = r - c * prm.splits;
        }
    }
    if constexpr (P > 1)
        while (cursor + 1 < prm.n_prob && tile >= prm.prob[cursor + 1].tile0) ++cursor;
    t.p = cursor;
    const DenseProblem &q = prm.prob[cursor];
    int local = tile - q.tile0, mb, nb;
    if (!TALL && (q.flags & kDenseSym)) {
        constexpr int kUnits = DenseShape<TALL>::kTileRows / TN;  // column tiles as wide as a row tile is high
        mb = 0;                                  // row by row of the upper triangle; squares on the diagonal are whole
        while (local >= q.nt - kUnits * mb) { local -= q.nt - kUnits * mb; ++mb; }
        nb = kUnits * mb + local;
    } else {
        const int per = kDenseGroupRows * q.nt, g = local / per, rem = local - g * per;
        const int rows = min(kDenseGroupRows, q.mt - g * kDenseGroupRows);
        nb = rem / rows;
        mb = g * kDenseGroupRows + rem - nb * rows;
    }
    t.m0 = mb * DenseShape<TALL>::kTileRows;
    t.n0 = nb * TN;
    t.two = TALL && t.m0 + 256 < q.M;
    t.skip = false;
    if (half >= 0) {
        t.skip = half == 1 && !t.two;
        t.two = false;
        t.m0 += 256 * half;
    }
    t.kb0 = 0;
    t.kb1 = q.nk;
    if (t.tail >= 0) {
        t.kb0 = (int)((long long)q.nk * t.split / prm.splits);
        t.kb1 = (int)((long long)q.nk * (t.split + 1) / prm.splits);
    }
    return t;
}

// A pair's part of the contraction of a tile that a cluster shares.
__device__ __forceinline__ void take_share(DenseTile &t, int sharer, int share)
{
    const int n = t.kb1;
    t.kb0 = n * sharer / share;
    t.kb1 = n * (sharer + 1) / share;
}

// ---- epilogue pieces: a warp holds 32 rows x 32 columns, one row a lane ----

// A warp's two staging buffers of 32 rows x 64 bytes, laid out as the 64-byte swizzle of a tensor map wants them (piece q
// of row r at epi_piece(r, q)).  Outputs leave by TMA: the warp writes its rows, one lane starts the copy, and the warp
// goes on with the other buffer; the map clips what lies outside the matrix.
struct Staging {
    unsigned char *base;
    int which;
    // The next buffer, free to be written: all groups but the latest have been read, and that one, committed for the other
    // buffer, is all that may be left.  So whoever takes a buffer commits one group for it, an empty one if nothing is copied.
    __device__ __forceinline__ unsigned char *take(int lane)
    {
        which ^= 1;
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
        return base + which * kEpiBufBytes;
    }
};
__device__ __forceinline__ void tile_send(unsigned char *buf, int lane, const CUtensorMap *map, int x, int y)
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                     ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(buf)), "r"(x), "r"(y) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ void tile_out(unsigned char *buf, int lane, const CUtensorMap *map, int x, int y, const uint4 (&w)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4 *>(buf + epi_piece(lane, q)) = w[q];
    tile_send(buf, lane, map, x, y);
}

// 32 rows x 64 bytes from global memory, four neighbouring lanes the 64 bytes of a row; `at` points at (first row of the
// warp, first column of the chunk); only pieces of 16 bytes that start at a valid column and row are read.
__device__ __forceinline__ void rows_load(int lane, const unsigned char *at, long long row_bytes, int rows_valid,
                                          int pieces_valid, uint4 (&raw)[4])
{
    const int q = lane & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int rr = 8 * j + (lane >> 2);
        raw[j] = make_uint4(0, 0, 0, 0);
        if (rr < rows_valid && q < pieces_valid) raw[j] = *reinterpret_cast<const uint4 *>(at + rr * row_bytes + q * 16);
    }
}
// ... and handed to the lanes that own the rows
__device__ __forceinline__ void rows_hand(unsigned char *buf, int lane, const uint4 (&raw)[4], uint4 (&own)[4])
{
    const int q = lane & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4 *>(buf + epi_piece(8 * j + (lane >> 2), q)) = raw[j];
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) own[k] = *reinterpret_cast<const uint4 *>(buf + epi_piece(lane, k));
    __syncwarp();
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&t);
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi)
{
    __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&t);
}
__device__ __forceinline__ float2 from_f16x2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float2 from_bf16x2(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

__device__ __forceinline__ void pack_bf16(const float (&v)[32], uint4 (&w)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        w[q] = make_uint4(bf16x2(v[8 * q], v[8 * q + 1]), bf16x2(v[8 * q + 2], v[8 * q + 3]),
                          bf16x2(v[8 * q + 4], v[8 * q + 5]), bf16x2(v[8 * q + 6], v[8 * q + 7]));
}
__device__ __forceinline__ void pack_f16(const float (&v)[32], uint4 (&w)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        w[q] = make_uint4(f16x2(v[8 * q], v[8 * q + 1]), f16x2(v[8 * q + 2], v[8 * q + 3]),
                          f16x2(v[8 * q + 4], v[8 * q + 5]), f16x2(v[8 * q + 6], v[8 * q + 7]));
}

__device__ __forceinline__ void activate_all(float (&v)[32], int act)
{
    if (act == MODSE_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 32; i += 2) activate2<MODSE_ACT_RELU>(v[i], v[i + 1]);
    } else if (act == MODSE_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 32; i += 2) activate2<MODSE_ACT_GELU>(v[i], v[i + 1]);
    } else if (act == MODSE_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 32; i += 2) activate2<MODSE_ACT_SILU>(v[i], v[i + 1]);
    }
}

// What a chunk of 32 rows (from r0) x 32 columns (from c0) reads from memory.  The first chunk's is requested before the
// accumulator is waited for, the next one's as soon as the registers of the present one are free.  Plain loads all: scales
// and bias may come from the kernel ahead, which may still be writing them when this one starts.
template <int MODE, bool F8> struct ChunkInputs {
    uint4 raw[MODE == DensePlain || MODE == DenseGram ? 1 : 4];      // residual, or the first input
    uint4 bias[MODE == DenseLinear ? 4 : 1];
    float sx;
};
enum : int { kLoadFirst = 1, kLoadBias = 2, kLoadAll = 3 };
template <int WHAT, int MODE, bool F8>
__device__ __forceinline__ void chunk_load(ChunkInputs<MODE, F8> &in, const DenseProblem &q, const LinearEpilogue &lin, int r0,
                                           int c0, int lane)
{
    const int rows = min(32, q.M - r0), pieces = (min(32, q.N - c0) + 7) >> 3;      // none where c0 lies outside
    if constexpr (MODE == DenseLinear) {
        if constexpr ((WHAT & kLoadFirst) != 0)
            if (lin.residual) rows_load(lane, (const unsigned char *)(lin.residual + (long long)r0 * q.N + c0), 2ll * q.N, rows, pieces, in.raw);
        if constexpr ((WHAT & kLoadBias) != 0) {
            if (lin.bias)
#pragma unroll
                for (int p = 0; p < 4; ++p) in.bias[p] = p < pieces ? *(reinterpret_cast<const uint4 *>(lin.bias + c0) + p) : make_uint4(0, 0, 0, 0);
            if constexpr (F8) in.sx = lane < rows ? lin.sx[r0 + lane] : 0.f;
        }
    } else if constexpr (MODE == DensePoly) {
        if constexpr ((WHAT & kLoadFirst) != 0)
            rows_load(lane, (const unsigned char *)((const __half *)q.in0 + (long long)r0 * q.ld_out + c0), 2 * q.ld_out, rows, pieces, in.raw);
    } else if constexpr (MODE == DenseStep) {
        const long long at = (long long)r0 * q.ld_in + c0;
        if constexpr ((WHAT & kLoadFirst) != 0)
            rows_load(lane, (const unsigned char *)((const __half *)q.in0 + at), 2 * q.ld_in, rows, pieces, in.raw);
    }
}

// Finishes the chunk and requests the inputs of the one that starts at column `next` (an outside column: of none); v: this
// lane's row.
template <int MODE, bool F8>
__device__ __forceinline__ void chunk_finish(ChunkInputs<MODE, F8> &in, const DenseProblem &q, const LinearEpilogue &lin,
                                             const CUtensorMap *o0, const CUtensorMap *o1, int r0, int c0, int next, int lane,
                                             Staging &stg, float (&v)[32])
{
    const int rows = min(32, q.M - r0), cols = min(32, q.N - c0);
    uint4 w[4];
    if constexpr (MODE == DenseLinear) {
        if constexpr (F8) {
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (4 * p < cols) {
                    const float4 f = *(reinterpret_cast<const float4 *>(lin.sw + c0) + p);
                    v[4 * p] *= in.sx * f.x; v[4 * p + 1] *= in.sx * f.y; v[4 * p + 2] *= in.sx * f.z; v[4 * p + 3] *= in.sx * f.w;
                }
        }
        if (lin.bias) {
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = from_bf16x2(word_of(in.bias[p], i));
                    v[8 * p + 2 * i] += f.x;
                    v[8 * p + 2 * i + 1] += f.y;
                }
        }
        chunk_load<kLoadBias>(in, q, lin, r0, next, lane);
        if (lin.z) {
            pack_bf16(v, w);
            tile_out(stg.take(lane), lane, o1, c0, r0, w);
        }
        activate_all(v, lin.act);
        unsigned char *buf = stg.take(lane);
        if (lin.residual) {
            uint4 own[4];
            rows_hand(buf, lane, in.raw, own);
            chunk_load<kLoadFirst>(in, q, lin, r0, next, lane);
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = from_bf16x2(word_of(own[p], i));
                    v[8 * p + 2 * i] += f.x;
                    v[8 * p + 2 * i + 1] += f.y;
                }
        }
        pack_bf16(v, w);
        tile_out(buf, lane, o0, c0, r0, w);
    } else if constexpr (MODE == DensePlain) {
        pack_bf16(v, w);
        tile_out(stg.take(lane), lane, o0, c0, r0, w);
    } else if constexpr (MODE == DenseGram || MODE == DensePoly) {
        unsigned char *buf = stg.take(lane);
        if constexpr (MODE == DensePoly) {
            uint4 own[4];
            rows_hand(buf, lane, in.raw, own);
            chunk_load<kLoadFirst>(in, q, lin, r0, next, lane);
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = from_f16x2(word_of(own[p], i));
                    v[8 * p + 2 * i] = fmaf(q.beta, f.x, q.alpha * v[8 * p + 2 * i]);
                    v[8 * p + 2 * i + 1] = fmaf(q.beta, f.y, q.alpha * v[8 * p + 2 * i + 1]);
                }
            if (c0 == r0) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += i == lane ? q.scale : 0.f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= q.alpha;
        }
        pack_f16(v, w);
        tile_out(buf, lane, o0, c0, r0, w);
        if ((c0 >> 8) > (r0 >> 8)) {
            // off the diagonal (in units of 256) the transposed block goes out the same way: a lane's values go down a column of the staging buffer
            buf = stg.take(lane);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                *reinterpret_cast<__half *>(buf + epi_piece(i, lane >> 3) + (lane & 7) * 2) = __float2half_rn(v[i]);
            tile_send(buf, lane, o0, r0, c0);
        }
    } else {
        unsigned char *buf = stg.take(lane);
        uint4 own[4];
        rows_hand(buf, lane, in.raw, own);
        chunk_load<kLoadFirst>(in, q, lin, r0, next, lane);
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = from_f16x2(word_of(own[p], i));
                v[8 * p + 2 * i] = fmaf(q.beta, f.x, q.alpha * v[8 * p + 2 * i]);
                v[8 * p + 2 * i + 1] = fmaf(q.beta, f.y, q.alpha * v[8 * p + 2 * i + 1]);
            }
        if (q.flags & kDenseLast) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= q.scale;
            pack_bf16(v, w);
            if (q.flags & kDenseTmaOut) {
                tile_out(buf, lane, o0, c0, r0, w);
            } else {
                // rows that TMA cannot write (any alignment): a warp writes one row after the other, a column a lane
#pragma unroll
                for (int p = 0; p < 4; ++p) *reinterpret_cast<uint4 *>(buf + epi_piece(lane, p)) = w[p];
                __syncwarp();
                __nv_bfloat16 *out = (__nv_bfloat16 *)q.out0 + (long long)r0 * q.ld_out + c0;
                if (lane < cols)
#pragma unroll 8
                    for (int r = 0; r < rows; ++r)
                        out[r * q.ld_out + lane] = *reinterpret_cast<const __nv_bfloat16 *>(buf + epi_piece(r, lane >> 3) + (lane & 7) * 2);
                __syncwarp();
                // an empty group in the place of this buffer's copy: Staging::take counts one for every buffer, and without
                // it the next one would be written while a copy of an earlier matrix's rows may still be reading it
                if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        } else {
            pack_f16(v, w);
            tile_out(buf, lane, o0, c0, r0, w);
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = from_f16x2(word_of(w[p], i));
                    v[8 * p + 2 * i] -= f.x;
                    v[8 * p + 2 * i + 1] -= f.y;
                }
            pack_f16(v, w);
            tile_out(stg.take(lane), lane, o1, c0, r0, w);
        }
    }
}

__device__ __forceinline__ void umma_f8_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accum)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accum)
        : "memory");
}

// fp32 accumulator; operand format bits: f16 0, bf16 1 (kind::f16), e4m3 0 (kind::f8f6f4); M = 256.
template <int TYPE>
__device__ __forceinline__ uint32_t dense_idesc(bool a_mn, bool b_mn, int n)
{
    constexpr uint32_t fmt = TYPE == DenseBf16 ? 1u : 0u;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | (16u << 24);
}

// Arrives on the barrier at the same offset in both CTAs of a pair (mask: their ranks in the cluster) once the MMAs issued
// so far are done.
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t mask)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)mask) : "memory");
}
__device__ __forceinline__ void st_cluster_f4(uint32_t addr, const float4 &v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// The epilogue warps of a tile that the pairs of a cluster share (one item a cluster): chunk ch of its TN / 32 column chunks
// is finished by pair ch % share.  What the other pairs send lies in the 8 KB that a stage of a 128-column tile leaves
// free, where no copy of the main loop writes, so that a warp sends as soon as its pair's products are done.
template <int MODE, int TYPE, int TN, int P>
__device__ __forceinline__ void finish_shared(const DenseParams<P> &prm, unsigned char *smem, uint32_t stage_base, DenseTail *st,
                                              const WaitCtx &wc, uint32_t tmem_base, int item, int sharer, int rank, int warp, int lane)
{
    using Sh = DenseShape<false>;
    constexpr int kChunks = TN / 64;                // 32-column chunks a warp reads; of them it finishes one at most
    constexpr uint32_t kChunkBytes = 32 * 32 * 4, kFreeAt = kDenseRows + TN / 2 * 128;
    static_assert(kFreeAt + 2 * kChunkBytes == Sh::kStageBytes && Sh::kStages * 2 >= 3 * 4 && kChunks == 2, "slots");
    const int share = prm.share;
    int cursor = 0;
    const DenseTile t = dense_decode<TN, false, P>(prm, item, cursor);
    const DenseProblem &q = prm.prob[t.p];
    const int quad = warp & 3, cq = (warp - kDenseFirstEpi) >> 2;
    const int r0 = t.m0 + rank * 128 + quad * 32, c0 = t.n0 + cq * (TN / 2);
    const uint32_t tacc = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(cq * (TN / 2));
    // what pair `sender` has of chunk ch, in the shared memory of the pair that finishes it
    auto slot = [&](int sender, int ch) {
        const int k = ((sender - (sender > ch % share)) * (TN / 32 / share) + ch / share) * 4 + quad;
        return (uint32_t)((k >> 1) * Sh::kStageBytes + kFreeAt + (k & 1) * kChunkBytes + lane * 16);
    };
    int own = -1;
    for (int c = 0; c < kChunks; ++c)
        if ((cq * kChunks + c) % share == sharer && c0 + 32 * c < q.N && r0 < q.M) own = c;
    ChunkInputs<MODE, TYPE == DenseE4m3> in;
    if (own >= 0) chunk_load<kLoadAll>(in, q, prm.lin, r0, c0 + 32 * own, lane);
    const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&st->tmem_full[0]), 0, wc));
    tc_fence_after();
    if (ok && r0 < q.M)
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
            const int ch = cq * kChunks + c, owner = ch % share;
            if (c0 + 32 * c >= q.N || owner == sharer) continue;
            uint32_t w[32];
            tmem_ld32(tacc + 32 * c, w);
            tmem_ld_wait();
            const uint32_t to = map_to_cta(stage_base + slot(sharer, ch), 2 * owner + rank);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                st_cluster_f4(to + 512 * j, make_float4(__uint_as_float(w[4 * j]), __uint_as_float(w[4 * j + 1]),
                                                        __uint_as_float(w[4 * j + 2]), __uint_as_float(w[4 * j + 3])));
        }
    __syncwarp();
    cluster_sync_all();                             // what the others sent has arrived
    if (!ok || own < 0) return;
    Staging stg{smem + (size_t)Sh::kStages * Sh::kStageBytes + (warp - kDenseFirstEpi) * kDenseEpiBytes, 0};
    const int ch = cq * kChunks + own;
    uint32_t w[32];
    tmem_ld32(tacc + 32 * own, w);
    tmem_ld_wait();
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = 0.f;
#pragma unroll 1
    for (int s = 0; s < share; ++s) {
        if (s == sharer) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(w[i]);
        } else {
            const float4 *src = reinterpret_cast<const float4 *>(smem + slot(s, ch));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 f = src[32 * j];
                v[4 * j] += f.x; v[4 * j + 1] += f.y; v[4 * j + 2] += f.z; v[4 * j + 3] += f.w;
            }
        }
    }
    chunk_finish(in, q, prm.lin, &prm.o0[t.p], &prm.o1[t.p], r0, c0 + 32 * own, q.N, lane, stg, v);
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

template <int MODE, int TYPE, int TN, bool TALL, bool SHARED, int P>
__device__ __forceinline__ void dense_gemm_body(const DenseParams<P> &prm)
{
    using Sh = DenseShape<TALL>;
    constexpr int kStages = Sh::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t pad = ((raw + 1023u) & ~1023u) - raw;
    unsigned char *smem = smem_raw + pad;
    const uint32_t stage_base = raw + pad;
    unsigned char *epi_bufs = smem + (size_t)kStages * Sh::kStageBytes;
    DenseTail *st = reinterpret_cast<DenseTail *>(epi_bufs + kDenseEpiWarps * kDenseEpiBytes);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int in_cluster = (int)cluster_ctarank(), rank = in_cluster & 1, leader = SHARED ? in_cluster & ~1 : 0, sharer = in_cluster >> 1;
    const int share = SHARED ? prm.share : 1;
    const int cluster_id = SHARED ? blockIdx.x / (2 * share) : blockIdx.x >> 1, n_clusters = SHARED ? gridDim.x / (2 * share) : gridDim.x >> 1;
    const uint32_t pair_mask = 3u << leader;
    constexpr int kElems = TYPE == DenseE4m3 ? 128 : 64;       // elements in 128 bytes
    constexpr int kHalf = TN / 2;                              // column-operand rows staged by each CTA
    constexpr uint32_t kColsAt = TALL ? 2 * kDenseRows : kDenseRows;      // column operand inside a stage

    if (tid == 0) {
        for (int i = 0; i < min(prm.n_prob, 4); ++i) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&prm.a[i])) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&prm.b[i])) : "memory");
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&st->full[s]), 1);
            mbar_init(smem_u32(&st->empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&st->tmem_full[a]), 1);
            mbar_init(smem_u32(&st->tmem_empty[a]), 2 * kDenseEpiWarps);
        }
        st->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&st->tmem_base)), "r"(kDenseTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                 // both CTAs' barriers exist before any remote arrival or copy completion
    tc_fence_after();
    wait_for_earlier_kernels();
    allow_next_kernel();
    // the first block clears the status word; a wait can expire a millisecond later at the earliest
    if (prm.clear_status && blockIdx.x == 0 && tid == 0) *prm.status = kDevOk;
    const uint32_t tmem_base = st->tmem_base;
    const WaitCtx wc{&st->abort_flag, prm.status, prm.wait_limit_ns};

    if (warp == 0) {
        // ===================== TMA producer (both CTAs) =====================
        if (lane == 0) {
            int stage = 0, cursor = 0;
            uint32_t phase = 0;
            long long issued = 0;
            bool ok = true;
            for (int round = 0; ok; ++round) {
                const int item = dense_item<P>(round, cluster_id, n_clusters, prm.items);
                if (item < 0 || item == prm.skip_item) break;
                DenseTile t = dense_decode<TN, TALL, P>(prm, item, cursor);
                if constexpr (SHARED) take_share(t, sharer, share);
                if (t.skip) continue;
                const int flags = prm.prob[t.p].flags;
                const CUtensorMap *am = &prm.a[t.p], *bm = &prm.b[t.p];
                const int ar = t.m0 + rank * 128, br = t.n0 + rank * kHalf, halves = t.two ? 2 : 1;
                const uint32_t bytes = 2u * (halves * kDenseRows + kHalf * 128u);      // of both CTAs
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!mbar_wait(smem_u32(&st->empty[stage]), phase ^ 1u, wc)) { ok = false; break; }
                    const uint32_t bar = map_to_cta(smem_u32(&st->full[stage]), leader);
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&st->full[stage]), bytes);
                    const uint32_t dst = stage_base + stage * Sh::kStageBytes;
                    for (int h = 0; h < halves; ++h) {
                        const uint32_t to = dst + h * kDenseRows;
                        const int row = ar + 256 * h;
                        if (flags & kDenseAMn) {
                            tma_load_2d_pair(to, am, bar, row, kb * 64);
                            tma_load_2d_pair(to + kBoxBytes, am, bar, row + 64, kb * 64);
                        } else {
                            tma_load_2d_pair(to, am, bar, kb * kElems, row);
                        }
                    }
                    if (flags & kDenseBMn) {
#pragma unroll
                        for (int i = 0; i < kHalf / 64; ++i)
                            tma_load_2d_pair(dst + kColsAt + i * kBoxBytes, bm, bar, br + 64 * i, kb * 64);
                    } else {
                        tma_load_2d_pair(dst + kColsAt, bm, bar, kb * kElems, br);
                    }
                    ++issued;
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok && rank == 0) {
                // the copies of both CTAs complete on the leader's barriers: it lets those in flight land
                const int n = issued < kStages ? (int)issued : kStages;
                for (int i = 1; i <= n; ++i) {
                    int s2 = stage - i;
                    uint32_t ph = phase;
                    if (s2 < 0) { s2 += kStages; ph ^= 1u; }
                    const unsigned long long tb = global_ns();
                    while (!mbar_try_wait(smem_u32(&st->full[s2]), ph) && global_ns() - tb < prm.wait_limit_ns) {}
                }
            }
        }
    } else if (warp == 1) {
        // ===================== MMA issuer (leader only) =====================
        if (lane == 0 && rank == 0) {
            int stage = 0, cursor = 0, it = 0;
            uint32_t phase = 0, used0 = 0, used1 = 0;      // how often each accumulator has been handed to the epilogue
            bool ok = true;
            for (int round = 0; ok; ++round) {
                const int item = dense_item<P>(round, cluster_id, n_clusters, prm.items);
                if (item < 0) break;
                DenseTile t = dense_decode<TN, TALL, P>(prm, item, cursor);
                if constexpr (SHARED) take_share(t, sharer, share);
                if (t.skip) continue;
                const int flags = prm.prob[t.p].flags;
                const bool a_mn = (flags & kDenseAMn) != 0, b_mn = (flags & kDenseBMn) != 0;
                const uint32_t a_step = a_mn ? (2048u >> 4) : (32u >> 4), b_step = b_mn ? (2048u >> 4) : (32u >> 4);
                const uint32_t idesc = dense_idesc<TYPE>(a_mn, b_mn, TN);
                // the four products of half h and the stage at `s` into accumulator columns `to`
                auto multiply = [&](int s, int h, uint32_t to, bool fresh) {
                    const uint32_t addr = stage_base + s * Sh::kStageBytes;
                    const uint64_t adesc = make_desc(addr + h * kDenseRows, a_mn), bdesc = make_desc(addr + kColsAt, b_mn);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const uint32_t more = (!fresh || ks > 0) ? 1u : 0u;
                        if constexpr (TYPE == DenseE4m3)
                            umma_f8_pair(to, adesc + (uint64_t)(ks * a_step), bdesc + (uint64_t)(ks * b_step), idesc, more);
                        else
                            umma_bf16_pair(to, adesc + (uint64_t)(ks * a_step), bdesc + (uint64_t)(ks * b_step), idesc, more);
                    }
                };
                if constexpr (!TALL) {
                    const int acc = it++ & 1;
                    uint32_t &used = acc ? used1 : used0;
                    if (!mbar_wait(smem_u32(&st->tmem_empty[acc]), (used & 1u) ^ 1u, wc)) { ok = false; break; }
                    ++used;
                    tc_fence_after();
                    for (int kb = t.kb0; kb < t.kb1; ++kb) {
                        if (!mbar_wait(smem_u32(&st->full[stage]), phase, wc)) { ok = false; break; }
                        tc_fence_after();
                        multiply(stage, 0, tmem_base + (uint32_t)(acc * kDenseAccCols), kb == t.kb0);
                        commit_to(smem_u32(&st->empty[stage]), pair_mask);
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    commit_to(smem_u32(&st->tmem_full[acc]), pair_mask);
                } else {
                    if (!mbar_wait(smem_u32(&st->tmem_empty[0]), (used0 & 1u) ^ 1u, wc)) { ok = false; break; }
                    ++used0;
                    tc_fence_after();
                    int kb = t.kb0;
                    if (t.two) {
                        // the first k-blocks into the first half while the second half's accumulator is still being
                        // drained, then the same stages into the second half
                        const int ahead = min(kStages, t.kb1 - t.kb0);
                        int s = stage;
                        uint32_t ph = phase;
                        for (int i = 0; i < ahead; ++i) {
                            if (!mbar_wait(smem_u32(&st->full[s]), ph, wc)) { ok = false; break; }
                            tc_fence_after();
                            multiply(s, 0, tmem_base, i == 0);
                            if (++s == kStages) { s = 0; ph ^= 1u; }
                        }
                        if (!ok) break;
                        if (t.kb0 + ahead == t.kb1) commit_to(smem_u32(&st->tmem_full[0]), pair_mask);
                        if (!mbar_wait(smem_u32(&st->tmem_empty[1]), (used1 & 1u) ^ 1u, wc)) { ok = false; break; }
                        ++used1;
                        tc_fence_after();
                        for (int i = 0; i < ahead; ++i) {
                            multiply(stage, 1, tmem_base + kDenseAccCols, i == 0);
                            commit_to(smem_u32(&st->empty[stage]), pair_mask);
                            if (++stage == kStages) { stage = 0; phase ^= 1u; }
                        }
                        kb += ahead;
                    }
                    for (; kb < t.kb1; ++kb) {
                        if (!mbar_wait(smem_u32(&st->full[stage]), phase, wc)) { ok = false; break; }
                        tc_fence_after();
                        multiply(stage, 0, tmem_base, kb == t.kb0);
                        if (kb + 1 == t.kb1) commit_to(smem_u32(&st->tmem_full[0]), pair_mask);
                        if (t.two) multiply(stage, 1, tmem_base + kDenseAccCols, false);
                        commit_to(smem_u32(&st->empty[stage]), pair_mask);
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    if (t.two) commit_to(smem_u32(&st->tmem_full[1]), pair_mask);
                }
            }
        }
    } else if (warp < kDenseFirstEpi) {
        // ===================== column sums of a [rows, cols] fp32 matrix beside the products =====================
        if constexpr (MODE == DensePlain) {
            const int step = 2 * (int)gridDim.x * 32;
            for (int c = (2 * (int)blockIdx.x + warp - 2) * 32 + lane; c < prm.sum.cols; c += step) {
                float t = 0.f;
#pragma unroll 8
                for (int r = 0; r < prm.sum.rows; ++r) t += __ldcg(prm.sum.part + (size_t)r * prm.sum.cols + c);
                prm.sum.out[c] = t;
            }
        }
    } else if constexpr (SHARED) {
        finish_shared<MODE, TYPE, TN>(prm, smem, stage_base, st, wc, tmem_base, cluster_id, sharer, rank, warp, lane);
    } else {
        // ===================== epilogue (both CTAs) =====================
        const int quad = warp & 3;                          // tensor-memory lanes this warp may read
        const int cq = (warp - kDenseFirstEpi) >> 2;        // which half of the tile's columns
        Staging stg{epi_bufs + (warp - kDenseFirstEpi) * kDenseEpiBytes, 0};
        const uint32_t leader_empty0 = map_to_cta(smem_u32(&st->tmem_empty[0]), leader);
        const uint32_t leader_empty1 = map_to_cta(smem_u32(&st->tmem_empty[1]), leader);
        constexpr int kChunks = TN / 64;                    // 32-column chunks a warp owns
        constexpr bool kF8 = TYPE == DenseE4m3;
        int cursor = 0, it = 0;
        uint32_t used0 = 0, used1 = 0;                      // how often each accumulator has been drained
        bool ok = true;
        for (int round = 0; ok; ++round) {
            const int item = dense_item<P>(round, cluster_id, n_clusters, prm.items);
            if (item < 0) break;
            const DenseTile t = dense_decode<TN, TALL, P>(prm, item, cursor);
            if (t.skip) continue;
            const DenseProblem &q = prm.prob[t.p];
            const CUtensorMap *o0 = &prm.o0[t.p], *o1 = &prm.o1[t.p];
            const int c0 = t.n0 + cq * kHalf, halves = t.two ? 2 : 1, first = TALL ? 0 : (it++ & 1);
#pragma unroll 1
            for (int h = 0; h < halves; ++h) {
                const int acc = TALL ? h : first, r0 = t.m0 + 256 * h + rank * 128 + quad * 32;
                const bool any = r0 < q.M && c0 < q.N;
                ChunkInputs<MODE, kF8> in;
                if (any && t.tail < 0) chunk_load<kLoadAll>(in, q, prm.lin, r0, c0, lane);
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&st->tmem_full[acc]), (acc ? used1 : used0) & 1u, wc))) { ok = false; break; }
                if (acc) ++used1; else ++used0;
                tc_fence_after();
                const uint32_t tacc = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * kDenseAccCols + cq * kHalf);
                // a cut tile's strip: 32 rows x kHalf columns, float4 j of all lanes side by side
                constexpr size_t kStrip = 32 * kHalf / 4, kPiece = 2 * kDenseEpiWarps * kStrip;
                const int strip_id = rank * kDenseEpiWarps + cq * 4 + quad;
                float4 *strip = nullptr;
                if (t.tail >= 0)
                    strip = reinterpret_cast<float4 *>(prm.partial) + (size_t)(t.tail * prm.splits) * kPiece + strip_id * kStrip + lane;
                if (any) {
#pragma unroll 1
                    for (int c = 0; c < kChunks; ++c) {
                        if (c0 + 32 * c >= q.N) break;
                        uint32_t w[32];
                        tmem_ld32(tacc + 32 * c, w);
                        tmem_ld_wait();
                        float v[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(w[i]);
                        if (t.tail < 0) {
                            chunk_finish(in, q, prm.lin, o0, o1, r0, c0 + 32 * c, c + 1 < kChunks ? c0 + 32 * c + 32 : q.N, lane, stg, v);
                        } else {
                            float4 *dst = strip + (size_t)t.split * kPiece + (size_t)c * 256;
#pragma unroll
                            for (int j = 0; j < 8; ++j) __stcg(dst + 32 * j, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(acc ? leader_empty1 : leader_empty0);
                if (t.tail >= 0 && any) {
                    __threadfence();
                    __syncwarp();
                    int seen = 0;
                    int *counter = prm.counters + t.tail * 2 * kDenseEpiWarps + strip_id;
                    if (lane == 0) seen = atomicAdd(counter, 1);
                    seen = __shfl_sync(0xFFFFFFFFu, seen, 0);
                    if (seen == prm.splits - 1) {
                        __threadfence();
                        if (lane == 0) *counter = 0;               // for the next launch
                        chunk_load<kLoadAll>(in, q, prm.lin, r0, c0, lane);
#pragma unroll 1
                        for (int c = 0; c < kChunks; ++c) {
                            if (c0 + 32 * c >= q.N) break;
                            float v[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = 0.f;
#pragma unroll 1
                            for (int s = 0; s < prm.splits; ++s) {
                                const float4 *src = strip + (size_t)s * kPiece + (size_t)c * 256;
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    const float4 f = __ldcg(src + 32 * j);
                                    v[4 * j] += f.x; v[4 * j + 1] += f.y; v[4 * j + 2] += f.z; v[4 * j + 3] += f.w;
                                }
                            }
                            chunk_finish(in, q, prm.lin, o0, o1, r0, c0 + 32 * c, c + 1 < kChunks ? c0 + 32 * c + 32 : q.N, lane, stg, v);
                        }
                    }
                }
            }
        }
        if (lane == 0)
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");     // the outputs have left shared memory
    }

    // the warps that finish a shared tile meet the other pairs' in the middle of it; the rest of the warps join them there
    if (SHARED && warp < kDenseFirstEpi) {
        __syncwarp();
        cluster_sync_all();
    }

    // ---- teardown: neither CTA leaves while its partner may still touch its shared or tensor memory ----
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kDenseTmemCols) : "memory");
    }
}

template <int MODE, int TYPE, int TN, bool TALL, int P>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kDenseThreads, 1)
dense_gemm_pair(const __grid_constant__ DenseParams<P> prm)
{
    dense_gemm_body<MODE, TYPE, TN, TALL, false, P>(prm);
}
// clusters of prm.share pairs, one tile each
template <int MODE, int TYPE, int TN, int P>
__global__ void __launch_bounds__(kDenseThreads, 1) dense_gemm_shared(const __grid_constant__ DenseParams<P> prm)
{
    dense_gemm_body<MODE, TYPE, TN, false, true, P>(prm);
}

// A 2-D tensor map: `cols` contiguous elements a row, boxes of 128 bytes x box_rows rows, 128-byte swizzle.
bool encode_operand(CUtensorMap *map, const DenseOperand &o, int type, int box_rows)
{
    EncodeTiledFn fn = get_encode();
    if (fn == nullptr) return false;
    const int esz = type == DenseE4m3 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(o.ld * esz)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / esz), (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = type == DenseE4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                   : type == DenseF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return fn(map, dt, 2, const_cast<void *>(o.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An output of 2-byte elements, written in boxes of 32 rows x 64 bytes with the 64-byte swizzle.
bool encode_output(CUtensorMap *map, const void *base, long long rows, long long cols, long long ld)
{
    EncodeTiledFn fn = get_encode();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(ld * 2)};
    const cuuint32_t box[2] = {32, 32}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles up to which clusters of two and of four pairs all find room at once (with 16 clusters of four the last ones waited
// for a place: 2048 x 2048, 64 tokens 19 us against 14).
constexpr int kDenseShare2 = 32, kDenseShare4 = 12;

// How a launch is cut: tile shape, whole tiles, pieces of the rest.
struct DensePlan {
    bool tall;
    int tn, tiles, full, splits, items, share;
};

int dense_nk(DenseType type, long long k) { return (int)((k + (type == DenseE4m3 ? 127 : 63)) / (type == DenseE4m3 ? 128 : 64)); }

// (A symmetric output has no tall form.)
long long dense_tiles(const DenseProblem &p, bool tall, int tn)
{
    const long long mt = (p.M + (tall ? 511 : 255)) / (tall ? 512 : 256), nt = (p.N + tn - 1) / tn;
    if (!(p.flags & kDenseSym)) return mt * nt;
    long long c = 0;
    for (long long m = 0; m < mt; ++m) c += nt - 256 / tn * m;
    return c;
}

DensePlan dense_plan(DenseType type, const DenseItem *items, int n, bool light, int sms, size_t partial_capacity)
{
    const int pairs = std::max(1, sms / 2);
    auto count = [&](bool tall, int tn) {
        long long tiles = 0;
        for (int i = 0; i < n; ++i) tiles += dense_tiles(items[i].p, tall, tn);
        return tiles;
    };
    DensePlan pl;
    pl.share = 1;
    // Tall tiles where they fill the GPU at least once and the epilogue that shows is a light one (a conversion and a store;
    // `light`) behind a long main loop.  A round of them takes about 1024 x 1.05 clocks a k-block and the epilogue, a round
    // of 256-row tiles 585 a k-block.  Measured, tall against not: dx and dw of 16384 x 2048 -> 5632 504 against 580 us,
    // the product alone 250 against 262, with K 5632 273 against 283; but 350 against 303 with bias, gelu and z, 293
    // against 282 with a residual, 205 against 148 from 8-bit rows, 56 against 58 with 16 k-blocks.
    const long long talls = light ? count(true, 256) : 0, squares = count(false, 256);
    const long long whole = talls / pairs, rest = talls % pairs;
    const double tall_rounds = (double)whole + (rest == 0 ? 0.0 : 2 * rest <= pairs ? 0.57 : 1.0);
    const double square_rounds = (double)((squares + pairs - 1) / pairs);
    int least_nk = 1 << 30;
    for (int i = 0; i < n; ++i) least_nk = std::min(least_nk, dense_nk(type, items[i].k));
    pl.tall = light && least_nk >= 24 && talls >= pairs && tall_rounds * 1.13 <= square_rounds * 0.585;
    if (pl.tall) {
        pl.tn = 256;
        pl.tiles = (int)talls;
        pl.full = (int)(whole * pairs);
        pl.splits = (rest > 0 && 2 * rest <= pairs) ? 2 : 1;
        pl.items = pl.full + (int)rest * pl.splits;
        return pl;
    }
    // 256-column tiles unless the whole output has less than half a tile for each CTA pair: then 128-column tiles, whose
    // epilogue, which shows in a launch of one round, is half as long
    pl.tn = squares * 2 <= pairs ? 128 : 256;
    pl.tiles = (int)count(false, pl.tn);
    pl.full = pl.tiles / pairs * pairs;
    const int left = pl.tiles - pl.full;
    pl.splits = 1;
    if (left > 0) {
        // One round over the pairs, as many pieces as the workspace holds, at least 16 k-blocks each: joining them costs
        // about 4.5 us, twelve k-blocks' time (704 x 704, 300 tokens: 11.7 us in three pieces, 7.2 whole).
        const long long held = (long long)(partial_capacity / ((size_t)256 * pl.tn * 4));
        const long long sp = std::min<long long>({std::min(pairs, kDenseMaxSplitItems) / left, least_nk / 16, 16, held / left});
        pl.splits = (int)std::max<long long>(1, sp);
    }
    // Few tiles: two or four pairs of a cluster on each, where that beats cutting the tiles (in us: 0.33 a k-block, 2 for
    // handing the chunks over, 4.5 for joining pieces through memory).  Measured, shared against cut or whole: 2048 x 2048
    // 10.1 against 14.7 us with 64 tokens and 11.7 against 16.1 with 512; 8448 x 1024 from 8-bit rows 11.6 against 17.5.
    // (With 1 us for the handing over, 512 x 2048 with 500 tokens is shared too: 7.5 us against 6.3.)
    if (pl.full == 0 && pl.tn == 128) {
        double best = pl.splits > 1 ? 0.33 * least_nk / pl.splits + 4.5 : 0.33 * least_nk;
        for (int share = 2; share <= 4; share *= 2) {
            const double cost = 0.33 * least_nk / share + 2.0;
            if (pl.tiles <= (share == 2 ? kDenseShare2 : kDenseShare4) * pairs / 74 && least_nk >= 2 * share && cost < best) {
                best = cost;
                pl.share = share;
                pl.splits = 1;
            }
        }
    }
    pl.items = pl.full + left * pl.splits;
    return pl;
}

template <int MODE, int TYPE, int TN, bool TALL, bool SHARED, int P>
cudaError_t launch_tn(const DensePlan &pl, const DenseItem *items, int n, const LinearEpilogue *lin, const DenseColumnSum *sum, void *ws, int head, cudaStream_t s)
{
    static_assert(!TALL || MODE == DensePlain || MODE == DenseLinear, "dense_decode has no tall form of symmetric outputs");
    DenseParams<P> prm;
    int tiles = 0;
    for (int i = 0; i < n; ++i) {
        const DenseItem &it = items[i];
        DenseProblem &q = prm.prob[i];
        q = it.p;
        q.nk = dense_nk((DenseType)TYPE, it.k);
        q.mt = (q.M + DenseShape<TALL>::kTileRows - 1) / DenseShape<TALL>::kTileRows;
        q.nt = (q.N + TN - 1) / TN;
        q.tile0 = tiles;
        tiles += (int)dense_tiles(q, TALL, TN);
        if (!encode_operand(&prm.a[i], it.a, TYPE, (q.flags & kDenseAMn) ? 64 : 128) ||
            !encode_operand(&prm.b[i], it.b, TYPE, (q.flags & kDenseBMn) ? 64 : TN / 2))
            return cudaErrorInvalidValue;
        bool ok = true;
        if constexpr (MODE == DenseLinear) {
            ok = encode_output(&prm.o0[i], lin->y, q.M, q.N, q.N) && (lin->z == nullptr || encode_output(&prm.o1[i], lin->z, q.M, q.N, q.N));
        } else if constexpr (MODE == DenseStep) {
            if (q.flags & kDenseLast) {
                // A copy of a box that the last column cuts ends at a multiple of 16 bytes, past that column (600 x 1100 in rows
                // of 1128: four columns beside the block were zeroed), so the width has to be a multiple of 8 as well.
                // (A tensor map's rows are less than 2^40 bytes apart; a matrix of one row may say more.)
                if ((((q.ld_out | q.N) & 7) | (reinterpret_cast<uintptr_t>(q.out0) & 15)) == 0 && q.ld_out < 1ll << 39) {
                    q.flags |= kDenseTmaOut;
                    ok = encode_output(&prm.o0[i], q.out0, q.M, q.N, q.ld_out);
                }
            } else {
                ok = encode_output(&prm.o0[i], q.out0, q.M, q.N, q.ld_in) && encode_output(&prm.o1[i], q.out1, q.M, q.N, q.ld_in);
            }
        } else {
            ok = encode_output(&prm.o0[i], q.out0, q.M, q.N, q.ld_out);
        }
        if (!ok) return cudaErrorInvalidValue;
    }
    const int pairs = std::max(1, device_sms() / 2);
    prm.lin = lin ? *lin : LinearEpilogue{};
    prm.n_prob = n;
    prm.full_tiles = pl.full;
    prm.splits = pl.splits;
    prm.items = pl.items;
    prm.share = pl.share;
    prm.status = (int *)ws;
    prm.counters = (int *)((unsigned char *)ws + kDenseCounterOffset);
    prm.partial = (float *)((unsigned char *)ws + kDenseHead);
    prm.wait_limit_ns = tc_wait_limit_ns();
    prm.clear_status = head == kDenseHeadRaw;
    prm.sum = sum ? *sum : DenseColumnSum{};
    prm.skip_item = tc_skip_tile(kTcDenseProducts);

    void (*kern)(DenseParams<P>);
    if constexpr (SHARED) kern = dense_gemm_shared<MODE, TYPE, TN, P>;
    else kern = dense_gemm_pair<MODE, TYPE, TN, TALL, P>;
    static unsigned long long attr_done = 0;      // bit per device ordinal (devices beyond 63 set it every time)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev > 63 || !((attr_done >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDenseSmem);
        if (e != cudaSuccess) return e;
        if (dev <= 63) attr_done |= 1ull << dev;
    }
    if (head == kDenseHeadRaw && !TALL && pl.splits > 1) {      // only cut tiles count arrivals
        e = cudaMemsetAsync(ws, 0, kDenseZeroBytes, s);
        if (e != cudaSuccess) return e;
    }
    if constexpr (SHARED) return launch_clusters(kern, 2 * pl.share, 2 * pl.share * prm.items, kDenseThreads, kDenseSmem, s, prm);
    return launch_overlapped(kern, 2 * std::min(pairs, prm.items), kDenseThreads, kDenseSmem, s, prm);
}

template <int MODE, int TYPE, int P>
cudaError_t launch_mode(const DenseItem *items, int n, const LinearEpilogue *lin, const DenseColumnSum *sum, void *ws, size_t cap, int head, cudaStream_t s)
{
    if (n > P) return cudaErrorInvalidValue;
    const bool light = MODE == DensePlain || (MODE == DenseLinear && TYPE == DenseBf16 && !lin->residual && !lin->z && lin->act <= MODSE_ACT_RELU);
    const DensePlan pl = dense_plan((DenseType)TYPE, items, n, light, device_sms(), cap);
    if constexpr (MODE == DensePlain || (MODE == DenseLinear && TYPE == DenseBf16))
        if (pl.tall) return launch_tn<MODE, TYPE, 256, true, false, P>(pl, items, n, lin, sum, ws, head, s);
    if (pl.share > 1)       // so few tiles are 128 columns wide
        return launch_tn<MODE, TYPE, 128, false, true, P>(pl, items, n, lin, sum, ws, head, s);
    if (pl.tn == 128) return launch_tn<MODE, TYPE, 128, false, false, P>(pl, items, n, lin, sum, ws, head, s);
    return launch_tn<MODE, TYPE, 256, false, false, P>(pl, items, n, lin, sum, ws, head, s);
}

}  // namespace

size_t dense_partial_bytes(DenseType type, const DenseItem *items, int n)
{
    const DensePlan pl = dense_plan(type, items, n, false, kDenseSms, ~(size_t)0 >> 1);
    return !pl.tall && pl.splits > 1 ? (size_t)(pl.items - pl.full) * 256 * pl.tn * 4 : 0;
}

size_t dense_partial_bound(DenseType type, const DenseItem *items, int n)
{
    // dense_plan cuts into at most one piece a pair, at least 16 k-blocks and at most 16 pieces a tile
    const long long pairs = kDenseSms / 2;
    long long squares = 0, narrow = 0;
    int least_nk = 1 << 30;
    for (int i = 0; i < n; ++i) {
        squares += dense_tiles(items[i].p, false, 256);
        narrow += dense_tiles(items[i].p, false, 128);
        least_nk = std::min(least_nk, dense_nk(type, items[i].k));
    }
    const long long each = std::min(least_nk / 16, 16);
    if (each < 2) return 0;
    return squares * 2 <= pairs ? (size_t)std::min(pairs, narrow * each) * 256 * 128 * 4 : (size_t)pairs * 256 * 256 * 4;
}

cudaError_t dense_launch(DenseMode mode, DenseType type, const DenseItem *list, int n, const LinearEpilogue *lin,
                         const DenseColumnSum *sum, void *ws, size_t partial_capacity, int head, cudaStream_t s)
{
    if (n < 1 || n > kDenseMaxProblems) return cudaErrorInvalidValue;
    // longest contraction first (see dense_item)
    DenseItem items[kDenseMaxProblems];
    std::copy(list, list + n, items);
    std::stable_sort(items, items + n, [](const DenseItem &a, const DenseItem &b) { return a.k > b.k; });
    switch (mode) {
    case DenseLinear:
        return type == DenseE4m3 ? launch_mode<DenseLinear, DenseE4m3, 1>(items, n, lin, sum, ws, partial_capacity, head, s)
                                 : launch_mode<DenseLinear, DenseBf16, 1>(items, n, lin, sum, ws, partial_capacity, head, s);
    case DensePlain: return launch_mode<DensePlain, DenseBf16, 2>(items, n, lin, sum, ws, partial_capacity, head, s);
    case DenseGram: return launch_mode<DenseGram, DenseF16, kDenseMaxProblems>(items, n, lin, sum, ws, partial_capacity, head, s);
    case DensePoly: return launch_mode<DensePoly, DenseF16, kDenseMaxProblems>(items, n, lin, sum, ws, partial_capacity, head, s);
    case DenseStep: return launch_mode<DenseStep, DenseF16, kDenseMaxProblems>(items, n, lin, sum, ws, partial_capacity, head, s);
    }
    return cudaErrorInvalidValue;
}

}  // namespace modse
