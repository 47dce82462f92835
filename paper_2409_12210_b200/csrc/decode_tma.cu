// modse_decode for bf16 layers whose extents are multiples of 64: weights come by TMA, column blocks of 64 elements (128
// bytes) of several rows at a time, and nothing that the inner loops read comes from global memory.
//
// The last point is what counts.  With 130 to 190 KB of weights in flight to an SM a row of x asked for beside them arrives
// only behind them, and the warps wait for it longer than for anything else.  So rows of x lie in shared memory before they
// are multiplied, and the gated hidden rows, which are used once by each group of 128 rows of W_down, come by TMA in the
// same stage as the weights.
//
// First kernel, up to eight tokens: units of eight hidden columns, whose rows of W_gate and W_up are one mma.sync fragment; the
// eight warps split the contraction, each with a ring that it fills for itself, and sums meet once a unit.  So there are enough
// units to go round 148 SMs evenly, and a block reads whole rows, 64 KB side by side, at a time.
// First kernel, more tokens: a fragment of weights would be read from shared memory once per eight tokens, and the rows of x with
// it; 64 columns' rows of W_gate and W_up and up to 32 rows of x are the operands of tcgen05 instead.
// Second kernel: 128 rows of W_down and 16 or 32 hidden rows are the operands of tcgen05 instructions as TMA leaves them, so no
// warp touches them.  What a block asks for is 128 bytes of each of 128 rows that lie far apart, so the blocks of a group of
// rows take its column blocks in turn: together they read a few KB of each row at a time.
//
// Both kernels of 32 tokens over eight experts of 5632 x 2048 (554 MB, 84 us at the rate of a plain copy): 118 us (153 as
// modse_forward).  Fragments straight from global memory 130, 16-byte asynchronous copies into rings 178, bulk copies of 256 bytes
// 270, one ring that all warps share 198, rows of x gathered by TMA (0.25 us for four rows) 376.  One token of the same layer
// (138 MB, 21 us): 38 us (91 as modse_forward), of which 4 are the routing, which every block does for itself, and 2 to 3 each the
// first data's way and the meeting of the blocks that share a group of rows, in both kernels.
//
// A fragment's rows lie 128 bytes apart in a stage, swizzled by TMA in 16-byte pieces.  Row i of a fragment's half plays row
// row_of(i) of the stage, so that the two rows that eight neighbouring lanes read lie in opposite halves of the banks.
#include <algorithm>

#include "decode.h"
#include "tc_stream.h"

namespace modse {
namespace decode {
namespace {

using namespace stream;
static_assert(kWarps == kTeamWarps, "the warps that take results are the first of the team");

constexpr int kSmemMost = 232448 - 6 * 1024;     // dynamic shared memory, beside what the kernels declare

struct Maps {
    CUtensorMap gate, up;        // [column block][row][64 elements], boxes of 8 rows and up_blocks blocks
    CUtensorMap gate64, up64;    // boxes of 64 rows x 64 elements
    CUtensorMap down;            // boxes of 128 rows x 64 elements
    CUtensorMap hidden;          // boxes of 16 rows x 64 elements
};

__device__ __forceinline__ int row_of(int g) { return (g >> 1) | ((g & 1) << 2); }

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void prefetch(const CUtensorMap &map) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory"); }
__device__ __forceinline__ uint4 lds(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// A column block of a fragment's sixteen rows times eight tokens.  rows: of the fragment's rows 0 .. 7 (unswizzled row 0), `second`
// bytes ahead of rows 8 .. 15; x: the lane's 16 bytes of both units of its token's row.
__device__ __forceinline__ void add_block(float (&acc)[4], uint32_t rows, uint32_t second, const uint4 (&x)[2])
{
    const int lane = threadIdx.x & 31, t = lane & 3, row = row_of(lane >> 2);
    uint4 a[2], b[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t at = rows + row * 128 + (((4 * h + t) ^ row) << 4);
        a[h] = lds(at);
        b[h] = lds(at + second);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo[4] = {a[h].x, b[h].x, a[h].y, b[h].y}, hi[4] = {a[h].z, b[h].z, a[h].w, b[h].w};
        mma_16816(acc, lo, x[h].x, x[h].y, false);
        mma_16816(acc, hi, x[h].z, x[h].w, false);
    }
}

// The rows of x of an expert, in shared memory where they fit: rows 64 bytes more than a multiple of 128 apart, so that the two
// rows that eight neighbouring lanes read lie in opposite halves of the banks.
struct Tokens {
    uint32_t at;
    int pitch, room;                     // bytes a row, rows
    bool held;
    // Every thread of the team calls it; what was held before is no longer needed.
    __device__ __forceinline__ void hold(const DecodeArgs &p, const Routing &r, int s)
    {
        const int count = r.first[s + 1] - r.first[s], row = 2 * p.m.d, pieces = row / 16;
        held = count <= room;
        team_sync();
        if (held)
            for (int i = threadIdx.x; i < count * pieces; i += kThreads) {
                const int c = i / pieces, at16 = (i - c * pieces) * 16;
                const uint4 v = *reinterpret_cast<const uint4 *>(p.x + (size_t)(r.pick[r.first[s] + c] / p.m.k) * row + at16);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + c * pitch + at16), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
            }
        team_sync();
    }
};

// ---- first kernel ----
constexpr int kUpBlocks = 4 /* at most, of a stage */, kUpBytes = kUpBlocks * kRows * 128, kUpDepth = 2;
constexpr int kUpRing = kWarps * kUpDepth * kUpBytes;

struct UpShared {
    unsigned long long full[kWarps][kUpDepth];
    float part[2][kWarps][8][kRows + 1];          // two of them, so that one meeting a unit is enough
    Routing r;
    float z[8 * kInBlockExperts];
    __align__(16) int idx[kMaxPicks], scan[kMaxPicks];
    int abort_flag;
};

__global__ void __launch_bounds__(kThreads, 1) decode_up_few(const __grid_constant__ DecodeArgs p, const __grid_constant__ Maps maps)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ UpShared sh;
    Routing &r = sh.r;
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int k = p.m.k, row = 2 * p.m.d, blocks = p.m.d / 64;
    if (threadIdx.x < kWarps * kUpDepth) mbar_init(smem_u32(&sh.full[0][0] + threadIdx.x), 1);
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        prefetch(maps.gate);
        prefetch(maps.up);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    fetch_router(p, row);
    wait_for_earlier_kernels();
    allow_next_kernel();
    route<__nv_bfloat16, 1>(p, sh.z, sh.part[0], sh.idx, sh.scan, r);
    if (blockIdx.x == 0) publish(p, r, sh.idx);
    const WaitCtx wc{&sh.abort_flag, p.status, p.wait_limit_ns};
    int all = 0;
    for (int s = 0; s < r.met; ++s) all += r.width[s] / kUnitCols;
    int begin, end;
    share_of(all, begin, end);
    // the warp's blocks of a unit's rows, in stages of stage_blocks; lane 0 starts the copies
    const int lo = blocks * warp / kWarps, hi = blocks * (warp + 1) / kWarps, stage_blocks = p.up_blocks;
    const uint32_t ring = stages + warp * (kUpDepth * kUpBytes), bar = smem_u32(sh.full[warp]);
    int in = 0, out = 0, pending = 0, step = lo;
    uint32_t phase = 0;
    bool ok = true;
    UnitCursor ahead{begin, 0, 0, 0}, at = ahead;
    bool more = lo < hi && begin < end && (int)blockIdx.x != p.skip_block && ahead.settle(r);
    auto push = [&] {                            // every lane is done with the stage
        if (!more || !ok) return;
        __syncwarp();
        if (lane == 0) {
            const int first = r.offset[ahead.s] + ahead.c0;
            const uint32_t to = ring + in * kUpBytes, on = bar + 8 * in;
            mbar_arrive_expect_tx(on, stage_blocks * (kRows * 128));
            tma_load_3d(to, &maps.gate, on, 0, first, step);
            tma_load_3d(to + stage_blocks * 1024, &maps.up, on, 0, first, step);
        }
        in = in + 1 == kUpDepth ? 0 : in + 1;
        ++pending;
        step += stage_blocks;
        if (step >= hi) {
            step = lo;
            more = ++ahead.u < end && ahead.settle(r);
        }
    };
    for (int i = 0; i < kUpDepth; ++i) push();
    const int pitch = row + 64;
    Tokens x{stages + kUpRing, pitch, p.x_room / pitch, false};
    float acc[4];
    int held = -1, count = 0;
    const unsigned char *mine = nullptr;         // the lane's row of x, where the rows are not held
    uint32_t cols = 0;                           // ... and where they are
    for (int round = 0; at.u < end && at.settle(r); ++at.u, ++round) {
        if (at.s != held) {
            held = at.s;
            count = r.first[at.s + 1] - r.first[at.s];
            const int q = min(g, count - 1);
            mine = p.x + (size_t)(r.pick[r.first[at.s] + q] / k) * row + t * 16;
            cols = x.at + q * pitch + t * 16;
            x.hold(p, r, at.s);
        }
        acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
        for (int b = lo; b < hi && ok; b += stage_blocks) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar + 8 * out, phase, wc));
            if (!ok) break;
            const uint32_t rows = ring + out * kUpBytes;
#pragma unroll
            for (int i = 0; i < kUpBlocks; ++i)
                if (i < stage_blocks && b + i < hi) {
                    uint4 v[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int from = (b + i) * 128 + h * kUnit;
                        v[h] = x.held ? lds(cols + from) : load_shared_rows(mine + from, true);
                    }
                    add_block(acc, rows + i * 1024, stage_blocks * 1024, v);
                }
            --pending;
            if (++out == kUpDepth) {
                out = 0;
                phase ^= 1u;
            }
            push();
        }
        auto &part = sh.part[round & 1];
        const int row8 = row_of(g);
#pragma unroll
        for (int i = 0; i < 4; ++i) part[warp][2 * t + (i & 1)][row8 + 8 * (i >> 1)] = acc[i];
        team_sync();
        if (threadIdx.x < count * kUnitCols) {
            const int i = threadIdx.x / kUnitCols, c = threadIdx.x % kUnitCols, q = r.first[at.s] + i;
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                a += part[w][i][c];
                b += part[w][i][c + kUnitCols];
            }
            // one rounding of the gated hidden value, as in modse_forward
            reinterpret_cast<__nv_bfloat16 *>(p.hidden + q * p.ld)[at.c0 + c] = __float2bfloat16_rn(gated(r.gate[r.pick[q]], a, b));
        }
    }
    // after a wait that expired the copies in flight land before the warp leaves, or the limit passes again
    for (; !ok && pending > 0; --pending) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(bar + 8 * out, phase) && global_ns() - t0 < p.wait_limit_ns) {}
        if (++out == kUpDepth) {
            out = 0;
            phase ^= 1u;
        }
    }
}

constexpr int kManyCols = 64;                    // hidden columns of a unit: 64 rows of W_gate over 64 of W_up

template <int N>
__global__ void __launch_bounds__(kTcThreads, 1) decode_up_many(const __grid_constant__ DecodeArgs p, const __grid_constant__ Maps maps)
{
    constexpr int NTM = N / 8;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Routing r;
    __shared__ Ring ring;
    __shared__ __align__(16) float out[N][kGroupRows];
    __shared__ __align__(16) int idx[kMaxPicks], scan[kMaxPicks];
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int k = p.m.k, blocks = p.m.d / 64;
    if (threadIdx.x == 0) {
        prefetch(maps.gate64);
        prefetch(maps.up64);
    }
    tc_begin<N>(ring, 2);
    fetch_router(p, 2 * p.m.d);
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (warp < kWarps) {
        // the logits and their partial sums, where the ring will be
        typedef float Part[kWarps][NTM * 8][kRows + 1];
        unsigned char *scratch = smem_raw + (stages - smem_u32(smem_raw));
        route<__nv_bfloat16, NTM>(p, reinterpret_cast<float *>(scratch + sizeof(Part)), *reinterpret_cast<Part *>(scratch), idx, scan, r);
        if (blockIdx.x == 0) publish(p, r, idx);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    const WaitCtx wc{&ring.abort_flag, p.status, p.wait_limit_ns};
    int all = 0;
    for (int s = 0; s < r.met; ++s) all += r.width[s] / kManyCols;
    int begin, end;
    share_of(all, begin, end);
    Place st(kTcStages), acc(2);
    int s = 0, base = 0;                         // the expert that unit u lies in, units ahead of it
    auto settle = [&](int u) {
        while (true) {
            const int units = r.width[s] / kManyCols;
            if (u - base < units) return (u - base) * kManyCols;
            base += units;
            ++s;
        }
    };
    if (warp >= kLoader) {
        // The weights come by TMA, the rows of x by the loading warp's lanes: 16 bytes a lane and piece, swizzled as TMA would (its
        // row gather takes 0.25 us for four rows).  The next stage's pieces are requested before this one's place is waited for.
        constexpr int P = N / 4;                 // pieces of a lane and column block: rows lane / 8 + 4 j
        const int piece = lane & 7, mine = warp - kLoader, pairs = (blocks + kPair - 1) / kPair;
        const int total = (int)blockIdx.x == p.skip_block ? 0 : (end - begin) * pairs;
        uint4 v[kPair][P];
        int count = 0, held = -1, c0 = 0, u = begin, b = mine;       // of the stage whose pieces are on their way: unit, pair of blocks
        const unsigned char *from[P];
        auto request = [&] {
            while (b >= pairs) {
                b -= pairs;
                ++u;
            }
            if (u >= end) return;
            c0 = settle(u);
            if (s != held) {
                held = s;
                count = r.first[s + 1] - r.first[s];
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const int q = min((lane >> 3) + 4 * j, count - 1);
                    from[j] = p.x + (size_t)(r.pick[r.first[s] + q] / k) * (2 * p.m.d) + piece * 16;
                }
            }
#pragma unroll
            for (int c = 0; c < kPair; ++c)
#pragma unroll
                for (int j = 0; j < P; ++j)
                    if (4 * j < count) v[c][j] = load_shared_rows(from[j] + (kPair * b + c) * 128, kPair * b + c < blocks);
        };
        st.skip(mine);
        request();
        int issued = 0;
        for (int i = mine; i < total; i += kLoaders) {
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&ring.empty[st.at]), st.phase ^ 1u, wc))) {
                if (lane == 0) drain(ring, st, issued, p.wait_limit_ns);
                break;
            }
            const uint32_t bar = smem_u32(&ring.full[st.at]), to = stages + st.at * Tc<N>::kStage;
            const int n = min(kPair, blocks - kPair * b);
            if (lane == 0) {
                const int first = r.offset[s] + c0;
                mbar_arrive_expect_tx(bar, n * kBlockBytes);
                for (int c = 0; c < n; ++c) {
                    tma_load_2d(to + c * kBlockBytes, &maps.gate64, bar, (kPair * b + c) * 64, first);
                    tma_load_2d(to + c * kBlockBytes + kBlockBytes / 2, &maps.up64, bar, (kPair * b + c) * 64, first);
                }
            }
#pragma unroll
            for (int c = 0; c < kPair; ++c)
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const int q = (lane >> 3) + 4 * j;
                    if (c < n && 4 * j < count)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                     ::"r"(to + Tc<N>::kTokens + c * N * 128 + q * 128 + ((piece ^ (q & 7)) << 4)), "r"(v[c][j].x), "r"(v[c][j].y),
                                       "r"(v[c][j].z), "r"(v[c][j].w) : "memory");
                }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            st.skip(kLoaders);
            ++issued;
            b += kLoaders;
            request();
        }
    } else if (warp == kIssuer) {
        if (lane == 0)
            for (int u = begin; u < end; ++u) {
                settle(u);
                if (!tc_multiply<N>(ring, st, acc, stages, blocks, r.first[s + 1] - r.first[s], wc)) break;
            }
    } else if (warp < kWarps / 2) {
        constexpr int kHalf = kThreads / 2;
        for (int u = begin; u < end; ++u) {
            const int c0 = settle(u), count = r.first[s + 1] - r.first[s];
            uint32_t v[N];
            const bool ok = tc_take<N>(ring, acc, v, wc);
            if (ok)
#pragma unroll
                for (int n = 0; n < N; ++n) out[n][32 * warp + lane] = __uint_as_float(v[n]);
            if (!half_sync(ok)) break;
            for (int i = threadIdx.x; i < count * kManyCols; i += kHalf) {
                const int q = i / kManyCols, c = i % kManyCols, at = r.first[s] + q;
                // one rounding of the gated hidden value, as in modse_forward
                reinterpret_cast<__nv_bfloat16 *>(p.hidden + at * p.ld)[c0 + c] =
                    __float2bfloat16_rn(gated(r.gate[r.pick[at]], out[q][c], out[q][c + kManyCols]));
            }
            half_sync(true);
        }
    }
    tc_end<N>(ring);
}

// ---- second kernel ----
// `share` blocks take the column blocks of all experts met, one after the other, of a group of rows in turn: what they ask for
// at a time lies side by side.
struct DownShare {
    int groups, share, member, first, step;      // the block's groups: first, first + step, ..
    __device__ __forceinline__ DownShare(int d, int per)
    {
        groups = (d + kGroupRows - 1) / kGroupRows;
        share = max(1, min((int)gridDim.x / groups, per / 2));
        step = max(1, (int)gridDim.x / share);
        member = blockIdx.x % share;
        first = (int)blockIdx.x / share < step ? (int)blockIdx.x / share : groups;
    }
    // the first of the column blocks from `upto` on that is the block's
    __device__ __forceinline__ int from(int upto) const { return upto + (member - upto % share + share) % share; }
};

template <int N>
__global__ void __launch_bounds__(kTcThreads, 1) decode_down_tma(const __grid_constant__ DecodeArgs p, const __grid_constant__ Maps maps)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ Routing r;
    __shared__ Ring ring;
    __shared__ int upto[kMaxPicks + 1];                       // column blocks ahead of each expert met
    __shared__ __align__(16) float out[N][kGroupRows];
    __shared__ int last;
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    if (tid == 0) {
        prefetch(maps.down);
        prefetch(maps.hidden);
    }
    tc_begin<N>(ring, 1);
    wait_for_earlier_kernels();
    allow_next_kernel();
    for (int i = tid; i < (int)(sizeof(Routing) / 4); i += kTcThreads) ((int *)&r)[i] = __ldcg((const int *)p.routing + i);
    __syncthreads();
    if (tid <= r.met) {
        int n = 0;
        for (int s = 0; s < tid; ++s) n += r.width[s] / 64;
        upto[tid] = n;
    }
    __syncthreads();
    const DownShare mine(p.m.d, upto[r.met]);
    const int groups = mine.groups, share = mine.share, step = mine.step, member = mine.member, first_group = mine.first;
    const WaitCtx wc{&ring.abort_flag, p.status, p.wait_limit_ns};
    Place st(kTcStages), acc(2);
    // the block's column blocks of expert s
    auto first_of = [&](int s) { return mine.from(upto[s]); };
    auto length_of = [&](int s) { return (upto[s + 1] - first_of(s) + share - 1) / share; };      // 0 or less: none
    if (warp >= kLoader) {
        if (lane == 0) {
            bool ok = true;
            int issued = 0, turn = warp - kLoader;       // the next of an expert's stages that is this thread's
            st.skip(turn);
            for (int group = first_group; ok && group < groups; group += step)
                for (int s = 0; ok && s < r.met; ++s) {
                    const int first = first_of(s), n = length_of(s), boxes = (r.first[s + 1] - r.first[s] + 15) / 16, col0 = r.offset[s];
                    const int pairs = (max(n, 0) + kPair - 1) / kPair;
                    for (; turn < pairs; turn += kLoaders) {
                        if (!mbar_wait(smem_u32(&ring.empty[st.at]), st.phase ^ 1u, wc)) { ok = false; break; }
                        const uint32_t bar = smem_u32(&ring.full[st.at]), to = stages + st.at * Tc<N>::kStage;
                        const int held = min(kPair, n - kPair * turn);
                        mbar_arrive_expect_tx(bar, held * (kBlockBytes + boxes * 2048));
                        for (int c = 0; c < held; ++c) {
                            const int col = (first + (kPair * turn + c) * share - upto[s]) * 64;
                            tma_load_2d(to + c * kBlockBytes, &maps.down, bar, col0 + col, group * kGroupRows);
                            for (int i = 0; i < boxes; ++i)
                                tma_load_2d(to + Tc<N>::kTokens + c * N * 128 + i * 2048, &maps.hidden, bar, col, r.first[s] + 16 * i);
                        }
                        st.skip(kLoaders);
                        ++issued;
                    }
                    turn -= pairs;
                }
            if (!ok) drain(ring, st, issued, p.wait_limit_ns);
        }
    } else if (warp == kIssuer) {
        if (lane == 0) {
            bool ok = true;
            for (int group = first_group; ok && group < groups; group += step)
                for (int s = 0; ok && s < r.met; ++s)
                    if (length_of(s) > 0) ok = tc_multiply<N>(ring, st, acc, stages, length_of(s), r.first[s + 1] - r.first[s], wc);
        }
    } else {
        bool ok = true;
        for (int group = first_group; group < groups; group += step) {
            if (warp < 4) {
                // a lane's own row of `out`: nobody else touches it before the meeting below
                float (*mine)[kGroupRows] = reinterpret_cast<float (*)[kGroupRows]>(&out[0][32 * warp + lane]);
                for (int tok = 0; tok < p.T; ++tok) mine[tok][0] = 0.f;
                for (int s = 0; s < r.met; ++s) {
                    if (length_of(s) <= 0) continue;
                    uint32_t v[N];
                    if (ok) ok = tc_take<N>(ring, acc, v, wc);
                    const int count = r.first[s + 1] - r.first[s];
                    if (ok)
#pragma unroll
                        for (int q = 0; q < N; ++q)
                            if (q < count) mine[r.pick[r.first[s] + q] / p.m.k][0] += __uint_as_float(v[q]);
                }
            }
            team_sync();
            leave_rows<kGroupRows>(p, group, &out[0][0], member, share, group * share, &last, p.y_f32 != 0);
            team_sync();                     // `out` and `last` have been read
        }
    }
    tc_end<N>(ring);
}

// ---- host ----
bool encode_3d(CUtensorMap *map, const void *base, long long rows, int d, int blocks)
{
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(d / 64)}, strides[2] = {(cuuint64_t)d * 2, 128};
    const cuuint32_t box[3] = {64, kUnitCols, (cuuint32_t)blocks};
    return encode(map, 3, base, dims, strides, box);
}

// One group of eight tokens: the first kernel on mma.sync, whose small units go round the SMs evenly; more: on tcgen05.
constexpr int kFewTokens = 8;

template <int N>
cudaError_t launch(DecodeArgs &a, const Maps &maps, int blocks, cudaStream_t s)
{
    static DeviceFlags done_few, done_up, done_down;
    cudaError_t e = allow_smem(decode_down_tma<N>, kTcSmem<N>, done_down);
    if (e != cudaSuccess) return e;
    if (N == 16 && a.T <= kFewTokens) {
        constexpr size_t most = kSmemMost - sizeof(UpShared);
        a.x_room = (int)(most - 1024 - kUpRing);
        e = allow_smem(decode_up_few, most, done_few);
        if (e == cudaSuccess) e = launch_overlapped(decode_up_few, blocks, kThreads, most, s, a, maps);
    } else {
        e = allow_smem(decode_up_many<N>, kTcSmem<N>, done_up);
        if (e == cudaSuccess) e = launch_overlapped(decode_up_many<N>, blocks, kTcThreads, kTcSmem<N>, s, a, maps);
    }
    return e != cudaSuccess ? e : launch_overlapped(decode_down_tma<N>, blocks, kTcThreads, kTcSmem<N>, s, a, maps);
}

}  // namespace

bool tma_takes(const LayerMeta &m)
{
    if (m.d % 64 != 0) return false;
    for (int e = 0; e <= m.N; ++e)
        if (m.hoff[e] % 64 != 0) return false;
    return true;
}

cudaError_t launch_tma(const DecodeArgs &args, int sms, cudaStream_t s)
{
    DecodeArgs a = args;
    Maps maps;
    // a warp's share of a row, up to kUpBlocks blocks at a time, as evenly as it goes
    const int share = (a.m.d / 64 + kWarps - 1) / kWarps, steps = (share + kUpBlocks - 1) / kUpBlocks;
    a.up_blocks = (share + steps - 1) / steps;
    const bool rows = a.T <= kFewTokens ? encode_3d(&maps.gate, a.w_gate, a.m.S, a.m.d, a.up_blocks) && encode_3d(&maps.up, a.w_up, a.m.S, a.m.d, a.up_blocks)
                                        : encode_2d(&maps.gate64, a.w_gate, a.m.S, a.m.d, 2ll * a.m.d, kManyCols) &&
                                          encode_2d(&maps.up64, a.w_up, a.m.S, a.m.d, 2ll * a.m.d, kManyCols);
    if (!rows || !encode_2d(&maps.down, a.w_down, a.m.d, a.m.S, 2ll * a.m.S, kGroupRows) ||
        !encode_2d(&maps.hidden, a.hidden, (long long)a.T * a.m.k, a.ld / 2, a.ld, 16))
        return cudaErrorInvalidValue;
    const int blocks = std::min(sms, kTmaBlocks);
    return a.T <= 16 ? launch<16>(a, maps, blocks, s) : launch<32>(a, maps, blocks, s);
}

}  // namespace decode
}  // namespace modse
