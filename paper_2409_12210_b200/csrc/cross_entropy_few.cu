// The logits of a few rows (up to 32) and their softmax sums: the part of modse_cross_entropy that reads the vocabulary's matrix.
//
// What bounds it is reading w once.  Tiles of 256 rows by 256 of the vocabulary would multiply zeros most of the time, and
// there would be too few of them to go round (125 for 32000, on 74 pairs of SMs).  Here rows of w are the rows of a
// tcgen05 product and the tokens its columns, and a tile is as high as gives each block the same number of them: at most 128
// rows, a multiple of eight (32000: 286 tiles of 112, two a block).  24 rows of 2048 over 32000: 32 to 33 us, 3 more as a
// dense product; 32 of 4096 over 128000: 172 us, 6.1 TB/s, against 195.
#include <algorithm>

#include "activations.h"
#include "cross_entropy.h"
#include "launch.h"
#include "tc_gemm.h"
#include "tc_stream.h"

namespace modse {
namespace {

using namespace stream;

constexpr float kLog2e = 1.4426950408889634f;

struct FewArgs {
    LossEpilogue loss;
    int *status;
    unsigned long long wait_limit_ns;
    int n, vocabulary, blocks /* of 64 columns */, height, tiles;
    int skip_tile;               // debugging: the tile whose weights are not asked for, nor any of its block behind it (-1: none)
};

template <int N>
__global__ void __launch_bounds__(kTcThreads, 1) loss_few_kernel(const __grid_constant__ FewArgs p, const __grid_constant__ CUtensorMap map_w,
                                                                 const __grid_constant__ CUtensorMap map_x)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ Ring ring;
    __shared__ __align__(16) float out[N][kGroupRows];
    __shared__ long long label[N];
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_w)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_x)) : "memory");
    }
    tc_begin<N>(ring, 1);
    wait_for_earlier_kernels();
    allow_next_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *p.status = kDevOk;
        *p.loss.counter = 0;
    }
    const WaitCtx wc{&ring.abort_flag, p.status, p.wait_limit_ns};
    Place st(kTcStages), acc(2);
    if (warp >= kLoader) {
        if (lane == 0) {
            const int pairs = (p.blocks + kPair - 1) / kPair, boxes = (p.n + 15) / 16;
            bool ok = true;
            int issued = 0, turn = warp - kLoader;       // the next of a tile's stages that is this thread's
            st.skip(turn);
            for (int tile = blockIdx.x; ok && tile < p.tiles && tile != p.skip_tile; tile += gridDim.x) {
                for (; turn < pairs; turn += kLoaders) {
                    if (!mbar_wait(smem_u32(&ring.empty[st.at]), st.phase ^ 1u, wc)) { ok = false; break; }
                    const uint32_t bar = smem_u32(&ring.full[st.at]), to = stages + st.at * Tc<N>::kStage;
                    const int held = min(kPair, p.blocks - kPair * turn);
                    mbar_arrive_expect_tx(bar, held * (p.height * 128 + boxes * 2048));
                    for (int c = 0; c < held; ++c) {
                        const int col = (kPair * turn + c) * 64;
                        tma_load_2d(to + c * kBlockBytes, &map_w, bar, col, tile * p.height);
                        for (int i = 0; i < boxes; ++i) tma_load_2d(to + Tc<N>::kTokens + c * N * 128 + i * 2048, &map_x, bar, col, 16 * i);
                    }
                    st.skip(kLoaders);
                    ++issued;
                }
                turn -= pairs;
            }
            if (!ok) drain(ring, st, issued, p.wait_limit_ns);
        }
    } else if (warp == kIssuer) {
        if (lane == 0)
            for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x)
                if (!tc_multiply<N>(ring, st, acc, stages, p.blocks, p.n, wc)) break;
    } else if (warp < kTeamWarps / 2) {
        if (threadIdx.x < N) label[threadIdx.x] = threadIdx.x < p.n ? p.loss.labels.at(threadIdx.x) : -1;
        for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
            uint32_t v[N];
            const bool ok = tc_take<N>(ring, acc, v, wc);
            if (ok)
#pragma unroll
                for (int t = 0; t < N; ++t) out[t][32 * warp + lane] = __uint_as_float(v[t]);
            if (!half_sync(ok)) break;
            // a warp takes the tile's logits of a token, four a lane; rows past the tile's or the vocabulary's last one are none
            const long long row0 = (long long)tile * p.height;
            const int rows = (int)min((long long)p.height, p.vocabulary - row0);
#pragma unroll 4
            for (int t = warp; t < p.n; t += kTeamWarps / 2) {
                const float4 f = *reinterpret_cast<const float4 *>(&out[t][4 * lane]);
                float z[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = 4 * lane + i < rows ? z[i] : -INFINITY;
                float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                // M as LossEpilogue::part has it
                const float m = fmaxf(fminf(top, 3.402823466e38f), -3.402823466e38f);
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += ex2_approx((z[i] - m) * kLog2e);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                if (lane == 0) {
                    __stcg(p.loss.part + (size_t)tile * p.n + t, make_float2(m, sum));
                    const long long at = label[t] - row0;
                    if (at >= 0 && at < rows) p.loss.picked[t] = out[t][at];
                }
            }
            half_sync(true);                 // `out` has been read
        }
    }
    tc_end<N>(ring);
}

template <int N>
cudaError_t launch(const FewArgs &a, const CUtensorMap &w, const CUtensorMap &x, cudaStream_t s)
{
    static DeviceFlags done;
    const cudaError_t e = allow_smem(loss_few_kernel<N>, kTcSmem<N>, done);
    return e != cudaSuccess ? e : launch_overlapped(loss_few_kernel<N>, std::min(a.tiles, kDenseSms), kTcThreads, kTcSmem<N>, s, a, w, x);
}

}  // namespace

// A tcgen05 instruction of 128 rows takes about 75 clocks however few of them are loaded, so low tiles of long rows are bound by
// those (8192 columns: 35 us a tile), where a dense product cuts the contraction: 32 rows of 8192 over 4700 (tiles of 32) take 40 us
// here and 32 there, over 10000 (of 72) 42 and 48; of 4096 over 2300 (of 16) 25 either way, of 2048 over 4700 17 and 21.
bool few_takes(int n, int d, int vocabulary) { return n <= kFewRows && (d <= 4096 || few_tiles(vocabulary).height >= 48); }

FewTiles few_tiles(int vocabulary)
{
    FewTiles t;
    const int most = kGroupRows * kDenseSms, each = (vocabulary + most - 1) / most, share = each * kDenseSms;      // tiles a block, in all
    t.height = ((vocabulary + share - 1) / share + 7) / 8 * 8;
    t.count = (vocabulary + t.height - 1) / t.height;
    return t;
}

cudaError_t launch_loss_few(int n, int d, int vocabulary, const void *x, const void *w, const LossEpilogue &loss, int *status, cudaStream_t s)
{
    const FewTiles t = few_tiles(vocabulary);
    CUtensorMap map_w, map_x;
    if (!encode_2d(&map_w, w, vocabulary, d, 2ll * d, t.height) || !encode_2d(&map_x, x, n, d, 2ll * d, 16)) return cudaErrorInvalidValue;
    const FewArgs a{loss, status, tc_wait_limit_ns(), n, vocabulary, (d + 63) / 64, t.height, t.count, tc_skip_tile(kTcDenseProducts)};
    return n <= 16 ? launch<16>(a, map_w, map_x, s) : launch<32>(a, map_w, map_x, s);
}

}  // namespace modse
