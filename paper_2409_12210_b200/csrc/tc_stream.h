// Few rows of tokens times many rows of weights on tcgen05, bound by the weights' way from memory: one ring of stages for a
// block, filled by TMA, multiplied by one thread.
//
// A stage is a column block of 128 rows of weights and the same columns of up to N rows of tokens, and as such the two
// operands of four tcgen05 instructions: the weights' rows are the rows of the product, the tokens its columns.
// Four threads fill the ring, every fourth stage each: waiting for a place and starting the copies takes one of them 0.3 us, in
// which HBM delivers 12 KB to an SM.
#pragma once

#include "tc_device.h"

namespace modse {
namespace stream {

constexpr int kGroupRows = 128;                  // of weights
constexpr int kBlockBytes = kGroupRows * 128;    // a column block of them
constexpr int kLoaders = 4, kTeamWarps = 8, kIssuer = kTeamWarps, kLoader = kIssuer + 1;
constexpr int kTcThreads = 32 * (kTeamWarps + 1 + kLoaders);      // eight warps for results and what comes before
// Two column blocks a stage, as far as there are two: handing a stage over costs the multiplying thread 0.2 us, as long as half a
// stage of weights takes to arrive.
constexpr int kPair = 2;
template <int N> struct Tc {
    static constexpr int kTokens = kPair * kBlockBytes;            // where a stage's rows of tokens begin
    static constexpr int kStage = kPair * (kBlockBytes + N * 128);
};
constexpr int kTcStages = 5;
template <int N> constexpr size_t kTcSmem = 1024 + (size_t)kTcStages * Tc<N>::kStage;
// A loading thread that waits for a place has seen the one `loaders` stages ahead of its own emptied; it must not be two fills
// ahead of it, which the one bit of a barrier's phase cannot tell from none.
static_assert(kTcStages >= kLoaders, "stages per loading thread");

struct Ring {
    unsigned long long full[kTcStages], empty[kTcStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
};
struct Place {                                   // of a role in a ring of `n`
    int n, at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ explicit Place(int size) : n(size) {}
    __device__ __forceinline__ void skip(int steps)
    {
        for (int i = 0; i < steps; ++i) next();
    }
    __device__ __forceinline__ void next()
    {
        if (++at == n) {
            at = 0;
            phase ^= 1u;
        }
    }
};

// fills: what has to arrive for a stage to be full beside the copies' bytes
template <int N> __device__ __forceinline__ void tc_begin(Ring &ring, int fills)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < kTcStages; ++i) {
            mbar_init(smem_u32(&ring.full[i]), fills);
            mbar_init(smem_u32(&ring.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ring.acc_full[i]), 1);
            mbar_init(smem_u32(&ring.acc_empty[i]), 4);
        }
        ring.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x >> 5 == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ring.tmem)), "r"(2 * N) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
}
template <int N> __device__ __forceinline__ void tc_end(const Ring &ring)
{
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x >> 5 == kIssuer) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(ring.tmem), "r"(2 * N) : "memory");
    }
}

// One thread's part of a run of `length` column blocks, `count` tokens, that are summed up in one accumulator: false if a wait
// expired.
template <int N>
__device__ __forceinline__ bool tc_multiply(Ring &ring, Place &st, Place &acc, uint32_t stages, int length, int count, const WaitCtx &wc)
{
    if (!mbar_wait(smem_u32(&ring.acc_empty[acc.at]), acc.phase ^ 1u, wc)) return false;
    tc_fence_after();
    const uint32_t idesc = make_idesc(false, false, count <= 16 ? 16 : N), to = ring.tmem + (uint32_t)(acc.at * N);
    for (int i = 0; i < length; i += kPair) {
        if (!mbar_wait(smem_u32(&ring.full[st.at]), st.phase, wc)) return false;
        tc_fence_after();
        const uint32_t at = stages + st.at * Tc<N>::kStage;
#pragma unroll
        for (int c = 0; c < kPair; ++c) {
            if (i + c >= length) break;
            const uint64_t a = make_desc(at + c * kBlockBytes, false), b = make_desc(at + Tc<N>::kTokens + c * N * 128, false);
#pragma unroll
            for (int q = 0; q < 4; ++q) umma_bf16(to, a + 2 * q, b + 2 * q, idesc, i + c > 0 || q > 0);
        }
        umma_commit(smem_u32(&ring.empty[st.at]));
        st.next();
    }
    umma_commit(smem_u32(&ring.acc_full[acc.at]));
    acc.next();
    return true;
}
// One of the team's first four warps takes its 32 rows of an accumulator: a row a lane.
template <int N>
__device__ __forceinline__ bool tc_take(Ring &ring, Place &acc, uint32_t (&v)[N], const WaitCtx &wc)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&ring.acc_full[acc.at]), acc.phase, wc))) return false;
    tc_fence_after();
    const uint32_t from = ring.tmem + ((uint32_t)(32 * warp) << 16) + (uint32_t)(acc.at * N);
    if constexpr (N == 16) tmem_ld16(from, v);
    else tmem_ld32(from, v);
    tmem_ld_wait();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ring.acc_empty[acc.at]));
    acc.next();
    return true;
}
// After a wait of a loading thread that expired: its copies in flight land before it leaves, or the limit passes again.
// st: the place that it waited for.
__device__ __forceinline__ void drain(Ring &ring, Place st, int issued, unsigned long long limit_ns)
{
    for (int i = 0; i < issued && i * kLoaders < st.n; ++i) {
        for (int j = 0; j < kLoaders; ++j)
            if (--st.at < 0) {
                st.at = st.n - 1;
                st.phase ^= 1u;
            }
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(smem_u32(&ring.full[st.at]), st.phase) && global_ns() - t0 < limit_ns) {}
    }
}

// Meeting of the team's first four warps; true if all say so.
__device__ __forceinline__ bool half_sync(bool v)
{
    int all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((int)v), "n"(32 * kTeamWarps / 2) : "memory");
    return all != 0;
}

// ---- host ----
inline bool encode(CUtensorMap *map, int rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    return encode_tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}
inline bool encode_2d(CUtensorMap *map, const void *base, long long rows, long long cols, long long ld_bytes, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld_bytes};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return encode(map, 2, base, dims, strides, box);
}

}  // namespace stream
}  // namespace modse
