// Launches that may begin before the kernel ahead of them in the stream has ended (programmatic dependent launch).
#pragma once

#include <cuda_runtime.h>

namespace modse {

// A kernel launched by launch_overlapped or launch_clusters sets itself up (barriers, tensor memory, address arithmetic)
// while the kernel ahead of it drains, and calls wait_for_earlier_kernels before it touches global memory: from there on
// everything the stream held before it has completed and is visible.  A kernel that calls allow_next_kernel lets one
// launched this way start its set-up as soon as SMs have room; without the call it may start when the blocks have left.
// What an earlier kernel writes is not read-only for the lifetime of a kernel that starts this early: it is read with plain
// loads, not through ld.global.nc (__ldg).
__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void allow_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Such a launch, with blocks in clusters of `cluster`.
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kern)(P...), int cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t s, A &&...args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A &&...args)
{
    return launch_clusters(kern, 1, grid, block, smem, s, args...);
}

}  // namespace modse
