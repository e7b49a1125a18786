// Launches that may begin while the kernel before them on the stream ends, as far as it lets them.
#pragma once
#include <cuda_runtime.h>
#include <string.h>

namespace ardiff {

// First in a kernel that launch_early() starts, before any access to memory: waits until all kernels before it are done and what they
// wrote can be read. Then lets the next one be set up: it waits here in turn.
__device__ __forceinline__ void begin_kernel() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Back to back, calls of a few microseconds are 1 to 2 us apart less than with plain launches.
template <typename K, typename... A>
inline bool launch_early(K kernel, unsigned grid, unsigned threads, unsigned cluster, size_t shared, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = shared; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess;
    return cudaGetLastError() == cudaSuccess && ok;
}

}  // namespace ardiff
