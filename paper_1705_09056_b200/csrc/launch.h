// Launches that follow one another on a stream as programmatic dependents: the next kernel's CTAs may be set up while
// the last ones of its predecessor still run, and wait in chain_wait() until that has finished and its writes are visible.
#pragma once
#include <cuda_runtime.h>

#include <utility>

namespace dpsgd {

// chain_next() at a kernel's start lets its successor begin (all CTAs are resident once the last has called it, so the
// successor takes no room from it); a kernel launched with launch_chained calls chain_wait() before it touches memory.  Only
// a kernel that waits is promised to see what the kernels before it have written, whatever they have waited for themselves.
__device__ __forceinline__ void chain_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// cluster: CTAs per cluster along x (1: none); the grid is a multiple of it.
template <typename... P, typename... A>
cudaError_t launch_chained_clusters(void (*kernel)(P...), int cluster, dim3 grid, unsigned threads, size_t smem,
                                    cudaStream_t stream, A&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

template <typename... P, typename... A>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream, A&&... args) {
    return launch_chained_clusters(kernel, 1, grid, threads, smem, stream, std::forward<A>(args)...);
}

}  // namespace dpsgd
