// Programmatic dependent launch: a kernel's blocks take their places while the last
// blocks of the kernel before it on the stream still run.
//
// Kernels launched by launch_dependent() begin with pdl_begin(): it waits until
// everything before them on the stream is complete and visible, and only then lets the
// next kernel's blocks in.  So a kernel reads and writes what it likes after
// pdl_begin(), as after an ordinary launch, and nothing before it; no kernel is more
// than one launch ahead.
#pragma once

#include <cuda_runtime.h>

#include <utility>

namespace crc {

__device__ __forceinline__ void pdl_begin() {
    asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
}

// cluster: CTAs of a cluster (1: none).
template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem,
                             cudaStream_t stream, unsigned cluster, A&&... args) {
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    c.attrs = at;
    c.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, std::forward<A>(args)...);
}

}  // namespace crc
