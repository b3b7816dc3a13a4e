// Launch of a kernel that may be set up while the kernel before it on the stream drains (programmatic stream serialization):
// it calls sm100::grid_dependency_wait() before it touches memory.  One exception: the second product of a few rows (few_rows_kernel with
// weights_settled) fetches weights before that.  The kernel ahead of it is the library's own first product, which does not write them
// and has itself waited for all before it (its launch_dependents comes behind its wait), so they are settled by then.
#pragma once
#include <cuda_runtime.h>

#include "sm100_ptx.cuh"

namespace atb {

template <class... Args>
cudaError_t launch_dependent(void (*kernel)(Args...), unsigned grid, unsigned block, unsigned cluster, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace atb
