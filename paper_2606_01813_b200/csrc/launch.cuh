// Host-side launch helper shared by the entry points.
#pragma once
#include <cuda_runtime.h>

namespace cadd {

// Launch with programmatic stream serialization: the grid may be set up and its CTAs dispatched while the previous
// kernel of the stream drains; every kernel launched this way starts with griddepcontrol.wait, which returns once the
// previous kernel has completed and its writes are visible (and at once when there is no such dependency).
// Costs a few microseconds more on the host than a plain launch, so launch-bound (small) problems ask for `overlap` = false.
template <typename... KArgs, typename... Args>
static cudaError_t launch_dependent(bool overlap, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
    if (!overlap) {
        kernel<<<grid, block, smem, st>>>(args...);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace cadd
