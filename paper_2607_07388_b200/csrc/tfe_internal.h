// Shared by the library's translation units; not part of the C ABI.
#ifndef TFE_INTERNAL_H
#define TFE_INTERNAL_H

#include <cuda_runtime.h>

#include "../../include/tfe.h"

// TFE_OK, or TFE_ERR_CUDA with the text kept for tfe_last_cuda_error() of this thread (the sticky error is cleared).
__attribute__((visibility("hidden"))) tfe_status tfe_note_cuda(cudaError_t e, const char *what);

#ifdef __CUDACC__
// Launch with programmatic stream serialisation: the launch is set up while the kernel before it on the stream drains.  Only for
// kernels that call tfe_wait_for_stream() before they read or write anything in device memory.  cluster: blocks per cluster.
template <typename... Params, typename... Args>
static inline tfe_status tfe_launch_serial(void (*kernel)(Params...), unsigned grid, unsigned threads, unsigned cluster, size_t smem,
                                           cudaStream_t stream, const char *what, const Args &...args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    return tfe_note_cuda(cudaLaunchKernelEx(&cfg, kernel, args...), what);
}
static __device__ __forceinline__ void tfe_wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif

#endif
