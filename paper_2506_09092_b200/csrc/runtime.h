// What the library's translation units share: device probing, the error text behind
// CUDALLM_ERR_CUDA and the launch helpers.  Defined in cudallm_gemm.cu.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/cudallm_gemm.h"

namespace cudallm {

constexpr int kRtMaxDevices = 64;

// Records `where` and the error's text for cudallm_strerror; returns CUDALLM_ERR_CUDA.
int rt_cuda_fail(cudaError_t e, const char *where);

// The current device, if it can run the kernels: its index and SM count.
int rt_current_device(int *dev, int *sm_count);

#define RT_CUDA_TRY(expr)                                              \
    do {                                                               \
        cudaError_t e__ = (expr);                                      \
        if (e__ != cudaSuccess) return cudallm::rt_cuda_fail(e__, #expr); \
    } while (0)

// Launch with programmatic stream serialisation (the kernel calls griddepcontrol.wait before it
// touches global memory): its launch latency hides behind the previous kernel of the stream.
template <typename... KArgs, typename... Args>
int rt_launch(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    RT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return CUDALLM_OK;
}

}  // namespace cudallm
