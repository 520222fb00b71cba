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

// 4-D tensor map of 16-bit values (fp16 if `f16`, else bf16): inner dimension first, strides of the
// outer three in bytes, boxes of 64 x 1 x rows x 1 values in the 128-byte swizzle, zero fill.
// Call rt_current_device first.
int rt_encode_rows(CUtensorMap *tm, const void *base, bool f16, const uint64_t (&dims)[4], const uint64_t (&strides)[3],
                   int rows);

// Host-side knobs of the kernels' bounded waits (cudallm_debug_set).
unsigned long long rt_wait_limit_ns();
bool rt_take_skip_loads();             // one-shot: the next attention launch loads nothing

// Where the attention kernels of device `dev` (current) report a wait that ran out.
int rt_attention_status_word(int dev, int **out);
// Status word of the attention kernels on device `dev` (current): read, and cleared if it was set; left alone (`host`
// too) where none of them has been launched.  Defined in xattn.cu.
int rt_xattn_status(int dev, int (&host)[2]);

#define RT_CUDA_TRY(expr)                                              \
    do {                                                               \
        cudaError_t e__ = (expr);                                      \
        if (e__ != cudaSuccess) return cudallm::rt_cuda_fail(e__, #expr); \
    } while (0)

// Launch with programmatic stream serialisation (the kernel calls griddepcontrol.wait before it
// touches global memory): its launch latency hides behind the previous kernel of the stream.
// rt_launch_cluster: the same in clusters of `cluster` CTAs along x.
template <typename... KArgs, typename... Args>
int rt_launch_cluster(void (*kernel)(KArgs...), dim3 grid, unsigned cluster, unsigned block, size_t smem, cudaStream_t stream,
                      const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
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
    RT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return CUDALLM_OK;
}
template <typename... KArgs, typename... Args>
int rt_launch(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream, const Args &...args)
{
    return rt_launch_cluster(kernel, grid, 1, block, smem, stream, args...);
}

}  // namespace cudallm
