// Shared host/device helpers of the library: status plumbing and launch checks.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include "war.h"

// Sticky device status word: the first device-side problem since the last war_device_status() call.
// It is one __device__ variable defined in war_api.cu; kernels of other translation units receive its
// address as an argument (war_status_word() resolves it once per device).
int* war_status_word();

__device__ __forceinline__ void war_set_device_status(int* status_word, int code) {
    atomicCAS(status_word, 0, code);
}

#define WAR_CUDA_TRY(expr)                                     \
    do {                                                       \
        cudaError_t e__ = (expr);                              \
        if (e__ != cudaSuccess) {                              \
            (void)cudaGetLastError();                          \
            return e__ == cudaErrorMemoryAllocation ? WAR_ERR_OOM : WAR_ERR_CUDA; \
        }                                                      \
    } while (0)

#define WAR_LAUNCH_CHECK()                                     \
    do {                                                       \
        cudaError_t e__ = cudaGetLastError();                  \
        if (e__ != cudaSuccess) return WAR_ERR_CUDA;           \
    } while (0)

// A launch that the device prepares while the kernel before it on the stream comes to its end.  The kernel begins with war_wait_before(),
// so it reads and writes nothing before that one is through and its results are there.
__device__ __forceinline__ void war_wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... Params, class... Args>
static inline war_status_t war_launch_behind(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    WAR_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...));
    return WAR_OK;
}

static inline int64_t war_ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
