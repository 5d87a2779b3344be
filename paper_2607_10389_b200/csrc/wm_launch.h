// Launch helpers of the host side.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/wm.h"

namespace wm {

// Launch a kernel that may start before the kernel enqueued just before it on the stream has
// finished (it waits inside, see grid_dep_wait).  `cluster`: blocks of a cluster.
template <typename... Params, typename... Args>
static void launch_after_clustered(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, uint32_t cluster, cudaStream_t s, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
static void launch_after(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args&&... args)
{
    launch_after_clustered(kernel, grid, block, smem, 1, s, static_cast<Params>(args)...);
}

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static inline wm_status launch_status()
{
    return cudaGetLastError() == cudaSuccess ? WM_OK : WM_ERR_CUDA;
}

}  // namespace wm
