// Launch of a kernel that may be placed while the one before it in the stream still runs: it waits for that one's completion itself
// (griddepcontrol.wait) before it touches global memory.
#ifndef CCL_LAUNCH_CUH_
#define CCL_LAUNCH_CUH_

#include "ccl_common.h"

namespace ccl {

// cluster: CTAs of a thread-block cluster (along the grid's first dimension)
template <typename... Params, typename... Args>
static ccl_status launch_early_clusters(void (*kernel)(Params...), dim3 grid, int threads, int cluster, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    count_launch();
    return CCL_OK;
}

template <typename... Params, typename... Args>
static ccl_status launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem_bytes, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem_bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    count_launch();
    return CCL_OK;
}

}  // namespace ccl

#endif  // CCL_LAUNCH_CUH_
