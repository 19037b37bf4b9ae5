// around.cuh -- launchers of what surrounds the expert layer (internal): the balance
// losses (balance.cu), the block norms (norm.cu) and AdamW (adamw.cu).
#pragma once

#include "common.cuh"

namespace vmoe {

// launch_kernel with `ranks` CTAs along x as a cluster.
template <typename... KArgs, typename... Args>
int launch_cluster(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, int ranks, cudaStream_t s, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...) == cudaSuccess ? VMOE_OK : VMOE_ERR_CUDA;
}

size_t balance_workspace(const Dims &p);
int launch_balance(const Dims &p, const float *logits, const int32_t *idx, const uint8_t *mask, int32_t *count,
                   int32_t *tokens, float *excess, float *loss, float *parts, cudaStream_t s);
int launch_balance_bwd(const Dims &p, const float *logits, const uint8_t *mask, const int32_t *count,
                       const int32_t *tokens, const float *excess, const float *dloss, float *dlogits, cudaStream_t s);
size_t norm_bwd_workspace(const Dims &p);
int launch_block_norm(const Dims &p, const vmoe_norm *n, const void *x, const void *y, const float *post_w,
                      const float *post_b, const float *gate, const float *pre_w, const float *pre_b, void *z, void *u,
                      float *post_stat, float *pre_stat, cudaStream_t s);
int launch_block_norm_bwd(const Dims &p, const vmoe_norm *n, const void *y, const void *z, const float *post_stat,
                          const float *pre_stat, const float *post_w, const float *post_b, const float *gate,
                          const float *pre_w, const void *dz, const void *du, void *dx, void *dy, float *dpost_w,
                          float *dpost_b, float *dgate, float *dpre_w, float *dpre_b, float *parts, cudaStream_t s);
int launch_adamw(int n, const vmoe_adamw_tensor *tensors, const vmoe_adamw_config *c, cudaStream_t s);

}  // namespace vmoe
