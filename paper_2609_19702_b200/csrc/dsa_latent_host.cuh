// What the translation units of the latent-cache calls share on the host.
#pragma once
#include <cmath>

#include "dsa_host.cuh"

namespace dsa {

// step: the call attends (and so needs lengths and a scale); the row calls only need to know where rows lie
inline int32_t check_latent(const dsa_latent* l, bool step) {
    if (!l) return DSA_ERR_INVALID_ARG;
    if (l->batch < 0 || l->max_seq_len < 0) return DSA_ERR_INVALID_ARG;
    if (l->dtype != DSA_BF16 && l->dtype != DSA_F32) return DSA_ERR_UNSUPPORTED;
    if (l->latent_dim != 256 && l->latent_dim != 512) return DSA_ERR_UNSUPPORTED;
    if (l->rope_dim < 8 || l->rope_dim > 64 || l->rope_dim % 8) return DSA_ERR_UNSUPPORTED;
    if (step && !(l->sm_scale > 0.f && std::isfinite(l->sm_scale))) return DSA_ERR_INVALID_ARG;
    if (l->batch == 0) return DSA_OK;
    if (!l->cache || !aligned16(l->cache) || (step && !l->seq_len)) return DSA_ERR_INVALID_ARG;
    const int64_t vec = l->dtype == DSA_BF16 ? 8 : 4;
    if (l->stride_batch < 0 || l->stride_token < l->latent_dim + l->rope_dim) return DSA_ERR_INVALID_ARG;
    if (l->stride_batch % vec || l->stride_token % vec) return DSA_ERR_INVALID_ARG;
    if (l->block_table) {
        if (l->block_size < 1 || l->max_blocks < 1 || l->num_blocks < 1) return DSA_ERR_INVALID_ARG;
        if ((int64_t)l->max_blocks * l->block_size < l->max_seq_len) return DSA_ERR_INVALID_ARG;
    }
    return DSA_OK;
}

// A launch that may begin while the one in front ends (its kernel waits for that one's writes itself).
template <class Kern, class... Args>
cudaError_t launch_clusters(Kern kern, int cluster, int64_t blocks, int threads, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}
template <class Kern, class... Args>
cudaError_t launch_dependent(Kern kern, int64_t blocks, int threads, size_t smem, cudaStream_t st, const Args&... args) {
    return launch_clusters(kern, 1, blocks, threads, smem, st, args...);
}

cudaError_t latent_prepare();                                // configure the kernels for the current device
cudaError_t prompt_prepare();

}  // namespace dsa
