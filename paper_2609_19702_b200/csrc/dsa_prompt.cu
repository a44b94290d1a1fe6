// Attention of prompts with expanded keys and values: argument checks and launch (dsa_latent_prompt).
#include <algorithm>
#include <cmath>

#include "dsa_latent_host.cuh"
#include "dsa_prompt_f32.cuh"

namespace {

using namespace dsa;

int32_t check_prompt(const dsa_prompt* p) {
    if (!p) return DSA_ERR_INVALID_ARG;
    if (p->batch < 0 || p->num_heads < 1 || p->q_tokens < 0 || p->kv_tokens < 0 || p->max_q_len < 0) return DSA_ERR_INVALID_ARG;
    if (p->dtype != DSA_BF16 && p->dtype != DSA_F32) return DSA_ERR_UNSUPPORTED;
    if ((p->nope_dim != 64 && p->nope_dim != 128) || p->value_dim != p->nope_dim) return DSA_ERR_UNSUPPORTED;
    if (p->rope_dim < 8 || p->rope_dim > 64 || p->rope_dim % 8) return DSA_ERR_UNSUPPORTED;
    if (!(p->sm_scale >= 0.f) || !std::isfinite(p->sm_scale)) return DSA_ERR_INVALID_ARG;
    if (p->num_heads > 1024 || p->batch > (1 << 20)) return DSA_ERR_UNSUPPORTED;
    const int64_t vec = p->dtype == DSA_BF16 ? 8 : 4;
    const int64_t strides[7] = {p->q_stride_token, p->q_stride_head, p->k_stride_token, p->k_stride_head, p->rope_stride_token,
                                p->v_stride_token, p->v_stride_head};
    for (int64_t s : strides)
        if (s < 0 || s % vec) return DSA_ERR_INVALID_ARG;
    if ((p->q_tokens > 1 && p->q_stride_token < p->nope_dim + p->rope_dim) ||
        (p->kv_tokens > 1 && (p->k_stride_token < p->nope_dim || p->rope_stride_token < p->rope_dim || p->v_stride_token < p->value_dim)))
        return DSA_ERR_INVALID_ARG;
    if (p->batch == 0 || p->q_tokens == 0 || p->max_q_len == 0) return DSA_OK;
    if (!p->q || !p->q_start || !aligned16(p->q)) return DSA_ERR_INVALID_ARG;
    if (p->kv_tokens > 0 && (!p->k_nope || !p->k_rope || !p->v)) return DSA_ERR_INVALID_ARG;
    if (!aligned16(p->k_nope) || !aligned16(p->k_rope) || !aligned16(p->v)) return DSA_ERR_INVALID_ARG;
    return DSA_OK;
}

template <typename T, int D>
cudaError_t configure_f32() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return configure_smem(dsa_prompt_f32_kernel<T, D>, PromptF32Cfg<D>::SMEM, done);
}
template <typename T, int D>
cudaError_t run_f32(const PromptArgs& g, int64_t blocks, cudaStream_t st) {
    const cudaError_t e = configure_f32<T, D>();
    return e != cudaSuccess ? e : launch_dependent(dsa_prompt_f32_kernel<T, D>, blocks, kStreamWarps * 32, PromptF32Cfg<D>::SMEM, st, g);
}

}  // namespace

namespace dsa {
cudaError_t prompt_prepare() {
    cudaError_t e = configure_f32<float, 64>();
    if (e == cudaSuccess) e = configure_f32<float, 128>();
    if (e == cudaSuccess) e = configure_f32<__nv_bfloat16, 64>();
    if (e == cudaSuccess) e = configure_f32<__nv_bfloat16, 128>();
    return e;
}
}  // namespace dsa

extern "C" {

int32_t dsa_latent_prompt(const dsa_prompt* p, void* out, float* lse, void* stream) {
    const int32_t rc = check_prompt(p);
    if (rc != DSA_OK) return rc;
    if (p->batch == 0 || p->q_tokens == 0 || p->max_q_len == 0) return DSA_OK;
    if (!out || !lse || !aligned16(out)) return DSA_ERR_INVALID_ARG;
    PromptArgs g = {};
    g.q = p->q; g.k = p->k_nope; g.kr = p->k_rope; g.v = p->v;
    g.q_tok = p->q_stride_token; g.q_head = p->q_stride_head;
    g.k_tok = p->k_stride_token; g.k_head = p->k_stride_head;
    g.r_tok = p->rope_stride_token;
    g.v_tok = p->v_stride_token; g.v_head = p->v_stride_head;
    g.q_start = p->q_start; g.kv_start = p->kv_start;
    g.batch = p->batch; g.H = p->num_heads; g.P = p->rope_dim;
    g.q_tokens = p->q_tokens; g.kv_tokens = p->kv_tokens;
    g.max_q_len = std::min(p->max_q_len, p->q_tokens);
    g.causal = p->causal ? 1 : 0;
    g.scale_log2 = (p->sm_scale > 0.f ? p->sm_scale : 1.f / std::sqrt((float)(p->nope_dim + p->rope_dim))) * LOG2E;
    g.out = out;
    g.lse = lse;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t blocks = ((int64_t)g.max_q_len + kPromptF32Block - 1) / kPromptF32Block * p->num_heads * p->batch;
    if (blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    cudaError_t e;
    if (p->dtype == DSA_BF16)
        e = p->nope_dim == 64 ? run_f32<__nv_bfloat16, 64>(g, blocks, st) : run_f32<__nv_bfloat16, 128>(g, blocks, st);
    else
        e = p->nope_dim == 64 ? run_f32<float, 64>(g, blocks, st) : run_f32<float, 128>(g, blocks, st);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

}  // extern "C"
