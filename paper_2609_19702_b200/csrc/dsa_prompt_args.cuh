// Arguments that the kernels of the prompt attention share (dsa_latent_prompt).
#pragma once
#include "dsa_common.cuh"

namespace dsa {

struct PromptArgs {
    const void* q;
    const void* k;
    const void* kr;
    const void* v;
    int64_t q_tok, q_head, k_tok, k_head, r_tok, v_tok, v_head;    // element strides
    const int* q_start;
    const int* kv_start;
    int batch, H, P;
    int q_tokens, kv_tokens, max_q_len;
    int causal;
    int sorted;                                    // bf16: blocks take the items in order of what they cost
    float scale_log2;
    void* out;                                     // [q_tokens, H, value_dim]
    float* lse;                                    // [q_tokens, H]
    int* wait_timeouts;
};

// Request b: its first query and key, how many of each.
__device__ __forceinline__ void prompt_range(const PromptArgs& g, int b, int& q0, int& nq, int& k0, int& nk) {
    q0 = max(0, min(g.q_start[b], g.q_tokens));
    nq = min(max(0, min(g.q_start[b + 1], g.q_tokens) - q0), g.max_q_len);
    const int* ks = g.kv_start ? g.kv_start : g.q_start;
    k0 = max(0, min(ks[b], g.kv_tokens));
    nk = max(0, min(ks[b + 1], g.kv_tokens) - k0);
}

}  // namespace dsa
