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
    int entries;                                   // > 0: the blocks of one head, at most, which a list names (see prompt_before);
                                                   // else max_q_len's for every request
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

// A list of the blocks of all requests without gaps: at most one a request more than the tokens fill, however loose max_q_len is.
// By every thread of a block, of which the first kPrListed have a request each: numbers `mine` of the threads before it.
constexpr int kPrListed = 256;
__device__ __forceinline__ int prompt_before(int mine, int* s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += x;
    }
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    int before = sum - mine;
    for (int w = 0; w < min(warp, kPrListed / 32); ++w) before += s_warp[w];
    return before;
}

}  // namespace dsa
