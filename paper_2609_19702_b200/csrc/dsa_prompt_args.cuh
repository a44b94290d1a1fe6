// Arguments that the kernels of the prompt attention share (dsa_latent_prompt).
#pragma once
#include "dsa_common.cuh"

namespace dsa {

// Every request has as many blocks as max_q_len takes; they are found by their numbers (see prompt_find); a list names them (see prompt_before)
constexpr int kPrByBound = 0, kPrByNumber = 1, kPrByList = 2;

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
    int blocks;                                    // how a block finds its work, one of
    int entries;                                   // kPrByList: blocks of one head, at most
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

// Blocks of `rows` queries, numbered so that a block finds its request without a table, and that there are as many as all
// tokens fill and one a request, however loose max_q_len is: request b's begin at q_start[b] / rows + b, and since n queries from
// row q on reach no further than block (q + n) / rows, the next request's begin behind the last of them.
// The block's request (-1: none) and which of its blocks it is (it may not have so many), by a whole warp: 32 requests are looked
// at at a time, so that a million of them take four dependent reads.
__device__ __forceinline__ int2 prompt_find(const int* q_start, int q_tokens, int batch, int rows, int e) {
    const int lane = threadIdx.x & 31;
    auto begins = [&](int b) { return max(0, min(q_start[b], q_tokens)) / rows + b; };
    int lo = 0, hi = batch;                        // (where starts ascend) begins(lo) <= e but for lo = 0, begins(hi) > e or hi = batch
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
        const int k = __popc(__ballot_sync(0xffffffffu, at < hi && begins(at) <= e));
        lo += k * step;
        hi = min(hi, lo + step);
    }
    const int number = e - begins(lo);
    return make_int2(number < 0 ? -1 : lo, number);
}

// A list of the blocks of all requests without gaps: at most one a request more than the tokens fill.
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
