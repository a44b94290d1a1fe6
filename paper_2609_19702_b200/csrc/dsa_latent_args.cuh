// Arguments that the kernels of the latent-cache attention share (dsa_latent_step).
#pragma once
#include "dsa_common.cuh"

namespace dsa {

struct LatentArgs {
    AttnArgs a;                                    // lengths, block table, strides, scale, outputs; H_q heads, a.k the cache, a.k_new
    const int* new_count;                          // [B] or NULL (N)
    int N, R, P;
    int rows;                                      // N * H_q: query rows of a request
    int row_tiles;                                 // blocks of query rows per request
};

// Lengths of request b: cached tokens, and new ones that exist and have room.  L2: read past an SM's L1, by who reads them before it
// waits for the kernel in front, so that nothing else keeps older ones from being found there.
template <bool L2 = false>
__device__ __forceinline__ void latent_lengths(const LatentArgs& g, int b, int& S, int& n) {
    const int raw = L2 ? __ldcg(g.a.seq_len + b) : g.a.seq_len[b];
    S = max(0, min(raw, g.a.max_seq_len));
    n = g.new_count ? max(0, min(L2 ? __ldcg(g.new_count + b) : g.new_count[b], g.N)) : g.N;
    n = raw < 0 ? 0 : min(n, g.a.max_seq_len - S);
}

// The rows of request b's new tokens go to the cache: tokens first, first + step, ... below n, by one warp.
template <typename T>
__device__ __forceinline__ void latent_append(const LatentArgs& g, int b, int S, int n, int first, int step, int lane) {
    const int vecs = (g.R + g.P) * (int)sizeof(T) / 16;
    for (int i = first; i < n; i += step) {
        if (!token_has_page(g.a, b, S + i)) continue;
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(g.a.k_new) + ((int64_t)b * g.N + i) * (g.R + g.P));
        uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<T*>(const_cast<void*>(g.a.k)) + token_offset(g.a, b, 0, S + i));
        for (int c = lane; c < vecs; c += 32) dst[c] = src[c];
    }
}

}  // namespace dsa
