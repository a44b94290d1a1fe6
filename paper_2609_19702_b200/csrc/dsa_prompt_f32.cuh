// Attention of the tokens of prompts with expanded keys and values, float32 (dsa_latent_prompt), by CUDA cores: see
// dsa_tile_f32.cuh.  A block has 32 queries of one (request, head) and takes the keys that they see tile by tile.
// Bound by the multiply-adds (see there): 4 prompts of up to 300 tokens, 8 heads of 64 + 32 numbers: 29 us, whose bytes
// would take 2.
#pragma once
#include "dsa_prompt_args.cuh"
#include "dsa_tile_f32.cuh"

namespace dsa {

template <int D>
struct PromptF32Cfg {
    static constexpr int LD = D + 64 + 4, LD_V = D + 4;                    // rows in shared memory, in floats
    static constexpr int SMEM = (2 * kTileRows * LD + kTileKeys * LD_V + TileF32<D>::SCRATCH) * 4;
};

template <int D>
__global__ void __launch_bounds__(kTileThreads, 2) dsa_prompt_f32_kernel(const PromptArgs g) {
    using C = PromptF32Cfg<D>;
    extern __shared__ __align__(16) float sm[];
    float* s_q = sm;
    float* s_k = s_q + kTileRows * C::LD;
    float* s_v = s_k + kTileKeys * C::LD;
    float* scratch = s_v + kTileKeys * C::LD_V;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x;
    const int tiles_q = (g.max_q_len + kTileRows - 1) / kTileRows;
    int idx = blockIdx.x;
    const int h = idx % g.H; idx /= g.H;
    int b = idx % g.batch, first = (tiles_q - 1 - idx / g.batch) * kTileRows;      // (the longest rows first)
    int q0, nq, k0, nk;
    if (g.blocks == kPrByNumber) {
        const int2 at = prompt_find(g.q_start, g.q_tokens, g.batch, kTileRows, idx);
        b = at.x;
        if (b < 0) return;
        prompt_range(g, b, q0, nq, k0, nk);
        first = ((nq + kTileRows - 1) / kTileRows - 1 - at.y) * kTileRows;
        if (first < 0) return;
    }
    prompt_range(g, b, q0, nq, k0, nk);
    // (the starts of the whole request decide which keys a query sees, whatever max_q_len leaves out)
    const int all_q = max(0, min(g.q_start[b + 1], g.q_tokens) - q0);
    if (first >= nq) return;
    auto limit = [&](int i) { return g.causal ? (int)max((int64_t)0, min((int64_t)nk, (int64_t)i + 1 + nk - all_q)) : nk; };
    const int row = tid >> 3;                                 // of a tile: eight threads a row, every eighth piece each
    {
        const bool there = first + row < nq;
        const float* src = reinterpret_cast<const float*>(g.q) + (int64_t)(q0 + (there ? first + row : 0)) * g.q_tok + h * g.q_head;
        for (int c = tid & 7; c < (D + g.P) / 4; c += 8) cp_async16(s_q + row * C::LD + c * 4, src + c * 4, there);
    }
    const int mine = first + row < nq ? limit(first + row) : 0, len = limit(min(first + kTileRows, nq) - 1);
    // K of a tile is on its way while the weights and the product of the tile before are worked out, V while the scores are
    auto copy_k = [&](int t) {
        const bool there = t * kTileKeys + row < len;
        const int64_t tok = there ? k0 + t * kTileKeys + row : 0;
        const float* k = reinterpret_cast<const float*>(g.k) + tok * g.k_tok + h * g.k_head;
        const float* kr = reinterpret_cast<const float*>(g.kr) + tok * g.r_tok;
        for (int c = tid & 7; c < D / 4; c += 8) cp_async16(s_k + row * C::LD + c * 4, k + c * 4, there);
        for (int c = tid & 7; c < g.P / 4; c += 8) cp_async16(s_k + row * C::LD + D + c * 4, kr + c * 4, there);
    };
    auto copy_v = [&](int t) {
        const bool there = t * kTileKeys + row < len;
        const float* v = reinterpret_cast<const float*>(g.v) + (there ? k0 + t * kTileKeys + row : (int64_t)0) * g.v_tok + h * g.v_head;
        for (int c = tid & 7; c < D / 4; c += 8) cp_async16(s_v + row * C::LD_V + c * 4, v + c * 4, there);
    };
    TileF32<D> st;
    st.clear();
    const int tiles = (len + kTileKeys - 1) / kTileKeys;
    if (tiles > 0) copy_k(0);
    cp_async_commit();
    if (tiles > 0) copy_v(0);
    cp_async_commit();
    for (int t = 0; t < tiles; ++t) {
        cp_async_wait<1>();
        __syncthreads();
        st.tile(s_q, s_k, s_v, C::LD, C::LD_V, D + g.P, g.scale_log2, scratch, [&](int) { return mine - t * kTileKeys; },
                [&] { if (t + 1 < tiles) copy_k(t + 1); cp_async_commit(); }, [] { cp_async_wait<1>(); });
        if (t + 1 < tiles) copy_v(t + 1);
        cp_async_commit();
    }
    cp_async_wait<0>();
    st.results(g.scale_log2, scratch,
               [&](int r) -> float* { return first + r < nq ? reinterpret_cast<float*>(g.out) + ((int64_t)(q0 + first + r) * g.H + h) * D : nullptr; },
               [&](int r, float lse) { if (first + r < nq) g.lse[(int64_t)(q0 + first + r) * g.H + h] = lse; });
}

}  // namespace dsa
