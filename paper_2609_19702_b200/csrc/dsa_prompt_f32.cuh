// Attention of the tokens of prompts with expanded keys and values, float32 (dsa_latent_prompt), by CUDA cores: see
// dsa_stream_f32.cuh.  A block has 32 queries of one (request, head), eight a warp, and streams the keys that they see.
#pragma once
#include "dsa_prompt_args.cuh"
#include "dsa_stream_f32.cuh"

namespace dsa {

constexpr int kPromptF32Rows = 8;                  // per warp
constexpr int kPromptF32Block = kPromptF32Rows * kStreamWarps;

template <int D>
struct PromptF32Cfg {
    static constexpr int LD_K = D + 64, ROW = LD_K + D;                    // [k_nope | k_rope | v]
    static constexpr int SMEM = 2 * kStreamTile * ROW * 4;
};

template <int D>
__global__ void __launch_bounds__(kStreamWarps * 32) dsa_prompt_f32_kernel(const PromptArgs g) {
    using C = PromptF32Cfg<D>;
    extern __shared__ __align__(16) float s_rows[];
    constexpr int ROWS = kPromptF32Rows;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tiles_q = (g.max_q_len + kPromptF32Block - 1) / kPromptF32Block;
    int idx = blockIdx.x;
    const int h = idx % g.H; idx /= g.H;
    const int b = idx % g.batch;
    const int first = (tiles_q - 1 - idx / g.batch) * kPromptF32Block;     // (the longest rows first)
    int q0, nq, k0, nk;
    prompt_range(g, b, q0, nq, k0, nk);
    // (the starts of the whole request decide which keys a query sees, whatever max_q_len leaves out)
    const int all_q = max(0, min(g.q_start[b + 1], g.q_tokens) - q0);
    if (first >= nq) return;
    const int row0 = first + warp * ROWS;
    StreamRows<ROWS, 1, 1> st;
    st.clear();
    int limit[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        limit[r] = 0;
        if (row0 + r >= nq) continue;
        limit[r] = g.causal ? (int)max((int64_t)0, min((int64_t)nk, (int64_t)row0 + r + 1 + nk - all_q)) : nk;
        const float* q = reinterpret_cast<const float*>(g.q) + (int64_t)(q0 + row0 + r) * g.q_tok + h * g.q_head;
        if (lane < D / 4) st.q[r][0] = load_piece(q + lane * 4);
        if (lane < g.P / 4) st.qr[r] = load_piece(q + D + lane * 4);
    }
    const int last = min(first + kPromptF32Block, nq) - 1;
    const int len = g.causal ? (int)max((int64_t)0, min((int64_t)nk, (int64_t)last + 1 + nk - all_q)) : nk;
    const int tiles = (len + kStreamTile - 1) / kStreamTile;
    auto stage = [&](int t) {
        const int row = tid >> 3, pos = t * kStreamTile + row;
        float* dst = s_rows + (t & 1) * kStreamTile * C::ROW + row * C::ROW;
        const bool there = pos < len;
        const int64_t tok = there ? k0 + pos : 0;
        const float* k = reinterpret_cast<const float*>(g.k) + tok * g.k_tok + h * g.k_head;
        const float* kr = reinterpret_cast<const float*>(g.kr) + tok * g.r_tok;
        const float* v = reinterpret_cast<const float*>(g.v) + tok * g.v_tok + h * g.v_head;
        for (int c = tid & 7; c < D / 4; c += 8) {
            cp_async16(dst + c * 4, k + c * 4, there);
            cp_async16(dst + C::LD_K + c * 4, v + c * 4, there);
        }
        for (int c = tid & 7; c < g.P / 4; c += 8) cp_async16(dst + D + c * 4, kr + c * 4, there);
        cp_async_commit();
    };
    if (tiles > 0) stage(0);
    for (int t = 0; t < tiles; ++t) {
        if (t + 1 < tiles) stage(t + 1); else cp_async_commit();
        cp_async_wait<1>();
        __syncthreads();
        const float* rows = s_rows + (t & 1) * kStreamTile * C::ROW;
        if (row0 < nq)
#pragma unroll 1
            for (int j = 0; j < kStreamTile; j += 4) {
                const float* k = rows + j * C::ROW;
                st.keys4(k, k + D, k + C::LD_K, C::ROW, C::ROW, C::ROW, D / 4, g.P / 4, D / 4, t * kStreamTile + j, limit, g.scale_log2, lane);
            }
        __syncthreads();
    }
    cp_async_wait<0>();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (row0 + r >= nq) continue;
        const int64_t orow = (int64_t)(q0 + row0 + r) * g.H + h;
        const float inv = st.l[r] == 0.f ? 0.f : 1.f / st.l[r];
        const float4 o = st.o[r][0];
        if (lane < D / 4)
            store_piece(reinterpret_cast<float*>(g.out) + orow * D + lane * 4,
                        st.l[r] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
        if (lane == 0) g.lse[orow] = st.lse(r, g.scale_log2);
    }
}

}  // namespace dsa
