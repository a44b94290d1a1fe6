// Attention of new tokens over a latent cache, float32 (dsa_latent_step), by CUDA cores: see dsa_stream_f32.cuh.
//
// A block has 16 of a request's query rows (token, head) and one piece of its keys, the cached tokens and the new ones as
// one sequence; pieces are merged by the combine kernel.  Rows of R + P floats are staged 16 at a time with 16-byte copies, the
// next tile under way while one is used; every row is key and value at once.
#pragma once
#include "dsa_latent_args.cuh"
#include "dsa_stream_f32.cuh"

namespace dsa {

constexpr int kLatentF32Rows = 4;                  // per warp
constexpr int kLatentF32Block = kLatentF32Rows * kStreamWarps;

template <int R>
struct LatentF32Cfg {
    static constexpr int SMEM = 2 * kStreamTile * (R + 64) * 4;
};

template <int R>
__global__ void __launch_bounds__(kStreamWarps * 32) dsa_latent_f32_kernel(const LatentArgs g) {
    extern __shared__ __align__(16) float s_rows[];
    constexpr int ROWS = kLatentF32Rows, VP = R / 128;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int piece = idx % g.a.n_split; idx /= g.a.n_split;
    const int rt = idx % g.row_tiles;
    const int b = idx / g.row_tiles;
    int S, n;
    latent_lengths(g, b, S, n);
    const int row0 = rt * kLatentF32Block + warp * ROWS;
    const int W = g.R + g.P, len = n > 0 ? S + n : 0;
    const int tiles = (len + kStreamTile - 1) / kStreamTile, per = (tiles + g.a.n_split - 1) / g.a.n_split;
    const int t0 = min(tiles, piece * per), t1 = min(tiles, t0 + per);

    StreamRows<ROWS, VP, VP> st;
    st.clear();
    int limit[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = row0 + r, token = row / g.a.H_q;
        limit[r] = row < g.rows && token < n ? S + token + 1 : 0;
        if (limit[r] == 0) continue;
        const float* q = reinterpret_cast<const float*>(g.a.q) + ((int64_t)b * g.rows + row) * W;
#pragma unroll
        for (int p = 0; p < VP; ++p) st.q[r][p] = load_piece(q + (lane + 32 * p) * 4);
        if (lane < g.P / 4) st.qr[r] = load_piece(q + R + lane * 4);
    }
    const int vecs = W / 4;
    auto stage = [&](int t) {
        float* dst = s_rows + (t & 1) * kStreamTile * (R + 64);
        // eight threads a row, every eighth piece each: one address per thread
        const int row = tid >> 3, pos = t * kStreamTile + row;
        const bool there = pos < len;
        const float* src = reinterpret_cast<const float*>(g.a.k);
        if (there)
            src = pos < S ? src + token_offset(g.a, b, 0, pos) : reinterpret_cast<const float*>(g.a.k_new) + ((int64_t)b * g.N + pos - S) * W;
        for (int c = tid & 7; c < vecs; c += 8) cp_async16(dst + row * (R + 64) + c * 4, src + c * 4, there);
        cp_async_commit();
    };
    if (t0 < t1) stage(t0);
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) stage(t + 1); else cp_async_commit();
        cp_async_wait<1>();
        __syncthreads();
        const float* rows = s_rows + (t & 1) * kStreamTile * (R + 64);
        if (row0 < g.rows)
#pragma unroll 1
            for (int j = 0; j < kStreamTile; j += 4) {
                const float* k = rows + j * (R + 64);
                st.keys4(k, k + R, k, R + 64, R + 64, R + 64, R / 4, g.P / 4, R / 4, t * kStreamTile + j, limit, g.a.scale_log2, lane);
            }
        __syncthreads();
    }
    cp_async_wait<0>();
    if (rt == 0) latent_append<float>(g, b, S, n, piece * kStreamWarps + warp, g.a.n_split * kStreamWarps, lane);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = row0 + r;
        if (row >= g.rows) continue;
        const int64_t orow = (int64_t)b * g.rows + row;
        const float inv = st.l[r] == 0.f ? 0.f : 1.f / st.l[r];
#pragma unroll
        for (int p = 0; p < VP; ++p) {
            float4 o = st.o[r][p];
            o = st.l[r] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            const int c = (lane + 32 * p) * 4;
            if (g.a.n_split > 1) store_piece(g.a.out_part + (orow * g.a.n_split + piece) * R + c, o);
            else store_piece(reinterpret_cast<float*>(g.a.out) + orow * R + c, o);
        }
        if (lane == 0) {
            if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + piece] = st.lse(r, g.a.scale_log2);
            else g.a.lse[orow] = st.lse(r, g.a.scale_log2);
        }
    }
}

}  // namespace dsa
