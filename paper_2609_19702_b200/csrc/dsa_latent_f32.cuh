// Attention of new tokens over a latent cache, float32 (dsa_latent_step), by CUDA cores: see dsa_tile_f32.cuh.
//
// A block has 32 of a request's query rows (token, head) and one piece of its keys, the cached tokens and the new ones as one
// sequence; pieces are merged by the kernel behind it.  Every staged row of R + P floats is key and value at once.
//
// Meant for checking a model in single precision, where the tensor cores have no exact form: bound by the multiply-adds of
// dsa_tile_f32.cuh and, for few rows, by the launch, the dependent reads and the merge.  4 requests x 20 heads x 3 tokens, R 256, lengths up to
// 1144: 19 us, of which the bytes would take 2.
#pragma once
#include "dsa_latent_args.cuh"
#include "dsa_tile_f32.cuh"

namespace dsa {

template <int R>
struct LatentF32Cfg {
    static constexpr int LD = R + 64 + 4;                                  // row in shared memory, in floats
    static constexpr int SMEM = (2 * kTileRows * LD + TileF32<R>::SCRATCH) * 4;
};

template <int R>
__global__ void __launch_bounds__(kTileThreads, R == 256 ? 2 : 1) dsa_latent_f32_kernel(const LatentArgs g) {
    using C = LatentF32Cfg<R>;
    extern __shared__ __align__(16) float sm[];
    float* s_q = sm;
    float* s_k = s_q + kTileRows * C::LD;
    float* scratch = s_k + kTileKeys * C::LD;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int piece = idx % g.a.n_split; idx /= g.a.n_split;
    const int rt = idx % g.row_tiles;
    const int b = idx / g.row_tiles;
    int S, n;
    latent_lengths(g, b, S, n);
    const int row0 = rt * kTileRows, W = g.R + g.P, vecs = W / 4, len = n > 0 ? S + n : 0;
    const int tiles = (len + kTileKeys - 1) / kTileKeys, per = (tiles + g.a.n_split - 1) / g.a.n_split;
    const int t0 = min(tiles, piece * per), t1 = row0 < n * g.a.H_q ? min(tiles, t0 + per) : t0;
    // row `tid / 8` of a tile: eight threads a row, every eighth piece each
    const int row = tid >> 3;
    if (t0 < t1) {
        const bool there = row0 + row < g.rows;
        const float* src = reinterpret_cast<const float*>(g.a.q) + ((int64_t)b * g.rows + (there ? row0 + row : 0)) * W;
        for (int c = tid & 7; c < vecs; c += 8) cp_async16(s_q + row * C::LD + c * 4, src + c * 4, there);
    }
    const int my_token = (row0 + row) / g.a.H_q;
    const int limit = row0 + row < g.rows && my_token < n ? S + my_token + 1 : 0;      // keys that the row sees
    TileF32<R> st;
    st.clear();
    for (int t = t0; t < t1; ++t) {
        const int pos = t * kTileKeys + row;
        const bool there = pos < len;
        const float* src = reinterpret_cast<const float*>(g.a.k);
        if (there)
            src = pos < S ? src + token_offset(g.a, b, 0, pos) : reinterpret_cast<const float*>(g.a.k_new) + ((int64_t)b * g.N + pos - S) * W;
        for (int c = tid & 7; c < vecs; c += 8) cp_async16(s_k + row * C::LD + c * 4, src + c * 4, there);
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
        st.tile(s_q, s_k, s_k, C::LD, C::LD, W, g.a.scale_log2, scratch, [&](int) { return limit - t * kTileKeys; }, [] {}, [] {});
    }
    if (rt == 0) latent_append<float>(g, b, S, n, piece * (kTileThreads / 32) + warp, g.a.n_split * (kTileThreads / 32), lane);
    const bool parts = g.a.n_split > 1;
    st.results(g.a.scale_log2, scratch,
               [&](int r) -> float* {
                   const int64_t orow = (int64_t)b * g.rows + row0 + r;
                   if (row0 + r >= g.rows) return nullptr;
                   return parts ? g.a.out_part + (orow * g.a.n_split + piece) * R : reinterpret_cast<float*>(g.a.out) + orow * R;
               },
               [&](int r, float lse) {
                   const int64_t orow = (int64_t)b * g.rows + row0 + r;
                   if (row0 + r >= g.rows) return;
                   if (parts) g.a.lse_part[orow * g.a.n_split + piece] = lse;
                   else g.a.lse[orow] = lse;
               });
}

// The pieces of a row joined: a warp has 128 of its dims, the weights exp(lse_i - max) over their sum from 32 lanes at a time.
// Bound by reading the pieces (rows x n_split x R floats, from L2), eight of them in flight.
constexpr int kLatF32MergeWarps = 4;

template <int R>
__global__ void __launch_bounds__(kLatF32MergeWarps * 32) dsa_latent_f32_merge_kernel(const LatentArgs g, int64_t rows) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x & 31, n = g.a.n_split;
    const int64_t at = (int64_t)blockIdx.x * kLatF32MergeWarps + (threadIdx.x >> 5), row = at / (R / 128);
    const int col = (int)(at % (R / 128)) * 128 + lane * 4;
    if (row >= rows) return;
    const float* lp = g.a.lse_part + row * n;
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, lp[i]);
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    float sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += 32) {
        const float v = i0 + lane < n ? lp[i0 + lane] : -INFINITY;
        const float w = v == -INFINITY ? 0.f : expf(v - top);         // (a piece without a number makes the row one)
        sum += w;
        const int m = min(32, n - i0);
        const float* op = g.a.out_part + (row * n + i0) * R + col;
#pragma unroll 8
        for (int j = 0; j < m; ++j) {
            const float wj = __shfl_sync(0xffffffffu, w, j);
            const float4 y = *reinterpret_cast<const float4*>(op + (int64_t)j * R);
            acc.x = fmaf(wj, y.x, acc.x); acc.y = fmaf(wj, y.y, acc.y); acc.z = fmaf(wj, y.z, acc.z); acc.w = fmaf(wj, y.w, acc.w);
        }
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(g.a.out) + row * R + col) =
        none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (col == 0) g.a.lse[row] = none ? -INFINITY : top + logf(sum);
}

}  // namespace dsa
