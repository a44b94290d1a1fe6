// Attention by CUDA cores for the float32 forms of the latent-cache calls: a warp owns ROWS query rows and streams keys.
//
// A lane holds the float4 pieces lane, lane + 32, ... of the rows' queries and of their O, so that a key's pieces are read
// once from shared memory by the warp, its scores with ROWS rows are ROWS partial sums per lane, and a halving exchange
// over the lanes finishes four keys' scores at a time.  The running maximum and sum are the same in all lanes; O is
// rescaled only when a maximum grows.  What bounds it: the multiply-adds of 128 lanes an SM and clock, and beside them the
// 40 exchange steps per four keys.
#pragma once
#include "dsa_common.cuh"

namespace dsa {

constexpr int kStreamWarps = 4;
constexpr int kStreamTile = 16;                    // keys per shared-memory tile, two of them in flight

__device__ __forceinline__ float4 load_piece(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void store_piece(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }

// KP / VP: pieces per lane of the keys' main part and of the values.
template <int ROWS, int KP, int VP>
struct StreamRows {
    float4 q[ROWS][KP], qr[ROWS];                  // (qr: the piece of the part that carries the position)
    float4 o[ROWS][VP];
    float m[ROWS], l[ROWS];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
            qr[r] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int p = 0; p < KP; ++p) q[r][p] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int p = 0; p < VP; ++p) o[r][p] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }

    // Four keys whose rows lie ld elements apart; row r sees the key at position pos + u if that is below limit[r].
    // main_vecs / rope_vecs / value_vecs: float4 pieces that the rows have.
    __device__ __forceinline__ void keys4(const float* k, const float* kr, const float* v, int ld_k, int ld_r, int ld_v, int main_vecs,
                                          int rope_vecs, int value_vecs, int pos, const int (&limit)[ROWS], float sl, int lane) {
        constexpr int V = ROWS * 4;
        float x[V];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float4 kk[KP], kq = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int p = 0; p < KP; ++p)
                kk[p] = lane + 32 * p < main_vecs ? load_piece(k + u * ld_k + (lane + 32 * p) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
            if (lane < rope_vecs) kq = load_piece(kr + u * ld_r + lane * 4);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float s = qr[r].x * kq.x;
                s = fmaf(qr[r].y, kq.y, s); s = fmaf(qr[r].z, kq.z, s); s = fmaf(qr[r].w, kq.w, s);
#pragma unroll
                for (int p = 0; p < KP; ++p) {
                    s = fmaf(q[r][p].x, kk[p].x, s); s = fmaf(q[r][p].y, kk[p].y, s);
                    s = fmaf(q[r][p].z, kk[p].z, s); s = fmaf(q[r][p].w, kk[p].w, s);
                }
                x[r * 4 + u] = s;
            }
        }
        group_sum_all<V, 32>(x, lane);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float mx = m[r];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (pos + u >= limit[r]) x[r * 4 + u] = -INFINITY;
                mx = fmaxf(mx, x[r * 4 + u]);
            }
            if (mx > m[r]) {                       // (the same in all lanes)
                const float alpha = exp2f((m[r] - mx) * sl);
                m[r] = mx;
                l[r] *= alpha;
#pragma unroll
                for (int p = 0; p < VP; ++p) { o[r][p].x *= alpha; o[r][p].y *= alpha; o[r][p].z *= alpha; o[r][p].w *= alpha; }
            }
            const float sub = m[r] == -INFINITY ? 0.f : m[r] * sl;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[r * 4 + u] = exp2f(fmaf(x[r * 4 + u], sl, -sub));
                l[r] += x[r * 4 + u];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int p = 0; p < VP; ++p) {
                if (lane + 32 * p >= value_vecs) continue;
                const float4 vv = load_piece(v + u * ld_v + (lane + 32 * p) * 4);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float w = x[r * 4 + u];
                    o[r][p].x = fmaf(w, vv.x, o[r][p].x); o[r][p].y = fmaf(w, vv.y, o[r][p].y);
                    o[r][p].z = fmaf(w, vv.z, o[r][p].z); o[r][p].w = fmaf(w, vv.w, o[r][p].w);
                }
            }
    }

    __device__ __forceinline__ float lse(int r, float sl) const { return l[r] == 0.f ? -INFINITY : (m[r] * sl + log2f(l[r])) * LN2; }
};

}  // namespace dsa
