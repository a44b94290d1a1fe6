// Attention by CUDA cores for the float32 forms of the latent-cache calls: 32 query rows of a block over tiles of 32 keys.
//
// Per tile: scores, a running maximum and sum per row, O rescaled and added to.  The scores' dims are dealt out to four groups
// of 64 threads, each thread with 4 x 4 scores, so that 8 reads of 16 bytes from shared memory feed 64 multiply-adds; the
// groups' sums meet in shared memory, where eight threads a row take the softmax.  For O every thread has some rows x some
// dims, two at a time.  What bounds it: the multiply-adds of 128 lanes an SM and clock, at 48 % of their rate where there are
// many blocks (one prompt of 1280 tokens, 32 heads of 128 + 64: 490 us); where there are few, reads, sums and three barriers
// one behind the other, 2.2 us a tile of 64-wide heads and 3.5 of 128-wide ones.
// Rows lie W + 4 floats apart, an odd number of 16-byte pieces, so that eight of them are read without a conflict.
#pragma once
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kTileRows = 32, kTileKeys = 32, kTileThreads = 256;

// VD: width of a value
template <int VD>
struct TileF32 {
    static constexpr int DG = VD / 4 < 64 ? VD / 4 : 64;                   // threads side by side along the dims
    static constexpr int F4 = VD / 4 / DG;                                 // pieces of four dims per thread
    static constexpr int RPT = kTileRows / (kTileThreads / DG);            // rows per thread
    static constexpr int LS = 36;                                          // row of the scores and weights, in floats
    static constexpr int SCRATCH = 4 * kTileRows * LS + kTileKeys * LS + 2 * kTileRows;   // floats of shared memory beside q and the keys

    ulonglong2 o[RPT][F4];                                                 // pairs of floats
    float m, l;                                                            // of row tid / 8 (the same in its eight threads)

    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int r = 0; r < RPT; ++r)
#pragma unroll
            for (int f = 0; f < F4; ++f) o[r][f] = make_ulonglong2(0ull, 0ull);
    }

    // One tile, by the whole block: q and k [32][ld] with `width` floats a row, v [32][ld_v]; row r sees the keys below seen(r).
    // Nobody writes q, k or v before it returns, but for k, which may be written from scores_done() on (where k is not v as well);
    // values() waits for this thread's copies of v.
    template <class Seen, class ScoresDone, class Values>
    __device__ __forceinline__ void tile(const float* q, const float* k, const float* v, int ld, int ld_v, int width, float sl, float* scratch, Seen seen, ScoresDone scores_done,
                                         Values values) {
        float* s_s = scratch;
        float* s_p = scratch + 4 * kTileRows * LS;
        float* s_alpha = s_p + kTileKeys * LS;
        const int tid = threadIdx.x;
        {
            const int g = tid >> 6, kg = tid & 7, rg = (tid >> 3) & 7;
            unsigned long long x[4][4] = {};               // (sums over even and odd dims)
            for (int c = g * 4; c < width; c += 16) {
                ulonglong2 a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = *reinterpret_cast<const ulonglong2*>(q + (rg + 8 * i) * ld + c);
                    b[i] = *reinterpret_cast<const ulonglong2*>(k + (kg + 8 * i) * ld + c);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][j] = fma_f32x2(a[i].x, b[j].x, fma_f32x2(a[i].y, b[j].y, x[i][j]));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 two = unpack_f32x2(x[i][j]);
                    s_s[(g * kTileRows + rg + 8 * i) * LS + kg + 8 * j] = two.x + two.y;
                }
        }
        __syncthreads();
        scores_done();
        {
            const int row = tid >> 3, key = (tid & 7) * 4, limit = seen(row);
            float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 y = *reinterpret_cast<const float4*>(s_s + (g * kTileRows + row) * LS + key);
                x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
            }
            float mx = m;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (key + i >= limit) x[i] = -INFINITY;
                mx = fmaxf(mx, x[i]);
            }
#pragma unroll
            for (int off = 4; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float alpha = mx == -INFINITY ? 1.f : exp2f((m - mx) * sl), sub = mx == -INFINITY ? 0.f : mx * sl;
            m = mx;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = exp2f(fmaf(x[i], sl, -sub));
                s_p[(key + i) * LS + row] = p;
                sum += p;
            }
#pragma unroll
            for (int off = 4; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            l = fmaf(l, alpha, sum);
            if ((tid & 7) == 0) s_alpha[row] = alpha;
        }
        values();
        __syncthreads();
        {
            const int dg = tid % DG, r0 = tid / DG * RPT;
#pragma unroll
            for (int r = 0; r < RPT; ++r) {
                const float alpha = s_alpha[r0 + r];
                const unsigned long long two = pack_f32x2(alpha, alpha);
#pragma unroll
                for (int f = 0; f < F4; ++f) { o[r][f].x = fma_f32x2(o[r][f].x, two, 0ull); o[r][f].y = fma_f32x2(o[r][f].y, two, 0ull); }
            }
#pragma unroll 4
            for (int j = 0; j < kTileKeys; ++j) {
                unsigned long long p[RPT];                     // (a weight twice)
                if constexpr (RPT >= 4) {
#pragma unroll
                    for (int r = 0; r < RPT; r += 4) {
                        const float4 y = *reinterpret_cast<const float4*>(s_p + j * LS + r0 + r);
                        p[r] = pack_f32x2(y.x, y.x); p[r + 1] = pack_f32x2(y.y, y.y); p[r + 2] = pack_f32x2(y.z, y.z); p[r + 3] = pack_f32x2(y.w, y.w);
                    }
                } else {
                    const float2 y = *reinterpret_cast<const float2*>(s_p + j * LS + r0);
                    p[0] = pack_f32x2(y.x, y.x); p[1] = pack_f32x2(y.y, y.y);
                }
#pragma unroll
                for (int f = 0; f < F4; ++f) {
                    const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(v + j * ld_v + (dg + f * DG) * 4);
#pragma unroll
                    for (int r = 0; r < RPT; ++r) { o[r][f].x = fma_f32x2(p[r], y.x, o[r][f].x); o[r][f].y = fma_f32x2(p[r], y.y, o[r][f].y); }
                }
            }
        }
        __syncthreads();
    }

    // out(row) gets the row's O over its sum (nullptr: no such row), lse(row, value) the log-sum.
    template <class Out, class Lse>
    __device__ __forceinline__ void results(float sl, float* scratch, Out out, Lse lse) {
        const int tid = threadIdx.x, row = tid >> 3;
        if ((tid & 7) == 0) {
            scratch[row] = l == 0.f ? 0.f : 1.f / l;
            lse(row, l == 0.f ? -INFINITY : (m * sl + log2f(l)) * LN2);
        }
        __syncthreads();
        const int dg = tid % DG, r0 = tid / DG * RPT;
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            float* dst = out(r0 + r);
            const float inv = scratch[r0 + r];
            if (dst)
#pragma unroll
                for (int f = 0; f < F4; ++f) {
                    const float2 a = unpack_f32x2(o[r][f].x), b = unpack_f32x2(o[r][f].y);
                    *reinterpret_cast<float4*>(dst + (dg + f * DG) * 4) =
                        inv == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(a.x * inv, a.y * inv, b.x * inv, b.y * inv);
                }
        }
    }
};

}  // namespace dsa
