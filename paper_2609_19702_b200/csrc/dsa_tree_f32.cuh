// Attention of a tree of drafted tokens over a cache, fp32 (dsa_tree_step; formulas in dsa_tree.cuh).
//
// fp32 inputs are multiplied in fp32 on the CUDA cores: the tensor cores would round them to tf32.  Per token
// and kv head 8 D bytes meet 2 D fused multiply-adds a query row: up to some 16 rows the copies are the bound,
// beyond them the multiply-adds and the shared-memory reads that feed them.  So there are two forms.  Measured: 8
// requests of 8 nodes, 20 heads of 64, up to 1144 tokens: 40 us, 7 of them the combine (49 MB; the few-row form is bound
// by issue slots -- some 370 instructions a warp and tile, 128 of them multiply-adds, and as much again for a block's
// set-up and results -- and by unequal lengths; the 32-row form took 122); 138 requests of 68 rows, 1000 tokens, D 128:
// 343 us for 4.8 GFLOP, bound by the reads of shared memory (352 with single multiply-adds).
//
// Few rows (up to 16): tiles of 32 tokens in a ring of three slots.  Eight threads share a token's scores, each
// an eighth of the dims for all rows (one read of K per multiply-add's row count, q from registers of the same
// address in all lanes), and exchange halves until each holds one or two rows' totals; O is cut into four dims
// per thread and 256 / (D / 4) groups of tokens, whose parts are added once at the end.
//
// More rows: 32 query rows a block and tiles of 64 tokens.  A warp's scores are 16 rows x 16 tokens, its lanes
// 4 x 8 of 4 rows x 2 tokens each, so that one read of q serves eight lanes and one of K four (on average 2.7
// cycles of shared memory a read, and 6 reads for 32 multiply-adds: these reads are what bounds it; lanes 2 x 16
// need more); scores are summed over even and odd dims, two multiply-adds in one; O as 16 rows x D / 4 dims.
// Groups of tokens and rows that do not exist are skipped.
//
// Rows in shared memory are padded by 16 bytes so that the eight rows a quarter-warp reads lie in different
// banks.  K rows are multiplied as they are (masked scores are replaced), rows of V that no node sees are
// staged as zeros: their weight is 0, but 0 x NaN is not.
#pragma once
#include "dsa_tree.cuh"

namespace dsa {

// Parents of the nodes lane and lane + 32 (-1: a root).
struct TreeParents { int up[2]; };
__device__ __forceinline__ TreeParents tree_parents(const TreeArgs& g, int b, int lane) {
    TreeParents t;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        const int p = i < g.N ? (g.parent ? g.parent[(int64_t)b * g.N + i] : i - 1) : -1;
        t.up[h] = (p >= 0 && p < i) ? p : -1;
    }
    return t;
}
// Ancestor sets of the nodes as 64-bit words (bit j: node j is node i or an ancestor of it), by one warp: every
// round doubles the length of the line that a word covers.
__device__ __forceinline__ void tree_lines(TreeParents t, unsigned long long* line_of, int lane) {
    unsigned long long m[2] = {1ull << lane, 1ull << (lane + 32)};
    int (&up)[2] = t.up;
#pragma unroll
    for (int round = 0; round < 6; ++round) {
        unsigned long long am[2];
        int au[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int src = up[h] & 31;
            const unsigned long long m0 = __shfl_sync(0xffffffffu, m[0], src), m1 = __shfl_sync(0xffffffffu, m[1], src);
            const int u0 = __shfl_sync(0xffffffffu, up[0], src), u1 = __shfl_sync(0xffffffffu, up[1], src);
            am[h] = up[h] < 0 ? 0ull : (up[h] < 32 ? m0 : m1);
            au[h] = up[h] < 0 ? -1 : (up[h] < 32 ? u0 : u1);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) { m[h] |= am[h]; up[h] = au[h]; }
    }
    line_of[lane] = m[0];
    line_of[lane + 32] = m[1];
}

constexpr int kTreeF32Rows = 32;
constexpr int kTreeF32Threads = 256;                       // few rows

template <int D>
struct TreeF32Cfg {
    static constexpr int LD = D + 4;                       // padded row of Q, K, V, in floats
    static constexpr int LP = kTreeTile + 4;               // padded row of the weights
    static constexpr int SMEM = (kTreeF32Rows * LD + 2 * kTreeTile * LD + kTreeF32Rows * LP + 4 * kTreeF32Rows) * 4;
};

template <int D>
__global__ void __launch_bounds__(kTreeF32Threads, 2) dsa_tree_f32_kernel(const TreeArgs g) {
    using C = TreeF32Cfg<D>;
    constexpr int DV = D / 4;                              // 16-byte pieces of a row
    constexpr int OD = D / 32;                             // dims of O per thread: 4, or 2
    extern __shared__ __align__(16) float sm[];
    float* s_q = sm;
    float* s_k = s_q + kTreeF32Rows * C::LD;
    float* s_v = s_k + kTreeTile * C::LD;
    float* s_p = s_v + kTreeTile * C::LD;
    float* s_max = s_p + kTreeF32Rows * C::LP;             // [token group][row]
    __shared__ unsigned long long line_of[kTreeMaxNodes];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int split = idx % g.a.n_split; idx /= g.a.n_split;
    const int rt = idx % g.row_tiles; idx /= g.row_tiles;
    const int kvh = idx % g.a.H_kv;
    const int b = idx / g.a.H_kv;
    const int G = g.G, per_tile = kTreeF32Rows / G, first_node = rt * per_tile;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    int S, L_p, n;
    tree_lengths(g, b, S, L_p, n);
    const int rows_all = min(per_tile, g.N - first_node) * G;
    const int rows = max(0, min(per_tile, n - first_node)) * G;
    const TreeSpan span = tree_span(g, S, L_p);
    const int per_split = (span.T + g.a.n_split - 1) / g.a.n_split;
    const int t0 = min(span.T, split * per_split), t1 = min(span.T, t0 + per_split);
    const int cached = t1 - t0, tiles = rows == 0 ? 0 : cached + (split == 0 ? 1 : 0);
    if (tiles == 0) {
        if (rows > 0) tree_append<float, D>(g, b, kvh, S, L_p, first_node + split + warp * g.a.n_split, 8 * g.a.n_split, min(n, first_node + per_tile), lane);
        tree_write_empty<float, D>(g, b, kvh, split, first_node, 0, rows_all, tid, kTreeF32Threads);
        return;
    }
    auto bounds = [&](int t, int& start, int& from, int& to) {
        start = 0; from = 0; to = n;
        if (t < cached) span.tile(t0 + t, start, from, to);
    };
    // K (and then V) rows of tile t; rows that nobody sees: zeros
    auto stage = [&](int t, bool is_v) {
        int start, from, to;
        bounds(t, start, from, to);
        const float* src = reinterpret_cast<const float*>(t < cached ? (is_v ? g.a.v : g.a.k) : (is_v ? g.a.v_new : g.a.k_new));
        // four threads a row, every fourth piece each: one address per thread
        const int row = tid >> 2, pos = start + row;
        const bool seen = pos >= from && pos < to;
        if (seen)
            src += t < cached ? token_offset(g.a, b, L_p, pos) + (int64_t)kvh * g.a.stride_head
                              : (((int64_t)b * g.N + pos) * g.a.H_kv + kvh) * D;
        float* dst = (is_v ? s_v : s_k) + row * C::LD;
#pragma unroll
        for (int j = 0; j < DV / 4; ++j) {
            const int c = ((tid & 3) + 4 * j) * 4;
            cp_async16(dst + c, src + c, seen);
        }
        cp_async_commit();
    };
    stage(0, false);
    stage(0, true);
    if (warp == 0) tree_lines(tree_parents(g, b, lane), line_of, lane);
    for (int i = tid; i < kTreeF32Rows * DV; i += kTreeF32Threads) {
        const int row = i / DV, c = (i - row * DV) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < rows)
            x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(g.a.q) +
                                                 (((int64_t)b * g.N + first_node + row / G) * g.a.H_q + kvh * G + row % G) * D + c);
        *reinterpret_cast<float4*>(s_q + row * C::LD + c) = x;
    }
    __syncthreads();

    const int kg = lane & 7, rg = lane >> 3;               // lane: tokens kg, kg + 8 of the warp's group; rows rg + 4 r of its half
    const int row0 = (warp & 1) * 16 + rg, group = warp >> 1;
    const int key0 = group * 16 + kg, dim0 = group * (D / 4) + kg * OD;
    const bool rows_here = (warp & 1) * 16 < rows;
    const float sl = g.a.scale_log2;
    float m[4], l[4], o[4][OD];
    unsigned long long own[4];
    int64_t win_lo[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < OD; ++c) o[r][c] = 0.f;
        const int row = row0 + 4 * r;
        own[r] = 0ull;
        win_lo[r] = 0;
        if (row >= rows) continue;
        const unsigned long long line = line_of[first_node + row / G];
        const int depth = __popcll(line) - 1;
        win_lo[r] = (int64_t)S + depth + 1 - g.a.mask.window;
        own[r] = line;                                     // (ancestors of a node that exists exist)
        if (g.windowed) {
            unsigned long long todo = line;
            while (todo) {
                const int j = __ffsll(todo) - 1;
                todo &= todo - 1;
                const int dj = __popcll(line_of[j]) - 1;
                if (depth - dj >= g.a.mask.window && (int64_t)S + dj >= (int64_t)L_p + g.a.mask.n_sink) own[r] &= ~(1ull << j);
            }
        }
    }

    for (int t = 0; t < tiles; ++t) {
        int start, from, to;
        bounds(t, start, from, to);
        const int count = to - start;                      // tokens of the tile that may be seen: [0, count)
        cp_async_wait<1>();                                // K is there (V may be on its way)
        __syncthreads();
        unsigned long long x2[4][2] = {};                  // (sums over even and odd dims)
        if (rows_here && group * 16 < count) {
#pragma unroll 4
            for (int c = 0; c < D; c += 4) {
                ulonglong2 q[4], k[2];
#pragma unroll
                for (int r = 0; r < 4; ++r) q[r] = *reinterpret_cast<const ulonglong2*>(s_q + (row0 + 4 * r) * C::LD + c);
#pragma unroll
                for (int j = 0; j < 2; ++j) k[j] = *reinterpret_cast<const ulonglong2*>(s_k + (key0 + 8 * j) * C::LD + c);
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < 2; ++j) x2[r][j] = fma_f32x2(q[r].x, k[j].x, fma_f32x2(q[r].y, k[j].y, x2[r][j]));
            }
        }
        float x[4][2];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 two = unpack_f32x2(x2[r][j]);
                x[r][j] = two.x + two.y;
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int key = key0 + 8 * j, pos = start + key;
                bool seen = row0 + 4 * r < rows && pos >= from && pos < to;
                if (t < cached) seen = seen && (t0 + t < span.T1 || pos >= win_lo[r]);
                else seen = seen && ((own[r] >> key) & 1ull) != 0;
                if (!seen) x[r][j] = -INFINITY;
                mx = fmaxf(mx, x[r][j]);
            }
#pragma unroll
            for (int off = 4; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            if (kg == 0) s_max[group * kTreeF32Rows + row0 + 4 * r] = mx;
        }
        __syncthreads();                                   // (K has been read for the last time)
        if (t + 1 < tiles) stage(t + 1, false); else cp_async_commit();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row0 + 4 * r;
            float m_new = m[r];
#pragma unroll
            for (int w = 0; w < 4; ++w) m_new = fmaxf(m_new, s_max[w * kTreeF32Rows + row]);
            const float sub = m_new == -INFINITY ? 0.f : m_new * sl;
            const float alpha = m_new == -INFINITY ? 1.f : exp2f((m[r] - m_new) * sl);
            m[r] = m_new;
            l[r] *= alpha;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float p = exp2f(fmaf(x[r][j], sl, -sub));
                l[r] += p;
                s_p[row * C::LP + key0 + 8 * j] = p;
            }
#pragma unroll
            for (int c = 0; c < OD; ++c) o[r][c] *= alpha;
        }
        cp_async_wait<1>();                                // V is there
        __syncthreads();
        if (rows_here)
#pragma unroll 2
            for (int j = 0; j < count; j += 4) {
                float4 p[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = *reinterpret_cast<const float4*>(s_p + (row0 + 4 * r) * C::LP + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[OD];
                    const float* src = s_v + (j + e) * C::LD + dim0;
                    if constexpr (OD == 4) {
                        const float4 y = *reinterpret_cast<const float4*>(src);
                        v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
                    } else {
                        const float2 y = *reinterpret_cast<const float2*>(src);
                        v[0] = y.x; v[1] = y.y;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float w = e == 0 ? p[r].x : e == 1 ? p[r].y : e == 2 ? p[r].z : p[r].w;
#pragma unroll
                        for (int c = 0; c < OD; ++c) o[r][c] = fmaf(w, v[c], o[r][c]);
                    }
                }
            }
        __syncthreads();                                   // V and the weights have been read
        if (t + 1 < tiles) stage(t + 1, true); else cp_async_commit();
    }
    cp_async_wait<0>();
    tree_append<float, D>(g, b, kvh, S, L_p, first_node + split + warp * g.a.n_split, 8 * g.a.n_split, min(n, first_node + per_tile), lane);
    // the rows' sums: over the lanes of a group, then over the groups
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int off = 4; off >= 1; off >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
        if (kg == 0) s_max[group * kTreeF32Rows + row0 + 4 * r] = l[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = row0 + 4 * r;
        if (row >= rows_all) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) sum += s_max[w * kTreeF32Rows + row];
        const int64_t orow = ((int64_t)b * g.N + first_node + row / G) * g.a.H_q + kvh * G + row % G;
        const bool none = sum == 0.f;
        const float inv = none ? 0.f : 1.f / sum;
        float* dst = (g.a.n_split > 1 ? g.a.out_part + (orow * g.a.n_split + split) * D : reinterpret_cast<float*>(g.a.out) + orow * D) + dim0;
#pragma unroll
        for (int c = 0; c < OD; ++c) o[r][c] = none ? 0.f : o[r][c] * inv;
        if constexpr (OD == 4) *reinterpret_cast<float4*>(dst) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
        else *reinterpret_cast<float2*>(dst) = make_float2(o[r][0], o[r][1]);
        if (dim0 == 0) {
            const float lse = none ? -INFINITY : (m[r] * sl + log2f(sum)) * LN2;
            if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + split] = lse;
            else g.a.lse[orow] = lse;
        }
    }
}

// ---- few rows -----------------------------------------------------------------------------------------
constexpr int kTreeFewTile = 32;                           // tokens per tile
constexpr int kTreeFewStages = 3;

template <int D, int ROWS>
struct TreeFewCfg {
    static constexpr int LD = D + 4;
    static constexpr int SLOT = 2 * kTreeFewTile * LD;     // K and V of a tile, in floats
    static constexpr int GROUPS = kTreeF32Threads / (D / 4);               // token groups of the O parts
    static constexpr int LQ = D + 4;
    static constexpr int FLOATS = kTreeFewStages * SLOT + ROWS * LQ + kTreeFewTile * ROWS + 8 * ROWS + 2 * ROWS;
    static constexpr int SMEM = FLOATS * 4;
    static_assert(8 * ROWS * D <= kTreeFewStages * SLOT, "the parts of O, one per warp, take the ring's place");
};

template <int D, int ROWS>
__global__ void __launch_bounds__(kTreeF32Threads, D == 64 && ROWS == 8 ? 4 : 2) dsa_tree_few_kernel(const TreeArgs g) {
    using C = TreeFewCfg<D, ROWS>;
    constexpr int DV = D / 4, PART = D / 8;                // float4 pieces of a row; dims per thread of the scores
    constexpr int RPL = ROWS / 8;                          // rows whose totals a thread ends up with
    extern __shared__ __align__(16) float sm[];
    float* s_ring = sm;
    float* s_q = s_ring + kTreeFewStages * C::SLOT;
    float* s_p = s_q + ROWS * C::LQ;                       // [token][row]
    float* s_max = s_p + kTreeFewTile * ROWS;              // [warp][row]
    float* s_m = s_max + 8 * ROWS;                         // [row] running maximum
    float* s_alpha = s_m + ROWS;
    __shared__ unsigned long long line_of[kTreeMaxNodes];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int split = idx % g.a.n_split; idx /= g.a.n_split;
    const int rt = idx % g.row_tiles; idx /= g.row_tiles;
    const int kvh = idx % g.a.H_kv;
    const int b = idx / g.a.H_kv;
    const int G = g.G, per_tile = ROWS / G, first_node = rt * per_tile;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    int S, L_p, n;
    tree_lengths(g, b, S, L_p, n);
    const int rows_all = min(per_tile, g.N - first_node) * G;
    const int rows = max(0, min(per_tile, n - first_node)) * G;
    const TreeSpan span = tree_span(g, S, L_p);
    const int halves = 2 * span.T;                         // 32-token tiles
    const int per_split = (halves + g.a.n_split - 1) / g.a.n_split;
    const int t0 = min(halves, split * per_split), t1 = min(halves, t0 + per_split);
    const int cached = t1 - t0;
    const int tiles = rows == 0 ? 0 : cached + (split == 0 ? (n + kTreeFewTile - 1) / kTreeFewTile : 0);
    if (tiles == 0) {
        if (rows > 0) tree_append<float, D>(g, b, kvh, S, L_p, first_node + split + warp * g.a.n_split, 8 * g.a.n_split, min(n, first_node + per_tile), lane);
        tree_write_empty<float, D>(g, b, kvh, split, first_node, 0, rows_all, tid, kTreeF32Threads);
        return;
    }
    auto bounds = [&](int t, int& start, int& from, int& to) {
        if (t < cached) {
            span.tile((t0 + t) >> 1, start, from, to);
            start += kTreeFewTile * ((t0 + t) & 1);
            from = max(from, start);
            to = min(to, start + kTreeFewTile);
        } else {
            start = (t - cached) * kTreeFewTile;
            from = start;
            to = min(n, start + kTreeFewTile);
        }
    };
    auto stage = [&](int t) {
        if (t < tiles) {
            int start, from, to;
            bounds(t, start, from, to);
            const float* k = reinterpret_cast<const float*>(t < cached ? g.a.k : g.a.k_new);
            const float* v = reinterpret_cast<const float*>(t < cached ? g.a.v : g.a.v_new);
            // eight threads a row, every eighth piece each: one address per thread
            const int row = tid >> 3, pos = start + row;
            const bool seen = pos >= from && pos < to;
            if (seen) {
                const int64_t off = t < cached ? token_offset(g.a, b, L_p, pos) + (int64_t)kvh * g.a.stride_head
                                               : (((int64_t)b * g.N + pos) * g.a.H_kv + kvh) * D;
                k += off;
                v += off;
            }
            float* dst = s_ring + (t % kTreeFewStages) * C::SLOT + row * C::LD;
#pragma unroll
            for (int j = 0; j < DV / 8; ++j) {
                const int c = ((tid & 7) + 8 * j) * 4;
                cp_async16(dst + c, k + c, seen);
                cp_async16(dst + kTreeFewTile * C::LD + c, v + c, seen);
            }
        }
        cp_async_commit();
    };
    stage(0);
    stage(1);
    if (warp == 0) tree_lines(tree_parents(g, b, lane), line_of, lane);
    for (int i = tid; i < ROWS * DV; i += kTreeF32Threads) {
        const int row = i / DV, c = (i - row * DV) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < rows)
            x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(g.a.q) +
                                                 (((int64_t)b * g.N + first_node + row / G) * g.a.H_q + kvh * G + row % G) * D + c);
        *reinterpret_cast<float4*>(s_q + row * C::LQ + c) = x;
    }
    if (tid < ROWS) { s_m[tid] = -INFINITY; }
    __syncthreads();

    // scores: token `key` of the tile, dims [part * PART, + PART); totals of rows part * RPL + r
    const int key = tid >> 3, part = tid & 7;
    const float sl = g.a.scale_log2;
    unsigned long long own[RPL];
    int64_t win_lo[RPL];
    bool alive[RPL];
    float l[RPL];
#pragma unroll
    for (int r = 0; r < RPL; ++r) {
        const int row = part * RPL + r;
        l[r] = 0.f;
        own[r] = 0ull;
        win_lo[r] = 0;
        alive[r] = row < rows;
        if (!alive[r]) continue;
        const unsigned long long line = line_of[first_node + row / G];
        const int depth = __popcll(line) - 1;
        win_lo[r] = (int64_t)S + depth + 1 - g.a.mask.window;
        own[r] = line;
        if (g.windowed) {
            unsigned long long todo = line;
            while (todo) {
                const int j = __ffsll(todo) - 1;
                todo &= todo - 1;
                const int dj = __popcll(line_of[j]) - 1;
                if (depth - dj >= g.a.mask.window && (int64_t)S + dj >= (int64_t)L_p + g.a.mask.n_sink) own[r] &= ~(1ull << j);
            }
        }
    }
    // O: dims oc .. oc + 3 of all rows, over the tokens og, og + GROUPS, ... of every tile
    const int oc = (tid % DV) * 4, og = tid / DV;
    float4 o[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) o[r] = make_float4(0.f, 0.f, 0.f, 0.f);

    for (int t = 0; t < tiles; ++t) {
        cp_async_wait<1>();
        __syncthreads();                                   // tile t is there for everybody, and tile t - 1 has been read
        stage(t + 2);
        const float* s_k = s_ring + (t % kTreeFewStages) * C::SLOT;
        const float* s_v = s_k + kTreeFewTile * C::LD;
        float x[ROWS] = {};
#pragma unroll
        for (int c = 0; c < PART; c += 4) {
            const int dim = part * 4 + c * 8;              // (pieces of 16 bytes in turn: the eight threads' reads are in a row)
            const float4 k = *reinterpret_cast<const float4*>(s_k + key * C::LD + dim);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float4 q = *reinterpret_cast<const float4*>(s_q + r * C::LQ + dim);
                x[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, x[r]))));
            }
        }
        // halving exchange over the eight threads
#pragma unroll
        for (int off = 4, cnt = ROWS; off >= 1; off >>= 1) {
            cnt /= 2;
            const bool up = (part & off) != 0;
#pragma unroll
            for (int r = 0; r < ROWS / 2; ++r)
                if (r < cnt) {
                    const float send = up ? x[r] : x[r + cnt];
                    const float keep = up ? x[r + cnt] : x[r];
                    x[r] = keep + __shfl_xor_sync(0xffffffffu, send, off);
                }
        }
        int start, from, to;
        bounds(t, start, from, to);
        const int pos = start + key;
#pragma unroll
        for (int r = 0; r < RPL; ++r) {
            bool seen = alive[r] && pos >= from && pos < to;
            if (t < cached) seen = seen && (((t0 + t) >> 1) < span.T1 || pos >= win_lo[r]);
            else seen = seen && ((own[r] >> pos) & 1ull) != 0;
            if (!seen) x[r] = -INFINITY;
            float mx = x[r];
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            if (lane < 8) s_max[warp * ROWS + part * RPL + r] = mx;
        }
        __syncthreads();
        float m_new[RPL];
#pragma unroll
        for (int r = 0; r < RPL; ++r) {
            const int row = part * RPL + r;
            const float m_old = s_m[row];
            float m = m_old;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = fmaxf(m, s_max[w * ROWS + row]);
            m_new[r] = m;
            const float sub = m == -INFINITY ? 0.f : m * sl;
            const float alpha = m == -INFINITY ? 1.f : exp2f((m_old - m) * sl);
            const float p = exp2f(fmaf(x[r], sl, -sub));
            l[r] = l[r] * alpha + p;
            s_p[key * ROWS + row] = p;
            if (key == 0) s_alpha[row] = alpha;
        }
        __syncthreads();
        if (key == 0)
#pragma unroll
            for (int r = 0; r < RPL; ++r) s_m[part * RPL + r] = m_new[r];
        bool same = true;
        float alpha[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) { alpha[r] = s_alpha[r]; same = same && alpha[r] == 1.f; }
        if (!same)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) { o[r].x *= alpha[r]; o[r].y *= alpha[r]; o[r].z *= alpha[r]; o[r].w *= alpha[r]; }
#pragma unroll
        for (int j = 0; j < kTreeFewTile / C::GROUPS; ++j) {
            const int tok = og + j * C::GROUPS;
            const float4 v = *reinterpret_cast<const float4*>(s_v + tok * C::LD + oc);
#pragma unroll
            for (int r4 = 0; r4 < ROWS; r4 += 4) {
                const float4 p = *reinterpret_cast<const float4*>(s_p + tok * ROWS + r4);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = r == 0 ? p.x : r == 1 ? p.y : r == 2 ? p.z : p.w;
                    o[r4 + r].x = fmaf(w, v.x, o[r4 + r].x);
                    o[r4 + r].y = fmaf(w, v.y, o[r4 + r].y);
                    o[r4 + r].z = fmaf(w, v.z, o[r4 + r].z);
                    o[r4 + r].w = fmaf(w, v.w, o[r4 + r].w);
                }
            }
        }
    }
    // sums over the tokens' threads, O over the token groups
#pragma unroll
    for (int r = 0; r < RPL; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 8);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 16);
    }
    cp_async_wait<0>();
    __syncthreads();                                       // the ring has been read for the last time
    float* s_o = s_ring;                                   // [warp][row][D]
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (DV == 16) {                                    // (a warp holds two token groups)
            o[r].x += __shfl_xor_sync(0xffffffffu, o[r].x, 16);
            o[r].y += __shfl_xor_sync(0xffffffffu, o[r].y, 16);
            o[r].z += __shfl_xor_sync(0xffffffffu, o[r].z, 16);
            o[r].w += __shfl_xor_sync(0xffffffffu, o[r].w, 16);
        }
        if (DV == 32 || lane < 16) *reinterpret_cast<float4*>(s_o + (warp * ROWS + r) * D + oc) = o[r];
    }
    if (lane < 8)
#pragma unroll
        for (int r = 0; r < RPL; ++r) s_max[warp * ROWS + part * RPL + r] = l[r];
    tree_append<float, D>(g, b, kvh, S, L_p, first_node + split + warp * g.a.n_split, 8 * g.a.n_split, min(n, first_node + per_tile), lane);
    __syncthreads();
    for (int i = tid; i < rows_all * DV; i += kTreeF32Threads) {
        const int row = i / DV, c = (i - row * DV) * 4;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += s_max[w * ROWS + row];
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 y = *reinterpret_cast<const float4*>(s_o + (j * ROWS + row) * D + c);
            x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        const bool none = sum == 0.f;
        const float inv = none ? 0.f : 1.f / sum;
        const int64_t orow = ((int64_t)b * g.N + first_node + row / G) * g.a.H_q + kvh * G + row % G;
        float* dst = g.a.n_split > 1 ? g.a.out_part + (orow * g.a.n_split + split) * D : reinterpret_cast<float*>(g.a.out) + orow * D;
        *reinterpret_cast<float4*>(dst + c) = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        if (c == 0) {
            const float lse = none ? -INFINITY : (s_m[row] * sl + log2f(sum)) * LN2;
            if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + split] = lse;
            else g.a.lse[orow] = lse;
        }
    }
}

}  // namespace dsa
