// Attention of a tree of drafted tokens over a cache, bf16 (dsa_tree_step).
//
//   x_ij = scale q_i . k_j over the cached tokens and the nodes of i's own line that the mask leaves,
//   lse_i = ln sum_j e^{x_ij},  out_i = sum_j e^{x_ij - lse_i} v_j.
//
// What bounds it: the cached K and V rows are read once per (request, kv head) -- D * 4 bytes per token --
// and every row meets N * G queries (4 N G D operations), so up to some 250 / N G = 64 queries the copy
// bandwidth is the bound by far, and from 256 on the tensor cores and the exponentials are near it too.
// One query token per request has too few rows for the 128-row tensor-core instruction; N drafted ones
// have 16 ... 512, so the products run on tcgen05 with the queries as the 128 rows of A.  Unused rows cost
// tensor time that nobody waits for: 64 keys x 128 rows x 128 dims take under 800 cycles of the tensor
// pipe, and their 32 KB take the SM 1300 cycles to fetch.
//
// A block handles 128 query rows (128 / G nodes) of one (request, kv head) and a range of its 64-token
// tiles.  Warp 4 copies K and V tiles into a ring of shared-memory slots with tensor-map copies (boxes of
// 64 elements x as many tokens as a page holds in one piece, 128-byte swizzle), warp 5 issues the products,
// warps 0-3 own the 128 rows, one thread per row (32 TMEM lanes per warp): they read S = Q K^T from TMEM,
// keep the running maximum and sum, and write P = e^{x - m} back to TMEM as bf16, where it is the A
// operand of O += P V.  S is double buffered: S(j + 1) is computed while tile j's softmax runs.  Warps
// whose 32 rows do not exist sit out.  TMEM: 2 x 64 columns of S (P takes the place of the S it came from) +
// D of O, 256 allocated; two blocks share an SM, so one's set-up and last tile hide behind the other's.
//
// The maximum that the exponentials are taken against trails the true one by at most 2^8 (it is replaced,
// and O rescaled, only when a row's maximum has grown beyond that): e^{x - m} then reaches at most 256,
// which fp32 sums and bf16 P hold as well as 1.  Sums are fp32 over the unrounded P; P is rounded to bf16
// (relative error 2^-9 per weight, averaging out over the row) because the tensor-core product takes
// operands of one 16-bit type.
//
// Rows of V that no node sees (behind the sequence, before the window, behind the last node) are zeroed in
// shared memory before the product: their P is 0, but 0 x NaN is not.
#pragma once
#include "dsa_common.cuh"

namespace dsa {

constexpr int kTreeMaxNodes = 64;
constexpr int kTreeTile = 64;                      // tokens per K / V tile
constexpr int kTreeRows = 128;                     // query rows per block: the M of the products
constexpr int kTreeThreads = 192;

struct TreeArgs {
    AttnArgs a;                                    // lengths, block table, strides, scale, outputs
    const int* parent;                             // [B, N] or NULL (a chain)
    const int* node_count;                         // [B] or NULL (N)
    int N, G;
    int row_tiles;                                 // blocks of kTreeRows query rows per (request, kv head)
    int windowed;                                  // 0: dense
    int box_tokens;                                // tokens per tensor-map box of the caches
    int align_tokens;                              // where a box may start: box_tokens (pages), 1 (contiguous)
    int blk_coord, head_coord;                     // 0: the map's outer / head dimension has one entry (stride 0)
};

struct TreeMaps {
    CUtensorMap q, k, v, k_new, v_new;
};

template <int D>
struct TreeCfg {
    static constexpr int HALVES = D / 64;                                  // 128-byte pieces of a row
    static constexpr int Q_HALF = kTreeRows * 128;
    static constexpr int Q_BYTES = HALVES * Q_HALF;
    static constexpr int KV_HALF = kTreeTile * 128;
    static constexpr int SLOT_BYTES = HALVES * KV_HALF;                    // one K or one V tile
    static constexpr int SLOTS = D == 128 ? 5 : 10;                        // two blocks per SM with either
    static constexpr int TAIL = 1024;                                      // barriers and node tables
    static constexpr int SMEM = Q_BYTES + SLOTS * SLOT_BYTES + TAIL;
    static constexpr int TMEM_COLS = 256;
    static constexpr int COL_S = 0, COL_O = 2 * kTreeTile;
};

// ---- tcgen05 and tensor-map wrappers ---------------------------------------------------------------
__device__ __forceinline__ void tma_box4(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3,
                                         unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
                 ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// D[tmem] (+)= A[smem] B[smem]^T
__device__ __forceinline__ void tc_mma_ss(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc) : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]^T
__device__ __forceinline__ void tc_mma_ts(unsigned d, unsigned a, unsigned long long b, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((unsigned)acc) : "memory");
}
__device__ __forceinline__ void tc_ld32(unsigned (&r)[32], unsigned addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tc_st32(unsigned addr, const unsigned (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                   "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory operand descriptor, 128-byte swizzle: atoms of 8 rows x 128 bytes.  `stride`: bytes from one
// 8-row atom to the next along the rows; `lead`: from one 64-element column block to the next (used where the
// 64 contiguous elements run along M / N and the operand is wider than they are).
__device__ __forceinline__ unsigned long long smem_desc(unsigned addr, unsigned lead, unsigned stride) {
    return (unsigned long long)((addr >> 4) & 0x3fffu) | ((unsigned long long)((lead >> 4) & 0x3fffu) << 16) |
           ((unsigned long long)((stride >> 4) & 0x3fffu) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: bf16 x bf16 -> fp32, M x N; b_mn: B's contiguous dimension is N, not K.
__host__ __device__ constexpr unsigned instr_desc(int M, int N, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((unsigned)(N >> 3) << 17) |
           ((unsigned)(M >> 4) << 24);
}

// ---- what a block works on, in 64-token tiles ---------------------------------------------------------
// The cached tokens that some node of the block sees: [0, P0) (dense: everything; windowed: prompt and
// sinks) and [lo, S).  Tiles 0 .. T1-1 start at 64 t, tiles T1 .. T-1 at lo_al + 64 (t - T1) with lo_al = lo
// rounded down to a whole box.
struct TreeSpan {
    int S, P0, lo, lo_al, T1, T;
    __device__ __forceinline__ void tile(int t, int& start, int& from, int& to) const {   // tokens [from, to) of it are seen
        if (t < T1) { start = t * kTreeTile; from = start; to = min(P0, start + kTreeTile); }
        else { start = lo_al + (t - T1) * kTreeTile; from = max(lo, start); to = min(S, start + kTreeTile); }
    }
};

// Lengths of request b: cached tokens, prompt, nodes that exist and have room.
__device__ __forceinline__ void tree_lengths(const TreeArgs& g, int b, int& S, int& L_p, int& n) {
    const int raw = g.a.seq_len[b];
    S = max(0, min(raw, g.a.max_seq_len));
    L_p = max(0, min(g.a.prompt_len[b], S));
    n = g.node_count ? max(0, min(g.node_count[b], g.N)) : g.N;
    n = raw < 0 ? 0 : min(n, g.a.max_seq_len - S);
}

__device__ __forceinline__ TreeSpan tree_span(const TreeArgs& g, int S, int L_p, int min_depth) {
    TreeSpan s;
    s.S = S;
    if (!g.windowed) {
        s.P0 = S; s.lo = s.lo_al = S;
    } else {
        s.P0 = L_p + min(g.a.mask.n_sink, S - L_p);
        s.lo = min(S, max(s.P0, S + min_depth + 1 - g.a.mask.window));
        s.lo_al = s.lo / g.align_tokens * g.align_tokens;
    }
    s.T1 = (s.P0 + kTreeTile - 1) / kTreeTile;
    s.T = s.T1 + (S - s.lo_al + kTreeTile - 1) / kTreeTile;
    if (s.lo >= S) s.T = s.T1;
    return s;
}

// Ancestor sets of the nodes as 64-bit words (bit j: node j is node i or an ancestor of it), by one warp: every
// round doubles the length of the line that a word covers.
__device__ __forceinline__ void tree_lines(const TreeArgs& g, int b, unsigned long long* line_of, int lane) {
    unsigned long long m[2];
    int up[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        m[h] = 1ull << i;
        int p = i < g.N ? (g.parent ? g.parent[(int64_t)b * g.N + i] : i - 1) : -1;
        up[h] = (p >= 0 && p < i) ? p : -1;
    }
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

// The nodes' K / V rows of kv head kvh to the cache, by `count` threads.
template <typename T, int D>
__device__ __forceinline__ void tree_append(const TreeArgs& g, int b, int kvh, int S, int L_p, int n, int tid, int count) {
    constexpr int VEC = 16 / (int)sizeof(T), CPR = D / VEC;
    T* kc = reinterpret_cast<T*>(const_cast<void*>(g.a.k));
    T* vc = reinterpret_cast<T*>(const_cast<void*>(g.a.v));
    for (int i = tid; i < n * CPR; i += count) {
        const int node = i / CPR, c = (i - node * CPR) * VEC;
        const int64_t src = (((int64_t)b * g.N + node) * g.a.H_kv + kvh) * D + c;
        const int64_t dst = token_offset(g.a, b, L_p, S + node) + (int64_t)kvh * g.a.stride_head + c;
        *reinterpret_cast<uint4*>(kc + dst) = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(g.a.k_new) + src);
        *reinterpret_cast<uint4*>(vc + dst) = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(g.a.v_new) + src);
    }
}

// Rows [r0, r1) of a block's query rows (row r: node first_node + r / G, head kvh * G + r % G) have nothing to
// attend to in this split: zeros and -inf, or an empty part for the combine.
template <typename T, int D>
__device__ __forceinline__ void tree_write_empty(const TreeArgs& g, int b, int kvh, int split, int first_node, int r0, int r1,
                                                 int tid, int count) {
    for (int r = r0 + tid; r < r1; r += count) {
        const int64_t row = ((int64_t)b * g.N + first_node + r / g.G) * g.a.H_q + kvh * g.G + r % g.G;
        if (g.a.n_split > 1) { g.a.lse_part[row * g.a.n_split + split] = -INFINITY; continue; }
        g.a.lse[row] = -INFINITY;
        T* out = reinterpret_cast<T*>(g.a.out) + row * D;
#pragma unroll
        for (int c = 0; c < D * (int)sizeof(T) / 16; ++c) reinterpret_cast<uint4*>(out)[c] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Wait for phase `parity` of `bar`, about a second at most.  False: this wait ran out, or another warp's did
// (*abort); the block then drains what it has in flight and ends.
__device__ __forceinline__ bool tree_wait(unsigned long long* bar, unsigned parity, volatile int* abort, int* wait_timeouts,
                                          int lane) {
    bool ok = mbar_try_wait(bar, parity);
    if (!ok) {
        const long long t0 = clock64();
        while (!(ok = mbar_try_wait(bar, parity))) {
            if (*abort) break;
            if (clock64() - t0 > kMbarWaitCycles) {
                *abort = 1;
                if (lane == 0 && wait_timeouts) atomicAdd(wait_timeouts, 1);
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, ok);                       // (one answer for the warp)
}

template <int D>
__global__ void __launch_bounds__(kTreeThreads, 2) dsa_tree_kernel(const TreeArgs g, const __grid_constant__ TreeMaps maps) {
    using C = TreeCfg<D>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + C::Q_BYTES + C::SLOTS * C::SLOT_BYTES);
    unsigned long long* full = bars;                          // a ring slot has landed
    unsigned long long* empty = bars + C::SLOTS;              // the products that read it are done
    unsigned long long* q_full = bars + 2 * C::SLOTS;
    unsigned long long* s_full = q_full + 1;                  // [2] scores are in TMEM
    unsigned long long* p_ready = q_full + 3;                 // [2] weights are in TMEM
    unsigned long long* pv_done = q_full + 5;                 // [2] O holds the tile
    unsigned long long* drained = q_full + 7;
    unsigned long long* line_of = q_full + 8;                 // [64]
    int* s_misc = reinterpret_cast<int*>(line_of + kTreeMaxNodes);   // [0] TMEM address, [1] abort, [2] lowest depth
    static_assert((2 * C::SLOTS + 8 + kTreeMaxNodes) * 8 + 12 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int rt = idx % g.row_tiles; idx /= g.row_tiles;
    const int kvh = idx % g.a.H_kv; idx /= g.a.H_kv;
    const int split = idx % g.a.n_split;
    const int b = idx / g.a.n_split;
    const int G = g.G, per_tile = kTreeRows / G, first_node = rt * per_tile;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    int S, L_p, n;
    tree_lengths(g, b, S, L_p, n);
    const int rows_all = min(per_tile, g.N - first_node) * G;              // rows that this block writes
    const int rows = max(0, min(per_tile, n - first_node)) * G;            // rows of nodes that exist
    if (rows == 0) {
        tree_write_empty<T, D>(g, b, kvh, split, first_node, 0, rows_all, tid, kTreeThreads);
        return;
    }
    const int active_warps = (rows + 31) / 32;
    if (warp == 0) {
        tree_lines(g, b, line_of, lane);
        __syncwarp();
        int d = kTreeMaxNodes;
        for (int i = first_node + lane; i < first_node + rows / G; i += 32) d = min(d, __popcll(line_of[i]) - 1);
        d = __reduce_min_sync(0xffffffffu, d);
        if (lane == 0) { s_misc[2] = d; s_misc[1] = 0; }
    } else if (warp == 5 && lane == 0) {
        for (int s = 0; s < C::SLOTS; ++s) { mbar_init(full + s, 1); mbar_init(empty + s, 1); }
        mbar_init(q_full, 1);
        for (int s = 0; s < 2; ++s) { mbar_init(s_full + s, 1); mbar_init(p_ready + s, active_warps); mbar_init(pv_done + s, 1); }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const TreeSpan span = tree_span(g, S, L_p, s_misc[2]);
    const int per_split = (span.T + g.a.n_split - 1) / g.a.n_split;
    const int t0 = min(span.T, split * per_split), t1 = min(span.T, t0 + per_split);
    const bool has_nodes = split == 0;                                      // the nodes' own rows: one tile more, the last
    const int cached = t1 - t0, tiles = cached + (has_nodes ? 1 : 0);
    if (tiles == 0) {
        tree_write_empty<T, D>(g, b, kvh, split, first_node, 0, rows_all, tid, kTreeThreads);
        return;
    }

    if (warp == 4) {
        // ---- copies -------------------------------------------------------------------------------
        const int r = g.box_tokens;
        if (lane == 0) {
            const int box_nodes = min(per_tile, g.N);
            mbar_expect_tx(q_full, (unsigned)(C::HALVES * box_nodes * G * 128));
            for (int h = 0; h < C::HALVES; ++h) tma_box4(s_q + h * C::Q_HALF, &maps.q, 64 * h, kvh * G, first_node, b, q_full);
        }
        __syncwarp();
        int issued = 0;
        // the page (or request) of this lane's boxes `lane` and `lane + 32` of tile t; loaded a tile ahead of its copies
        auto ids_of = [&](int t, int (&blk)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                blk[h] = g.blk_coord ? b : 0;
                const int j = lane + 32 * h;
                if (t < cached && g.a.block_table && j * r < kTreeTile) {
                    int start, from, to;
                    span.tile(t0 + t, start, from, to);
                    const int bi = min((start + j * r) / g.a.block_size, g.a.max_blocks - 1);
                    blk[h] = max(0, min(g.a.block_table[(int64_t)b * g.a.max_blocks + bi], g.a.num_blocks - 1)) * g.blk_coord;
                }
            }
        };
        auto issue = [&](int t, bool is_v, const int (&blk)[2]) -> bool {
            const int s = issued % C::SLOTS;
            if (issued >= C::SLOTS && !tree_wait(empty + s, (issued / C::SLOTS - 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
            unsigned char* dst = s_ring + s * C::SLOT_BYTES;
            if (t < cached) {
                int start, from, to;
                span.tile(t0 + t, start, from, to);
                const int j0 = (from - start) / r, j1 = (to - start + r - 1) / r;
                if (lane == 0) mbar_expect_tx(full + s, (unsigned)((j1 - j0) * C::HALVES * r * 128));
                __syncwarp();
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) {
                    const int j = lane + 32 * h2;
                    if (j < j0 || j >= j1) continue;
                    const int pos = start + j * r;
                    const int tok = g.a.block_table ? pos % g.a.block_size : pos;
                    for (int h = 0; h < C::HALVES; ++h)
                        tma_box4(dst + h * C::KV_HALF + j * r * 128, is_v ? &maps.v : &maps.k, 64 * h, tok, kvh * g.head_coord,
                                 blk[h2], full + s);
                }
            } else if (lane == 0) {
                mbar_expect_tx(full + s, (unsigned)(C::HALVES * g.N * 128));
                for (int h = 0; h < C::HALVES; ++h)
                    tma_box4(dst + h * C::KV_HALF, is_v ? &maps.v_new : &maps.k_new, 64 * h, 0, kvh, b, full + s);
            }
            __syncwarp();
            ++issued;
            return true;
        };
        int id0[2], id1[2], id2[2];
        ids_of(0, id0);
        ids_of(1, id1);
        bool ok = issue(0, false, id0) && (tiles < 2 || issue(1, false, id1));
        for (int t = 0; ok && t < tiles; ++t) {
            ids_of(t + 2, id2);
            ok = issue(t, true, id0) && (t + 2 >= tiles || issue(t + 2, false, id2));
#pragma unroll
            for (int h = 0; h < 2; ++h) { id0[h] = id1[h]; id1[h] = id2[h]; }
        }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        volatile int no_abort = 0;
        tree_wait(q_full, 0u, &no_abort, nullptr, lane);
        for (int c = max(0, issued - C::SLOTS); c < issued; ++c)
            if (!tree_wait(full + c % C::SLOTS, (c / C::SLOTS) & 1, &no_abort, nullptr, lane)) break;
    } else {
        if (warp == 5) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
            tc_fence_before();
        }
        asm volatile("bar.sync 1, 160;" ::: "memory");
        tc_fence_after();
        const unsigned tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
        if (warp == 5) {
            // ---- products ---------------------------------------------------------------------------
            constexpr unsigned kIdescS = instr_desc(kTreeRows, kTreeTile, false), kIdescO = instr_desc(kTreeRows, D, true);
            int used = 0;
            auto scores = [&](int t) -> bool {
                const int s = used % C::SLOTS;
                if (!tree_wait(full + s, (used / C::SLOTS) & 1, abort, g.a.wait_timeouts, lane)) return false;
                tc_fence_after();
                if (lane == 0) {
                    const unsigned qa = smem_u32(s_q), ka = smem_u32(s_ring + s * C::SLOT_BYTES);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        tc_mma_ss(tmem + C::COL_S + (t & 1) * kTreeTile,
                                  smem_desc(qa + (kk / 4) * C::Q_HALF + (kk % 4) * 32, 16, 1024),
                                  smem_desc(ka + (kk / 4) * C::KV_HALF + (kk % 4) * 32, 16, 1024), kIdescS, kk > 0);
                    tc_commit(empty + s);
                    tc_commit(s_full + (t & 1));
                }
                __syncwarp();
                ++used;
                return true;
            };
            auto values = [&](int t) -> bool {
                if (!tree_wait(p_ready + (t & 1), (t >> 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
                const int s = used % C::SLOTS;
                if (!tree_wait(full + s, (used / C::SLOTS) & 1, abort, g.a.wait_timeouts, lane)) return false;
                unsigned char* v = s_ring + s * C::SLOT_BYTES;
                // rows of V that nobody sees: zero, whatever the cache or the slot held there
                int lo = 0, hi = n;
                if (t < cached) {
                    int start;
                    span.tile(t0 + t, start, lo, hi);
                    lo -= start; hi -= start;
                }
                if (lo > 0 || hi < kTreeTile) {
                    for (int i = lane; i < kTreeTile * 8; i += 32) {
                        const int row = i >> 3;
                        if (row >= lo && row < hi) continue;
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h)
                            *reinterpret_cast<uint4*>(v + h * C::KV_HALF + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                tc_fence_after();
                if (lane == 0) {
                    const unsigned va = smem_u32(v);
#pragma unroll
                    for (int kk = 0; kk < kTreeTile / 16; ++kk)
                        tc_mma_ts(tmem + C::COL_O, tmem + C::COL_S + (t & 1) * kTreeTile + kk * 8,
                                  smem_desc(va + kk * 2048, C::KV_HALF, 1024), kIdescO, t > 0 || kk > 0);
                    tc_commit(empty + s);
                    tc_commit(pv_done + (t & 1));
                }
                __syncwarp();
                ++used;
                return true;
            };
            bool ok = tree_wait(q_full, 0u, abort, g.a.wait_timeouts, lane) && scores(0) && (tiles < 2 || scores(1));
            for (int t = 0; ok && t < tiles; ++t) ok = values(t) && (t + 2 >= tiles || scores(t + 2));
            if (!ok) {                                       // TMEM is given back only when no product uses it
                if (lane == 0) tc_commit(drained);
                __syncwarp();
                volatile int no_abort = 0;
                tree_wait(drained, 0u, &no_abort, nullptr, lane);
            }
        } else {
            // ---- softmax: one thread per query row --------------------------------------------------
            if (has_nodes && rt == 0) tree_append<T, D>(g, b, kvh, S, L_p, n, tid, 128);
            const int row = tid;                              // of the block's 128
            const int node = first_node + row / G;
            const bool alive = row < rows;
            const bool work = warp < active_warps;
            const unsigned lane_base = (unsigned)(warp * 32) << 16;
            const float sl = g.a.scale_log2;
            float m_ref = -INFINITY, l = 0.f;                 // (m_ref in units of the raw scores)
            bool ok = true;
            if (work) {
                const unsigned long long line = alive ? line_of[node] : 0ull;
                const int depth = __popcll(line) - 1;
                // the first cached position of the window (dense: everything is in [0, P0))
                const int64_t win_lo = (int64_t)S + depth + 1 - g.a.mask.window;
                unsigned long long own = line & (n < 64 ? (1ull << n) - 1ull : ~0ull);
                if (g.windowed && alive) {
                    // drafted tokens of the own line that the window has left behind (sinks stay)
                    unsigned long long keep = own, todo = own;
                    while (todo) {
                        const int j = __ffsll(todo) - 1;
                        todo &= todo - 1;
                        const int dj = __popcll(line_of[j]) - 1;
                        if (depth - dj >= g.a.mask.window && (int64_t)S + dj >= (int64_t)L_p + g.a.mask.n_sink) keep &= ~(1ull << j);
                    }
                    own = keep;
                }
                for (int t = 0; t < tiles; ++t) {
                    const int buf = t & 1;
                    if (!tree_wait(s_full + buf, (t >> 1) & 1, abort, g.a.wait_timeouts, lane)) { ok = false; break; }
                    tc_fence_after();
                    const unsigned s_addr = tmem + lane_base + C::COL_S + buf * kTreeTile;
                    unsigned x0[32], x1[32];
                    tc_ld32(x0, s_addr);
                    tc_ld32(x1, s_addr + 32);
                    unsigned long long see;
                    if (t < cached) {
                        int start, from, to;
                        span.tile(t0 + t, start, from, to);
                        int c0 = 0, c1 = to - start;
                        if (t0 + t >= span.T1) c0 = (int)max((int64_t)from, min((int64_t)to, win_lo)) - start;
                        if (!alive) c1 = 0;
                        see = c1 >= 64 ? ~0ull : (1ull << c1) - 1ull;
                        see = c0 >= 64 ? 0ull : (c0 > 0 ? (see >> c0) << c0 : see);
                    } else {
                        see = own;
                    }
                    tc_wait_ld();
                    if (__any_sync(0xffffffffu, see != ~0ull)) {
                        const unsigned lo = (unsigned)see, hi = (unsigned)(see >> 32);
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (!((lo >> i) & 1u)) x0[i] = 0xff800000u;
                            if (!((hi >> i) & 1u)) x1[i] = 0xff800000u;
                        }
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        mx[i & 1] = fmaxf(mx[i & 1], __uint_as_float(x0[i]));
                        mx[2 + (i & 1)] = fmaxf(mx[2 + (i & 1)], __uint_as_float(x1[i]));
                    }
                    const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    // (-inf - -inf is NaN: compares false, nothing to rescale)
                    if (__any_sync(0xffffffffu, (m_tile - m_ref) * sl > 8.f)) {
                        const float m_new = fmaxf(m_ref, m_tile);
                        const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m_ref - m_new) * sl);
                        m_ref = m_new;
                        l *= alpha;
                        if (t > 0) {
                            if (!tree_wait(pv_done + ((t - 1) & 1), ((t - 1) >> 1) & 1, abort, g.a.wait_timeouts, lane)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                unsigned o[32];
                                tc_ld32(o, tmem + lane_base + C::COL_O + c);
                                tc_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tc_st32(tmem + lane_base + C::COL_O + c, o);
                            }
                        }
                    }
                    const float sub = m_ref == -INFINITY ? 0.f : m_ref * sl;
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
                    unsigned pk[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const unsigned a0 = i < 16 ? x0[2 * i] : x1[2 * i - 32], a1 = i < 16 ? x0[2 * i + 1] : x1[2 * i - 31];
                        const float p0 = fast_exp2(fmaf(__uint_as_float(a0), sl, -sub));
                        const float p1 = fast_exp2(fmaf(__uint_as_float(a1), sl, -sub));
                        sum[i & 3] += p0 + p1;
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(pk[i]) : "f"(p1), "f"(p0));
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tc_st32(s_addr, pk);
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_ready + buf);
                }
                if (ok) ok = tree_wait(pv_done + ((tiles - 1) & 1), ((tiles - 1) >> 1) & 1, abort, g.a.wait_timeouts, lane);
                tc_fence_after();
            }
            // ---- results --------------------------------------------------------------------------
            if (work && ok) {
                const bool mine = row < rows_all;
                const bool none = l == 0.f;                    // nothing seen: zeros and -inf
                const float inv = none ? 0.f : 1.f / l;
                const int64_t orow = ((int64_t)b * g.N + node) * g.a.H_q + kvh * G + row % G;
                const float lse = none ? -INFINITY : (m_ref * sl + log2f(l)) * LN2;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned o[32];
                    tc_ld32(o, tmem + lane_base + C::COL_O + c);
                    tc_wait_ld();
                    if (mine) {
                        float f[32];
    #pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = none ? 0.f : __uint_as_float(o[i]) * inv;
                        if (g.a.n_split > 1) {
                            float* dst = g.a.out_part + (orow * g.a.n_split + split) * D + c;
    #pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<float4*>(dst + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
                        } else {
                            T* dst = reinterpret_cast<T*>(g.a.out) + orow * D + c;
    #pragma unroll
                            for (int i = 0; i < 32; i += 8) {
                                unsigned w[4];
    #pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(f[i + 2 * k + 1]), "f"(f[i + 2 * k]));
                                *reinterpret_cast<uint4*>(dst + i) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                    __syncwarp();
                }
                if (mine) {
                    if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + split] = lse;
                    else g.a.lse[orow] = lse;
                }
            } else if (!work) {
                // rows of nodes that do not exist, beyond the last warp with rows
                const int first = active_warps * 32;
                tree_write_empty<T, D>(g, b, kvh, split, first_node, first, rows_all, tid - first, 128 - first);
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;"
                     ::"r"((unsigned)*reinterpret_cast<volatile int*>(s_misc)), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
