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
// whose 32 rows do not exist sit out.  Warps 6 and 7 append the nodes' rows to the cache meanwhile (by the
// softmax warps, before their first tile, that took 6 us of a 60 us block).  TMEM: 2 x 64 columns of S (P
// takes the place of the S it came from) + D of O, 256 allocated; two blocks share an SM, so one's set-up
// and last tile hide behind the other's.
//
// Work is cut along the cached tokens where there are fewer blocks than places, or where their number leaves
// the last wave of blocks half empty: the 2, 4 or 8 blocks of a thread-block cluster share the tiles of one
// (request, kv head) and merge their states through distributed shared memory, without partial results in
// HBM or a second launch.  Only where eight are too few (a long sequence under one or two heads) partial
// results go to the workspace and the combine kernel.
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
constexpr int kTreeThreads = 256;

struct TreeArgs {
    AttnArgs a;                                    // lengths, block table, strides, scale, outputs
    const int* parent;                             // [B, N] or NULL (a chain)
    const int* node_count;                         // [B] or NULL (N)
    int N, G;
    int row_tiles;                                 // blocks of kTreeRows query rows per (request, kv head)
    int windowed;                                  // 0: dense
    int box_tokens;                                // tokens per tensor-map box of the caches
    int box_shift;                                 // and its logarithm
    int align_tokens;                              // where a box may start: box_tokens (pages), 1 (contiguous)
    int cluster;                                   // blocks that share the tiles and merge on chip (1: none; else n_split is 1)
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
    static constexpr int PART_LD = D + 4;                                  // row of a partial result, in floats
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
// The cached tokens that some node of the request sees: [0, P0) (dense: everything; windowed: prompt and
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

__device__ __forceinline__ TreeSpan tree_span(const TreeArgs& g, int S, int L_p) {
    TreeSpan s;
    s.S = S;
    if (!g.windowed) {
        s.P0 = S; s.lo = s.lo_al = S;
    } else {
        s.P0 = L_p + min(g.a.mask.n_sink, S - L_p);
        s.lo = min(S, max(s.P0, S + 1 - g.a.mask.window));          // (a root's window)
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

// K / V rows of the nodes first, first + step, ... below n, kv head kvh, to the cache, by `count` threads.
template <typename T, int D>
__device__ __forceinline__ void tree_append(const TreeArgs& g, int b, int kvh, int S, int L_p, int first, int step, int n, int tid,
                                            int count) {
    constexpr int VEC = 16 / (int)sizeof(T), CPR = D / VEC;
    T* kc = reinterpret_cast<T*>(const_cast<void*>(g.a.k));
    T* vc = reinterpret_cast<T*>(const_cast<void*>(g.a.v));
#pragma unroll 4
    for (int i = tid; i < (n - first + step - 1) / step * CPR; i += count) {
        const int node = first + i / CPR * step, c = i % CPR * VEC;
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

// ---- thread-block clusters ---------------------------------------------------------------------------
__device__ __forceinline__ void tree_cluster_barrier() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned tree_peer(const void* p, unsigned rank) {   // p in the shared memory of block `rank`
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 tree_peer_f2(unsigned addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 tree_peer_f4(unsigned addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
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
    int* s_misc = reinterpret_cast<int*>(line_of + kTreeMaxNodes);   // [0] TMEM address, [1] abort
    static_assert((2 * C::SLOTS + 8 + kTreeMaxNodes) * 8 + 8 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;
    // after the last product, for a merge within the cluster: O (rows padded against bank conflicts) and per row
    // (maximum in base-2 units, sum)
    float* s_part = reinterpret_cast<float*>(s_ring);
    float2* s_ml = reinterpret_cast<float2*>(s_q);
    static_assert(kTreeRows * C::PART_LD * 4 <= C::SLOTS * C::SLOT_BYTES, "the partial result takes the ring's place");

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int pieces = g.cluster * g.a.n_split;               // (one of the two is 1)
    const int piece = idx % pieces; idx /= pieces;
    const int rt = idx % g.row_tiles; idx /= g.row_tiles;
    const int kvh = idx % g.a.H_kv;
    const int b = idx / g.a.H_kv;
    const int G = g.G, per_tile = kTreeRows / G, first_node = rt * per_tile;

    // set-up that reads nothing: it may run while the launch in front finishes
    if (warp == 4 && lane == 0) {
        for (int s = 0; s < C::SLOTS; ++s) { mbar_init(full + s, 1); mbar_init(empty + s, 1); }
        mbar_init(q_full, 1);
        for (int s = 0; s < 2; ++s) { mbar_init(s_full + s, 1); mbar_init(pv_done + s, 1); }
        mbar_init(drained, 1);
        s_misc[1] = 0;
    } else if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_fence_before();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    int S, L_p, n;
    tree_lengths(g, b, S, L_p, n);
    const int rows_all = min(per_tile, g.N - first_node) * G;              // rows that this block writes
    const int rows = max(0, min(per_tile, n - first_node)) * G;            // rows of nodes that exist
    const int active_warps = (rows + 31) / 32;                              // warps with rows
    const TreeSpan span = tree_span(g, S, L_p);
    const int per_piece = (span.T + pieces - 1) / pieces;
    const int t0 = min(span.T, piece * per_piece), t1 = min(span.T, t0 + per_piece);
    const bool has_nodes = piece == 0;                                      // the nodes' own rows: one tile more, the last
    const int cached = t1 - t0;
    const int tiles = rows == 0 ? 0 : cached + (has_nodes ? 1 : 0);

    float m_ref = -INFINITY, l = 0.f;                         // softmax threads: maximum (of the raw scores) and sum of their row
    unsigned tmem = 0;
    if (warp == 4) {
        // ---- copies -------------------------------------------------------------------------------
        if (lane == 0) {
            for (int s = 0; s < 2; ++s) mbar_init(p_ready + s, max(active_warps, 1));
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("bar.arrive 1, 192;" ::: "memory");      // (the barriers are ready)
        if (tiles > 0) {
            if (lane == 0) {
                const int box_nodes = min(per_tile, g.N);
                mbar_expect_tx(q_full, (unsigned)(C::HALVES * box_nodes * G * 128));
                for (int h = 0; h < C::HALVES; ++h) tma_box4(s_q + h * C::Q_HALF, &maps.q, 64 * h, kvh * G, first_node, b, q_full);
            }
            __syncwarp();
            const int shift = g.box_shift;
            // where this lane's boxes `lane` and `lane + 32` of a tile come from: (page or request, token in it);
            // looked up two tiles ahead of their copies
            struct Where { int blk[2], tok[2]; };
            auto where = [&](int t) -> Where {
                Where w;
                int start = 0, from, to;
                if (t < cached) span.tile(t0 + t, start, from, to);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int pos = start + ((lane + 32 * h) << shift);
                    w.blk[h] = g.blk_coord ? b : 0;
                    w.tok[h] = pos;
                    if (g.a.block_table) {
                        const int bi = pos / g.a.block_size;
                        w.tok[h] = pos - bi * g.a.block_size;
                        if (t < cached && ((lane + 32 * h) << shift) < kTreeTile)
                            w.blk[h] = max(0, min(__ldg(g.a.block_table + (int64_t)b * g.a.max_blocks + min(bi, g.a.max_blocks - 1)),
                                                  g.a.num_blocks - 1)) * g.blk_coord;
                    }
                }
                return w;
            };
            int issued = 0, slot = 0, round = 0;
            auto issue = [&](int t, bool is_v, const Where& w) -> bool {
                if (round > 0 && !tree_wait(empty + slot, (round - 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
                unsigned char* dst = s_ring + slot * C::SLOT_BYTES;
                unsigned long long* bar = full + slot;
                if (t < cached) {
                    int start, from, to;
                    span.tile(t0 + t, start, from, to);
                    const int j0 = (from - start) >> shift, j1 = (to - start + (1 << shift) - 1) >> shift;
                    if (lane == 0) mbar_expect_tx(bar, (unsigned)(((j1 - j0) * C::HALVES) << shift) * 128u);
                    __syncwarp();
                    const CUtensorMap* map = is_v ? &maps.v : &maps.k;
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const int j = lane + 32 * h2;
                        if (j >= j0 && j < j1) {
#pragma unroll
                            for (int h = 0; h < C::HALVES; ++h)
                                tma_box4(dst + h * C::KV_HALF + ((j << shift) * 128), map, 64 * h, w.tok[h2], kvh * g.head_coord,
                                         w.blk[h2], bar);
                        }
                        if (shift >= 1) break;
                    }
                } else if (lane == 0) {
                    mbar_expect_tx(bar, (unsigned)(C::HALVES * g.N * 128));
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h)
                        tma_box4(dst + h * C::KV_HALF, is_v ? &maps.v_new : &maps.k_new, 64 * h, 0, kvh, b, bar);
                }
                __syncwarp();
                ++issued;
                if (++slot == C::SLOTS) { slot = 0; ++round; }
                return true;
            };
            Where w0 = where(0), w1 = where(1), w2 = where(2);
            bool ok = issue(0, false, w0) && (tiles < 2 || issue(1, false, w1));
            for (int t = 0; ok && t < tiles; ++t) {
                const Where w3 = where(t + 3);
                ok = issue(t, true, w0) && (t + 2 >= tiles || issue(t + 2, false, w2));
                w0 = w1; w1 = w2; w2 = w3;
            }
            // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
            volatile int no_abort = 0;
            tree_wait(q_full, 0u, &no_abort, nullptr, lane);
            for (int c = max(0, issued - C::SLOTS); c < issued; ++c)
                if (!tree_wait(full + c % C::SLOTS, (c / C::SLOTS) & 1, &no_abort, nullptr, lane)) break;
        }
    } else if (warp >= 6) {
        // ---- the nodes' rows to the cache: every block those of its own nodes, the pieces in turn ----------------
        tree_append<T, D>(g, b, kvh, S, L_p, first_node + piece, pieces, min(n, first_node + per_tile), tid - 192, 64);
    } else {
        if (warp == 0) tree_lines(g, b, line_of, lane);
        asm volatile("bar.sync 1, 192;" ::: "memory");
        tc_fence_after();
        tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
        if (warp == 5) {
            // ---- products ---------------------------------------------------------------------------
            constexpr unsigned kIdescS = instr_desc(kTreeRows, kTreeTile, false), kIdescO = instr_desc(kTreeRows, D, true);
            int slot = 0, round = 0;                         // of the ring
            auto next_slot = [&]() { if (++slot == C::SLOTS) { slot = 0; ++round; } };
            auto scores = [&](int t) -> bool {
                const int s = slot;
                if (!tree_wait(full + s, round & 1, abort, g.a.wait_timeouts, lane)) return false;
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
                next_slot();
                return true;
            };
            auto values = [&](int t) -> bool {
                if (!tree_wait(p_ready + (t & 1), (t >> 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
                const int s = slot;
                if (!tree_wait(full + s, round & 1, abort, g.a.wait_timeouts, lane)) return false;
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
                next_slot();
                return true;
            };
            bool ok = tiles > 0 && tree_wait(q_full, 0u, abort, g.a.wait_timeouts, lane) && scores(0) && (tiles < 2 || scores(1));
            for (int t = 0; ok && t < tiles; ++t) ok = values(t) && (t + 2 >= tiles || scores(t + 2));
            if (!ok && tiles > 0) {                          // TMEM is given back only when no product uses it
                if (lane == 0) tc_commit(drained);
                __syncwarp();
                volatile int no_abort = 0;
                tree_wait(drained, 0u, &no_abort, nullptr, lane);
            }
        } else {
            // ---- softmax: one thread per query row --------------------------------------------------
            const int row = tid;                              // of the block's 128
            const int node = first_node + row / G;
            const bool alive = row < rows;
            const bool work = tiles > 0 && warp < active_warps;
            const unsigned lane_base = (unsigned)(warp * 32) << 16;
            const float sl = g.a.scale_log2;
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
                        pk[i] = pack_bf16(p0, p1);
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
            if (g.cluster > 1) {
                // (merged below)
            } else if (work && ok) {
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
                            float* dst = g.a.out_part + (orow * g.a.n_split + piece) * D + c;
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
                                    w[k] = pack_bf16(f[i + 2 * k], f[i + 2 * k + 1]);
                                *reinterpret_cast<uint4*>(dst + i) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                    __syncwarp();
                }
                if (mine) {
                    if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + piece] = lse;
                    else g.a.lse[orow] = lse;
                }
            } else if (!work) {
                // rows of nodes that do not exist, beyond the last warp with rows; all rows where there is nothing to see
                const int first = tiles > 0 ? active_warps * 32 : 0;
                tree_write_empty<T, D>(g, b, kvh, piece, first_node, first, rows_all, tid - first, 128 - first);
            }
        }
        tc_fence_before();
    }
    if (g.cluster > 1) {
        // ---- merge: out = sum_i e^{m_i - M} O_i / sum_i e^{m_i - M} l_i over the cluster's blocks --------------
        __syncthreads();                                      // the ring and Q have been read for the last time
        if (warp < 4) {
            s_ml[tid] = make_float2(l == 0.f ? -INFINITY : m_ref * g.a.scale_log2, l);
            if (tiles > 0 && warp < active_warps) {
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned o[32];
                    tc_ld32(o, tmem + ((unsigned)(warp * 32) << 16) + C::COL_O + c);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<uint4*>(s_part + tid * C::PART_LD + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                }
                tc_fence_before();
            }
        }
        tree_cluster_barrier();
        constexpr int LPR = D / 4, RPW = 32 / LPR;            // lanes per row (four dims each), rows per warp
        const int sub = lane / LPR, c4 = (lane % LPR) * 4;
        for (int r = piece + (warp * RPW + sub) * g.cluster; r < rows_all; r += 8 * RPW * g.cluster) {
            float m_max = -INFINITY;
            for (int i = 0; i < g.cluster; ++i) m_max = fmaxf(m_max, tree_peer_f2(tree_peer(s_ml + r, i)).x);
            float sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int i = 0; i < g.cluster; ++i) {
                const float2 ml = tree_peer_f2(tree_peer(s_ml + r, i));
                if (ml.y == 0.f) continue;                    // (a piece that saw nothing has no O either)
                const float w = fast_exp2(ml.x - m_max);
                const float4 o = tree_peer_f4(tree_peer(s_part + r * C::PART_LD + c4, i));
                sum = fmaf(w, ml.y, sum);
                acc.x = fmaf(w, o.x, acc.x); acc.y = fmaf(w, o.y, acc.y);
                acc.z = fmaf(w, o.z, acc.z); acc.w = fmaf(w, o.w, acc.w);
            }
            const bool none = sum == 0.f;
            const float inv = none ? 0.f : 1.f / sum;
            const int64_t orow = ((int64_t)b * g.N + first_node + r / G) * g.a.H_q + kvh * G + r % G;
            *reinterpret_cast<uint2*>(reinterpret_cast<T*>(g.a.out) + orow * D + c4) =
                none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (c4 == 0) g.a.lse[orow] = none ? -INFINITY : (m_max + log2f(sum)) * LN2;
        }
        tree_cluster_barrier();                               // nobody leaves while its shared memory may be read
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;"
                     ::"r"((unsigned)*reinterpret_cast<volatile int*>(s_misc)), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
