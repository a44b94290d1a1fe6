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
// Measured (one call in a replayed sequence): 32 x 32 nodes, 32 heads, up to 4160 paged tokens: 193 us, 5.8 TB/s; 8 x 16
// nodes, 32 / 8 heads, up to 8190 tokens: 46 us, 4.4 TB/s (the longest sequence's blocks are waited for); 64 x 16
// nodes, window of 512: 152 us, 5.3 TB/s; 16 x 64 nodes, 64 / 8 heads: 126 us, 0.83 PFLOP/s; 1 x 4 nodes: 9.8 us.  The fourth
// is bound by the chain of a tile -- a softmax thread takes 1700 cycles for its 64 scores (64 exponentials at 4 a cycle and
// scheduler are 512 of them), the products 640 per block, and two blocks overlap but half of it -- and by the clock, which
// the power limit lowers to 1.7 GHz.  Two threads per row with half a tile each, and so 80 registers, were slower (154 us).
//
// A block handles 128 query rows (128 / G nodes) of one (request, kv head) and a range of its 64-token
// tiles.  Warps 4 and 6 copy K and V tiles into a ring of shared-memory slots each with tensor-map copies (boxes of
// 64 elements x as many tokens as a page holds in one piece, 128-byte swizzle; issuing a tile's copies from
// 16-token pages takes a warp some 700 cycles, and one warp for both fell behind), warp 5 issues the products,
// warps 0-3 own the 128 rows, one thread per row (32 TMEM lanes per warp): they read S = Q K^T from TMEM,
// keep the running maximum and sum, and write P = e^{x - m} back to TMEM as bf16, where it is the A
// operand of O += P V.  S is double buffered: S(j + 1) is computed while tile j's softmax runs.  Warps
// whose 32 rows do not exist sit out.  Warp 7 appends the nodes' rows to the cache meanwhile (by the softmax
// warps, before their first tile, that took 6 us of a 60 us block).  TMEM: 2 x 64 columns of S (P
// takes the place of the S it came from) + D of O, 256 allocated; two blocks share an SM, so one's set-up
// and last tile hide behind the other's.
//
// A block's set-up, its first copies and its results take some 10 us that nobody else uses on a short sequence.  So
// blocks are persistent: a running one takes over the next block that has not been launched yet (cluster launch
// control), its copying warp runs ahead into the next item, and the ring never drains.  Sequences differ in length,
// and a taken-over block goes to whoever is done first; the longest sequences go first (198 -> 194 us for 32 x 32 nodes; up
// to 256 requests, which a block puts in order itself), so that none of them is begun last and waited for alone.
//
// Where there are fewer blocks than places, the cached tokens are cut: the 2, 4 or 8 blocks of a thread-block cluster
// share the tiles of one (request, kv head) and merge their states through distributed shared memory, without partial
// results in HBM or a second launch.  Only where eight are too few (a long sequence under one or two heads) partial
// results go to the workspace and the combine kernel.
//
// The maximum that the exponentials are taken against trails the true one by at most 2^8 (it is replaced,
// and O rescaled, only when a row's maximum has grown beyond that): e^{x - m} then reaches at most 256,
// which fp32 sums and bf16 P hold as well as 1.  Sums are fp32 over the unrounded P; P is rounded to bf16
// (relative error up to 2^-8 per weight, averaging out over the row) because the tensor-core product takes
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
constexpr int kTreeSorted = 256;                   // requests, at most, that a block puts in order (one per thread)

struct TreeArgs {
    AttnArgs a;                                    // lengths, block table, strides, scale, outputs
    const int* parent;                             // [B, N] or NULL (a chain)
    const int* node_count;                         // [B] or NULL (N)
    int batch, N, G, g_shift;                      // G: a power of two
    int row_tiles;                                 // blocks of kTreeRows query rows per (request, kv head)
    int windowed;                                  // 0: dense
    int box_tokens;                                // tokens per tensor-map box of the caches
    int box_shift;                                 // and its logarithm
    unsigned page_mul;                             // position / block_size = (position * page_mul) >> page_shift
    int page_shift;
    int align_tokens;                              // where a box may start: box_tokens (pages), 1 (contiguous)
    int cluster;                                   // blocks that share the tiles and merge on chip (1: none; else n_split is 1)
    int sorted;                                    // requests are taken in the order of their tiles, most first
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
    static constexpr int K_SLOTS = D == 128 ? 3 : 5, V_SLOTS = D == 128 ? 2 : 5;   // two blocks per SM with either
    static constexpr int SLOTS = K_SLOTS + V_SLOTS;
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
// Shared-memory operand descriptors, 128-byte swizzle: atoms of 8 rows x 128 bytes, 1024 bytes from one to the next
// along the rows; `lead`: bytes from one 64-element column block to the next, where the 64 contiguous elements run
// along N and the operand is wider than they are.  The upper half is the same for all of them.
constexpr unsigned kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ unsigned desc_low(unsigned addr, unsigned lead) { return ((addr >> 4) & 0x3fffu) | ((lead >> 4) << 16); }
// Instruction descriptor: bf16 x bf16 -> fp32, M x N; b_mn: B's contiguous dimension is N, not K.
__host__ __device__ constexpr unsigned instr_desc(int M, int N, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((unsigned)(N >> 3) << 17) |
           ((unsigned)(M >> 4) << 24);
}
// D[tmem] (+)= A[smem] B[smem]^T
__device__ __forceinline__ void tc_mma_ss(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"((unsigned)acc), "r"(kDescHigh) : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]^T
__device__ __forceinline__ void tc_mma_ts(unsigned d, unsigned a, unsigned b_low, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}"
                 ::"r"(d), "r"(a), "r"(b_low), "r"(idesc), "r"((unsigned)acc), "r"(kDescHigh) : "memory");
}
// one lane of the warp, the same every time (products and their commits come from one thread)
__device__ __forceinline__ bool elect_one() {
    unsigned yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes != 0;
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
        s.lo_al = s.lo & -g.align_tokens;                                   // (a power of two)
    }
    s.T1 = (s.P0 + kTreeTile - 1) / kTreeTile;
    s.T = s.T1 + (S - s.lo_al + kTreeTile - 1) / kTreeTile;
    if (s.lo >= S) s.T = s.T1;
    return s;
}

// K / V rows of the nodes first, first + step, ... below n, kv head kvh, to the cache, by one warp: every lane looks up
// one node's place (-1: it has no page, and its rows are dropped), then the rows are copied eight 512-byte steps at a time.
template <typename T, int D>
__device__ __forceinline__ void tree_append(const TreeArgs& g, int b, int kvh, int S, int L_p, int first, int step, int n, int lane) {
    constexpr int VEC = 16 / (int)sizeof(T), CPR = D / VEC, PAIR = 2 * CPR;        // 16-byte pieces of a K and a V row
    for (int base = first; base < n; base += 32 * step) {
        const int64_t node0 = (int64_t)b * g.N + base;
        const int count = min(32, (n - base + step - 1) / step);
        const int pos = S + base + lane * step;
        const int64_t place = lane < count && token_has_page(g.a, b, pos) ? token_offset(g.a, b, L_p, pos) + (int64_t)kvh * g.a.stride_head : -1;
        for (int i0 = 0; i0 < count * PAIR; i0 += 8 * 32) {
            uint4 x[8];
            int64_t dst[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + 32 * j + lane, r = i / PAIR, c = i % CPR * VEC;
                const int64_t at = __shfl_sync(0xffffffffu, place, min(r, 31));
                dst[j] = at < 0 ? -1 : at + c;
                if (r < count)
                    x[j] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(i % PAIR < CPR ? g.a.k_new : g.a.v_new) +
                                                           ((node0 + r * step) * g.a.H_kv + kvh) * D + c);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + 32 * j + lane;
                if (i / PAIR < count && dst[j] >= 0)
                    *reinterpret_cast<uint4*>(reinterpret_cast<T*>(const_cast<void*>(i % PAIR < CPR ? g.a.k : g.a.v)) + dst[j]) = x[j];
            }
        }
    }
}

// Rows [r0, r1) of a block's query rows (row r: node first_node + r / G, head kvh * G + r % G) have nothing to
// attend to in this split: zeros and -inf, or an empty part for the combine.
template <typename T, int D>
__device__ __forceinline__ void tree_write_empty(const TreeArgs& g, int b, int kvh, int split, int first_node, int r0, int r1,
                                                 int tid, int count) {
    for (int r = r0 + tid; r < r1; r += count) {
        const int64_t row = ((int64_t)b * g.N + first_node + (r >> g.g_shift)) * g.a.H_q + kvh * g.G + (r & (g.G - 1));
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

// two floats in one instruction (each rounded on its own)
__device__ __forceinline__ unsigned long long pack_f32x2(float lo, float hi) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpack_f32x2(unsigned long long v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ unsigned long long fma_f32x2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add_f32x2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// ---- dynamic scheduling: a running block takes over blocks that have not been launched yet --------------------
__device__ __forceinline__ void steal_block(void* response, unsigned long long* bar) {      // one thread
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");            // (the last response has been read)
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(smem_u32(response)), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ int stolen_block(const void* response) {         // its index, or -1: there is none any more
    unsigned ok;
    int x;
    asm volatile("{\n.reg .b128 r;\n.reg .pred p;\n"
                 "ld.shared.b128 r, [%2];\n"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
                 "selp.u32 %0, 1, 0, p;\n"
                 "mov.b32 %1, 0;\n"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
                 : "=r"(ok), "=r"(x) : "r"(smem_u32(response)) : "memory");
    return ok ? x : -1;
}

// What a block works on: the piece `piece` of the tiles that the nodes of row tile `rt` of (b, kvh) see.
struct TreeItem {
    int index, b, kvh, rt, piece, S, L_p, n;                  // index < 0: nothing any more
};
// Its tiles: [t0, t0 + cached) of the request's, then (has_nodes) the nodes' own rows.
struct TreeWork {
    TreeSpan span;
    int t0, cached, tiles, first_node;
    int rows_all, rows;                                       // rows that the block writes; rows of nodes that exist
};
struct TreeInfo {
    TreeItem item;
    TreeWork work;
    signed char up[kTreeMaxNodes];                            // parents of the nodes, -1: a root
};

template <int D>
__global__ void __launch_bounds__(kTreeThreads, 2) dsa_tree_kernel(const TreeArgs g, const __grid_constant__ TreeMaps maps) {
    using C = TreeCfg<D>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + C::Q_BYTES + C::SLOTS * C::SLOT_BYTES);
    unsigned char* s_vring = s_ring + C::K_SLOTS * C::SLOT_BYTES;
    unsigned long long* k_full = bars;                        // a ring slot has landed
    unsigned long long* v_full = bars + C::K_SLOTS;
    unsigned long long* k_empty = bars + C::SLOTS;            // the products that read it are done
    unsigned long long* v_empty = k_empty + C::K_SLOTS;
    unsigned long long* s_full = bars + 2 * C::SLOTS;         // [2] scores are in TMEM
    unsigned long long* p_ready = s_full + 2;                 // [2] weights are in TMEM
    unsigned long long* pv_done = s_full + 4;                 // [2] O holds the tile
    unsigned long long* info_full = s_full + 6;               // [2] the next item is known
    unsigned long long* info_empty = s_full + 8;              // [2] every warp has read it
    unsigned long long* q_full = s_full + 10;                 // q has landed
    unsigned long long* q_empty = s_full + 11;                // the scores of an item's last tile are done
    unsigned long long* o_free = s_full + 12;                 // O has been read
    unsigned long long* stolen = s_full + 13;
    uint4* s_response = reinterpret_cast<uint4*>(s_full + 14);
    unsigned long long* drained = s_full + 16;
    TreeInfo* s_info = reinterpret_cast<TreeInfo*>(s_full + 17);                 // [2]
    int* s_misc = reinterpret_cast<int*>(s_info + 2);         // [0] TMEM address, [1] abort
    unsigned char* s_order = reinterpret_cast<unsigned char*>(s_misc + 2);       // [kTreeSorted] requests, most tiles first
    static_assert((2 * C::SLOTS + 17) * 8 + 2 * sizeof(TreeInfo) + 8 + kTreeSorted <= C::TAIL, "tail of the shared memory");
    static_assert((2 * C::SLOTS) % 2 == 0, "the response lies on 16 bytes");
    volatile int* abort = s_misc + 1;
    // after the last product, for a merge within the cluster: O (rows padded against bank conflicts) and per row
    // (maximum in base-2 units, sum)
    float* s_part = reinterpret_cast<float*>(s_ring);
    float2* s_ml = reinterpret_cast<float2*>(s_q);
    static_assert(kTreeRows * C::PART_LD * 4 <= C::SLOTS * C::SLOT_BYTES, "the partial result takes the ring's place");

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int pieces = g.cluster * g.a.n_split;               // (one of the two is 1)
    const int G = g.G, per_tile = kTreeRows >> g.g_shift;

    // set-up that reads nothing: it may run while the launch in front finishes
    if (warp == 4 && lane == 0) {
        for (int s = 0; s < 2 * C::SLOTS; ++s) mbar_init(bars + s, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
            mbar_init(info_full + s, 1); mbar_init(info_empty + s, 7);
        }
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(o_free, 4);
        mbar_init(stolen, 1); mbar_init(drained, 1);
        s_misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_fence_before();
    }
    // Rows of q that no copy fills: zeros.  Nobody reads their results, but what the products multiply there costs power
    // and so clock (64 x 16 nodes with a window, over and over: 164 us with leftovers, 156 with zeros).
    {
        const int filled = min(per_tile, g.N) * G * 8;        // 16-byte pieces of a half
        for (int i = filled + tid; i < kTreeRows * 8; i += kTreeThreads)
#pragma unroll
            for (int h = 0; h < C::HALVES; ++h) *reinterpret_cast<uint4*>(s_q + h * C::Q_HALF + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    if (g.sorted) {
        // the place of request `tid` among all of them (a request's tiles and its index make a key; nothing has come yet)
        unsigned* s_key = reinterpret_cast<unsigned*>(s_ring);
        unsigned key = 0;
        if (tid < g.batch) {
            int S, L_p, n;
            tree_lengths(g, tid, S, L_p, n);
            key = ((n > 0 ? (unsigned)min(tree_span(g, S, L_p).T, 0x3fffff) + 1u : 0u) << 8) | (255u - (unsigned)tid);
        }
        s_key[tid] = key;
        __syncthreads();
        int before = 0;
        for (int j = 0; j < g.batch; j += 4) {
            const uint4 other = *reinterpret_cast<const uint4*>(s_key + j);      // (behind the last request: 0)
            before += (other.x > key) + (other.y > key) + (other.z > key) + (other.w > key);
        }
        if (tid < g.batch) s_order[before] = (unsigned char)tid;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // (tiles are copied to where the keys were)
        __syncthreads();
    }

    // the item number `i` of this block, once the copying warp has found it; false: there is none, or give up
    TreeItem it = {};
    TreeWork w = {};
    auto next_item = [&](int i) -> bool {
        if (!tree_wait(info_full + (i & 1), (i >> 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
        it = s_info[i & 1].item;
        w = s_info[i & 1].work;
        return it.index >= 0;
    };
    auto item_read = [&](int i) {                             // this warp needs item i's description no longer
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty + (i & 1));
    };

    // ---- copies of K and V tiles -------------------------------------------------------------------------
    // A tile is 64 >> box_shift boxes of HALVES pieces; piece p = box * HALVES + half is copied by lane p % 32.
    // Where this lane's pieces of a tile come from: (page or request, token in it), looked up tiles ahead of the copies.
    constexpr int PIECES = kTreeTile * C::HALVES / 32;        // per lane, with boxes of one token
    struct Where { int blk[PIECES], tok[PIECES]; };
    const int n_pieces = (kTreeTile >> g.box_shift) * C::HALVES;
    auto where = [&](int t, Where& r) {
        int start = 0, from, to;
        if (t < w.cached) w.span.tile(w.t0 + t, start, from, to);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (k > 0 && 32 * k >= n_pieces) break;
            const int box = (lane + 32 * k) / C::HALVES;
            const int pos = start + (box << g.box_shift);
            r.blk[k] = g.blk_coord ? it.b : 0;
            r.tok[k] = pos;
            if (g.a.block_table) {
                const int bi = (int)(((unsigned long long)(unsigned)pos * g.page_mul) >> g.page_shift);
                r.tok[k] = pos - bi * g.a.block_size;
                // (as the table has it: put into range when the copy is made, so that nobody waits for it here)
                if (t < w.cached && (box << g.box_shift) < kTreeTile)
                    r.blk[k] = g.a.block_table[(int64_t)it.b * g.a.max_blocks + min(bi, g.a.max_blocks - 1)];
            }
        }
    };
    auto copy_tile = [&](int t, const Where& r, const CUtensorMap* cached_map, const CUtensorMap* new_map, unsigned char* dst,
                         unsigned long long* bar) {
        if (t < w.cached) {
            int start, from, to;
            w.span.tile(w.t0 + t, start, from, to);
            const int j0 = (from - start) >> g.box_shift, j1 = (to - start + (1 << g.box_shift) - 1) >> g.box_shift;
            if (lane == 0) mbar_expect_tx(bar, (unsigned)(((j1 - j0) * C::HALVES) << g.box_shift) * 128u);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                if (k > 0 && 32 * k >= n_pieces) break;
                const int box = (lane + 32 * k) / C::HALVES, h = lane % C::HALVES;
                if (box < j0 || box >= j1) continue;
                const int blk = g.a.block_table ? max(0, min(r.blk[k], g.a.num_blocks - 1)) * g.blk_coord : r.blk[k];
                tma_box4(dst + h * C::KV_HALF + ((box << g.box_shift) * 128), cached_map, 64 * h, r.tok[k], it.kvh * g.head_coord, blk, bar);
            }
        } else {
            if (lane == 0) mbar_expect_tx(bar, (unsigned)(C::HALVES * g.N * 128));
            __syncwarp();
            if (lane < C::HALVES) tma_box4(dst + lane * C::KV_HALF, new_map, 64 * lane, 0, it.kvh, it.b, bar);
        }
        __syncwarp();
    };
    // a ring of `slots` slots: the next one, free again
    struct Ring { int slot, round, issued; };
    auto next_free = [&](Ring& ring, unsigned long long* empty) -> bool {
        return ring.round == 0 || tree_wait(empty + ring.slot, (ring.round - 1) & 1, abort, g.a.wait_timeouts, lane);
    };
    auto advance = [&](Ring& ring, int slots) {
        ++ring.issued;
        if (++ring.slot == slots) { ring.slot = 0; ++ring.round; }
    };
    // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
    auto drain = [&](const Ring& ring, unsigned long long* full, int slots) {
        volatile int no_abort = 0;
        for (int c = max(0, ring.issued - slots); c < ring.issued; ++c)
            if (!tree_wait(full + c % slots, (c / slots) & 1, &no_abort, nullptr, lane)) break;
    };

    float m_ref = -INFINITY, l = 0.f;                         // softmax threads: maximum (of the raw scores) and sum of their row
    if (warp == 4) {
        // ---- what to work on; copies of q and K -----------------------------------------------------
        Ring ring = {0, 0, 0};
        bool ok = true;
        int live = 0;                                         // items with tiles so far
        it.index = (int)blockIdx.x;
        for (int i = 0; ok; ++i) {
            int up[2] = {-1, -1};                             // parents of the nodes lane and lane + 32
            if (it.index >= 0) {
                int idx = it.index;
                it.piece = idx % pieces; idx /= pieces;
                it.rt = idx % g.row_tiles; idx /= g.row_tiles;
                it.kvh = idx % g.a.H_kv;
                it.b = g.sorted ? s_order[idx / g.a.H_kv] : idx / g.a.H_kv;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int node = lane + 32 * h;
                    if (node < g.N) up[h] = g.parent ? g.parent[(int64_t)it.b * g.N + node] : node - 1;
                    if (up[h] >= node) up[h] = -1;
                }
                tree_lengths(g, it.b, it.S, it.L_p, it.n);
            }
            if (i >= 2) ok = tree_wait(info_empty + (i & 1), ((i >> 1) - 1) & 1, abort, g.a.wait_timeouts, lane);
            if (!ok) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) s_info[i & 1].up[lane + 32 * h] = (signed char)max(up[h], -1);
            if (it.index >= 0) {
                w.first_node = it.rt * per_tile;
                w.rows_all = min(per_tile, g.N - w.first_node) << g.g_shift;
                w.rows = max(0, min(per_tile, it.n - w.first_node)) << g.g_shift;
                w.span = tree_span(g, it.S, it.L_p);
                const int per_piece = pieces > 1 ? (w.span.T + pieces - 1) / pieces : w.span.T;
                w.t0 = min(w.span.T, it.piece * per_piece);
                w.cached = min(w.span.T, w.t0 + per_piece) - w.t0;
                w.tiles = w.rows == 0 ? 0 : w.cached + (it.piece == 0 ? 1 : 0);
            }
            if (lane == 0) { s_info[i & 1].item = it; s_info[i & 1].work = w; }
            __syncwarp();
            if (lane == 0) mbar_arrive(info_full + (i & 1));
            if (it.index < 0) break;
            // the next item is taken over when this one's copies are nearly all on their way: late, so that it goes to
            // whoever has room for it, but early enough to know its lengths and pages in time
            bool asked = g.cluster > 1;
            auto ask = [&]() {
                if (!asked && lane == 0) steal_block(s_response, stolen);
                asked = true;
            };
            if (w.tiles > 0) {
                Where r0, r1, r2;
                where(0, r0);
                where(1, r1);
                if (live > 0) ok = tree_wait(q_empty, (live - 1) & 1, abort, g.a.wait_timeouts, lane);
                if (ok && lane == 0) {
                    const int box_nodes = min(per_tile, g.N);
                    mbar_expect_tx(q_full, (unsigned)(C::HALVES * box_nodes * G * 128));
                    for (int h = 0; h < C::HALVES; ++h) tma_box4(s_q + h * C::Q_HALF, &maps.q, 64 * h, it.kvh * G, w.first_node, it.b, q_full);
                }
                __syncwarp();
                if (ok) ++live;
                for (int t = 0; ok && t < w.tiles; ++t) {
                    if (t + 3 >= w.tiles) ask();
                    where(t + 2, r2);
                    ok = next_free(ring, k_empty);
                    if (!ok) break;
                    copy_tile(t, r0, &maps.k, &maps.k_new, s_ring + ring.slot * C::SLOT_BYTES, k_full + ring.slot);
                    advance(ring, C::K_SLOTS);
                    r0 = r1;
                    r1 = r2;
                }
            }
            ask();
            it.index = -1;
            if (g.cluster == 1) {
                volatile int no_abort = 0;                    // (the response is waited for whatever else has happened)
                if (tree_wait(stolen, i & 1, &no_abort, g.a.wait_timeouts, lane)) it.index = stolen_block(s_response);
                else { *abort = 1; ok = false; }
            }
        }
        volatile int no_abort = 0;
        if (live > 0) tree_wait(q_full, (live - 1) & 1, &no_abort, nullptr, lane);
        drain(ring, k_full, C::K_SLOTS);
    } else if (warp == 6) {
        // ---- copies of V ----------------------------------------------------------------------------
        Ring ring = {0, 0, 0};
        bool ok = true;
        for (int i = 0; ok && next_item(i); ++i) {
            item_read(i);
            if (w.tiles == 0) continue;
            Where r0, r1, r2;
            where(0, r0);
            where(1, r1);
            for (int t = 0; t < w.tiles; ++t) {
                where(t + 2, r2);
                ok = next_free(ring, v_empty);
                if (!ok) break;
                copy_tile(t, r0, &maps.v, &maps.v_new, s_vring + ring.slot * C::SLOT_BYTES, v_full + ring.slot);
                advance(ring, C::V_SLOTS);
                r0 = r1;
                r1 = r2;
            }
        }
        drain(ring, v_full, C::V_SLOTS);
    } else if (warp == 7) {
        // ---- the nodes' rows to the cache: every block those of its own nodes, the pieces in turn ----------------
        for (int i = 0; next_item(i); ++i) {
            item_read(i);
            const int first = it.rt * per_tile;
            tree_append<T, D>(g, it.b, it.kvh, it.S, it.L_p, first + it.piece, pieces, min(it.n, first + per_tile), lane);
        }
    } else if (warp == 5) {
        // ---- products ---------------------------------------------------------------------------
        constexpr unsigned kIdescS = instr_desc(kTreeRows, kTreeTile, false), kIdescO = instr_desc(kTreeRows, D, true);
        const unsigned q_desc = desc_low(smem_u32(s_q), 16), k_desc = desc_low(smem_u32(s_ring), 16);
        const unsigned v_desc = desc_low(smem_u32(s_vring), C::KV_HALF);
        int k_slot = 0, k_round = 0, v_slot = 0, v_round = 0;  // of the rings
        int done = 0;                                         // tiles of the items before this one
        auto scores = [&](int t) -> bool {
            const int s = k_slot, buf = (done + t) & 1;
            if (!tree_wait(k_full + s, k_round & 1, abort, g.a.wait_timeouts, lane)) return false;
            tc_fence_after();
            if (elect_one()) {
                const unsigned qa = q_desc, ka = k_desc + s * (C::SLOT_BYTES / 16), d = tmem + C::COL_S + buf * kTreeTile;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    tc_mma_ss(d, qa + ((kk / 4) * C::Q_HALF + (kk % 4) * 32) / 16, ka + ((kk / 4) * C::KV_HALF + (kk % 4) * 32) / 16,
                              kIdescS, kk > 0);
                tc_commit(k_empty + s);
                tc_commit(s_full + buf);
                if (t == w.tiles - 1) tc_commit(q_empty);
            }
            __syncwarp();
            if (++k_slot == C::K_SLOTS) { k_slot = 0; ++k_round; }
            return true;
        };
        auto values = [&](int t) -> bool {
            const int gt = done + t, buf = gt & 1;
            if (!tree_wait(p_ready + buf, (gt >> 1) & 1, abort, g.a.wait_timeouts, lane)) return false;
            const int s = v_slot;
            if (!tree_wait(v_full + s, v_round & 1, abort, g.a.wait_timeouts, lane)) return false;
            unsigned char* v = s_vring + s * C::SLOT_BYTES;
            // rows of V that nobody sees: zero, whatever the cache or the slot held there
            int lo = 0, hi = it.n;
            if (t < w.cached) {
                int start;
                w.span.tile(w.t0 + t, start, lo, hi);
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
            if (elect_one()) {
                const unsigned va = v_desc + s * (C::SLOT_BYTES / 16), pa = tmem + C::COL_S + buf * kTreeTile;
#pragma unroll
                for (int kk = 0; kk < kTreeTile / 16; ++kk)
                    tc_mma_ts(tmem + C::COL_O, pa + kk * 8, va + kk * (2048 / 16), kIdescO, t > 0 || kk > 0);
                tc_commit(v_empty + s);
                tc_commit(pv_done + buf);
            }
            __syncwarp();
            if (++v_slot == C::V_SLOTS) { v_slot = 0; ++v_round; }
            return true;
        };
        int live = 0;
        bool ok = true;
        for (int i = 0; next_item(i); ++i) {
            item_read(i);
            if (w.tiles == 0) continue;
            ok = tree_wait(q_full, live & 1, abort, g.a.wait_timeouts, lane) && scores(0) && (w.tiles < 2 || scores(1));
            // (the first product of P and V replaces the last item's O)
            if (ok && live > 0) ok = tree_wait(o_free, (live - 1) & 1, abort, g.a.wait_timeouts, lane);
            for (int t = 0; ok && t < w.tiles; ++t) ok = values(t) && (t + 2 >= w.tiles || scores(t + 2));
            if (!ok) break;
            done += w.tiles;
            ++live;
        }
        if (__any_sync(0xffffffffu, !ok || *abort)) {         // TMEM is given back only when no product uses it
            if (elect_one()) tc_commit(drained);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained, 0u, &no_abort, nullptr, lane);
        }
    } else {
        // ---- softmax: one thread per query row --------------------------------------------------
        const int row = tid;                                  // of the block's 128
        const unsigned lane_base = (unsigned)(warp * 32) << 16;
        const float sl = g.a.scale_log2;
        int done = 0;                                         // tiles of the items before this one
        bool ok = true;
        for (int i = 0; ok && next_item(i); ++i) {
            m_ref = -INFINITY;
            l = 0.f;
            const bool work = w.tiles > 0 && warp * 32 < w.rows;     // a warp without rows only keeps step
            const int node = w.first_node + (row >> g.g_shift);
            const bool alive = row < w.rows;                  // (a row that does not exist computes along, unmasked, and decides nothing)
            unsigned long long own = alive ? 0ull : ~0ull;    // drafted tokens that the row's node sees
            int64_t win_lo = INT64_MIN;                       // and where the window begins (dense: everything is in [0, P0))
            if (work && alive) {
                const signed char* up = s_info[i & 1].up;
                int depth = 0;                                // (ancestors of a node that exists exist)
                for (int j = node; j >= 0; j = up[j], ++depth) own |= 1ull << j;
                --depth;
                win_lo = (int64_t)it.S + depth + 1 - g.a.mask.window;
                if (g.windowed) {
                    // tokens of the own line that the window has left behind (sinks stay): `back` positions behind
                    const int64_t sinks = (int64_t)it.L_p + g.a.mask.n_sink - it.S;       // depths below this are sinks
                    int back = 0;
                    for (int j = node; j >= 0; j = up[j], ++back)
                        if (back >= g.a.mask.window && depth - back >= sinks) own &= ~(1ull << j);
                }
            }
            item_read(i);
            if (w.tiles == 0) {
                if (g.cluster == 1) tree_write_empty<T, D>(g, it.b, it.kvh, it.piece, w.first_node, 0, w.rows_all, tid, 128);
                continue;
            }
            for (int t = 0; ok && t < w.tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                ok = tree_wait(s_full + buf, (gt >> 1) & 1, abort, g.a.wait_timeouts, lane);
                if (!ok) break;
                if (!work) {
                    if (lane == 0) mbar_arrive(p_ready + buf);
                    continue;
                }
                tc_fence_after();
                const unsigned s_addr = tmem + lane_base + C::COL_S + buf * kTreeTile;
                unsigned x0[32], x1[32];
                tc_ld32(x0, s_addr);
                tc_ld32(x1, s_addr + 32);
                unsigned long long see;
                if (t < w.cached) {
                    int start, from, to;
                    w.span.tile(w.t0 + t, start, from, to);
                    int c0 = 0, c1 = to - start;
                    if (w.t0 + t >= w.span.T1) c0 = (int)max((int64_t)from, min((int64_t)to, win_lo)) - start;
                    see = c1 >= 64 ? ~0ull : (1ull << c1) - 1ull;
                    see = c0 >= 64 ? 0ull : (c0 > 0 ? (see >> c0) << c0 : see);
                } else {
                    see = own;
                }
                tc_wait_ld();
                if (__any_sync(0xffffffffu, see != ~0ull)) {
                    const unsigned lo = (unsigned)see, hi = (unsigned)(see >> 32);
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        if (!((lo >> k) & 1u)) x0[k] = 0xff800000u;
                        if (!((hi >> k) & 1u)) x1[k] = 0xff800000u;
                    }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 32; k += 4)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {             // (maxima of three)
                        mx[h] = fmaxf(fmaxf(mx[h], __uint_as_float(x0[k + 2 * h])), __uint_as_float(x0[k + 2 * h + 1]));
                        mx[2 + h] = fmaxf(fmaxf(mx[2 + h], __uint_as_float(x1[k + 2 * h])), __uint_as_float(x1[k + 2 * h + 1]));
                    }
                const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                // (-inf - -inf is NaN: compares false, nothing to rescale)
                if (__any_sync(0xffffffffu, alive && (m_tile - m_ref) * sl > 8.f)) {
                    const float m_new = fmaxf(m_ref, m_tile);
                    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m_ref - m_new) * sl);
                    m_ref = m_new;
                    l *= alpha;
                    if (t > 0) {
                        ok = tree_wait(pv_done + ((gt - 1) & 1), ((gt - 1) >> 1) & 1, abort, g.a.wait_timeouts, lane);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            unsigned o[32];
                            tc_ld32(o, tmem + lane_base + C::COL_O + c);
                            tc_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tc_st32(tmem + lane_base + C::COL_O + c, o);
                        }
                    }
                }
                const float sub = m_ref == -INFINITY ? 0.f : m_ref * sl;
                const unsigned long long sl2 = pack_f32x2(sl, sl), sub2 = pack_f32x2(-sub, -sub);
                unsigned long long sum[2] = {0ull, 0ull};
                unsigned pk[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const unsigned a0 = k < 16 ? x0[2 * k] : x1[2 * k - 32], a1 = k < 16 ? x0[2 * k + 1] : x1[2 * k - 31];
                    const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(a0), __uint_as_float(a1)), sl2, sub2));
                    const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                    sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                    pk[k] = pack_bf16(p0, p1);
                }
                const float2 both = unpack_f32x2(add_f32x2(sum[0], sum[1]));
                l += both.x + both.y;
                tc_st32(s_addr, pk);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready + buf);
            }
            if (!ok) break;
            done += w.tiles;
            ok = tree_wait(pv_done + ((done - 1) & 1), ((done - 1) >> 1) & 1, abort, g.a.wait_timeouts, lane);
            tc_fence_after();
            if (g.cluster > 1) break;                         // (one item, merged below)
            // ---- results ------------------------------------------------------------------------
            if (work) {
                const bool mine = ok && row < w.rows_all;
                const bool none = !alive || l == 0.f;          // nothing seen: zeros and -inf
                const float inv = none ? 0.f : 1.f / l;
                const int64_t orow = ((int64_t)it.b * g.N + node) * g.a.H_q + it.kvh * G + (row & (G - 1));
                const float lse = none ? -INFINITY : (m_ref * sl + log2f(l)) * LN2;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned o[32];
                    tc_ld32(o, tmem + lane_base + C::COL_O + c);
                    tc_wait_ld();
                    if (mine) {
                        float f[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) f[k] = none ? 0.f : __uint_as_float(o[k]) * inv;
                        if (g.a.n_split > 1) {
                            float* dst = g.a.out_part + (orow * g.a.n_split + it.piece) * D + c;
#pragma unroll
                            for (int k = 0; k < 32; k += 4)
                                *reinterpret_cast<float4*>(dst + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
                        } else {
                            T* dst = reinterpret_cast<T*>(g.a.out) + orow * D + c;
#pragma unroll
                            for (int k = 0; k < 32; k += 8)
                                *reinterpret_cast<uint4*>(dst + k) = make_uint4(pack_bf16(f[k], f[k + 1]), pack_bf16(f[k + 2], f[k + 3]),
                                                                                pack_bf16(f[k + 4], f[k + 5]), pack_bf16(f[k + 6], f[k + 7]));
                        }
                    }
                    __syncwarp();
                }
                tc_fence_before();
                if (mine) {
                    if (g.a.n_split > 1) g.a.lse_part[orow * g.a.n_split + it.piece] = lse;
                    else g.a.lse[orow] = lse;
                }
            } else {
                // rows of nodes that do not exist, beyond the last warp with rows
                const int first = (w.rows + 31) / 32 * 32;
                tree_write_empty<T, D>(g, it.b, it.kvh, it.piece, w.first_node, first, w.rows_all, tid - first, 128 - first);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
        }
    }
    __syncthreads();                                          // (every role has come to its end)
    if (g.cluster > 1) {
        // ---- merge: out = sum_i e^{m_i - M} O_i / sum_i e^{m_i - M} l_i over the cluster's blocks --------------
        it = s_info[0].item;
        w = s_info[0].work;
        if (warp < 4) {
            const bool none = tid >= w.rows || l == 0.f;
            s_ml[tid] = none ? make_float2(-INFINITY, 0.f) : make_float2(m_ref * g.a.scale_log2, l);
            if (w.tiles > 0 && warp * 32 < w.rows) {
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned o[32];
                    tc_ld32(o, tmem + ((unsigned)(warp * 32) << 16) + C::COL_O + c);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<uint4*>(s_part + tid * C::PART_LD + c + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                }
                tc_fence_before();
            }
        }
        tree_cluster_barrier();
        constexpr int LPR = D / 4, RPW = 32 / LPR;            // lanes per row (four dims each), rows per warp
        const int sub = lane / LPR, c4 = (lane % LPR) * 4;
        for (int r = it.piece + (warp * RPW + sub) * g.cluster; r < w.rows_all; r += 8 * RPW * g.cluster) {
            float m_max = -INFINITY;
            for (int i = 0; i < g.cluster; ++i) m_max = fmaxf(m_max, tree_peer_f2(tree_peer(s_ml + r, i)).x);
            float sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int i = 0; i < g.cluster; ++i) {
                const float2 ml = tree_peer_f2(tree_peer(s_ml + r, i));
                if (ml.y == 0.f) continue;                    // (a piece that saw nothing has no O either)
                const float wt = fast_exp2(ml.x - m_max);
                const float4 o = tree_peer_f4(tree_peer(s_part + r * C::PART_LD + c4, i));
                sum = fmaf(wt, ml.y, sum);
                acc.x = fmaf(wt, o.x, acc.x); acc.y = fmaf(wt, o.y, acc.y);
                acc.z = fmaf(wt, o.z, acc.z); acc.w = fmaf(wt, o.w, acc.w);
            }
            const bool none = sum == 0.f;
            const float inv = none ? 0.f : 1.f / sum;
            const int64_t orow = ((int64_t)it.b * g.N + w.first_node + (r >> g.g_shift)) * g.a.H_q + it.kvh * G + (r & (G - 1));
            *reinterpret_cast<uint2*>(reinterpret_cast<T*>(g.a.out) + orow * D + c4) =
                none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (c4 == 0) g.a.lse[orow] = none ? -INFINITY : (m_max + log2f(sum)) * LN2;
        }
        tree_cluster_barrier();                               // nobody leaves while its shared memory may be read
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
