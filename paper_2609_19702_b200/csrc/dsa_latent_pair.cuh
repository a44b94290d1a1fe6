// Attention of new tokens over a latent cache, bf16, more than 64 query rows (dsa_latent_step): two blocks, one product.
//
// The mathematics of dsa_latent.cuh with M = 128: 64 query rows in either block of a cluster of two, tiles of 128 keys.  What
// bounds blocks of 64 rows here is that every SM reads every key for half the rows that a product can have, and takes the
// tensor pipe twice as long as M = 128 does (N 64 at 33 cycles for 64 rows; the pair form, N 128 at 33 for 128).  In the pair
// form each block brings half of B: for S half of the keys, all of their columns; for O += W V half of the dims, of all keys.  So
// a block copies its own 64 keys whole, and once the scores are done, fetches the other block's keys again (from L2) for its
// half of the dims only, into the columns of its own keys that the other half of the dims took.  A block's shared memory sees
// 3 / 2 of its keys' bytes that way, against 2 / 1 with a block for each half of the rows.
//
// Measured: 32 requests x 128 heads, lengths 1024 to 8190 (179 MB of rows, 28 us at the measured copy rate; 41 GFLOP, 24 at
// the matrix rate): 61 us, with blocks of 64 rows 77.  16 x 128 heads with up to four tokens: 50 us, and 57.  Copies by threads, as the
// blocks of 64 rows have them, take 74 here: their arrivals have to be passed on to the other block.  A tile takes as long as
// its chain of landing, scores, softmax, the other keys' values, products: two tiles in flight are all that fits beside q,
// and do not cover all of it.
#pragma once
#include "dsa_latent.cuh"

namespace dsa {

constexpr int kPairTile = 128;                     // tokens per tile: 64 a block
constexpr int kPairRows = 128;                     // query rows per item: 64 a block
constexpr int kPairThreads = 256;

template <int R>
struct PairCfg {
    using W = LatentCfg<R>;
    static constexpr int P2_BYTES = kLatRows * 128;                        // weights of the tile's second half
    static constexpr int SMEM = W::Q_BYTES + W::SLOTS * W::SLOT + P2_BYTES + W::TAIL;
    static constexpr int COL_S = R / 2, TMEM_COLS = R == 512 ? 512 : 256;  // 2 x 64 columns of S behind O
    static_assert(COL_S + 2 * 64 <= TMEM_COLS, "tensor memory");
    static_assert(SMEM <= 232448, "shared memory of an SM");
};

// On a barrier of either block.  The release has block scope, the default: what an arrival hands over (weights, zeroed rows,
// scores and O that have been read) lies in this block's own shared and tensor memory, and no thread of the other block loads it.
// Its products do, in this SM and by the asynchronous proxy, and the proxy or tcgen05 fence in front of the arrival orders the
// writes (or reads) before them.  Nothing in global memory is handed over, and that is what a release at cluster scope waits
// for: 1300 cycles, 32 x 128 heads 79 us instead of 65.
__device__ __forceinline__ void pair_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// a copy to this block's shared memory that completes on a barrier of either block
__device__ __forceinline__ void pair_box3(void* dst, const CUtensorMap* map, int c0, int c1, int c2, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
// Where the 64 cached tokens from position `pos` on lie, as far as a lane sees to it: of box `lane` (page or request, token in
// it).  Looked up tiles ahead of the copies.
struct PairWhere {
    int blk, tok;
};
__device__ __forceinline__ PairWhere pair_where(const LatentTcArgs& g, int b, int pos, bool cached, int lane) {
    const AttnArgs& a = g.l.a;
    PairWhere w = {g.blk_coord ? b : 0, pos + (lane << g.box_shift)};
    if (a.block_table) {
        const int bi = (int)(((unsigned long long)(unsigned)w.tok * g.page_mul) >> g.page_shift);
        w.tok -= bi * a.block_size;
        // (as the table has it: put into range when the copy is made, so that nobody waits for it here)
        if ((lane << g.box_shift) < kLatTile && cached) w.blk = a.block_table[(int64_t)b * a.max_blocks + min(bi, a.max_blocks - 1)];
    }
    return w;
}
// one arrival on the barrier at this offset in both blocks when the products issued so far are done
__device__ __forceinline__ void pair_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((unsigned short)3) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T with 128 rows, 64 of them and half of B's in either block
__device__ __forceinline__ void tc_mma_pair(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"((unsigned)acc), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tc_mma_pair_add(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc) {
    asm volatile("{\n.reg .b64 a, b;\nmov.b64 a, {%1, %4};\nmov.b64 b, {%2, %4};\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, 1;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(kDescHigh) : "memory");
}
template <int R>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) dsa_latent_pair_kernel(const LatentTcArgs g, const __grid_constant__ LatentMaps maps) {
    using W = LatentCfg<R>;
    using C = PairCfg<R>;
    using Seg = LatentSeg<kPairTile>;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + W::Q_BYTES;
    unsigned char* s_p2 = s_ring + W::SLOTS * W::SLOT;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(s_p2 + C::P2_BYTES);
    constexpr int LANDS = W::SLOTS * W::LAND, PARTS = W::SLOTS * W::GROUPS;
    // in the first block of the pair, whose warps issue the products:
    unsigned long long* full = bars;                          // [slot][LAND] has landed in both blocks
    unsigned long long* p_ready = bars + LANDS;               // [2] weights are in shared memory
    unsigned long long* v_ready = p_ready + 2;                // [2] the values that the other block's keys have are there
    unsigned long long* q_full = p_ready + 4;
    unsigned long long* o_free = p_ready + 5;                 // O has been read
    unsigned long long* drained = p_ready + 6;                // [2]
    // in both:
    unsigned long long* empty = p_ready + 8;                  // [slot][GROUPS] the products that read it are done
    unsigned long long* s_full = empty + PARTS;               // [2] scores are in TMEM
    unsigned long long* pv_done = s_full + 2;                 // [2] O holds the tile
    unsigned long long* q_empty = s_full + 4;                 // the scores of a share's last tile are done
    unsigned long long* info_full = s_full + 5;               // [2] the next share is known
    unsigned long long* info_empty = s_full + 7;              // [2] every warp has read it
    unsigned long long* v_land = s_full + 9;                  // the other keys' values have landed here
    unsigned long long* swap_full = s_full + 10;              // [2] the two warps of a row have written to s_pair
    Seg* s_info = reinterpret_cast<Seg*>(s_full + 12);        // [2]
    float* s_pair = reinterpret_cast<float*>(s_info + 2);     // [2][128] maxima and sums that the two halves of a row exchange
    int* s_misc = reinterpret_cast<int*>(s_pair + 256);       // [0] TMEM address, [1] abort, [2..] first request, its first unit, units, set-up units
    int2* s_scan = reinterpret_cast<int2*>(s_misc + 8);       // [8]
    static_assert((LANDS + PARTS + 20) * 8 + 2 * sizeof(Seg) + 1024 + 96 <= W::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const LatentArgs& l = g.l;
    unsigned rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const bool leader = rank == 0;
    const int share = (int)blockIdx.x >> 1;

    if (warp == 4 && lane == 0) {
        for (int s = 0; s < LANDS; ++s) mbar_init(full + s, 1);
        for (int s = 0; s < PARTS; ++s) mbar_init(empty + s, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(p_ready + s, 8); mbar_init(v_ready + s, 2); mbar_init(drained + s, 1);
            mbar_init(s_full + s, 1); mbar_init(pv_done + s, 1);
            mbar_init(info_full + s, 1); mbar_init(info_empty + s, 7); mbar_init(swap_full + s, 2);
        }
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(o_free, 8); mbar_init(v_land, 1);
        s_misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 6) {
        if (lane < 3)
            asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &maps.q : lane == 1 ? &maps.cache : &maps.fresh) : "memory");
    } else if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        tc_fence_before();
    }
    __syncthreads();
    tree_cluster_barrier();                                           // (the other block's barriers are there)
    tc_fence_after();
    const unsigned tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    latent_first<kPairTile, kPairRows>(g, share, s_scan, s_misc + 2);

    Seg sg;
    auto next_seg = [&](int i) -> bool {
        if (!tree_wait(info_full + (i & 1), (i >> 1) & 1, abort, l.a.wait_timeouts, lane)) return false;
        sg = s_info[i & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty + (i & 1));
        return sg.b >= 0;
    };
    // tokens of tile t that block h of the pair has
    auto half_count = [&](int t, int h) { return max(0, min(kLatTile, sg.count(t) - h * kLatTile)); };
    auto where = [&](int t, int h) { return pair_where(g, sg.b, (sg.t0 + t) * kPairTile + h * kLatTile, sg.cached(t), lane); };
    // boxes of block h's keys of tile t, and their rows; a tile of new tokens is one box of N rows, the first block's
    auto used_boxes = [&](int t, int h) { return sg.cached(t) ? (half_count(t, h) + (1 << g.box_shift) - 1) >> g.box_shift : h == 0 ? 1 : 0; };
    auto used_rows = [&](int t, int h) { return sg.cached(t) ? used_boxes(t, h) << g.box_shift : h == 0 ? l.N : 0; };
    // `nch` columns, column(i) of the rows to place(i) of the slot, of block h's keys of tile t
    auto copy_cols = [&](int t, int h, const PairWhere& w, unsigned char* dst, int nch, auto column, auto place, auto bar) {
        const int used = used_boxes(t, h);
        if (!sg.cached(t)) {
            if (lane < nch && used > 0) pair_box3(dst + place(lane) * W::CHUNK, &maps.fresh, 64 * column(lane), 0, sg.b, bar(lane));
        } else {
            for (int p0 = 0; p0 < used * nch; p0 += 32) {
                const int p = p0 + lane, n = p / nch, i = p - n * nch;
                int blk = __shfl_sync(0xffffffffu, w.blk, n & 31);
                const int tok = __shfl_sync(0xffffffffu, w.tok, n & 31);
                if (l.a.block_table) blk = max(0, min(blk, l.a.num_blocks - 1)) * g.blk_coord;
                if (p < used * nch) pair_box3(dst + place(i) * W::CHUNK + ((n << g.box_shift) * 128), &maps.cache, 64 * column(i), tok, blk, bar(i));
            }
        }
        __syncwarp();
    };

    if (warp == 4) {
        // ---- what to work on; copies of q and of this block's keys -------------------------------------------
        const int setup = s_misc[5];
        LatentCursor<kPairTile, kPairRows> cur = {s_misc[2], s_misc[3], s_misc[4]};
        int slot = 0, round = 0, issued = 0, live = 0;
        bool ok = true;
        for (int i = 0; ok; ++i) {
            sg = cur.next(l, setup);
            if (i >= 2) ok = tree_wait(info_empty + (i & 1), ((i >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) s_info[i & 1] = sg;
            __syncwarp();
            if (lane == 0) mbar_arrive(info_full + (i & 1));
            if (sg.b < 0) break;
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            const int q_row = sg.b * l.rows + sg.rt * kPairRows + (int)rank * kLatRows;
            PairWhere at0, at1;
            at0 = where(0, (int)rank);
            const int q_before = live;
            if (lane < W::CH)
                asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];"
                             ::"l"(&maps.q), "r"(64 * lane), "r"(q_row), "r"(0) : "memory");
            auto copy_q = [&]() -> bool {
                if (live > 0 && !tree_wait(q_empty, (live - 1) & 1, abort, l.a.wait_timeouts, lane)) return false;
                if (leader && lane == 0) mbar_expect_tx(q_full, (unsigned)(2 * W::Q_BYTES));
                __syncwarp();
                if (lane < W::CH) pair_box3(s_q + lane * kLatRows * 128, &maps.q, 64 * lane, q_row, 0, tree_peer(q_full, 0));
                __syncwarp();
                ++live;
                return true;
            };
            if (live == 0) ok = copy_q();
            for (int t = 0; ok && t < tiles; ++t) {
                if (t + 1 < tiles) at1 = where(t + 1, (int)rank);
                const unsigned rows = (unsigned)(used_rows(t, 0) + used_rows(t, 1));
                unsigned char* dst = s_ring + slot * W::SLOT;
#pragma unroll 1
                for (int gr = 0; ok && gr < W::GROUPS; ++gr) {
                    if (round > 0) ok = tree_wait(empty + slot * W::GROUPS + gr, (round - 1) & 1, abort, l.a.wait_timeouts, lane);
                    if (!ok) break;
                    const int c0 = gr * 4, nch = gr == W::GROUPS - 1 ? W::CH - c0 : 4;
                    if (leader && lane < W::LAND && 3 * lane >= c0 && 3 * lane < c0 + nch)    // parts that begin in this group
                        mbar_expect_tx(full + slot * W::LAND + lane, (unsigned)(min(3, W::CH - 3 * lane) * 128) * rows);
                    __syncwarp();
                    copy_cols(t, (int)rank, at0, dst, nch, [&](int c) { return c0 + c; }, [&](int c) { return c0 + c; },
                              [&](int c) { return tree_peer(full + slot * W::LAND + (c0 + c) / 3, 0); });
                }
                issued += W::LAND;
                if (++slot == W::SLOTS) { slot = 0; ++round; }
                if (ok && t == 0 && live == q_before) ok = copy_q();
                at0 = at1;
            }
        }
        // no copy is in flight when the pair ends (in a healthy run the products have waited for all of them)
        if (leader) {
            volatile int no_abort = 0;
            if (live > 0) tree_wait(q_full, (live - 1) & 1, &no_abort, nullptr, lane);
            for (int c = max(0, issued - LANDS); c < issued; ++c)
                if (!tree_wait(full + c % LANDS, (c / LANDS) & 1, &no_abort, nullptr, lane)) break;
        }
    } else if (warp == 6) {
        // ---- values of the other block's keys -----------------------------------------------------------------
        // A product with V needs all 128 keys of the block's half of the dims.  When the scores are done, half of what this
        // block's own keys brought is of no more use: the columns of the other half's dims.  The other block's keys take
        // their place, with the columns of this half: columns {0, 1}, {4, 5} of keys 0-63 stand at 0, 1, 4, 5 and of keys
        // 64-127 at 2, 3, 6, 7 in the first block, {2, 3}, {6, 7} in the second.
        int done = 0, slot = 0, landed = 0;
        bool ok = true;
        const int other = 1 - (int)rank;
        constexpr int COLS = R / 128;                         // columns that come from the other keys
        const int to = leader ? 2 : 0, from = leader ? 0 : 2;
        auto pick = [](int c, int base) { return (c >> 1) * 4 + (c & 1) + base; };
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            PairWhere at0, at1;
            at0 = where(0, other);
            for (int t = 0; ok && t < tiles; ++t) {
                if (t + 1 < tiles) at1 = where(t + 1, other);
                const int gt = done + t, buf = gt & 1, rows = used_rows(t, other);
                ok = tree_wait(s_full + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                unsigned char* dst = s_ring + slot * W::SLOT;
                if (rows > 0) {
                    if (lane == 0) mbar_expect_tx(v_land, (unsigned)(COLS * 128 * rows));
                    __syncwarp();
                    copy_cols(t, other, at0, dst, COLS, [&](int c) { return pick(c, from); }, [&](int c) { return pick(c, to); },
                              [&](int) { return smem_u32(v_land); });
                }
                // rows behind the last token, up to where the product stops: zero, whatever the cache or the slot held
                auto zero = [&](int count, int base) {
                    if (!(count & 15)) return;
                    const int pieces = (16 - (count & 15)) * 8;
                    for (int x = lane; x < pieces * COLS; x += 32) {
                        const int c = x / pieces, at = x - c * pieces;
                        *reinterpret_cast<uint4*>(dst + pick(c, base) * W::CHUNK + count * 128 + at * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                };
                zero(half_count(t, (int)rank), from);
                if (rows > 0) {
                    ok = tree_wait(v_land, landed & 1, abort, l.a.wait_timeouts, lane);
                    ++landed;
                    if (!ok) break;
                    zero(half_count(t, other), to);
                }
                __syncwarp();
                if (lane == 0) pair_arrive(tree_peer(v_ready + buf, 0));
                if (++slot == W::SLOTS) slot = 0;
                at0 = at1;
            }
            done += tiles;
        }
        if (!ok && landed > 0) {
            volatile int no_abort = 0;
            tree_wait(v_land, (landed - 1) & 1, &no_abort, nullptr, lane);
        }
    } else if (warp == 5 && !leader) {
        // ---- the new tokens' rows to the cache; query rows that no item has ----------------------------------------
        for (int i = 0; next_seg(i); ++i) latent_rest<R, kPairRows>(l, sg, sg.rt, (sg.n * l.a.H_q + kPairRows - 1) / kPairRows, lane);
    } else if (warp == 5) {
        // ---- scores, by the first block -------------------------------------------------------------------------
        constexpr unsigned kIdescS = instr_desc(kPairRows, kPairTile, false);
        const unsigned q_desc = desc_low(smem_u32(s_q), 16), k_desc = desc_low(smem_u32(s_ring), 16);
        int done = 0, slot = 0, round = 0, live = 0;
        bool ok = true;
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            ok = tree_wait(q_full, live & 1, abort, l.a.wait_timeouts, lane);
            ++live;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                // (this buffer of S has been read; and both blocks have said so of the values, before either says it again)
                if (gt >= 2)
                    ok = tree_wait(p_ready + buf, ((gt >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane) &&
                         tree_wait(v_ready + buf, ((gt >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                const unsigned d = tmem + C::COL_S + buf * 64;
#pragma unroll
                for (int p = 0; p < W::LAND; ++p) {
                    constexpr int kCols = 3;
                    const int c0 = p * kCols, nch = W::CH - c0 < kCols ? W::CH - c0 : kCols;
                    ok = ok && tree_wait(full + slot * W::LAND + p, round & 1, abort, l.a.wait_timeouts, lane);
                    if (!ok) break;
                    if (elect_one()) {
                        const unsigned qa = q_desc + c0 * kLatRows * 128 / 16, ka = k_desc + (slot * W::SLOT + c0 * W::CHUNK) / 16;
                        if (p == 0) tc_mma_pair(d, qa, ka, kIdescS, false);
                        else tc_mma_pair_add(d, qa, ka, kIdescS);
#pragma unroll
                        for (int k = 1; k < 4 * kCols; ++k)
                            if (k / 4 < nch) tc_mma_pair_add(d, qa + ((k / 4) * kLatRows * 128 + (k % 4) * 32) / 16, ka + ((k / 4) * W::CHUNK + (k % 4) * 32) / 16, kIdescS);
                        if (p == W::LAND - 1) {
                            pair_commit(s_full + buf);
                            if (t == tiles - 1) pair_commit(q_empty);
                        }
                    }
                    __syncwarp();
                }
                if (++slot == W::SLOTS) { slot = 0; ++round; }
            }
            done += tiles;
        }
        // TMEM is given back only when no product uses it
        if (__any_sync(0xffffffffu, !ok || *abort)) {
            if (elect_one())
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(drained)) : "memory");
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained, 0u, &no_abort, nullptr, lane);
        }
    } else if (warp == 7) {
        // ---- products with V, by the first block ----------------------------------------------------------------
        constexpr unsigned kIdescO = instr_desc(kPairRows, 256, true);
        const unsigned ring_desc = desc_low(smem_u32(s_ring), 16), v_desc = desc_low(smem_u32(s_ring), W::CHUNK), p2_desc = desc_low(smem_u32(s_p2), 16);
        int done = 0, slot = 0, live = 0;
        bool ok = true;
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            if (tiles == 0 || !leader) continue;
            // (the first product replaces the last share's O)
            if (live > 0) ok = tree_wait(o_free, (live - 1) & 1, abort, l.a.wait_timeouts, lane);
            ++live;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                ok = tree_wait(p_ready + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane) &&
                     tree_wait(v_ready + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const int steps = (sg.count(t) + 15) / 16;
                    const unsigned va = v_desc + slot * (W::SLOT / 16), pa = ring_desc + (slot * W::SLOT + (W::CH - 1) * W::CHUNK) / 16;
#pragma unroll
                    for (int nb = 0; nb < R / 256; ++nb) {
                        tc_mma_pair(tmem + nb * 128, pa, va + nb * 4 * W::CHUNK / 16, kIdescO, t > 0);
#pragma unroll
                        for (int kk = 1; kk < 8; ++kk)
                            if (kk < steps)
                                tc_mma_pair_add(tmem + nb * 128, kk < 4 ? pa + kk * 2 : p2_desc + (kk - 4) * 2,
                                                va + ((nb * 4 + (kk < 4 ? 0 : 2)) * W::CHUNK + (kk & 3) * 2048) / 16, kIdescO);
                        pair_commit(empty + slot * W::GROUPS + nb);
                    }
                    pair_commit(pv_done + buf);
                }
                __syncwarp();
                if (++slot == W::SLOTS) slot = 0;
            }
            done += tiles;
        }
        if (leader && __any_sync(0xffffffffu, !ok || *abort)) {
            if (elect_one())
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(drained + 1)) : "memory");
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained + 1, 0u, &no_abort, nullptr, lane);
        }
    } else {
        // ---- softmax: two threads per query row, half of the tile's keys each ----------------------------------------
        const int half = warp >> 1, row = (warp & 1) * 32 + lane;
        const unsigned lane_base = (unsigned)(warp * 32) << 16;
        const float sl = l.a.scale_log2;
        int done = 0, slot = 0, swaps = 0;
        bool ok = true;
        // a number from either thread of a row to the other one
        auto swap = [&](float mine, float& theirs) -> bool {
            float* at = s_pair + (swaps & 1) * 128;
            at[tid] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(swap_full + (warp & 1));
            const bool fine = tree_wait(swap_full + (warp & 1), swaps & 1, abort, l.a.wait_timeouts, lane);
            theirs = at[tid ^ 64];
            ++swaps;
            return fine;
        };
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles(), my_row = (int)rank * kLatRows + row;
            const bool alive = my_row < sg.rows;
            const int token = (sg.rt * kPairRows + my_row) / l.a.H_q;
            float m_ref = -INFINITY, sum_l = 0.f;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                ok = tree_wait(s_full + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                unsigned x[2][32];
                tc_ld32(x[0], tmem + lane_base + C::COL_S + buf * 64);
                tc_ld32(x[1], tmem + lane_base + C::COL_S + buf * 64 + 32);
                // (a row that does not exist computes along, unmasked, and decides nothing)
                int seen = kPairTile;
                if (alive) seen = sg.cached(t) ? sg.count(t) : token + 1;
                seen -= half * kLatTile;
                tc_wait_ld();
                tc_fence_before();
                if (__any_sync(0xffffffffu, seen < kLatTile)) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c * 32 + k >= seen) x[c][k] = 0xff800000u;
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 32; k += 4)
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        mx[h] = fmaxf(fmaxf(mx[h], __uint_as_float(x[h & 1][k + (h & 2)])), __uint_as_float(x[h & 1][k + (h & 2) + 1]));
                float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), m_other;
                ok = swap(m_tile, m_other);
                if (!ok) break;
                m_tile = fmaxf(m_tile, m_other);
                // O holds the tile before, and what its second half's weights were in may be written again
                if (gt > 0) ok = tree_wait(pv_done + ((gt - 1) & 1), ((gt - 1) >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                // (-inf - -inf is NaN: compares false, nothing to rescale; both warps of the rows decide alike)
                if (__any_sync(0xffffffffu, alive && (m_tile - m_ref) * sl > 8.f)) {
                    const float m_new = fmaxf(m_ref, m_tile);
                    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m_ref - m_new) * sl);
                    m_ref = m_new;
                    sum_l *= alpha;
                    if (t > 0) {
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < R / 2; c += 32) {
                            unsigned o[32];
                            tc_ld32(o, tmem + lane_base + c);
                            tc_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tc_st32(tmem + lane_base + c, o);
                        }
                        tc_wait_st();
                        tc_fence_before();
                    }
                }
                const float sub = m_ref == -INFINITY ? 0.f : m_ref * sl;
                const unsigned long long sl2 = pack_f32x2(sl, sl), sub2 = pack_f32x2(-sub, -sub);
                unsigned long long sum[2] = {0ull, 0ull};
                // weights of the first 64 keys take the place of the slot's r part, which the scores were the last to read
                unsigned char* p_row = (half == 0 ? s_ring + slot * W::SLOT + (W::CH - 1) * W::CHUNK : s_p2) + row * 128;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    unsigned pk[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[c][2 * k]), __uint_as_float(x[c][2 * k + 1])), sl2, sub2));
                        const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                        sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                        pk[k] = pack_bf16(p0, p1);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<uint4*>(p_row + (((c * 4 + k) ^ (row & 7)) * 16)) = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
                }
                const float2 both = unpack_f32x2(add_f32x2(sum[0], sum[1]));
                sum_l += both.x + both.y;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) pair_arrive(tree_peer(p_ready + buf, 0));
                if (++slot == W::SLOTS) slot = 0;
            }
            if (!ok) break;
            float total = 0.f;
            if (tiles > 0) {
                done += tiles;
                ok = tree_wait(pv_done + ((done - 1) & 1), ((done - 1) >> 1) & 1, abort, l.a.wait_timeouts, lane) && swap(sum_l, total);
                if (!ok) break;
                tc_fence_after();
                total += sum_l;
            }
            const int first = sg.rt * kPairRows + (int)rank * kLatRows;
            latent_results<R>(g, tmem + lane_base, (int64_t)sg.b * l.rows + first + row, max(0, min(kLatRows, l.rows - first)), row, half,
                              sg.part < 0 ? -1 : (share * 2 + (int)rank) * 2 + sg.part, tiles > 0, alive, m_ref * sl, total);
            if (tiles == 0) continue;
            if (lane == 0) pair_arrive(tree_peer(o_free, 0));
        }
    }
    __syncthreads();                                          // (every role has come to its end)
    tree_cluster_barrier();                                           // nobody leaves while its shared memory or barriers may be used
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
