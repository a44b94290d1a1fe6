// Attention of the tokens of prompts with expanded keys and values, bf16 (dsa_latent_prompt).
//
// S = Q [K | K_rope]^T over D + 64 numbers (what K_rope has fewer arrives as zeros), O += W V, with the lagging reference and the
// roundings of dsa_latent.cuh.  K_rope's rows are one column of a tile, read once for all heads from where they lie; k_nope and v
// are read through their strides, so the two parts of one product's rows need no copy.
//
// What bounds it: the tensor pipe, 2 (D + 64 + D) operations a query and key, and beside it the softmax, an exponential for each.
// A block has 256 queries as two halves of 128 (M 128, one thread a row), each with a warp that issues its products, so that one
// half's softmax runs under the other's products.  A half has 80 columns of scores and 40 of weights of its own beside O's (2 x
// 128 + 256 = 512 columns with D 128): the scores of tile j + 1 are there when the softmax of tile j is done, and 80 keys are the
// most that leaves room for.  Weights go back through tensor memory (A of the second product), not through shared memory, whose bytes
// the products need: K and V of a tile are read by either half, q with every tile.  Tiles of 96 keys whose weights
// take the scores' columns: 84 us for the prompt below instead of 81, and 75 instead of 68 for the batch.
// Blocks are persistent and take over those not launched yet, so that an item's first copies run under the last one's products;
// where a list of the items fits, the dearest come first, and a ragged batch leaves no SM behind.  The rows that do not fill a block are the
// request's first ones, which see the fewest keys.
//
// Measured: one prompt of 4160 tokens, 16 heads: 80 us, 1.1 PFLOP/s or 65 % of the measured matrix rate (which is for bursts: in a row of such
// calls the power limit holds the clock at 1650 MHz, 92 us).  24 prompts of up to 600 tokens behind prefixes of up to 512, 16 heads:
// 64 us, where keys and values alone (185 MB) would take 29: halves that are not full, and beginnings and ends of short items.
#pragma once
#include "dsa_prompt_args.cuh"
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kPrTile = 80;                        // keys per tile: scores, weights and O of 256 queries fill the tensor memory
constexpr int kPrRows = 128;                       // query rows per half of a block: the M of the products
constexpr int kPrBlock = 2 * kPrRows;
constexpr int kPrThreads = 352;
constexpr int kPrPassed = 4096;                    // blocks without a query that a running block passes over before it says so
static_assert(kPrListed <= kPrThreads && kPrListed <= 256, "a request and an entry a thread, a byte for either in a name");

struct PromptMaps {
    CUtensorMap q, k, kr, v;
    int q_head, k_head, v_head;                    // 0: the map's head dimension has one entry (stride 0)
};

template <int D>
struct PromptCfg {
    static constexpr int KC = D / 64 + 1, VC = D / 64;                     // 64-element columns of a key (the last: k_rope), a value
    static constexpr int COL = kPrTile * 128, Q_COL = kPrRows * 128;       // bytes of one column of a tile, of a half's queries
    static constexpr int Q_BYTES = 2 * KC * Q_COL;
    static constexpr int K_SLOTS = D == 128 ? 3 : 4, V_SLOTS = D == 128 ? 2 : 4;   // tiles in flight
    static constexpr int K_SLOT = KC * COL, V_SLOT = VC * COL, RING_BYTES = K_SLOTS * K_SLOT + V_SLOTS * V_SLOT;
    static constexpr int TAIL = 1024;
    static constexpr int SMEM = Q_BYTES + RING_BYTES + TAIL;
    static constexpr int COL_P = kPrTile, COL_HALF = 128, COL_O = 256, TMEM_COLS = 512;    // a half: scores, then weights; O of both
    static_assert(COL_P + kPrTile / 2 <= COL_HALF, "tensor memory");
    static_assert(SMEM <= 232448, "shared memory of an SM");
};

__device__ __forceinline__ void tma_col(void* dst, const CUtensorMap* map, int c0, int c1, int c2, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar)) : "memory");
}

// What a block works on: 256 queries of one (request, head), in two halves.
struct PromptItem {
    int h, row0, k0, nk, n_tiles;                  // head (< 0: nothing any more), first query's row, first key, keys, key tiles that any query sees
    int shift;                                     // query i of the item sees the first clamp(i + shift, 0, nk) keys
    int rows[2], len[2], tiles[2];                 // of either half: queries, keys that any of them sees, tiles of those
};

// BLOCKS: how a block finds its work (forms of their own, because what one of them does not need cost it 2 to 5 % with short prompts)
template <int D, int BLOCKS>
__global__ void __launch_bounds__(kPrThreads, 1) dsa_prompt_kernel(const PromptArgs g, const __grid_constant__ PromptMaps maps) {
    using C = PromptCfg<D>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned char* s_vring = s_ring + C::K_SLOTS * C::K_SLOT;
    constexpr int SLOTS = C::K_SLOTS + C::V_SLOTS;
    unsigned long long* k_full = reinterpret_cast<unsigned long long*>(s_ring + C::RING_BYTES);    // a tile's K has landed
    unsigned long long* v_full = k_full + C::K_SLOTS;
    unsigned long long* k_empty = k_full + SLOTS;             // the products of either half that read it are done
    unsigned long long* v_empty = k_empty + C::K_SLOTS;
    unsigned long long* q_full = k_full + 2 * SLOTS;          // [2] a half's queries
    unsigned long long* s_full = q_full + 2;                  // [2] scores are in TMEM
    unsigned long long* p_ready = q_full + 4;                 // [2] weights are in TMEM
    unsigned long long* pv_done = q_full + 6;                 // [2] O holds the tile
    unsigned long long* drained = q_full + 8;                 // [2]
    unsigned long long* s_read = q_full + 10;                 // [2] the scores have been read
    unsigned long long* q_empty = q_full + 12;                // [2] the scores of an item's last tile are done
    unsigned long long* o_free = q_full + 14;                 // [2] O has been read
    unsigned long long* info_full = q_full + 16;              // [2] the next item is known
    unsigned long long* info_empty = q_full + 18;             // [2] every warp has read it
    unsigned long long* stolen = q_full + 20;
    uint4* s_response = reinterpret_cast<uint4*>(q_full + 22);
    PromptItem* s_info = reinterpret_cast<PromptItem*>(q_full + 24);           // [2]
    int* s_misc = reinterpret_cast<int*>(s_info + 2);         // [0] TMEM address, [1] abort
    unsigned short* s_list = reinterpret_cast<unsigned short*>(s_misc + 2);    // [kPrListed] request | number << 8; 0xffff: nothing
    static_assert((2 * SLOTS + 24) * 8 + 2 * sizeof(PromptItem) + 8 + 2 * kPrListed <= C::TAIL, "tail of the shared memory");
    static_assert((2 * SLOTS + 22) % 2 == 0, "the response lies on 16 bytes");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (warp == 8 && lane == 0) {
        for (int s = 0; s < SLOTS; ++s) { mbar_init(k_full + s, 1); mbar_init(k_empty + s, 2); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full + s, 1); mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
            mbar_init(drained + s, 1); mbar_init(s_read + s, 4); mbar_init(q_empty + s, 1); mbar_init(o_free + s, 4);
            mbar_init(info_full + s, 1); mbar_init(info_empty + s, 10);
        }
        mbar_init(stolen, 1);
        s_misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    // Rows of 256 queries are numbered from the requests' ends.  false: the request has none of this number.
    auto describe = [&](int b, int from_end, PromptItem& it) -> bool {
        int q0, nq, nk;
        prompt_range(g, b, q0, nq, it.k0, nk);
        // the request's last rows are in blocks of kPrBlock from the end; the first rows, with the fewest keys, are what is left
        const int tile = (nq + kPrBlock - 1) / kPrBlock - 1 - from_end;
        if (tile < 0) return false;
        const int first = tile == 0 ? 0 : nq - (from_end + 1) * kPrBlock, n_rows = tile == 0 ? nq - from_end * kPrBlock : kPrBlock;
        // (the starts of the whole request decide which keys a query sees, whatever max_q_len leaves out)
        const int all_q = max(0, min(g.q_start[b + 1], g.q_tokens) - q0);
        it.row0 = q0 + first;
        it.nk = nk;
        it.shift = g.causal ? nk - (all_q - first - 1) : nk;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            it.rows[s] = max(0, min(kPrRows, n_rows - s * kPrRows));
            const int last = g.causal ? s * kPrRows + it.rows[s] - 1 : 0;
            it.len[s] = it.rows[s] > 0 ? max(0, min(nk, last + it.shift)) : 0;
            it.tiles[s] = (it.len[s] + kPrTile - 1) / kPrTile;
        }
        it.n_tiles = max(it.tiles[0], it.tiles[1]);
        return true;
    };
    if constexpr (BLOCKS == kPrByList) {
        // A list of the items of one head, without gaps and by what they cost, the dearest first: a tile of both halves takes some 2500
        // cycles, of one 1400, the ends of an item 3000.  (a request a thread, then an entry a thread)
        int* s_cost = reinterpret_cast<int*>(smem);
        int* s_name = s_cost + kPrListed;
        int* s_warp = s_name + kPrListed;
        int q0, nq, k0, nk, rows = 0;
        if (tid < kPrListed) {
            s_cost[tid] = -1;
            if (tid < g.batch) {
                prompt_range(g, tid, q0, nq, k0, nk);
                rows = (nq + kPrBlock - 1) / kPrBlock;
            }
        }
        const int first = prompt_before(rows, s_warp);
        PromptItem it = {};
        for (int k = 0; k < rows && first + k < g.entries; ++k) {
            describe(tid, k, it);
            s_cost[first + k] = 6 + 3 * it.n_tiles + 2 * min(it.tiles[0], it.tiles[1]);
            s_name[first + k] = tid | k << 8;
        }
        __syncthreads();
        if (tid < g.entries) {
            const int mine = s_cost[tid];
            int place = 0;
#pragma unroll 8
            for (int k = 0; k < g.entries; ++k) place += s_cost[k] > mine || (s_cost[k] == mine && k < tid);
            s_list[place] = mine < 0 ? 0xffff : (unsigned short)s_name[tid];
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // (copies take s_cost's place)
        __syncthreads();
    }

    // item number `i` of this block, once the copying warp has found it; nullptr: give up
    auto item = [&](int i) -> const PromptItem* {
        return tree_wait(info_full + (i & 1), (i >> 1) & 1, abort, g.wait_timeouts, lane) ? s_info + (i & 1) : nullptr;
    };
    auto item_read = [&](int i) {                             // this warp needs item i's description no longer
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty + (i & 1));
    };

    if (warp == 8) {
        // ---- what to work on; copies of q, K(0), V(0), K(1), V(1), ... ----------------------------------------
        // Blocks are persistent: a running one takes over the next that has not been launched yet, and begins its copies while
        // the products of the last one run.
        PromptItem it = {};
        int issued = 0, k_issued = 0, live[2] = {0, 0}, idx = (int)blockIdx.x, asked = 0, answered = 0;
        bool ok = true;
        auto ask = [&]() {
            __syncwarp();                                     // (every lane has read the last response, whose place the next one takes)
            if (lane == 0) steal_block(s_response, stolen);
            __syncwarp();
            ++asked;
        };
        auto answer = [&]() -> bool {
            volatile int no_abort = 0;                        // (the response is waited for whatever else has happened)
            ++answered;
            if (!tree_wait(stolen, (asked - 1) & 1, &no_abort, g.wait_timeouts, lane)) { *abort = 1; return false; }
            idx = stolen_block(s_response);
            return true;
        };
        for (int i = 0; ok; ++i) {
            it.h = -1;
            int passed = 0;
            while (ok && idx >= 0) {                          // (blocks without a query are passed over)
                const int e = idx / g.H;
                int2 at;                                      // request (-1: none), which of its blocks
                if constexpr (BLOCKS == kPrByList) {
                    const int name = s_list[e];
                    at = make_int2(name == 0xffff ? -1 : name & 255, name >> 8);
                } else if constexpr (BLOCKS == kPrByNumber) {
                    at = prompt_find(g.q_start, g.q_tokens, g.batch, kPrBlock, e);
                } else {
                    at = make_int2(e % g.batch, e / g.batch);
                }
                if (at.x >= 0 && describe(at.x, at.y, it)) {
                    it.h = idx % g.H;
                    break;
                }
                if (BLOCKS != kPrByList && ++passed == kPrPassed) break;         // (a list is short)
                ask();
                ok = answer();
            }
            // Nobody waits for the end of a long run of blocks without a query, which a batch of 2^20 requests and 1024 heads could make
            // longer than a wait may take (some 0.5 us a block): now and then the others get an item without a row.
            if (BLOCKS != kPrByList && passed == kPrPassed) it = PromptItem{};
            if (!ok) break;
            if (i >= 2) ok = tree_wait(info_empty + (i & 1), ((i >> 1) - 1) & 1, abort, g.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) s_info[i & 1] = it;
            __syncwarp();
            if (lane == 0) mbar_arrive(info_full + (i & 1));
            if (it.h < 0) break;
            const int h = it.h;
            auto copy_q = [&]() {
#pragma unroll
                for (int s = 0; ok && s < 2; ++s) {
                    if (it.tiles[s] == 0) continue;
                    if (live[s] > 0) ok = tree_wait(q_empty + s, (live[s] - 1) & 1, abort, g.wait_timeouts, lane);
                    if (!ok) break;
                    ++live[s];
                    if (lane == 0) {
                        mbar_expect_tx(q_full + s, (unsigned)(C::KC * C::Q_COL));
                        for (int c = 0; c < C::KC; ++c)
                            tma_col(s_q + (s * C::KC + c) * C::Q_COL, &maps.q, 64 * c, h * maps.q_head, it.row0 + s * kPrRows, q_full + s);
                    }
                    __syncwarp();
                }
            };
            if (i == 0) copy_q();
            for (int j = 0; ok && j < it.n_tiles; ++j) {
                const int ks = issued % C::K_SLOTS, k_round = issued / C::K_SLOTS, vs = issued % C::V_SLOTS, v_round = issued / C::V_SLOTS;
                const int tok = it.k0 + j * kPrTile;
                if (j + 1 == it.n_tiles) ask();               // late, so that it goes to whoever has room for it
                if (k_round > 0) ok = tree_wait(k_empty + ks, (k_round - 1) & 1, abort, g.wait_timeouts, lane);
                if (ok && lane == 0) {
                    mbar_expect_tx(k_full + ks, (unsigned)C::K_SLOT);
                    for (int c = 0; c < C::KC - 1; ++c) tma_col(s_ring + ks * C::K_SLOT + c * C::COL, &maps.k, 64 * c, h * maps.k_head, tok, k_full + ks);
                    tma_col(s_ring + ks * C::K_SLOT + (C::KC - 1) * C::COL, &maps.kr, 0, 0, tok, k_full + ks);
                }
                __syncwarp();
                if (!ok) break;
                ++k_issued;
                if (j == 0 && i > 0) copy_q();                // (behind the first keys, which need not wait for the last item's scores)
                if (ok && v_round > 0) ok = tree_wait(v_empty + vs, (v_round - 1) & 1, abort, g.wait_timeouts, lane);
                if (ok && lane == 0) {
                    mbar_expect_tx(v_full + vs, (unsigned)C::V_SLOT);
                    for (int c = 0; c < C::VC; ++c) tma_col(s_vring + vs * C::V_SLOT + c * C::COL, &maps.v, 64 * c, h * maps.v_head, tok, v_full + vs);
                }
                __syncwarp();
                if (ok) ++issued;
            }
            if (it.n_tiles == 0) ask();
            if (ok) ok = answer();
        }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        if (asked > answered) answer();
        volatile int no_abort = 0;
        for (int s = 0; s < 2; ++s)
            if (live[s] > 0) tree_wait(q_full + s, (live[s] - 1) & 1, &no_abort, nullptr, lane);
        for (int c = max(0, k_issued - C::K_SLOTS); c < k_issued; ++c)
            if (!tree_wait(k_full + c % C::K_SLOTS, (c / C::K_SLOTS) & 1, &no_abort, nullptr, lane)) break;
        for (int c = max(0, issued - C::V_SLOTS); c < issued; ++c)
            if (!tree_wait(v_full + c % C::V_SLOTS, (c / C::V_SLOTS) & 1, &no_abort, nullptr, lane)) break;
    } else if (warp >= 9) {
        // ---- products of a half, S = Q K(j) and O += P V(j), a warp for either half ------------------------------
        // Scores have columns of their own, so those of tile j + 1 are computed as soon as tile j's have been read, while their
        // weights are worked out: the softmax of a half never waits for a product, and the tensor pipe never for a softmax.
        constexpr unsigned kIdescS = instr_desc(kPrRows, kPrTile, false), kIdescO = instr_desc(kPrRows, D, true);
        const int s = warp - 9;
        const unsigned q_desc = desc_low(smem_u32(s_q), 16) + s * C::KC * (C::Q_COL / 16), k_desc = desc_low(smem_u32(s_ring), 16);
        const unsigned v_desc = desc_low(smem_u32(s_vring), C::COL);
        const unsigned s_addr = tmem + s * C::COL_HALF, p_addr = s_addr + C::COL_P, o_addr = tmem + C::COL_O + s * D;
        bool ok = true;
        int first = 0, mine = 0, live = 0;                    // tiles of the items before this one, this half's of them; items that it had tiles of
        for (int i = 0; ok; ++i) {
            const PromptItem* it = item(i);
            if (!it || it->h < 0) break;
            const int tiles = it->tiles[s], n_tiles = it->n_tiles, len = it->len[s], nk = it->nk;
            item_read(i);
            for (int j = 0; ok && j <= n_tiles && n_tiles > 0; ++j) {
                if (j < n_tiles) {                            // scores of tile j
                    const int slot = (first + j) % C::K_SLOTS;
                    ok = tree_wait(k_full + slot, ((first + j) / C::K_SLOTS) & 1, abort, g.wait_timeouts, lane);
                    if (ok && j < tiles) {
                        if (j == 0) ok = tree_wait(q_full + s, live & 1, abort, g.wait_timeouts, lane);
                        if (ok && mine + j > 0) ok = tree_wait(s_read + s, (mine + j - 1) & 1, abort, g.wait_timeouts, lane);
                    }
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        if (j < tiles) {
#pragma unroll
                            for (int c = 0; c < C::KC; ++c) {
                                const unsigned qa = q_desc + c * (C::Q_COL / 16), ka = k_desc + (slot * C::K_SLOT + c * C::COL) / 16;
                                if (c == 0) tc_mma_ss(s_addr, qa, ka, kIdescS, false);
                                else tc_mma_ss_add(s_addr, qa, ka, kIdescS);
#pragma unroll
                                for (int kk = 1; kk < 4; ++kk) tc_mma_ss_add(s_addr, qa + kk * 2, ka + kk * 2, kIdescS);
                            }
                            tc_commit(s_full + s);
                            if (j + 1 == tiles) tc_commit(q_empty + s);
                        }
                        tc_commit(k_empty + slot);
                    }
                    __syncwarp();
                }
                if (j == 0) continue;
                const int v = j - 1, slot = (first + v) % C::V_SLOTS;        // values of the tile before
                ok = tree_wait(v_full + slot, ((first + v) / C::V_SLOTS) & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                const int count = min(kPrTile, len - v * kPrTile), there = nk - v * kPrTile, steps = (count + 15) / 16;
                if (v < tiles) {
                    // values behind the request's last key, up to where the product stops: zero, whatever they were
                    if (there < steps * 16) {
                        const int pieces = (steps * 16 - there) * 8;
                        for (int x = lane; x < pieces * C::VC; x += 32) {
                            const int c = x / pieces, p = x - c * pieces;
                            *reinterpret_cast<uint4*>(s_vring + slot * C::V_SLOT + c * C::COL + there * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    // (the first product replaces the last item's O)
                    if (v == 0 && live > 0) ok = tree_wait(o_free + s, (live - 1) & 1, abort, g.wait_timeouts, lane);
                    if (ok) ok = tree_wait(p_ready + s, (mine + v) & 1, abort, g.wait_timeouts, lane);
                    if (!ok) break;
                }
                tc_fence_after();
                if (elect_one()) {
                    if (v < tiles) {
                        const unsigned va = v_desc + slot * (C::V_SLOT / 16);
                        tc_mma_ts(o_addr, p_addr, va, kIdescO, v > 0);
                        if (steps == kPrTile / 16) {
#pragma unroll
                            for (int kk = 1; kk < kPrTile / 16; ++kk) tc_mma_ts_add(o_addr, p_addr + kk * 8, va + kk * (2048 / 16), kIdescO);
                        } else {
                            for (int kk = 1; kk < steps; ++kk) tc_mma_ts_add(o_addr, p_addr + kk * 8, va + kk * (2048 / 16), kIdescO);
                        }
                        tc_commit(pv_done + s);
                    }
                    tc_commit(v_empty + slot);
                }
                __syncwarp();
            }
            first += n_tiles;
            mine += tiles;
            if (tiles > 0) ++live;
        }
        if (__any_sync(0xffffffffu, !ok || *abort)) {         // TMEM is given back only when no product uses it
            if (elect_one()) tc_commit(drained + s);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained + s, 0u, &no_abort, nullptr, lane);
        }
    } else {
        // ---- softmax: one thread per query row, four warps per half -----------------------------------------
        const int s = warp >> 2, row = tid & 127;
        const unsigned lane_base = (unsigned)((warp & 3) * 32) << 16;
        const unsigned s_addr = tmem + lane_base + s * C::COL_HALF, p_addr = s_addr + C::COL_P, o_addr = tmem + lane_base + C::COL_O + s * D;
        const float sl = g.scale_log2;
        int done = 0;                                         // tiles of the items before this one
        bool ok = true;
        for (int i = 0; ok; ++i) {
            const PromptItem* it = item(i);
            if (!it || it->h < 0) break;
            const int tiles = it->tiles[s], rows = it->rows[s], h = it->h, row0 = it->row0 + s * kPrRows;
            const bool alive = row < rows;
            // (a row that does not exist computes along and decides nothing)
            const int sees = alive ? max(0, min(it->nk, it->shift + (g.causal ? s * kPrRows + row : 0))) : 0x7fffffff;
            item_read(i);
            float m_ref = -INFINITY, sum_l = 0.f;
            for (int j = 0; ok && j < tiles; ++j) {
                const int gt = done + j;
                ok = tree_wait(s_full + s, gt & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                constexpr int PARTS = kPrTile / 16;
                unsigned x[PARTS][16];
#pragma unroll
                for (int c = 0; c < PARTS; ++c) tc_ld16(x[c], s_addr + 16 * c);
                tc_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_read + s);
                const int seen = sees - j * kPrTile;
                if (__any_sync(0xffffffffu, seen < kPrTile)) {
#pragma unroll
                    for (int c = 0; c < PARTS; ++c)
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (c * 16 + k >= seen) x[c][k] = 0xff800000u;
                }
                float mx[PARTS];
#pragma unroll
                for (int c = 0; c < PARTS; ++c) mx[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
                for (int k = 2; k < 16; k += 2)
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) mx[c] = fmaxf(fmaxf(mx[c], __uint_as_float(x[c][k])), __uint_as_float(x[c][k + 1]));
                float m_tile = mx[0];
#pragma unroll
                for (int c = 1; c < PARTS; ++c) m_tile = fmaxf(m_tile, mx[c]);
                // (-inf - -inf is NaN: compares false, nothing to rescale)
                const bool grow = __any_sync(0xffffffffu, alive && (m_tile - m_ref) * sl > 8.f);
                float alpha = 1.f;
                if (grow) {
                    const float m_new = fmaxf(m_ref, m_tile);
                    if (m_new != -INFINITY) alpha = fast_exp2((m_ref - m_new) * sl);
                    m_ref = m_new;
                    sum_l *= alpha;
                }
                const float sub = m_ref == -INFINITY ? 0.f : m_ref * sl;
                const unsigned long long sl2 = pack_f32x2(sl, sl), sub2 = pack_f32x2(-sub, -sub);
                unsigned long long sum[2] = {0ull, 0ull};
                unsigned pk[PARTS][8];
#pragma unroll
                for (int c = 0; c < PARTS; ++c)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[c][2 * k]), __uint_as_float(x[c][2 * k + 1])), sl2, sub2));
                        const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                        sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                        pk[c][k] = pack_bf16(p0, p1);
                    }
                // only now: O holds the tile before, and that tile's weights may be written over
                if (gt > 0) ok = tree_wait(pv_done + s, (gt - 1) & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                if (grow && j > 0) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        unsigned o[16];
                        tc_ld16(o, o_addr + c);
                        tc_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                        tc_st16(o_addr + c, o);
                    }
                }
#pragma unroll
                for (int c = 0; c < PARTS; ++c) tc_st8(p_addr + 8 * c, pk[c]);
                const float2 both = unpack_f32x2(add_f32x2(sum[0], sum[1]));
                sum_l += both.x + both.y;
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready + s);
            }
            // ---- results ----------------------------------------------------------------------------------------
            if (!ok) break;
            if (tiles > 0) {
                done += tiles;
                ok = tree_wait(pv_done + s, (done - 1) & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
            }
            if ((warp & 3) * 32 < rows) {
                const bool none = sum_l == 0.f;                    // nothing seen: zeros and -inf
                const float inv = none ? 0.f : 1.f / sum_l;
                const int64_t orow = (int64_t)(row0 + row) * g.H + h;
                T* dst = reinterpret_cast<T*>(g.out) + orow * D;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned x[32];
                    if (tiles > 0) {
                        tc_ld32(x, o_addr + c);
                        tc_wait_ld();
                    }
                    if (alive)
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            unsigned y[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                y[e] = none ? 0u : pack_bf16(__uint_as_float(x[k + 2 * e]) * inv, __uint_as_float(x[k + 2 * e + 1]) * inv);
                            *reinterpret_cast<uint4*>(dst + c + k) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    __syncwarp();
                }
                if (alive) g.lse[orow] = none ? -INFINITY : (m_ref * sl + log2f(sum_l)) * LN2;
            }
            if (tiles > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_free + s);
            }
        }
    }
    __syncthreads();                                          // (every role has come to its end)
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
