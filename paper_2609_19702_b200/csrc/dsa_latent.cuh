// Attention of new tokens over a latent cache, bf16 (dsa_latent_step).
#pragma once
#include "dsa_latent_args.cuh"
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kLatTile = 64;                       // tokens per tile
constexpr int kLatRows = 64;                       // query rows per block: the M of the products
constexpr int kLatThreads = 256;

struct LatentTcArgs {
    LatentArgs l;
    int groups;                                    // blocks that share the keys of a row tile
    int min_units;                                 // units of work that a block takes at least
    int box_tokens, box_shift;                     // tokens per tensor-map box of the cache, and its logarithm
    unsigned page_mul;                             // position / block_size = (position * page_mul) >> page_shift
    int page_shift;
    int blk_coord;                                 // 0: the map's outer dimension has one entry (stride 0)
    int* sched;                                    // workspace: [B + 1] units before each request, then the quota
    float2* part_ml;                               // [groups * row_tiles * 2][64] maximum (base 2) and sum
    float4* part_o;                                // [groups * row_tiles * 2][R / 4][64]
};

struct LatentMaps {
    CUtensorMap q, cache, fresh;
};

template <int R>
struct LatentCfg {
    static constexpr int CH = R / 64 + 1;                                  // 128-byte columns of a row (the last: r)
    static constexpr int CHUNK = kLatTile * 128;
    static constexpr int SLOT = CH * CHUNK;
    static constexpr int Q_BYTES = CH * kLatRows * 128;
    static constexpr int SLOTS = R == 512 ? 2 : 4;
    static constexpr int GROUPS = R / 256;                                 // parts of a slot that land and are freed on their own
    static constexpr int TAIL = 2048;
    static constexpr int SMEM = Q_BYTES + SLOTS * SLOT + TAIL;
    static constexpr int COL_S = R / 2, TMEM_COLS = R == 512 ? 512 : 256;
    static_assert(SMEM <= 232448, "shared memory of an SM");
};

__device__ __forceinline__ void tma_box3(void* dst, const CUtensorMap* map, int c0, int c1, int c2, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar)) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T with 64 rows: the first half of the N columns in lanes 0-63, the second in lanes 64-127
__device__ __forceinline__ void tc_mma_ws(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"((unsigned)acc), "r"(kDescHigh) : "memory");
}
// one look at phase `parity` of the barrier
__device__ __forceinline__ bool mbar_test(unsigned long long* bar, unsigned parity) {
    unsigned done;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return __all_sync(0xffffffffu, done != 0);
}
// Units of work of a request: its cached tiles and one for the new tokens (or for having nothing to do).
__device__ __forceinline__ int latent_units(int S, int n) { return n > 0 ? (S + kLatTile - 1) / kLatTile + 1 : 1; }

// A block's share of one request: units [t0, t1) of `units`.
struct LatentSeg {
    int b, S, n, t0, t1, units, rows, part;        // b < 0: nothing any more.  rows: query rows of tokens that exist.  part: where the
                                                   // partial result goes, -1: the block has the whole request
    __device__ __forceinline__ int tiles() const { return rows > 0 ? t1 - t0 : 0; }
    __device__ __forceinline__ int count(int t) const {                    // tokens of tile t (of this share)
        return t0 + t < units - 1 ? min(kLatTile, S - (t0 + t) * kLatTile) : n;
    }
};

template <int R>
__global__ void __launch_bounds__(kLatThreads, 1) dsa_latent_kernel(const LatentTcArgs g, const __grid_constant__ LatentMaps maps) {
    using C = LatentCfg<R>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(s_ring + C::SLOTS * C::SLOT);
    constexpr int PARTS = C::SLOTS * C::GROUPS;
    unsigned long long* full = bars;                          // [slot][group] has landed
    unsigned long long* empty = bars + PARTS;                 // [slot][group] the products that read it are done
    unsigned long long* s_full = bars + 2 * PARTS;            // [2] scores are in TMEM
    unsigned long long* p_ready = s_full + 2;                 // [2] weights are in shared memory
    unsigned long long* pv_done = s_full + 4;                 // [2] O holds the tile
    unsigned long long* info_full = s_full + 6;               // [2] the next share is known
    unsigned long long* info_empty = s_full + 8;              // [2] every warp has read it
    unsigned long long* q_full = s_full + 10;
    unsigned long long* q_empty = s_full + 11;                // the scores of a share's last tile are done
    unsigned long long* o_free = s_full + 12;                 // O has been read
    unsigned long long* drained = s_full + 13;
    unsigned long long* pair = s_full + 14;                   // [2] the two warps of a row have written to s_pair
    LatentSeg* s_info = reinterpret_cast<LatentSeg*>(s_full + 16);             // [2]
    float* s_pair = reinterpret_cast<float*>(s_info + 2);     // [2][128] maxima and sums that the two halves of a row exchange
    int* s_misc = reinterpret_cast<int*>(s_pair + 256);       // [0] TMEM address, [1] abort, [2..] first request, units before it, total
    int* s_scan = s_misc + 8;                                 // [8]
    static_assert((2 * PARTS + 16) * 8 + 2 * sizeof(LatentSeg) + 1024 + 64 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const LatentArgs& l = g.l;
    const int rt = (int)blockIdx.x % l.row_tiles, group = (int)blockIdx.x / l.row_tiles;

    if (warp == 4 && lane == 0) {
        for (int s = 0; s < 2 * PARTS; ++s) mbar_init(bars + s, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
            mbar_init(info_full + s, 1); mbar_init(info_empty + s, 6);
            mbar_init(pair + s, 2);
        }
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(o_free, 4); mbar_init(drained, 1);
        s_misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 5) {
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

    // ---- this block's share: the units of all requests end to end, cut into equal pieces -----------------------------
    {
        const int B = l.a.B, per = (B + kLatThreads - 1) / kLatThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
        int sum = 0;
        for (int b = b0; b < b1; ++b) {
            int S, n;
            latent_lengths(l, b, S, n);
            sum += latent_units(S, n);
        }
        int before = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += x;
        }
        if (lane == 31) s_scan[warp] = before;
        before -= sum;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < kLatThreads / 32; ++w) {
            if (w < warp) before += s_scan[w];
            total += s_scan[w];
        }
        const int quota = max(g.min_units, (total + g.groups - 1) / g.groups);
        const int first = min(total, group * quota);          // (group * quota < total + groups * min_units)
        if (tid == 0) {
            s_misc[2] = -1;
            s_misc[4] = min(total, first + quota);
            if (blockIdx.x == 0) { g.sched[B] = total; g.sched[B + 1] = quota; }
        }
        __syncthreads();
        for (int b = b0; b < b1; ++b) {
            int S, n;
            latent_lengths(l, b, S, n);
            const int units = latent_units(S, n);
            if (first >= before && first < before + units) { s_misc[2] = b; s_misc[3] = first - before; }
            if (blockIdx.x == 0) g.sched[b] = before;
            before += units;
        }
        if (tid == 0) s_misc[5] = first;
    }
    __syncthreads();

    LatentSeg sg;
    auto next_seg = [&](int i) -> bool {
        if (!tree_wait(info_full + (i & 1), (i >> 1) & 1, abort, l.a.wait_timeouts, lane)) return false;
        sg = s_info[i & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty + (i & 1));
        return sg.b >= 0;
    };

    if (warp == 4) {
        // ---- what to work on; copies of q and of the cached rows ------------------------------------------
        int b = s_misc[2], at = s_misc[3], left = s_misc[4] - s_misc[5];
        int slot = 0, round = 0, issued = 0, live = 0;
        bool ok = true;
        for (int i = 0; ok; ++i) {
            sg.b = left > 0 ? b : -1;
            if (sg.b >= 0) {
                latent_lengths(l, b, sg.S, sg.n);
                sg.units = latent_units(sg.S, sg.n);
                sg.t0 = at;
                sg.t1 = min(sg.units, at + left);
                sg.rows = max(0, min(kLatRows, sg.n * l.a.H_q - rt * kLatRows));
                sg.part = sg.t0 == 0 && sg.t1 == sg.units ? -1 : ((int)blockIdx.x * 2 + (sg.t0 > 0 ? 0 : 1));
                left -= sg.t1 - sg.t0;
                at = 0;
                ++b;
            }
            if (i >= 2) ok = tree_wait(info_empty + (i & 1), ((i >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) s_info[i & 1] = sg;
            __syncwarp();
            if (lane == 0) mbar_arrive(info_full + (i & 1));
            if (sg.b < 0) break;
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            // where this lane's boxes of a tile come from: (page or request, token in it)
            const int boxes = kLatTile >> g.box_shift;
            auto where = [&](int t, int (&blk)[2], int (&tok)[2]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int box = lane + 32 * h, pos = (sg.t0 + t) * kLatTile + (box << g.box_shift);
                    blk[h] = g.blk_coord ? sg.b : 0;
                    tok[h] = pos;
                    if (l.a.block_table) {
                        const int bi = (int)(((unsigned long long)(unsigned)pos * g.page_mul) >> g.page_shift);
                        tok[h] = pos - bi * l.a.block_size;
                        if (box < boxes && sg.t0 + t < sg.units - 1)
                            blk[h] = l.a.block_table[(int64_t)sg.b * l.a.max_blocks + min(bi, l.a.max_blocks - 1)];
                    }
                }
            };
            int blk0[2], tok0[2], blk1[2], tok1[2];
            where(0, blk0, tok0);
            if (live > 0) ok = tree_wait(q_empty, (live - 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(q_full, (unsigned)C::Q_BYTES);
            __syncwarp();
            if (lane < C::CH) tma_box3(s_q + lane * kLatRows * 128, &maps.q, 64 * lane, sg.b * l.rows + rt * kLatRows, 0, q_full);
            ++live;
            for (int t = 0; ok && t < tiles; ++t) {
                if (t + 1 < tiles) where(t + 1, blk1, tok1);
                const bool cached = sg.t0 + t < sg.units - 1;
                const int used = cached ? (sg.count(t) + g.box_tokens - 1) >> g.box_shift : 1;     // boxes
                unsigned char* dst = s_ring + slot * C::SLOT;
#pragma unroll 1
                for (int gr = 0; ok && gr < C::GROUPS; ++gr) {
                    if (round > 0) ok = tree_wait(empty + slot * C::GROUPS + gr, (round - 1) & 1, abort, l.a.wait_timeouts, lane);
                    if (!ok) break;
                    const int c0 = gr * 4, nch = gr == C::GROUPS - 1 ? C::CH - c0 : 4;
                    unsigned long long* bar = full + slot * C::GROUPS + gr;
                    if (lane == 0) mbar_expect_tx(bar, (unsigned)(nch * 128) * (cached ? (unsigned)(used << g.box_shift) : (unsigned)l.N));
                    __syncwarp();
                    if (!cached) {
                        if (lane < nch) tma_box3(dst + (c0 + lane) * C::CHUNK, &maps.fresh, 64 * (c0 + lane), 0, sg.b, bar);
                    } else {
                        for (int p0 = 0; p0 < used * nch; p0 += 32) {
                            const int p = p0 + lane, box = p / nch, c = c0 + p - box * nch;
                            int blk = __shfl_sync(0xffffffffu, blk0[0], box & 31), tok = __shfl_sync(0xffffffffu, tok0[0], box & 31);
                            const int blk_h = __shfl_sync(0xffffffffu, blk0[1], box & 31), tok_h = __shfl_sync(0xffffffffu, tok0[1], box & 31);
                            if (box >= 32) { blk = blk_h; tok = tok_h; }
                            if (l.a.block_table) blk = max(0, min(blk, l.a.num_blocks - 1)) * g.blk_coord;
                            if (p < used * nch) tma_box3(dst + c * C::CHUNK + ((box << g.box_shift) * 128), &maps.cache, 64 * c, tok, blk, bar);
                        }
                    }
                    __syncwarp();
                    ++issued;
                }
                if (++slot == C::SLOTS) { slot = 0; ++round; }
#pragma unroll
                for (int h = 0; h < 2; ++h) { blk0[h] = blk1[h]; tok0[h] = tok1[h]; }
            }
        }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        volatile int no_abort = 0;
        if (live > 0) tree_wait(q_full, (live - 1) & 1, &no_abort, nullptr, lane);
        for (int c = max(0, issued - PARTS); c < issued; ++c)
            if (!tree_wait(full + c % PARTS, (c / PARTS) & 1, &no_abort, nullptr, lane)) break;
    } else if (warp == 5) {
        // ---- products -----------------------------------------------------------------------------------
        constexpr unsigned kIdescS = instr_desc(kLatRows, kLatTile, false), kIdescO = instr_desc(kLatRows, 256, true);
        const unsigned q_desc = desc_low(smem_u32(s_q), 16), k_desc = desc_low(smem_u32(s_ring), 16), v_desc = desc_low(smem_u32(s_ring), C::CHUNK);
        // Scores run up to a tile ahead of the products with V, into the next share if need be: each has its own place in
        // the shares, and whichever can go on does, scores first.
        LatentSeg sp = {};                                    // the share of the products with V
        int si = 0, pi = 0;                                   // shares begun by either
        int ts = 0, tp = 0, s_tiles = 0, p_tiles = 0;         // tiles of it
        int gs = 0, gp = 0, gr = 0;                           // tiles in all; the part of a slot that the scores are at
        int s_slot = 0, s_round = 0, p_slot = 0;
        int s_live = 0, p_live = 0;                           // shares with tiles
        bool s_end = false;
        LatentSeg pend[2];
        long long idle = clock64();
        bool ok = true;
        while (ok && !(s_end && gp == gs)) {
            bool moved = false;
            if (!s_end && ts == s_tiles && si - pi < 2) {     // the scores' next share
                if (mbar_test(info_full + (si & 1), (si >> 1) & 1)) {
                    const LatentSeg x = s_info[si & 1];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(info_empty + (si & 1));
                    pend[0] = pend[1];
                    pend[1] = x;
                    moved = true;
                    if (x.b < 0) { s_end = true; s_tiles = ts = 0; }
                    else { sg = x; s_tiles = x.tiles(); ts = 0; ++si; }
                }
            }
            if (tp == p_tiles && pi < si) {                   // the next share of the products with V: the older one that waits
                sp = si - pi == 2 ? pend[0] : pend[1];
                if (s_end) sp = pend[0];
                p_tiles = sp.tiles();
                tp = 0;
                ++pi;
                moved = true;
            }
            if (ts < s_tiles && gs <= gp + 1 && mbar_test(full + s_slot * C::GROUPS + gr, s_round & 1) &&
                (ts > 0 || gr > 0 || mbar_test(q_full, s_live & 1))) {
                // rows behind the last token, up to where the product with V stops: zero, whatever the cache or the slot held
                const int c0 = gr * 4, nch = gr == C::GROUPS - 1 ? C::CH - c0 : 4, count = sg.count(ts);
                if (count & 15) {
                    const int pieces = (16 - (count & 15)) * 8;
                    for (int i = lane; i < pieces * nch; i += 32) {
                        const int c = i / pieces, p = i - c * pieces;
                        *reinterpret_cast<uint4*>(s_ring + s_slot * C::SLOT + (c0 + c) * C::CHUNK + count * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                tc_fence_after();
                const int buf = gs & 1;
                const bool last = gr == C::GROUPS - 1;
                if (elect_one()) {
                    const unsigned ka = k_desc + s_slot * (C::SLOT / 16), d = tmem + C::COL_S + buf * (kLatTile / 2);
                    for (int c = c0; c < c0 + nch; ++c)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            tc_mma_ws(d, q_desc + (c * kLatRows * 128 + kk * 32) / 16, ka + (c * C::CHUNK + kk * 32) / 16, kIdescS, c > 0 || kk > 0);
                    if (last) {
                        tc_commit(s_full + buf);
                        if (ts == s_tiles - 1) tc_commit(q_empty);
                    }
                }
                __syncwarp();
                if (last) {
                    gr = 0;
                    if (++s_slot == C::SLOTS) { s_slot = 0; ++s_round; }
                    if (ts == s_tiles - 1) ++s_live;
                    ++ts;
                    ++gs;
                } else {
                    ++gr;
                }
                moved = true;
            } else if (tp < p_tiles && gp < gs && mbar_test(p_ready + (gp & 1), (gp >> 1) & 1) &&
                       (tp > 0 || p_live == 0 || mbar_test(o_free, (p_live - 1) & 1))) {
                tc_fence_after();
                if (elect_one()) {
                    const int steps = (sp.count(tp) + 15) / 16;
                    const unsigned va = v_desc + p_slot * (C::SLOT / 16), pa = k_desc + (p_slot * C::SLOT + (C::CH - 1) * C::CHUNK) / 16;
                    for (int nb = 0; nb < R / 256; ++nb) {
                        for (int kk = 0; kk < steps; ++kk)
                            tc_mma_ws(tmem + nb * 128, pa + kk * 2, va + (nb * 4 * C::CHUNK + kk * 2048) / 16, kIdescO, tp > 0 || kk > 0);
                        tc_commit(empty + p_slot * C::GROUPS + nb);
                    }
                    tc_commit(pv_done + (gp & 1));
                }
                __syncwarp();
                if (++p_slot == C::SLOTS) p_slot = 0;
                if (tp == p_tiles - 1) ++p_live;
                ++tp;
                ++gp;
                moved = true;
            }
            if (moved) { idle = clock64(); continue; }
            const bool late = clock64() - idle > kMbarWaitCycles;
            if (late && lane == 0) {
                *abort = 1;
                if (l.a.wait_timeouts) atomicAdd(l.a.wait_timeouts, 1);
            }
            ok = !__any_sync(0xffffffffu, late || *abort);
        }
        if (__any_sync(0xffffffffu, !ok || *abort)) {         // TMEM is given back only when no product uses it
            if (elect_one()) tc_commit(drained);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained, 0u, &no_abort, nullptr, lane);
        }
    } else if (warp == 6) {
        // ---- the new tokens' rows to the cache, by the blocks that have their unit -----------------------------
        for (int i = 0; next_seg(i); ++i)
            if (sg.t1 == sg.units) latent_append<T>(l, sg.b, sg.S, sg.n, rt, l.row_tiles, lane);
    } else if (warp < 4) {
        // ---- softmax: two threads per query row, half of the tile's keys each -------------------------------
        const int half = warp >> 1, row = (warp & 1) * 32 + lane;
        const unsigned lane_base = (unsigned)(warp * 32) << 16;
        const float sl = l.a.scale_log2;
        const int token = (rt * kLatRows + row) / l.a.H_q;
        int done = 0, slot = 0, swaps = 0;
        bool ok = true;
        // a number from either thread of a row to the other one
        auto swap = [&](float mine, float& other) -> bool {
            float* at = s_pair + (swaps & 1) * 128;
            at[tid] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(pair + (warp & 1));
            const bool fine = tree_wait(pair + (warp & 1), swaps & 1, abort, l.a.wait_timeouts, lane);
            other = at[tid ^ 64];
            ++swaps;
            return fine;
        };
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            const bool alive = row < sg.rows;
            float m_ref = -INFINITY, sum_l = 0.f;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                ok = tree_wait(s_full + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                unsigned x[32];
                tc_ld32(x, tmem + lane_base + C::COL_S + buf * (kLatTile / 2));
                // (a row that does not exist computes along, unmasked, and decides nothing)
                int seen = kLatTile;
                if (alive) seen = sg.t0 + t < sg.units - 1 ? sg.count(t) : token + 1;
                seen -= half * 32;
                const unsigned see = seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u;
                tc_wait_ld();
                tc_fence_before();
                if (__any_sync(0xffffffffu, see != ~0u)) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (!((see >> k) & 1u)) x[k] = 0xff800000u;
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 32; k += 8)
#pragma unroll
                    for (int h = 0; h < 4; ++h) mx[h] = fmaxf(fmaxf(mx[h], __uint_as_float(x[k + 2 * h])), __uint_as_float(x[k + 2 * h + 1]));
                float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), m_other;
                ok = swap(m_tile, m_other);
                if (!ok) break;
                m_tile = fmaxf(m_tile, m_other);
                // (-inf - -inf is NaN: compares false, nothing to rescale; both warps of the rows decide alike)
                if (__any_sync(0xffffffffu, alive && (m_tile - m_ref) * sl > 8.f)) {
                    const float m_new = fmaxf(m_ref, m_tile);
                    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m_ref - m_new) * sl);
                    m_ref = m_new;
                    sum_l *= alpha;
                    if (t > 0) {
                        ok = tree_wait(pv_done + ((gt - 1) & 1), ((gt - 1) >> 1) & 1, abort, l.a.wait_timeouts, lane);
                        if (!ok) break;
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
                unsigned pk[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), sl2, sub2));
                    const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                    sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                    pk[k] = pack_bf16(p0, p1);
                }
                const float2 both = unpack_f32x2(add_f32x2(sum[0], sum[1]));
                sum_l += both.x + both.y;
                // the weights take the place of the slot's r part, which the scores were the last to read
                unsigned char* p_row = s_ring + slot * C::SLOT + (C::CH - 1) * C::CHUNK + row * 128;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<uint4*>(p_row + (((half * 4 + k) ^ (row & 7)) * 16)) = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready + buf);
                if (++slot == C::SLOTS) slot = 0;
            }
            if (!ok) break;
            const int rows_all = min(kLatRows, l.rows - rt * kLatRows);
            const int64_t orow = (int64_t)sg.b * l.rows + rt * kLatRows + row;
            if (tiles == 0) {
                if (sg.part < 0 && row < rows_all) {          // nothing to attend with: zeros and -inf
                    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<T*>(l.a.out) + orow * R) + half * (R / 16);
#pragma unroll 8
                    for (int c = 0; c < R / 16; ++c) dst[c] = make_uint4(0u, 0u, 0u, 0u);
                    if (half == 0) l.a.lse[orow] = -INFINITY;
                }
                continue;
            }
            done += tiles;
            ok = tree_wait(pv_done + ((done - 1) & 1), ((done - 1) >> 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            tc_fence_after();
            float total;
            ok = swap(sum_l, total);
            if (!ok) break;
            total += sum_l;
            const bool none = !alive || total == 0.f;         // nothing seen: zeros and -inf
            const float inv = none ? 0.f : 1.f / total;
#pragma unroll 1
            for (int c = 0; c < R / 2; c += 32) {
                unsigned o[32];
                tc_ld32(o, tmem + lane_base + c);
                tc_wait_ld();
                const int dim = (c >> 7) * 256 + half * 128 + (c & 127);
                if (sg.part >= 0) {
                    float4* dst = g.part_o + ((int64_t)sg.part * (R / 4) + dim / 4) * kLatRows + row;
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        dst[(k / 4) * kLatRows] = make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3]));
                } else if (row < rows_all) {
                    float f[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = none ? 0.f : __uint_as_float(o[k]) * inv;
                    T* dst = reinterpret_cast<T*>(l.a.out) + orow * R + dim;
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
                        *reinterpret_cast<uint4*>(dst + k) = make_uint4(pack_bf16(f[k], f[k + 1]), pack_bf16(f[k + 2], f[k + 3]),
                                                                        pack_bf16(f[k + 4], f[k + 5]), pack_bf16(f[k + 6], f[k + 7]));
                }
                __syncwarp();
            }
            tc_fence_before();
            if (half == 0) {
                if (sg.part >= 0) g.part_ml[(int64_t)sg.part * kLatRows + row] = none ? make_float2(-INFINITY, 0.f) : make_float2(m_ref * sl, total);
                else if (row < rows_all) l.a.lse[orow] = none ? -INFINITY : (m_ref * sl + log2f(total)) * LN2;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
        }
    }
    __syncthreads();                                          // (every role has come to its end)
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

// Merges the partial results of requests that several blocks share: out = sum_i e^{m_i - M} O_i / sum_i e^{m_i - M} l_i.
// A block: 64 dims of one (request, row tile); a warp has 8 rows x 4 pieces of four dims, so that it reads and writes whole sectors.
template <int R>
__global__ void __launch_bounds__(256) dsa_latent_merge_kernel(const LatentTcArgs g) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const LatentArgs& l = g.l;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int d0 = (idx % (R / 64)) * 64; idx /= R / 64;
    const int rt = idx % l.row_tiles, b = idx / l.row_tiles;
    const int u0 = g.sched[b], u1 = g.sched[b + 1], quota = g.sched[l.a.B + 1];
    const int g0 = u0 / quota, g1 = (u1 - 1) / quota;
    if (g0 == g1) return;
    int S, n;
    latent_lengths(l, b, S, n);
    const int row = warp * 8 + lane / 4, c4 = lane % 4;
    if (rt * kLatRows + row >= l.rows) return;
    const bool alive = row < n * l.a.H_q - rt * kLatRows;
    const int64_t orow = (int64_t)b * l.rows + rt * kLatRows + row;
    auto part = [&](int gi) { return (int64_t)(gi * l.row_tiles + rt) * 2 + (gi == g0 ? 1 : 0); };
    float top = -INFINITY, sum = 0.f;
    float4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (alive) {
        for (int gi = g0; gi <= g1; ++gi) top = fmaxf(top, g.part_ml[part(gi) * kLatRows + row].x);
#pragma unroll 2
        for (int gi = g0; gi <= g1; ++gi) {
            const float2 ml = g.part_ml[part(gi) * kLatRows + row];
            const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - top);
            sum = fmaf(w, ml.y, sum);
            const float4* o = g.part_o + (part(gi) * (R / 4) + d0 / 4 + c4) * kLatRows + row;
            if (ml.y == 0.f) continue;                        // (a part that saw nothing)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 x = o[k * 4 * kLatRows];
                acc[k].x = fmaf(w, x.x, acc[k].x); acc[k].y = fmaf(w, x.y, acc[k].y);
                acc[k].z = fmaf(w, x.z, acc[k].z); acc[k].w = fmaf(w, x.w, acc[k].w);
            }
        }
    }
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(l.a.out) + orow * R + d0 + c4 * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<uint2*>(out + k * 16) = none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(acc[k].x * inv, acc[k].y * inv), pack_bf16(acc[k].z * inv, acc[k].w * inv));
    if (d0 == 0 && c4 == 0) l.a.lse[orow] = none ? -INFINITY : (top + log2f(sum)) * LN2;
}

}  // namespace dsa
