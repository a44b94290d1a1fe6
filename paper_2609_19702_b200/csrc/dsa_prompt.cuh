// Attention of the tokens of prompts with expanded keys and values, bf16 (dsa_latent_prompt).
#pragma once
#include "dsa_prompt_args.cuh"
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kPrTile = 96;                        // keys per tile: two tiles of K and V fit beside 256 queries
constexpr int kPrRows = 128;                       // query rows per half of a block: the M of the products
constexpr int kPrBlock = 2 * kPrRows;
constexpr int kPrThreads = 352;

struct PromptMaps {
    CUtensorMap q, k, kr, v;
    int q_head, k_head, v_head;                    // 0: the map's head dimension has one entry (stride 0)
};

template <int D>
struct PromptCfg {
    static constexpr int KC = D / 64 + 1, VC = D / 64;                     // 64-element columns of a key (the last: k_rope), a value
    static constexpr int COL = kPrTile * 128, Q_COL = kPrRows * 128;       // bytes of one column of a tile, of a half's queries
    static constexpr int Q_BYTES = 2 * KC * Q_COL;
    static constexpr int SLOTS = D == 128 ? 2 : 4, RING = SLOTS * (KC + VC);   // tiles in flight, and their columns
    static constexpr int TAIL = 1024;
    static constexpr int SMEM = Q_BYTES + RING * COL + TAIL;
    static constexpr int COL_O = 2 * kPrTile, TMEM_COLS = 512;
    static_assert(SMEM <= 232448, "shared memory of an SM");
};

__device__ __forceinline__ void tma_col(void* dst, const CUtensorMap* map, int c0, int c1, int c2, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar)) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kPrThreads, 1) dsa_prompt_kernel(const PromptArgs g, const __grid_constant__ PromptMaps maps) {
    using C = PromptCfg<D>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned long long* full = reinterpret_cast<unsigned long long*>(s_ring + C::RING * C::COL);   // [SLOTS][2] a tile's K / V has landed
    unsigned long long* empty = full + 2 * C::SLOTS;          // [SLOTS][2] the products of either half that read it are done
    unsigned long long* q_full = empty + 2 * C::SLOTS;             // [2] a half's queries
    unsigned long long* s_full = q_full + 2;                  // [2] scores are in TMEM
    unsigned long long* p_ready = q_full + 4;                 // [2] weights are in TMEM
    unsigned long long* pv_done = q_full + 6;                 // [2] O holds the tile
    unsigned long long* drained = q_full + 8;                 // [2]
    unsigned long long* turn = q_full + 10;                   // [2] the other half has issued its products
    int* s_misc = reinterpret_cast<int*>(q_full + 12);        // [0] TMEM address, [1] abort
    static_assert((4 * C::SLOTS + 12) * 8 + 8 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int h = idx % g.H; idx /= g.H;
    const int b = idx % g.batch;
    const int from_end = idx / g.batch;                       // (the rows with the most keys first)

    if (warp == 8 && lane == 0) {
        for (int s = 0; s < 2 * C::SLOTS; ++s) { mbar_init(full + s, 1); mbar_init(empty + s, 2); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full + s, 1); mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
            mbar_init(drained + s, 1); mbar_init(turn + s, 1);
        }
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

    int q0, nq, k0, nk;
    prompt_range(g, b, q0, nq, k0, nk);
    // the request's last rows are in blocks of kPrBlock from the end; the first rows, with the fewest keys, are what is left
    const int tiles_r = (nq + kPrBlock - 1) / kPrBlock, tile = tiles_r - 1 - from_end;
    const int first = tile <= 0 ? 0 : nq - (from_end + 1) * kPrBlock, n_rows = tile < 0 ? 0 : tile == 0 ? nq - from_end * kPrBlock : kPrBlock;
    // (the starts of the whole request decide which keys a query sees, whatever max_q_len leaves out)
    const int all_q = max(0, min(g.q_start[b + 1], g.q_tokens) - q0);
    // keys that query i sees: the first `limit(i)`
    auto limit = [&](int i) { return g.causal ? (int)max((int64_t)0, min((int64_t)nk, (int64_t)i + 1 + nk - all_q)) : nk; };
    int rows[2], len[2], tiles[2];                            // of either half: queries, keys that any of them sees, tiles of those
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        rows[s] = max(0, min(kPrRows, n_rows - s * kPrRows));
        len[s] = rows[s] > 0 ? limit(first + s * kPrRows + rows[s] - 1) : 0;
        tiles[s] = (len[s] + kPrTile - 1) / kPrTile;
    }
    const int n_tiles = max(tiles[0], tiles[1]);

    if (warp == 8) {
        // ---- copies: K(0), V(0), K(1), V(1), ... -----------------------------------------------------------
        int issued = 0;
        bool ok = true;
        if (lane == 0)
#pragma unroll 1
            for (int s = 0; s < 2; ++s)
                if (tiles[s] > 0) {
                    mbar_expect_tx(q_full + s, (unsigned)(C::KC * C::Q_COL));
                    for (int c = 0; c < C::KC; ++c)
                        tma_col(s_q + (s * C::KC + c) * C::Q_COL, &maps.q, 64 * c, h * maps.q_head, q0 + first + s * kPrRows, q_full + s);
                }
        __syncwarp();
        for (int j = 0; ok && j < n_tiles; ++j) {
            const int slot = j % C::SLOTS, round = j / C::SLOTS, tok = k0 + j * kPrTile;
            unsigned char* dst = s_ring + slot * (C::KC + C::VC) * C::COL;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                unsigned long long* bar = full + 2 * slot + v;
                if (ok && round > 0) ok = tree_wait(empty + 2 * slot + v, (round - 1) & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(bar, (unsigned)((v ? C::VC : C::KC) * C::COL));
                    if (v == 0) {
                        for (int c = 0; c < C::KC - 1; ++c) tma_col(dst + c * C::COL, &maps.k, 64 * c, h * maps.k_head, tok, bar);
                        tma_col(dst + (C::KC - 1) * C::COL, &maps.kr, 0, 0, tok, bar);
                    } else {
                        for (int c = 0; c < C::VC; ++c) tma_col(dst + (C::KC + c) * C::COL, &maps.v, 64 * c, h * maps.v_head, tok, bar);
                    }
                }
                __syncwarp();
                ++issued;
            }
        }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        volatile int no_abort = 0;
        for (int s = 0; s < 2; ++s)
            if (tiles[s] > 0) tree_wait(q_full + s, 0u, &no_abort, nullptr, lane);
        for (int c = max(0, issued - 2 * C::SLOTS); c < issued; ++c)
            if (!tree_wait(full + c % (2 * C::SLOTS), (c / (2 * C::SLOTS)) & 1, &no_abort, nullptr, lane)) break;
    } else if (warp >= 9) {
        // ---- products of a half: O += P V(j), S = Q K(j + 1).  A warp for either half, so that what the one waits for and works
        // out is behind the other's products.
        constexpr unsigned kIdescS = instr_desc(kPrRows, kPrTile, false), kIdescO = instr_desc(kPrRows, D, true);
        const int s = warp - 9;
        const unsigned q_desc = desc_low(smem_u32(s_q), 16) + s * C::KC * (C::Q_COL / 16), k_desc = desc_low(smem_u32(s_ring), 16);
        const unsigned v_desc = desc_low(smem_u32(s_ring), C::COL), s_addr = tmem + s * kPrTile, o_addr = tmem + C::COL_O + s * D;
        bool ok = true;
        // Step j: O += P V(j) and S = Q K(j + 1), issued in one go.  The halves take turns, so that one's softmax runs while the
        // other's products do; left to themselves they fall in step, and the tensor pipe waits for both.  The weights, which come
        // last, are waited for last: every look at a barrier costs some 250 cycles behind the products that are still queued.
        for (int j = -1; ok && j < n_tiles; ++j) {
            const bool pv = j >= 0 && j < tiles[s], next = j + 1 < tiles[s], last = j + 1 >= n_tiles;
            const int vs = j < 0 ? 0 : j % C::SLOTS, ks = (j + 1) % C::SLOTS;
            if (!last) ok = tree_wait(full + 2 * ks, ((j + 1) / C::SLOTS) & 1, abort, g.wait_timeouts, lane);
            if (ok && j >= 0) ok = tree_wait(full + 2 * vs + 1, (j / C::SLOTS) & 1, abort, g.wait_timeouts, lane);
            if (ok && j < 0 && next) ok = tree_wait(q_full + s, 0u, abort, g.wait_timeouts, lane);
            if (!ok) break;
            const int count = min(kPrTile, len[s] - j * kPrTile), there = nk - j * kPrTile, steps = (count + 15) / 16;
            // values behind the request's last key, up to where the product stops: zero, whatever they were
            if (pv && there < steps * 16) {
                const int pieces = (steps * 16 - there) * 8;
                for (int i = lane; i < pieces * C::VC; i += 32) {
                    const int c = i / pieces, p = i - c * pieces;
                    *reinterpret_cast<uint4*>(s_ring + (vs * (C::KC + C::VC) + C::KC + c) * C::COL + there * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            if (s == 1 || j >= 0) ok = tree_wait(turn + s, (s == 1 ? j + 1 : j) & 1, abort, g.wait_timeouts, lane);
            if (ok && pv) ok = tree_wait(p_ready + s, j & 1, abort, g.wait_timeouts, lane);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                if (pv) {
                    const unsigned va = v_desc + (vs * (C::KC + C::VC) + C::KC) * (C::COL / 16);
                    tc_mma_ts(o_addr, s_addr, va, kIdescO, j > 0);
                    if (steps == kPrTile / 16) {
#pragma unroll
                        for (int kk = 1; kk < kPrTile / 16; ++kk) tc_mma_ts_add(o_addr, s_addr + kk * 8, va + kk * (2048 / 16), kIdescO);
                    } else {
                        for (int kk = 1; kk < steps; ++kk) tc_mma_ts_add(o_addr, s_addr + kk * 8, va + kk * (2048 / 16), kIdescO);
                    }
                    tc_commit(pv_done + s);
                }
                if (next) {
#pragma unroll
                    for (int c = 0; c < C::KC; ++c) {
                        const unsigned qa = q_desc + c * (C::Q_COL / 16), ka = k_desc + (ks * (C::KC + C::VC) + c) * (C::COL / 16);
                        if (c == 0) tc_mma_ss(s_addr, qa, ka, kIdescS, false);
                        else tc_mma_ss_add(s_addr, qa, ka, kIdescS);
#pragma unroll
                        for (int kk = 1; kk < 4; ++kk) tc_mma_ss_add(s_addr, qa + kk * 2, ka + kk * 2, kIdescS);
                    }
                    tc_commit(s_full + s);
                }
                mbar_arrive(turn + 1 - s);
                if (j >= 0) tc_commit(empty + 2 * vs + 1);
                if (!last) tc_commit(empty + 2 * ks);
            }
            __syncwarp();
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
        const unsigned s_addr = tmem + lane_base + s * kPrTile, o_addr = tmem + lane_base + C::COL_O + s * D;
        const float sl = g.scale_log2;
        const bool alive = row < rows[s];
        const int sees = alive ? limit(first + s * kPrRows + row) : 0x7fffffff;   // (a row that does not exist computes along and decides nothing)
        float m_ref = -INFINITY, sum_l = 0.f;
        bool ok = true;
        for (int j = 0; ok && j < tiles[s]; ++j) {
            ok = tree_wait(s_full + s, j & 1, abort, g.wait_timeouts, lane);
            if (!ok) break;
            tc_fence_after();
            unsigned x[3][32];
#pragma unroll
            for (int c = 0; c < 3; ++c) tc_ld32(x[c], s_addr + 32 * c);
            tc_wait_ld();
            const int seen = sees - j * kPrTile;
            if (__any_sync(0xffffffffu, seen < kPrTile)) {
#pragma unroll
                for (int c = 0; c < 3; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (c * 32 + k >= seen) x[c][k] = 0xff800000u;
            }
            float mx[3] = {-INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < 32; k += 2)
#pragma unroll
                for (int c = 0; c < 3; ++c) mx[c] = fmaxf(fmaxf(mx[c], __uint_as_float(x[c][k])), __uint_as_float(x[c][k + 1]));
            const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), mx[2]);
            // (-inf - -inf is NaN: compares false, nothing to rescale)
            if (__any_sync(0xffffffffu, alive && (m_tile - m_ref) * sl > 8.f)) {
                const float m_new = fmaxf(m_ref, m_tile);
                const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m_ref - m_new) * sl);
                m_ref = m_new;
                sum_l *= alpha;
                if (j > 0) {
                    ok = tree_wait(pv_done + s, (j - 1) & 1, abort, g.wait_timeouts, lane);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        unsigned o[32];
                        tc_ld32(o, o_addr + c);
                        tc_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                        tc_st32(o_addr + c, o);
                    }
                }
            }
            const float sub = m_ref == -INFINITY ? 0.f : m_ref * sl;
            const unsigned long long sl2 = pack_f32x2(sl, sl), sub2 = pack_f32x2(-sub, -sub);
            unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                unsigned pk[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[c][2 * k]), __uint_as_float(x[c][2 * k + 1])), sl2, sub2));
                    const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                    sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                    pk[k] = pack_bf16(p0, p1);
                }
                tc_st16(s_addr + 16 * c, pk);
            }
            const float2 both = unpack_f32x2(add_f32x2(sum[0], sum[1]));
            sum_l += both.x + both.y;
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + s);
        }
        // ---- results ------------------------------------------------------------------------------------
        if (ok && tiles[s] > 0) ok = tree_wait(pv_done + s, (tiles[s] - 1) & 1, abort, g.wait_timeouts, lane);
        tc_fence_after();
        if (ok && (warp & 3) * 32 < rows[s]) {
            const bool none = sum_l == 0.f;                    // nothing seen: zeros and -inf
            const float inv = none ? 0.f : 1.f / sum_l;
            const int64_t orow = (int64_t)(q0 + first + s * kPrRows + row) * g.H + h;
            T* dst = reinterpret_cast<T*>(g.out) + orow * D;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                unsigned o[32];
                if (tiles[s] > 0) {
                    tc_ld32(o, o_addr + c);
                    tc_wait_ld();
                }
                if (alive) {
                    float f[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = none ? 0.f : __uint_as_float(o[k]) * inv;
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
                        *reinterpret_cast<uint4*>(dst + c + k) = make_uint4(pack_bf16(f[k], f[k + 1]), pack_bf16(f[k + 2], f[k + 3]),
                                                                            pack_bf16(f[k + 4], f[k + 5]), pack_bf16(f[k + 6], f[k + 7]));
                }
                __syncwarp();
            }
            if (alive) g.lse[orow] = none ? -INFINITY : (m_ref * sl + log2f(sum_l)) * LN2;
        }
        tc_fence_before();
    }
    __syncthreads();                                          // (every role has come to its end)
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

}  // namespace dsa
