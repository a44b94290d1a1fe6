// Attention of the tokens of prompts with expanded keys and values, bf16 (dsa_latent_prompt).
#pragma once
#include "dsa_prompt_args.cuh"
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kPrTile = 128;                       // keys per tile
constexpr int kPrRows = 128;                       // query rows per half of a block: the M of the products
constexpr int kPrBlock = 2 * kPrRows;
constexpr int kPrThreads = 320;

struct PromptMaps {
    CUtensorMap q, k, kr, v;
    int q_head, k_head, v_head;                    // 0: the map's head dimension has one entry (stride 0)
};

template <int D>
struct PromptCfg {
    static constexpr int KC = D / 64 + 1, VC = D / 64;                     // 64-element columns of a key (the last: k_rope), a value
    static constexpr int COL = kPrTile * 128;                              // bytes of one column of a tile
    static constexpr int Q_BYTES = 2 * KC * COL;
    static constexpr int RING = D == 128 ? 8 : 9;
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
    unsigned long long* full = reinterpret_cast<unsigned long long*>(s_ring + C::RING * C::COL);   // [RING] a column has landed
    unsigned long long* empty = full + C::RING;               // [RING] the products that read it are done
    unsigned long long* q_full = empty + C::RING;             // [2] a half's queries
    unsigned long long* s_full = q_full + 2;                  // [2] scores are in TMEM
    unsigned long long* p_ready = q_full + 4;                 // [2] weights are in TMEM
    unsigned long long* pv_done = q_full + 6;                 // [2] O holds the tile
    unsigned long long* drained = q_full + 8;
    int* s_misc = reinterpret_cast<int*>(q_full + 9);         // [0] TMEM address, [1] abort
    static_assert((2 * C::RING + 9) * 8 + 8 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tiles_q = (g.max_q_len + kPrBlock - 1) / kPrBlock;
    int idx = blockIdx.x;
    const int h = idx % g.H; idx /= g.H;
    const int b = idx % g.batch;
    const int first = (tiles_q - 1 - idx / g.batch) * kPrBlock;            // (the rows with the most keys first)

    if (warp == 8 && lane == 0) {
        for (int s = 0; s < 2 * C::RING; ++s) mbar_init(full + s, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full + s, 1); mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
        }
        mbar_init(drained, 1);
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
    // (the starts of the whole request decide which keys a query sees, whatever max_q_len leaves out)
    const int all_q = max(0, min(g.q_start[b + 1], g.q_tokens) - q0);
    // keys that query i sees: the first `limit(i)`
    auto limit = [&](int i) { return g.causal ? (int)max((int64_t)0, min((int64_t)nk, (int64_t)i + 1 + nk - all_q)) : nk; };
    int rows[2], len[2], tiles[2];                            // of either half: queries, keys that any of them sees, tiles of those
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        rows[s] = max(0, min(kPrRows, nq - first - s * kPrRows));
        len[s] = rows[s] > 0 ? limit(first + s * kPrRows + rows[s] - 1) : 0;
        tiles[s] = (len[s] + kPrTile - 1) / kPrTile;
    }
    const int n_tiles = max(tiles[0], tiles[1]);

    if (warp == 8) {
        // ---- copies: the columns of K(0), V(0), K(1), V(1), ... -------------------------------------------
        int slot = 0, round = 0, issued = 0;
        bool ok = true;
        if (lane == 0)
#pragma unroll 1
            for (int s = 0; s < 2; ++s)
                if (tiles[s] > 0) {
                    mbar_expect_tx(q_full + s, (unsigned)(C::KC * C::COL));
                    for (int c = 0; c < C::KC; ++c)
                        tma_col(s_q + (s * C::KC + c) * C::COL, &maps.q, 64 * c, h * maps.q_head, q0 + first + s * kPrRows, q_full + s);
                }
        __syncwarp();
        for (int j = 0; ok && j < n_tiles; ++j)
#pragma unroll 1
            for (int c = 0; ok && c < C::KC + C::VC; ++c) {
                if (round > 0) ok = tree_wait(empty + slot, (round - 1) & 1, abort, g.wait_timeouts, lane);
                if (!ok) break;
                if (lane == 0) {
                    unsigned char* dst = s_ring + slot * C::COL;
                    mbar_expect_tx(full + slot, (unsigned)C::COL);
                    const int tok = k0 + j * kPrTile;
                    if (c < C::KC - 1) tma_col(dst, &maps.k, 64 * c, h * maps.k_head, tok, full + slot);
                    else if (c == C::KC - 1) tma_col(dst, &maps.kr, 0, 0, tok, full + slot);
                    else tma_col(dst, &maps.v, 64 * (c - C::KC), h * maps.v_head, tok, full + slot);
                }
                __syncwarp();
                ++issued;
                if (++slot == C::RING) { slot = 0; ++round; }
            }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        volatile int no_abort = 0;
        for (int s = 0; s < 2; ++s)
            if (tiles[s] > 0) tree_wait(q_full + s, 0u, &no_abort, nullptr, lane);
        for (int c = max(0, issued - C::RING); c < issued; ++c)
            if (!tree_wait(full + c % C::RING, (c / C::RING) & 1, &no_abort, nullptr, lane)) break;
    } else if (warp == 9) {
        // ---- products: O_A += P_A V(j), S_A = Q_A K(j + 1), and the same for B ------------------------------
        constexpr unsigned kIdescS = instr_desc(kPrRows, kPrTile, false), kIdescO = instr_desc(kPrRows, D, true), kIdescO64 = instr_desc(kPrRows, 64, true);
        const unsigned q_desc = desc_low(smem_u32(s_q), 16), k_desc = desc_low(smem_u32(s_ring), 16), v_desc = desc_low(smem_u32(s_ring), C::COL);
        bool ok = true;
        // a tile's columns: (KC + VC) j + c in the order of the copies
        auto wait_col = [&](int c) { return tree_wait(full + c % C::RING, (c / C::RING) & 1, abort, g.wait_timeouts, lane); };
        auto free_cols = [&](int c, int n) {
            if (elect_one())
                for (int i = 0; i < n; ++i) tc_commit(empty + (c + i) % C::RING);
            __syncwarp();
        };
        auto scores = [&](int s, int j) -> bool {
            const int c0 = (C::KC + C::VC) * j;
            if (j == 0 && !tree_wait(q_full + s, 0u, abort, g.wait_timeouts, lane)) return false;
#pragma unroll
            for (int c = 0; c < C::KC; ++c) {
                if (!wait_col(c0 + c)) return false;
                tc_fence_after();
                if (elect_one()) {
                    const unsigned qa = q_desc + (s * C::KC + c) * (C::COL / 16), ka = k_desc + ((c0 + c) % C::RING) * (C::COL / 16);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) tc_mma_ss(tmem + s * kPrTile, qa + kk * 2, ka + kk * 2, kIdescS, c > 0 || kk > 0);
                    if (c == C::KC - 1) tc_commit(s_full + s);
                }
                __syncwarp();
            }
            return true;
        };
        auto values = [&](int s, int j) -> bool {
            const int c0 = (C::KC + C::VC) * j + C::KC;
            if (!tree_wait(p_ready + s, j & 1, abort, g.wait_timeouts, lane)) return false;
#pragma unroll
            for (int c = 0; c < C::VC; ++c)
                if (!wait_col(c0 + c)) return false;
            // values behind the request's last key, up to where the product stops: zero, whatever they were
            const int count = min(kPrTile, len[s] - j * kPrTile), there = nk - j * kPrTile;
            const int steps = (count + 15) / 16;
            if (there < steps * 16) {
                const int pieces = (steps * 16 - there) * 8;
                for (int i = lane; i < pieces * C::VC; i += 32) {
                    const int c = i / pieces, p = i - c * pieces;
                    *reinterpret_cast<uint4*>(s_ring + ((c0 + c) % C::RING) * C::COL + there * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            tc_fence_after();
            if (elect_one()) {
                const unsigned o = tmem + C::COL_O + s * D, p = tmem + s * kPrTile;
                const int slot = c0 % C::RING;
                if (C::VC == 1 || slot + 1 < C::RING) {
                    const unsigned va = v_desc + slot * (C::COL / 16);
                    for (int kk = 0; kk < steps; ++kk) tc_mma_ts(o, p + kk * 8, va + kk * (2048 / 16), kIdescO, j > 0 || kk > 0);
                } else {                                      // the two columns are the ring's last and first
                    for (int c = 0; c < C::VC; ++c) {
                        const unsigned va = v_desc + ((c0 + c) % C::RING) * (C::COL / 16);
                        for (int kk = 0; kk < steps; ++kk) tc_mma_ts(o + c * 64, p + kk * 8, va + kk * (2048 / 16), kIdescO64, j > 0 || kk > 0);
                    }
                }
                tc_commit(pv_done + s);
            }
            __syncwarp();
            return true;
        };
        for (int s = 0; ok && s < 2; ++s)
            if (tiles[s] > 0) ok = scores(s, 0);
        if (ok && n_tiles > 0) free_cols(0, C::KC);
        for (int j = 0; ok && j < n_tiles; ++j) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (ok && j < tiles[s]) ok = values(s, j);
                if (ok && s == 1) free_cols((C::KC + C::VC) * j + C::KC, C::VC);
                if (ok && j + 1 < tiles[s]) ok = scores(s, j + 1);
                if (ok && s == 1 && j + 1 < n_tiles) free_cols((C::KC + C::VC) * (j + 1), C::KC);
            }
        }
        if (__any_sync(0xffffffffu, !ok || *abort)) {         // TMEM is given back only when no product uses it
            if (elect_one()) tc_commit(drained);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained, 0u, &no_abort, nullptr, lane);
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
            unsigned x[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tc_ld32(x[c], s_addr + 32 * c);
            tc_wait_ld();
            const int seen = sees - j * kPrTile;
            if (__any_sync(0xffffffffu, seen < kPrTile)) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (c * 32 + k >= seen) x[c][k] = 0xff800000u;
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < 32; k += 2)
#pragma unroll
                for (int c = 0; c < 4; ++c) mx[c] = fmaxf(fmaxf(mx[c], __uint_as_float(x[c][k])), __uint_as_float(x[c][k + 1]));
            const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
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
            for (int half = 0; half < 2; ++half) {
                unsigned pk[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const unsigned* from = x[half * 2 + k / 16] + (k % 16) * 2;
                    const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(from[0]), __uint_as_float(from[1])), sl2, sub2));
                    const float p0 = fast_exp2(y.x), p1 = fast_exp2(y.y);
                    sum[k & 1] = add_f32x2(sum[k & 1], pack_f32x2(p0, p1));
                    pk[k] = pack_bf16(p0, p1);
                }
                tc_st32(s_addr + 32 * half, pk);
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
