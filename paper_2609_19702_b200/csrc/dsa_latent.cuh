// Attention of new tokens over a latent cache, bf16 (dsa_latent_step).
//
// A cached row is key and value of all heads at once, so the query rows (token, head) of a request are the M of two products over the
// same tile of keys in shared memory: S = Q K^T over the R + P numbers of a row, and O += W V with V the first R of them and
// W = 2^(x - m), x the scores in base-2 units.  m, a row's reference, follows its running maximum only when that has grown by more
// than 8: a weight is then at most 2^8, O and the sums are float32 and bear that, and O is seldom rescaled.  W is rounded to bf16,
// the type that V has in the product (relative error of half a step whatever m is); the sum that divides O is of the weights
// before that rounding, in float32.
//
// What bounds it: reading the rows once.  A tile of 64 keys is 73.7 KB (R 512, P 64): 1.7 us of one SM's share of HBM, and about
// 1800 cycles, 1 us, of its tensor pipe (36 products of N 64 at 33 cycles, 8 of N 256 at 80).  So 64 query rows fit under the
// copies, and few rows cost the same; more than 64 are the pair kernel's.  The M of 64 is the .ws form: a half of the N
// columns in either half of the tensor memory's lanes, so that four warps have two threads a row, for softmax and results.
// Shared memory holds q (73.7 KB) and two tiles (four with R 256); what a slot cannot wait for is cut up: a tile lands
// in parts of three 128-byte columns, the scores of each part begin as it lands, and its halves are freed one by one as the products
// with V have read them.  W takes the place of the slot's r column, which only the scores read.  Scores and products with V are
// issued by a warp each, because every look at a barrier costs an issuing warp some 250 cycles behind queued products.
// Rows are copied by 128 threads, 16 bytes at a time: tensor-map copies, with boxes within a page, take 70 to 90 cycles each at
// the least and arrive later (64 x 16 heads, threads / tensor maps: pages of 64: 64.7 / 68 us, 16: 65 / 81, 24: 65 / 118, 1: 69 / 212,
// one request of 600 tokens 11.3 / 13.1).
//
// Measured: 64 requests x 16 heads, lengths up to 8190 (304 MB of rows, 47 us at the measured copy rate): 64.7 us, 4.7 TB/s.  Some
// 4 us go by before the first tile has landed (lengths, then pages, then rows), 3 to 5 in the merge of the parts and its launch, the
// rest in begun and ended items.  One request of about 600 tokens: 11 us, four dependent reads and one launch.
#pragma once
#include "dsa_latent_args.cuh"
#include "dsa_tc.cuh"

namespace dsa {

constexpr int kLatTile = 64;                       // tokens per tile
constexpr int kLatRows = 64;                       // query rows per block: the M of the products
constexpr int kLatThreads = 384;
constexpr int kRowLoaders = 128;                   // of them: copy rows of the cache
constexpr int kLatMergeThreads = 256;

struct LatentTcArgs {
    LatentArgs l;
    int groups;                                    // shares that the work is cut into, or
    int cluster;                                   // > 0: blocks of a cluster that have one item to themselves
    int min_units;                                 // units of work that a block takes at least
    int box_shift;                                 // pairs: logarithm of the tokens per tensor-map copy of the cache
    unsigned page_mul;                             // position / block_size = (position * page_mul) >> page_shift
    int page_shift;
    int q_rows;                                    // rows of q per copy: fewer than a block's where a request has fewer
    int blk_coord;                                 // pairs: 0: the map's outer dimension has one entry (stride 0)
    float2* part_ml;                               // workspace: [blocks * 2][64] maximum (base 2) and sum
    float4* part_o;                                // [blocks * 2][R / 4][64]
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
    static constexpr int LAND = (CH + 2) / 3;                              // parts of a slot that land on their own: three columns each
    static constexpr int GROUPS = R / 256;                                 // and that are freed on their own: what a product with V reads
    static constexpr int TAIL = 2048;
    static constexpr int SMEM = Q_BYTES + SLOTS * SLOT + TAIL;
    static constexpr int PART_LD = R + 4;                                  // row of a partial result in shared memory, in floats
    static_assert(kLatRows * PART_LD * 4 <= SLOTS * SLOT, "the partial result takes the ring's place");
    static constexpr int COL_S = R / 2, TMEM_COLS = R == 512 ? 512 : 256;
    static_assert(SMEM <= 232448, "shared memory of an SM");
};

__device__ __forceinline__ void tma_box3(void* dst, const CUtensorMap* map, int c0, int c1, int c2, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar)) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T with 64 rows: the first half of the N columns in lanes 0-63, the second in lanes 64-127.  Two
// forms, because what goes with a predicate costs the issuing lane more than the product costs the tensor pipe (56 against 33
// cycles with N = 64).
__device__ __forceinline__ void tc_mma_ws(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"((unsigned)acc), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tc_mma_ws_add(unsigned d, unsigned a_low, unsigned b_low, unsigned idesc) {
    asm volatile("{\n.reg .b64 a, b;\nmov.b64 a, {%1, %4};\nmov.b64 b, {%2, %4};\n"
                 "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], a, b, %3, 1;\n}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(kDescHigh) : "memory");
}
// ---- shares -------------------------------------------------------------------------------------------------
// The work is a list of items: for every request the row tiles (ROWS query rows) that have tokens which exist, for each of them
// a unit per key tile (KT tokens; the last unit: the new tokens).  End to end they are cut into shares of equal size, one per
// block (or pair of blocks), so that every one has the same number of tiles whatever the lengths are.  An item that is cut
// leaves partial results, which the merge kernel joins.
// To begin an item costs about as much as two tiles (its q, the last one's results), so where shares are large every item counts
// two units more, at its front.
template <int KT, int ROWS, bool L2 = false>
struct LatentItems {
    int S, n, items, units;                        // of a request: lengths, items, and units of each
    __device__ __forceinline__ LatentItems(const LatentArgs& l, int b) {
        latent_lengths<L2>(l, b, S, n);
        items = n > 0 ? (n * l.a.H_q + ROWS - 1) / ROWS : 1;
        units = n > 0 ? (S + KT - 1) / KT + 1 : 1;
    }
};

struct LatentShares {
    int before, quota, setup;                      // units in front of request `b0`; of a share; that an item counts for its beginning
};

// By every thread of a block: units in front of request b0, where a thread has the stretch [b0, b1) of them, in order.
// s_scan: shared, two numbers per warp.
template <int KT, int ROWS, bool L2 = false>
__device__ __forceinline__ LatentShares latent_shares(const LatentArgs& l, int groups, int min_units, int b0, int b1, int2* s_scan) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    int sum = 0, items = 0;
    for (int b = b0; b < b1; ++b) {
        const LatentItems<KT, ROWS, L2> x(l, b);
        sum += x.items * x.units;
        items += x.items;
    }
    int before = sum, items_before = items;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, before, off), y = __shfl_up_sync(0xffffffffu, items_before, off);
        if (lane >= off) { before += x; items_before += y; }
    }
    if (lane == 31) s_scan[warp] = make_int2(before, items_before);
    before -= sum;
    items_before -= items;
    __syncthreads();
    int total = 0, all = 0;
    for (int w = 0; w < warps; ++w) {
        const int2 x = s_scan[w];
        if (w < warp) { before += x.x; items_before += x.y; }
        total += x.x;
        all += x.y;
    }
    LatentShares r;
    r.setup = total >= 8 * groups ? 2 : 0;
    r.before = before + r.setup * items_before;
    r.quota = max(min_units, (total + r.setup * all + groups - 1) / groups);
    return r;
}

// What a share has of one item: tiles [t0, t1) of `all`, the last of which are the new tokens.
template <int KT>
struct LatentSeg {
    int b, rt, S, n, t0, t1, all, rows, part;      // b < 0: nothing any more.  rows: query rows of tokens that exist (of the item's).
                                                   // part: 0 / 1, the partial result's place; -1: the whole item
    int zeros;                                     // > 0: the request's query rows from here on have no item, and this share sees to them
    __device__ __forceinline__ int tiles() const { return t1 - t0; }
    __device__ __forceinline__ bool cached(int t) const { return t0 + t < all - 1; }
    __device__ __forceinline__ int count(int t) const { return cached(t) ? min(KT, S - (t0 + t) * KT) : n; }   // tokens of its tile t
};

// A share's place in the list, moved on from item to item by one warp.
template <int KT, int ROWS>
struct LatentCursor {
    int b, at, left;                               // request, unit of it, units left
    __device__ __forceinline__ LatentSeg<KT> next(const LatentArgs& l, int setup) {
        LatentSeg<KT> sg = {};
        sg.b = -1;
        if (left <= 0) return sg;
        const LatentItems<KT, ROWS> x(l, b);
        const int units = x.units + setup, pos = at % units, end = min(units, pos + left);
        sg.b = b;
        sg.rt = at / units;
        sg.S = x.S;
        sg.n = x.n;
        sg.all = x.n > 0 ? x.units : 0;
        sg.t0 = min(sg.all, max(0, pos - setup));
        sg.t1 = min(sg.all, max(0, end - setup));
        sg.rows = min(ROWS, x.n * l.a.H_q - sg.rt * ROWS);
        sg.part = pos == 0 && end == units ? -1 : pos > 0 ? 0 : 1;
        sg.zeros = at == 0 && x.items * ROWS < l.rows ? x.items * ROWS : 0;
        left -= end - pos;
        at += end - pos;
        if (at == x.items * units) { ++b; at = 0; }
        return sg;
    }
};

// By a whole block: where share `share` begins.  place: shared; request (-1: it is empty), unit of it, units, set-up units.
template <int KT, int ROWS>
__device__ __forceinline__ void latent_first(const LatentTcArgs& g, int share, int2* s_scan, int* place) {
    const LatentArgs& l = g.l;
    const int tid = threadIdx.x, B = l.a.B, per = (B + (int)blockDim.x - 1) / (int)blockDim.x, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    if (tid == 0) { place[0] = -1; place[2] = 0; }
    const LatentShares sh = latent_shares<KT, ROWS>(l, g.groups, g.min_units, b0, b1, s_scan);      // (has a barrier)
    const int first = share * sh.quota;                       // (below 2^31: see the host's bound of the units)
    int before = sh.before;
    for (int b = b0; b < b1; ++b) {
        const LatentItems<KT, ROWS> x(l, b);
        const int units = x.items * (x.units + sh.setup);
        if (first >= before && first < before + units) { place[0] = b; place[1] = first - before; }
        // (units left in the list: the last request knows)
        if (b == B - 1) place[2] = max(0, min(sh.quota, before + units - first));
        before += units;
    }
    if (tid == 0) place[3] = sh.setup;
    __syncthreads();
}

// What is left to one warp of a share: the new tokens' rows to the cache (by the shares that have their tile: tokens first,
// first + step, ...), and zeros for the query rows that no item has.
template <int R, int ROWS, int KT>
__device__ __forceinline__ void latent_rest(const LatentArgs& l, const LatentSeg<KT>& sg, int first, int step, int lane) {
    if (sg.t1 == sg.all) latent_append<__nv_bfloat16>(l, sg.b, sg.S, sg.n, first, step, lane);
    if (sg.zeros > 0) {
        uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(l.a.out) + ((int64_t)sg.b * l.rows + sg.zeros) * R);
        const int pieces = (l.rows - sg.zeros) * (R / 8);
        for (int i = lane; i < pieces; i += 32) out[i] = make_uint4(0u, 0u, 0u, 0u);
        for (int r = sg.zeros + lane; r < l.rows; r += 32) l.a.lse[(int64_t)sg.b * l.rows + r] = -INFINITY;
    }
}

// The results of 64 query rows by the four warps that have their TMEM lanes, two threads a row (half 0 / 1: dims 0-127 / 128-255 of
// every 256): to out and lse, or, part >= 0, what the merge needs (in s_part and s_ml, where the blocks of a cluster merge).  m: the
// reference in base-2 units, total: the row's sum.
template <int R>
__device__ __forceinline__ void latent_results(const LatentTcArgs& g, unsigned tmem, int64_t orow, int rows_all, int row, int half, int part,
                                               bool any, bool alive, float m, float total, float* s_part = nullptr, float2* s_ml = nullptr) {
    const LatentArgs& l = g.l;
    const bool none = !alive || total == 0.f;                 // nothing seen: zeros and -inf
    const float inv = none ? 0.f : 1.f / total;
    const bool mine = part >= 0 ? alive && any : row < rows_all;           // (of a part nobody reads the other rows)
    if (__any_sync(0xffffffffu, mine)) {
        unsigned o[2][32];                                    // (the next columns are on their way while these are stored)
        if (any) tc_ld32(o[0], tmem);
#pragma unroll
        for (int c = 0; c < R / 2; c += 32) {
            const unsigned* x = o[(c / 32) & 1];
            if (any) {
                tc_wait_ld();
                if (c + 32 < R / 2) tc_ld32(o[(c / 32 + 1) & 1], tmem + c + 32);
            }
            if (mine) {
                const int dim = (c >> 7) * 256 + half * 128 + (c & 127);
                if (part >= 0 && s_part) {
                    float4* dst = reinterpret_cast<float4*>(s_part + row * LatentCfg<R>::PART_LD + dim);
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        dst[k / 4] = make_float4(__uint_as_float(x[k]), __uint_as_float(x[k + 1]), __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                } else if (part >= 0) {
                    float4* dst = g.part_o + ((int64_t)part * (R / 4) + dim / 4) * kLatRows + row;
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        dst[(k / 4) * kLatRows] = make_float4(__uint_as_float(x[k]), __uint_as_float(x[k + 1]), __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                } else {
                    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(l.a.out) + orow * R + dim;
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        unsigned y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[e] = none ? 0u : pack_bf16(__uint_as_float(x[k + 2 * e]) * inv, __uint_as_float(x[k + 2 * e + 1]) * inv);
                        *reinterpret_cast<uint4*>(dst + k) = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                }
            }
            __syncwarp();
        }
        tc_fence_before();
    }
    if (half == 0) {
        if (part >= 0) (s_ml ? s_ml + row : g.part_ml + (int64_t)part * kLatRows + row)[0] = none ? make_float2(-INFINITY, 0.f) : make_float2(m, total);
        else if (row < rows_all) l.a.lse[orow] = none ? -INFINITY : (m + log2f(total)) * LN2;
    }
    __syncwarp();
}

// Copies of 16 rows of a tile by one warp, straight from where each of them lies.  Eight lanes have 128 bytes (a column) of a row, so that a copy of
// 16 bytes by every lane is four whole lines in either memory; rows behind the last token arrive as zeros.  A tile's
// rows cost 16 such copies a column with addresses that are worked out once, about what a tensor-map copy of the same bytes takes,
// and it is the same whatever the pages are.
template <int R>
struct LatentRows {
    static constexpr int ROWS = kLatTile / (kRowLoaders / 32), K = ROWS / 4;
    const LatentArgs& l;
    int first, piece, row4;                                   // first row; this lane's piece of a column, its row of every four
    unsigned to[K];                                           // its places in a tile
    const __nv_bfloat16* from[K];
    bool there[K];
    __device__ __forceinline__ LatentRows(const LatentArgs& args, unsigned char* ring, int w, int lane) : l(args), first(w * ROWS), piece(lane & 7), row4(lane >> 3) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = first + 4 * k + row4;
            to[k] = smem_u32(ring) + r * 128 + ((piece ^ (r & 7)) * 16);
        }
    }
    // What a lane sees to: row first + lane % 16 of tile t: its page (or request) and token.  Ahead of at().
    __device__ __forceinline__ void find(const LatentTcArgs& g, const LatentSeg<kLatTile>& sg, int t, int& page, int& token) const {
        page = sg.b;
        token = (sg.t0 + t) * kLatTile + first + ((int)threadIdx.x & (ROWS - 1));
        if (!l.a.block_table || !sg.cached(t)) return;
        const int bi = (int)(((unsigned long long)(unsigned)token * g.page_mul) >> g.page_shift);
        token -= bi * l.a.block_size;
        page = l.a.block_table[(int64_t)sg.b * l.a.max_blocks + min(bi, l.a.max_blocks - 1)];
    }
    // The rows of tile t, which find() has looked up.
    __device__ __forceinline__ void at(const LatentTcArgs& g, const LatentSeg<kLatTile>& sg, int t, int page, int token) {
        using T = __nv_bfloat16;
        const T* cache = reinterpret_cast<const T*>(l.a.k);
        if (l.a.block_table) page = max(0, min(page, l.a.num_blocks - 1));
        const T* mine = sg.cached(t) ? cache + page * l.a.stride_b + token * l.a.stride_tok
                                     : reinterpret_cast<const T*>(l.a.k_new) + ((int64_t)sg.b * l.N + first + ((int)threadIdx.x & (ROWS - 1))) * (l.R + l.P);
        const int count = sg.count(t) - first;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = 4 * k + row4;
            const T* x = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), r)) + piece * 8;
            there[k] = r < count;
            from[k] = there[k] ? x : cache;                   // (an address that is there; nothing is read)
        }
    }
    // Column c of the rows to a slot.
    __device__ __forceinline__ void copy(int slot, int c) const {
        using C = LatentCfg<R>;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool some = there[k] && (c < C::CH - 1 || piece < l.P / 8);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                         ::"r"(to[k] + slot * C::SLOT + c * C::CHUNK), "l"(some ? from[k] + c * 64 : from[k]), "r"(some ? 16 : 0) : "memory");
        }
    }
};

template <int R>
__global__ void __launch_bounds__(kLatThreads, 1) dsa_latent_kernel(const LatentTcArgs g, const __grid_constant__ LatentMaps maps) {
    using C = LatentCfg<R>;
    using Seg = LatentSeg<kLatTile>;
    using T = __nv_bfloat16;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* s_q = smem;
    unsigned char* s_ring = smem + C::Q_BYTES;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(s_ring + C::SLOTS * C::SLOT);
    constexpr int LANDS = C::SLOTS * C::LAND, PARTS = C::SLOTS * C::GROUPS;
    unsigned long long* full = bars;                          // [slot][LAND] has landed
    unsigned long long* empty = bars + LANDS;                 // [slot][GROUPS] the products that read it are done
    unsigned long long* s_full = empty + PARTS;               // [2] scores are in TMEM
    unsigned long long* p_ready = s_full + 2;                 // [2] weights are in shared memory
    unsigned long long* pv_done = s_full + 4;                 // [2] O holds the tile
    unsigned long long* info_full = s_full + 6;               // [2] the next share is known
    unsigned long long* info_empty = s_full + 8;              // [2] every warp has read it
    unsigned long long* q_full = s_full + 10;
    unsigned long long* q_empty = s_full + 11;                // the scores of a share's last tile are done
    unsigned long long* o_free = s_full + 12;                 // O has been read
    unsigned long long* drained = s_full + 13;                // [2]
    unsigned long long* pair = s_full + 15;                   // [2] the two warps of a row have written to s_pair
    Seg* s_info = reinterpret_cast<Seg*>(s_full + 18);        // [2]
    float* s_pair = reinterpret_cast<float*>(s_info + 2);     // [2][128] maxima and sums that the two halves of a row exchange
    int* s_misc = reinterpret_cast<int*>(s_pair + 256);       // [0] TMEM address, [1] abort, [2..] first request, its first unit, units, set-up units
    int2* s_scan = reinterpret_cast<int2*>(s_misc + 8);       // [kLatThreads / 32]
    static_assert((LANDS + PARTS + 18) * 8 + 2 * sizeof(Seg) + 1024 + 32 + kLatThreads / 4 <= C::TAIL, "tail of the shared memory");
    volatile int* abort = s_misc + 1;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const LatentArgs& l = g.l;
    const int share = (int)blockIdx.x;
    // a cluster's merge: O of this block's part (rows padded against bank conflicts) and per row (maximum in base-2 units, sum)
    float* s_part = reinterpret_cast<float*>(s_ring);
    float2* s_ml = reinterpret_cast<float2*>(s_q);

    if (warp == 4 && lane == 0) {
        for (int s = 0; s < LANDS; ++s) mbar_init(full + s, kRowLoaders);
        for (int s = 0; s < PARTS; ++s) mbar_init(empty + s, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1); mbar_init(p_ready + s, 4); mbar_init(pv_done + s, 1);
            mbar_init(info_full + s, 1); mbar_init(info_empty + s, 7);
            mbar_init(pair + s, 2); mbar_init(drained + s, 1);
        }
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(o_free, 4);
        s_misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 6) {
        if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q) : "memory");
    } else if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(s_misc)), "r"((unsigned)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_fence_before();
    }
    // rows of q that no copy fills: zeros (nobody reads their results, but leftovers would cost power)
    for (int i = g.q_rows * 8 + tid; i < kLatRows * 8; i += kLatThreads)
#pragma unroll
        for (int c = 0; c < C::CH; ++c) *reinterpret_cast<uint4*>(s_q + c * kLatRows * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = (unsigned)*reinterpret_cast<volatile int*>(s_misc);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    bool merged = false;                                      // several blocks of the cluster have parts of the item
    int item_b = 0, item_rt = 0;
    if (g.cluster > 0) {
        const int rank = share % g.cluster, item = share / g.cluster;
        item_b = item / l.row_tiles;
        item_rt = item % l.row_tiles;
        // (the request's pages are fetched into L2 while its lengths are read: from cold caches 17.6 -> 17.1 us, one request of 600 tokens)
        if (l.a.block_table && warp >= 8) {
            const int at = (tid - 256) * 32;
            if (at < l.a.max_blocks) asm volatile("prefetch.global.L2 [%0];" ::"l"(l.a.block_table + (int64_t)item_b * l.a.max_blocks + at) : "memory");
        }
        const LatentItems<kLatTile, kLatRows> x(l, item_b);
        const int per = (x.units + g.cluster - 1) / g.cluster, left = item_rt < x.items ? max(0, min(per, x.units - rank * per)) : 0;
        merged = item_rt < x.items && x.units > per;
        if (tid == 0) { s_misc[2] = item_b; s_misc[3] = item_rt * x.units + rank * per; s_misc[4] = left; s_misc[5] = 0; }
        if (merged && left == 0 && tid < kLatRows) s_ml[tid] = make_float2(-INFINITY, 0.f);
        __syncthreads();
    } else {
        latent_first<kLatTile, kLatRows>(g, share, s_scan, s_misc + 2);
    }

    Seg sg;
    auto next_seg = [&](int i) -> bool {
        if (!tree_wait(info_full + (i & 1), (i >> 1) & 1, abort, l.a.wait_timeouts, lane)) return false;
        sg = s_info[i & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty + (i & 1));
        return sg.b >= 0;
    };

    if (warp == 4) {
        // ---- what to work on; copies of q ---------------------------------------------------------------------
        const int setup = s_misc[5];
        LatentCursor<kLatTile, kLatRows> cur = {s_misc[2], s_misc[3], s_misc[4]};
        int live = 0;
        bool ok = true;
        for (int i = 0; ok; ++i) {
            sg = cur.next(l, setup);
            if (i >= 2) ok = tree_wait(info_empty + (i & 1), ((i >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) s_info[i & 1] = sg;
            __syncwarp();
            if (lane == 0) mbar_arrive(info_full + (i & 1));
            if (sg.b < 0) break;
            if (sg.tiles() == 0) continue;
            // q is fetched into L2 now, and to its place when the scores of the share before are done
            if (lane < C::CH)
                asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];"
                             ::"l"(&maps.q), "r"(64 * lane), "r"(sg.b * l.rows + sg.rt * kLatRows), "r"(0) : "memory");
            if (live > 0) ok = tree_wait(q_empty, (live - 1) & 1, abort, l.a.wait_timeouts, lane);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(q_full, (unsigned)(C::CH * 128 * g.q_rows));
            __syncwarp();
            if (lane < C::CH) tma_box3(s_q + lane * kLatRows * 128, &maps.q, 64 * lane, sg.b * l.rows + sg.rt * kLatRows, 0, q_full);
            __syncwarp();
            ++live;
        }
        // no copy is in flight when the block ends (in a healthy run the products have waited for all of them)
        volatile int no_abort = 0;
        if (live > 0) tree_wait(q_full, (live - 1) & 1, &no_abort, nullptr, lane);
    } else if (warp == 5) {
        // ---- scores ---------------------------------------------------------------------------------------
        constexpr unsigned kIdescS = instr_desc(kLatRows, kLatTile, false);
        const unsigned q_desc = desc_low(smem_u32(s_q), 16), k_desc = desc_low(smem_u32(s_ring), 16);
        int done = 0, slot = 0, round = 0, live = 0;          // tiles of the shares before this one; shares with tiles
        bool ok = true;
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            ok = tree_wait(q_full, live & 1, abort, l.a.wait_timeouts, lane);
            ++live;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                // (this buffer of S has been read)
                if (gt >= 2) ok = tree_wait(p_ready + buf, ((gt >> 1) - 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                const unsigned d = tmem + C::COL_S + buf * (kLatTile / 2);
#pragma unroll
                for (int p = 0; p < C::LAND; ++p) {
                    constexpr int kCols = 3;
                    const int c0 = p * kCols, nch = C::CH - c0 < kCols ? C::CH - c0 : kCols;
                    ok = ok && tree_wait(full + slot * C::LAND + p, round & 1, abort, l.a.wait_timeouts, lane);
                    if (!ok) break;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (what was copied by threads, to the products)
                    if (elect_one()) {
                        const unsigned qa = q_desc + c0 * kLatRows * 128 / 16, ka = k_desc + (slot * C::SLOT + c0 * C::CHUNK) / 16;
                        if (p == 0) tc_mma_ws(d, qa, ka, kIdescS, false);
                        else tc_mma_ws_add(d, qa, ka, kIdescS);
#pragma unroll
                        for (int k = 1; k < 4 * kCols; ++k)
                            if (k / 4 < nch) tc_mma_ws_add(d, qa + ((k / 4) * kLatRows * 128 + (k % 4) * 32) / 16, ka + ((k / 4) * C::CHUNK + (k % 4) * 32) / 16, kIdescS);
                        if (p == C::LAND - 1) {
                            tc_commit(s_full + buf);
                            if (t == tiles - 1) tc_commit(q_empty);
                        }
                    }
                    __syncwarp();
                }
                if (++slot == C::SLOTS) { slot = 0; ++round; }
            }
            done += tiles;
        }
        // TMEM is given back only when no product uses it
        if (__any_sync(0xffffffffu, !ok || *abort)) {
            if (elect_one()) tc_commit(drained);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained, 0u, &no_abort, nullptr, lane);
        }
    } else if (warp == 7) {
        // ---- products with V, by a warp of their own: each of the two goes on as soon as what it needs is there --------
        constexpr unsigned kIdescO = instr_desc(kLatRows, 256, true);
        const unsigned ring_desc = desc_low(smem_u32(s_ring), 16), v_desc = desc_low(smem_u32(s_ring), C::CHUNK);
        int done = 0, slot = 0, live = 0;
        bool ok = true;
        for (int i = 0; ok && next_seg(i); ++i) {
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            // (the first product replaces the last share's O)
            if (live > 0) ok = tree_wait(o_free, (live - 1) & 1, abort, l.a.wait_timeouts, lane);
            ++live;
            for (int t = 0; ok && t < tiles; ++t) {
                const int gt = done + t, buf = gt & 1;
                ok = tree_wait(p_ready + buf, (gt >> 1) & 1, abort, l.a.wait_timeouts, lane);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const int steps = (sg.count(t) + 15) / 16;
                    const unsigned va = v_desc + slot * (C::SLOT / 16), pa = ring_desc + (slot * C::SLOT + (C::CH - 1) * C::CHUNK) / 16;
#pragma unroll
                    for (int nb = 0; nb < R / 256; ++nb) {
                        tc_mma_ws(tmem + nb * 128, pa, va + nb * 4 * C::CHUNK / 16, kIdescO, t > 0);
#pragma unroll
                        for (int kk = 1; kk < 4; ++kk)
                            if (kk < steps) tc_mma_ws_add(tmem + nb * 128, pa + kk * 2, va + (nb * 4 * C::CHUNK + kk * 2048) / 16, kIdescO);
                        tc_commit(empty + slot * C::GROUPS + nb);
                    }
                    tc_commit(pv_done + buf);
                }
                __syncwarp();
                if (++slot == C::SLOTS) slot = 0;
            }
            done += tiles;
        }
        if (__any_sync(0xffffffffu, !ok || *abort)) {
            if (elect_one()) tc_commit(drained + 1);
            __syncwarp();
            volatile int no_abort = 0;
            tree_wait(drained + 1, 0u, &no_abort, nullptr, lane);
        }
    } else if (warp == 6) {
        // ---- the new tokens' rows to the cache, by the blocks that have their unit -----------------------------
        for (int i = 0; next_seg(i); ++i) latent_rest<R, kLatRows>(l, sg, sg.rt, (sg.n * l.a.H_q + kLatRows - 1) / kLatRows, lane);
    } else if (warp >= 8) {
        // ---- copies of rows, cached and new ones, 16 of a tile by each warp ---------------------------------------
        // (by a place in the list of their own, since they are ahead of those who learn of the items from one another)
        LatentRows<R> rows(l, s_ring, warp - 8, lane);
        LatentCursor<kLatTile, kLatRows> cur = {s_misc[2], s_misc[3], s_misc[4]};
        const int setup = s_misc[5];
        int slot = 0, round = 0;
        bool ok = true;
        while (ok && (sg = cur.next(l, setup)).b >= 0) {
            const int tiles = sg.tiles();
            if (tiles == 0) continue;
            int page, token;
            rows.find(g, sg, 0, page, token);
            for (int t = 0; ok && t < tiles; ++t) {
                rows.at(g, sg, t, page, token);
                if (t + 1 < tiles) rows.find(g, sg, t + 1, page, token);
#pragma unroll
                for (int c = 0; c < C::CH; ++c) {
                    if (c % 4 == 0 && c / 4 < C::GROUPS && round > 0)
                        ok = ok && tree_wait(empty + slot * C::GROUPS + c / 4, (round - 1) & 1, abort, l.a.wait_timeouts, lane);
                    if (!ok) break;
                    rows.copy(slot, c);
                    if (c % 3 == 2 || c == C::CH - 1) cp_async_arrive_on(full + slot * C::LAND + c / 3);
                }
                if (++slot == C::SLOTS) { slot = 0; ++round; }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp < 4) {
        // ---- softmax: two threads per query row, half of the tile's keys each -------------------------------
        const int half = warp >> 1, row = (warp & 1) * 32 + lane;
        const unsigned lane_base = (unsigned)(warp * 32) << 16;
        const float sl = l.a.scale_log2;
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
            const int token = (sg.rt * kLatRows + row) / l.a.H_q;
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
                if (alive) seen = sg.cached(t) ? sg.count(t) : token + 1;
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
            float total = 0.f;
            if (tiles > 0) {
                done += tiles;
                ok = tree_wait(pv_done + ((done - 1) & 1), ((done - 1) >> 1) & 1, abort, l.a.wait_timeouts, lane) && swap(sum_l, total);
                if (!ok) break;
                tc_fence_after();
                total += sum_l;
            }
            latent_results<R>(g, tmem + lane_base, (int64_t)sg.b * l.rows + sg.rt * kLatRows + row, min(kLatRows, l.rows - sg.rt * kLatRows), row,
                              half, sg.part < 0 ? -1 : share * 2 + sg.part, tiles > 0, alive, m_ref * sl, total, g.cluster > 0 ? s_part : nullptr,
                              g.cluster > 0 ? s_ml : nullptr);
            if (tiles == 0) continue;
            if (lane == 0) mbar_arrive(o_free);
        }
    }
    __syncthreads();                                          // (every role has come to its end)
    if (g.cluster > 1 && merged) {
        // out = sum_i e^{m_i - M} O_i / sum_i e^{m_i - M} l_i over the cluster's blocks, which share the rows
        tree_cluster_barrier();
        constexpr int PIECES = R / 128;                       // of a row, a warp each: every lane has four dims, of all blocks at once
        const int rank = share % g.cluster, tasks = min(kLatRows, l.rows - item_rt * kLatRows) * PIECES;
        for (int task = rank * (kLatThreads / 32) + warp; task < tasks; task += kLatThreads / 32 * g.cluster) {
            const int r = task / PIECES, c = task % PIECES * 128 + lane * 4;
            float2 ml[8];
            float4 o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
                if (i < g.cluster) {
                    ml[i] = tree_peer_f2(tree_peer(s_ml + r, i));
                    o[i] = tree_peer_f4(tree_peer(s_part + r * C::PART_LD + c, i));
                }
            }
            float top = -INFINITY, sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (ml[i].y == 0.f) continue;                 // (a part that saw nothing has no O either)
                const float w = fast_exp2(ml[i].x - top);
                sum = fmaf(w, ml[i].y, sum);
                acc.x = fmaf(w, o[i].x, acc.x); acc.y = fmaf(w, o[i].y, acc.y);
                acc.z = fmaf(w, o[i].z, acc.z); acc.w = fmaf(w, o[i].w, acc.w);
            }
            const bool none = sum == 0.f;
            const float inv = none ? 0.f : 1.f / sum;
            const int64_t orow = (int64_t)item_b * l.rows + item_rt * kLatRows + r;
            *reinterpret_cast<uint2*>(reinterpret_cast<T*>(l.a.out) + orow * R + c) =
                none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (c == 0) l.a.lse[orow] = none ? -INFINITY : (top + log2f(sum)) * LN2;
        }
        tree_cluster_barrier();                               // nobody leaves while its shared memory may be read
    }
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)C::TMEM_COLS));
    }
}

// Merges the partial results of items that several shares have: out = sum_i e^{m_i - M} O_i / sum_i e^{m_i - M} l_i.
// A block: 64 dims of 64 query rows; a warp has 8 rows x 4 pieces of four dims, so that it reads and writes whole sectors.
// Which parts there are is worked out before the wait for the kernel in front, while that still runs: it begins its successors
// when everything in front of it is done, so the lengths that it has read are there to be read here.
template <int R, int KT, int ROWS>
__global__ void __launch_bounds__(kLatMergeThreads) dsa_latent_merge_kernel(const LatentTcArgs g) {
    __shared__ int2 s_scan[kLatMergeThreads / 32];
    __shared__ int s_before;
    constexpr int PER = ROWS / kLatRows;                      // blocks that have an item's rows
    const LatentArgs& l = g.l;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int idx = blockIdx.x;
    const int d0 = (idx % (R / 64)) * 64; idx /= R / 64;
    const int rt = idx % l.row_tiles, b = idx / l.row_tiles;
    const int B = l.a.B, per = (B + kLatMergeThreads - 1) / kLatMergeThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const LatentItems<KT, ROWS, true> x(l, b);
    const LatentShares sh = latent_shares<KT, ROWS, true>(l, g.groups, g.min_units, b0, b1, s_scan);
    if (b >= b0 && b < b1) {
        int before = sh.before;
        for (int i = b0; i < b; ++i) {
            const LatentItems<KT, ROWS, true> x(l, i);
            before += x.items * (x.units + sh.setup);
        }
        s_before = before;
    }
    __syncthreads();
    const int first = s_before + rt / PER * (x.units + sh.setup), g0 = first / sh.quota, g1 = (first + x.units + sh.setup - 1) / sh.quota;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    if (g0 == g1 || rt / PER >= x.items) return;
    const int row = warp * 8 + lane / 4, c4 = lane % 4;
    if (rt * kLatRows + row >= l.rows) return;
    const bool alive = row < x.n * l.a.H_q - rt * kLatRows;
    const int64_t orow = (int64_t)b * l.rows + rt * kLatRows + row;
    auto part = [&](int gi) { return (int64_t)(gi * PER + rt % PER) * 2 + (gi == g0 ? 1 : 0); };
    float top = -INFINITY, sum = 0.f;
    float4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (alive) {
        for (int from = g0; from <= g1; from += 2) {          // (the loads of two parts at a time)
            float2 ml[2];
            float4 y[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t p = part(min(from + j, g1));
                ml[j] = g.part_ml[p * kLatRows + row];
                const float4* o = g.part_o + (p * (R / 4) + d0 / 4 + c4) * kLatRows + row;
#pragma unroll
                for (int k = 0; k < 4; ++k) y[j][k] = o[k * 4 * kLatRows];
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (from + j > g1 || ml[j].y == 0.f) continue;    // (a part that saw nothing)
                const float next = fmaxf(top, ml[j].x), keep = fast_exp2(top - next), w = fast_exp2(ml[j].x - next);
                top = next;
                sum = fmaf(sum, keep, w * ml[j].y);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    acc[k].x = fmaf(acc[k].x, keep, w * y[j][k].x); acc[k].y = fmaf(acc[k].y, keep, w * y[j][k].y);
                    acc[k].z = fmaf(acc[k].z, keep, w * y[j][k].z); acc[k].w = fmaf(acc[k].w, keep, w * y[j][k].w);
                }
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
