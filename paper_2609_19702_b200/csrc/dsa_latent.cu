// New tokens over a latent cache: argument checks, launch plan and launch (dsa_latent_step).
#include <algorithm>

#include "dsa_latent.cuh"
#include "dsa_latent_pair.cuh"
#include "dsa_latent_f32.cuh"
#include "dsa_latent_host.cuh"

namespace {

using namespace dsa;

struct LatentPlan {
    int rows, row_tiles;                           // query rows of a request, blocks of them
    int n_split;                                   // float32: pieces of a request's keys
    bool pairs;                                    // bf16: pairs of blocks with 128 query rows
    int groups;                                    // and shares of the work, or
    int cluster;                                   // blocks of a cluster with an item to itself (0: shares)
    int64_t blocks;
    size_t ws_out_bytes, ws_total;                 // float32: partial outputs, and their log-sums behind them
    size_t ws_ml_bytes;                            // bf16: maxima and sums, and partial outputs behind them
};

constexpr int kLatMinUnits = 2;                    // tiles that a block takes at least (see LatentTcArgs)

// Tokens per tensor-map copy of the cache: a box must not cross the end of a page, so the largest power of two that divides it.
int latent_box(const dsa_latent* l) {
    int box = kLatTile;
    if (l->block_table)
        while (l->block_size % box) box /= 2;
    return box;
}

int32_t make_latent_plan(const dsa_latent* l, int32_t heads, int32_t max_new, LatentPlan* pl) {
    const int32_t rc = check_latent(l, true);
    if (rc != DSA_OK) return rc;
    if (heads < 1 || max_new < 1) return DSA_ERR_INVALID_ARG;
    if (max_new > DSA_LATENT_MAX_NEW || heads > 1024) return DSA_ERR_UNSUPPORTED;
    if (l->max_seq_len > 0x7fff0000) return DSA_ERR_UNSUPPORTED;     // (positions a tile or N further stay below 2^31)
    *pl = LatentPlan{};
    pl->rows = heads * max_new;
    if (l->dtype == DSA_BF16) {
        pl->row_tiles = (pl->rows + kLatRows - 1) / kLatRows;
        // (an upper bound of the units on the device, and of those that beginnings count for)
        const int64_t tiles = ((int64_t)l->max_seq_len + kLatTile - 1) / kLatTile + 1, items = std::max<int64_t>(1, (int64_t)l->batch * pl->row_tiles);
        const int64_t units = items * (tiles + 2), sms = std::max(host_sm_count(), 1);
        if (units > (1 << 30)) return DSA_ERR_UNSUPPORTED;
        // More than 64 query rows: pairs, but where a page allows only boxes of less than 16 tokens, whose copies cost 70 to 90 cycles
        // each however little they bring.  32 x 128 heads, pairs / blocks of 64 rows, whose threads copy row by row: pages of 64:
        // 61 / 77 us, 16: 67 / 78, 24: 87 / 78, 1: 146 / 79.
        pl->pairs = pl->rows > kLatRows && latent_box(l) >= 16;
        const int per = pl->pairs ? 2 : 1;
        pl->groups = (int)std::max<int64_t>(1, std::min<int64_t>(sms / per, units / (per * per * kLatMinUnits)));
        pl->blocks = (int64_t)pl->groups * per;
        // (waits of up to one item's share: 2^18 tiles take half of the second that a wait may)
        if (std::min(tiles, units / pl->groups) > (1 << 18)) return DSA_ERR_UNSUPPORTED;
        // Few items, or items of few tiles: a cluster has each of them to itself and merges on chip, without partial results in HBM
        // or a second launch.  In us, with `t` the bound of an item's tiles: a launch, 1.4 to 1.5 a tile of a block, and the merge's
        // reads; against shares, which are of one size whatever the lengths, but start later, write parts (the more of an item,
        // the longer its merge) and need the merge kernel.  Measured, shares / best cluster (lengths spread up to the bound): 16
        // heads, 9 requests, 17 tiles: 17.2 / 12.4 (8 blocks), 65 tiles: 24.8 / 20.1 (8); 18 requests, 33 tiles: 20.6 / 20.3 (4), 65:
        // 26.6 / 34.3; 64 requests, 2 tiles: 12.6 / 9.0 (1), 5: 15.8 / 13.2 (2), 17: 21.9 / 23.9, 65: 42.2 / 60.3; 128 heads, one
        // request, 33 tiles: 14.7 / 17.1 (8), 9 requests, 17 tiles: 20.6 / 18.5 (4); 37 requests, 10 tiles: 25.6 / 22.8 (1).
        const float t = (float)tiles, all = (float)(items * tiles) / (float)sms;
        float best = pl->pairs ? 13.f + 10.f * all / (all + 1.f) + 0.7f * all
                               : 10.5f + std::min(3.f, t / 2.f) + 1.03f * all + 0.35f * std::min(t / 2.f, (float)sms / (float)items);
        const float merge = 0.018f * (float)(std::min(pl->rows, kLatRows) * l->latent_dim / 128);
        // (clusters that are on the device at once: an SM holds one block, and a cluster's SMs lie close together)
        const int64_t most[4] = {sms, sms * 7 / 15, sms * 7 / 33, sms / 10};
        for (int i = 0, c = 1; i < 4; ++i, c *= 2) {
            const float cost = (c > 1 ? 8.f + merge : 6.5f) + (c > 2 ? 1.35f : 1.5f) * (float)((tiles + c - 1) / c);
            if (items <= most[i] && cost < best) { best = cost; pl->cluster = c; }
        }
        if (pl->cluster) {
            pl->pairs = false;
            pl->groups = 1;
            pl->blocks = items * pl->cluster;
        }
        if (pl->groups > 1) {
            pl->ws_ml_bytes = (size_t)pl->blocks * 2 * kLatRows * sizeof(float2);
            pl->ws_total = pl->ws_ml_bytes + (size_t)pl->blocks * 2 * kLatRows * l->latent_dim * sizeof(float);
        }
        return DSA_OK;
    }
    pl->row_tiles = (pl->rows + kTileRows - 1) / kTileRows;
    const int64_t items = std::max<int64_t>(1, (int64_t)l->batch * pl->row_tiles);
    const int64_t tiles = ((int64_t)l->max_seq_len + max_new + kTileKeys - 1) / kTileKeys;
    const int64_t places = 3 * (int64_t)host_sm_count();
    pl->n_split = (int)std::max<int64_t>(1, std::min<int64_t>({(places + items / 2) / items, tiles / 2, (int64_t)kMaxSplits}));
    pl->blocks = items * pl->n_split;
    if (pl->blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    if (pl->n_split > 1) {
        const size_t parts = (size_t)l->batch * pl->rows * pl->n_split;
        pl->ws_out_bytes = (parts * l->latent_dim * sizeof(float) + 255) / 256 * 256;
        pl->ws_total = pl->ws_out_bytes + (parts * sizeof(float) + 255) / 256 * 256;
    }
    return DSA_OK;
}

// A view of rows of `width` elements for the tensor-map copies: 64 elements (128 bytes) of `box` rows per copy, 128-byte
// swizzle; what a copy asks for beyond the view arrives as zeros.
bool encode_rows(TensorMapEncodeFn encode, CUtensorMap* map, const void* base, int64_t width, int64_t rows, int64_t outer,
                 int64_t row_stride, int64_t outer_stride, int box) {
    const int64_t most = 0xffffffffLL;
    if (rows < 1 || rows > most || outer < 1 || outer > most) return false;
    if (row_stride >= (1LL << 39) || outer_stride <= 0 || outer_stride >= (1LL << 39)) return false;
    const cuuint64_t n[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)outer};
    const cuuint64_t pitch[2] = {(cuuint64_t)row_stride * 2, (cuuint64_t)outer_stride * 2};
    const cuuint32_t bx[3] = {64u, (cuuint32_t)box, 1u}, step[3] = {1u, 1u, 1u};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), n, pitch, bx, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int32_t build_latent_maps(const dsa_latent* l, const LatentPlan& pl, const void* q, const void* c_new, LatentTcArgs* g, LatentMaps* m) {
    const TensorMapEncodeFn encode = host_tensor_map_encoder();
    if (!encode) return DSA_ERR_UNSUPPORTED;
    const int64_t W = l->latent_dim + l->rope_dim, tokens = l->block_table ? l->block_size : std::max(l->max_seq_len, 1);
    const int box = latent_box(l);
    for (g->box_shift = 0; (1 << g->box_shift) < box;) ++g->box_shift;
    // division of positions (below 2^31) by the page size: with 2^s >= d the product by ceil(2^(31 + s) / d) is exact
    const unsigned d = l->block_table ? (unsigned)l->block_size : 1u;
    for (g->page_shift = 31; (1ull << (g->page_shift - 31)) < d;) ++g->page_shift;
    g->page_mul = (unsigned)(((1ull << g->page_shift) + d - 1) / d);
    g->q_rows = std::min(kLatRows, (pl.rows + 7) / 8 * 8);
    g->blk_coord = l->stride_batch > 0 ? 1 : 0;    // (a stride of 0: a dimension of one entry)
    const int64_t outer = g->blk_coord ? (l->block_table ? l->num_blocks : l->batch) : 1;
    bool ok = encode_rows(encode, &m->q, q, W, (int64_t)l->batch * pl.rows, 1, W, W, g->q_rows);
    if (pl.pairs)
        ok = ok && encode_rows(encode, &m->cache, l->cache, W, tokens, outer, l->stride_token, g->blk_coord ? l->stride_batch : l->stride_token, box) &&
             encode_rows(encode, &m->fresh, c_new, W, g->l.N, l->batch, W, (int64_t)g->l.N * W, g->l.N);
    return ok ? DSA_OK : DSA_ERR_UNSUPPORTED;      // (an extent or stride beyond what a tensor map holds)
}

template <int R>
cudaError_t configure() {
    static std::atomic<bool> done[kMaxDevices] = {}, done_f32[kMaxDevices] = {};
    static std::atomic<bool> done_pair[kMaxDevices] = {};
    cudaError_t e = configure_smem(dsa_latent_kernel<R>, LatentCfg<R>::SMEM, done);
    if (e == cudaSuccess) e = configure_smem(dsa_latent_pair_kernel<R>, PairCfg<R>::SMEM, done_pair);
    if (e == cudaSuccess) e = configure_smem(dsa_latent_f32_kernel<R>, LatentF32Cfg<R>::SMEM, done_f32);
    return e;
}
template <int R>
cudaError_t run_bf16(const LatentTcArgs& g, const LatentMaps& m, bool pairs, int64_t blocks, cudaStream_t st) {
    cudaError_t e = configure<R>();
    if (e != cudaSuccess) return e;
    e = pairs ? launch_dependent(dsa_latent_pair_kernel<R>, blocks, kPairThreads, PairCfg<R>::SMEM, st, g, m)
              : launch_clusters(dsa_latent_kernel<R>, std::max(g.cluster, 1), blocks, kLatThreads, LatentCfg<R>::SMEM, st, g, m);
    if (e != cudaSuccess || g.groups == 1) return e;
    const int64_t merge = (int64_t)g.l.a.B * g.l.row_tiles * (R / 64);
    return pairs ? launch_dependent(dsa_latent_merge_kernel<R, kPairTile, kPairRows>, merge, kLatMergeThreads, 0, st, g)
                 : launch_dependent(dsa_latent_merge_kernel<R, kLatTile, kLatRows>, merge, kLatMergeThreads, 0, st, g);
}
template <int R>
cudaError_t run_f32(const LatentArgs& g, int64_t blocks, cudaStream_t st) {
    cudaError_t e = configure<R>();
    if (e != cudaSuccess) return e;
    e = launch_dependent(dsa_latent_f32_kernel<R>, blocks, kTileThreads, LatentF32Cfg<R>::SMEM, st, g);
    if (e != cudaSuccess || g.a.n_split == 1) return e;
    const int64_t rows = (int64_t)g.a.B * g.rows, warps = rows * (R / 128);
    return launch_dependent(dsa_latent_f32_merge_kernel<R>, (warps + kLatF32MergeWarps - 1) / kLatF32MergeWarps, kLatF32MergeWarps * 32, 0, st, g, rows);
}

}  // namespace

namespace dsa {
cudaError_t latent_prepare() {
    cudaError_t e = configure<256>();
    if (e == cudaSuccess) e = configure<512>();
    return e;
}
}  // namespace dsa

extern "C" {

int32_t dsa_latent_workspace_size(const dsa_latent* latent, int32_t num_heads, int32_t max_new, size_t* bytes) {
    if (!bytes) return DSA_ERR_INVALID_ARG;
    LatentPlan pl;
    const int32_t rc = make_latent_plan(latent, num_heads, max_new, &pl);
    if (rc != DSA_OK) return rc;
    *bytes = pl.ws_total;
    return DSA_OK;
}

int32_t dsa_latent_step(const dsa_latent* latent, int32_t num_heads, int32_t max_new, const void* q, const void* c_new,
                        const int32_t* new_count, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    LatentPlan pl;
    const int32_t rc = make_latent_plan(latent, num_heads, max_new, &pl);
    if (rc != DSA_OK) return rc;
    if (latent->batch == 0) return DSA_OK;
    if (!q || !c_new || !out || !lse) return DSA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(c_new) || !aligned16(out)) return DSA_ERR_INVALID_ARG;
    if (pl.ws_total > 0) {
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return DSA_ERR_INVALID_ARG;
        if (workspace_bytes < pl.ws_total) return DSA_ERR_WORKSPACE_TOO_SMALL;
    }
    LatentArgs g = {};
    g.a.q = q;
    g.a.k = latent->cache;
    g.a.k_new = c_new;
    g.a.stride_b = latent->stride_batch;
    g.a.stride_tok = latent->stride_token;
    g.a.seq_len = latent->seq_len;
    g.a.block_table = latent->block_table;
    g.a.max_blocks = latent->max_blocks;
    g.a.block_size = latent->block_size;
    g.a.num_blocks = latent->num_blocks;
    g.a.max_seq_len = latent->max_seq_len;
    g.a.B = latent->batch;
    g.a.H_q = num_heads;
    g.a.H_kv = 1;
    g.a.scale_log2 = latent->sm_scale * LOG2E;
    g.a.n_split = pl.n_split;
    g.new_count = new_count;
    g.N = max_new;
    g.R = latent->latent_dim;
    g.P = latent->rope_dim;
    g.rows = pl.rows;
    g.row_tiles = pl.row_tiles;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (latent->dtype == DSA_BF16) {
        LatentTcArgs t = {};
        g.a.out = out;
        g.a.lse = lse;
        e = host_wait_timeouts_address(&g.a.wait_timeouts);
        if (e != cudaSuccess) return host_cuda_fail(e);
        t.l = g;
        t.groups = pl.groups;
        t.cluster = pl.cluster;
        t.min_units = kLatMinUnits;
        unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
        t.part_ml = reinterpret_cast<float2*>(ws);
        t.part_o = reinterpret_cast<float4*>(ws + pl.ws_ml_bytes);
        LatentMaps m;
        const int32_t built = build_latent_maps(latent, pl, q, c_new, &t, &m);
        if (built != DSA_OK) return built;
        e = latent->latent_dim == 256 ? run_bf16<256>(t, m, pl.pairs, pl.blocks, st) : run_bf16<512>(t, m, pl.pairs, pl.blocks, st);
        return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
    }
    if (pl.n_split > 1) {
        g.a.out_part = reinterpret_cast<float*>(workspace);
        g.a.lse_part = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(workspace) + pl.ws_out_bytes);
    }
    g.a.out = out;
    g.a.lse = lse;
    e = latent->latent_dim == 256 ? run_f32<256>(g, pl.blocks, st) : run_f32<512>(g, pl.blocks, st);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

}  // extern "C"
