// Drafted tokens: argument checks, launch plan and launch of the tree attention (dsa_tree_step).
#include "dsa_host.cuh"

#include <algorithm>
#include <cmath>

#include "dsa_tree.cuh"
#include "dsa_tree_f32.cuh"

namespace {

using namespace dsa;

struct TreePlan {
    int G, row_tiles;
    int rows;                                      // query rows per block
    int n_split;                                   // pieces whose partial results go through the workspace (1: none)
    int cluster;                                   // or blocks of a cluster that merge on chip (1: none)
    int64_t blocks;
    int box_tokens, align_tokens;
    size_t ws_out_bytes, ws_total;
};

// How many blocks of a cluster should share the tiles of one (request, kv head, 128 rows).  The estimate: waves of
// blocks x the time of one, in units of a tile, where a block's set-up costs about four tiles and a merge two more.
// Without clusters blocks take over each other's work and there are no waves; with them a last wave that is only part
// full costs a full one (32 x 32 heads of up to 4160 tokens: 204 us without, 227 in twos; 8 x 8 heads of 8190 tokens: 102
// without, 60 in twos, 46 in fours).  The lengths on the device are not known here and may be shorter than the bound:
// what counts is their ratio.
int choose_cluster(int64_t items, int64_t tiles, int64_t places) {
    int best = 1;
    double best_cost = std::max(1.0, (double)items / (double)places) * (4.0 + (double)tiles);
    for (int c = 2; c <= 8 && tiles >= 2 * c; c *= 2) {
        const int64_t waves = (items * c + places - 1) / places;
        const double cost = (double)waves * (6.0 + (double)((tiles + c - 1) / c));
        if (cost < best_cost) { best = c; best_cost = cost; }
    }
    return best;
}

int32_t make_tree_plan(const dsa_problem* p, const dsa_diag_params* d, const dsa_tree* tree, TreePlan* pl) {
    int32_t rc = host_check_problem(p);
    if (rc != DSA_OK) return rc;
    rc = host_check_diag(p, d);
    if (rc != DSA_OK) return rc;
    if (!tree || tree->max_nodes < 1) return DSA_ERR_INVALID_ARG;
    if (tree->max_nodes > DSA_TREE_MAX_NODES) return DSA_ERR_UNSUPPORTED;
    if (p->ring_size > 0) return DSA_ERR_UNSUPPORTED;
    if (p->max_seq_len > 0x7fff0000) return DSA_ERR_UNSUPPORTED;     // (positions a tile or a tree further stay below 2^31)
    if (d && d->mode != DSA_MASK_WINDOW) return DSA_ERR_UNSUPPORTED;
    const int N = tree->max_nodes;
    pl->G = p->num_q_heads / p->num_kv_heads;
    pl->rows = p->dtype == DSA_BF16 ? kTreeRows : N * pl->G <= 8 ? 8 : N * pl->G <= 16 ? 16 : kTreeF32Rows;
    pl->row_tiles = (N * pl->G + pl->rows - 1) / pl->rows;

    // a box of the caches' tensor maps must not cross the end of a page: the largest power of two that divides it
    pl->box_tokens = kTreeTile;
    pl->align_tokens = 1;
    if (p->block_table) {
        while (p->block_size % pl->box_tokens) pl->box_tokens /= 2;
        pl->align_tokens = pl->box_tokens;
    }

    // upper bound of the cached tiles that a block's nodes see
    int64_t tiles = ((int64_t)p->max_seq_len + kTreeTile - 1) / kTreeTile;
    if (d) {
        const int64_t lp = p->max_prompt_len > 0 ? std::min(p->max_prompt_len, p->max_seq_len) : p->max_seq_len;
        const int64_t seen = (lp + d->n_sink + kTreeTile - 1) / kTreeTile + ((int64_t)d->window + N + 2 * kTreeTile - 1) / kTreeTile;
        tiles = std::min(tiles, seen);
    }
    tiles = std::max<int64_t>(tiles, 1);
    const int64_t items = std::max<int64_t>(1, (int64_t)p->batch * p->num_kv_heads * pl->row_tiles);
    int64_t want = 1;
    pl->cluster = 1;
    const bool bf16 = p->dtype == DSA_BF16;
    if (p->split_tokens > 0) {
        const int64_t per = (p->split_tokens + (int64_t)kTreeTile - 1) / kTreeTile;
        want = (tiles + per - 1) / per;
    } else {
        int64_t places = 2 * (int64_t)host_sm_count();               // two blocks share an SM
        if (bf16) {
            pl->cluster = choose_cluster(items, tiles, places);
            // eight blocks are too few where even they leave most places empty and have many tiles each
            if (pl->cluster == 8 && items * 16 <= places && tiles >= 8 * 16) {
                want = std::min(places / items, tiles / 4);
                pl->cluster = 1;
            }
        } else {
            // fp32: about as many blocks as there are places, none below two tiles
            if (pl->rows == 8 && p->head_dim == 64) places *= 2;      // (four blocks share an SM)
            want = std::min((places + items / 2) / items, std::max<int64_t>(1, tiles / 2));
            want = std::max<int64_t>(want, 1);
        }
    }
    if (want > kMaxSplits) return DSA_ERR_UNSUPPORTED;
    pl->n_split = (int)want;
    pl->blocks = items * want * pl->cluster;
    if (pl->blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    pl->ws_out_bytes = pl->ws_total = 0;
    if (want > 1) {
        const size_t parts = (size_t)p->batch * N * p->num_q_heads * want;
        pl->ws_out_bytes = (parts * p->head_dim * sizeof(float) + 255) / 256 * 256;
        pl->ws_total = pl->ws_out_bytes + (parts * sizeof(float) + 255) / 256 * 256;
    }
    return DSA_OK;
}

// Views for the tensor-map copies: 64 elements (128 bytes) of a row per box, 128-byte swizzle.
bool encode_view(TensorMapEncodeFn encode, CUtensorMap* map, const void* base, const int64_t (&dims)[4],
                 const int64_t (&stride_elems)[3], const int (&box)[4]) {
    cuuint64_t n[4], pitch[3];
    cuuint32_t bx[4], step[4] = {1u, 1u, 1u, 1u};
    for (int i = 0; i < 4; ++i) {
        if (dims[i] < 1 || dims[i] > 0xffffffffLL) return false;
        n[i] = (cuuint64_t)dims[i];
        bx[i] = (cuuint32_t)box[i];
    }
    for (int i = 0; i < 3; ++i) {
        if (stride_elems[i] <= 0 || stride_elems[i] >= (1LL << 39)) return false;
        pitch[i] = (cuuint64_t)stride_elems[i] * 2;
    }
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), n, pitch, bx, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int32_t build_tree_maps(const dsa_problem* p, const dsa_tree* tree, const TreePlan& pl, const void* k_new, const void* v_new,
                        TreeArgs* g, TreeMaps* m) {
    const TensorMapEncodeFn encode = host_tensor_map_encoder();
    if (!encode) return DSA_ERR_UNSUPPORTED;
    const int64_t D = p->head_dim, Hq = p->num_q_heads, Hkv = p->num_kv_heads, N = tree->max_nodes, B = p->batch;
    // caches: [page or request][head][token][D]; a stride of 0 (all requests or heads read the same) is a
    // dimension of one entry
    g->blk_coord = p->stride_batch > 0 ? 1 : 0;
    g->head_coord = p->stride_head > 0 ? 1 : 0;
    const int64_t tokens = p->block_table ? p->block_size : std::max(p->max_seq_len, 1);
    const int64_t outer = g->blk_coord ? (p->block_table ? p->num_blocks : B) : 1;
    const int64_t cache_dims[4] = {D, tokens, g->head_coord ? Hkv : 1, outer};
    const int64_t cache_strides[3] = {p->stride_token, g->head_coord ? p->stride_head : p->stride_token,
                                      g->blk_coord ? p->stride_batch : p->stride_token};
    const int cache_box[4] = {64, pl.box_tokens, 1, 1};
    const int64_t new_dims[4] = {D, N, Hkv, B};
    const int64_t new_strides[3] = {Hkv * D, D, N * Hkv * D};
    const int new_box[4] = {64, (int)N, 1, 1};
    const int64_t q_dims[4] = {D, Hq, N, B};
    const int64_t q_strides[3] = {D, Hq * D, N * Hq * D};
    const int q_box[4] = {64, pl.G, (int)std::min<int64_t>(N, kTreeRows / pl.G), 1};
    const bool ok = encode_view(encode, &m->k, p->k_cache, cache_dims, cache_strides, cache_box) &&
                    encode_view(encode, &m->v, p->v_cache, cache_dims, cache_strides, cache_box) &&
                    encode_view(encode, &m->k_new, k_new, new_dims, new_strides, new_box) &&
                    encode_view(encode, &m->v_new, v_new, new_dims, new_strides, new_box) &&
                    encode_view(encode, &m->q, p->q, q_dims, q_strides, q_box);
    return ok ? DSA_OK : DSA_ERR_UNSUPPORTED;      // (an extent or stride beyond what a tensor map holds)
}

template <class Kern, class... Args>
cudaError_t launch_tree(Kern kern, int64_t blocks, int threads, int smem, int cluster, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int D>
cudaError_t configure_bf16() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return configure_smem(dsa_tree_kernel<D>, TreeCfg<D>::SMEM, done);
}
template <int D>
cudaError_t configure_f32() {
    static std::atomic<bool> done[kMaxDevices] = {}, done8[kMaxDevices] = {}, done16[kMaxDevices] = {};
    cudaError_t e = configure_smem(dsa_tree_f32_kernel<D>, TreeF32Cfg<D>::SMEM, done);
    if (e == cudaSuccess) e = configure_smem(dsa_tree_few_kernel<D, 8>, TreeFewCfg<D, 8>::SMEM, done8);
    if (e == cudaSuccess) e = configure_smem(dsa_tree_few_kernel<D, 16>, TreeFewCfg<D, 16>::SMEM, done16);
    return e;
}
template <int D>
cudaError_t run_bf16(const TreeArgs& g, const TreeMaps& m, int64_t blocks, cudaStream_t st) {
    const cudaError_t e = configure_bf16<D>();
    return e != cudaSuccess ? e : launch_tree(dsa_tree_kernel<D>, blocks, kTreeThreads, TreeCfg<D>::SMEM, g.cluster, st, g, m);
}
template <int D>
cudaError_t run_f32(const TreeArgs& g, int rows, int64_t blocks, cudaStream_t st) {
    const cudaError_t e = configure_f32<D>();
    if (e != cudaSuccess) return e;
    if (rows == 8) return launch_tree(dsa_tree_few_kernel<D, 8>, blocks, kTreeF32Threads, TreeFewCfg<D, 8>::SMEM, 1, st, g);
    if (rows == 16) return launch_tree(dsa_tree_few_kernel<D, 16>, blocks, kTreeF32Threads, TreeFewCfg<D, 16>::SMEM, 1, st, g);
    return launch_tree(dsa_tree_f32_kernel<D>, blocks, kTreeF32Threads, TreeF32Cfg<D>::SMEM, 1, st, g);
}

}  // namespace

namespace dsa {
cudaError_t tree_prepare() {
    cudaError_t e = configure_bf16<64>();
    if (e == cudaSuccess) e = configure_bf16<128>();
    if (e == cudaSuccess) e = configure_f32<64>();
    if (e == cudaSuccess) e = configure_f32<128>();
    return e;
}
}  // namespace dsa

extern "C" {

int32_t dsa_tree_workspace_size(const dsa_problem* problem, const dsa_diag_params* diag, const dsa_tree* tree, size_t* bytes) {
    if (!bytes) return DSA_ERR_INVALID_ARG;
    TreePlan pl;
    const int32_t rc = make_tree_plan(problem, diag, tree, &pl);
    if (rc != DSA_OK) return rc;
    *bytes = pl.ws_total;
    return DSA_OK;
}

int32_t dsa_tree_step(const dsa_problem* problem, const dsa_diag_params* diag, const dsa_tree* tree, const void* k_new,
                      const void* v_new, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    TreePlan pl;
    int32_t rc = make_tree_plan(problem, diag, tree, &pl);
    if (rc != DSA_OK) return rc;
    if (problem->batch == 0) return DSA_OK;
    if (!k_new || !v_new || !out || !lse) return DSA_ERR_INVALID_ARG;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(out)) return DSA_ERR_INVALID_ARG;
    if (pl.ws_total > 0) {
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return DSA_ERR_INVALID_ARG;
        if (workspace_bytes < pl.ws_total) return DSA_ERR_WORKSPACE_TOO_SMALL;
    }
    TreeArgs g = {};
    host_cache_args(problem, &g.a);
    g.a.k_new = k_new;
    g.a.v_new = v_new;
    g.a.n_split = pl.n_split;
    g.a.mask.window = diag ? diag->window : 0;
    g.a.mask.n_sink = diag ? diag->n_sink : 0;
    g.windowed = diag ? 1 : 0;
    g.parent = tree->parent;
    g.node_count = tree->node_count;
    g.N = tree->max_nodes;
    g.G = pl.G;
    for (g.g_shift = 0; (1 << g.g_shift) < pl.G;) ++g.g_shift;
    g.row_tiles = pl.row_tiles;
    g.box_tokens = pl.box_tokens;
    for (g.box_shift = 0; (1 << g.box_shift) < pl.box_tokens;) ++g.box_shift;
    g.batch = problem->batch;
    g.cluster = pl.cluster;
    // where blocks take over work, the longest sequences go first: a long one that is begun last is waited for alone
    g.sorted = pl.cluster == 1 && pl.blocks > 2 * (int64_t)host_sm_count() && problem->batch > 1 && problem->batch <= kTreeSorted;
    // division of positions (below 2^31) by the page size: with 2^s >= d the product by ceil(2^(31 + s) / d) is exact
    const unsigned d = problem->block_table ? (unsigned)problem->block_size : 1u;
    for (g.page_shift = 31; (1ull << (g.page_shift - 31)) < d;) ++g.page_shift;
    g.page_mul = (unsigned)(((1ull << g.page_shift) + d - 1) / d);
    g.align_tokens = pl.align_tokens;
    if (pl.n_split > 1) {
        g.a.out_part = reinterpret_cast<float*>(workspace);
        g.a.lse_part = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(workspace) + pl.ws_out_bytes);
    } else {
        g.a.out = out;
        g.a.lse = lse;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (problem->dtype == DSA_BF16) {
        e = host_wait_timeouts_address(&g.a.wait_timeouts);
        if (e != cudaSuccess) return host_cuda_fail(e);
        TreeMaps m;
        rc = build_tree_maps(problem, tree, pl, k_new, v_new, &g, &m);
        if (rc != DSA_OK) return rc;
        e = problem->head_dim == 64 ? run_bf16<64>(g, m, pl.blocks, st) : run_bf16<128>(g, m, pl.blocks, st);
    } else {
        e = problem->head_dim == 64 ? run_f32<64>(g, pl.rows, pl.blocks, st) : run_f32<128>(g, pl.rows, pl.blocks, st);
    }
    if (e != cudaSuccess) return host_cuda_fail(e);
    if (pl.n_split > 1)
        return host_launch_combine(g.a.out_part, g.a.lse_part, (int64_t)problem->batch * g.N * problem->num_q_heads,
                                   problem->head_dim, pl.n_split, out, lse, problem->dtype, st);
    return DSA_OK;
}

}  // extern "C"
