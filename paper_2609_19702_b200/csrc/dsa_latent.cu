// New tokens over a latent cache: argument checks, launch plan and launch (dsa_latent_step).
#include <algorithm>

#include "dsa_latent_f32.cuh"
#include "dsa_latent_host.cuh"

namespace {

using namespace dsa;

struct LatentPlan {
    int rows, row_tiles;                           // query rows of a request, blocks of them
    int n_split;                                   // float32: pieces of a request's keys
    int64_t blocks;
    size_t ws_out_bytes, ws_total;
};

int32_t make_latent_plan(const dsa_latent* l, int32_t heads, int32_t max_new, LatentPlan* pl) {
    const int32_t rc = check_latent(l, true);
    if (rc != DSA_OK) return rc;
    if (heads < 1 || max_new < 1) return DSA_ERR_INVALID_ARG;
    if (max_new > DSA_LATENT_MAX_NEW || heads > 1024) return DSA_ERR_UNSUPPORTED;
    if (l->max_seq_len > 0x7fff0000) return DSA_ERR_UNSUPPORTED;     // (positions a tile or N further stay below 2^31)
    *pl = LatentPlan{};
    pl->rows = heads * max_new;
    pl->row_tiles = (pl->rows + kLatentF32Block - 1) / kLatentF32Block;
    const int64_t items = std::max<int64_t>(1, (int64_t)l->batch * pl->row_tiles);
    const int64_t tiles = ((int64_t)l->max_seq_len + max_new + kStreamTile - 1) / kStreamTile;
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

template <typename T, int R>
cudaError_t configure_f32() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return configure_smem(dsa_latent_f32_kernel<T, R>, LatentF32Cfg<R>::SMEM, done);
}
template <typename T, int R>
cudaError_t run_f32(const LatentArgs& g, int64_t blocks, cudaStream_t st) {
    const cudaError_t e = configure_f32<T, R>();
    return e != cudaSuccess ? e : launch_dependent(dsa_latent_f32_kernel<T, R>, blocks, kStreamWarps * 32, LatentF32Cfg<R>::SMEM, st, g);
}

}  // namespace

namespace dsa {
cudaError_t latent_prepare() {
    cudaError_t e = configure_f32<float, 256>();
    if (e == cudaSuccess) e = configure_f32<float, 512>();
    if (e == cudaSuccess) e = configure_f32<__nv_bfloat16, 256>();
    if (e == cudaSuccess) e = configure_f32<__nv_bfloat16, 512>();
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
    if (pl.n_split > 1) {
        g.a.out_part = reinterpret_cast<float*>(workspace);
        g.a.lse_part = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(workspace) + pl.ws_out_bytes);
    } else {
        g.a.out = out;
        g.a.lse = lse;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (latent->dtype == DSA_BF16)
        e = latent->latent_dim == 256 ? run_f32<__nv_bfloat16, 256>(g, pl.blocks, st) : run_f32<__nv_bfloat16, 512>(g, pl.blocks, st);
    else
        e = latent->latent_dim == 256 ? run_f32<float, 256>(g, pl.blocks, st) : run_f32<float, 512>(g, pl.blocks, st);
    if (e != cudaSuccess) return host_cuda_fail(e);
    if (pl.n_split > 1)
        return host_launch_combine(g.a.out_part, g.a.lse_part, (int64_t)latent->batch * pl.rows, latent->latent_dim, pl.n_split, out,
                                   lse, latent->dtype, st);
    return DSA_OK;
}

}  // extern "C"
