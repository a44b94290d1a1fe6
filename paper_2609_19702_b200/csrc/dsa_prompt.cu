// Attention of prompts with expanded keys and values: argument checks and launch (dsa_latent_prompt).
#include <algorithm>
#include <cmath>

#include "dsa_latent_host.cuh"
#include "dsa_prompt.cuh"
#include "dsa_prompt_f32.cuh"

namespace {

using namespace dsa;

int32_t check_prompt(const dsa_prompt* p) {
    if (!p) return DSA_ERR_INVALID_ARG;
    if (p->batch < 0 || p->num_heads < 1 || p->q_tokens < 0 || p->kv_tokens < 0 || p->max_q_len < 0) return DSA_ERR_INVALID_ARG;
    if (p->dtype != DSA_BF16 && p->dtype != DSA_F32) return DSA_ERR_UNSUPPORTED;
    if ((p->nope_dim != 64 && p->nope_dim != 128) || p->value_dim != p->nope_dim) return DSA_ERR_UNSUPPORTED;
    if (p->rope_dim < 8 || p->rope_dim > 64 || p->rope_dim % 8) return DSA_ERR_UNSUPPORTED;
    if (!(p->sm_scale >= 0.f) || !std::isfinite(p->sm_scale)) return DSA_ERR_INVALID_ARG;
    if (p->num_heads > 1024 || p->batch > (1 << 20)) return DSA_ERR_UNSUPPORTED;
    const int64_t vec = p->dtype == DSA_BF16 ? 8 : 4;
    const int64_t strides[7] = {p->q_stride_token, p->q_stride_head, p->k_stride_token, p->k_stride_head, p->rope_stride_token,
                                p->v_stride_token, p->v_stride_head};
    for (int64_t s : strides)
        if (s < 0 || s % vec) return DSA_ERR_INVALID_ARG;
    if ((p->q_tokens > 1 && p->q_stride_token < p->nope_dim + p->rope_dim) ||
        (p->kv_tokens > 1 && (p->k_stride_token < p->nope_dim || p->rope_stride_token < p->rope_dim || p->v_stride_token < p->value_dim)))
        return DSA_ERR_INVALID_ARG;
    // (a half without queries waits while the other half goes through a request's keys: 2^25 take half of the second that a wait may)
    if (p->dtype == DSA_BF16 && p->kv_tokens > (1 << 25)) return DSA_ERR_UNSUPPORTED;
    if (p->batch == 0 || p->q_tokens == 0 || p->max_q_len == 0) return DSA_OK;
    if (!p->q || !p->q_start || !aligned16(p->q)) return DSA_ERR_INVALID_ARG;
    if (p->kv_tokens > 0 && (!p->k_nope || !p->k_rope || !p->v)) return DSA_ERR_INVALID_ARG;
    if (!aligned16(p->k_nope) || !aligned16(p->k_rope) || !aligned16(p->v)) return DSA_ERR_INVALID_ARG;
    return DSA_OK;
}

// A view [tokens][heads][width] for the tensor-map copies: 64 elements (128 bytes) of one head and `box` tokens per copy,
// 128-byte swizzle; what a copy asks for beyond the view arrives as zeros.  head: 1, or 0 where all heads read the same rows.
bool encode_heads(TensorMapEncodeFn encode, CUtensorMap* map, const void* base, int64_t width, int64_t heads, int64_t tokens,
                  int64_t head_stride, int64_t token_stride, int box, int* head) {
    const int64_t most = 0xffffffffLL;
    if (tokens < 1 || tokens > most) return false;
    if (tokens == 1) token_stride = width + 64;    // (never used: any stride will do)
    token_stride = (token_stride + 7) / 8 * 8;
    *head = heads > 1 && head_stride > 0;
    if (token_stride >= (1LL << 39) || head_stride >= (1LL << 39)) return false;
    const cuuint64_t n[3] = {(cuuint64_t)width, (cuuint64_t)(*head ? heads : 1), (cuuint64_t)tokens};
    const cuuint64_t pitch[2] = {(cuuint64_t)(*head ? head_stride : token_stride) * 2, (cuuint64_t)token_stride * 2};
    const cuuint32_t bx[3] = {64u, 1u, (cuuint32_t)box}, step[3] = {1u, 1u, 1u};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), n, pitch, bx, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int BLOCKS>
cudaError_t configure_bf16() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return configure_smem(dsa_prompt_kernel<D, BLOCKS>, PromptCfg<D>::SMEM, done);
}
template <int D>
cudaError_t configure_f32() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return configure_smem(dsa_prompt_f32_kernel<D>, PromptF32Cfg<D>::SMEM, done);
}
template <int D>
cudaError_t configure() {
    cudaError_t e = configure_bf16<D, kPrByBound>();
    if (e == cudaSuccess) e = configure_bf16<D, kPrByNumber>();
    if (e == cudaSuccess) e = configure_bf16<D, kPrByList>();
    if (e == cudaSuccess) e = configure_f32<D>();
    return e;
}
template <int D>
cudaError_t run(const PromptArgs& g, const PromptMaps& m, bool bf16, int64_t blocks, cudaStream_t st) {
    const cudaError_t e = configure<D>();
    if (e != cudaSuccess) return e;
    if (!bf16) return launch_dependent(dsa_prompt_f32_kernel<D>, blocks, kTileThreads, PromptF32Cfg<D>::SMEM, st, g);
    if (g.blocks == kPrByList) return launch_dependent(dsa_prompt_kernel<D, kPrByList>, blocks, kPrThreads, PromptCfg<D>::SMEM, st, g, m);
    if (g.blocks == kPrByNumber) return launch_dependent(dsa_prompt_kernel<D, kPrByNumber>, blocks, kPrThreads, PromptCfg<D>::SMEM, st, g, m);
    return launch_dependent(dsa_prompt_kernel<D, kPrByBound>, blocks, kPrThreads, PromptCfg<D>::SMEM, st, g, m);
}

}  // namespace

namespace dsa {
cudaError_t prompt_prepare() {
    cudaError_t e = configure<64>();
    if (e == cudaSuccess) e = configure<128>();
    return e;
}
}  // namespace dsa

extern "C" {

int32_t dsa_latent_prompt(const dsa_prompt* p, void* out, float* lse, void* stream) {
    const int32_t rc = check_prompt(p);
    if (rc != DSA_OK) return rc;
    if (p->batch == 0 || p->q_tokens == 0 || p->max_q_len == 0) return DSA_OK;
    if (!out || !lse || !aligned16(out)) return DSA_ERR_INVALID_ARG;
    PromptArgs g = {};
    g.q = p->q; g.k = p->k_nope; g.kr = p->k_rope; g.v = p->v;
    g.q_tok = p->q_stride_token; g.q_head = p->q_stride_head;
    g.k_tok = p->k_stride_token; g.k_head = p->k_stride_head;
    g.r_tok = p->rope_stride_token;
    g.v_tok = p->v_stride_token; g.v_head = p->v_stride_head;
    g.q_start = p->q_start; g.kv_start = p->kv_start;
    g.batch = p->batch; g.H = p->num_heads; g.P = p->rope_dim;
    g.q_tokens = p->q_tokens; g.kv_tokens = p->kv_tokens;
    g.max_q_len = std::min(p->max_q_len, p->q_tokens);
    g.causal = p->causal ? 1 : 0;
    g.scale_log2 = (p->sm_scale > 0.f ? p->sm_scale : 1.f / std::sqrt((float)(p->nope_dim + p->rope_dim))) * LOG2E;
    g.out = out;
    g.lse = lse;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool bf16 = p->dtype == DSA_BF16;
    const int rows = bf16 ? kPrBlock : kTileRows;
    // Blocks of a head: max_q_len's for every request, or, found by their numbers, what the tokens fill and one a request.  The first
    // where it is not many more: it takes no search and puts the long items first, but a block without a query costs half a
    // microsecond.  In us, by bound / by number: bf16, 1000 prompts of up to 300, 4 heads, 1.3 times as many: 169 / 175, 1.9
    // times: 184 / 175; 40 of up to 3000, 8 heads, 1.7 times: 359 / 320; 300 of up to 130, 128 heads, 66 times: 12249 / 885.
    // float32, 600 of up to 100, 16 heads, 1.6 times: 730 / 760, 2.7 times: 778 / 760.
    const int64_t grid = ((int64_t)g.max_q_len + rows - 1) / rows * p->batch, filled = (int64_t)p->q_tokens / rows + p->batch;
    g.blocks = (bf16 ? 2 * grid >= 3 * filled : grid >= 2 * filled) || grid * p->num_heads > 0x7fffffffLL ? kPrByNumber : kPrByBound;
    int64_t entries = g.blocks == kPrByNumber ? filled : grid;
    // bf16 lists what a thread a request and an entry can name, and sorts it, so that none of the long items is begun last (24
    // prompts of up to 600 tokens behind prefixes of up to 512, 16 heads: 66 -> 63.7 us; 64 of up to 300 with a bound of all
    // tokens: 198 -> 56); very many even out.
    const int64_t listed = std::min(grid, filled);
    if (bf16 && p->batch > 1 && p->batch <= kPrListed && listed <= kPrListed && (listed * p->num_heads > host_sm_count() || listed < grid)) {
        g.blocks = kPrByList;
        g.entries = (int)listed;
        entries = listed;
    }
    const int64_t blocks = entries * p->num_heads;
    if (blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    PromptMaps m = {};
    cudaError_t e;
    if (bf16) {
        e = host_wait_timeouts_address(&g.wait_timeouts);
        if (e != cudaSuccess) return host_cuda_fail(e);
        const TensorMapEncodeFn encode = host_tensor_map_encoder();
        if (!encode) return DSA_ERR_UNSUPPORTED;
        int one;
        // (without any key no copy of a key is made, and the views may be those of q)
        const bool keys = p->kv_tokens > 0;
        const int64_t kv = keys ? p->kv_tokens : 1, W = p->nope_dim + p->rope_dim, H = p->num_heads;
        const bool ok = encode_heads(encode, &m.q, p->q, W, H, p->q_tokens, p->q_stride_head, p->q_stride_token, kPrRows, &m.q_head) &&
                        encode_heads(encode, &m.k, keys ? p->k_nope : p->q, p->nope_dim, H, kv, p->k_stride_head, p->k_stride_token, kPrTile, &m.k_head) &&
                        encode_heads(encode, &m.kr, keys ? p->k_rope : p->q, p->rope_dim, 1, kv, 0, p->rope_stride_token, kPrTile, &one) &&
                        encode_heads(encode, &m.v, keys ? p->v : p->q, p->value_dim, H, kv, p->v_stride_head, p->v_stride_token, kPrTile, &m.v_head);
        if (!ok) return DSA_ERR_UNSUPPORTED;       // (an extent or stride beyond what a tensor map holds)
    }
    e = p->nope_dim == 64 ? run<64>(g, m, bf16, blocks, st) : run<128>(g, m, bf16, blocks, st);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

}  // extern "C"
