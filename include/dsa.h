/*
 * dsa.h -- C ABI of the diagonal-aware sparse decode-attention library for NVIDIA B200 (sm_100a).
 *
 * One call = one decode step of one transformer layer: every request of a batch has ONE query
 * token per head and attends over its KV cache.  The sparse call keeps the whole prompt and,
 * inside a recent window of the decode (image) tokens, drops the keys that lie on the skipped
 * diagonals -- keys at fixed distances behind the query -- so that dropped keys are never read
 * from memory.  (Paper: "Understanding and Exploiting Diagonal Attention Sparsity in
 * Autoregressive Image Generation", Section 4 and Algorithm 1.)
 *
 * Conventions
 *   - Every tensor pointer is a DEVICE pointer owned by the caller; it must stay valid until the
 *     work queued on `stream` has finished.  The dsa_problem / dsa_diag_params structs themselves
 *     are HOST memory, read during the call only.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*, NULL = default stream);
 *     the library never synchronises and allocates no device memory.  It reads no environment
 *     variable and carries no result from one call to the next (the one piece of device state that
 *     outlives a call is a diagnostic counter, see dsa_wait_timeouts()); what it does remember per
 *     device are idempotent set-up caches (which kernel variants have been configured, the SM
 *     count, the addresses of the built-in scratch array and of that counter, the driver entry
 *     point that encodes tensor maps), written with atomics, so calls may come from several host
 *     threads.  Scratch comes from the caller's `workspace` (device, 256-byte aligned), sized
 *     by dsa_workspace_size(); it may be reused by the next call on the same stream.  The one
 *     exception is dsa_decode_attention_static_scratch(), whose scratch is a fixed array inside
 *     the library image.
 *   - Arguments are checked on the host before anything is launched.  Values that live in
 *     device memory (seq_len, prompt_len, block ids, skip offsets) cannot be checked there;
 *     kernels clamp them into range instead, so bad values give wrong numbers, not faults.
 *   - Return value: DSA_OK or a negative dsa_status.  After DSA_ERR_CUDA the CUDA error code is
 *     available from dsa_last_cuda_error().
 *   - The first launch of each kernel variant on a device also configures it (one-time
 *     attribute and address queries that must not happen inside a stream capture): call
 *     dsa_prepare() once per device, or make the first call of a given shape, before capturing.
 *   - There is no CPU path: without a CUDA device every compute call fails with DSA_ERR_CUDA.
 *
 * Positions.  For request b, prompt_len[b] = L_p tokens of prompt come first in the cache and
 * are always attended.  p = seq_len[b] - prompt_len[b] decode tokens follow, the last of which
 * is the token being decoded (its K/V are already in the cache); Algorithm 1's 0-based step is
 * t = p - 1.  A key at cache position s >= L_p lies o = seq_len - 1 - s tokens behind the query.
 */
#ifndef DSA_H
#define DSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DSA_VERSION 101  /* 101: dsa_problem.plan_flags promise bit, dsa_diag_params.skip_bitmap, dsa_plan_info grew */

/* exported symbols (the library is built with hidden visibility for everything else) */
#if defined(__GNUC__)
#define DSA_API __attribute__((visibility("default")))
#else
#define DSA_API
#endif

typedef enum dsa_status {
    DSA_OK = 0,
    DSA_ERR_INVALID_ARG = -1,         /* null pointer, bad size, bad stride, N_att > window ...   */
    DSA_ERR_UNSUPPORTED = -2,         /* head_dim not 64/128, group size not 1/2/4/8, window too   */
                                      /* large for a LIST mask, ...                                */
    DSA_ERR_WORKSPACE_TOO_SMALL = -3,
    DSA_ERR_CUDA = -4                 /* a CUDA runtime call failed; see dsa_last_cuda_error()     */
} dsa_status;

typedef enum dsa_dtype { DSA_BF16 = 0, DSA_F32 = 1 } dsa_dtype;

typedef enum dsa_mask_mode {
    DSA_MASK_WINDOW = 0,  /* prompt + the `window` most recent decode tokens, nothing skipped      */
    DSA_MASK_GRID = 1,    /* skipped diagonals derived from the raster grid (see dsa_diag_params)  */
    DSA_MASK_LIST = 2     /* skipped diagonals given per head as a list of distances               */
} dsa_mask_mode;

/*
 * The attention problem (inputs of Algorithm 1: the prompt KV cache K_p,V_p and the decode KV
 * cache K,V, stored back to back per request, plus the query of the current step).
 */
typedef struct dsa_problem {
    int32_t batch;             /* B, number of requests (>= 0)                                     */
    int32_t num_q_heads;       /* H_q                                                              */
    int32_t num_kv_heads;      /* H_kv; H_q / H_kv must be 1, 2, 4 or 8.  Query head h reads kv    */
                               /* head h / (H_q / H_kv)                                            */
    int32_t head_dim;          /* D: 64 or 128                                                     */
    int32_t dtype;             /* dsa_dtype of q, k_cache, v_cache and out                         */
    float sm_scale;            /* logit scale; 0 means 1/sqrt(D)                                   */
    const void *q;             /* [B, H_q, D] contiguous                                           */
    const void *k_cache;       /* keys;   rows of D contiguous elements, 16-byte aligned           */
    const void *v_cache;       /* values; same layout and strides as k_cache                       */
    /* Element strides.  Contiguous cache (block_table == NULL): token s of request b, kv head g
     * starts at b*stride_batch + s*stride_token + g*stride_head (stride_batch may be 0 to let all
     * requests read one cache).  Paged cache: token s lives in block
     * id = block_table[b*max_blocks + s/block_size] at
     * id*stride_batch + (s % block_size)*stride_token + g*stride_head.
     * All strides must be multiples of 16 bytes. */
    int64_t stride_batch;
    int64_t stride_token;
    int64_t stride_head;
    const int32_t *seq_len;    /* [B] tokens in the cache, prompt included                         */
    const int32_t *prompt_len; /* [B] L_p; values above seq_len[b] are read as seq_len[b]          */
    const int32_t *block_table;/* [B, max_blocks] or NULL                                          */
    int32_t max_blocks;        /* row length of block_table                                        */
    int32_t block_size;        /* tokens per block (> 0 when paged)                                */
    int32_t num_blocks;        /* blocks in the pool; block ids are clamped to [0, num_blocks)     */
    int32_t max_seq_len;       /* HOST upper bound of seq_len[b]; sizes the launch.  Longer        */
                               /* sequences are read as if they ended there                        */
    int32_t max_prompt_len;    /* HOST upper bound of prompt_len[b], or 0 if unknown (the sparse   */
                               /* call then plans for max_seq_len kept tokens)                     */
    int32_t split_tokens;      /* kept tokens handled by one thread block; 0 = library chooses.    */
                               /* Rounded up to the tile size, at most 1024                        */
    /* Bounded cache (the eviction step of Algorithm 1, phase 3; footprint N_r + L_p of Section 4's
     * cost analysis).  ring_size == 0: every token is stored at its logical position.
     * ring_size > 0: the prompt and the first ring_sinks decode tokens are stored at their logical
     * positions; decode token j >= ring_sinks is stored at position
     * L_p + ring_sinks + (j - ring_sinks) mod ring_size, overwriting the token that left the
     * window ring_size steps earlier.  seq_len stays the LOGICAL length.  Needs
     * max_prompt_len > 0; sparse calls need window <= ring_size and n_sink <= ring_sinks; the
     * dense call is refused.  The cache then needs max_prompt_len + ring_sinks + ring_size
     * tokens per request instead of max_seq_len; a device prompt_len[b] above max_prompt_len is
     * read as max_prompt_len, so that no row is addressed outside that region. */
    int32_t ring_size;
    int32_t ring_sinks;
    /* 0 in production: the library chooses the launch plan.  Comparison runs and tests may force
     * single planner decisions with the DSA_PLAN_* bits below; results never depend on them
     * beyond summation order. */
    uint32_t plan_flags;
} dsa_problem;

#define DSA_PLAN_CUDA_CORES    0x01u  /* bf16 through the CUDA-core kernel instead of the tensor-core one */
#define DSA_PLAN_NO_ITEM_WARPS 0x02u  /* small launches: split + combine, never four warps on one item   */
#define DSA_PLAN_RING_DEEP     0x04u  /* two-heads-per-block kernel: keep the 3-stage ring               */
#define DSA_PLAN_RING_SHALLOW  0x08u  /* two-heads-per-block kernel: take the 2-stage ring               */
#define DSA_PLAN_GROUP         0x10u  /* take the head-group / per-head-list kernels wherever they can run */
#define DSA_PLAN_NO_GROUP      0x20u  /* never take them                                                 */
#define DSA_PLAN_GROUP_W4      0x40u  /* forced head-group kernel: 4 warps per block instead of 2        */
#define DSA_PLAN_NO_CLUSTER    0x80u  /* small launches: never let a thread-block cluster share a work item */
#define DSA_PLAN_CLUSTER2      0x10000u /* small launches (several warps per item): clusters of 2 blocks  */
#define DSA_PLAN_CLUSTER4      0x20000u /*                                           clusters of 4 blocks  */
#define DSA_PLAN_GATHER        0x40000u /* head-group kernel, 4 warps: stage tiles by tensor-map gather copies */
                                        /* (TMA, four scattered rows per copy) where the cache has a 2-D view */
#define DSA_PLAN_NO_GATHER     0x80000u /* never do                                                        */
#define DSA_PLAN_PRODUCERS     0x100000u /* head-group kernel, 4 warps: a producer warp beside every consumer warp */
#define DSA_PLAN_NO_PRODUCERS  0x200000u /* never                                                       */
/* Not a planner switch but a promise about the stream: no launch that can still be running when this
 * call's kernel starts writes seq_len, prompt_len, block_table or the skip lists (skip_offsets and
 * skip_bitmap; a call with `select` writes both, for its own layer).  The attention kernels
 * chain with programmatic dependent launch and let their successor start before they have waited for
 * their own predecessor, so "still running" means: the launch just before this call and, if that is an
 * attention call of this library, the launches before it in turn, back to the first launch that does
 * not let its successor in early (a projection, dsa_advance_seq_len: those complete before anything
 * behind them starts).  dsa_append_kv does let its successor in early and, when it advances, writes
 * seq_len: the call behind it cannot make the promise.  In a decode loop of fused steps every layer's
 * call but the one that follows dsa_advance_seq_len can.
 * The head-group, per-head-list, several-warps-per-item and cluster kernels then work out which rows to
 * read BEFORE they wait for the launch in front, and touch q, the new rows and the caches only after;
 * the other kernels (producer-warp and tensor-map forms, one warp per item, CUDA cores) ignore it. */
#define DSA_PLAN_METADATA_STABLE 0x800000u
#define DSA_PLAN_HEADS_PER_WARP_SHIFT 8  /* forced head-group kernel: kv heads per warp in bits 8..15    */
#define DSA_PLAN_HEADS_PER_WARP_MASK  0xff00u

/*
 * Which decode keys are kept (Algorithm 1 with its data-dependent selection made an input).
 *
 * With t = p - 1, the window holds the distances o = 0 .. min(t, window - 1) (the `window` = N_r
 * most recent decode tokens, the current one included).  m = window - n_att diagonals are
 * skipped in steady state.  Algorithm 1 selects them one per step from step n_att - 1 on, and an
 * entry selected at step s is skipped from step s + 1 on; so at step t the first
 * n_act = clamp(t - (n_att - 1), 0, m) selected distances are skipped.  A key chosen at step s
 * with cache index j keeps the distance s - j at every later step (the "+1" shift of skip_idx).
 *
 *   LIST  skip_offsets[b][mask_head][k] is the distance of the k-th selection, in selection
 *         order; it must be a valid trace: 0 <= o_k <= n_att - 1 + k (0-based k), no repeats.
 *         mask_heads is 1 (all heads share), H_kv (per kv head) or H_q (per query head, the
 *         paper's setting; with grouped queries a KV row is read if any head of its group keeps
 *         it, the other heads ignore it).
 *   GRID  the trace is generated from the grid instead of being passed: with
 *         stride = grid_w + row_extra tokens per image row, the column distance of o is
 *         d(o) = min(o mod stride, stride - o mod stride) and every selection step skips the
 *         attended key with the largest (d(o), o).  Same mask for all heads.  (Not in the
 *         paper: a data-free stand-in for its argmin that keeps the diagonals next to the
 *         multiples of the row stride.)
 *   WINDOW nothing skipped (n_att is ignored).  This is the paper's SlidingWindow baseline.
 *
 * Selection (the choice of the next skipped key in Algorithm 1, phase 2, fused into the attention
 * pass as in Section 5.1).  With `select` set, a request whose step t lies in N_att-1 .. N_r-2 also gets
 * the next trace entry: among the decode keys it attends (sinks excluded) the one with the lowest
 * softmax weight -- the lowest logit; equal logits go to the lowest cache index -- is found per
 * query head and its distance is written to skip_offsets[b][h][t - (N_att-1)], which takes effect
 * from the next step on.  Calling the sparse call once per decode step with the same buffer thus
 * grows the trace exactly as Algorithm 1 grows skip_idx.  Entries are decided on float32 logits;
 * -1 is written if there is no candidate.  Requests outside those steps are left untouched.
 *
 * Sinks (Section 5.1, the "Diagonal + sink4" variant and the StreamingLLM baseline): the first
 * n_sink decode tokens are kept at every step in addition to what the mode keeps, and are never
 * counted against n_att: in steady state n_att + n_sink decode keys are attended.  WINDOW with
 * n_sink = 4 is StreamingLLM (4 sinks + recent window); GRID or LIST with n_sink = 4 is
 * Diagonal + sink4 with n_att = budget - 4.
 */
typedef struct dsa_diag_params {
    int32_t mode;                 /* dsa_mask_mode                                                 */
    int32_t window;               /* N_r >= 1                                                      */
    int32_t n_att;                /* N_att, 1 <= n_att <= window                                   */
    int32_t grid_w;               /* GRID: image tokens per row                                    */
    int32_t row_extra;            /* GRID: row-end / separator tokens per row (>= 0)               */
    int32_t *skip_offsets;        /* LIST: device [B, mask_heads, trace_len] int32 (written when   */
                                  /* `select` is set, otherwise only read)                         */
    int32_t mask_heads;           /* LIST: 1, H_kv or H_q                                          */
    int32_t trace_len;            /* LIST: entries per trace, >= window - n_att                    */
    int32_t n_sink;               /* first decode tokens always kept (>= 0; 0 = none)              */
    int32_t select;               /* LIST, mask_heads == H_q: also run the phase-2 selection       */
    uint32_t *skip_bitmap;        /* LIST, optional (NULL: none): device [B, mask_heads, ceil(window / 32)]  */
                                  /* words; bit o of a head's row is set iff distance o is one of its        */
                                  /* ACTIVE skip_offsets entries (the first n_act).  The same information    */
                                  /* as the list, in the form the per-head-list kernel wants: it then reads  */
                                  /* window / 8 bytes per head instead of scattering the list into a bitmap  */
                                  /* itself.  dsa_build_skip_bitmap() fills it from skip_offsets; calls with */
                                  /* `select` keep it up to date (they set the bit of every entry they       */
                                  /* write).  The caller clears it together with the list when a request     */
                                  /* starts over.  Kernels other than the per-head-list one read the list.   */
} dsa_diag_params;

/* What a call will launch (filled by dsa_query_plan; for reporting and for tests). */
typedef struct dsa_plan_info {
    int32_t split_tokens;   /* kept tokens per work item                                           */
    int32_t n_split;        /* splits per (request, kv head); 1 = results written directly         */
    int32_t launches;       /* kernels launched by the call (1, or 2 with the combine)             */
    int32_t grid_blocks;    /* thread blocks of the attention kernel                               */
    int32_t smem_bytes;     /* dynamic shared memory per block                                     */
    int32_t tile_tokens;    /* tokens per staged K/V tile                                          */
    int32_t stages;         /* tiles in flight per block (per warp for the tensor-core kernel)     */
    int32_t tensor_cores;   /* 1: tensor-core kernel (bf16), one warp per work item;               */
                            /* 0: CUDA-core kernel (fp32), one 128-thread block per work item      */
    int32_t work_items;     /* (request, kv head, split) items                                     */
    int32_t item_warps;     /* warps that share one work item (4 in small tensor-core launches,    */
                            /* merged in shared memory; else 1)                                    */
    int32_t heads_per_block;/* head-group tensor-core kernel: kv heads that share the one row list */
                            /* a block builds (its warps stream heads_per_block / block_warps      */
                            /* heads each, back to back); 0: another kernel                        */
    int32_t block_warps;    /* warps per thread block that compute (producer_warps come on top)     */
    int32_t per_head_lists; /* 1: the per-head-list tensor-core kernel (list masks per head, fused  */
                            /* selection): shared tables per block, one candidate list per head    */
    int32_t cluster_blocks; /* blocks of a thread-block cluster that share one work item and merge */
                            /* through distributed shared memory (small launches); 1: no cluster   */
    int32_t tensor_map_copies; /* 1: the head-group kernel stages its tiles with tensor-map gather  */
                            /* copies (TMA) completing on mbarriers; 0: 16-byte cp.async copies    */
    int32_t producer_warps; /* warps per block that only issue copies (one per consumer warp, handing */
                            /* tiles over through mbarriers); 0: every warp copies and computes       */
} dsa_plan_info;

DSA_API int32_t dsa_version(void);
DSA_API const char *dsa_status_string(int32_t status);
/* CUDA error code recorded by the last failing call of this thread (0 if none). */
DSA_API int32_t dsa_last_cuda_error(void);
/* Number of bounded waits that gave up on the current device since the library was loaded.  The
 * tensor-map kernel waits for each tile on an mbarrier for about a second at most; a copy that
 * never lands makes it count here, stop waiting and run to its end, so that the context stays
 * usable (the numbers of that call are then wrong).  0 in a healthy run.  count_out: host pointer.
 * Synchronises with the device (a copy from a device symbol): not for use inside a capture. */
DSA_API int32_t dsa_wait_timeouts(int32_t *count_out);
/* Measuring hook: the sparse / dense call (diag NULL: dense) with the arithmetic taken out.  The launch
 * has the plan's grid, builds the same row lists and stages the same K / V tiles through the same
 * shared-memory rings, but a landed tile is only read once; what it leaves in out / lse (and the
 * workspace) is meaningless.  Its time is what the staging alone costs for this very problem -- the
 * attention call's own speed of light.  DSA_ERR_UNSUPPORTED unless the plan is the four-warp head-group
 * kernel (dsa_plan_info.block_warps == 4, per_head_lists == 0).  Arguments as dsa_decode_attention_sparse. */
DSA_API int32_t dsa_debug_copy_only(const dsa_problem *problem, const dsa_diag_params *diag, void *out, float *lse,
                                    void *workspace, size_t workspace_bytes, void *stream);
/* Fills diag->skip_bitmap from diag->skip_offsets for the requests' current seq_len: row (b, mask head)
 * gets the bits of that head's first n_act entries that lie in [0, window), all other bits are cleared.
 * LIST mode only; both pointers required.  Asynchronous on `stream`. */
DSA_API int32_t dsa_build_skip_bitmap(const dsa_problem *problem, const dsa_diag_params *diag, void *stream);
/* Test hook for that mechanism: launches one warp on `stream` that waits, with the same bound, on an
 * mbarrier nothing ever arrives on.  The wait runs out after about a second, the counter above goes
 * up by one, the kernel ends and the context stays usable.  Asynchronous like every launch. */
DSA_API int32_t dsa_debug_wait_giveup(void *stream);

/*
 * Configure every kernel variant of the library for the CURRENT device (a few hundred one-time
 * attribute calls, the SM count and the address of the built-in scratch array of
 * dsa_decode_attention_static_scratch; no launch, no allocation).  Optional: calls do it lazily
 * for what they need; required only before a stream capture whose calls would otherwise be the
 * first of their shape on this device.
 */
DSA_API int32_t dsa_prepare(void);

/* Bytes of workspace the attention calls need for `problem` (diag == NULL: dense call). */
DSA_API int32_t dsa_workspace_size(const dsa_problem *problem, const dsa_diag_params *diag, size_t *bytes);

/* The launch plan the attention calls will use for `problem` (diag == NULL: dense call). */
DSA_API int32_t dsa_query_plan(const dsa_problem *problem, const dsa_diag_params *diag, dsa_plan_info *info);

/*
 * Dense decode attention (the paper's baseline; Algorithm 1's Attn over every cached token):
 *   s_j = sm_scale * q_h . k_j  for j in [0, seq_len),  lse = ln sum_j e^{s_j},
 *   out = sum_j e^{s_j - lse} v_j.
 * out [B, H_q, D] in problem->dtype; lse [B, H_q] float32, natural log.  A request with
 * seq_len <= 0 gets out = 0, lse = -inf.
 */
DSA_API int32_t dsa_decode_attention_dense(const dsa_problem *problem, void *out, float *lse,
                                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Diagonal-aware sparse decode attention (Algorithm 1, one step t for every request):
 *   Attn(Q_t, K_p + K[idx], V_p + V[idx]) with idx = window - skip_idx,
 * softmax taken jointly over the prompt keys and the kept decode keys.  Only kept rows are read.
 * Outputs as for the dense call.
 */
DSA_API int32_t dsa_decode_attention_sparse(const dsa_problem *problem, const dsa_diag_params *diag,
                                    void *out, float *lse,
                                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * One decode step's attention with the step's inputs and results in HOST memory (the call a
 * serving loop makes when the scheduler lives on the CPU; the KV cache, which is decode state,
 * stays on the device).  Not in the paper; it is the dense (diag == NULL) or sparse call above
 * wrapped in the copies a step needs, all queued on `stream`:
 *   host_q -> problem->q, host_seq_len -> problem->seq_len, host_prompt_len -> problem->prompt_len,
 *   host_block_table -> problem->block_table (paged caches only; NULL otherwise),
 *   attention into dev_out / dev_lse, then dev_out -> host_out, dev_lse -> host_lse.
 * The device pointers inside `problem` are therefore WRITTEN by this call.  Host buffers should
 * be pinned for the copies to be asynchronous; they must stay valid, and host_out / host_lse
 * must not be read, until the stream has been synchronised by the caller.
 */
DSA_API int32_t dsa_decode_attention_host_io(const dsa_problem *problem, const dsa_diag_params *diag,
                                             const void *host_q, const int32_t *host_seq_len,
                                             const int32_t *host_prompt_len, const int32_t *host_block_table,
                                             void *dev_out, float *dev_lse, void *host_out, float *host_lse,
                                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * The same step as dsa_decode_attention_host_io, with the large transfers folded into the
 * kernels (not in the paper): the attention kernels read q from, and write out / lse to, the
 * caller's PINNED host buffers directly over the bus (mapped, zero-copy), so no separate q upload
 * precedes the attention and no download follows it.  What every head of a request re-reads
 * (host_seq_len, host_prompt_len, host_block_table) is still copied into the device arrays named
 * in `problem`, which are therefore WRITTEN.  problem->q is scratch: when the plan splits the
 * keys of one (request, kv head) over several work items, q is first copied there so that it
 * crosses the bus once; otherwise it is left untouched.
 * host_q, host_out and host_lse must be page-locked host memory that the device can address
 * (cudaHostAlloc / cudaHostRegister; checked with cudaPointerGetAttributes before anything is
 * queued: DSA_ERR_INVALID_ARG otherwise), host_q and host_out 16-byte aligned.  They must stay valid, and
 * host_out / host_lse must not be read, until the caller has synchronised the stream.
 */
DSA_API int32_t dsa_decode_attention_host_mapped(const dsa_problem *problem, const dsa_diag_params *diag,
                                                 const void *host_q, const int32_t *host_seq_len,
                                                 const int32_t *host_prompt_len, const int32_t *host_block_table,
                                                 void *host_out, float *host_lse,
                                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Merge split-KV partial results (not in the paper; the exact identity that a softmax over a
 * union of key sets is the lse-weighted mix of the softmaxes over the parts):
 *   lse = ln sum_i e^{lse_i},  out = sum_i e^{lse_i - lse} out_i.
 * out_part [B, H_q, n_split, D] float32, lse_part [B, H_q, n_split] float32 (natural log; a
 * part with lse_i = -inf is empty and its out_i is not read).  out [B, H_q, D] in out_dtype,
 * lse [B, H_q] float32 (may be NULL).
 */
DSA_API int32_t dsa_combine_splits(const float *out_part, const float *lse_part,
                           int32_t batch, int32_t num_q_heads, int32_t head_dim, int32_t n_split,
                           void *out, float *lse, int32_t out_dtype, void *stream);

/*
 * Append the K/V rows of the token being decoded (the cache write that precedes attention in a
 * decode step; with a bounded cache this is also Algorithm 1's eviction, since the new token
 * takes the slot of the one that left the window).  k_new, v_new: device [B, H_kv, D] in
 * problem->dtype.  The rows of request b go to logical position seq_len[b] (the value BEFORE
 * the call); a request whose seq_len is already max_seq_len is left alone.  With advance != 0
 * seq_len[b] is then incremented on the device by the same kernel, so that a captured sequence
 * "append, attend" can be replayed step after step without the host touching seq_len.
 */
DSA_API int32_t dsa_append_kv(const dsa_problem *problem, const void *k_new, const void *v_new,
                              int32_t advance, void *stream);

/*
 * One decode step of one layer in a single launch (plus the combine when the plan splits):
 * dsa_append_kv followed by the dense (diag == NULL) or sparse attention call, fused.  Not a
 * method of its own: Algorithm 1's "K.append(K_t)" and "Attn(Q_t, K_p + K[idx], ...)" of one
 * step, issued together.
 *   seq_len[b] counts the tokens ALREADY cached, without the token being decoded, and is not
 *   modified: a model's layers share one seq_len array, which the caller advances once per token
 *   after its last layer (dsa_advance_seq_len).
 *   k_new, v_new: device [B, H_kv, D] in problem->dtype, 16-byte aligned.  The rows of request b
 *   are written to logical position seq_len[b] of the cache and the request attends over
 *   seq_len[b] + 1 tokens, the mask taking p = seq_len[b] + 1 - prompt_len[b].  A request whose
 *   seq_len is already max_seq_len has no room: its token is dropped and it attends over what
 *   is cached, exactly as dsa_append_kv followed by attention would do.
 * For bf16 the attention kernel itself reads the current token's rows from k_new / v_new and
 * stores them to the cache; for float32 the rows are stored by a launch of their own first.
 * Everything else (outputs, workspace, plan, fused selection, bounded caches) as for the
 * attention calls.
 */
DSA_API int32_t dsa_decode_step(const dsa_problem *problem, const dsa_diag_params *diag,
                                const void *k_new, const void *v_new, void *out, float *lse,
                                void *workspace, size_t workspace_bytes, void *stream);

/*
 * seq_len[b] += 1 for every request below `max_seq_len` (device array of `batch` int32), queued on
 * `stream`: the once-per-token counterpart of dsa_decode_step, so that a captured token step
 * (every layer's dsa_decode_step, then this) can be replayed without the host touching seq_len.
 */
DSA_API int32_t dsa_advance_seq_len(int32_t *seq_len, int32_t batch, int32_t max_seq_len, void *stream);

/*
 * The kept cache positions, produced by the same device code that the sparse attention kernel
 * uses to decide which rows to read (Algorithm 1: K_p, then window - skip_idx as positions).
 * Positions are LOGICAL (before any ring mapping).
 * idx_out [B, mask_heads, max_kept] int32, ascending, entries beyond the count untouched;
 * count_out [B, mask_heads] int32 holds the full count even when it exceeds max_kept.
 * mask_heads is diag->mask_heads for LIST and 1 otherwise; diag == NULL reports the dense set.
 */
DSA_API int32_t dsa_debug_kept_indices(const dsa_problem *problem, const dsa_diag_params *diag,
                               int32_t *idx_out, int32_t *count_out, int32_t max_kept,
                               void *stream);

/*
 * The attention calls above for callers that cannot hand over a workspace.  (The paper has no
 * counterpart: this is a packaging variant of the two calls, not another method.)
 *
 * Who needs it: code that must not allocate device memory at the point of the call -- an
 * extension running inside a host application's allocation-free section, a latency-critical
 * serving loop that forbids allocator calls, a process whose device memory was carved up
 * completely at start-up.  The split-KV partial results go to a fixed DSA_STATIC_SCRATCH_MAX-byte
 * array inside the library image instead of a caller workspace; the call itself allocates and
 * frees nothing.  The price: each GPU that loads the library carries those bytes until the
 * process exits, whether or not this entry point is ever used.
 *
 * diag == NULL runs the dense call, otherwise the sparse call; q, caches, out and lse are passed
 * exactly as above and results are identical to dsa_decode_attention_dense / _sparse.
 * Problems whose partials exceed the array are refused with DSA_ERR_WORKSPACE_TOO_SMALL and
 * nothing is launched; dsa_workspace_size() tells the size in advance.
 * The first call on each device (or dsa_prepare() before it) looks up the array's device address,
 * with that device current; let that happen before any stream capture begins.
 * All calls share the one array and it keeps whatever the last call left there; nothing in it
 * needs clearing between calls.  Two calls whose kernels can run at the same time on one GPU
 * (different streams, different host threads) would overwrite each other's partials: keep calls
 * of this entry point ordered on one stream per GPU.
 */
#define DSA_STATIC_SCRATCH_MAX (8u << 20)
DSA_API int32_t dsa_decode_attention_static_scratch(const dsa_problem *problem, const dsa_diag_params *diag,
                                                    void *out, float *lse, void *stream);

/* ==== Drafted tokens: several tokens of a request decoded in one pass ===============================
 *
 * A decode step with drafted tokens (speculative decoding; not in the paper) is, for every layer,
 * dsa_tree_step; after the last layer dsa_verify_tree, which says which of the drafted tokens stand;
 * and dsa_compact_kv, which moves their K/V rows up behind the cached ones and gives the new seq_len.
 * The page calls below it keep the block table of a paged cache in step with that on the device:
 * dsa_reserve_pages before a pass, dsa_release_pages after it, dsa_fork_pages to branch a request.
 *
 * All conventions above hold.  The calls in this part read nothing that the stream's earlier work may
 * still be writing, and (unlike the attention calls) start none of their successors early before their
 * own predecessors have finished.  With regard to the promise DSA_PLAN_METADATA_STABLE, those that write
 * seq_len, prompt_len or a block table (compact, fork, release, reserve) are like dsa_advance_seq_len: the
 * call directly behind one of them cannot make it, since only a kernel that waits for the launch in front
 * is certain to see what that has written; the calls behind that one can.
 */

/* The drafted tokens ("nodes") of every request and what hangs on what. */
typedef struct dsa_tree {
    int32_t max_nodes;         /* N: nodes a request has room for in q, k_new, ..., 1 .. DSA_TREE_MAX_NODES */
    const int32_t *parent;     /* device [B, N]: the node that node i follows, in [0, i); any other value    */
                               /* (-1) makes node i a root that follows the cached tokens directly.          */
                               /* NULL: a chain, parent[i] = i - 1                                           */
    const int32_t *node_count; /* device [B]: nodes 0 .. node_count[b]-1 of the request exist (clamped to    */
                               /* [0, N]); NULL: all N                                                       */
} dsa_tree;
#define DSA_TREE_MAX_NODES 64

/* Bytes of workspace dsa_tree_step needs (diag as there). */
DSA_API int32_t dsa_tree_workspace_size(const dsa_problem *problem, const dsa_diag_params *diag, const dsa_tree *tree,
                                        size_t *bytes);

/*
 * dsa_decode_step for a tree of drafted tokens: appends the nodes' K/V rows to the cache and lets every
 * node attend over the cached tokens and over its own line (its ancestors and itself):
 *   x_j = sm_scale * q_i . k_j over the tokens j that node i sees,  lse_i = ln sum_j e^{x_j},
 *   out_i = sum_j e^{x_j - lse_i} v_j.
 * With S = seq_len[b] (tokens already cached; not modified) node i at depth d (roots: 0) has logical
 * position S + d.  diag == NULL: it sees every cached token and its whole line.  diag->mode ==
 * DSA_MASK_WINDOW: of both, the tokens fewer than `window` positions behind it, the prompt, and the
 * first n_sink decode tokens.  Other modes are refused (DSA_ERR_UNSUPPORTED), and so is a bounded
 * cache (ring_size > 0), whose slots the rejected rows would have overwritten.
 *   problem->q [B, N, H_q, D], k_new / v_new [B, N, H_kv, D], out [B, N, H_q, D], lse [B, N, H_q]:
 *   contiguous, the first four 16-byte aligned.  Of problem->plan_flags nothing is used; split_tokens
 *   is honoured (cached tokens per thread block, rounded up to 64).
 *   The rows of node i go to cache position S + i whatever the tree's shape (dsa_compact_kv puts the
 *   accepted ones in order).  Nodes without room (S + i >= max_seq_len) are dropped like those at and
 *   behind node_count[b]: nothing is appended, out = 0, lse = -inf; k_new, v_new and q of such nodes may
 *   hold anything.  A negative seq_len drops all nodes.
 *   A node whose page is missing (its entry in the block table is outside [0, num_blocks), after
 *   dsa_reserve_pages found none for instance) is computed, but its rows are stored nowhere.
 *   dsa_verify_tree does not know which nodes have room and pages: a caller whose requests can run out of them
 *   leaves such nodes out of node_count, on the device, between dsa_reserve_pages and this call (none where
 *   status[b] is not 0 or seq_len[b] negative; else at most max_seq_len - seq_len[b]), and gives both calls the
 *   same.  dsa_compact_kv counts no row that is missing.
 *   Cached rows that no node of the request sees may hold anything (NaN included); a NaN or infinity in
 *   the V row of a token that some node sees reaches the other nodes of the request as well.
 */
DSA_API int32_t dsa_tree_step(const dsa_problem *problem, const dsa_diag_params *diag, const dsa_tree *tree,
                              const void *k_new, const void *v_new, void *out, float *lse,
                              void *workspace, size_t workspace_bytes, void *stream);

/* What dsa_verify_tree checks the drafted tokens against. */
typedef struct dsa_verify {
    int32_t batch;             /* B                                                                          */
    int32_t vocab;             /* V >= 1                                                                     */
    int32_t dtype;             /* dsa_dtype of target_probs and draft_probs                                  */
    const int32_t *tokens;     /* device [B, N]: the token drafted at each node (node 0's is not read)       */
    const void *target_probs;  /* device, row (b, i) at (b*N + i) * target_stride: the target's distribution */
                               /* of the token that follows node i (greedy: any scores, logits for instance) */
    int64_t target_stride;     /* elements, >= V                                                             */
    const void *draft_probs;   /* device, likewise: the distribution that node i's children were drawn from, */
                               /* each on its own; NULL: the children were chosen, not drawn                 */
    int64_t draft_stride;
    const float *uniforms;     /* device [B, N] in [0, 1): [b][i] decides about node i, [b][0] the last      */
                               /* token.  NULL: greedy                                                       */
} dsa_verify;

/*
 * Which drafted tokens stand.  Node 0 is the last token that is settled already; the walk starts there.
 * At a node c with target row p (and draft row q) the children of c are tested in index order; the first
 * that is accepted becomes c, and where none is the walk ends and the token behind c is chosen:
 *   greedy         a child stands iff its token is the (lowest) argmax of p; the token behind c is that argmax.
 *   sampled        v = p, W = 1.  Child i with token x stands iff u_i W q(x) < v(x); otherwise
 *                  v <- max(v - W q, 0), W <- sum v.  (The rejection sampling that leaves the target's
 *                  distribution unchanged.)
 *   chosen (draft_probs NULL)  the same with q a point: child i stands iff u_i W < v(x); otherwise
 *                  W <- W - v(x), v(x) <- 0.
 * The token behind c is then the lowest k with v(0) + ... + v(k) > u_0 sum v (v = p again where nothing is
 * left of v; -1 where p has no positive entry either).  Sums and products are fp64, so that the order of
 * the additions decides about nothing.  Tokens outside [0, V) never stand and change nothing.
 * Greedy: a NaN counts as -inf.  Probabilities are finite and not negative (subnormal floats count as 0); a
 * row with others gives some token or -1, and no fault.
 *   path [B, N] int32: the nodes that stand, node 0 first, -1 behind them; accepted [B]: how many they
 *   are; next_token [B].  A request without nodes gets accepted = 0, next_token = -1.
 * path / accepted are what dsa_compact_kv takes as keep / keep_count.  No workspace.
 */
DSA_API int32_t dsa_verify_tree(const dsa_verify *verify, const dsa_tree *tree, int32_t *path, int32_t *accepted,
                                int32_t *next_token, void *stream);

/*
 * Moves kept tokens together: for i < keep_count[b] the K and V rows at position base[b] + keep[b][i] go to
 * position base[b] + i, in place.  keep [B, max_keep] device, ascending without repeats (so keep[b][i] >= i; max_keep at
 * most 2^30, B * max_keep at most 2^32);
 * keep_count [B] device, clamped to [0, max_keep]; base [B] device, or NULL for 0.  After a verified tree:
 * base = seq_len, keep = path.  To drop tokens for good: base = NULL, keep = the positions that stay.
 * len_out [B] device or NULL: base[b] + (the clamped) keep_count[b], but no further than the first kept row that the
 * cache does not have or has no place for (a position outside [0, max_seq_len) or without a page): a length never counts
 * rows that were stored nowhere.  It may be seq_len, base or keep_count itself.
 * The cache is that of `problem` (q and max_seq_len's sense as elsewhere: rows at positions outside
 * [0, max_seq_len), or whose page is missing, are neither read nor written; refused for bounded caches); with num_layers > 1 the
 * layers' caches lie stride_layer elements apart behind k_cache and v_cache and one call serves all of them.
 * A list that is not ascending gives wrong rows, not faults.  Rows move in place, for every request that reads
 * them: a page that several block-table entries name must not lie behind the first row that moves.
 */
DSA_API int32_t dsa_compact_kv(const dsa_problem *problem, int32_t num_layers, int64_t stride_layer,
                               const int32_t *base, const int32_t *keep, const int32_t *keep_count, int32_t max_keep,
                               int32_t *len_out, void *stream);

/* The pages of a paged cache: a page is free while its count is 0 (a negative count is left as it is, but for the
 * lowest max_blocks numbers there are, which dsa_reserve_pages uses while it runs).  Pages are taken lowest index
 * first, so that equal calls give equal tables.  All arrays on the device; the caller zeroes ref_count to begin with
 * (and fills block tables with -1, the mark of an entry without a page).  Calls on one pool are ordered by
 * the caller: one stream, or events. */
typedef struct dsa_page_pool {
    int32_t num_blocks;        /* pages of the pool                                                          */
    int32_t block_size;        /* tokens per page                                                            */
    int32_t *ref_count;        /* [num_blocks] block-table entries that name the page                        */
} dsa_page_pool;

/*
 * Gives every row of block_table [batch, max_blocks] the pages that it lacks to hold seq_len[b] +
 * extra_tokens tokens (rows with a negative seq_len: none).  Rows are served in order; status[b] is 0, or
 * the number of pages the row lacks and did not get: a row whose demand goes beyond what is left, then,
 * gets nothing, and neither does any row behind it that lacks pages; a row longer than max_blocks gets
 * nothing by itself.  Entries that are not -1 (any negative value counts as -1) are left as they are.
 * At most 4000 rows per call (more: DSA_ERR_UNSUPPORTED).
 */
DSA_API int32_t dsa_reserve_pages(const dsa_page_pool *pool, int32_t *block_table, int32_t batch, int32_t max_blocks,
                                  const int32_t *seq_len, int32_t extra_tokens, int32_t *status, void *stream);

/*
 * Gives back the pages behind the first keep_tokens[b] tokens of every row (negative: none of them;
 * keep_tokens NULL: all pages of all rows): the entries become -1 and the pages' counts fall by one.
 */
DSA_API int32_t dsa_release_pages(const dsa_page_pool *pool, int32_t *block_table, int32_t batch, int32_t max_blocks,
                                  const int32_t *keep_tokens, void *stream);

/*
 * Branches requests: row dst[i] of problem's block table becomes a continuation of row src[i], i < n.  The
 * pages that src[i] has filled are shared (their counts rise); its part-filled last page is copied, in all
 * layers, to a fresh page; the entries behind it become -1; seq_len and prompt_len of dst[i] become those
 * of src[i].  (These arrays of `problem` are therefore WRITTEN.)  What row dst[i] held is overwritten without
 * being given back: release it first.  One source may have many branches.  New tokens of either go to pages of its
 * own; rows within the shared length are not to be written again (moved, or taken back and appended anew) while the
 * other lives.
 * status[i]: 0; 1: no free page was left for it, nothing was changed; 2: refused, nothing was changed:
 * src[i] or dst[i] is no row of the table, a page within src[i]'s length is missing (its entry is outside
 * [0, num_blocks)), or dst[i] is also src or an earlier dst of the same call.
 * workspace: 16 * n bytes, 256-byte aligned.  num_layers, stride_layer as for dsa_compact_kv.
 */
DSA_API int32_t dsa_fork_pages(const dsa_page_pool *pool, const dsa_problem *problem, int32_t num_layers,
                               int64_t stride_layer, const int32_t *src, const int32_t *dst, int32_t n, int32_t *status,
                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * Copies whole pages src[i] -> dst[i], i < n, of all layers (device arrays; pairs with an index outside the
 * pool are skipped).  No page may be the destination of two pairs, or destination and source.
 */
DSA_API int32_t dsa_copy_pages(const dsa_problem *problem, int32_t num_layers, int64_t stride_layer,
                               const int32_t *src, const int32_t *dst, int32_t n, void *stream);

/* ==== Latent caches: one shared row a token ==========================================================
 *
 * A latent cache holds ONE row a token for all heads: latent_dim numbers c_j that every head's keys and
 * values are linear maps of, and rope_dim more, r_j, that carry the position (not in the paper).
 * Two forms of the same attention:
 *   absorbed  the maps have been multiplied into the query and come off the result afterwards, so that all
 *             heads attend over the cached rows themselves: dsa_latent_step, for new tokens over a cache;
 *   expanded  keys and values are computed per head: dsa_latent_prompt, for the tokens of prompts, where that
 *             costs fewer operations (2 (nope_dim + rope_dim + value_dim) a query and key against
 *             2 (2 latent_dim + rope_dim)).
 * dsa_map_tokens says where the tokens of a ragged batch go in a cache (pages from dsa_reserve_pages), and
 * dsa_store_rows / dsa_gather_rows take their rows there or back.
 *
 * All conventions above hold, and those of the drafted-token calls with regard to predecessors, successors
 * and DSA_PLAN_METADATA_STABLE (dsa_map_tokens and dsa_store_rows write no lengths and no tables).
 */
typedef struct dsa_latent {
    int32_t batch;             /* B                                                                          */
    int32_t latent_dim;        /* R: 256 or 512                                                              */
    int32_t rope_dim;          /* P: a multiple of 8 in 8 .. 64                                              */
    int32_t dtype;             /* dsa_dtype of cache, q, c_new, out                                          */
    float sm_scale;            /* logit scale, > 0: 1/sqrt of the heads' width BEFORE absorption             */
    void *cache;               /* rows of R + P contiguous elements [c | r], 16-byte aligned                 */
    int64_t stride_batch;      /* element strides as in dsa_problem: token s of request b at                 */
    int64_t stride_token;      /* b*stride_batch + s*stride_token, or with a block_table in page             */
                               /* block_table[b*max_blocks + s/block_size].  Multiples of 16 bytes           */
    const int32_t *seq_len;    /* [B] tokens in the cache                                                    */
    const int32_t *block_table;/* [B, max_blocks] or NULL                                                    */
    int32_t max_blocks;
    int32_t block_size;
    int32_t num_blocks;
    int32_t max_seq_len;       /* HOST upper bound of seq_len[b]; longer sequences are read as ending there  */
} dsa_latent;

#define DSA_LATENT_MAX_NEW 64

/* Bytes of workspace dsa_latent_step needs for max_new tokens a request and num_heads heads. */
DSA_API int32_t dsa_latent_workspace_size(const dsa_latent *latent, int32_t num_heads, int32_t max_new, size_t *bytes);

/*
 * One pass of up to max_new (N, 1 .. DSA_LATENT_MAX_NEW) new tokens a request: appends their rows to the
 * cache and lets every token i attend, with all heads, over the S = seq_len[b] cached tokens and the new
 * tokens 0 .. i.  With the query row of head h split as q = [a | e]:
 *   x_j = sm_scale * (a . c_j + e . r_j),  lse = ln sum_j e^{x_j},  out = sum_j e^{x_j - lse} c_j.
 *   q [B, N, num_heads, R + P], c_new [B, N, R + P], out [B, N, num_heads, R], lse [B, N, num_heads] float32:
 *   contiguous, the first three 16-byte aligned.
 *   new_count [B] device or NULL: tokens 0 .. new_count[b]-1 of the request exist (clamped to [0, N]); NULL: all N.
 *   Token i's row goes to position S + i; seq_len is not modified.  Tokens without room (S + i >= max_seq_len)
 *   are dropped like those at and behind new_count[b]: nothing is appended, out = 0, lse = -inf; their q and
 *   c_new rows may hold anything.  A negative seq_len drops all.  A token whose page is missing is computed, but
 *   its row is stored nowhere.  Cached rows behind S may hold anything (NaN included); a NaN or infinity in a row
 *   that some of the request's new tokens see may reach the other ones.  num_heads: at most 1024.  bf16: bounds that
 *   allow a block more than 2^24 tokens of one sequence are unsupported (a wait in the kernel could pass its limit).
 *   workspace: 256-byte aligned, dsa_latent_workspace_size() bytes.
 */
DSA_API int32_t dsa_latent_step(const dsa_latent *latent, int32_t num_heads, int32_t max_new, const void *q,
                                const void *c_new, const int32_t *new_count, void *out, float *lse,
                                void *workspace, size_t workspace_bytes, void *stream);

/* A ragged batch of prompts with keys and values expanded per head. */
typedef struct dsa_prompt {
    int32_t batch;             /* B                                                                          */
    int32_t num_heads;         /* H                                                                          */
    int32_t nope_dim;          /* numbers of a key that each head has for itself: 64 or 128 ...              */
    int32_t value_dim;         /* ... and of a value: the same                                               */
    int32_t rope_dim;          /* numbers of a key that all heads share: a multiple of 8 in 8 .. 64          */
    int32_t dtype;             /* dsa_dtype of q, k_nope, k_rope, v and out                                  */
    float sm_scale;            /* logit scale; 0 means 1/sqrt(nope_dim + rope_dim)                           */
    int32_t q_tokens;          /* rows of q, out and lse                                                     */
    int32_t kv_tokens;         /* rows of k_nope, k_rope and v                                               */
    int32_t max_q_len;         /* HOST upper bound of a request's queries (q_tokens will do: however loose   */
                               /* it is, the launch is sized by q_tokens and batch as well).  Queries beyond */
                               /* it are left out (out and lse stay as they were)                            */
    /* Rows of a token and head, contiguous, 16-byte aligned, at token*stride_token + head*stride_head
     * elements (multiples of 16 bytes): q [.., nope_dim + rope_dim], the others as they are named. */
    const void *q;
    int64_t q_stride_token, q_stride_head;
    const void *k_nope;
    int64_t k_stride_token, k_stride_head;
    const void *k_rope;        /* one row a token                                                            */
    int64_t rope_stride_token;
    const void *v;
    int64_t v_stride_token, v_stride_head;
    const int32_t *q_start;    /* device [B + 1], ascending: request b has the query rows                    */
                               /* q_start[b] .. q_start[b+1]-1 ...                                           */
    const int32_t *kv_start;   /* ... and the keys kv_start[b] .. kv_start[b+1]-1; NULL: q_start             */
    int32_t causal;            /* 0: every query sees all keys of its request; else query i of Lq, with Lk   */
                               /* keys, sees the keys j <= i + Lk - Lq (its own is the last)                 */
} dsa_prompt;

/*
 * Attention of the tokens of a ragged batch, per head h:
 *   x_ij = sm_scale * q_i . [k_nope_j | k_rope_j],  lse_i = ln sum_j e^{x_ij},  out_i = sum_j e^{x_ij - lse_i} v_j
 * over the keys that query i sees.  out [q_tokens, H, value_dim] (16-byte aligned), lse [q_tokens, H] float32: contiguous.
 * A query that sees no key (Lk < Lq) gets out = 0, lse = -inf.  Rows that belong to no request are left as they were.  Starts
 * are clamped into [0, q_tokens] / [0, kv_tokens].  Keys and values that no query of the request sees may hold anything; a NaN
 * or infinity in the v row of a key that some query sees may reach the other queries of the request.  num_heads: at most 1024,
 * batch 2^20, kv_tokens 2^25 (bf16; a wait in the kernel could pass its limit).  No workspace.
 */
DSA_API int32_t dsa_latent_prompt(const dsa_prompt *prompt, void *out, float *lse, void *stream);

/* The tokens of a ragged batch and the cache they belong to. */
typedef struct dsa_token_map {
    int32_t batch;             /* B                                                                          */
    int32_t max_tokens;        /* entries of slot, position, request; tokens beyond them are left out        */
    const int32_t *count;      /* device [B]: tokens of each request in the batch (negative: none)           */
    const int32_t *base;       /* device [B]: position of its first one (seq_len), or NULL for 0             */
    const int32_t *block_table;/* device [B, max_blocks], or NULL: request b has the slots                   */
                               /* b*max_seq_len .. (b+1)*max_seq_len-1                                       */
    int32_t max_blocks;
    int32_t block_size;
    int32_t num_blocks;
    int32_t max_seq_len;       /* tokens a request has room for                                              */
} dsa_token_map;

/*
 * Lays the tokens of the requests end to end: start[b] is the number of tokens before request b, start[B] all of
 * them (both at most max_tokens), and for its token k (entry t = start[b] + k):
 *   request[t] = b, position[t] = base[b] + k, slot[t] = page * block_size + position % block_size with the page
 *   that block_table names, or -1: no room (position outside [0, max_seq_len)) or no page (entry outside [0, num_blocks)).
 * Entries behind the last token: -1 in all three.  start [B + 1], position and request [max_tokens] int32, slot
 * [max_tokens] int64; position and request may be NULL.
 * start is what dsa_prompt takes as q_start / kv_start, slot what the row calls take.  With base NULL and count the
 * cached lengths the map names the tokens in the cache.  batch: at most 8192.
 */
DSA_API int32_t dsa_map_tokens(const dsa_token_map *map, int32_t *start, int64_t *slot, int32_t *position,
                               int32_t *request, void *stream);

/*
 * Copies rows of R + P elements between a batch and a latent cache: row t, at rows + t*row_stride elements (a multiple of
 * 16 bytes, 16-byte aligned), goes to (store) or comes from (gather) the token at slot[t], t < count.  slot: device int64,
 * as dsa_map_tokens gives it: page slot / block_size with a block_table, else request slot / max_seq_len.  Rows whose slot lies
 * outside the cache are skipped: nothing is stored, or the batch's row stays as it was.  No two rows of a store may have the
 * same slot.  Of `latent` seq_len, sm_scale and the table's entries are not used.
 */
DSA_API int32_t dsa_store_rows(const dsa_latent *latent, const int64_t *slot, int32_t count, const void *rows,
                               int64_t row_stride, void *stream);
DSA_API int32_t dsa_gather_rows(const dsa_latent *latent, const int64_t *slot, int32_t count, void *rows,
                                int64_t row_stride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DSA_H */
