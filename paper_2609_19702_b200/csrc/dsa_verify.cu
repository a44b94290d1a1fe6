// Verification of drafted tokens against the target's probabilities (dsa_verify_tree).
//
// The walk down the tree is a chain of decisions, and a decision needs two numbers only, p(x) and q(x) of the
// child's token: they are fetched for all nodes at once before the walk starts.  A row of the vocabulary is
// read in whole only where a child was turned down (the residual max(v - W q, 0) and its sum) and where the
// walk ends (the sum that the last token is drawn from; the last rejection's own pass serves for that), so a
// walk that accepts reads nothing but its end.  Greedy decoding reads the row of every node on the path, and
// has the row of the likeliest next one (the first child's) brought into L2 meanwhile.
//
// What bounds it: one or two rows of p and q per request, some 100 KB to 1 MB, and then the latency of the
// passes, one after the other.  So a request is worked on by a cluster of up to 8 blocks, each with a
// contiguous piece of the vocabulary cut into one run per warp, and blocks exchange nothing but one sum per
// warp through distributed shared memory.  The residual of the current node stays in the blocks' shared memory,
// every thread its own entries, so that a second rejection reads q only and the draw reads nothing (in
// registers it cost so many that one block filled an SM: 60 us against 26 for 64 requests x 65536 entries).
// Pieces that shared memory cannot hold (vocabularies beyond some 220000 entries) are read again in every pass
// and the residual is recomputed from the k weights W.
//
// Sums are in double precision: with 32 bits the token at the border of a cumulative sum would hang on the
// order of the additions (at 65536 entries and 24 bits once in some hundred draws), with 53 it does not.
#include "dsa_host.cuh"

#include <algorithm>

namespace {

using namespace dsa;

constexpr int kVerifyMaxCluster = 8;
constexpr int kVerifyMaxNodes = DSA_TREE_MAX_NODES;
constexpr int kVerifyKeepBytes = 216 * 1024;       // of a block's shared memory for the residual

struct VerifyArgs {
    const int* tokens;
    const void* p;
    const void* q;
    int64_t p_stride, q_stride;
    const float* u;
    const int* parent;
    const int* node_count;
    int N, V;
    int run;                       // vocabulary entries per warp, a multiple of 128
    int* path;
    int* accepted;
    int* next_token;
};

// Four consecutive entries of a row from index i on (i a multiple of 4); beyond `end`: zeros.
template <typename T>
__device__ __forceinline__ void load4(const T* row, int i, int end, bool vec, float (&f)[4]) {
    if (vec && i + 4 <= end) {
        if constexpr (sizeof(T) == 4) {
            const float4 x = *reinterpret_cast<const float4*>(row + i);
            f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(row + i);
            f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xffff0000u);
            f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = i + k < end ? (float)row[i + k] : 0.f;
}

__device__ __forceinline__ unsigned map_to_rank(unsigned addr, unsigned rank) {
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// What is left of the target's row at the current node: v_0 = p, v_{k+1} = max(v_k - W_k q, 0), or p with
// the turned-down tokens taken out.
struct Residual {
    int k;                         // rejections at this node
    const double* weight;          // shared: W_0 .. W_{k-1}
    const int* out;                // shared: the k turned-down tokens (draft given as points)
    __device__ __forceinline__ double with_draft(double p, double q) const {
        for (int r = 0; r < k; ++r) p = fmax(fma(-weight[r], q, p), 0.0);
        return p;
    }
    __device__ __forceinline__ double with_points(double p, int x) const {
        for (int r = 0; r < k; ++r)
            if (out[r] == x) p = 0.0;
        return p;
    }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
__device__ __forceinline__ double warp_prefix(double v, int lane) {          // inclusive
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v += o;
    }
    return v;
}
// (score, index): the larger score, of equal ones the lower index; kNone: no entry yet
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ void take_better(float& best, int& arg, float o, int oi) {
    if (oi != kNone && (arg == kNone || o > best || (o == best && oi < arg))) { best = o; arg = oi; }
}

// W warps per block; KEEP: the residual is kept (dynamic shared memory, 8 bytes per entry of the block's piece)
template <typename T, int W, bool GREEDY, bool KEEP>
__global__ void __launch_bounds__(32 * W, 32 / W) dsa_verify_kernel(const VerifyArgs a) {
    constexpr int kRuns = kVerifyMaxCluster * W;
    // one sum (greedy: best score and its index) per warp of the cluster, two sets: the blocks may be one pass apart
    __shared__ double s_sum[2][kRuns];
    __shared__ float s_best[2][kRuns];
    __shared__ int s_arg[2][kRuns];
    extern __shared__ __align__(16) double s_left[];
    __shared__ double s_weight[kVerifyMaxNodes];
    __shared__ int s_out[kVerifyMaxNodes];
    __shared__ int s_token[kVerifyMaxNodes], s_parent[kVerifyMaxNodes], s_path[kVerifyMaxNodes];
    __shared__ float s_u[kVerifyMaxNodes], s_p[kVerifyMaxNodes], s_q[kVerifyMaxNodes];

    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned rank, blocks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const int b = blockIdx.x / blocks;
    const int n = a.node_count ? max(0, min(a.node_count[b], a.N)) : a.N;
    const T* p0 = reinterpret_cast<const T*>(a.p);
    const T* q0 = reinterpret_cast<const T*>(a.q);
    const bool points = a.q == nullptr;
    if (tid < a.N) {
        const int64_t i = (int64_t)b * a.N + tid;
        const int x = a.tokens[i];
        int up = a.parent ? a.parent[i] : tid - 1;
        if (up < 0 || up >= tid) up = -1;
        s_token[tid] = x;
        s_parent[tid] = up;
        s_u[tid] = GREEDY ? 0.f : a.u[i];
        const bool valid = up >= 0 && x >= 0 && x < a.V;
        const int64_t row = (int64_t)b * a.N + max(up, 0);
        s_p[tid] = valid && !GREEDY ? (float)p0[row * a.p_stride + x] : 0.f;
        s_q[tid] = valid && !GREEDY && !points ? (float)q0[row * a.q_stride + x] : 0.f;
        s_path[tid] = -1;
    }
    __syncthreads();
    if (n == 0) {                                            // (the same for every block of the cluster)
        if (rank == 0) {
            if (tid < a.N) a.path[(int64_t)b * a.N + tid] = -1;
            if (tid == 0) { a.accepted[b] = 0; a.next_token[b] = -1; }
        }
        return;
    }
    if (blocks > 1) cluster_barrier();                       // every block has started: its shared memory may be written

    const int slot = (int)rank * W + warp;                   // this warp's run of the vocabulary: [lo, hi)
    const int n_runs = (int)blocks * W, per_lane = (n_runs + 31) / 32;
    const int lo = (int)min((int64_t)slot * a.run, (int64_t)a.V), hi = (int)min((int64_t)(slot + 1) * a.run, (int64_t)a.V);
    int pass = 0;
    auto meet = [&]() {                                      // what the warps have published is there
        if (blocks > 1) cluster_barrier(); else __syncthreads();
    };
    auto rows_of = [&](int node, const T*& p, const T*& q, bool& vec) {
        const int64_t row = (int64_t)b * a.N + node;
        p = p0 + row * a.p_stride;
        q = points ? p : q0 + row * a.q_stride;
        constexpr uintptr_t mask = 4 * sizeof(T) - 1;
        vec = ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & mask) == 0;
    };
    double* kept = s_left + warp * a.run;                    // what is left of the current node's row: this warp's run
    int held = -1;                                           // the node that it belongs to
    // the sum of what is left at `node` after res.k rejections; leaves the warps' sums in s_sum[(pass - 1) & 1]
    auto sum_left = [&](int node, const Residual& res) -> double {
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        double acc[4] = {0.0, 0.0, 0.0, 0.0};
        const bool need_q = !points && res.k > 0;
        // a node's first pass follows its first rejection, and every one its own: `kept` lacks the last one only
        const bool fresh = !KEEP || held != node || res.k == 0;
        const double w = KEEP && need_q ? -res.weight[res.k - 1] : 0.0;
#pragma unroll 4
        for (int i = lo + 4 * lane; i < hi; i += 128) {
            float fp[4], fq[4] = {0.f, 0.f, 0.f, 0.f};
            double x[4];
            if (fresh) load4(p, i, hi, vec, fp);
            if (need_q) load4(q, i, hi, vec, fq);
            if (fresh) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (double)fp[e];
            } else {
                const double2 x0 = *reinterpret_cast<const double2*>(kept + (i - lo)), x1 = *reinterpret_cast<const double2*>(kept + (i - lo) + 2);
                x[0] = x0.x; x[1] = x0.y; x[2] = x1.x; x[3] = x1.y;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (KEEP && need_q) x[e] = fmax(fma(w, (double)fq[e], x[e]), 0.0);
                else if (need_q) x[e] = res.with_draft(x[e], fq[e]);
                else if (points) x[e] = res.with_points(x[e], i + e);
                acc[e] += x[e];
            }
            if (KEEP) {
                *reinterpret_cast<double2*>(kept + (i - lo)) = make_double2(x[0], x[1]);
                *reinterpret_cast<double2*>(kept + (i - lo) + 2) = make_double2(x[2], x[3]);
            }
        }
        held = node;
        const double mine = warp_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
        if (lane < (int)blocks)
            asm volatile("st.shared::cluster.f64 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_sum[pass & 1][slot]), lane)), "d"(mine) : "memory");
        meet();
        double total = 0.0;                                  // (the same additions in every warp of every block)
        for (int w = lane * per_lane; w < min(n_runs, (lane + 1) * per_lane); ++w) total += s_sum[pass & 1][w];
        ++pass;
        return warp_sum(total);
    };
    // the lowest index whose cumulative sum exceeds u * total; the warps' sums are in s_sum[(pass - 1) & 1]
    auto draw = [&](int node, const Residual& res, float u, double total) {
        const double* sums = s_sum[(pass - 1) & 1];
        const double goal = (double)u * total;
        const int w0 = lane * per_lane, w1 = min(n_runs, w0 + per_lane);
        double mine = 0.0;
        for (int w = w0; w < w1; ++w) mine += sums[w];
        const double upto_run = warp_prefix(mine, lane);
        int hit_run = kNone, last_run = -1;
        double at_run = upto_run - mine, at_hit = 0.0, at_last = 0.0;
        for (int w = w0; w < w1; ++w) {
            const double s = sums[w];
            if (s > 0.0) {
                last_run = w; at_last = at_run;
                if (hit_run == kNone && at_run + s > goal) { hit_run = w; at_hit = at_run; }
            }
            at_run += s;
        }
        int run = __reduce_min_sync(0xffffffffu, hit_run);
        const bool hit = run != kNone;
        if (!hit) run = __reduce_max_sync(0xffffffffu, last_run);    // (rounding: the last run with anything in it)
        if (run != slot) return;                             // (every warp finds the same run; the one it belongs to goes on)
        double before = __shfl_sync(0xffffffffu, hit ? at_hit : at_last, run / per_lane);
        int found = -1, last = -1;
        // 128 entries in order, four a lane: the first that takes the sum beyond the goal, and the last that is not 0
        auto look = [&](int i, const double (&x)[4]) {
            const double four = (x[0] + x[1]) + (x[2] + x[3]);
            const double upto = warp_prefix(four, lane);
            double at = before + (upto - four);
            int first = kNone, some = -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                at += x[e];
                if (x[e] > 0.0) {
                    some = i + e;
                    if (at > goal) first = min(first, i + e);
                }
            }
            first = __reduce_min_sync(0xffffffffu, first);
            last = max(last, __reduce_max_sync(0xffffffffu, some));
            if (found < 0 && first != kNone) found = first;
            before += __shfl_sync(0xffffffffu, upto, 31);
        };
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        const bool need_q = !points && res.k > 0;
        for (int i0 = lo; i0 < hi && found < 0; i0 += 128) {
            const int i = i0 + 4 * lane;
            double x[4] = {0.0, 0.0, 0.0, 0.0};
            if (i < hi) {
                if (KEEP) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = kept[i - lo + e];
                } else {
                    float fp[4], fq[4] = {0.f, 0.f, 0.f, 0.f};
                    load4(p, i, hi, vec, fp);
                    if (need_q) load4(q, i, hi, vec, fq);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = need_q ? res.with_draft(fp[e], fq[e]) : points ? res.with_points(fp[e], i + e) : (double)fp[e];
                }
            }
            look(i, x);
        }
        if (found < 0) found = last;                         // (rounding: the last entry with anything in it)
        if (lane == 0) a.next_token[b] = found;
    };
    // the lowest index of the largest score at `node`; `next` (or -1): the node whose row is wanted next, likely
    auto best_of = [&](int node, int next) -> int {
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        if (next >= 0) {                                     // one line of the next row per lane and step
            const T* ahead = p0 + ((int64_t)b * a.N + next) * a.p_stride;
            for (int i = lo + lane * (128 / (int)sizeof(T)); i < hi; i += 32 * (128 / (int)sizeof(T)))
                asm volatile("prefetch.global.L2 [%0];" ::"l"(ahead + i));
        }
        float best = -INFINITY;
        int arg = kNone;
#pragma unroll 4
        for (int i = lo + 4 * lane; i < hi; i += 128) {
            float f[4];
            load4(p, i, hi, vec, f);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < hi && (f[e] > best || arg == kNone)) { best = f[e]; arg = i + e; }
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1)
            take_better(best, arg, __shfl_xor_sync(0xffffffffu, best, off), __shfl_xor_sync(0xffffffffu, arg, off));
        if (lane < (int)blocks) {
            asm volatile("st.shared::cluster.f32 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_best[pass & 1][slot]), lane)), "f"(best) : "memory");
            asm volatile("st.shared::cluster.u32 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_arg[pass & 1][slot]), lane)), "r"(arg) : "memory");
        }
        meet();
        best = -INFINITY;
        arg = kNone;
        for (int w = lane * per_lane; w < min(n_runs, (lane + 1) * per_lane); ++w) take_better(best, arg, s_best[pass & 1][w], s_arg[pass & 1][w]);
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1)
            take_better(best, arg, __shfl_xor_sync(0xffffffffu, best, off), __shfl_xor_sync(0xffffffffu, arg, off));
        ++pass;
        return arg;
    };
    auto first_child = [&](int node) -> int {
        for (int i = node + 1; i < n; ++i)
            if (s_parent[i] == node) return i;
        return -1;
    };

    // ---- the walk: every thread of every block takes the same decisions ----------------------------
    int cur = 0, length = 1;
    Residual res{0, s_weight, s_out};
    double weight = 1.0;                                     // W of the next test
    bool summed = false;                                     // s_sum holds the sums for (cur, res)
    int best = 0;
    if constexpr (GREEDY) best = best_of(0, first_child(0));
    if (tid == 0) s_path[0] = 0;
    for (int i = 1; i < n; ++i) {
        if (s_parent[i] != cur) continue;
        const int x = s_token[i];
        bool stands;
        if constexpr (GREEDY) {
            stands = x == best;
        } else {
            if (x < 0 || x >= a.V) continue;
            const double q = points ? 1.0 : (double)s_q[i];
            const double left = points ? res.with_points(s_p[i], x) : res.with_draft(s_p[i], q);
            stands = (double)s_u[i] * weight * q < left;
            if (!stands) {
                __syncthreads();                             // (the last reads of the lists are done)
                if (tid == 0) { s_weight[res.k] = weight; s_out[res.k] = x; }
                __syncthreads();
                ++res.k;
                if (points) {
                    weight -= left;
                } else {
                    weight = sum_left(cur, res);
                    summed = true;
                }
            }
        }
        if (stands) {
            cur = i;
            if (tid == 0) s_path[length] = i;
            ++length;
            if constexpr (GREEDY) best = best_of(cur, first_child(cur));
            res.k = 0;
            weight = 1.0;
            summed = false;
        }
    }
    if constexpr (GREEDY) {
        if (rank == 0 && tid == 0) a.next_token[b] = best;
    } else {
        double total = weight;
        if (!summed) total = sum_left(cur, res);
        if (!(total > 0.0) && res.k > 0) {                   // nothing is left of v: the target's row itself
            res.k = 0;
            total = sum_left(cur, res);
        }
        if (total > 0.0) draw(cur, res, s_u[0], total);
        else if (rank == 0 && tid == 0) a.next_token[b] = -1;
    }
    __syncthreads();
    if (rank == 0) {
        if (tid < a.N) a.path[(int64_t)b * a.N + tid] = s_path[tid];
        if (tid == 0) a.accepted[b] = length;
    }
    if (blocks > 1) cluster_barrier();                       // nobody leaves while its shared memory may be written
}

template <typename T, int W, bool GREEDY, bool KEEP>
cudaError_t configure_verify() {
    static std::atomic<bool> done[kMaxDevices] = {};
    return KEEP ? configure_smem(dsa_verify_kernel<T, W, GREEDY, KEEP>, kVerifyKeepBytes, done) : cudaSuccess;
}

template <typename T, int W, bool GREEDY, bool KEEP>
cudaError_t launch_verify(const VerifyArgs& a, int batch, int blocks, cudaStream_t st) {
    const cudaError_t e = configure_verify<T, W, GREEDY, KEEP>();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)batch * blocks));
    cfg.blockDim = dim3(32 * W);
    cfg.dynamicSmemBytes = KEEP ? (size_t)W * a.run * sizeof(double) : 0;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)blocks;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = blocks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, dsa_verify_kernel<T, W, GREEDY, KEEP>, a);
}

template <typename T>
cudaError_t run_verify(VerifyArgs& a, int batch, cudaStream_t st) {
    // Four warps and 512 entries each are enough for small vocabularies; else sixteen, and as many blocks (up to
    // eight) as keep a warp's run at 512 entries, whatever the batch: a pass is all latency, so that more and
    // shorter ones at a time are the faster way through many requests as well.
    const bool greedy = a.u == nullptr;
    const int warps = a.V <= 2048 ? 4 : 16;
    int blocks = 1;
    while (blocks < kVerifyMaxCluster && (int64_t)blocks * warps * 512 < a.V) blocks *= 2;
    const int runs = blocks * warps;
    a.run = ((a.V + runs - 1) / runs + 127) / 128 * 128;
    const bool keep = (int64_t)warps * a.run * 8 <= kVerifyKeepBytes;
    if (warps == 4) return greedy ? launch_verify<T, 4, true, false>(a, batch, blocks, st) : launch_verify<T, 4, false, true>(a, batch, blocks, st);
    if (greedy) return launch_verify<T, 16, true, false>(a, batch, blocks, st);
    return keep ? launch_verify<T, 16, false, true>(a, batch, blocks, st) : launch_verify<T, 16, false, false>(a, batch, blocks, st);
}

}  // namespace

namespace dsa {
cudaError_t verify_prepare() {
    cudaError_t e = configure_verify<float, 4, false, true>();
    if (e == cudaSuccess) e = configure_verify<float, 16, false, true>();
    if (e == cudaSuccess) e = configure_verify<__nv_bfloat16, 4, false, true>();
    if (e == cudaSuccess) e = configure_verify<__nv_bfloat16, 16, false, true>();
    return e;
}
}  // namespace dsa

extern "C" int32_t dsa_verify_tree(const dsa_verify* v, const dsa_tree* tree, int32_t* path, int32_t* accepted,
                                   int32_t* next_token, void* stream) {
    if (!v || !tree || v->batch < 0 || v->vocab < 1 || tree->max_nodes < 1) return DSA_ERR_INVALID_ARG;
    if (tree->max_nodes > DSA_TREE_MAX_NODES) return DSA_ERR_UNSUPPORTED;
    if (v->dtype != DSA_BF16 && v->dtype != DSA_F32) return DSA_ERR_UNSUPPORTED;
    if (v->target_stride < v->vocab || (v->draft_probs && v->draft_stride < v->vocab)) return DSA_ERR_INVALID_ARG;
    if (v->vocab > (1 << 30) || v->batch > (1 << 26)) return DSA_ERR_UNSUPPORTED;
    if (v->batch == 0) return DSA_OK;
    if (!v->tokens || !v->target_probs || !path || !accepted || !next_token) return DSA_ERR_INVALID_ARG;
    const uintptr_t esize = v->dtype == DSA_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(v->target_probs) % esize || reinterpret_cast<uintptr_t>(v->draft_probs) % esize)
        return DSA_ERR_INVALID_ARG;
    if (v->draft_probs && !v->uniforms) return DSA_ERR_INVALID_ARG;      // (greedy decoding knows no draft probabilities)
    VerifyArgs a = {};
    a.tokens = v->tokens;
    a.p = v->target_probs;
    a.q = v->draft_probs;
    a.p_stride = v->target_stride;
    a.q_stride = v->draft_stride;
    a.u = v->uniforms;
    a.parent = tree->parent;
    a.node_count = tree->node_count;
    a.N = tree->max_nodes;
    a.V = v->vocab;
    a.path = path;
    a.accepted = accepted;
    a.next_token = next_token;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = v->dtype == DSA_BF16 ? run_verify<__nv_bfloat16>(a, v->batch, st) : run_verify<float>(a, v->batch, st);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}
