// Verification of drafted tokens against the target's probabilities (dsa_verify_tree).
//
// The walk down the tree is a chain of decisions, and a decision needs two numbers only, p(x) and q(x) of the
// child's token: they are fetched for all nodes at once before the walk starts.  A row of the vocabulary is
// read in whole only where a child was turned down (the residual max(v - W q, 0) and its sum) and where the
// walk ends (the sum that the last token is drawn from; the last rejection's own pass serves for that), so a
// walk that accepts reads nothing but its end.  Greedy decoding reads the row of every node on the path.
//
// What bounds it: one or two rows of p and q per request, some 100 KB to 1 MB, and then the latency of the
// passes, one after the other.  So a request is worked on by a cluster of up to 8 blocks, each with a
// contiguous piece of the vocabulary cut into one run per warp, and blocks exchange nothing but one sum per
// warp through distributed shared memory.  The residual after k rejections is recomputed from p, q and the k
// weights W in every pass; nothing is stored.
//
// Sums are in double precision: with 32 bits the token at the border of a cumulative sum would hang on the
// order of the additions (at 65536 entries and 24 bits once in some hundred draws), with 53 it does not.
#include "dsa_host.cuh"

#include <algorithm>

namespace {

using namespace dsa;

constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCluster = 8;
constexpr int kVerifyMaxNodes = DSA_TREE_MAX_NODES;

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

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) dsa_verify_kernel(const VerifyArgs a) {
    // one sum (greedy: best score and its index) per warp of the cluster, two sets: the blocks may be one pass apart
    __shared__ double s_sum[2][kVerifyMaxCluster * kVerifyWarps];
    __shared__ float s_best[2][kVerifyMaxCluster * kVerifyWarps];
    __shared__ int s_arg[2][kVerifyMaxCluster * kVerifyWarps];
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
    const bool greedy = a.u == nullptr, points = a.q == nullptr;
    if (tid < a.N) {
        const int64_t i = (int64_t)b * a.N + tid;
        const int x = a.tokens[i];
        int up = a.parent ? a.parent[i] : tid - 1;
        if (up < 0 || up >= tid) up = -1;
        s_token[tid] = x;
        s_parent[tid] = up;
        s_u[tid] = greedy ? 0.f : a.u[i];
        const bool valid = up >= 0 && x >= 0 && x < a.V;
        const int64_t row = (int64_t)b * a.N + max(up, 0);
        s_p[tid] = valid && !greedy ? (float)p0[row * a.p_stride + x] : 0.f;
        s_q[tid] = valid && !greedy && !points ? (float)q0[row * a.q_stride + x] : 0.f;
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

    cluster_barrier();                                       // every block has started: its shared memory may be written
    const int slot = (int)rank * kVerifyWarps + warp;        // this warp's run of the vocabulary: [lo, hi)
    const int n_runs = (int)blocks * kVerifyWarps, per_lane = (n_runs + 31) / 32;
    const int lo = (int)min((int64_t)slot * a.run, (int64_t)a.V), hi = (int)min((int64_t)(slot + 1) * a.run, (int64_t)a.V);
    int pass = 0;
    auto publish_sum = [&](double v) {
        if (lane < (int)blocks)
            asm volatile("st.shared::cluster.f64 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_sum[pass & 1][slot]), lane)), "d"(v) : "memory");
    };
    auto rows_of = [&](int node, const T*& p, const T*& q, bool& vec) {
        const int64_t row = (int64_t)b * a.N + node;
        p = p0 + row * a.p_stride;
        q = points ? p : q0 + row * a.q_stride;
        constexpr uintptr_t mask = 4 * sizeof(T) - 1;
        vec = ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & mask) == 0;
    };
    // the sum of what is left at `node` after res.k rejections; leaves the warps' sums in s_sum[(pass - 1) & 1]
    auto sum_left = [&](int node, const Residual& res) -> double {
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        double acc[4] = {0.0, 0.0, 0.0, 0.0};
        const bool need_q = !points && res.k > 0;
#pragma unroll 2
        for (int i = lo + 4 * lane; i < hi; i += 128) {
            float fp[4], fq[4] = {0.f, 0.f, 0.f, 0.f};
            load4(p, i, hi, vec, fp);
            if (need_q) load4(q, i, hi, vec, fq);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[e] += need_q ? res.with_draft(fp[e], fq[e]) : points ? res.with_points(fp[e], i + e) : (double)fp[e];
        }
        double v = (acc[0] + acc[1]) + (acc[2] + acc[3]);
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
        publish_sum(v);
        cluster_barrier();
        double total = 0.0;                                  // (the same additions in every warp of every block)
        for (int w = lane * per_lane; w < min(n_runs, (lane + 1) * per_lane); ++w) total += s_sum[pass & 1][w];
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
        ++pass;
        return total;
    };
    // the lowest index whose cumulative sum exceeds u * total; the warps' sums are in s_sum[(pass - 1) & 1]
    auto draw = [&](int node, const Residual& res, float u, double total) {
        const double* sums = s_sum[(pass - 1) & 1];
        const double goal = (double)u * total;
        const int w0 = lane * per_lane, w1 = min(n_runs, w0 + per_lane);
        double mine = 0.0;
        for (int w = w0; w < w1; ++w) mine += sums[w];
        double upto = mine;                                  // inclusive prefix over the lanes
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const double o = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += o;
        }
        int hit_run = 0x7fffffff, last_run = -1;
        double at_run = upto - mine, at_hit = 0.0, at_last = 0.0;
        for (int w = w0; w < w1; ++w) {
            const double s = sums[w];
            if (s > 0.0) {
                last_run = w; at_last = at_run;
                if (hit_run == 0x7fffffff && at_run + s > goal) { hit_run = w; at_hit = at_run; }
            }
            at_run += s;
        }
        int run = __reduce_min_sync(0xffffffffu, hit_run);
        const bool hit = run != 0x7fffffff;
        if (!hit) run = __reduce_max_sync(0xffffffffu, last_run);    // (rounding: the last run with anything in it)
        if (run != slot) return;                             // (every warp finds the same run; the one it belongs to goes on)
        double before = __shfl_sync(0xffffffffu, hit ? at_hit : at_last, run / per_lane);
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        const bool need_q = !points && res.k > 0;
        int found = -1, last = -1;
        for (int i0 = lo; i0 < hi && found < 0; i0 += 128) {
            const int i = i0 + 4 * lane;
            float fp[4] = {0.f, 0.f, 0.f, 0.f}, fq[4] = {0.f, 0.f, 0.f, 0.f};
            if (i < hi) {
                load4(p, i, hi, vec, fp);
                if (need_q) load4(q, i, hi, vec, fq);
            }
            double v[4];
            mine = 0.0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = need_q ? res.with_draft(fp[e], fq[e]) : points ? res.with_points(fp[e], i + e) : (double)fp[e];
                mine += v[e];
            }
            upto = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const double o = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += o;
            }
            double at = before + (upto - mine);
            int first = 0x7fffffff, some = -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                at += v[e];
                if (v[e] > 0.0) {
                    some = i + e;
                    if (at > goal) first = min(first, i + e);
                }
            }
            first = __reduce_min_sync(0xffffffffu, first);
            last = max(last, __reduce_max_sync(0xffffffffu, some));
            if (first != 0x7fffffff) found = first;
            before += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (found < 0) found = last;                         // (rounding: the last entry with anything in it)
        if (lane == 0) a.next_token[b] = found;
    };
    // the lowest index of the largest score at `node`
    auto best_of = [&](int node) -> int {
        const T *p, *q;
        bool vec;
        rows_of(node, p, q, vec);
        float best = -INFINITY;
        int arg = 0x7fffffff;
#pragma unroll 4
        for (int i = lo + 4 * lane; i < hi; i += 128) {
            float f[4];
            load4(p, i, hi, vec, f);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < hi && (f[e] > best || arg == 0x7fffffff)) { best = f[e]; arg = i + e; }
        }
        auto better = [](float x, int ix, float y, int iy) { return x > y || (x == y && ix < iy) || iy == 0x7fffffff; };
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, best, off);
            const int oi = __shfl_xor_sync(0xffffffffu, arg, off);
            if (oi != 0x7fffffff && better(o, oi, best, arg)) { best = o; arg = oi; }
        }
        if (lane < (int)blocks) {
            asm volatile("st.shared::cluster.f32 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_best[pass & 1][slot]), lane)), "f"(best) : "memory");
            asm volatile("st.shared::cluster.u32 [%0], %1;"
                         ::"r"(map_to_rank(smem_u32(&s_arg[pass & 1][slot]), lane)), "r"(arg) : "memory");
        }
        cluster_barrier();
        best = -INFINITY;
        arg = 0x7fffffff;
        for (int w = 0; w < n_runs; ++w) {
            const float o = s_best[pass & 1][w];
            const int oi = s_arg[pass & 1][w];
            if (oi != 0x7fffffff && better(o, oi, best, arg)) { best = o; arg = oi; }
        }
        ++pass;
        return arg;
    };

    // ---- the walk: every thread of every block takes the same decisions ----------------------------
    int cur = 0, length = 1;
    Residual res{0, s_weight, s_out};
    double weight = 1.0;                                     // W of the next test
    bool summed = false;                                     // s_sum holds the sums for (cur, res)
    int best = greedy ? best_of(0) : 0;
    if (tid == 0) s_path[0] = 0;
    for (int i = 1; i < n; ++i) {
        if (s_parent[i] != cur) continue;
        const int x = s_token[i];
        bool stands;
        if (greedy) {
            stands = x == best;
        } else {
            if (x < 0 || x >= a.V) continue;
            const double q = points ? 1.0 : (double)s_q[i];
            const double v = points ? res.with_points(s_p[i], x) : res.with_draft(s_p[i], q);
            stands = (double)s_u[i] * weight * q < v;
            if (!stands) {
                __syncthreads();                             // (the last reads of the lists are done)
                if (tid == 0) { s_weight[res.k] = weight; s_out[res.k] = x; }
                __syncthreads();
                ++res.k;
                if (points) {
                    weight -= v;
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
            if (greedy) best = best_of(cur);
            res.k = 0;
            weight = 1.0;
            summed = false;
        }
    }
    if (greedy) {
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
    cluster_barrier();                                       // nobody leaves while its shared memory may be written
}

template <typename T>
cudaError_t launch_verify(const VerifyArgs& a, int batch, int blocks, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)batch * blocks));
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)blocks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, dsa_verify_kernel<T>, a);
}

}  // namespace

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
    // blocks per request: pieces of some 8192 entries, as long as the device has room for all blocks at once
    int blocks = 1;
    while (blocks < kVerifyMaxCluster && (int64_t)blocks * 8192 < v->vocab &&
           (int64_t)v->batch * blocks * 2 <= 4 * (int64_t)host_sm_count())
        blocks *= 2;
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
    const int runs = blocks * kVerifyWarps;
    a.run = ((v->vocab + runs - 1) / runs + 127) / 128 * 128;
    a.path = path;
    a.accepted = accepted;
    a.next_token = next_token;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = v->dtype == DSA_BF16 ? launch_verify<__nv_bfloat16>(a, v->batch, blocks, st)
                                               : launch_verify<float>(a, v->batch, blocks, st);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}
