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
// warp through distributed shared memory.  The residual of the current node stays in their shared memory, every
// thread its own entries, so that a second rejection reads q only and the draw reads nothing; pieces too large for
// that (vocabularies beyond some 220000 entries) are read again in every pass and the residual is recomputed from
// the k weights W.
//
// Precision: with 24-bit sums the token at the border of a cumulative sum would hang on the order of the additions
// (at 65536 entries once in some hundred draws).  Entries and sums are fp64; floats are widened by their bits, since the
// unit that converts is much narrower than the one that adds (pairs of floats, high and low, took 38 us where this takes
// 35).  One warp of a block walks the tree and tells the others what to do.
//
// Measured: 64 requests of 32 nodes, 65536 entries, sampled: 35-40 us, one to five passes a request (33 MB; a pass is
// 3.3 us: 1 us of loads, 1 us of arithmetic and shared memory, the rest the meeting of the blocks and the next decision,
// and the 512 blocks need two rounds of SMs).  One request, 16384 entries: 7 us.  Greedy, 32 requests of 16 nodes: 22 us,
// 2.5 us a node on the path; taking a node and its first child in one pass was slower (24-26 us: the rows that are then
// read in vain cost more than the passes saved), and so were 8 warps a block (one round: 34 us instead of 28).
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

// ---- fp64 -------------------------------------------------------------------------------------------------
// A float as a double, by its bits (the unit that converts is a fourth as wide as the one that adds; a subnormal
// float counts as 0).
__device__ __forceinline__ double widen(float f) {
    const int x = __float_as_int(f);
    const bool some = (x & 0x7f800000) != 0;
    return __hiloint2double(some ? ((x >> 3) & 0x8fffffff) + 0x38000000 : 0, some ? x << 29 : 0);
}
__device__ __forceinline__ double reject(double v, double w, double q) { return fmax(__fma_rn(-w, q, v), 0.); }

__device__ __forceinline__ double warp_sum(double v) {                      // lane 0's order of additions, for every lane
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) v += __shfl_down_sync(0xffffffffu, v, off);
    return __shfl_sync(0xffffffffu, v, 0);
}
__device__ __forceinline__ double warp_prefix(double v, int lane) {         // of the lanes before this one
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v += o;
    }
    const double up = __shfl_up_sync(0xffffffffu, v, 1);
    return lane > 0 ? up : 0.;
}
// (score, index): the larger score, of equal ones the lower index; kNone: no entry yet
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ void take_better(float& best, int& arg, float o, int oi) {
    if (oi != kNone && (arg == kNone || o > best || (o == best && oi < arg))) { best = o; arg = oi; }
}

// What the blocks' warps are told to do next: sum what is left at `node` after `k` rejections; draw from it (warp
// `run` of the cluster, whose entries begin at the cumulative sum `before`, looks for `goal`); or nothing any more.
enum : int { kSum, kDraw, kDone };
struct Task {
    int what, node, k, run;
    double before, goal;
};

// W warps per block; KEEP: the residual is kept (dynamic shared memory, 8 bytes per entry of the block's piece)
template <typename T, int W, bool GREEDY, bool KEEP>
__global__ void __launch_bounds__(32 * W, (GREEDY ? 48 : 32) / W) dsa_verify_kernel(const VerifyArgs a) {
    constexpr int kRuns = kVerifyMaxCluster * W;
    // one sum (greedy: best score and its index) per warp of the cluster, two sets: the blocks may be one pass apart
    __shared__ double s_sum[2][kRuns];
    __shared__ float s_best[2][kRuns];
    __shared__ int s_arg[2][kRuns];
    __shared__ Task s_task;
    __shared__ double s_weight[kVerifyMaxNodes];               // W of the rejections at the current node
    __shared__ int s_out[kVerifyMaxNodes];                   // and the turned-down tokens (draft given as points)
    __shared__ int s_token[kVerifyMaxNodes], s_parent[kVerifyMaxNodes], s_path[kVerifyMaxNodes];
    __shared__ unsigned s_children[2 * kVerifyMaxNodes];     // of every node, a bit each
    __shared__ float s_u[kVerifyMaxNodes], s_p[kVerifyMaxNodes], s_q[kVerifyMaxNodes];
    extern __shared__ __align__(16) double s_left[];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned rank, blocks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    if (blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // (this block has started)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x / blocks;
    const int n = a.node_count ? max(0, min(a.node_count[b], a.N)) : a.N;
    const T* p0 = reinterpret_cast<const T*>(a.p);
    const T* q0 = reinterpret_cast<const T*>(a.q);
    const bool points = a.q == nullptr;
    if (tid < 2 * kVerifyMaxNodes) s_children[tid] = 0u;
    __syncthreads();
    if (tid < a.N) {
        const int64_t i = (int64_t)b * a.N + tid;
        const int x = a.tokens[i];
        int up = a.parent ? a.parent[i] : tid - 1;
        if (up < 0 || up >= tid) up = -1;
        s_token[tid] = x;
        s_parent[tid] = up;
        if (up >= 0 && tid < n) atomicOr(&s_children[2 * up + (tid >> 5)], 1u << (tid & 31));
        s_u[tid] = GREEDY ? 0.f : a.u[i];
        const bool valid = up >= 0 && x >= 0 && x < a.V;
        const int64_t row = (int64_t)b * a.N + max(up, 0);
        s_p[tid] = valid && !GREEDY ? (float)p0[row * a.p_stride + x] : 0.f;
        s_q[tid] = valid && !GREEDY && !points ? (float)q0[row * a.q_stride + x] : 0.f;
        s_path[tid] = tid == 0 && n > 0 ? 0 : -1;
    }
    __syncthreads();
    // every block has started: its shared memory may be written
    if (blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

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
    int length = n > 0 ? 1 : 0;                              // of the path

    if constexpr (GREEDY) {
        // the lowest index of the largest score at `node`; `next` (or -1): the node whose row is wanted next, likely
        auto best_of = [&](int node, int next) -> int {
            const T *p, *q;
            bool vec;
            rows_of(node, p, q, vec);
            if (next >= 0) {                                 // one line of the next row per lane and step
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
                for (int e = 0; e < 4; ++e) {
                    const float score = fmaxf(f[e], -INFINITY);               // (a NaN counts as -inf)
                    if (i + e < hi && (score > best || arg == kNone)) { best = score; arg = i + e; }
                }
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
            for (int w = lane * per_lane; w < min(n_runs, (lane + 1) * per_lane); ++w)
                take_better(best, arg, s_best[pass & 1][w], s_arg[pass & 1][w]);
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1)
                take_better(best, arg, __shfl_xor_sync(0xffffffffu, best, off), __shfl_xor_sync(0xffffffffu, arg, off));
            ++pass;
            return arg;
        };
        auto first_child = [&](int node) -> int {
            const unsigned low = s_children[2 * node], high = s_children[2 * node + 1];
            return low ? __ffs(low) - 1 : high ? 31 + __ffs(high) : -1;
        };
        int best = -1;
        if (n > 0) best = best_of(0, first_child(0));
        int cur = 0;
        for (int i = 1; i < n; ++i) {                        // (every thread of every block takes the same decisions)
            if (s_parent[i] != cur || s_token[i] != best) continue;
            cur = i;
            if (tid == 0) s_path[length] = i;
            ++length;
            best = best_of(cur, first_child(cur));
        }
        if (rank == 0 && tid == 0) a.next_token[b] = best;
    } else {
        double* kept = s_left + warp * a.run;                  // what is left of the current node's row: this warp's run
        int held = -1;                                       // the node that it belongs to
        // one entry after k rejections, from p and q
        auto left_of = [&](float p, float q, int x, int k) -> double {
            double v = widen(p);
            if (points) {
                for (int r = 0; r < k; ++r)
                    if (s_out[r] == x) v = 0.;
            } else {
                for (int r = 0; r < k; ++r) v = reject(v, s_weight[r], widen(q));
            }
            return v;
        };
        double runs_before = 0.;                       // warp 0: the sum of the runs before this lane's
        // the sum of what is left at `node` after k rejections; leaves the warps' sums in s_sum[(pass - 1) & 1]
        auto sum_left = [&](int node, int k) -> double {
            const T *p, *q;
            bool vec;
            rows_of(node, p, q, vec);
            double acc[4] = {};
            const bool need_q = !points && k > 0;
            // a node's first pass follows its first rejection, and every one its own: `kept` lacks the last one only
            const bool fresh = !KEEP || held != node || k == 0;
            const double w = KEEP && need_q ? s_weight[k - 1] : 0.;
            for (int i0 = lo; i0 < hi; i0 += 512) {          // four stretches of 128 entries: all loads, then the arithmetic
                float fp[16], fq[16];
                if (fresh) {
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        float f[4];
                        load4(p, min(i0 + 128 * s + 4 * lane, hi), hi, vec, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) fp[4 * s + e] = f[e];
                    }
                }
                if (need_q) {
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        float f[4];
                        load4(q, min(i0 + 128 * s + 4 * lane, hi), hi, vec, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) fq[4 * s + e] = f[e];
                    }
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int i = i0 + 128 * s + 4 * lane;
                    if (i >= hi) break;
                    double x[4];
                    if (KEEP && !fresh) {
                        const double2 x0 = *reinterpret_cast<const double2*>(kept + (i - lo)), x1 = *reinterpret_cast<const double2*>(kept + (i - lo) + 2);
                        x[0] = x0.x; x[1] = x0.y; x[2] = x1.x; x[3] = x1.y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = reject(x[e], w, widen(fq[4 * s + e]));
                    } else if (KEEP && need_q) {             // the first rejection at a node: W is 1
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = fmax(widen(fp[4 * s + e]) - widen(fq[4 * s + e]), 0.);
                    } else if (KEEP && k == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = widen(fp[4 * s + e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = left_of(fp[4 * s + e], need_q ? fq[4 * s + e] : 0.f, i + e, k);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] += x[e];
                    if (KEEP) {
                        *reinterpret_cast<double2*>(kept + (i - lo)) = make_double2(x[0], x[1]);
                        *reinterpret_cast<double2*>(kept + (i - lo) + 2) = make_double2(x[2], x[3]);
                    }
                }
            }
            held = node;
            acc[0] += acc[1];
            acc[2] += acc[3];
            acc[0] += acc[2];
            const double mine = warp_sum(acc[0]);
            if (lane < (int)blocks)
                asm volatile("st.shared::cluster.f64 [%0], %1;"
                             ::"r"(map_to_rank(smem_u32(&s_sum[pass & 1][slot]), lane)), "d"(mine) : "memory");
            meet();
            double total = 0.;
            if (warp == 0) {                                 // (the same additions in warp 0 of every block)
                double own[4];                                 // per_lane is at most 4
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int at = lane * per_lane + w;
                    own[w] = w < per_lane && at < n_runs ? s_sum[pass & 1][at] : 0.;
                }
                double other = own[2];
                total = own[0];
                total += own[1];
                other += own[3];
                total += other;
                runs_before = warp_prefix(total, lane);
                total += runs_before;
                total = __shfl_sync(0xffffffffu, total, 31);
            }
            ++pass;
            return total;
        };
        // this warp's entries hold the lowest index whose cumulative sum exceeds the goal: which it is
        auto draw = [&](const Task& task) {
            const T *p, *q;
            bool vec;
            rows_of(task.node, p, q, vec);
            auto entries = [&](int i, double (&x)[4]) {        // four entries from i on
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = 0.;
                if (i >= hi) return;
                if constexpr (KEEP) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = kept[i - lo + e];
                } else {
                    float fp[4], fq[4] = {0.f, 0.f, 0.f, 0.f};
                    load4(p, i, hi, vec, fp);
                    if (!points && task.k > 0) load4(q, i, hi, vec, fq);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = left_of(fp[e], fq[e], i + e, task.k);
                }
            };
            double before = task.before, before_last = task.before;
            int at = lo, last = lo;                          // the stretch of 128 entries; the last one with anything in it
            bool hit = false;
            for (; at < hi; at += 128) {
                double x[4];
                entries(at + 4 * lane, x);
                for (int e = 1; e < 4; ++e) x[0] += x[e];
                const double sum = warp_sum(x[0]);
                if (sum > 0.) {
                    last = at;
                    before_last = before;
                    before += sum;
                    if (before > task.goal) { hit = true; break; }
                }
            }
            // (rounding may leave the goal unreached: the last entry with anything in it then)
            double x[4];
            const int i = last + 4 * lane;
            entries(i, x);
            double four = x[0];
            for (int e = 1; e < 4; ++e) four += x[e];
            double upto = before_last;
            upto += warp_prefix(four, lane);
            int first = kNone, some = -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                upto += x[e];
                if (x[e] > 0.) {
                    some = i + e;
                    if (hit && upto > task.goal) first = min(first, i + e);
                }
            }
            first = __reduce_min_sync(0xffffffffu, first);
            some = __reduce_max_sync(0xffffffffu, some);
            if (lane == 0) a.next_token[b] = first != kNone ? first : some;
        };

        // warp 0 walks the tree (of every block the same way, on the same sums)
        int cur = 0, k = 0;
        unsigned low = 0, high = 0;                          // the children of cur that are still to be tested
        double weight = 1.;                            // W of the next test
        bool summed = false;                                 // s_sum holds the sums for (cur, k), and weight their total
        const double zero = 0.;
        if (n > 0) { low = s_children[0]; high = s_children[1]; }
        auto next_task = [&](double sum) -> Task {             // `sum`: of the task before, if it was a sum
            if (n == 0) {
                if (rank == 0 && lane == 0) a.next_token[b] = -1;
                return Task{kDone, 0, 0, 0, zero, zero};
            }
            if (summed) weight = sum;
            while (low | high) {
                const int i = low ? __ffs(low) - 1 : 31 + __ffs(high);
                if (low) low &= low - 1; else high &= high - 1;
                const int x = s_token[i];
                if (x < 0 || x >= a.V) continue;
                const float q = points ? 1.f : s_q[i];
                const double left = left_of(s_p[i], q, x, k);
                if (left > weight * s_u[i] * q) {
                    cur = i;
                    if (lane == 0) s_path[length] = i;
                    ++length;
                    k = 0;
                    weight = 1.;
                    summed = false;
                    low = s_children[2 * i];
                    high = s_children[2 * i + 1];
                    continue;
                }
                if (lane == 0) { s_weight[k] = weight; s_out[k] = x; }
                __syncwarp();
                ++k;
                if (points) {
                    weight -= left;
                } else {
                    summed = true;
                    return Task{kSum, cur, k, 0, zero, zero};
                }
            }
            if (!summed) {                                   // the sum at the last node
                summed = true;
                return Task{kSum, cur, k, 0, zero, zero};
            }
            if (!(weight > 0.)) {
                if (k > 0) {                                 // nothing is left of v: the target's row itself
                    k = 0;
                    return Task{kSum, cur, 0, 0, zero, zero};
                }
                if (rank == 0 && lane == 0) a.next_token[b] = -1;
                return Task{kDone, 0, 0, 0, zero, zero};
            }
            // the warp whose run takes the cumulative sum beyond the goal
            const double* sums = s_sum[(pass - 1) & 1];
            const double goal = weight * s_u[0];
            const int w0 = lane * per_lane, w1 = min(n_runs, w0 + per_lane);
            double at_run = runs_before, before = zero;
            int hit_run = kNone, last_run = -1;
            for (int w = w0; w < w1 && hit_run == kNone; ++w) {
                if (sums[w] > 0.) {
                    last_run = w;
                    before = at_run;
                    at_run += sums[w];
                    if (at_run > goal) hit_run = w;
                }
            }
            int run = __reduce_min_sync(0xffffffffu, hit_run);
            if (run == kNone) run = __reduce_max_sync(0xffffffffu, last_run);    // (rounding: the last run with anything in it)
            const int from = run / per_lane;
            return Task{kDraw, cur, k, run, __shfl_sync(0xffffffffu, before, from), goal};
        };
        double sum = 0.;
        for (;;) {
            if (warp == 0) {
                const Task next = next_task(sum);
                if (lane == 0) s_task = next;
            }
            __syncthreads();
            const Task task = s_task;
            if (task.what == kSum) {
                sum = sum_left(task.node, task.k);           // (meets, so that the next task finds this one read)
            } else {
                if (task.what == kDraw && task.run == slot) draw(task);
                break;
            }
        }
    }
    __syncthreads();
    // (the last writes to another block's shared memory lie before the last meeting: a block may leave)
    if (rank == 0) {
        if (tid < a.N) a.path[(int64_t)b * a.N + tid] = s_path[tid];
        if (tid == 0) a.accepted[b] = length;
    }
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
    // Small vocabularies: four warps a request (beyond 2048 entries they would have longer runs than the 512 below).
    // Else sixteen, and as many blocks (up to eight) as keep a warp's run at 512 entries, whatever the batch: a pass is all
    // latency, and more blocks per request beat fewer at every batch (64 requests, 65536 entries: 38 us as 8 x 16 warps; as
    // 8 x 8 warps 38 too, and 34 instead of 28 for half the requests).
    const bool greedy = a.u == nullptr;
    auto fit = [&](int warps, int run) {
        int blocks = 1;
        while (blocks < kVerifyMaxCluster && (int64_t)blocks * warps * run < a.V) blocks *= 2;
        a.run = ((a.V + blocks * warps - 1) / (blocks * warps) + 127) / 128 * 128;
        return blocks;
    };
    if (a.V <= 2048) {
        const int blocks = fit(4, 512);
        return greedy ? launch_verify<T, 4, true, false>(a, batch, blocks, st) : launch_verify<T, 4, false, true>(a, batch, blocks, st);
    }
    const int blocks = fit(16, 512);
    if (greedy) return launch_verify<T, 16, true, false>(a, batch, blocks, st);
    if (16 * (int64_t)a.run * (int)sizeof(double) <= kVerifyKeepBytes) return launch_verify<T, 16, false, true>(a, batch, blocks, st);
    return launch_verify<T, 16, false, false>(a, batch, blocks, st);
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
