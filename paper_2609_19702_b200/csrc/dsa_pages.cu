// Pages and rows of a cache: moving kept rows together, copying, sharing, taking and giving back pages
// (dsa_compact_kv, dsa_copy_pages, dsa_fork_pages, dsa_reserve_pages, dsa_release_pages).
//
// Rows and pages are moved at copy bandwidth: what bounds them is 2 x the bytes moved.  Measured: 218 MB of kept rows
// moved up (16 requests, dropped tokens): 78 us, 5.6 TB/s read and written; three accepted rows of 64 requests: 6.9 us for
// 25 MB; 32 branches with their last pages and the pages given back before: 19.6 us for 31 MB, bound by three launches, the
// planning block and copies that have one token's rows in flight at a time (201 MB of whole pages: 36.5 us with 16 tokens
// a page, 78 with 128).  A page pool is one
// array of counts; a free page is one whose count is 0 and pages are taken lowest index first.  Giving pages
// back is then nothing but independent decrements, in any order and from any number of blocks, and two runs
// of the same calls leave the same tables, which a stack of free pages filled by atomics would not.
#include "dsa_host.cuh"

#include <algorithm>

namespace {

using namespace dsa;

constexpr int kCopyThreads = 128;
constexpr int kCopyBatch = 8;                      // rows a thread has in flight
constexpr int kListRows = 64;                      // rows whose places a block works out at a time
constexpr int kPoolThreads = 1024;

struct CacheArgs {
    AttnArgs a;
    int64_t stride_layer;
    int esize;                                     // bytes per element
    int row_vecs;                                  // 16-byte pieces of one token's heads
    int head_vecs;                                 // and of one head
};

// Piece `col` of a token's heads, as a byte offset behind the token's.
__device__ __forceinline__ int64_t piece_offset(const CacheArgs& c, int col) {
    const int head = col / c.head_vecs;
    return ((int64_t)head * c.a.stride_head) * c.esize + (int64_t)(col - head * c.head_vecs) * 16;
}

// Whether the cache has the token at position `pos` of request b.
__device__ __forceinline__ bool row_in_cache(const CacheArgs& c, int b, int64_t pos) {
    return pos >= 0 && pos < c.a.max_seq_len && token_has_page(c.a, b, (int)pos);
}

// How many kept rows of a request, from the first one on, the cache has and has a place for: what its length may
// count.  By a whole block; s_stored is shared.
__device__ __forceinline__ int rows_stored(const CacheArgs& c, int b, int64_t first, const int* list, int count, int* s_stored) {
    if (threadIdx.x == 0) *s_stored = count;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += blockDim.x)
        if (!row_in_cache(c, b, first + list[i]) || !row_in_cache(c, b, first + i)) { atomicMin(s_stored, i); break; }
    __syncthreads();
    return *s_stored;
}

// ---- rows of a request move up ----------------------------------------------------------------------
// One block: 128 of the 16-byte columns of one request's rows, in `planes` of the layers' K and V caches, and one
// stretch of kListRows rows of the list; the rows' places (page lookups) are worked out once and shared by the planes.
//
// Kept positions ascend, so what stays in place is a prefix of the list, and where the first row that moves comes from
// beyond all places that are written, no row is read from a place that another one is written to: the rows may move in
// any order, and blocks take a stretch each.  Else (a list that overlaps its own destination) one block takes all
// stretches in order: a thread takes its column through all rows, so what it overwrites it has read itself, and since
// keep[i] >= i a batch of loads never needs what the batch before it has yet to store.
__global__ void __launch_bounds__(kCopyThreads, 8) dsa_compact_kernel(const CacheArgs c, const int* base, const int* keep,
                                                                      const int* keep_count, int max_keep, int col_blocks,
                                                                      int planes, int plane_groups, int stretches, int layers,
                                                                      int* len_out) {
    __shared__ int64_t s_src[kListRows], s_dst[kListRows];
    __shared__ int s_n, s_first, s_stored;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31;
    int idx = blockIdx.x;
    const int col = (idx % col_blocks) * kCopyThreads + tid; idx /= col_blocks;
    const int group = idx % plane_groups; idx /= plane_groups;
    const int stretch = idx % stretches;
    const int b = idx / stretches;
    const int* list = keep + (int64_t)b * max_keep;
    const int count = max(0, min(keep_count[b], max_keep));
    const int64_t first = base ? base[b] : 0;
    if (len_out && idx == b * stretches && blockIdx.x % (col_blocks * plane_groups) == 0) {
        const int stored = rows_stored(c, b, first, list, count, &s_stored);
        if (tid == 0) len_out[b] = (int)first + stored;
    }
    if (stretch * kListRows >= count) return;
    // the prefix that stays (keep[i] - i never falls)
    if (tid == 0) s_first = count;
    __syncthreads();
    for (int i = tid; i < count; i += kCopyThreads)
        if (list[i] != i) { atomicMin(&s_first, i); break; }
    __syncthreads();
    const int stays = s_first;
    if (stays >= count) return;
    const bool any_order = list[stays] >= count;
    if (!any_order && stretch > 0) return;
    const bool mine = col < c.row_vecs;
    const int64_t column = mine ? piece_offset(c, col) : 0;
    const int p0 = group * planes, p1 = min(2 * layers, p0 + planes);
    const int from = any_order ? stretch * kListRows : 0, to = any_order ? min(count, from + kListRows) : count;
    for (int i0 = max(from, stays / kListRows * kListRows); i0 < to; i0 += kListRows) {
        __syncthreads();
        if (tid < 32) {                            // the rows of this stretch that move, in order
            int n = 0;
            for (int i = i0 + lane; i - lane < min(to, i0 + kListRows); i += 32) {
                bool moves = false;
                int64_t src = 0, dst = 0;
                if (i < to) {
                    const int64_t at = first + list[i], goal = first + i;
                    moves = at != goal && row_in_cache(c, b, at) && row_in_cache(c, b, goal);
                    if (moves) {
                        src = token_offset(c.a, b, 0, (int)at) * c.esize;
                        dst = token_offset(c.a, b, 0, (int)goal) * c.esize;
                    }
                }
                const unsigned ballot = __ballot_sync(0xffffffffu, moves);
                if (moves) {
                    const int at = n + __popc(ballot & ((1u << lane) - 1u));
                    s_src[at] = src;
                    s_dst[at] = dst;
                }
                n += __popc(ballot);
            }
            if (lane == 0) s_n = n;
        }
        __syncthreads();
        const int n = s_n;
        if (!mine || n == 0) continue;
        auto plane = [&](int p) -> unsigned char* {
            return reinterpret_cast<unsigned char*>(const_cast<void*>((p & 1) ? c.a.v : c.a.k)) +
                   (int64_t)(p >> 1) * c.stride_layer * c.esize + column;
        };
        // (plane, row) pairs, a plane's rows one behind the other
        const int total = n * (p1 - p0);
        int p_load = p0, i_load = 0, p_store = p0, i_store = 0;
        unsigned char *at_load = plane(p0), *at_store = plane(p0);
        for (int done = 0; done < total; done += kCopyBatch) {
            uint4 x[kCopyBatch];
            const int m = min(kCopyBatch, total - done);
#pragma unroll
            for (int k = 0; k < kCopyBatch; ++k)
                if (k < m) {
                    x[k] = *reinterpret_cast<const uint4*>(at_load + s_src[i_load]);
                    if (++i_load == n) { i_load = 0; if (++p_load < p1) at_load = plane(p_load); }
                }
#pragma unroll
            for (int k = 0; k < kCopyBatch; ++k)
                if (k < m) {
                    *reinterpret_cast<uint4*>(at_store + s_dst[i_store]) = x[k];
                    if (++i_store == n) { i_store = 0; if (++p_store < p1) at_store = plane(p_store); }
                }
        }
    }
}

__global__ void __launch_bounds__(kCopyThreads) dsa_compact_len_kernel(const CacheArgs c, const int* base, const int* keep,
                                                                       const int* keep_count, int max_keep, int* len_out) {
    __shared__ int s_stored;
    const int b = blockIdx.x, first = base ? base[b] : 0;
    const int stored = rows_stored(c, b, first, keep + (int64_t)b * max_keep, max(0, min(keep_count[b], max_keep)), &s_stored);
    if (threadIdx.x == 0) len_out[b] = first + stored;     // (every thread has read base and keep_count, which it may be)
}

// ---- whole or part-filled pages --------------------------------------------------------------------------
// What a fork has to do, as worked out by the planning kernel.
struct ForkItem {
    int from_page, to_page;                        // to_page < 0: no page is copied
    int tokens;                                    // of the page that are copied
    int ok;                                        // 0: refused or no page left
};

struct ForkArgs {
    const int* src;
    const int* dst;
    int* table;
    int* seq_len;
    int* prompt_len;
    int* ref_count;
    int* status;
    int n, batch, max_blocks, num_blocks, block_size, max_seq_len;
    ForkItem* items;
};

// Exclusive prefix sums over a block of kPoolThreads threads, and the total.
__device__ __forceinline__ int block_prefix(int mine, int* s_warp, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += o;
    }
    __syncthreads();                               // s_warp free again
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    const int of_warp = s_warp[lane];              // (32 warps)
    int warps = of_warp;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, warps, off);
        if (lane >= off) warps += o;
    }
    total = __shfl_sync(0xffffffffu, warps, 31);
    return __shfl_sync(0xffffffffu, warps - of_warp, warp) + upto - mine;
}

// The counts of eight neighbouring pages from p on (a multiple of eight); beyond the pool: not free.
__device__ __forceinline__ void eight_counts(const int* ref_count, int p, int num_blocks, int (&r)[8]) {
    if (num_blocks - p >= 8 && (reinterpret_cast<uintptr_t>(ref_count) & 15) == 0) {
        const int4 a = *reinterpret_cast<const int4*>(ref_count + p), b = *reinterpret_cast<const int4*>(ref_count + p + 4);
        r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w; r[4] = b.x; r[5] = b.y; r[6] = b.z; r[7] = b.w;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) r[k] = p + k < num_blocks ? ref_count[p + k] : 1;
    }
}

// Free pages in ascending order: take(rank, page) for the first `want` of them; returns how many there were
// (counted no further than `want`).  One block of kPoolThreads threads.
template <class F>
__device__ __forceinline__ int free_pages(const int* ref_count, int num_blocks, int want, int* s_warp, F&& take) {
    int found = 0;
    for (int64_t p0 = 0; p0 < num_blocks && found < want; p0 += 8 * kPoolThreads) {
        const int64_t p = p0 + 8 * (int64_t)threadIdx.x;
        int r[8], mine = 0;
        if (p < num_blocks) {
            eight_counts(ref_count, (int)p, num_blocks, r);
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += r[k] == 0;
        }
        int total;
        int rank = found + block_prefix(mine, s_warp, total);
        if (p < num_blocks)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (r[k] == 0) {
                    if (rank < want) take(rank, (int)p + k);
                    ++rank;
                }
        found += total;
    }
    return min(found, want);
}

// Which branches can be made and which fresh page each gets: one block.
__global__ void __launch_bounds__(kPoolThreads) dsa_fork_plan_kernel(const ForkArgs f) {
    __shared__ int s_warp[32];
    __shared__ int s_src[kPoolThreads], s_dst[kPoolThreads];
    __shared__ bool s_bad[kPoolThreads];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // fresh pages wanted, in order; an item's rank among them is kept in to_page until the pages are known
    int want = 0;
    for (int i0 = 0; i0 < f.n; i0 += kPoolThreads) {
        const int i = i0 + tid;
        ForkItem it = {0, -1, 0, 0};
        const int s = i < f.n ? f.src[i] : -1, d = i < f.n ? f.dst[i] : -1;
        bool ok = s >= 0 && s < f.batch && d >= 0 && d < f.batch;
        int len = 0;
        if (ok) len = max(0, min(f.seq_len[s], f.max_seq_len));
        for (int j0 = 0; j0 < f.n; j0 += kPoolThreads) {    // (against all branches, a thousand at a time)
            __syncthreads();
            if (j0 + tid < f.n) { s_src[tid] = f.src[j0 + tid]; s_dst[tid] = f.dst[j0 + tid]; }
            __syncthreads();
            if (ok)
                for (int j = 0; j < min(kPoolThreads, f.n - j0); ++j) ok = ok && s_src[j] != d && (j0 + j >= i || s_dst[j] != d);
        }
        // every page within the source's length has to be there: a warp per branch looks its row through
        __syncthreads();
        s_src[tid] = s;
        s_dst[tid] = ok ? len / f.block_size + (len % f.block_size != 0) : 0;
        __syncthreads();
        for (int j = warp; j < min(kPoolThreads, f.n - i0); j += 32) {
            const int* row = f.table + (int64_t)s_src[j] * f.max_blocks;
            bool bad = false;
#pragma unroll 4
            for (int e = lane; e < s_dst[j]; e += 32) {
                const int id = row[e];
                bad |= id < 0 || id >= f.num_blocks;
            }
            bad = __any_sync(0xffffffffu, bad);
            if (lane == 0) s_bad[j] = bad;
        }
        __syncthreads();
        ok = ok && !s_bad[tid];
        if (ok) {
            it.tokens = len % f.block_size;
            it.from_page = it.tokens ? f.table[(int64_t)s * f.max_blocks + len / f.block_size] : 0;
            it.ok = 1;
        }
        int total;
        const int rank = want + block_prefix(it.ok && it.tokens, s_warp, total);
        if (it.ok && it.tokens) it.to_page = rank;
        want += total;
        if (i < f.n) f.items[i] = it;
    }
    // the pages themselves, over the ranks: item lists are as long as the call, so every rank looks its item up
    __syncthreads();
    int* fresh = reinterpret_cast<int*>(f.status); // (status holds page ids until the items have taken them)
    const int got = free_pages(f.ref_count, f.num_blocks, want, s_warp, [&](int rank, int page) { fresh[rank] = page; });
    __syncthreads();
    for (int i0 = 0; i0 < f.n; i0 += kPoolThreads) {
        const int i = i0 + tid;
        if (i >= f.n) continue;
        ForkItem it = f.items[i];
        if (it.to_page >= 0) {
            if (it.to_page < got) it.to_page = fresh[it.to_page];
            else { it.to_page = -1; it.ok = -1; }
            f.items[i] = it;
        }
    }
    __syncthreads();
    for (int i = tid; i < f.n; i += kPoolThreads) {
        const ForkItem it = f.items[i];
        f.status[i] = it.ok > 0 ? 0 : (it.ok < 0 ? 1 : 2);
    }
}

// Blocks of the copy kernel: (pair, layer, K or V, 128 columns); the pair's first block also makes the row.
__global__ void __launch_bounds__(kCopyThreads) dsa_fork_copy_kernel(const CacheArgs c, const ForkArgs f, int col_blocks,
                                                                     int layers) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x;
    int idx = blockIdx.x;
    const int col = (idx % col_blocks) * kCopyThreads + tid;
    const bool first_col = idx % col_blocks == 0; idx /= col_blocks;
    const bool is_v = idx & 1; idx >>= 1;
    const int layer = idx % layers;
    const int i = idx / layers;
    const ForkItem it = f.items[i];
    if (it.ok <= 0) return;
    if (first_col && !is_v && layer == 0) {
        const int s = f.src[i], d = f.dst[i];
        const int len = max(0, min(f.seq_len[s], f.max_seq_len));
        const int full = len / f.block_size;
        for (int e = tid; e < f.max_blocks; e += kCopyThreads) {
            int id = -1;
            if (e < full) {
                id = f.table[(int64_t)s * f.max_blocks + e];
                if (id >= 0 && id < f.num_blocks) atomicAdd(&f.ref_count[id], 1);
            } else if (e == full && it.to_page >= 0) {
                id = it.to_page;
                f.ref_count[id] = 1;
            }
            f.table[(int64_t)d * f.max_blocks + e] = id;
        }
        if (tid == 0) {
            f.seq_len[d] = f.seq_len[s];
            f.prompt_len[d] = f.prompt_len[s];
        }
    }
    if (it.to_page < 0 || col >= c.row_vecs) return;
    const int from = max(0, min(it.from_page, c.a.num_blocks - 1));
    unsigned char* cache = reinterpret_cast<unsigned char*>(const_cast<void*>(is_v ? c.a.v : c.a.k)) +
                           (int64_t)layer * c.stride_layer * c.esize + piece_offset(c, col);
    const unsigned char* src = cache + (int64_t)from * c.a.stride_b * c.esize;
    unsigned char* dst = cache + (int64_t)it.to_page * c.a.stride_b * c.esize;
    const int64_t step = c.a.stride_tok * c.esize;
#pragma unroll 8
    for (int t = 0; t < it.tokens; ++t) *reinterpret_cast<uint4*>(dst + t * step) = *reinterpret_cast<const uint4*>(src + t * step);
}

__global__ void __launch_bounds__(kCopyThreads) dsa_copy_pages_kernel(const CacheArgs c, const int* src, const int* dst,
                                                                      int col_blocks, int layers) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int idx = blockIdx.x;
    const int col = (idx % col_blocks) * kCopyThreads + (int)threadIdx.x; idx /= col_blocks;
    const bool is_v = idx & 1; idx >>= 1;
    const int layer = idx % layers;
    const int i = idx / layers;
    const int from = src[i], to = dst[i];
    if (from < 0 || from >= c.a.num_blocks || to < 0 || to >= c.a.num_blocks || from == to || col >= c.row_vecs) return;
    unsigned char* cache = reinterpret_cast<unsigned char*>(const_cast<void*>(is_v ? c.a.v : c.a.k)) +
                           (int64_t)layer * c.stride_layer * c.esize + piece_offset(c, col);
    const unsigned char* s = cache + (int64_t)from * c.a.stride_b * c.esize;
    unsigned char* d = cache + (int64_t)to * c.a.stride_b * c.esize;
    const int64_t step = c.a.stride_tok * c.esize;
#pragma unroll 8
    for (int t = 0; t < c.a.block_size; ++t) *reinterpret_cast<uint4*>(d + t * step) = *reinterpret_cast<const uint4*>(s + t * step);
}

// ---- taking and giving back ------------------------------------------------------------------------------
// One block per row; an entry is taken out with an exchange, so that a page is given back once whatever runs.
__global__ void dsa_release_kernel(int* table, int max_blocks, const int* keep_tokens, int* ref_count, int num_blocks,
                                   int block_size) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x;
    const int keep = keep_tokens ? keep_tokens[b] : 0;
    if (keep < 0) return;
    const int first = (int)min(((int64_t)keep + block_size - 1) / block_size, (int64_t)max_blocks);
    for (int e = first + (int)threadIdx.x; e < max_blocks; e += blockDim.x) {
        int* entry = table + (int64_t)b * max_blocks + e;
        if (*entry < 0) continue;
        const int id = atomicExch(entry, -1);
        if (id >= 0 && id < num_blocks && atomicSub(&ref_count[id], 1) <= 0) atomicAdd(&ref_count[id], 1);
    }
}

// A granted page is marked with its row's entry in its count until the tables are written.  The marks are the lowest
// numbers there are: a count that is negative already is none of them, and its page is not free either.
constexpr int kMark = -0x7fffffff - 1;             // + entry, below max_blocks

// Pages for rows that lack some: one block.  Dynamic shared memory: per row its first lacking entry and the
// running sum of what rows lack (3 ints per row).
__global__ void __launch_bounds__(kPoolThreads) dsa_reserve_kernel(int* table, int batch, int max_blocks, const int* seq_len,
                                                                   int extra, int* ref_count, int num_blocks, int block_size,
                                                                   int* status) {
    extern __shared__ int s_rows[];
    int* s_lacks = s_rows;                         // [batch] entries that the row lacks; later the sum before the row
    int* s_first = s_rows + batch;                 // [batch] the first of them
    int* s_need = s_rows + 2 * batch;              // [batch] entries that the row needs; -1: it gets nothing
    __shared__ int s_warp[32];
    __shared__ int s_granted, s_total;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // what every row lacks: eight lanes a row
    const int sub = lane & 7;
    for (int b0 = 0; b0 < batch; b0 += kPoolThreads / 8) {
        const int b = b0 + (tid >> 3);
        int lacks = 0, first = 0x7fffffff, need = 0;
        if (b < batch) {
            const int len = seq_len[b];
            const int64_t want = len < 0 ? 0 : ((int64_t)len + extra + block_size - 1) / block_size;
            need = (int)min(want, (int64_t)0x7fffffff);
            for (int e = sub; e < min(need, max_blocks); e += 8)
                if (table[(int64_t)b * max_blocks + e] < 0) { ++lacks; first = min(first, e); }
        }
#pragma unroll
        for (int off = 4; off >= 1; off >>= 1) {
            lacks += __shfl_xor_sync(0xffffffffu, lacks, off);
            first = min(first, __shfl_xor_sync(0xffffffffu, first, off));
        }
        if (b < batch && sub == 0) {
            const bool long_row = need > max_blocks;
            status[b] = long_row ? lacks + (need - max_blocks) : lacks;
            s_lacks[b] = long_row ? 0 : lacks;
            s_first[b] = first;
            s_need[b] = long_row ? -1 : need;
        }
    }
    __syncthreads();
    // running sums: s_lacks[b] becomes the pages wanted by the rows before b
    if (warp == 0) {
        int sum = 0;
        for (int b0 = 0; b0 < batch; b0 += 32) {
            const int mine = b0 + lane < batch ? s_lacks[b0 + lane] : 0;
            int upto = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto = upto > 0x7fffffff - o ? 0x7fffffff : upto + o;
            }
            if (b0 + lane < batch) s_lacks[b0 + lane] = sum + (upto - mine);
            sum += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) { s_total = sum; s_granted = 0; }
    }
    __syncthreads();
    const int total = s_total;
    // how many free pages there are (no further than what is wanted), then how many rows that serves
    const int found = free_pages(ref_count, num_blocks, total, s_warp, [](int, int) {});
    for (int b = tid; b < batch; b += kPoolThreads) {
        const int upto = b + 1 < batch ? s_lacks[b + 1] : total;
        if (upto <= found) {
            atomicMax(&s_granted, upto);
            if (s_need[b] >= 0) status[b] = 0;
        } else if (upto == s_lacks[b] && s_need[b] >= 0) {
            status[b] = 0;                         // lacks nothing
        }
    }
    __syncthreads();
    const int granted = s_granted;
    auto row_of = [&](int rank) {                  // the last row with s_lacks[row] <= rank
        int lo = 0, hi = batch - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_lacks[mid] <= rank) lo = mid; else hi = mid - 1;
        }
        return lo;
    };
    free_pages(ref_count, num_blocks, granted, s_warp, [&](int rank, int page) {
        const int lo = row_of(rank);
        int k = rank - s_lacks[lo];
        const int next = lo + 1 < batch ? s_lacks[lo + 1] : total;
        int* row = table + (int64_t)lo * max_blocks;
        int e = s_first[lo];
        if (s_need[lo] - e == next - s_lacks[lo]) {
            e += k;                                // no hole: the row's pages end before its first lacking entry
        } else {
            // a row with holes: its k-th lacking entry, counted before any of them is filled (see below)
            for (; e < max_blocks - 1; ++e)
                if (row[e] < 0 && k-- == 0) break;
        }
        ref_count[page] = kMark + e;               // (the tables are written when all ranks have counted)
    });
    __syncthreads();
    // the marked pages are the first `granted` free ones, in order: rank and row again
    int at = 0;
    for (int64_t p0 = 0; p0 < num_blocks && at < granted; p0 += 8 * kPoolThreads) {
        const int64_t p = p0 + 8 * (int64_t)tid;
        int r[8], mine = 0;
        if (p < num_blocks) {
            eight_counts(ref_count, (int)p, num_blocks, r);
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += r[k] < kMark + max_blocks;
        }
        int n;
        int rank = at + block_prefix(mine, s_warp, n);
        if (p < num_blocks)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (r[k] < kMark + max_blocks) {
                    if (rank < granted) table[(int64_t)row_of(rank) * max_blocks + (r[k] - kMark)] = (int)p + k;
                    ref_count[p + k] = 1;
                    ++rank;
                }
        at += n;
    }
}

// ---- host ------------------------------------------------------------------------------------------------
int32_t cache_args(const dsa_problem* p, int32_t num_layers, int64_t stride_layer, CacheArgs* c) {
    const int32_t rc = host_check_problem(p);
    if (rc != DSA_OK) return rc;
    if (num_layers < 1) return DSA_ERR_INVALID_ARG;
    if (p->ring_size > 0) return DSA_ERR_UNSUPPORTED;
    if (num_layers > (1 << 16) || p->num_kv_heads > (1 << 16)) return DSA_ERR_UNSUPPORTED;
    const int esize = p->dtype == DSA_BF16 ? 2 : 4;
    if (num_layers > 1 && (stride_layer < 1 || stride_layer * esize % 16)) return DSA_ERR_INVALID_ARG;
    *c = CacheArgs{};
    host_cache_args(p, &c->a);
    c->stride_layer = num_layers > 1 ? stride_layer : 0;
    c->esize = esize;
    c->head_vecs = p->head_dim * esize / 16;
    c->row_vecs = p->num_kv_heads * c->head_vecs;
    return DSA_OK;
}

template <class Kern, class... Args>
int32_t launch(Kern kern, int64_t blocks, int threads, size_t smem, cudaStream_t st, bool behind_own, const Args&... args) {
    if (blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind_own ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, args...);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

int32_t check_pool(const dsa_page_pool* pool, const void* table, int32_t batch, int32_t max_blocks) {
    if (!pool || pool->num_blocks < 1 || pool->block_size < 1 || batch < 0 || max_blocks < 1) return DSA_ERR_INVALID_ARG;
    if (!pool->ref_count || (batch > 0 && !table)) return DSA_ERR_INVALID_ARG;
    if ((int64_t)batch * max_blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;
    return DSA_OK;
}

}  // namespace

extern "C" {

int32_t dsa_compact_kv(const dsa_problem* problem, int32_t num_layers, int64_t stride_layer, const int32_t* base,
                       const int32_t* keep, const int32_t* keep_count, int32_t max_keep, int32_t* len_out, void* stream) {
    CacheArgs c;
    int32_t rc = cache_args(problem, num_layers, stride_layer, &c);
    if (rc != DSA_OK) return rc;
    if (max_keep < 0) return DSA_ERR_INVALID_ARG;
    if (max_keep > (1 << 30) || (int64_t)problem->batch * max_keep > (1LL << 32)) return DSA_ERR_UNSUPPORTED;
    if (problem->batch == 0) return DSA_OK;
    if (!keep_count || (max_keep > 0 && !keep)) return DSA_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool own_launch = len_out && (max_keep == 0 || base == len_out || keep_count == len_out);
    if (max_keep > 0) {
        const int col_blocks = (c.row_vecs + kCopyThreads - 1) / kCopyThreads;
        const int stretches = (max_keep + kListRows - 1) / kListRows;
        // planes per block: enough of them for some eight loads in flight, as long as there are blocks for every SM
        int planes = std::max(1, std::min(2 * (int)num_layers, 8 / std::min(max_keep, 8)));
        while (planes > 1 && (int64_t)problem->batch * col_blocks * stretches * ((2 * num_layers + planes - 1) / planes) < 4 * host_sm_count())
            planes /= 2;
        const int groups = (2 * (int)num_layers + planes - 1) / planes;
        rc = launch(dsa_compact_kernel, (int64_t)problem->batch * stretches * groups * col_blocks, kCopyThreads, 0, st, true, c, base,
                    keep, keep_count, (int)max_keep, col_blocks, planes, groups, stretches, (int)num_layers,
                    own_launch ? (int32_t*)nullptr : len_out);
        if (rc != DSA_OK) return rc;
    }
    // (a launch of its own where len_out is base or keep_count, which every block of the other one reads)
    if (own_launch)
        rc = launch(dsa_compact_len_kernel, problem->batch, kCopyThreads, 0, st, false, c, base, keep, keep_count, (int)max_keep,
                    len_out);
    return rc;
}

int32_t dsa_reserve_pages(const dsa_page_pool* pool, int32_t* block_table, int32_t batch, int32_t max_blocks,
                          const int32_t* seq_len, int32_t extra_tokens, int32_t* status, void* stream) {
    const int32_t rc = check_pool(pool, block_table, batch, max_blocks);
    if (rc != DSA_OK) return rc;
    if (extra_tokens < 0) return DSA_ERR_INVALID_ARG;
    if (batch == 0) return DSA_OK;
    if (!seq_len || !status) return DSA_ERR_INVALID_ARG;
    const size_t smem = (size_t)batch * 3 * sizeof(int);
    if (smem > 47 * 1024) return DSA_ERR_UNSUPPORTED;        // (some 4000 rows)
    return launch(dsa_reserve_kernel, 1, kPoolThreads, smem, reinterpret_cast<cudaStream_t>(stream), true, block_table, (int)batch,
                  (int)max_blocks, seq_len, (int)extra_tokens, pool->ref_count, (int)pool->num_blocks, (int)pool->block_size,
                  status);
}

int32_t dsa_release_pages(const dsa_page_pool* pool, int32_t* block_table, int32_t batch, int32_t max_blocks,
                          const int32_t* keep_tokens, void* stream) {
    const int32_t rc = check_pool(pool, block_table, batch, max_blocks);
    if (rc != DSA_OK) return rc;
    if (batch == 0) return DSA_OK;
    return launch(dsa_release_kernel, batch, 128, 0, reinterpret_cast<cudaStream_t>(stream), true, block_table, (int)max_blocks,
                  keep_tokens, pool->ref_count, (int)pool->num_blocks, (int)pool->block_size);
}

int32_t dsa_fork_pages(const dsa_page_pool* pool, const dsa_problem* problem, int32_t num_layers, int64_t stride_layer,
                       const int32_t* src, const int32_t* dst, int32_t n, int32_t* status, void* workspace,
                       size_t workspace_bytes, void* stream) {
    CacheArgs c;
    int32_t rc = cache_args(problem, num_layers, stride_layer, &c);
    if (rc != DSA_OK) return rc;
    if ((!problem->block_table && problem->batch > 0) || n < 0) return DSA_ERR_INVALID_ARG;
    rc = check_pool(pool, problem->block_table, problem->batch, problem->max_blocks);
    if (rc != DSA_OK) return rc;
    if (pool->num_blocks != problem->num_blocks || pool->block_size != problem->block_size) return DSA_ERR_INVALID_ARG;
    if (problem->batch == 0 || n == 0) return DSA_OK;
    if (!src || !dst || !status) return DSA_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return DSA_ERR_INVALID_ARG;
    if (workspace_bytes < (size_t)n * sizeof(ForkItem)) return DSA_ERR_WORKSPACE_TOO_SMALL;
    ForkArgs f = {};
    f.src = src;
    f.dst = dst;
    f.table = const_cast<int32_t*>(problem->block_table);
    f.seq_len = const_cast<int32_t*>(problem->seq_len);
    f.prompt_len = const_cast<int32_t*>(problem->prompt_len);
    f.ref_count = pool->ref_count;
    f.status = status;
    f.n = n;
    f.batch = problem->batch;
    f.max_blocks = problem->max_blocks;
    f.num_blocks = problem->num_blocks;
    f.block_size = problem->block_size;
    f.max_seq_len = problem->max_seq_len;
    f.items = reinterpret_cast<ForkItem*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int col_blocks = (c.row_vecs + kCopyThreads - 1) / kCopyThreads;
    const int64_t blocks = (int64_t)n * num_layers * 2 * col_blocks;
    if (blocks > 0x7fffffffLL) return DSA_ERR_UNSUPPORTED;   // (before the plan is made: a refused call changes nothing)
    rc = launch(dsa_fork_plan_kernel, 1, kPoolThreads, 0, st, true, f);
    if (rc != DSA_OK) return rc;
    return launch(dsa_fork_copy_kernel, blocks, kCopyThreads, 0, st, true, c, f, col_blocks, (int)num_layers);
}

int32_t dsa_copy_pages(const dsa_problem* problem, int32_t num_layers, int64_t stride_layer, const int32_t* src,
                       const int32_t* dst, int32_t n, void* stream) {
    CacheArgs c;
    const int32_t rc = cache_args(problem, num_layers, stride_layer, &c);
    if (rc != DSA_OK) return rc;
    if ((!problem->block_table && problem->batch > 0) || n < 0) return DSA_ERR_INVALID_ARG;
    if (problem->batch == 0 || n == 0) return DSA_OK;
    if (!src || !dst) return DSA_ERR_INVALID_ARG;
    const int col_blocks = (c.row_vecs + kCopyThreads - 1) / kCopyThreads;
    return launch(dsa_copy_pages_kernel, (int64_t)n * num_layers * 2 * col_blocks, kCopyThreads, 0,
                  reinterpret_cast<cudaStream_t>(stream), true, c, src, dst, col_blocks, (int)num_layers);
}

}  // extern "C"
