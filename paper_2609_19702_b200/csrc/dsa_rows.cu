// Tokens of a ragged batch and their rows in a latent cache (dsa_map_tokens, dsa_store_rows, dsa_gather_rows).
#include "dsa_host.cuh"

#include <algorithm>

#include "dsa_latent_host.cuh"

namespace {

using namespace dsa;

// ---- which request, position and slot every token has ---------------------------------------------------
// Every block adds up the counts of all requests itself (a few reads per thread; no second launch, no wait on another
// block), keeps the starts in shared memory, and looks the requests of its own stretch of tokens up there by bisection.
// What bounds it is the chain of dependent reads -- counts, base, table -- for small batches and 16 written bytes a token
// for large ones.  Measured: 8 requests, one token each: 2.4 us in a row of replayed calls; 256 requests of up to 512: 3.1 (with 1024
// tokens a block 5.3).
constexpr int kMapThreads = 256;
constexpr int kMapTokens = 256;                    // of a block
constexpr int kMapBatch = 8192;                    // requests, at most: their starts lie in shared memory

struct MapArgs {
    const int* count;
    const int* base;
    const int* table;
    int batch, max_tokens, max_blocks, block_size, num_blocks, max_seq_len;
    int* start;
    int64_t* slot;
    int* position;
    int* request;
};

__global__ void __launch_bounds__(kMapThreads) dsa_map_kernel(const MapArgs m) {
    extern __shared__ int s_start[];               // [batch + 1]
    __shared__ int64_t s_warp[kMapThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // starts: a thread adds up a stretch of requests, the block the stretches
    const int per = (m.batch + kMapThreads - 1) / kMapThreads;
    const int b0 = min(m.batch, tid * per), b1 = min(m.batch, b0 + per);
    int64_t sum = 0;
    for (int b = b0; b < b1; ++b) sum += max(m.count[b], 0);
    int64_t before = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, before, off);
        if (lane >= off) before += x;
    }
    if (lane == 31) s_warp[warp] = before;
    before -= sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    for (int b = b0; b < b1; ++b) {
        s_start[b] = (int)min(before, (int64_t)m.max_tokens);
        before += max(m.count[b], 0);
    }
    if (tid == kMapThreads - 1) s_start[m.batch] = (int)min(before, (int64_t)m.max_tokens);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int b = tid; b <= m.batch; b += kMapThreads) m.start[b] = s_start[b];
    const int total = s_start[m.batch];
    const int t0 = blockIdx.x * kMapTokens, t1 = min(m.max_tokens, t0 + kMapTokens);
    for (int t = t0 + tid; t < t1; t += kMapThreads) {
        int b = -1, position = -1;
        int64_t slot = -1;
        if (t < total) {
            int hi = m.batch;                      // the last request that starts at or before t: start[b] <= t < start[b + 1]
            b = 0;
            while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (s_start[mid] <= t) b = mid; else hi = mid;
            }
            const int64_t at = (int64_t)(m.base ? m.base[b] : 0) + (t - s_start[b]);
            position = (int)min(at, (int64_t)0x7fffffff);
            if (at >= 0 && at < m.max_seq_len) {
                if (!m.table) {
                    slot = (int64_t)b * m.max_seq_len + at;
                } else {
                    const int e = (int)at / m.block_size;
                    const int page = e < m.max_blocks ? m.table[(int64_t)b * m.max_blocks + e] : -1;
                    if (page >= 0 && page < m.num_blocks) slot = (int64_t)page * m.block_size + ((int)at - e * m.block_size);
                }
            }
        }
        m.slot[t] = slot;
        if (m.position) m.position[t] = position;
        if (m.request) m.request[t] = b;
    }
}

// ---- rows to and from their slots ----------------------------------------------------------------------
// Bound by 2 x the bytes of the rows.  A block takes 8 rows (their places looked up once, by 8 threads) and copies them as one run
// of 16-byte pieces, five pieces in flight per thread (8 rows of 1152 bytes are 4.5 a thread: one turn).  Measured: 64 requests of up
// to 512 rows, 38 MB moved: 9.6 us, 3.9 TB/s; with 16 rows and 256 threads 10.6, with 32 rows 11.8, with 4 rows and 64 threads 10.4.
// The places, then the rows, then the writes follow one another; these calls have 4096 blocks, half of them with rows, where the device
// holds 1332 at a time (52 registers a thread), so that there are one and a half rounds of that.  Beyond L2: 592 MB moved, 137 us,
// 4.3 TB/s.
constexpr int kRowThreads = 128;
constexpr int kRowsPerBlock = 8;
constexpr int kRowFlight = 5;

struct RowArgs {
    unsigned char* cache;
    unsigned char* rows;
    const int64_t* slot;
    int64_t stride_batch, stride_token, row_stride; // bytes
    int64_t slots;                                  // of the cache
    int per_page, count, vecs;                      // tokens of a page or request; rows; 16-byte pieces of one
};

template <bool STORE>
__global__ void __launch_bounds__(kRowThreads) dsa_rows_kernel(const RowArgs c) {
    __shared__ int64_t s_at[kRowsPerBlock];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * kRowsPerBlock;
    const int n = (int)min((int64_t)kRowsPerBlock, c.count - t0);
    if (tid < n) {
        const int64_t s = c.slot[t0 + tid];
        const int64_t page = s / c.per_page;
        s_at[tid] = s < 0 || s >= c.slots ? -1 : page * c.stride_batch + (s - page * c.per_page) * c.stride_token;
    }
    __syncthreads();
    const int pieces = n * c.vecs;
    for (int i0 = tid; i0 < pieces; i0 += kRowThreads * kRowFlight) {
        uint4 x[kRowFlight];
        unsigned char* to[kRowFlight];
#pragma unroll
        for (int k = 0; k < kRowFlight; ++k) {
            const int i = i0 + k * kRowThreads, r = min(i, pieces - 1) / c.vecs;
            const int64_t at = s_at[r], col = (int64_t)(min(i, pieces - 1) - r * c.vecs) * 16;
            unsigned char* in_cache = c.cache + at + col;
            unsigned char* in_batch = c.rows + (t0 + r) * c.row_stride + col;
            to[k] = i >= pieces || at < 0 ? nullptr : STORE ? in_cache : in_batch;
            if (to[k]) x[k] = *reinterpret_cast<const uint4*>(STORE ? in_batch : in_cache);
        }
#pragma unroll
        for (int k = 0; k < kRowFlight; ++k)
            if (to[k]) *reinterpret_cast<uint4*>(to[k]) = x[k];
    }
}

int32_t copy_rows(const dsa_latent* l, const int64_t* slot, int32_t count, void* rows, int64_t row_stride, void* stream, bool store) {
    const int32_t rc = check_latent(l, false);
    if (rc != DSA_OK) return rc;
    if (count < 0) return DSA_ERR_INVALID_ARG;
    if (count == 0 || l->batch == 0) return DSA_OK;
    const int width = l->latent_dim + l->rope_dim, esize = l->dtype == DSA_BF16 ? 2 : 4;
    if (!slot || !rows || !aligned16(rows) || (reinterpret_cast<uintptr_t>(slot) & 7u)) return DSA_ERR_INVALID_ARG;
    if (row_stride < width || row_stride * esize % 16) return DSA_ERR_INVALID_ARG;
    RowArgs c = {};
    c.cache = reinterpret_cast<unsigned char*>(l->cache);
    c.rows = reinterpret_cast<unsigned char*>(rows);
    c.slot = slot;
    c.stride_batch = l->stride_batch * esize;
    c.stride_token = l->stride_token * esize;
    c.row_stride = row_stride * esize;
    c.per_page = l->block_table ? l->block_size : std::max(l->max_seq_len, 1);
    c.slots = l->block_table ? (int64_t)l->num_blocks * l->block_size : (int64_t)l->batch * l->max_seq_len;
    c.count = count;
    c.vecs = width * esize / 16;
    const int64_t blocks = ((int64_t)count + kRowsPerBlock - 1) / kRowsPerBlock;
    const cudaError_t e = store ? launch_dependent(dsa_rows_kernel<true>, blocks, kRowThreads, 0, reinterpret_cast<cudaStream_t>(stream), c)
                                : launch_dependent(dsa_rows_kernel<false>, blocks, kRowThreads, 0, reinterpret_cast<cudaStream_t>(stream), c);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

}  // namespace

extern "C" {

int32_t dsa_map_tokens(const dsa_token_map* map, int32_t* start, int64_t* slot, int32_t* position, int32_t* request, void* stream) {
    if (!map || map->batch < 0 || map->max_tokens < 0 || map->max_seq_len < 0) return DSA_ERR_INVALID_ARG;
    if (map->batch > kMapBatch || map->max_tokens > 0x7fffffff - kMapTokens) return DSA_ERR_UNSUPPORTED;
    if (map->block_table && (map->block_size < 1 || map->max_blocks < 1 || map->num_blocks < 1)) return DSA_ERR_INVALID_ARG;
    if (!start || (map->batch > 0 && !map->count) || (map->max_tokens > 0 && !slot) || (reinterpret_cast<uintptr_t>(slot) & 7u)) return DSA_ERR_INVALID_ARG;
    MapArgs m = {};
    m.count = map->count;
    m.base = map->base;
    m.table = map->block_table;
    m.batch = map->batch;
    m.max_tokens = map->max_tokens;
    m.max_blocks = map->max_blocks;
    m.block_size = map->block_table ? map->block_size : 1;
    m.num_blocks = map->num_blocks;
    m.max_seq_len = map->max_seq_len;
    m.start = start;
    m.slot = slot;
    m.position = position;
    m.request = request;
    const int64_t blocks = std::max<int64_t>(1, ((int64_t)map->max_tokens + kMapTokens - 1) / kMapTokens);
    const cudaError_t e = launch_dependent(dsa_map_kernel, blocks, kMapThreads, (size_t)(map->batch + 1) * sizeof(int),
                                           reinterpret_cast<cudaStream_t>(stream), m);
    return e == cudaSuccess ? DSA_OK : host_cuda_fail(e);
}

int32_t dsa_store_rows(const dsa_latent* latent, const int64_t* slot, int32_t count, const void* rows, int64_t row_stride, void* stream) {
    return copy_rows(latent, slot, count, const_cast<void*>(rows), row_stride, stream, true);
}

int32_t dsa_gather_rows(const dsa_latent* latent, const int64_t* slot, int32_t count, void* rows, int64_t row_stride, void* stream) {
    return copy_rows(latent, slot, count, rows, row_stride, stream, false);
}

}  // extern "C"
