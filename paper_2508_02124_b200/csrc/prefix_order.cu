// The order of prefixes (include/dma.h, dma_prefix_order): of every prefix and query head the w keys of the largest delta, sorted.
//
// The weakest kept key of each (prefix, head) is found as decoding finds it (cache4_select.cu); what lies above it is collected and sorted in chunks of kChunk positions, and,
// where a prefix may have several chunks, each entry's place is the sum of its places in all of them.
#include <algorithm>

#include "cache4_decode.cuh"

namespace dma {
namespace {

constexpr int kChunk = 4096, kThreads = 512;

struct Order {
    const float* delta;
    const int32_t *table, *len;
    int32_t *slot, *order_len;
    float* weight;
    int64_t ld, order_ld;
    const unsigned long long* weakest;       // NULL: all are kept
    unsigned long long* run;                 // [nseq * Hq, cap]: the chunks' sorted entries, wherever there was room
    int32_t *run_at, *run_len, *room;        // [nseq * Hq, chunks], [nseq * Hq]
    int nseq, Hq, w, page_log, num_pages, max_blocks, chunks, cap;
    __device__ __forceinline__ int visible(int s) const { return min(max(len[s], 0), max_blocks << page_log); }
};

// Rows for the selection, the lists' lengths, cleared counters. A CTA per prefix.
__global__ void __launch_bounds__(256) order_rows_kernel(Order P, int32_t* seq, int32_t* pos, int32_t* status) {
    __shared__ int total;
    pdl_enter();
    const int s = blockIdx.x, n = P.visible(s), blocks = (n + (1 << P.page_log) - 1) >> P.page_log;
    if (s == 0 && threadIdx.x < kWsHeaderBytes / 4) status[threadIdx.x] = 0;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    int mine = 0;
    for (int b = threadIdx.x; b < blocks; b += 256)
        if ((unsigned)P.table[s * P.ld + b] < (unsigned)P.num_pages) mine += min(n - (b << P.page_log), 1 << P.page_log);
    atomicAdd(&total, mine);
    for (int h = threadIdx.x; h < P.Hq; h += 256) P.room[s * P.Hq + h] = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        seq[s] = s;
        pos[s] = n - 1;
        P.order_len[s] = min(P.w, total);
    }
}

__global__ void __launch_bounds__(kThreads) order_sort_kernel(Order P) {
    __shared__ unsigned long long e[kChunk];
    __shared__ int count, base;
    const int tid = threadIdx.x, lane = tid & 31, chunk = blockIdx.x % P.chunks, item = blockIdx.x / P.chunks, s = item / P.Hq, h = item % P.Hq;
    pdl_enter();
    const int n = P.visible(s), j0 = chunk * kChunk, j1 = min(n, j0 + kChunk);
    const int32_t* pages = P.table + s * P.ld;
    const unsigned long long least = P.weakest ? P.weakest[item] : 0ull;
    if (tid == 0) count = 0;
    __syncthreads();
    for (int b = j0; b < j1; b += kThreads) {
        const int j = b + tid;
        unsigned long long key = 0;
        if (j < j1) {
            const int page = pages[j >> P.page_log];
            if ((unsigned)page < (unsigned)P.num_pages)
                key = order_key(__float_as_uint(P.delta[(((size_t)page * P.Hq + h) << P.page_log) + (j & ((1 << P.page_log) - 1))]) & 0x7FFFFFFFu, j);
        }
        const bool kept = key != 0 && key >= least;
        const uint32_t m = __ballot_sync(0xffffffffu, kept);
        int at = 0;
        if (lane == 0 && m) at = atomicAdd(&count, __popc(m));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(m & ((1u << lane) - 1u));
        if (kept) e[at] = key;
    }
    __syncthreads();
    const int c = count;
    int size = 2;
    while (size < c) size *= 2;
    for (int i = c + tid; i < size; i += kThreads) e[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int x = k / 2; x > 0; x /= 2) {
            for (int i = tid; i < size / 2; i += kThreads) {
                const int a = 2 * i - (i & (x - 1));
                const unsigned long long u = e[a], v = e[a + x];
                if ((u < v) == ((a & k) == 0)) { e[a] = v; e[a + x] = u; }
            }
            __syncthreads();
        }
    if (P.chunks > 1) {
        if (tid == 0) {
            base = atomicAdd(&P.room[item], c);
            P.run_at[blockIdx.x] = base;
            P.run_len[blockIdx.x] = c;
        }
        __syncthreads();
        for (int i = tid; i < c && base + i < P.cap; i += kThreads) P.run[(size_t)item * P.cap + base + i] = e[i];
        return;
    }
    for (int i = tid; i < c && i < P.cap; i += kThreads) {
        const int j = (int)(0xFFFFFFFFu - (uint32_t)e[i]);
        P.slot[item * P.order_ld + i] = (pages[j >> P.page_log] << P.page_log) + (j & ((1 << P.page_log) - 1));
        P.weight[item * P.order_ld + i] = __uint_as_float((uint32_t)(e[i] >> 32));
    }
}

__global__ void __launch_bounds__(256) order_merge_kernel(Order P) {
    const int item = blockIdx.x / P.chunks, chunk = blockIdx.x % P.chunks, s = item / P.Hq;
    pdl_enter();
    const unsigned long long* run = P.run + (size_t)item * P.cap;
    const int32_t *at = P.run_at + item * P.chunks, *len = P.run_len + item * P.chunks, *pages = P.table + s * P.ld;
    const int from = at[chunk], count = min(len[chunk], P.cap - from);
    for (int i = threadIdx.x; i < count; i += 256) {
        const unsigned long long key = run[from + i];
        int place = i;
        for (int c = 0; c < P.chunks; ++c) {
            if (c == chunk) continue;
            const unsigned long long* other = run + at[c];
            int lo = 0, hi = min(len[c], P.cap - at[c]);
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (other[mid] > key) lo = mid + 1; else hi = mid;
            }
            place += lo;
        }
        if (place >= P.cap) continue;
        const int j = (int)(0xFFFFFFFFu - (uint32_t)key);
        P.slot[item * P.order_ld + place] = (pages[j >> P.page_log] << P.page_log) + (j & ((1 << P.page_log) - 1));
        P.weight[item * P.order_ld + place] = __uint_as_float((uint32_t)(key >> 32));
    }
}

struct Layout {
    size_t seq, pos, weakest, room, at, len, run, total;
    int chunks, cap;
    explicit Layout(const Cache& C) {
        const int64_t capacity = (int64_t)C.max_blocks << C.page_log, items = (int64_t)C.nseq * C.Hq;
        chunks = (int)((capacity + kChunk - 1) / kChunk);
        cap = (int)std::min<int64_t>(C.w, capacity);
        size_t x = kWsHeaderBytes;
        auto take = [&](size_t bytes) { const size_t at = x; x += (bytes + 255) / 256 * 256; return at; };
        seq = take((size_t)C.nseq * 4);
        pos = take((size_t)C.nseq * 4);
        weakest = take((size_t)items * 8);
        room = take((size_t)items * 4);
        at = take((size_t)items * chunks * 4);
        len = take((size_t)items * chunks * 4);
        run = take((size_t)items * cap * 8);
        total = x;
    }
};

}  // namespace

size_t prefix_order_ws_bytes(const Cache& C) { return Layout(C).total; }

int launch_prefix_order(const Cache& C0, const float* delta, const int32_t* table, const int32_t* len, int32_t* slot, float* weight, int64_t order_ld, int32_t* order_len,
                        void* ws, cudaStream_t st) {
    Cache C = C0;
    C.rows = C.nseq;
    const Layout L(C);
    char* p = (char*)ws;
    const bool select = L.cap < ((int64_t)C.max_blocks << C.page_log);
    Order P = {delta, table, len, slot, order_len, weight, C.table_ld, order_ld, select ? (unsigned long long*)(p + L.weakest) : nullptr, (unsigned long long*)(p + L.run),
               (int32_t*)(p + L.at), (int32_t*)(p + L.len), (int32_t*)(p + L.room), C.nseq, C.Hq, C.w, C.page_log, C.num_pages, C.max_blocks, L.chunks, L.cap};
    int rc = launch_overlapped(order_rows_kernel, dim3(C.nseq), dim3(256), 0, st, 1, P, (int32_t*)(p + L.seq), (int32_t*)(p + L.pos), (int32_t*)p);
    if (rc) return rc;
    if (select) {
        const Rows R = {table, (const int32_t*)(p + L.seq), (const int32_t*)(p + L.pos), delta, C.table_ld, C.nseq, C.page_log, C.num_pages, C.max_blocks, C.Hq};
        if ((rc = launch_cache4_select(C, R, (unsigned long long*)(p + L.weakest), Plan{}, st))) return rc;
    }
    const unsigned grid = (unsigned)((int64_t)C.nseq * C.Hq * L.chunks);
    if ((rc = launch_overlapped(order_sort_kernel, dim3(grid), dim3(kThreads), 0, st, 1, P))) return rc;
    return L.chunks > 1 ? launch_overlapped(order_merge_kernel, dim3(grid), dim3(256), 0, st, 1, P) : DMA_OK;
}

}  // namespace dma
