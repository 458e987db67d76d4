// The order of prefixes (include/dma.h, dma_prefix_order): of every prefix and query head the w keys of the largest delta, sorted.
//
// The weakest kept key of each (prefix, head) is found as decoding finds it (cache4_select.cu); what is not below it is collected and sorted, by a CTA per (prefix, head) or in chunks.
#include <algorithm>
#include <type_traits>

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

// f(pattern, position, slot) for the keys of [j0, j1) (multiples of 8), eight of a thread side by side in one page (pages have 16 keys and more); keys in pages outside the pool are left out.
template <int NT, typename F>
__device__ __forceinline__ void sweep(const Order& P, int s, int h, int j0, int j1, F f) {
    const int32_t* pages = P.table + s * P.ld;
    const int mask = (1 << P.page_log) - 1;
    for (int b = j0; b < j1; b += NT * 8) {
        const int j = b + threadIdx.x * 8, page = j < j1 ? pages[j >> P.page_log] : -1;
        uint4 u[2];
        const bool there = (unsigned)page < (unsigned)P.num_pages;
        if (there) {
            const uint4* from = reinterpret_cast<const uint4*>(P.delta + (((size_t)page * P.Hq + h) << P.page_log) + (j & mask));
            u[0] = from[0];
            u[1] = from[1];
        }
        unsigned long long key[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4& x = u[i / 4];
            key[i] = there && j + i < j1 ? order_key((i % 4 == 0 ? x.x : i % 4 == 1 ? x.y : i % 4 == 2 ? x.z : x.w) & 0x7FFFFFFFu, j + i) : 0ull;
        }
        f(key);
    }
}

// The kept ones among a thread's keys to shared memory, in no order; `count` is moved on.
template <int NT>
__device__ __forceinline__ void collect(const unsigned long long (&key)[8], unsigned long long least, unsigned long long* to, int room, int* count) {
    const int lane = threadIdx.x & 31;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += key[i] != 0 && key[i] >= least;
    int at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += y;
    }
    int base = 0;
    if (lane == 31 && at) base = atomicAdd(count, at);
    at += __shfl_sync(0xffffffffu, base, 31) - mine;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (key[i] != 0 && key[i] >= least) {
            if (at < room) to[at] = key[i];
            ++at;
        }
}

__device__ __forceinline__ void put(const Order& P, int item, int s, int place, unsigned long long key) {
    const int j = (int)(0xFFFFFFFFu - (uint32_t)key);
    P.slot[item * P.order_ld + place] = (P.table[s * P.ld + (j >> P.page_log)] << P.page_log) + (j & ((1 << P.page_log) - 1));
    P.weight[item * P.order_ld + place] = __uint_as_float((uint32_t)(key >> 32));
}

// Lists of up to E * 1024 entries by a CTA per (prefix, head): what is kept is collected in shared memory and sorted by a bitonic network, E entries side by side per thread. Exchanges over fewer
// than 32 E places stay in registers and shuffles; the others, 15 of 66 for 2048, go through shared memory.
template <int E>
__global__ void __launch_bounds__(1024) order_held_kernel(Order P) {
    constexpr int NT = 1024, N = E * NT;
    extern __shared__ unsigned long long e[];                     // [2][N]
    __shared__ int count;
    const int tid = threadIdx.x, item = blockIdx.x, s = item / P.Hq, h = item % P.Hq;
    pdl_enter();
    const int n = P.visible(s);
    const unsigned long long least = P.weakest ? P.weakest[item] : 0ull;
    if (tid == 0) count = 0;
    for (int i = tid; i < N; i += NT) e[i] = 0;
    __syncthreads();
    sweep<NT>(P, s, h, 0, n, [&](const unsigned long long (&key)[8]) { collect<NT>(key, least, e, N, &count); });
    __syncthreads();
    unsigned long long v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = e[tid * E + i];
    int buf = 1;
#pragma unroll 1
    for (int k = 2; k <= N; k *= 2) {
#pragma unroll 1
        for (int x = k / 2; x >= 32 * E; x /= 2) {                // other warps'
            unsigned long long* to = e + buf * N;
#pragma unroll
            for (int i = 0; i < E; ++i) to[i * NT + tid] = v[i];
            __syncthreads();
            const bool high = ((tid * E & x) == 0) == ((tid * E & k) == 0);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const unsigned long long o = to[i * NT + (tid ^ x / E)];
                v[i] = (o > v[i]) == high ? o : v[i];
            }
            buf ^= 1;
        }
#pragma unroll 1
        for (int x = min(k / 2, 16 * E); x >= E; x /= 2) {        // other lanes'
            const bool high = ((tid * E & x) == 0) == ((tid * E & k) == 0);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const unsigned long long o = __shfl_xor_sync(0xffffffffu, v[i], x / E);
                v[i] = (o > v[i]) == high ? o : v[i];
            }
        }
#pragma unroll
        for (int x = E / 2; x > 0; x /= 2)
            if (x < k) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (!(i & x)) {
                        const bool down = ((tid * E + i) & k) == 0;
                        const unsigned long long a = v[i], b = v[i | x];
                        const bool turn = (a < b) == down;
                        v[i] = turn ? b : a;
                        v[i | x] = turn ? a : b;
                    }
            }
    }
    const int c = min(count, P.cap);
    unsigned long long* out = e + buf * N;
#pragma unroll
    for (int i = 0; i < E; ++i) out[i * NT + tid] = v[i];
    __syncthreads();
    for (int i = tid; i < c; i += NT) put(P, item, s, i, out[i % E * NT + i / E]);
}

// Longer lists, and few long prefixes: chunks of kChunk positions, sorted in shared memory, and each entry's place as the sum of its places in all of them.
__global__ void __launch_bounds__(kThreads) order_sort_kernel(Order P) {
    __shared__ unsigned long long e[kChunk];
    __shared__ int count, base;
    const int tid = threadIdx.x, chunk = blockIdx.x % P.chunks, item = blockIdx.x / P.chunks, s = item / P.Hq, h = item % P.Hq;
    pdl_enter();
    const int n = P.visible(s), j0 = min(n, chunk * kChunk), j1 = min(n, j0 + kChunk);
    const unsigned long long least = P.weakest ? P.weakest[item] : 0ull;
    if (tid == 0) count = 0;
    __syncthreads();
    sweep<kThreads>(P, s, h, j0, j1, [&](const unsigned long long (&key)[8]) { collect<kThreads>(key, least, e, kChunk, &count); });
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
    if (tid == 0) {
        base = atomicAdd(&P.room[item], c);
        P.run_at[blockIdx.x] = base;
        P.run_len[blockIdx.x] = c;
    }
    __syncthreads();
    for (int i = tid; i < c && base + i < P.cap; i += kThreads) P.run[(size_t)item * P.cap + base + i] = e[i];
}

__global__ void __launch_bounds__(256) order_merge_kernel(Order P) {
    constexpr int kTogether = 4;                                  // chunks searched side by side
    const int item = blockIdx.x / P.chunks, chunk = blockIdx.x % P.chunks, s = item / P.Hq;
    pdl_enter();
    const unsigned long long* run = P.run + (size_t)item * P.cap;
    const int32_t *at = P.run_at + item * P.chunks, *len = P.run_len + item * P.chunks;
    const int from = at[chunk], count = min(len[chunk], P.cap - from);
    for (int i = threadIdx.x; i < count; i += 256) {
        const unsigned long long key = run[from + i];
        int place = i;
        for (int c0 = 0; c0 < P.chunks; c0 += kTogether) {
            int lo[kTogether], hi[kTogether], start[kTogether];
            bool more = false;
#pragma unroll
            for (int y = 0; y < kTogether; ++y) {
                const int c = c0 + y;
                const bool other = c < P.chunks && c != chunk;
                start[y] = other ? at[c] : 0;
                lo[y] = 0;
                hi[y] = other ? min(len[c], P.cap - start[y]) : 0;
                more |= lo[y] < hi[y];
            }
            while (more) {
                more = false;
#pragma unroll
                for (int y = 0; y < kTogether; ++y)
                    if (lo[y] < hi[y]) {
                        const int mid = (lo[y] + hi[y]) >> 1;
                        if (run[start[y] + mid] > key) lo[y] = mid + 1; else hi[y] = mid;
                        more |= lo[y] < hi[y];
                    }
            }
#pragma unroll
            for (int y = 0; y < kTogether; ++y) place += lo[y];
        }
        if (place < P.cap) put(P, item, s, place, key);
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
    const int64_t items = (int64_t)C.nseq * C.Hq;
    auto held = [&](auto e_tag) {
        constexpr int E = decltype(e_tag)::value, smem = 2 * E * 1024 * 8;
        if (cudaFuncSetAttribute(order_held_kernel<E>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return (int)DMA_ERR_CUDA;
        return launch_overlapped(order_held_kernel<E>, dim3((unsigned)items), dim3(1024), smem, st, 1, P);
    };
    if (L.cap <= 8192 && (L.chunks <= 16 || items >= 148)) {
        if (L.cap <= 1024) return held(std::integral_constant<int, 1>{});
        if (L.cap <= 2048) return held(std::integral_constant<int, 2>{});
        if (L.cap <= 4096) return held(std::integral_constant<int, 4>{});
        return held(std::integral_constant<int, 8>{});
    }
    const unsigned grid = (unsigned)(items * L.chunks);
    if ((rc = launch_overlapped(order_sort_kernel, dim3(grid), dim3(kThreads), 0, st, 1, P))) return rc;
    return launch_overlapped(order_merge_kernel, dim3(grid), dim3(256), 0, st, 1, P);
}

}  // namespace dma
