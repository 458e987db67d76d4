// The order of prefixes (include/dma.h, dma_prefix_order): of every prefix and query head the w keys of the largest delta, sorted.
//
// The weakest kept key of each (prefix, head) is found as decoding finds it (cache4_select.cu); what is not below it is collected and sorted, by a CTA per (prefix, head) where shared memory
// holds the list, 8192 entries, else in chunks of it. Ordering is round trips and instructions, not memory: 32 heads of 16K keys, w = 2048: 16 us (rows 2, selection 6.4, lists 7.8; the
// weights' bytes 0.4); five prefixes of up to 64K, w = 4096: 38 to 49 us (2, 20, 18 to 24; bytes 4.6). In chunks the first takes 33 us; 16 prefixes of 16K, w = 4096, 110 instead of 49; one of 256K 63
// instead of 54, one of 1M, w = 8192, 155 either way. In chunks one of 256K, w = 16384, takes 91 us, one of 1M 157.
#include <algorithm>
#include <type_traits>

#include "cache4_decode.cuh"

namespace dma {
namespace {

constexpr int kHeld = 8192, kChunk = 4096, kSpan = 4096;

struct Order {
    const float* delta;
    const int32_t *table, *len;
    int32_t *slot, *order_len;
    float* weight;
    int64_t ld, order_ld;
    const unsigned long long* weakest;       // NULL: all are kept
    unsigned long long* run;                 // [nseq * Hq, cap]: entries of lists that no CTA holds
    int32_t* room;                           // [nseq * Hq]: how many there are
    int Hq, w, page_log, num_pages, max_blocks, spans, chunks, cap;
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

// f(patterns, position, how many there are, where they lie) for the keys of [j0, j1) (j0 a multiple of 16), sixteen of a thread side by side in one page (pages have 16 keys and more).
template <int NT, typename F>
__device__ __forceinline__ void sweep(const Order& P, int s, int h, int j0, int j1, F f) {
    const int32_t* pages = P.table + s * P.ld;
    const int mask = (1 << P.page_log) - 1;
    auto page_of = [&](int j) { return j < j1 ? pages[j >> P.page_log] : -1; };
    int next = page_of(j0 + threadIdx.x * 16);
#pragma unroll 1
    for (int b = j0; b < j1; b += NT * 16) {
        const int j = b + threadIdx.x * 16, page = next;
        const bool there = (unsigned)page < (unsigned)P.num_pages;
        const uint32_t* from = reinterpret_cast<const uint32_t*>(P.delta) + (((size_t)(there ? page : 0) * P.Hq + h) << P.page_log) + (j & mask);
        uint32_t u[16];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (there) x = *reinterpret_cast<const uint4*>(from + i);
            u[i] = x.x; u[i + 1] = x.y; u[i + 2] = x.z; u[i + 3] = x.w;
        }
        next = page_of(j + NT * 16);
        f(u, j, there ? min(16, j1 - j) : 0, from);
    }
}

// The kept ones among a thread's `n` keys from position j on to `to`, in no order; `count` is moved on. Few are kept as a rule: a thread reads them again one by one (all sixteen
// in turn, with keys compared in 64 bits: 160 lists of 64K keys 35 us instead of 27).
__device__ __forceinline__ void collect(const uint32_t (&u)[16], int j, int n, const uint32_t* from, unsigned long long least, unsigned long long* to, int room, int* count) {
    const int lane = threadIdx.x & 31;
    // the weakest kept key's pattern and position: keys of the same weight are kept up to there
    const int pattern = (int)(least >> 32);
    const uint32_t last = 0xFFFFFFFFu - (uint32_t)least;
    auto above = [&](int than) {
        uint32_t flags = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) flags |= (uint32_t)((int)(u[i] & 0x7FFFFFFFu) > than) << i;
        return flags;
    };
    uint32_t flags = above((uint32_t)j <= last ? pattern - 1 : pattern);
    if ((uint32_t)j <= last && last < (uint32_t)j + 15u) flags &= above(pattern) | ((2u << (last - (uint32_t)j)) - 1u);
    flags &= (1u << max(n, 0)) - 1u;
    const int mine = __popc(flags);
    int at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += y;
    }
    int base = 0;
    if (lane == 31 && at) base = atomicAdd(count, at);
    at += __shfl_sync(0xffffffffu, base, 31) - mine;
    for (; flags; flags &= flags - 1u, ++at) {
        const int i = __ffs(flags) - 1;
        if (at < room) to[at] = order_key(from[i] & 0x7FFFFFFFu, j + i);
    }
}

__device__ __forceinline__ void put(const Order& P, int item, int s, int place, unsigned long long key) {
    const int j = (int)(0xFFFFFFFFu - (uint32_t)key);
    P.slot[item * P.order_ld + place] = (P.table[s * P.ld + (j >> P.page_log)] << P.page_log) + (j & ((1 << P.page_log) - 1));
    P.weight[item * P.order_ld + place] = __uint_as_float((uint32_t)(key >> 32));
}

// Numbers of a CTA, E side by side per thread, in descending order by a bitonic network; buf: 2 E NT places. Exchanges over fewer than 32 E places stay in registers and shuffles.
template <int NT, int E>
__device__ void sort_down(unsigned long long (&v)[E], unsigned long long* buf) {
    constexpr int N = E * NT;
    const int tid = threadIdx.x;
    int which = 0;
#pragma unroll 1
    for (int k = 2; k <= N; k *= 2) {
#pragma unroll 1
        for (int x = k / 2; x >= 32 * E; x /= 2) {                // other warps'
            unsigned long long* to = buf + which * N;
#pragma unroll
            for (int i = 0; i < E; ++i) to[i * NT + tid] = v[i];
            __syncthreads();
            const bool high = ((tid * E & x) == 0) == ((tid * E & k) == 0);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const unsigned long long o = to[i * NT + (tid ^ x / E)];
                v[i] = (o > v[i]) == high ? o : v[i];
            }
            which ^= 1;
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
}

// Lists of up to E * NT entries by a CTA per (prefix, head). What is kept is collected in shared memory, dealt into as many bins between the smallest and the largest weight as the list may
// have entries, and ranked within its bin; where a bin has many (weights that crowd), sorted by a bitonic network instead (2048 entries: 6 us more).
template <int NT, int E>
__global__ void __launch_bounds__(NT, 1024 / NT) order_held_kernel(Order P) {
    constexpr int N = E * NT, kCrowd = 48;
    extern __shared__ unsigned long long e[];                     // [2][N] entries, [N] bins
    __shared__ int count, crowd;
    __shared__ uint32_t lowest, highest;
    __shared__ int part[NT / 32];
    int* bins = reinterpret_cast<int*>(e + 2 * N);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, item = blockIdx.x, s = item / P.Hq, h = item % P.Hq;
    pdl_enter();
    const int n = P.visible(s);
    const unsigned long long least = P.weakest ? P.weakest[item] : 0ull;
    if (tid == 0) { count = 0; crowd = 0; lowest = ~0u; highest = 0u; }
    for (int i = tid; i < N; i += NT) bins[i] = 0;
    __syncthreads();
    sweep<NT>(P, s, h, 0, n, [&](const uint32_t (&u)[16], int j, int m, const uint32_t* from) { collect(u, j, m, from, least, e, N, &count); });
    __syncthreads();
    const int c = min(count, P.cap);
    uint32_t lo = ~0u, hi = 0u;
    for (int i = tid; i < c; i += NT) {
        lo = min(lo, (uint32_t)(e[i] >> 32));
        hi = max(hi, (uint32_t)(e[i] >> 32));
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { atomicMin(&lowest, lo); atomicMax(&highest, hi); }
    __syncthreads();
    lo = lowest;
    const float scale = (float)(N - 1) / fmaxf((float)(highest - lo), 1.0f);
    auto bin_of = [&](unsigned long long key) { return N - 1 - min(N - 1, (int)((float)((uint32_t)(key >> 32) - lo) * scale)); };     // (the largest first; never falls as the weight does)
    int where[E];                                                 // in its bin, as they come
    int most = 0;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i * NT + tid < c) {
            where[i] = atomicAdd(&bins[bin_of(e[i * NT + tid])], 1);
            most = max(most, where[i]);
        }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) atomicMax(&crowd, most);
    __syncthreads();
    if (crowd >= kCrowd) {
        unsigned long long v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = tid * E + i < c ? e[tid * E + i] : 0ull;
        __syncthreads();
        sort_down<NT, E>(v, e);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (tid * E + i < c) put(P, item, s, tid * E + i, v[i]);
        return;
    }
    // bins to places
    int mine[E], sum = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        mine[i] = sum;
        sum += bins[tid * E + i];
    }
    int x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int before = x - sum;
    for (int i = 0; i < NT / 32; ++i) before += i < warp ? part[i] : 0;
#pragma unroll
    for (int i = 0; i < E; ++i) bins[tid * E + i] = before + mine[i];
    __syncthreads();
    unsigned long long* dealt = e + N;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i * NT + tid < c) dealt[bins[bin_of(e[i * NT + tid])] + where[i]] = e[i * NT + tid];
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < c; i += NT) {
        const unsigned long long key = dealt[i];
        const int bin = bin_of(key), from = bins[bin], to = bin + 1 < N ? bins[bin + 1] : c;
        int place = from;
        for (int o = from; o < to; ++o) place += dealt[o] > key;
        put(P, item, s, place, key);
    }
}

// Longer lists. What is kept is collected as it comes, a CTA per kSpan positions, and sorted in chunks; an entry's place is the sum of its places in all of them.
__global__ void __launch_bounds__(kSpan / 16) order_collect_kernel(Order P) {
    const int span = blockIdx.x % P.spans, item = blockIdx.x / P.spans, s = item / P.Hq, h = item % P.Hq;
    pdl_enter();
    const int n = P.visible(s), j0 = min(n, span * kSpan), j1 = min(n, j0 + kSpan);
    const unsigned long long least = P.weakest ? P.weakest[item] : 0ull;
    sweep<kSpan / 16>(P, s, h, j0, j1, [&](const uint32_t (&u)[16], int j, int m, const uint32_t* from) { collect(u, j, m, from, least, P.run + (size_t)item * P.cap, P.cap, &P.room[item]); });
}

__global__ void __launch_bounds__(1024) order_sort_kernel(Order P) {
    constexpr int E = kChunk / 1024;
    extern __shared__ unsigned long long e[];                     // [2][kChunk]
    const int chunk = blockIdx.x % P.chunks, item = blockIdx.x / P.chunks, from = chunk * kChunk + threadIdx.x * E;
    pdl_enter();
    const int count = min(P.room[item], P.cap);
    if (count <= chunk * kChunk) return;
    unsigned long long* run = P.run + (size_t)item * P.cap;
    unsigned long long v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = from + i < count ? run[from + i] : 0ull;
    sort_down<1024, E>(v, e);
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (from + i < count) run[from + i] = v[i];
}

__global__ void __launch_bounds__(1024) order_merge_kernel(Order P) {
    constexpr int kTogether = 4;                                  // chunks searched side by side
    const int part = blockIdx.x % P.chunks, item = blockIdx.x / P.chunks, s = item / P.Hq;
    pdl_enter();
    const unsigned long long* run = P.run + (size_t)item * P.cap;
    const int count = min(P.room[item], P.cap), end = min(count, (part + 1) * kChunk);
    for (int i = part * kChunk + threadIdx.x; i < end; i += 1024) {
        const unsigned long long key = run[i];
        int place = i - part * kChunk;
        for (int c0 = 0; c0 * kChunk < count; c0 += kTogether) {
            int lo[kTogether], hi[kTogether];
            bool more = false;
#pragma unroll
            for (int y = 0; y < kTogether; ++y) {
                const int c = c0 + y;
                lo[y] = 0;
                hi[y] = c == part ? 0 : max(0, min(count - c * kChunk, kChunk));
                more |= hi[y] > 0;
            }
            while (more) {
                more = false;
#pragma unroll
                for (int y = 0; y < kTogether; ++y)
                    if (lo[y] < hi[y]) {
                        const int mid = (lo[y] + hi[y]) >> 1;
                        if (run[(c0 + y) * kChunk + mid] > key) lo[y] = mid + 1; else hi[y] = mid;
                        more |= lo[y] < hi[y];
                    }
            }
#pragma unroll
            for (int y = 0; y < kTogether; ++y) place += lo[y];
        }
        put(P, item, s, place, key);
    }
}

struct Layout {
    size_t seq, pos, weakest, room, run, total;
    int spans, chunks, cap;
    explicit Layout(const Cache& C) {
        const int64_t capacity = (int64_t)C.max_blocks << C.page_log, items = (int64_t)C.nseq * C.Hq;
        cap = (int)std::min<int64_t>(C.w, capacity);
        spans = (int)((capacity + kSpan - 1) / kSpan);
        chunks = (cap + kChunk - 1) / kChunk;
        size_t x = kWsHeaderBytes;
        auto take = [&](size_t bytes) { const size_t at = x; x += (bytes + 255) / 256 * 256; return at; };
        seq = take((size_t)C.nseq * 4);
        pos = take((size_t)C.nseq * 4);
        weakest = take((size_t)items * 8);
        room = take((size_t)items * 4);
        run = take(cap > kHeld ? (size_t)items * cap * 8 : 0);
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
               (int32_t*)(p + L.room), C.Hq, C.w, C.page_log, C.num_pages, C.max_blocks, L.spans, L.chunks, L.cap};
    int rc = launch_overlapped(order_rows_kernel, dim3(C.nseq), dim3(256), 0, st, 1, P, (int32_t*)(p + L.seq), (int32_t*)(p + L.pos), (int32_t*)p);
    if (rc) return rc;
    if (select) {
        const Rows R = {table, (const int32_t*)(p + L.seq), (const int32_t*)(p + L.pos), delta, C.table_ld, C.nseq, C.page_log, C.num_pages, C.max_blocks, C.Hq};
        if ((rc = launch_cache4_select(C, R, (unsigned long long*)(p + L.weakest), Plan{}, st))) return rc;
    }
    const int64_t items = (int64_t)C.nseq * C.Hq;
    auto held = [&](auto n_tag, auto e_tag) {
        constexpr int NT = decltype(n_tag)::value, E = decltype(e_tag)::value, smem = E * NT * 20;
        auto kernel = order_held_kernel<NT, E>;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return (int)DMA_ERR_CUDA;
        return launch_overlapped(kernel, dim3((unsigned)items), dim3(NT), smem, st, 1, P);
    };
    // More lists than SMs: smaller CTAs, several per SM (2048 lists of 1024 entries 26 us, of 1024 threads 72; 512 of 4096 30 and 37). Else all the threads that a CTA may have (32 of 4096
    // from 256K keys 29 us, of 512 threads 36).
    if (L.cap <= kHeld) {
        using std::integral_constant;
        const bool many = items > 148;
        if (L.cap <= 1024) return many ? held(integral_constant<int, 256>{}, integral_constant<int, 4>{}) : held(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
        if (L.cap <= 2048) return many ? held(integral_constant<int, 512>{}, integral_constant<int, 4>{}) : held(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
        if (L.cap <= 4096) return many ? held(integral_constant<int, 512>{}, integral_constant<int, 8>{}) : held(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
        return held(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
    }
    if ((rc = launch_overlapped(order_collect_kernel, dim3((unsigned)(items * L.spans)), dim3(kSpan / 16), 0, st, 1, P))) return rc;
    const unsigned grid = (unsigned)(items * L.chunks);
    constexpr int smem = 2 * kChunk * 8;
    if (cudaFuncSetAttribute(order_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return DMA_ERR_CUDA;
    if ((rc = launch_overlapped(order_sort_kernel, dim3(grid), dim3(1024), smem, st, 1, P))) return rc;
    return launch_overlapped(order_merge_kernel, dim3(grid), dim3(1024), 0, st, 1, P);
}

}  // namespace dma
