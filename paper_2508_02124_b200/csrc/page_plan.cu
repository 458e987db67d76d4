// Pages for requests of new lengths (include/dma.h, dma_page_plan): block table, ring of free pages, row and slot maps.
//
// With held = ceil(lens / P), hold = ceil(want / P): a request needs max(0, hold - held) pages, brings max(0, want - lens) rows and gives
// max(0, held - hold) pages back. Whether it is granted, and where its pages and rows lie, follows from running sums over the requests:
//   page_plan_kernel   one CTA: the sums, a thread per request, 1024 requests at a time; then a thread per page taken, per page given back
//                      and, in small calls, per row, each of which finds its request by a search in the sums
//   page_rows_kernel   the rows of large calls, on the whole chip
// Bound by latency: three dependent trips to memory (lengths, ring, table) and the barriers of the sums.
#include <algorithm>
#include <climits>

#include "paged.cuh"

namespace dma {
namespace {

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;

struct PlanShared {
    int64_t part[3][kPlanWarps];
    int closed[kPlanWarps];
    int refused[kPlanWarps];
    int64_t take[kPlanThreads + 1], back[kPlanThreads + 1];        // pages taken / given back before each request of this turn
    int held[kPlanThreads], hold[kPlanThreads];
};

// Inclusive running sum over the CTA; `total` of all threads. One barrier; `part` is not used again before the next one.
__device__ __forceinline__ int64_t running_sum(int64_t x, int64_t* part, int64_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int64_t p = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, p, o);
        if (lane >= o) p += y;
    }
    total = __shfl_sync(0xffffffffu, p, 31);
    const int64_t before = __shfl_sync(0xffffffffu, p, max(warp - 1, 0));
    return x + (warp ? before : 0);
}

// the last i in [0, n) with first[i] <= x (first[0] <= x, ascending)
template <typename T>
__device__ __forceinline__ int find_last(const T* first, int n, T x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Row t of the plan. cu: rows before each request (monotone, cu[nseq] = total). A request without rows has the offset of its successor,
// so the last request with cu <= t is the one that t belongs to.
__device__ __forceinline__ void write_row(int t, int seq, int pos_end, int next, const int32_t* table, int64_t ld, int page_log, int num_pages,
                                          int32_t* row_seq, int32_t* row_pos, int32_t* slot) {
    const int pos = pos_end - (next - t);
    const int page = table[seq * ld + (pos >> page_log)];
    row_seq[t] = seq;
    row_pos[t] = pos;
    slot[t] = (unsigned)page < (unsigned)num_pages ? (page << page_log) + (pos & ((1 << page_log) - 1)) : -1;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const int32_t* lens, const int32_t* want, int32_t* table, int32_t* ring, const int32_t* pool,
                                                                 int32_t* lens_out, int32_t* pool_out, int32_t* cu, int32_t* row_seq, int32_t* row_pos, int32_t* slot,
                                                                 int nseq, int rows, int page_log, int num_pages, int max_blocks, int64_t ld, int rows_here) {
    __shared__ PlanShared S;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_enter(lens, want, table, ring, pool, lens_out, pool_out, cu, row_seq, row_pos, slot);
    const int head = (pool[0] % num_pages + num_pages) % num_pages, free = min(max(pool[1], 0), num_pages);
    const int capacity = max_blocks << page_log, mask = (1 << page_log) - 1;
    int64_t asked = 0, asked_rows = 0, taken = 0, given = 0;        // by the requests of the turns before
    int rows_granted = INT_MAX;                                     // rows before the first request refused for rows
    int refused = 0;
    auto wrap = [&](int64_t i) {                                    // (beyond twice the ring only where the pool's words are not what an earlier call left)
        if (i >= num_pages) i -= num_pages;
        return (int)(i < num_pages ? i : i % num_pages);
    };
    for (int base = 0; base < nseq; base += kPlanThreads) {
        const int r = base + tid;
        const bool real = r < nseq;
        const int n = real ? lens[r] : 0, m = real ? want[r] : 0;
        bool good = n >= 0 && n <= capacity && m >= 0 && m <= capacity;
        // (n and m up to 2^31 - 1: no sum with the page size)
        const int held = good ? (n >> page_log) + ((n & mask) != 0) : 0, hold = good ? (m >> page_log) + ((m & mask) != 0) : 0;
        const int need = max(hold - held, 0), back = max(held - hold, 0);
        int64_t sum_need, sum_rows, sum_back;
        const int64_t before_need = asked + running_sum(need, S.part[0], sum_need) - need;
        good = good && (need == 0 || before_need + need <= free);
        int fresh = good ? max(m - n, 0) : 0;
        const int64_t before_rows = asked_rows + running_sum(fresh, S.part[1], sum_rows) - fresh;
        const bool late = fresh > 0 && before_rows + fresh > rows;
        // (what the first late request finds before it was all granted, and nothing behind it is)
        const int mine = late ? (int)min(before_rows, (int64_t)INT_MAX) : INT_MAX;
        const int first = __reduce_min_sync(0xffffffffu, mine);
        if (late) good = false;
        const int bad = __popc(__ballot_sync(0xffffffffu, real && !good));
        if (lane == 0) { S.closed[warp] = first; S.refused[warp] = bad; }
        const int64_t before_back = running_sum(good ? back : 0, S.part[2], sum_back) - (good ? back : 0);       // (its barrier: closed, refused)
        rows_granted = min(rows_granted, __reduce_min_sync(0xffffffffu, S.closed[lane]));
        refused += __reduce_add_sync(0xffffffffu, S.refused[lane]);
        // pages: a granted request finds all that was asked before it granted; a refused one takes none
        S.take[tid] = min(before_need, (int64_t)free) - taken;
        S.back[tid] = before_back;
        S.held[tid] = held;
        S.hold[tid] = good ? hold : held;
        if (real) {
            const int now = good ? m : n;
            lens_out[r] = now;
            cu[r] = (int)min(before_rows, (int64_t)rows_granted);
        }
        __syncthreads();
        // A request refused for pages, or late, has hold = held here, and the sums behind it say nothing any more: what is taken ends with the last granted one.
        int64_t last = 0;
        if (good && need > 0) last = before_need + need;
#pragma unroll
        for (int o = 16; o; o >>= 1) last = max(last, (int64_t)__shfl_xor_sync(0xffffffffu, last, o));
        if (lane == 0) S.part[0][warp] = last;
        __syncthreads();
        last = S.part[0][lane];
#pragma unroll
        for (int o = 16; o; o >>= 1) last = max(last, (int64_t)__shfl_xor_sync(0xffffffffu, last, o));
        const int turn = min(nseq - base, kPlanThreads);
        const int64_t until = max(last, taken);
        for (int64_t i = tid; i < until - taken; i += kPlanThreads) {
            const int k = find_last(S.take, turn, i);
            table[(base + k) * ld + S.held[k] + (i - S.take[k])] = ring[wrap(head + taken + i)];
        }
        for (int64_t i = tid; i < sum_back; i += kPlanThreads) {
            const int k = find_last(S.back, turn, i);
            ring[wrap((int64_t)head + free + given + i)] = table[(base + k) * ld + S.hold[k] + (i - S.back[k])];
        }
        asked += sum_need;
        asked_rows += sum_rows;
        taken = until;
        given += sum_back;
        __syncthreads();                        // the turn's shared memory has been read
    }
    const int total = (int)min(asked_rows, (int64_t)rows_granted);
    if (tid == 0) {
        cu[nseq] = total;
        pool_out[0] = wrap(head + taken);
        pool_out[1] = (int)min(free - taken + given, (int64_t)num_pages);
        pool_out[2] = refused;
        pool_out[3] = total;
    }
    if (!rows_here) return;
    __syncthreads();                            // table, lens_out and cu of this CTA
    for (int t = tid; t < rows; t += kPlanThreads) {
        if (t < total) {
            const int k = find_last(cu, nseq, t);
            write_row(t, k, lens_out[k], cu[k + 1], table, ld, page_log, num_pages, row_seq, row_pos, slot);
        } else {
            row_seq[t] = row_pos[t] = slot[t] = -1;
        }
    }
}

// A CTA takes kRowsPerCta rows; its requests' offsets, where they are few, are searched in shared memory.
constexpr int kRowThreads = 256, kRowsPerCta = 1024, kStaged = 2048;
__global__ void __launch_bounds__(kRowThreads) page_rows_kernel(const int32_t* table, const int32_t* lens_out, const int32_t* cu, int32_t* row_seq, int32_t* row_pos,
                                                                int32_t* slot, int nseq, int rows, int page_log, int num_pages, int64_t ld) {
    __shared__ int32_t staged[kStaged];
    __shared__ int ends[2];
    const int tid = threadIdx.x, t0 = blockIdx.x * kRowsPerCta, t1 = min(rows, t0 + kRowsPerCta);
    pdl_enter(table, lens_out, cu, row_seq, row_pos, slot);
    const int total = cu[nseq];
    if (t0 < total) {
        if (tid < 64 && tid % 32 == 0) ends[tid / 32] = find_last(cu, nseq, tid == 0 ? t0 : min(t1, total) - 1);
        __syncthreads();
        const int k0 = ends[0], n = ends[1] + 1 - k0;
        const bool in_smem = n < kStaged;
        if (in_smem) {
            for (int i = tid; i <= n; i += kRowThreads) staged[i] = cu[k0 + i];
            __syncthreads();
        }
        for (int t = t0 + tid; t < min(t1, total); t += kRowThreads) {
            const int k = in_smem ? find_last(staged, n, t) : find_last(cu + k0, n, t);
            write_row(t, k0 + k, lens_out[k0 + k], in_smem ? staged[k + 1] : cu[k0 + k + 1], table, ld, page_log, num_pages, row_seq, row_pos, slot);
        }
    }
    for (int t = max(t0, total) + tid; t < t1; t += kRowThreads) row_seq[t] = row_pos[t] = slot[t] = -1;
}

}  // namespace

int launch_page_plan(const Cache& C, const int32_t* lens, const int32_t* want, int32_t* table, int32_t* ring, const int32_t* pool, int32_t* lens_out,
                     int32_t* pool_out, int32_t* cu, int32_t* row_seq, int32_t* row_pos, int32_t* slot, cudaStream_t st) {
    constexpr int kRowsHere = 4096;
    const bool here = C.rows <= kRowsHere;
    const int rc = launch_overlapped(page_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, 1, lens, want, table, ring, pool, lens_out, pool_out, cu, row_seq,
                                     row_pos, slot, C.nseq, C.rows, C.page_log, C.num_pages, C.max_blocks, C.table_ld, here ? 1 : 0);
    if (rc || here) return rc;
    return launch_overlapped(page_rows_kernel, dim3((C.rows + kRowsPerCta - 1) / kRowsPerCta), dim3(kRowThreads), 0, st, 1, table, lens_out, cu, row_seq, row_pos,
                             slot, C.nseq, C.rows, C.page_log, C.num_pages, C.table_ld);
}

}  // namespace dma
