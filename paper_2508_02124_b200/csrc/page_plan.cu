// Pages for requests of new lengths (include/dma.h, dma_page_plan): block table, ring of free pages, row and slot maps.
//
// With held = ceil(lens / P), hold = ceil(want / P): a request needs max(0, hold - held) pages, brings max(0, want - lens) rows and gives
// max(0, held - hold) pages back. Whether it is granted, and where its pages and rows lie, follows from running sums over the requests, a thread per
// request, 1024 requests at a time; a thread per page taken, per page given back and per row then finds its request by a search in the sums.
// Every CTA forms the sums, which takes it less time than waiting for another's, and takes its share of the pages and rows: a row's page is its table's entry or, where the call
// takes it, the ring's, so that no CTA waits for another's writes. One CTA where there is little to write.
// Bound by latency: three dependent trips to memory (lengths, ring or table, maps) and the barriers of the sums. us: 64 requests of a decoding step 5.3; 1000 requests, 50 000 rows and
// as many pages given back 7.9 (by one CTA 51, and its rows by a second kernel 6).
#include <algorithm>
#include <climits>

#include "paged.cuh"

namespace dma {
namespace {

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;

struct PlanShared {
    int64_t part[3][kPlanWarps], back[kPlanThreads];               // back: pages given back before each request of this turn
    int closed[kPlanWarps], refused[kPlanWarps], last[kPlanWarps];
    int take[kPlanThreads], row[kPlanThreads];                     // pages taken, rows before each request of this turn
    int lens[kPlanThreads], held[kPlanThreads], hold[kPlanThreads];
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

// state: lens_out and pool_out are written (by the first CTA); maps: everything else is.
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const int32_t* lens, const int32_t* want, int32_t* table, int32_t* ring, const int32_t* pool,
                                                                 int32_t* lens_out, int32_t* pool_out, int32_t* cu, int32_t* row_seq, int32_t* row_pos, int32_t* slot,
                                                                 int nseq, int rows, int page_log, int num_pages, int max_blocks, int64_t ld, bool state, bool maps) {
    __shared__ PlanShared S;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t begin = (int64_t)blockIdx.x * kPlanThreads + tid, stride = (int64_t)gridDim.x * kPlanThreads;
    const bool first_cta = blockIdx.x == 0;
    pdl_enter(lens, want, table, ring, pool, lens_out, pool_out, cu, row_seq, row_pos, slot);
    const int pool_head = pool[0], pool_free = pool[1];
    const int head = (pool_head % num_pages + num_pages) % num_pages, free = min(max(pool_free, 0), num_pages);
    const int capacity = max_blocks << page_log, mask = (1 << page_log) - 1;
    int64_t asked = 0, asked_rows = 0, given = 0;                   // by the requests of the turns before
    int taken = 0, total = 0, refused = 0;                          // pages, rows granted; requests refused
    int rows_granted = INT_MAX;                                     // rows before the first request refused for rows
    auto wrap = [&](int64_t i) {                                    // (beyond twice the ring only where the pool's words are not what an earlier call left)
        if (i >= num_pages) i -= num_pages;
        return (int)(i < num_pages ? i : i % num_pages);
    };
    for (int base = 0; base < nseq; base += kPlanThreads) {
        const int r = base + tid, turn = min(nseq - base, kPlanThreads);
        const bool real = r < nseq;
        const int n = real ? lens[r] : 0, m = real ? want[r] : 0;
        bool good = n >= 0 && n <= capacity && m >= 0 && m <= capacity;
        // (n and m up to 2^31 - 1: no sum with the page size)
        const int held = good ? (n >> page_log) + ((n & mask) != 0) : 0, hold = good ? (m >> page_log) + ((m & mask) != 0) : 0;
        const int need = max(hold - held, 0), back = max(held - hold, 0);
        int64_t sum_need, sum_rows, sum_back;
        const int64_t before_need = asked + running_sum(need, S.part[0], sum_need) - need;
        good = good && (need == 0 || before_need + need <= free);
        const int fresh = good ? max(m - n, 0) : 0;
        const int64_t before_rows = asked_rows + running_sum(fresh, S.part[1], sum_rows) - fresh;
        const bool late = fresh > 0 && before_rows + fresh > rows;
        // (what the first late request finds before it was all granted, and nothing behind it is)
        const int first = __reduce_min_sync(0xffffffffu, late ? (int)min(before_rows, (int64_t)INT_MAX) : INT_MAX);
        if (late) good = false;
        // a request refused for pages, or late, ends what is taken: the sums behind it say nothing any more
        const int last = __reduce_max_sync(0xffffffffu, good && need > 0 ? (int)(before_need + need) : 0);
        const int bad = __popc(__ballot_sync(0xffffffffu, real && !good));
        if (lane == 0) { S.closed[warp] = first; S.refused[warp] = bad; S.last[warp] = last; }
        const int64_t before_back = running_sum(good ? back : 0, S.part[2], sum_back) - (good ? back : 0);       // (its barrier: closed, refused, last)
        rows_granted = min(rows_granted, __reduce_min_sync(0xffffffffu, S.closed[lane]));
        refused += __reduce_add_sync(0xffffffffu, S.refused[lane]);
        const int until = max(taken, __reduce_max_sync(0xffffffffu, S.last[lane]));
        const int row = (int)min(before_rows, (int64_t)rows_granted);
        asked += sum_need;
        asked_rows += sum_rows;
        const int row_end = (int)min(asked_rows, (int64_t)rows_granted);
        if (real && first_cta) {
            if (state) lens_out[r] = good ? m : n;
            if (maps) cu[r] = row;
        }
        if (maps) {
            // A request finds all that was asked before it granted, or takes nothing itself: behind the last page taken every offset lies behind it too.
            S.take[tid] = (int)min(before_need, (int64_t)free) - taken;
            S.back[tid] = before_back;
            S.row[tid] = row;
            S.lens[tid] = n;
            S.held[tid] = held;
            S.hold[tid] = good ? hold : held;
            __syncthreads();
            for (int64_t i = begin; i < until - taken; i += stride) {
                const int k = find_last(S.take, turn, (int)i);
                table[(base + k) * ld + S.held[k] + ((int)i - S.take[k])] = ring[wrap((int64_t)head + taken + i)];
            }
            for (int64_t i = begin; i < sum_back; i += stride) {
                const int k = find_last(S.back, turn, i);
                ring[wrap((int64_t)head + free + given + i)] = table[(base + k) * ld + S.hold[k] + (i - S.back[k])];
            }
            // (a request without rows has the offset of its successor: the last one with its offset at or before the row is the row's)
            for (int64_t t = total + begin; t < row_end; t += stride) {
                const int k = find_last(S.row, turn, (int)t), pos = S.lens[k] + ((int)t - S.row[k]), b = pos >> page_log, had = S.held[k];
                const int page = b < had ? table[(base + k) * ld + b] : ring[wrap((int64_t)head + taken + S.take[k] + (b - had))];
                row_seq[t] = base + k;
                row_pos[t] = pos;
                slot[t] = (unsigned)page < (unsigned)num_pages ? (page << page_log) + (pos & mask) : -1;
            }
        }
        taken = until;
        given += sum_back;
        total = row_end;
        __syncthreads();                        // the turn's shared memory has been read
    }
    if (first_cta && tid == 0) {
        if (maps) cu[nseq] = total;
        if (state) {
            pool_out[0] = wrap((int64_t)head + taken);
            pool_out[1] = (int)min((int64_t)free - taken + given, (int64_t)num_pages);
            pool_out[2] = refused;
            pool_out[3] = total;
        }
    }
    if (maps)
        for (int64_t t = total + begin; t < rows; t += stride) row_seq[t] = row_pos[t] = slot[t] = -1;
}

bool apart(const int32_t* a, const int32_t* b, size_t n) { return a + n <= b || b + n <= a; }

}  // namespace

int launch_page_plan(const Cache& C, const int32_t* lens, const int32_t* want, int32_t* table, int32_t* ring, const int32_t* pool, int32_t* lens_out,
                     int32_t* pool_out, int32_t* cu, int32_t* row_seq, int32_t* row_pos, int32_t* slot, cudaStream_t st) {
    // Lengths and pool that are updated in place are written when every CTA has read them: by a second kernel where there are several.
    const bool in_place = !(apart(lens, lens_out, C.nseq) && apart(want, lens_out, C.nseq) && apart(pool, pool_out, 4));
    // Several CTAs where there may be much to write, a thread per row or page (us of one CTA and of this many, replayed: 64 requests that bring 4096 rows and hold up to 512 pages 7.3 and 5.1, in
    // place, with 2 to set it up, 9.3 and 10.6; 16 that bring 8192 rows 9.3 and 4.9, in place 11.2 and 10.5; decoding steps of 64 to 1000 requests the same either way).
    const int64_t most = (int64_t)C.rows + (int64_t)C.nseq * C.max_blocks;
    const bool little = C.rows <= (in_place ? 4096 : 1024) && most <= 64 * 1024;
    const int ctas = little ? 1 : (int)std::min<int64_t>(148, (most + kPlanThreads - 1) / kPlanThreads);
    const bool two = ctas > 1 && in_place;
    int rc = launch_overlapped(page_plan_kernel, dim3(ctas), dim3(kPlanThreads), 0, st, 1, lens, want, table, ring, pool, lens_out, pool_out, cu, row_seq, row_pos,
                               slot, C.nseq, C.rows, C.page_log, C.num_pages, C.max_blocks, C.table_ld, !two, true);
    if (rc || !two) return rc;
    return launch_overlapped(page_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, 1, lens, want, table, ring, pool, lens_out, pool_out, cu, row_seq, row_pos, slot,
                             C.nseq, C.rows, C.page_log, C.num_pages, C.max_blocks, C.table_ld, true, false);
}

}  // namespace dma
