// Selection for dma_cache4_decode (include/dma.h): every (row, query head) keeps the w visible keys with the largest dynamic weight delta, ties to the lower index. What the
// attention needs is the weakest kept key, as a 64-bit order key: a key is kept iff its order key is not below it.
//
// Kernels
//   select_held_kernel   rows that a CTA's registers hold
//   select_kernel        longer ones, by a sample and a sweep; a cluster per row where there are few
//   plan_kernel          the attention's shares of the work, where nothing is selected (else the selection's first CTA makes them)
//
// Measured, 32 heads, us: one row of 16384 keys 6.0, of 262144 25, of 1048576 49; 64 rows of 1 to 16K 41; 256 of 4096 68; 64 of 65536 178. Bound by barriers and round trips where there
// are few rows, by instructions where there are many (64 rows of 1 to 16K: 63 % of the issue slots, 43 per 32 keys, the fixed part of a row included; the weights' bytes alone would take
// a fifth of the time). All weights equal: 7 for the one row, 48 for the 64; quarters of whole numbers: 12 and 120.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "cache4_decode.cuh"
#include "cache4_sample.h"

namespace dma {
namespace {

namespace cg = cooperative_groups;

__device__ __forceinline__ int row_units(const Plan& P, int n) {
    if (n < 0) return 0;
    const float drop = n > P.w ? 1.0f - (float)P.w / (float)n : 0.0f, all = n > P.w ? 1.0f - powf(drop, (float)P.heads) : 1.0f;
    // (the fixed cost of an item, its queries and its end, is about that of a unit)
    return (int)ceilf((float)n * (0.15f + 0.85f * all) / (float)(1 << P.unit_log)) + 1;
}

template <int NT>
__device__ void make_plan(const Rows& R, int rows, const Plan& P) {
    __shared__ int part[NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int carry = 0;
    for (int base = 0; base < rows; base += NT) {
        const int t = base + tid;
        int r, units = 0;
        if (t < rows) {
            const int n = R.visible(t, r);
            units = row_units(P, n) * P.per_row;
        }
        int x = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) part[warp] = x;
        __syncthreads();
        int before = 0, all = 0;
        for (int i = 0; i < NT / 32; ++i) {
            before += i < warp ? part[i] : 0;
            all += part[i];
        }
        if (t < rows) P.ustart[t] = carry + before + x - units;
        carry += all;
        __syncthreads();
    }
    if (tid == 0) P.ustart[rows] = carry;
    for (int i = tid; i < rows * P.per_row; i += NT) P.tickets[i] = 0;
}

__global__ void __launch_bounds__(1024) plan_kernel(Rows R, int rows, Plan P) {
    pdl_enter(R.seq, R.pos, P.ustart, P.tickets);
    make_plan<1024>(R, rows, P);
}

// (the pattern of keys in pages outside the pool: fewer than w others, which are all kept)
__device__ __forceinline__ unsigned long long threshold(unsigned long long found) { return found >> 32 ? found : 0ull; }

// The weakest kept key of a (row, query head). A sample brackets its delta (4.5 standard deviations of the sample's rank to either side); one sweep over the row
// counts the keys above the bracket and notes those inside, a few per cent, each thread in slots of its own; the need-th of these is found by
// a histogram over the bracket and a ranking of the bin's keys. Rows of up to kSample keys are their own sample: the bracket is one bin. A bracket that misses, or holds too
// many (weights that crowd), is replaced by a bin of a histogram of the row, and the row is swept again; equal weights are counted by index.
constexpr int kShared = 512, kRank = 128;                // overflow slots, most keys ranked against each other
// slots per thread (512 threads of 12: rows of 64K, w = 8192, are swept twice, 277 us for 64 rows; of 20: 181)
__host__ __device__ constexpr int own_slots(int threads) { return threads == 256 ? 16 : 20; }
constexpr int kBins = 1024;
template <int NT>
struct alignas(16) HeldShared {
    unsigned long long cand[kRank];
    int hist[kBins];
    uint32_t wmin[NT / 32], wmax[NT / 32];
    int part[NT / 32], above[NT / 32];
    int bin[2], need, count, ncand, nmore;
    unsigned long long found;
};
template <int NT, bool kCluster>
struct alignas(16) SelectShared : HeldShared<NT> {
    int sum[kCluster ? kBins : 1];                                // a cluster's row's bins
    uint2 own[own_slots(NT) * NT], more[kShared];                          // (pattern, index) of keys inside the bracket
    int total[2][3];                                              // this CTA's keys above the bracket and inside, and its overflow; of the last two sweeps
};
// The bracket's ranks of the sample, to either side of the expected one; and whether the slots take the row's part between them, with a quarter to spare.
constexpr int kPer = 8;                                           // a thread's keys of the sample
__host__ __device__ __forceinline__ float bracket(int n, int w, int sample) {
    const float q = (float)w / (float)n;
    return 4.5f * sqrtf(q * (float)sample * (1.0f - q)) + 4.0f;
}
__host__ __device__ __forceinline__ bool collects(int n, float dev, int threads, int sample, int ctas) {
    return (float)n * (2.0f * dev + 1.0f) <= 0.75f * (float)sample * (float)((own_slots(threads) - 4) * threads) * (float)ctas;
}
__device__ __forceinline__ int shift_of(uint32_t width) { return max(0, 22 - __clz((int)width)); }       // kBins bins over width + 1 patterns

// The descending running count of the bins in hist: a thread's bins are kBins - 1 - tid kBins / NT and those below it, `excl` keys lie above them. The bins are zeroed again. One barrier.
template <int NT>
__device__ __forceinline__ void scan_bins(HeldShared<NT>& S, int* hist, int& excl, int (&c)[kBins / NT]) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, top = kBins - 1 - tid * (kBins / NT);
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kBins / NT; ++i) { c[i] = hist[top - i]; hist[top - i] = 0; sum += c[i]; }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) S.part[warp] = incl;
    __syncthreads();
    excl = __reduce_add_sync(0xffffffffu, lane < warp && lane < NT / 32 ? S.part[lane] : 0) + incl - sum;
}
// whether one of the thread's bins holds rank `want` (from 1): which, how many keys it holds and how many lie above it
template <int NT>
__device__ __forceinline__ bool bin_of(int want, int excl, const int (&c)[kBins / NT], int& bin, int& before, int& count) {
    bool mine = false;
#pragma unroll
    for (int i = 0; i < kBins / NT; ++i) {
        if (excl < want && want <= excl + c[i]) { bin = kBins - 1 - threadIdx.x * (kBins / NT) - i; before = excl; count = c[i]; mine = true; }
        excl += c[i];
    }
    return mine;
}
// the CTA's least and largest pattern; one barrier
template <int NT>
__device__ __forceinline__ void range_of(HeldShared<NT>& S, uint32_t& umin, uint32_t& umax) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    umin = __reduce_min_sync(0xffffffffu, umin);
    umax = __reduce_max_sync(0xffffffffu, umax);
    if (lane == 0) { S.wmin[warp] = umin; S.wmax[warp] = umax; }
    __syncthreads();
    umin = __reduce_min_sync(0xffffffffu, S.wmin[lane % (NT / 32)]);
    umax = __reduce_max_sync(0xffffffffu, S.wmax[lane % (NT / 32)]);
}
// The need-th largest of the first `count` candidates. One barrier behind their last write is the caller's.
template <int NT>
__device__ __forceinline__ unsigned long long rank_candidates(HeldShared<NT>& S, int count, int need) {
    const int tid = threadIdx.x;
    for (int i = tid; i < count; i += NT) {
        const unsigned long long k = S.cand[i];
        int before = 0;
        for (int e = 0; e < count; ++e) before += S.cand[e] > k;
        if (before == need - 1) S.found = k;
    }
    __syncthreads();
    return S.found;
}

// The need-th (from 1) of the order keys in [base, base + nbins << s), of which there are `count`. each(f): f(order key) for the thread's keys, others among them.
// Called behind a barrier after the last use of part, bin, need and count.
template <int NT, typename Each>
__device__ __forceinline__ unsigned long long find_weakest(HeldShared<NT>& S, Each&& each, unsigned long long base, int s, int nbins, int count, int need) {
    const int tid = threadIdx.x;
    while (count > kRank) {
        each([&](unsigned long long x) {
            const unsigned long long bin = (x - base) >> s;
            if (x >= base && bin < (unsigned long long)nbins) atomicAdd(&S.hist[bin], 1);
        });
        __syncthreads();
        int excl, c[kBins / NT], bin, before, in_bin;
        scan_bins<NT>(S, S.hist, excl, c);
        if (bin_of<NT>(need, excl, c, bin, before, in_bin)) { S.bin[0] = bin; S.need = need - before; S.count = in_bin; }
        __syncthreads();
        base += (unsigned long long)S.bin[0] << s;
        need = S.need;
        count = S.count;
        const int narrower = max(0, s - 10);
        nbins = 1 << (s - narrower);
        s = narrower;
        __syncthreads();
    }
    each([&](unsigned long long x) {
        if (x >= base && (x - base) >> s < (unsigned long long)nbins) {
            const int at = atomicAdd(&S.ncand, 1);
            if (at < kRank) S.cand[at] = x;
        }
    });
    __syncthreads();
    return rank_candidates<NT>(S, count, need);
}

template <int NT, bool kCluster>
__global__ void __launch_bounds__(NT, 1024 / NT) select_kernel(Rows R, int rows, int w, unsigned long long* weakest, Plan P) {
    extern __shared__ __align__(16) uint8_t select_smem[];
    SelectShared<NT, kCluster>& S = *reinterpret_cast<SelectShared<NT, kCluster>*>(select_smem);
    constexpr int kSample = kPer * NT, kWarps = NT / 32, kOwn = own_slots(NT);
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nrank = kCluster ? (int)cluster.num_blocks() : 1, rank = kCluster ? (int)cluster.block_rank() : 0;
    for (int i = tid; i < kBins; i += NT) S.hist[i] = 0;
    if (tid == 0) { S.ncand = S.nmore = 0; S.bin[0] = S.bin[1] = -1; }
    pdl_enter(R.table, R.seq, R.pos, R.delta, weakest, P.ustart, P.tickets);
    int item = blockIdx.x / nrank;
    if (P.ustart && item-- == 0) {
        if (rank == 0) make_plan<NT>(R, rows, P);
        return;
    }
    const int t = item / R.Hq, h = item % R.Hq;
    int r;
    const int n = R.visible(t, r);
    if (n <= w) {                                                 // every key
        if (tid == 0 && rank == 0) weakest[item] = 0ull;
        return;
    }
    const int32_t* pages = R.table + r * R.ld;
    const float* plane = R.delta + ((size_t)h << R.page_log);
    const int stride = R.Hq << R.page_log;                        // floats between pages (checked: a page's weights are fewer than 2^31)
    // sample (by every CTA of a cluster, the same one)
    uint32_t lo = 0u, hi = 0x7FFFFFFFu;
    bool collect;
    {
        uint32_t u[kPer], umin = 0x7FFFFFFFu, umax = 0u;
        // four neighbours from each of kSample / 4 scattered places (single keys take four times the sectors, which were the larger part of what the kernel waited for)
        const bool whole = n <= kSample;
        const uint32_t quads = (uint32_t)n / 4;
        uint32_t at[kPer / 4];
        int pg[kPer / 4];
#pragma unroll
        for (int k = 0; k < kPer / 4; ++k) {
            const uint32_t i = k * NT + tid;
            at[k] = 4 * (whole ? i : sample_quad(i, quads, kSample / 4));
            pg[k] = at[k] < (uint32_t)n ? pages[at[k] >> R.page_log] : -1;
        }
#pragma unroll
        for (int k = 0; k < kPer / 4; ++k) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if ((unsigned)pg[k] < (unsigned)R.num_pages) v = *reinterpret_cast<const uint4*>(plane + (size_t)pg[k] * stride + (at[k] & (uint32_t)R.mask()));
            const uint32_t four[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) u[4 * k + e] = at[k] + e < (uint32_t)n ? four[e] & 0x7FFFFFFFu : 0xFFFFFFFFu;
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (u[k] != 0xFFFFFFFFu) { umin = min(umin, u[k]); umax = max(umax, u[k]); }
        range_of<NT>(S, umin, umax);
        const int shift = shift_of(umax - umin);
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (u[k] != 0xFFFFFFFFu) atomicAdd(&S.hist[(u[k] - umin) >> shift], 1);
        __syncthreads();
        int excl, c[kBins / NT];
        scan_bins<NT>(S, S.hist, excl, c);
        const float mid = (float)w / (float)n * kSample, dev = bracket(n, w, kSample);
        const int r0 = whole ? w : (int)(mid - dev), r1 = whole ? w : (int)(mid + dev) + 1;
        int bin, before, count;
        if (bin_of<NT>(r0, excl, c, bin, before, count)) S.bin[0] = bin;
        if (bin_of<NT>(r1, excl, c, bin, before, count)) S.bin[1] = bin;
        __syncthreads();
        // (where the slots do not take what lies inside, the bracket's bins are counted first)
        collect = whole || collects(n, dev, NT, kSample, nrank);
        // (a rank beyond the sample: no bracket on that side)
        if (S.bin[0] >= 0 && r0 >= 1) hi = min(umin + ((uint32_t)(S.bin[0] + 1) << shift) - 1u, 0x7FFFFFFFu);
        if (S.bin[1] >= 0) lo = umin + ((uint32_t)S.bin[1] << shift);
    }
    // f(patterns, index of the first) for four neighbouring keys of a page per thread and step; keys beyond the row read as `beyond`
    const int chunks = (n + 3) / 4;
    auto sweep = [&](uint32_t beyond, auto&& f) {
        constexpr int kAhead = 4;
        int page[kAhead];
        auto pages_at = [&](int i0) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = i0 + k * NT + tid;
                page[k] = i < chunks ? pages[(4 * i) >> R.page_log] : -1;
            }
        };
        const int step = NT * kAhead * nrank;
        pages_at(rank * NT * kAhead);
        for (int i0 = rank * NT * kAhead; i0 < chunks; i0 += step) {
            uint4 u[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                u[k] = make_uint4(0u, 0u, 0u, 0u);
                if ((unsigned)page[k] < (unsigned)R.num_pages) u[k] = *reinterpret_cast<const uint4*>(plane + (size_t)page[k] * stride + (4 * (i0 + k * NT + tid) & R.mask()));
            }
            pages_at(i0 + step);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int j = 4 * (i0 + k * NT + tid);
                uint32_t v[4] = {u[k].x & 0x7FFFFFFFu, u[k].y & 0x7FFFFFFFu, u[k].z & 0x7FFFFFFFu, u[k].w & 0x7FFFFFFFu};
                if (j + 4 > n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j + e >= n) v[e] = beyond;
                }
                f(v, j);
            }
        }
    };
    uint2* own;
    int need, nmore, count, shift;
    unsigned long long found;
    int* bins = S.hist;                                           // of the whole row, after a merge
    auto merge = [&]() {
        if (nrank == 1) {
            __syncthreads();
            return;
        }
        bins = S.sum;
        cluster.sync();
        for (int i = tid; i < kBins; i += NT) {
            int all = 0;
            for (int q = 0; q < nrank; ++q) all += cluster.map_shared_rank(S.hist, q)[i];
            S.sum[i] = all;
        }
        cluster.sync();
        for (int i = tid; i < kBins; i += NT) S.hist[i] = 0;
        __syncthreads();
    };
    // the bin that holds the need-th: where it begins, its keys, and the rank in it
    auto narrow = [&](uint32_t& from) {
        int excl, c[kBins / NT], bin, before, in_bin;
        scan_bins<NT>(S, bins, excl, c);
        if (bin_of<NT>(need, excl, c, bin, before, in_bin)) { S.bin[0] = bin; S.need = need - before; S.count = in_bin; }
        __syncthreads();
        from += (uint32_t)S.bin[0] << shift;
        need = S.need;
        count = S.count;
        __syncthreads();
    };
    // Many equal weights, of which the first by index are kept: bins over n - 1 - index, two sweeps for a million keys.
    auto by_index = [&](uint32_t pattern) {
        uint32_t from = 0u, nbins = kBins;
        for (shift = shift_of((uint32_t)n - 1u);;) {
            sweep(pattern ^ 1u, [&](const uint32_t (&v)[4], int j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bin = ((uint32_t)(n - 1 - j - e) - from) >> shift;
                    if (v[e] == pattern && bin < nbins) atomicAdd(&S.hist[bin], 1);
                }
            });
            merge();
            narrow(from);
            if (shift == 0) return n - 1 - (int)from;
            const int narrower = max(0, shift - 10);
            nbins = 1u << (shift - narrower);
            shift = narrower;
        }
    };
    for (int turn = 0;; ++turn) {
        // One sweep: what lies below the bracket is counted by the sign of its distance; what lies inside goes into bins, or is noted by predicated stores, without a branch
        // per key (with a branch and two comparisons per key, the sweep was 50 of the 62 instructions that 32 keys took).
        if (turn == 16) {                                         // (five narrow any row to one pattern: weights that change under the call)
            if (nrank > 1) cluster.sync();
            found = order_key(lo, INT32_MAX);
            if (rank != 0) return;
            break;
        }
        uint32_t below = 0u, seen = 0u;
        int in = 0;
        own = S.own + tid;
        uint2* const own_end = own + (kOwn - 4) * NT;
        const uint32_t width = hi - lo, beyond = lo > 0u ? 0u : 0xFFFFFFFFu;      // (below the bracket, wherever that is)
        shift = shift_of(width);
        if (collect) {
            sweep(beyond, [&](const uint32_t (&v)[4], int j) {
                seen += 4;
                if (own <= own_end) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t d = v[e] - lo;
                        below += d >> 31;
                        if (d <= width) { *own = make_uint2(v[e], (uint32_t)(j + e)); own += NT; }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t d = v[e] - lo;
                        below += d >> 31;
                        if (d <= width) {
                            const int at = atomicAdd(&S.nmore, 1);
                            if (at < kShared) S.more[at] = make_uint2(v[e], (uint32_t)(j + e));
                            ++in;
                        }
                    }
                }
            });
            in += (int)(own - (S.own + tid)) / NT;
        } else {
            sweep(beyond, [&](const uint32_t (&v)[4], int) {
                seen += 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t d = v[e] - lo;
                    below += d >> 31;
                    if (d <= width) { atomicAdd(&S.hist[d >> shift], 1); ++in; }
                }
            });
        }
        const int sum_above = __reduce_add_sync(0xffffffffu, (int)(seen - below) - in), sum_in = __reduce_add_sync(0xffffffffu, in);
        if (lane == 0) { S.above[warp] = sum_above; S.part[warp] = sum_in; }
        __syncthreads();
        int inside = __reduce_add_sync(0xffffffffu, lane < kWarps ? S.part[lane] : 0), above = __reduce_add_sync(0xffffffffu, lane < kWarps ? S.above[lane] : 0);
        nmore = S.nmore;
        bool over = nmore > kShared;
        if (nrank > 1) {
            int* mine = S.total[turn & 1];
            if (tid == 0) { mine[0] = above; mine[1] = inside; mine[2] = over; }
            cluster.sync();
            above = inside = 0;
            for (int q = 0; q < nrank; ++q) {
                const int* x = cluster.map_shared_rank(mine, q);
                above += x[0];
                inside += x[1];
                over = over || x[2];
            }
        }
        __syncthreads();                                          // (part, above and nmore have been read)
        need = w - above;
        if (need < 1 || need > inside) {                          // the bracket missed: the part of the row beside it, by bins
            if (!collect)
                for (int i = tid; i < kBins; i += NT) S.hist[i] = 0;
            if (need < 1) { lo = hi + 1u; hi = 0x7FFFFFFFu; } else { hi = lo - 1u; lo = 0u; }
            if (tid == 0) S.nmore = 0;
            collect = false;
            __syncthreads();
            continue;
        }
        if (lo == hi && (!collect || over)) {                     // equal weights
            if (nrank > 1) cluster.sync();                        // (no CTA leaves while another may still read its totals)
            if (!collect) {                                       // (counted into the first bin)
                if (tid == 0) S.hist[0] = 0;
                __syncthreads();
            }
            found = order_key(lo, inside == n ? need - 1 : by_index(lo));
            if (rank != 0) return;
            break;
        }
        if (!collect) {                                           // the threshold's bin is the new bracket
            merge();
            narrow(lo);
            hi = min(hi, lo + ((1u << shift) - 1u));
            collect = lo == hi ? false : (int64_t)count <= (int64_t)(kOwn - 4) * NT * nrank / 2;
            if (lo == hi && count <= kRank) collect = true;
            continue;
        }
        if (over) {                                               // too many (weights that crowd): by bins
            if (tid == 0) S.nmore = 0;
            collect = false;
            __syncthreads();
            continue;
        }
        // the keys inside: the bin that holds the need-th, then its order keys
        auto inside_keys = [&](auto&& f) {
            for (uint2* x = S.own + tid; x < own; x += NT) f(*x);
            for (int i = tid; i < nmore; i += NT) f(S.more[i]);
        };
        inside_keys([&](uint2 x) { atomicAdd(&S.hist[(x.x - lo) >> shift], 1); });
        merge();
        narrow(lo);
        if (nrank == 1) {
            found = find_weakest<NT>(S, [&](auto&& f) {
                inside_keys([&](uint2 x) { if ((x.x - lo) >> shift == 0u) f(order_key(x.x, (int)x.y)); });
            }, (unsigned long long)lo << 32, 32 + shift - 10, 1 << 10, count, need);
            break;
        }
        if (count <= kRank) {                                     // they meet in the first CTA
            SelectShared<NT, kCluster>* first = cluster.map_shared_rank(&S, 0);
            inside_keys([&](uint2 x) { if ((x.x - lo) >> shift == 0u) first->cand[atomicAdd(&first->ncand, 1)] = order_key(x.x, (int)x.y); });
            cluster.sync();
            if (rank != 0) return;
            found = rank_candidates<NT>(S, count, need);
            break;
        }
        hi = min(hi, lo + ((1u << shift) - 1u));                  // a bin that holds many: swept again
        if (tid == 0) S.nmore = 0;
        collect = false;
        __syncthreads();
    }
    if (tid == 0) weakest[item] = threshold(found);
}

// The same for rows that the registers hold: NT threads with kKeys keys each. The row is read in one go, a
// histogram of all its keys over their range finds the threshold's bin, and that bin is ranked: a third of the sample's and the sweep's instructions, and fewer
// barriers and round trips, which is what counts for few rows.
template <int NT, int kKeys>
__global__ void __launch_bounds__(NT, 1024 / NT) select_held_kernel(Rows R, int rows, int w, unsigned long long* weakest, Plan P) {
    static_assert(NT <= kBins, "a thread has a bin at least");
    extern __shared__ __align__(16) uint8_t select_smem[];
    HeldShared<NT>& S = *reinterpret_cast<HeldShared<NT>*>(select_smem);
    const int tid = threadIdx.x;
    for (int i = tid; i < kBins; i += NT) S.hist[i] = 0;
    if (tid == 0) S.ncand = 0;
    pdl_enter(R.table, R.seq, R.pos, R.delta, weakest, P.ustart, P.tickets);
    int item = blockIdx.x;
    if (P.ustart && item-- == 0) {
        make_plan<NT>(R, rows, P);
        return;
    }
    const int t = item / R.Hq, h = item % R.Hq;
    int r;
    const int n = R.visible(t, r);
    if (n <= w) {                                                 // every key
        if (tid == 0) weakest[item] = 0ull;
        return;
    }
    const int32_t* pages = R.table + r * R.ld;
    const float* plane = R.delta + ((size_t)h << R.page_log);
    const int stride = R.Hq << R.page_log;
    auto index = [&](int k) { return 4 * ((k >> 2) * NT + tid) + (k & 3); };
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    constexpr int kTogether = kKeys < 16 ? kKeys : 16;            // keys of a thread on their way at a time
    uint32_t u[kKeys], umin = 0x7FFFFFFFu, umax = 0u;
#pragma unroll
    for (int k0 = 0; k0 < kKeys; k0 += kTogether) {
        int page[kTogether / 4];
#pragma unroll
        for (int k = 0; k < kTogether / 4; ++k) page[k] = index(k0 + 4 * k) < n ? pages[index(k0 + 4 * k) >> R.page_log] : -1;
#pragma unroll
        for (int k = 0; k < kTogether; k += 4) {
            const int j = index(k0 + k), pg = page[k / 4];
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if ((unsigned)pg < (unsigned)R.num_pages) v = *reinterpret_cast<const uint4*>(plane + (size_t)pg * stride + (j & R.mask()));
            u[k0 + k] = j < n ? v.x & 0x7FFFFFFFu : kNone;
            u[k0 + k + 1] = j + 1 < n ? v.y & 0x7FFFFFFFu : kNone;
            u[k0 + k + 2] = j + 2 < n ? v.z & 0x7FFFFFFFu : kNone;
            u[k0 + k + 3] = j + 3 < n ? v.w & 0x7FFFFFFFu : kNone;
        }
    }
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        umin = min(umin, u[k]);                                   // (kNone: no minimum, and as an int no maximum)
        umax = (uint32_t)max((int)umax, (int)u[k]);
    }
    range_of<NT>(S, umin, umax);                                  // (its barrier: the histogram is zero)
    // the bin that holds the need-th, then, while it holds many keys of several patterns, the bins of its own range
    uint32_t lo = umin, nbins = kBins, pattern = 0u;
    int shift = shift_of(umax - umin), need = w, count;
    bool by_index = false;                                        // keys of one pattern, of which the first by index are kept: u holds n - 1 - index
    for (;;) {
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            const uint32_t bin = (u[k] - lo) >> shift;            // (kNone: beyond the bins, since its distance to any key is 2^31 at least)
            if (bin < nbins) atomicAdd(&S.hist[bin], 1);
        }
        int excl, c[kBins / NT], bin, before, in_bin;
        __syncthreads();
        scan_bins<NT>(S, S.hist, excl, c);
        if (bin_of<NT>(need, excl, c, bin, before, in_bin)) { S.bin[0] = bin; S.need = need - before; S.count = in_bin; }
        __syncthreads();
        lo += (uint32_t)S.bin[0] << shift;
        need = S.need;
        count = S.count;
        if (count <= kRank) break;
        if (shift == 0) {                                         // equal weights
            by_index = true;
            pattern = lo;
#pragma unroll
            for (int k = 0; k < kKeys; ++k) u[k] = u[k] == pattern ? (uint32_t)(n - 1 - index(k)) : kNone;
            lo = 0u;
            nbins = kBins;
            shift = shift_of((uint32_t)n - 1u);
        } else {
            const int narrower = max(0, shift - 10);
            nbins = 1u << (shift - narrower);
            shift = narrower;
        }
        __syncthreads();                                          // (bin, need and count have been read)
    }
#pragma unroll
    for (int k = 0; k < kKeys; ++k)
        if ((u[k] - lo) >> shift == 0u) S.cand[atomicAdd(&S.ncand, 1)] = order_key(by_index ? pattern : u[k], index(k));
    __syncthreads();
    const unsigned long long found = rank_candidates<NT>(S, count, need);
    if (tid == 0) weakest[item] = threshold(found);
}

int select_launch(void (*kernel)(Rows, int, int, unsigned long long*, Plan), int threads, size_t bytes, int cluster, const Cache& C, const Rows& R,
                  unsigned long long* weakest, const Plan& plan, cudaStream_t st) {
    if (bytes > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(kernel, dim3((unsigned)(((int64_t)C.rows * C.Hq + (plan.ustart ? 1 : 0)) * cluster)), dim3(threads), bytes, st, cluster, R, C.rows, C.w, weakest, plan);
}
}  // namespace

// The form by the table's capacity, which bounds the rows' lengths (and with w their brackets), and by the number of (row, head) items. us of one form and of
// the next, 32 heads, rows of the capacity, w a quarter of it:
//   up to 2K     held by 256 threads; by 1024 for 13 rows 4.5 against 9.2, for one row 3.7 against 3.9
//   up to 4K     held by 1024 threads where every item has an SM (4 rows 4.1; by 256 4.7), else by 256 (5 rows 4.8 against 6.2; 13 rows 6.6 against 11.5)
//   up to 16K    held by 1024 threads where two items per SM are all (one row of 16K 6.3; swept 7.8. 9 rows 13.6 against 14.0; 10 rows 17.7 against 17.1)
//   beyond       swept: by 256 threads where there are many items and the bracket fits their slots (64 rows of 16K 57; by 512 70), else by 512 (64 rows of 32K 108 against 144), whose
//                cluster is as large as the bracket needs (9 rows of 256K, w = 8192: two CTAs 92, one, which sweeps twice, 133; 32 of 128K, w = 32K: 208 against 267). Where no cluster's slots would do, or a
//                grid does not take so many clusters, 256 threads again (64 rows of 64K, two sweeps 264 against 281).
//                Few rows take larger clusters: of 16K keys per CTA where an SM has one (one row of 64K: four CTAs 12.5, two 14.0, eight 16.6), of 32K where it has two (2 rows of 128K:
//                four 22.7, two 24.6; 4 rows of 32K: two 18.8, one 14.5; one row of 256K: eight 24.6, two 36).
int launch_cache4_select(const Cache& C, const Rows& R, unsigned long long* weakest, const Plan& plan, cudaStream_t st) {
    constexpr int K = 1024, kSms = 148;
    const int capacity = C.max_blocks << C.page_log;
    const int64_t items = (int64_t)C.rows * C.Hq;
    auto held = [&](auto nt, auto kernel) { return select_launch(kernel, nt, sizeof(HeldShared<nt>), 1, C, R, weakest, plan, st); };
    constexpr std::integral_constant<int, 256> t256{};
    constexpr std::integral_constant<int, 1024> t1024{};
    if (capacity <= 2 * K) return held(t256, select_held_kernel<256, 8>);
    if (capacity <= 4 * K) return items <= kSms ? held(t1024, select_held_kernel<1024, 4>) : held(t256, select_held_kernel<256, 16>);
    const bool few = items <= 2 * kSms;
    if (few && capacity <= 8 * K) return held(t1024, select_held_kernel<1024, 8>);
    if (few && capacity <= 16 * K) return held(t1024, select_held_kernel<1024, 16>);
    auto fits = [&](int threads, int ctas) { return collects(capacity, bracket(capacity, C.w, kPer * threads), threads, kPer * threads, ctas); };
    int cluster = 1;
    while (cluster < 8 && !fits(512, cluster)) cluster *= 2;
    const bool one_sweep = fits(512, cluster) && (items + 1) * cluster <= INT32_MAX;       // (what a grid takes)
    if (!few && (fits(256, 1) || !one_sweep)) return select_launch(select_kernel<256, false>, 256, sizeof(SelectShared<256, false>), 1, C, R, weakest, plan, st);
    while (cluster < 8 && items * cluster * 2 <= 2 * kSms && capacity / (2 * cluster) >= (items * cluster * 2 <= kSms ? 16 : 32) * K) cluster *= 2;
    if (cluster == 1) return select_launch(select_kernel<512, false>, 512, sizeof(SelectShared<512, false>), 1, C, R, weakest, plan, st);
    return select_launch(select_kernel<512, true>, 512, sizeof(SelectShared<512, true>), cluster, C, R, weakest, plan, st);
}

int launch_cache4_plan(const Cache& C, const Rows& R, const Plan& plan, cudaStream_t st) {
    return launch_overlapped(plan_kernel, dim3(1), dim3(1024), 0, st, 1, R, C.rows, plan);
}

}  // namespace dma
