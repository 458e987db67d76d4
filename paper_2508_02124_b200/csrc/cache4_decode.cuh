// What the selection and the attention of dma_cache4_decode share: the rows' keys, their order, and how the attention's work is cut.
#pragma once

#include "paged.cuh"

namespace dma {

// (delta descending, index ascending) as one unsigned compare; delta > 0, so its pattern orders like its value. The sign is masked, and keys in
// pages outside the pool count as 0: behind all others.
__device__ __forceinline__ unsigned long long order_key(uint32_t u, int j) { return (unsigned long long)u << 32 | (0xFFFFFFFFu - (uint32_t)j); }

// What a kernel needs to find its row's keys.
struct Rows {
    const int32_t *table, *seq, *pos;
    const float* delta;
    int64_t ld;
    int nseq, page_log, num_pages, max_blocks, Hq;
    __device__ __forceinline__ int mask() const { return (1 << page_log) - 1; }
    // keys that row t sees; -1: padding, the row is left as it is
    __device__ __forceinline__ int visible(int t, int& r) const {
        r = seq[t];
        if ((unsigned)r >= (unsigned)nseq) return -1;
        return min(max(pos[t], -1), (max_blocks << page_log) - 1) + 1;
    }
};

// What every row's attention is cut by: units of about the same work, dealt out to the CTAs in equal shares. ustart[t]: units before row t, over all its
// `per_row` items. A key costs its test, and its expansion where some head of the group keeps it; the heads' kept keys are taken to be independent.
// (By keys alone, rows that keep all theirs took up to twice a long row's time.)
struct Plan { int32_t* ustart; int32_t* tickets; int per_row, unit_log, heads, w; };

// weakest[rows * Hq]: the order key of every (row, query head)'s weakest kept key, 0 where it keeps all. The plan, where it has arrays, is made on the way.
int launch_cache4_select(const Cache& C, const Rows& R, unsigned long long* weakest, const Plan& plan, cudaStream_t st);
int launch_cache4_plan(const Cache& C, const Rows& R, const Plan& plan, cudaStream_t st);

}  // namespace dma
