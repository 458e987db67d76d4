// What the kernels of dma_cache_decode share: a row's own keys, the prefixes' orders, the rows grouped by prefix, pieces of a row's attention.
#pragma once

#include "paged.cuh"

namespace dma {

struct DecodeArgs {
    const void *q, *kv;
    const float* delta;
    const int32_t *table, *seq, *pos, *prefix;
    const int32_t *order_slot, *order_len;
    const float* order_weight;
    void* o;
    float* lse;
    int64_t ld, order_ld, qs_row, qs_head, os_row, os_head;
    float scale;
    int rows, nseq, nprefix, Hq, Hkv, G, w, page_log, num_pages, max_blocks;
    // workspace
    int32_t* status;
    int* cut;                    // [rows * Hq]: entries of its prefix' order that a row's head keeps
    unsigned long long* least;   // [rows * Hq]: the order key of the weakest own key that it keeps, or one between that and the next
    float* piece;                // [rows * Hq][pieces][D + 2]: maximum, sum and weighted values of a part of the keys; the first piece: own keys
    int pieces;
    int *first, *members;        // [nprefix + 1]: scratch; [tiles * tile_rows]: the rows of each tile
    int4* tiles;                 // (prefix, rows of it, listed keys, -)
    int* ntiles;
    int tile_rows;
    // keys that row t sees of its own sequence; -1: the row is left as it is
    __device__ __forceinline__ int own(int t, int& r) const {
        r = seq[t];
        if ((unsigned)r >= (unsigned)nseq) return -1;
        return min(max(pos[t], -1), (max_blocks << page_log) - 1) + 1;
    }
    // the row's prefix, -1 where it has none, and how many of its keys are listed
    __device__ __forceinline__ int listed(int t, int& n) const {
        n = 0;
        if (nprefix == 0) return -1;
        const int g = prefix[t];
        if ((unsigned)g >= (unsigned)nprefix) return -1;
        n = (int)max((int64_t)0, min((int64_t)min(order_len[g], w), order_ld));
        return n > 0 ? g : -1;
    }
    __device__ __forceinline__ float* piece_of(int t, int h, int i, int d) const { return piece + ((size_t)(t * Hq + h) * pieces + i) * (d + 2); }
};

__device__ __forceinline__ void team_sync(int id, int threads) {
    if (threads > 32) asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
    else __syncwarp();
}

// What a CTA of the rows' own keys works on: the heads head0 .. head1 - 1 of a (row, KV head), `heads` of them, or all, per CTA.
struct OwnRow {
    int t, hk, head0, head1, n, listed;
    const int32_t* pages;
    // false: the row is left as it is. The loads that do not depend on each other go out together.
    __device__ __forceinline__ bool find(const DecodeArgs& A, int cta, int heads) {
        const int parts = (A.G + heads - 1) / heads;
        t = cta / (A.Hkv * parts);
        hk = cta / parts % A.Hkv;
        head0 = cta % parts * heads;
        head1 = min(A.G, head0 + heads);
        const int r = A.seq[t], p = A.pos[t], g = A.nprefix ? A.prefix[t] : -1;
        if ((unsigned)r >= (unsigned)A.nseq) return false;
        n = min(max(p, -1), (A.max_blocks << A.page_log) - 1) + 1;
        pages = A.table + r * A.ld;
        listed = 0;
        if ((unsigned)g < (unsigned)A.nprefix) listed = (int)max((int64_t)0, min((int64_t)min(A.order_len[g], A.w), A.order_ld));
        return true;
    }
    // all keys are kept, whatever their weights
    __device__ __forceinline__ bool keeps_all(const DecodeArgs& A) const { return (int64_t)listed + n <= A.w; }
};

// f(position, slot, patterns) for a head's own keys j0 .. j1 - 1 (j0 a multiple of 16), 512 at a time: a lane has 16 of them, side by side in one page (pages have 16 keys and more).
// Patterns of places without a key: -2
template <typename F>
__device__ __forceinline__ void sweep_own(const DecodeArgs& A, const OwnRow& R, int h, int j0, int j1, F f) {
    const int lane = threadIdx.x & 31, mask = (1 << A.page_log) - 1;
    auto page_of = [&](int j) { return j < j1 ? R.pages[j >> A.page_log] : -1; };
    int next = page_of(j0 + 16 * lane);
#pragma unroll 1
    for (int b = j0; b < j1; b += 512) {
        const int j = b + 16 * lane, page = next, slot = (page << A.page_log) + (j & mask);
        const bool there = (unsigned)page < (unsigned)A.num_pages;
        int u[16];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            int4 x = make_int4(-2, -2, -2, -2);
            if (there) x = *reinterpret_cast<const int4*>(A.delta + (((size_t)page * A.Hq + h) << A.page_log) + (j & mask) + i);
            u[i] = x.x; u[i + 1] = x.y; u[i + 2] = x.z; u[i + 3] = x.w;
        }
        next = page_of(j + 512);
        if (b + 512 > j1)
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = j + i < j1 ? u[i] : -2;
        f(j, slot, u);
    }
}

// Warps of a row's heads: one per head of a group, eight at most; teams of them, and fewer heads per CTA, where all make fewer than `fill` per SM or where a team would have more than `most` keys per warp.
struct Teams {
    int heads, team, warps;      // of a CTA: heads (or all, in turn), warps per head, warps
    int64_t ctas;
    Teams(const Cache& C, int fill, int64_t most) {
        const int64_t capacity = (int64_t)C.max_blocks << C.page_log;
        heads = team = 1;
        while (heads < C.G && heads < 8) heads *= 2;
        const int all = heads;
        auto count = [&](int per) { return (int64_t)C.rows * C.Hkv * (per == all ? 1 : (C.G + per - 1) / per); };
        while (team < 8 && (count(heads) * heads * team * 2 <= fill * 148 || capacity > most * team)) {
            team *= 2;
            if (heads * team > 8) heads /= 2;
        }
        warps = heads * team;
        ctas = count(heads);
        if (heads == all) heads = C.G;
    }
};

// What each row keeps, of its prefix and of its own keys; the rows grouped by prefix.
int launch_cuts(const Cache& C, const DecodeArgs& A, cudaStream_t st);
// Attention over the rows' own keys: the row's results where it has no prefix, else its first piece. The next kernel may start beside it.
int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st);
// Attention over the prefixes and the sum of the pieces; on the tensor cores tiles of 128 rows and one piece
int launch_prefix_simt(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st);
int launch_prefix_tc(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st);

}  // namespace dma
