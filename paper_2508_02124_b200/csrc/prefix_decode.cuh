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

// Attention over the rows' own keys, and what each keeps of its prefix: the row's last part where it has no prefix, else its first piece.
int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st);
// Attention over the prefixes and the sum of the pieces; on the tensor cores tiles of 128 rows and one piece
int launch_prefix_simt(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st);
int launch_prefix_tc(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st);

}  // namespace dma
