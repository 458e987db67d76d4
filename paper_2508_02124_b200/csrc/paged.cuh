// The paged caches (include/dma.h, dma_cache_t): resolved descriptor, launchers, addressing of pages and slots.
#pragma once

#include "common.cuh"

namespace dma {

constexpr int kGroup = 64;             // channels that share a scale and a zero

// query heads of a group that dma_cache4_append takes: their sampling weights and z lie in 48 KB of shared memory
constexpr int append_heads(int d) { return d == 128 ? 76 : 96; }

// dma_cache_t with defaults resolved
struct Cache {
    int Hq, Hkv, G, d, w, dtype, flags;
    int page_size, page_log, num_pages, max_blocks, nseq, rows;
    float scale;
    int64_t table_ld;
    int64_t qs[2], ks[2], vs[2], os[2];       // row and head strides in elements
};

int resolve_pages(const dma_cache_t* c, Cache* out);       // pages, sequences and rows only
int resolve_cache(const dma_cache_t* c, Cache* out);       // all of it

int launch_page_plan(const Cache& C, const int32_t* lens, const int32_t* want, int32_t* table, int32_t* ring, const int32_t* pool, int32_t* lens_out,
                     int32_t* pool_out, int32_t* cu, int32_t* row_seq, int32_t* row_pos, int32_t* slot, cudaStream_t st);
int launch_cache4_append(const Cache& C, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld,
                         const int32_t* slot, uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st);
int launch_cache4_read(const Cache& C, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* slot, void* K, void* V,
                       float* delta_out, int64_t delta_ld, cudaStream_t st);
size_t cache4_decode_ws_bytes(const Cache& C);
int launch_cache4_decode(const Cache& C, const void* q, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* table,
                         const int32_t* row_seq, const int32_t* row_pos, void* o, float* lse, void* ws, cudaStream_t st);

// dma_rotation_t with defaults resolved; no frequencies: nothing is rotated
struct Rotation {
    const float* inv_freq;
    int rot, interleaved;
    float scale;
};
int launch_cache_append(const Cache& C, const Rotation& rot, const void* q, const void* K, const void* V, const float* W, const float* A, const float* delta_new,
                        int64_t delta_ld, const int32_t* slot, const int32_t* pos, const int32_t* prefix, const int32_t* prefix_len, int nprefix, void* q_out, void* kv,
                        float* delta, cudaStream_t st);
size_t prefix_order_ws_bytes(const Cache& C);              // of C.nseq prefixes
int launch_prefix_order(const Cache& C, const float* delta, const int32_t* table, const int32_t* len, int32_t* slot, float* weight, int64_t order_ld, int32_t* order_len,
                        void* ws, cudaStream_t st);
size_t cache_decode_ws_bytes(const Cache& C, int nprefix);
int launch_cache_decode(const Cache& C, const void* q, const void* kv, const float* delta, const int32_t* table, const int32_t* row_seq, const int32_t* row_pos,
                        const int32_t* row_prefix, int nprefix, const int32_t* order_slot, const float* order_weight, int64_t order_ld, const int32_t* order_len,
                        void* o, float* lse, void* ws, cudaStream_t st);

// Key rows of the pool: row (page, head, place) of codes takes d bytes (K's codes, V's), of scales 2 d / 64 pairs of bf16; of a cache
// in the element type 2 d elements.
__device__ __forceinline__ size_t key_row(int page, int head, int place, int Hkv, int page_log) {
    return (((size_t)page * Hkv + head) << page_log) + place;
}
// a pair (s, z) as loaded
__device__ __forceinline__ float pair_s(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float pair_z(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

// one of the two is a NaN or an infinity (all ones in the exponent carry into the sign's place)
__device__ __forceinline__ bool odd_pair(uint32_t p) { return (((p & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0u; }

}  // namespace dma
