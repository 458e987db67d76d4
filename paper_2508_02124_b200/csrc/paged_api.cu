// C-ABI entry points of the paged caches (include/dma.h): argument validation, defaults, dispatch.
#include <algorithm>
#include <cmath>

#include "paged.cuh"

namespace dma {

int resolve_pages(const dma_cache_t* c, Cache* o) {
    if (!c) return DMA_ERR_NULL;
    if (c->rows < 1 || c->nseq < 1 || c->num_pages < 1 || c->max_blocks < 1) return DMA_ERR_SHAPE;
    if (c->nseq > (1 << 30)) return DMA_ERR_SHAPE;                 // (the plan counts them by 1024, in 32 bits)
    int lg = 4;
    while (lg < 8 && (1 << lg) != c->page_size) ++lg;
    if ((1 << lg) != c->page_size) return DMA_ERR_UNSUPPORTED;
    if (((int64_t)c->num_pages << lg) > INT32_MAX || ((int64_t)c->max_blocks << lg) > (1 << 30)) return DMA_ERR_SHAPE;
    if (c->table_ld != 0 && c->table_ld < c->max_blocks) return DMA_ERR_SHAPE;
    o->page_size = c->page_size; o->page_log = lg; o->num_pages = c->num_pages; o->max_blocks = c->max_blocks;
    o->nseq = c->nseq; o->rows = c->rows;
    o->table_ld = c->table_ld ? c->table_ld : c->max_blocks;
    return DMA_OK;
}

static bool row_strides(const int64_t in[2], int64_t out[2], int H, int d) {
    if (in[0] == 0 && in[1] == 0) {
        out[0] = (int64_t)H * d; out[1] = d;
        return true;
    }
    for (int i = 0; i < 2; ++i) {
        if (in[i] <= 0 || in[i] % 8) return false;
        out[i] = in[i];
    }
    return true;
}

int resolve_cache(const dma_cache_t* c, Cache* o) {
    const int rc = resolve_pages(c, o);
    if (rc) return rc;
    if (c->Hq < 1 || c->Hkv < 1 || c->Hq % c->Hkv || c->w < 1) return DMA_ERR_SHAPE;
    if ((int64_t)c->rows * c->Hq > INT32_MAX / 2 || (int64_t)c->Hq * c->page_size > INT32_MAX || c->Hkv > 65535) return DMA_ERR_SHAPE;
    if (c->d != 64 && c->d != 128) return DMA_ERR_UNSUPPORTED;
    if (c->dtype != DMA_BF16 && c->dtype != DMA_FP32) return DMA_ERR_UNSUPPORTED;
    if (c->flags & ~DMA_FLAG_SIMT) return DMA_ERR_UNSUPPORTED;
    if (!(c->softmax_scale >= 0.0f) || std::isinf(c->softmax_scale)) return DMA_ERR_SHAPE;
    o->Hq = c->Hq; o->Hkv = c->Hkv; o->G = c->Hq / c->Hkv; o->d = c->d; o->w = c->w; o->dtype = c->dtype; o->flags = c->flags;
    o->scale = c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->d);
    if (!row_strides(c->q_stride, o->qs, c->Hq, c->d) || !row_strides(c->k_stride, o->ks, c->Hkv, c->d) ||
        !row_strides(c->v_stride, o->vs, c->Hkv, c->d) || !row_strides(c->o_stride, o->os, c->Hq, c->d))
        return DMA_ERR_ALIGN;
    return DMA_OK;
}

template <typename... Ts>
static bool aligned(uintptr_t to, Ts... ptrs) {
    return ((((uintptr_t)ptrs & (to - 1)) == 0) && ...);
}

static int sm100() {
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return DMA_ERR_CUDA;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return DMA_ERR_CUDA;
    return major == 10 ? DMA_OK : DMA_ERR_CUDA;
}

}  // namespace dma

using namespace dma;

extern "C" {

int dma_cache4_bytes(const dma_cache_t* c, size_t* codes, size_t* scales, size_t* delta) {
    Cache C;
    const int rc = resolve_cache(c, &C);
    if (rc) return rc;
    const size_t keys = (size_t)C.num_pages << C.page_log;
    if (codes) *codes = keys * C.Hkv * C.d;
    if (scales) *scales = keys * C.Hkv * (C.d / kGroup) * 8;
    if (delta) *delta = keys * C.Hq * sizeof(float);
    return DMA_OK;
}

int dma_page_plan(const dma_cache_t* c, const int32_t* lens, const int32_t* want, int32_t* block_table, int32_t* free_pages,
                  const int32_t* pool, int32_t* lens_out, int32_t* pool_out, int32_t* cu_rows, int32_t* row_seq, int32_t* row_pos,
                  int32_t* slot, void* cuda_stream) {
    Cache C;
    int rc = resolve_pages(c, &C);
    if (rc) return rc;
    if (!lens || !want || !block_table || !free_pages || !pool || !lens_out || !pool_out || !cu_rows || !row_seq || !row_pos || !slot)
        return DMA_ERR_NULL;
    if (!aligned(4, lens, want, block_table, free_pages, pool, lens_out, pool_out, cu_rows, row_seq, row_pos, slot)) return DMA_ERR_ALIGN;
    if ((rc = sm100())) return rc;
    return launch_page_plan(C, lens, want, block_table, free_pages, pool, lens_out, pool_out, cu_rows, row_seq, row_pos, slot, (cudaStream_t)cuda_stream);
}

int dma_cache4_append(const dma_cache_t* c, const void* K, const void* V, const float* W_delta, const float* A, const float* delta_new,
                      int64_t delta_ld, const int32_t* slot, void* codes, void* scales, float* delta, void* cuda_stream) {
    Cache C;
    int rc = resolve_cache(c, &C);
    if (rc) return rc;
    if (!K || !V || !slot || !codes || !scales || !delta || (!delta_new && (!W_delta || !A))) return DMA_ERR_NULL;
    if (!aligned(16, K, V, W_delta, codes, scales, delta) || !aligned(4, A, delta_new, slot)) return DMA_ERR_ALIGN;
    if (delta_new && delta_ld < C.rows) return DMA_ERR_SHAPE;
    if (C.G > append_heads(C.d)) return DMA_ERR_UNSUPPORTED;
    if ((rc = sm100())) return rc;
    return launch_cache4_append(C, K, V, W_delta, A, delta_new, delta_ld, slot, (uint8_t*)codes, (__nv_bfloat16*)scales, delta, (cudaStream_t)cuda_stream);
}

int dma_cache4_read(const dma_cache_t* c, const void* codes, const void* scales, const float* delta, const int32_t* slot, void* K,
                    void* V, float* delta_out, int64_t delta_ld, void* cuda_stream) {
    Cache C;
    int rc = resolve_cache(c, &C);
    if (rc) return rc;
    if (!codes || !scales || !slot || !K || !V || (delta_out && !delta)) return DMA_ERR_NULL;
    if (!aligned(16, K, V, codes, scales, delta) || !aligned(4, slot, delta_out)) return DMA_ERR_ALIGN;
    if (delta_out && delta_ld < C.rows) return DMA_ERR_SHAPE;
    if ((rc = sm100())) return rc;
    return launch_cache4_read(C, (const uint8_t*)codes, (const __nv_bfloat16*)scales, delta, slot, K, V, delta_out, delta_ld, (cudaStream_t)cuda_stream);
}

int dma_cache4_decode_workspace(const dma_cache_t* c, size_t* bytes) {
    Cache C;
    const int rc = resolve_cache(c, &C);
    if (rc) return rc;
    if (!bytes) return DMA_ERR_NULL;
    *bytes = cache4_decode_ws_bytes(C);
    return DMA_OK;
}

int dma_cache4_decode(const dma_cache_t* c, const void* q, const void* codes, const void* scales, const float* delta,
                      const int32_t* block_table, const int32_t* row_seq, const int32_t* row_pos, void* o, float* lse, void* ws,
                      size_t ws_bytes, void* cuda_stream) {
    Cache C;
    int rc = resolve_cache(c, &C);
    if (rc) return rc;
    if (!q || !codes || !scales || !delta || !block_table || !row_seq || !row_pos || !o || !lse) return DMA_ERR_NULL;
    if (!aligned(16, q, codes, scales, delta, o) || !aligned(4, block_table, row_seq, row_pos, lse)) return DMA_ERR_ALIGN;
    if (!ws || ws_bytes < cache4_decode_ws_bytes(C) || !aligned(16, ws)) return DMA_ERR_WORKSPACE;
    if ((rc = sm100())) return rc;
    return launch_cache4_decode(C, q, (const uint8_t*)codes, (const __nv_bfloat16*)scales, delta, block_table, row_seq, row_pos, o, lse, ws,
                                (cudaStream_t)cuda_stream);
}

int dma_cache_bytes(const dma_cache_t* c, size_t* kv, size_t* delta) {
    Cache C;
    const int rc = resolve_cache(c, &C);
    if (rc) return rc;
    const size_t keys = (size_t)C.num_pages << C.page_log;
    if (kv) *kv = keys * C.Hkv * 2 * C.d * (C.dtype == DMA_BF16 ? 2 : 4);
    if (delta) *delta = keys * C.Hq * sizeof(float);
    return DMA_OK;
}

int dma_cache_append(const dma_cache_t* c, const dma_rotation_t* rotation, const void* q, const void* K, const void* V, const float* W_delta,
                     const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot, const int32_t* row_pos,
                     const int32_t* row_prefix, const int32_t* prefix_len, int32_t nprefix, void* q_out, void* kv, float* delta, void* cuda_stream) {
    Cache C;
    int rc = resolve_cache(c, &C);
    if (rc) return rc;
    if (!K || !V || !slot || !kv || !delta || (!delta_new && (!W_delta || !A)) || (q == nullptr) != (q_out == nullptr)) return DMA_ERR_NULL;
    Rotation rot = {};
    if (nprefix == 0) row_prefix = prefix_len = nullptr;           // (an empty array may have no address)
    if (rotation) {
        if (!rotation->inv_freq || !row_pos || (row_prefix == nullptr) != (prefix_len == nullptr)) return DMA_ERR_NULL;
        if (rotation->rot < 16 || rotation->rot > C.d || nprefix < 0 || !std::isfinite(rotation->scale)) return DMA_ERR_SHAPE;
        if (rotation->rot % 16) return DMA_ERR_UNSUPPORTED;
        rot = {rotation->inv_freq, rotation->rot, rotation->interleaved != 0, rotation->scale != 0.0f ? rotation->scale : 1.0f};
    } else {
        if (q) return DMA_ERR_UNSUPPORTED;
        row_pos = row_prefix = prefix_len = nullptr;
    }
    if (!delta_new && C.G > append_heads(C.d)) return DMA_ERR_UNSUPPORTED;
    if (q && q == q_out && C.rows * C.Hq > 1 && (C.qs[0] != C.os[0] || C.qs[1] != C.os[1])) return DMA_ERR_SHAPE;
    if (!aligned(16, q, K, V, W_delta, q_out, kv, delta) || !aligned(4, A, delta_new, slot, rot.inv_freq, row_pos, row_prefix, prefix_len)) return DMA_ERR_ALIGN;
    if (delta_new && delta_ld < C.rows) return DMA_ERR_SHAPE;
    if ((rc = sm100())) return rc;
    return launch_cache_append(C, rot, q, K, V, W_delta, A, delta_new, delta_ld, slot, row_pos, row_prefix, prefix_len, nprefix, q_out, kv, delta, (cudaStream_t)cuda_stream);
}

// A prefix' list and its sorted chunks are counted in 32 bits.
static int resolve_order(const dma_cache_t* c, Cache* C) {
    const int rc = resolve_cache(c, C);
    if (rc) return rc;
    const int64_t items = (int64_t)C->nseq * C->Hq;
    if (items > INT32_MAX / 2 || items * ((((int64_t)C->max_blocks << C->page_log) + 4095) / 4096) > INT32_MAX) return DMA_ERR_SHAPE;
    return DMA_OK;
}

int dma_prefix_order_workspace(const dma_cache_t* c, size_t* bytes) {
    Cache C;
    const int rc = resolve_order(c, &C);
    if (rc) return rc;
    if (!bytes) return DMA_ERR_NULL;
    *bytes = prefix_order_ws_bytes(C);
    return DMA_OK;
}

int dma_prefix_order(const dma_cache_t* c, const float* delta, const int32_t* block_table, const int32_t* prefix_len, int32_t* order_slot,
                     float* order_weight, int64_t order_ld, int32_t* order_len, void* ws, size_t ws_bytes, void* cuda_stream) {
    Cache C;
    int rc = resolve_order(c, &C);
    if (rc) return rc;
    if (!delta || !block_table || !prefix_len || !order_slot || !order_weight || !order_len) return DMA_ERR_NULL;
    if (!aligned(16, delta) || !aligned(4, block_table, prefix_len, order_slot, order_weight, order_len)) return DMA_ERR_ALIGN;
    if (order_ld < std::min<int64_t>(C.w, (int64_t)C.max_blocks << C.page_log)) return DMA_ERR_SHAPE;
    if (!ws || ws_bytes < prefix_order_ws_bytes(C) || !aligned(16, ws)) return DMA_ERR_WORKSPACE;
    if ((rc = sm100())) return rc;
    return launch_prefix_order(C, delta, block_table, prefix_len, order_slot, order_weight, order_ld, order_len, ws, (cudaStream_t)cuda_stream);
}

// The rows of all tiles, of which there are min(rows, nprefix + rows / 8) at most, are counted in 32 bits.
static int resolve_decode(const dma_cache_t* c, int32_t nprefix, Cache* C) {
    const int rc = resolve_cache(c, C);
    if (rc) return rc;
    if (nprefix < 0 || nprefix > (1 << 30) || std::min<int64_t>(C->rows, (int64_t)nprefix + C->rows / 8) >= (1 << 24)) return DMA_ERR_SHAPE;
    return DMA_OK;
}

int dma_cache_decode_workspace(const dma_cache_t* c, int32_t nprefix, size_t* bytes) {
    Cache C;
    const int rc = resolve_decode(c, nprefix, &C);
    if (rc) return rc;
    if (!bytes) return DMA_ERR_NULL;
    *bytes = cache_decode_ws_bytes(C, nprefix);
    return DMA_OK;
}

int dma_cache_decode(const dma_cache_t* c, const void* q, const void* kv, const float* delta, const int32_t* block_table, const int32_t* row_seq,
                     const int32_t* row_pos, const int32_t* row_prefix, int32_t nprefix, const int32_t* order_slot, const float* order_weight,
                     int64_t order_ld, const int32_t* order_len, void* o, float* lse, void* ws, size_t ws_bytes, void* cuda_stream) {
    Cache C;
    int rc = resolve_decode(c, nprefix, &C);
    if (rc) return rc;
    if (!q || !kv || !delta || !block_table || !row_seq || !row_pos || !o || !lse) return DMA_ERR_NULL;
    if (nprefix > 0 && (!row_prefix || !order_slot || !order_weight || !order_len)) return DMA_ERR_NULL;
    if (!aligned(16, q, kv, delta, o) || !aligned(4, block_table, row_seq, row_pos, lse)) return DMA_ERR_ALIGN;
    if (nprefix > 0 && !aligned(4, row_prefix, order_slot, order_weight, order_len)) return DMA_ERR_ALIGN;
    if (nprefix > 0 && order_ld < 1) return DMA_ERR_SHAPE;
    if (!ws || ws_bytes < cache_decode_ws_bytes(C, nprefix) || !aligned(16, ws)) return DMA_ERR_WORKSPACE;
    if ((rc = sm100())) return rc;
    return launch_cache_decode(C, q, kv, delta, block_table, row_seq, row_pos, row_prefix, nprefix, order_slot, order_weight, order_ld, order_len, o, lse, ws,
                               (cudaStream_t)cuda_stream);
}

}  // extern "C"
