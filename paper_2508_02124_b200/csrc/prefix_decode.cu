// dma_cache_decode (include/dma.h): the calls' launches; the second step on the CUDA cores (fp32, and bf16 on request): the rows of a prefix, eight at a time, over a head's list, which is
// cut into 16 splits; then the sum of the pieces. Three rows behind 250 keys, fp32: 4.7 and 5.1 us, round trips. One row behind 16K keys, w = 2048, 32 heads: 18 and 10; four 24 and 10.
#include <algorithm>

#include "delta_fixed.cuh"
#include "prefix_decode.cuh"

namespace dma {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kKeys = 32, kSplits = 16;

// A CTA per (tile of eight rows, head, split). Keys lie in shared memory as fp32, 32 at a time; a warp has a row: a lane per key for the scores, D / 32 channels per lane for the
// values.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) simt_kernel(DecodeArgs A) {
    constexpr int P = D + 4, C = D / 32;
    __shared__ __align__(16) float sK[kKeys][P], sV[kKeys][D], sQ[kWarps][D];
    __shared__ float sW[kKeys];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, split = blockIdx.y, nsplit = gridDim.y;
    pdl_enter();
    const int tile = blockIdx.x / A.Hq, h = blockIdx.x % A.Hq, hk = h / A.G;
    if (tile >= *A.ntiles) return;
    const int4 rows = A.tiles[tile];
    const bool active = warp < rows.y;
    const int t = A.members[tile * kWarps + min(warp, rows.y - 1)], n = rows.z;
    const int cut = A.cut[t * A.Hq + h], nslots = A.num_pages << A.page_log;
    const int32_t* slot = A.order_slot + ((int64_t)rows.x * A.Hq + h) * A.order_ld;
    const float* weight = A.order_weight + ((int64_t)rows.x * A.Hq + h) * A.order_ld;
    const T *q = (const T*)A.q + t * A.qs_row + h * A.qs_head, *kv = (const T*)A.kv;
    for (int x = lane; x < D; x += 32) sQ[warp][x] = to_f32(q[x]) * A.scale;
    float m = -INFINITY, l = 0.0f, acc[C];
#pragma unroll
    for (int x = 0; x < C; ++x) acc[x] = 0.0f;
    for (int base = split * kKeys; base < n; base += nsplit * kKeys) {
        __syncthreads();
        for (int i = tid; i < kKeys * (D / 8); i += kThreads) {
            const int key = i / (D / 8), c = i % (D / 8) * 8;
            float k[8] = {}, v[8] = {};
            const int at = base + key < n ? slot[base + key] : -1;
            if ((unsigned)at < (unsigned)nslots) {
                const T* row = kv + key_row(at >> A.page_log, hk, at & ((1 << A.page_log) - 1), A.Hkv, A.page_log) * (2 * D) + c;
                load8(row, k);
                load8(row + D, v);
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                sK[key][c + x] = k[x];
                sV[key][c + x] = v[x];
            }
            if (c == 0) sW[key] = (unsigned)at < (unsigned)nslots ? weight[base + key] : -INFINITY;
        }
        __syncthreads();
        if (!active) continue;
        float s = 0.0f;
#pragma unroll 4
        for (int x = 0; x < D; x += 4) {
            const float4 a = *reinterpret_cast<const float4*>(&sQ[warp][x]), b = *reinterpret_cast<const float4*>(&sK[lane][x]);
            s = fmaf(a.x, b.x, s); s = fmaf(a.y, b.y, s); s = fmaf(a.z, b.z, s); s = fmaf(a.w, b.w, s);
        }
        const bool kept = base + lane < cut;
        s = kept ? s + sW[lane] : -INFINITY;
        float top = s;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        top = fmaxf(m, top);
        const float ref = top == -INFINITY ? 0.0f : top, fade = m == -INFINITY ? 0.0f : expf(m - ref), p = kept ? expf(s - ref) : 0.0f;
        m = top;
        float sum = p;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        l = l * fade + sum;
#pragma unroll
        for (int x = 0; x < C; ++x) acc[x] = fade == 0.0f ? 0.0f : acc[x] * fade;
        const int count = max(0, min(cut - base, kKeys));
        for (int i = 0; i < count; ++i) {                         // (only kept keys: others' values may be anything)
            const float pi = __shfl_sync(0xffffffffu, p, i);
#pragma unroll
            for (int x = 0; x < C; ++x) acc[x] = fmaf(pi, sV[i][lane + 32 * x], acc[x]);
        }
    }
    if (!active) return;
    float* out = A.piece_of(t, h, 1 + split, D);
    if (lane == 0) { out[0] = m; out[1] = l; }
#pragma unroll
    for (int x = 0; x < C; ++x) out[2 + lane + 32 * x] = acc[x];
}

// A warp per (row, head) whose row has a prefix.
template <typename T, int D>
__global__ void __launch_bounds__(256) simt_sum_kernel(DecodeArgs A) {
    const int lane = threadIdx.x & 31, item = blockIdx.x * 8 + (threadIdx.x >> 5), t = item / A.Hq, h = item % A.Hq;
    pdl_enter();
    int r, n;
    if (item >= A.rows * A.Hq || A.own(t, r) < 0 || A.listed(t, n) < 0) return;
    float top = -INFINITY, sum = 0.0f;
    for (int i = 0; i < A.pieces; ++i) top = fmaxf(top, A.piece_of(t, h, i, D)[0]);
    float acc[D / 32] = {};
    for (int i = 0; i < A.pieces; ++i) {
        const float* p = A.piece_of(t, h, i, D);
        const float f = p[0] == -INFINITY ? (p[1] == 0.0f ? 0.0f : 1.0f) : expf(p[0] - top);
        if (f == 0.0f) continue;
        sum += p[1] * f;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) acc[x] += p[2 + lane + 32 * x] * f;
    }
    T* o = (T*)A.o + t * A.os_row + h * A.os_head;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) store_as(o + lane + 32 * x, sum == 0.0f ? 0.0f : acc[x] / sum);
    if (lane == 0) A.lse[item] = sum == 0.0f ? -INFINITY : top + logf(sum);
}

struct Layout {
    size_t cut, piece, first, members, tiles, ntiles, total;
    int pieces, tile_rows, max_tiles;
    bool simt;
    Layout(const Cache& C, int nprefix) {
        simt = C.dtype != DMA_BF16 || (C.flags & DMA_FLAG_SIMT);
        tile_rows = simt ? kWarps : 128;
        pieces = simt ? 1 + kSplits : 1;
        max_tiles = (int)std::min<int64_t>(C.rows, (int64_t)nprefix + C.rows / tile_rows);
        size_t x = kWsHeaderBytes;
        auto take = [&](size_t bytes) { const size_t at = x; x += (bytes + 255) / 256 * 256; return at; };
        cut = take((size_t)C.rows * C.Hq * 4);
        piece = take((size_t)C.rows * C.Hq * pieces * (C.d + 2) * 4);
        first = take((size_t)(nprefix + 1) * 4);
        members = take((size_t)max_tiles * tile_rows * 4);
        tiles = take((size_t)max_tiles * 16);
        ntiles = take(4);
        total = x;
    }
};

template <typename T, int D>
int prefix_simt(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st) {
    const int rc = launch_overlapped(simt_kernel<T, D>, dim3((unsigned)(max_tiles * C.Hq), A.pieces - 1), dim3(kThreads), 0, st, 1, A);
    return rc ? rc : launch_overlapped(simt_sum_kernel<T, D>, dim3((unsigned)((C.rows * C.Hq + 7) / 8)), dim3(256), 0, st, 1, A);
}

}  // namespace

int launch_prefix_simt(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? prefix_simt<__nv_bfloat16, 128> : prefix_simt<__nv_bfloat16, 64>) : (C.d == 128 ? prefix_simt<float, 128> : prefix_simt<float, 64>);
    return f(C, A, max_tiles, st);
}

size_t cache_decode_ws_bytes(const Cache& C, int nprefix) { return Layout(C, nprefix).total; }

int launch_cache_decode(const Cache& C, const void* q, const void* kv, const float* delta, const int32_t* table, const int32_t* row_seq, const int32_t* row_pos,
                        const int32_t* row_prefix, int nprefix, const int32_t* order_slot, const float* order_weight, int64_t order_ld, const int32_t* order_len,
                        void* o, float* lse, void* ws, cudaStream_t st) {
    const Layout L(C, nprefix);
    char* p = (char*)ws;
    const DecodeArgs A = {q, kv, delta, table, row_seq, row_pos, row_prefix, order_slot, order_len, order_weight, o, lse, C.table_ld, order_ld, C.qs[0], C.qs[1], C.os[0], C.os[1],
                          C.scale, C.rows, C.nseq, nprefix, C.Hq, C.Hkv, C.G, C.w, C.page_log, C.num_pages, C.max_blocks, (int32_t*)p, (int*)(p + L.cut), (float*)(p + L.piece),
                          L.pieces, (int*)(p + L.first), (int*)(p + L.members), (int4*)(p + L.tiles), (int*)(p + L.ntiles), L.tile_rows};
    const int rc = launch_own_keys(C, A, st);
    if (rc || nprefix == 0) return rc;
    return L.simt ? launch_prefix_simt(C, A, L.max_tiles, st) : launch_prefix_tc(C, A, L.max_tiles, st);
}

}  // namespace dma
