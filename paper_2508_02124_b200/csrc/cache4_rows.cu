// Rows into and out of the paged 4-bit cache (include/dma.h, dma_cache4_append, dma_cache4_read).
//
// A group of d / 8 lanes owns a row of one KV head, 8 channels of K and of V per lane, as in the kernels that form delta: a lane's eight
// codes are one 32-bit word, eight lanes hold the 64 channels of a scale.
#include <algorithm>
#include <type_traits>

#include "delta_fixed.cuh"
#include "paged.cuh"

namespace dma {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// The codes of a lane's eight channels, and the (s, z) pair of its group of eight lanes. All in fp32, rounded operation by operation:
// the halves keep every difference in range.
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t& pair) {
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int c = 1; c < 8; ++c) { lo = min_nan(lo, x[c]); hi = max_nan(hi, x[c]); }
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, m));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    const float z = round_bf16(lo), zh = __fmul_rn(z, 0.5f);
    const float s = max_nan(0.0f, round_bf16(__fdiv_rn(__fsub_rn(__fmul_rn(hi, 0.5f), zh), 7.5f)));
    const float sh = __fmul_rn(s, 0.5f);
    pair = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(s)) | (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(z)) << 16;
    uint32_t word = 0u;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float n = rintf(__fdiv_rn(__fsub_rn(__fmul_rn(x[c], 0.5f), zh), sh));
        word |= (uint32_t)(int)fminf(fmaxf(n, 0.0f), 15.0f) << (4 * c);        // (fmaxf: 0 where n is NaN)
    }
    return word;
}

// Tiles of kRows rows of KV head blockIdx.y, taken in turn. z of the tile's (head, row) pairs goes through shared memory; then a thread per
// pair forms delta.
template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kThreads) cache4_append_kernel(const T* K, const T* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld,
                                                                 const int32_t* slot, uint8_t* codes, uint32_t* scales, float* delta, int rows, int Hq, int Hkv, int G,
                                                                 int64_t ks_row, int64_t ks_head, int64_t vs_row, int64_t vs_head, int page_log, int nslots) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    extern __shared__ float smem[];
    float* sW = smem;                     // [G][D]
    float* sZ = smem + G * D;             // [G][kRows]
    __shared__ int sSlot[kRows];
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(K, V, W, A, delta_new, slot, codes, scales, delta);
    if (!delta_new)
        for (int i = tid; i < G * D; i += kThreads) sW[i] = W[(size_t)hk * G * D + i];
    const int place_mask = (1 << page_log) - 1, ntiles = (rows + kRows - 1) / kRows;
    for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
        const int t0 = tile * kRows, n = min(kRows, rows - t0);
        __syncthreads();                  // W; the last tile's z and slots have been read
        for (int r = warp * RPW + grp; r < kRows; r += 8 * RPW) {
            const int t = t0 + r;
            const bool real = r < n;
            const int at = real ? slot[t] : -1;
            const bool in = (unsigned)at < (unsigned)nslots;
            float k[8], v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) k[c] = v[c] = 0.0f;
            if (in) {
                load8(K + t * ks_row + hk * ks_head + sub * 8, k);
                load8(V + t * vs_row + hk * vs_head + sub * 8, v);
            }
            if (!delta_new) {
                for (int g = 0; g < G; ++g) {
                    float p = 0.0f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) p = __fmaf_rn(v[c], sW[g * D + sub * 8 + c], p);
#pragma unroll
                    for (int m = 1; m < LPR; m <<= 1) p = __fadd_rn(p, __shfl_xor_sync(0xffffffffu, p, m));
                    if (sub == 0) sZ[g * kRows + r] = p;
                }
            }
            uint32_t kp, vp;
            const uint32_t kw = quantise(k, kp), vw = quantise(v, vp);
            if (sub == 0) sSlot[r] = in ? at : -1;
            if (in) {
                const size_t row = key_row(at >> page_log, hk, at & place_mask, Hkv, page_log);
                *reinterpret_cast<uint32_t*>(codes + row * D + sub * 4) = kw;
                *reinterpret_cast<uint32_t*>(codes + row * D + D / 2 + sub * 4) = vw;
                if (sub % 8 == 0) {
                    scales[row * (D / 32) + sub / 8] = kp;
                    scales[row * (D / 32) + D / 64 + sub / 8] = vp;
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < G * kRows; i += kThreads) {
            const int g = i / kRows, r = i % kRows, h = hk * G + g, at = sSlot[r];
            if (at < 0) continue;
            const float x = delta_new ? delta_new[h * delta_ld + t0 + r] : delta_fixed(sZ[i], A[h]);
            delta[(((size_t)(at >> page_log) * Hq + h) << page_log) + (at & place_mask)] = x;
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

__device__ __forceinline__ void expand(uint32_t word, uint32_t pair, float (&x)[8]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = __fmaf_rn(pair_s(pair), (float)(word >> (4 * c) & 15u), pair_z(pair));
}

template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kThreads) cache4_read_kernel(const uint8_t* codes, const uint32_t* scales, const float* delta, const int32_t* slot, T* K, T* V,
                                                               float* delta_out, int64_t delta_ld, int rows, int Hq, int Hkv, int G, int64_t ks_row, int64_t ks_head,
                                                               int64_t vs_row, int64_t vs_head, int page_log, int nslots) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(codes, scales, delta, slot, K, V, delta_out);
    const int place_mask = (1 << page_log) - 1, t0 = blockIdx.x * kRows, n = min(kRows, rows - t0);
    for (int r = warp * RPW + grp; r < n; r += 8 * RPW) {
        const int t = t0 + r, at = slot[t];
        if ((unsigned)at >= (unsigned)nslots) continue;
        const size_t row = key_row(at >> page_log, hk, at & place_mask, Hkv, page_log);
        float k[8], v[8];
        expand(*reinterpret_cast<const uint32_t*>(codes + row * D + sub * 4), scales[row * (D / 32) + sub / 8], k);
        expand(*reinterpret_cast<const uint32_t*>(codes + row * D + D / 2 + sub * 4), scales[row * (D / 32) + D / 64 + sub / 8], v);
        store8(K + t * ks_row + hk * ks_head + sub * 8, k);
        store8(V + t * vs_row + hk * vs_head + sub * 8, v);
    }
    if (!delta_out) return;
    for (int i = tid; i < G * kRows; i += kThreads) {
        const int r = i % kRows, h = hk * G + i / kRows;
        if (r >= n) continue;
        const int at = slot[t0 + r];
        if ((unsigned)at < (unsigned)nslots) delta_out[h * delta_ld + t0 + r] = delta[(((size_t)(at >> page_log) * Hq + h) << page_log) + (at & place_mask)];
    }
}

template <typename T, int D>
int append(const Cache& C, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
           uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    constexpr int kRows = 32;
    const size_t smem = (size_t)C.G * (D + kRows) * sizeof(float);
    if (smem > 48 * 1024) return DMA_ERR_UNSUPPORTED;
    const int tiles = (C.rows + kRows - 1) / kRows;
    return launch_overlapped(cache4_append_kernel<T, D, kRows>, dim3(tiles, C.Hkv), dim3(kThreads), smem, st, 1, (const T*)K, (const T*)V, W, A, delta_new, delta_ld,
                             slot, codes, (uint32_t*)scales, delta, C.rows, C.Hq, C.Hkv, C.G, C.ks[0], C.ks[1], C.vs[0], C.vs[1], C.page_log,
                             C.num_pages << C.page_log);
}

template <typename T, int D>
int read(const Cache& C, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* slot, void* K, void* V, float* delta_out,
         int64_t delta_ld, cudaStream_t st) {
    constexpr int kRows = 32;
    return launch_overlapped(cache4_read_kernel<T, D, kRows>, dim3((C.rows + kRows - 1) / kRows, C.Hkv), dim3(kThreads), 0, st, 1, codes, (const uint32_t*)scales, delta,
                             slot, (T*)K, (T*)V, delta_out, delta_ld, C.rows, C.Hq, C.Hkv, C.G, C.ks[0], C.ks[1], C.vs[0], C.vs[1], C.page_log,
                             C.num_pages << C.page_log);
}

}  // namespace

int launch_cache4_append(const Cache& C, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
                         uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? append<__nv_bfloat16, 128> : append<__nv_bfloat16, 64>) : (C.d == 128 ? append<float, 128> : append<float, 64>);
    return f(C, K, V, W, A, delta_new, delta_ld, slot, codes, scales, delta, st);
}

int launch_cache4_read(const Cache& C, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* slot, void* K, void* V,
                       float* delta_out, int64_t delta_ld, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? read<__nv_bfloat16, 128> : read<__nv_bfloat16, 64>) : (C.d == 128 ? read<float, 128> : read<float, 64>);
    return f(C, codes, scales, delta, slot, K, V, delta_out, delta_ld, st);
}

}  // namespace dma
