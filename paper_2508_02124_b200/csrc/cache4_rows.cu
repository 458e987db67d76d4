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
// A division takes a dozen instructions, sixteen of them per lane more than all else; so the quotients are products with the reciprocal, each within 4e-6 of the definition's for
// quotients below 16 (three roundings of 2^-24). Both round to the same code unless the product lies that near to a half; then, and for scales so small that their own
// rounding to bf16 is coarse, or not finite, the lane divides.
template <bool kExactZero>
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t& pair) {
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int c = 1; c < 8; ++c) { lo = min_nan(lo, x[c]); hi = max_nan(hi, x[c]); }
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, m));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    const float z = kExactZero ? lo : round_bf16(lo), zh = __fmul_rn(z, 0.5f);
    const float s = max_nan(0.0f, round_bf16(__fdiv_rn(__fsub_rn(__fmul_rn(hi, 0.5f), zh), 7.5f)));
    const float sh = __fmul_rn(s, 0.5f);
    pair = (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xffff0000u);
    const float inv = __frcp_rn(sh);
    bool near = !(s >= 1e-30f && s <= 1e37f);
    float n[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        float q = __fmul_rn(__fmaf_rn(x[c], 0.5f, -zh), inv);
        if (!kExactZero) q = fmaxf(q, 0.0f);                      // (a zero that bf16 rounded up; with an exact one no value lies below it)
        n[c] = __fadd_rn(__fadd_rn(q, 12582912.0f), -12582912.0f);
        near = near || !(fabsf(q - n[c]) <= 0.49999f);
    }
    if (near) {
#pragma unroll
        for (int c = 0; c < 8; ++c) n[c] = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(__fmul_rn(x[c], 0.5f), zh), sh)), 0.0f), 15.0f);        // (fmaxf: 0 where it is NaN)
    }
    // four codes as one number, exactly: 2^23 + them
    const float w0 = fmaf(fmaf(fmaf(n[3], 16.0f, n[2]), 16.0f, n[1]), 16.0f, n[0]) + 8388608.0f, w1 = fmaf(fmaf(fmaf(n[7], 16.0f, n[6]), 16.0f, n[5]), 16.0f, n[4]) + 8388608.0f;
    return __byte_perm(__float_as_uint(w0), __float_as_uint(w1), 0x5410);
}

// Tiles of kRows rows of KV head blockIdx.y, taken in turn; a warp requests its next rows before it works on those it has. z of the tile's (head, row) pairs goes
// through shared memory; then a thread per pair forms delta, while the next tile's rows are worked on (two buffers, one barrier per tile).
template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) cache4_append_kernel(const T* K, const T* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld,
                                                                 const int32_t* slot, uint8_t* codes, uint32_t* scales, float* delta, int rows, int Hq, int Hkv, int G,
                                                                 int64_t ks_row, int64_t ks_head, int64_t vs_row, int64_t vs_head, int page_log, int nslots) {
    constexpr int LPR = D / 8, RPW = 32 / LPR, kPass = kRows / (8 * RPW);
    using Raw = typename RawOf<T>::type;
    extern __shared__ float smem[];
    float* sW = smem;                     // [G][D]
    float* sZ = smem + G * D;             // [2][G][kRows]
    __shared__ int sSlot[2][kRows];
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(K, V, W, A, delta_new, slot, codes, scales, delta);
    const int place_mask = (1 << page_log) - 1, ntiles = (rows + kRows - 1) / kRows;
    const T* Kh = K + hk * ks_head + sub * 8;
    const T* Vh = V + hk * vs_head + sub * 8;
    Raw k_next, v_next;
    int at_next;
    auto request = [&](int tile, int pass) {
        const int t = tile * kRows + (pass * 8 + warp) * RPW + grp;
        k_next = Raw{};
        v_next = Raw{};
        at_next = -1;
        if (tile < ntiles && t < rows) {
            k_next = load_raw8(Kh + t * ks_row);
            v_next = load_raw8(Vh + t * vs_row);
            at_next = slot[t];
        }
    };
    request(blockIdx.x, 0);
    if (!delta_new) {
        // (a lane's eight weights in two halves, each next to the other lanes' same half: a group's 16-byte reads meet every bank once)
        for (int i = tid; i < G * D; i += kThreads) sW[i / D * D + (i >> 2 & 1) * (D / 2) + i % D / 8 * 4 + (i & 3)] = W[(size_t)hk * G * D + i];
        __syncthreads();
    }
    int buf = 0;
    for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x, buf ^= 1) {
        const int t0 = tile * kRows;
        float* zs = sZ + buf * G * kRows;
        for (int pass = 0; pass < kPass; ++pass) {
            const int r = (pass * 8 + warp) * RPW + grp, at = at_next;
            const bool in = (unsigned)at < (unsigned)nslots;
            float v[8];
            uint32_t kp, vp, kw, vw;
            {
                float k[8];
                widen8(k_next, k);
                widen8(v_next, v);
                if (pass + 1 < kPass) request(tile, pass + 1); else request(tile + gridDim.x, 0);
                kw = quantise<sizeof(T) == 2>(k, kp);
            }
            vw = quantise<sizeof(T) == 2>(v, vp);
            if (sub == 0) sSlot[buf][r] = in ? at : -1;
            if (in) {
                const size_t row = key_row(at >> page_log, hk, at & place_mask, Hkv, page_log);
                *reinterpret_cast<uint32_t*>(codes + row * D + sub * 4) = kw;
                *reinterpret_cast<uint32_t*>(codes + row * D + D / 2 + sub * 4) = vw;
                if (sub % 8 == 0) {
                    scales[row * (D / 32) + sub / 8] = kp;
                    scales[row * (D / 32) + D / 64 + sub / 8] = vp;
                }
            }
            if (!delta_new) {
                // heads in blocks of 4 (then 2, then 1), as in the other kernels that form delta
                auto block = [&](int g0, auto nb_tag) {
                    constexpr int NB = decltype(nb_tag)::value;
                    float p[NB];
#pragma unroll
                    for (int q = 0; q < NB; ++q) {
                        const float4 wa = *reinterpret_cast<const float4*>(sW + (g0 + q) * D + sub * 4), wb = *reinterpret_cast<const float4*>(sW + (g0 + q) * D + D / 2 + sub * 4);
                        const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
                        float a = 0.0f;
#pragma unroll
                        for (int c = 0; c < 8; ++c) a = __fmaf_rn(v[c], w[c], a);
                        p[q] = a;
                    }
                    int mine = 0;             // head of the block this lane ends up with: the low bits of sub, reversed
#pragma unroll
                    for (int m = 1, t = NB >> 1; m < NB; m <<= 1, t >>= 1) mine |= (sub & m) ? t : 0;
                    block_reduce<NB, LPR>(p, sub);
                    if (sub < NB) zs[(g0 + mine) * kRows + r] = p[0];
                };
                int g0 = 0;
                for (; g0 + 4 <= G; g0 += 4) block(g0, std::integral_constant<int, 4>{});
                if (g0 + 2 <= G) { block(g0, std::integral_constant<int, 2>{}); g0 += 2; }
                if (g0 < G) block(g0, std::integral_constant<int, 1>{});
            }
        }
        __syncthreads();                      // z and slots of this tile are complete (and the other buffers' readers of two tiles ago are long done)
        for (int i = tid; i < G * kRows; i += kThreads) {
            const int g = i / kRows, r = i % kRows, h = hk * G + g, at = sSlot[buf][r];
            if (at < 0) continue;
            const float x = delta_new ? delta_new[h * delta_ld + t0 + r] : delta_fixed(zs[i], A[h]);
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

template <typename T, int D, int kRows>
int append_tiles(const Cache& C, int ctas, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
                 uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    const size_t smem = (size_t)C.G * (D + 2 * kRows) * sizeof(float);
    if (smem > 48 * 1024) return DMA_ERR_UNSUPPORTED;
    return launch_overlapped(cache4_append_kernel<T, D, kRows>, dim3(ctas, C.Hkv), dim3(kThreads), smem, st, 1, (const T*)K, (const T*)V, W, A, delta_new, delta_ld, slot, codes,
                             (uint32_t*)scales, delta, C.rows, C.Hq, C.Hkv, C.G, C.ks[0], C.ks[1], C.vs[0], C.vs[1], C.page_log, C.num_pages << C.page_log);
}
// Tiles of 64 rows on four CTAs per SM; of a pass's rows where that leaves SMs without one.
template <typename T, int D>
int append(const Cache& C, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
           uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    constexpr int kPassRows = 8 * 32 / (D / 8), kTile = 64;
    const int tiles = (C.rows + kTile - 1) / kTile, most = (4 * 148 + C.Hkv - 1) / C.Hkv;
    const bool large = (int64_t)tiles * C.Hkv >= 148 && (size_t)C.G * (D + 2 * kTile) * sizeof(float) <= 48 * 1024;
    if (large) return append_tiles<T, D, kTile>(C, std::min(tiles, most), K, V, W, A, delta_new, delta_ld, slot, codes, scales, delta, st);
    return append_tiles<T, D, kPassRows>(C, std::min((C.rows + kPassRows - 1) / kPassRows, most), K, V, W, A, delta_new, delta_ld, slot, codes, scales, delta, st);
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
