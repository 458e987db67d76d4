// Rows into and out of the paged 4-bit cache (include/dma.h, dma_cache4_append, dma_cache4_read).
//
// Append: a group of d / 16 lanes owns a row of one KV head, 16 channels of K and of V per lane: two words of codes, four lanes to the 64 channels of a scale. Bound by
// latency: 61 % of the issue slots and 32 % of the warps active, neither memory nor a pipe at its limit; 18 instructions per warp and 32 values. 16384 rows of 8 heads, d = 128: 31 us,
// 2.9 TB/s, where the bytes alone take 13 (57 with divisions beside ties, 45 with 8 channels per lane: what a row takes beside its values is shared by fewer of them).
// Read: d / 8 lanes, a word of codes each. 14336 rows 16.6 us, 4.7 TB/s: below the copy's rate by the two dependent trips, slot and codes, that every CTA of several waves begins with.
#include <algorithm>
#include <type_traits>

#include "delta_fixed.cuh"
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kThreads = 256, kAppendThreads = 128;

__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// 16 channels as loaded, and widened
template <typename T> struct Raw16 { typename RawOf<T>::type a, b; };
template <typename T>
__device__ __forceinline__ Raw16<T> load_raw16(const T* p) { return {load_raw8(p), load_raw8(p + 8)}; }
template <typename T>
__device__ __forceinline__ void widen16(const Raw16<T>& r, float (&x)[2][8]) { widen8(r.a, x[0]); widen8(r.b, x[1]); }

// lo and hi over the four lanes of a group, of K and of V
__device__ __forceinline__ void group_range(const Raw16<float>& k, const Raw16<float>& v, float (&lo)[2], float (&hi)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float x[2][8];
        widen16(i ? v : k, x);
        lo[i] = hi[i] = x[0][0];
#pragma unroll
        for (int c = 1; c < 16; ++c) { lo[i] = min_nan(lo[i], x[c / 8][c % 8]); hi[i] = max_nan(hi[i], x[c / 8][c % 8]); }
#pragma unroll
        for (int m = 1; m < 4; m <<= 1) {
            lo[i] = min_nan(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], m));
            hi[i] = max_nan(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], m));
        }
    }
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) { uint32_t r; asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { uint32_t r; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
// (two numbers per instruction, and K's and V's together through the lanes)
__device__ __forceinline__ void group_range(const Raw16<__nv_bfloat16>& k, const Raw16<__nv_bfloat16>& v, float (&lo)[2], float (&hi)[2]) {
    auto all = [](auto&& f, const Raw16<__nv_bfloat16>& r) { return f(f(f(r.a.x, r.a.y), f(r.a.z, r.a.w)), f(f(r.b.x, r.b.y), f(r.b.z, r.b.w))); };
    const uint32_t k0 = all(min2, k), v0 = all(min2, v), k1 = all(max2, k), v1 = all(max2, v);
    uint32_t a = min2(__byte_perm(k0, v0, 0x5410), __byte_perm(k0, v0, 0x7632)), b = max2(__byte_perm(k1, v1, 0x5410), __byte_perm(k1, v1, 0x7632));
#pragma unroll
    for (int m = 1; m < 4; m <<= 1) {
        a = min2(a, __shfl_xor_sync(0xffffffffu, a, m));
        b = max2(b, __shfl_xor_sync(0xffffffffu, b, m));
    }
    lo[0] = __uint_as_float(a << 16); lo[1] = __uint_as_float(a & 0xffff0000u);
    hi[0] = __uint_as_float(b << 16); hi[1] = __uint_as_float(b & 0xffff0000u);
}

// The codes of a lane's 16 channels, and the (s, z) pair of its group: the definition, in fp32, rounded operation by operation; the halves keep every difference in range.
// A division takes a dozen instructions, sixteen of them per lane more than all else. A quotient a / b is therefore the product q with b's rounded reciprocal y and one
// correction, q + (a - q b) y (Markstein, "Computation of elementary functions on the IBM RISC System/6000", 1990). The remainder is exact, and before its own rounding the sum is
// within 2^-45 of the quotient, so that it rounds to the quotient's rounding unless the quotient is as near to a midpoint between two numbers. It never is: b is half a bf16 number
// or 7.5, of 8 bits at most, a has 24, and a midpoint m has 25 with its last one set. m b then has 25 bits at least without trailing zeros, is not a, and as multiples of one unit
// below 2^33 the two differ by 2^-33 at least. So the codes are the divisions' bits. (Without the correction 0.2 % of bf16 values are ties that the product misses.) Two values per
// instruction. Ranges at the ends of fp32's, and what is not finite, are divided; rows that are not stored (`used`) may come out as anything.
template <bool kExactZero>
__device__ __forceinline__ uint2 quantise(const float (&x)[2][8], float lo, float hi, bool used, uint32_t& pair) {
    const float z = kExactZero ? lo : round_bf16(lo), zh = __fmul_rn(z, 0.5f), range = __fsub_rn(__fmul_rn(hi, 0.5f), zh);
    if (kExactZero && range == 0.0f) {                            // equal values: 0 / 0, code 0
        pair = __float_as_uint(z) & 0xffff0000u;
        return make_uint2(0u, 0u);
    }
    if (!(range >= 1e-28f && range <= 1e38f) && used) {
        const float s = max_nan(0.0f, round_bf16(__fdiv_rn(range, 7.5f))), sh = __fmul_rn(s, 0.5f);
        pair = (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xffff0000u);
        uint32_t word[2] = {0u, 0u};
#pragma unroll
        for (int c = 0; c < 16; ++c)                              // (fmaxf: 0 where the quotient is NaN)
            word[c / 8] |= (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(__fmul_rn(x[c / 8][c % 8], 0.5f), zh), sh)), 0.0f), 15.0f) << (4 * (c % 8));
        return make_uint2(word[0], word[1]);
    }
    constexpr float kSeventh = 1.0f / 7.5f;
    float q0 = __fmul_rn(range, kSeventh);
    q0 = __fmaf_rn(__fmaf_rn(-q0, 7.5f, range), kSeventh, q0);
    const float s = round_bf16(q0), sh = __fmul_rn(s, 0.5f), y = __frcp_rn(sh);
    pair = (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xffff0000u);
    const float2 half = make_float2(0.5f, 0.5f), zz = make_float2(-zh, -zh), b = make_float2(-sh, -sh), yy = make_float2(y, y), up = make_float2(12582912.0f, 12582912.0f),
                 down = make_float2(-12582912.0f, -12582912.0f), by16 = make_float2(16.0f, 16.0f);
    uint32_t word[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float2 n[4];                                              // codes c and c + 4
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float2 a = ptx::fma2(make_float2(x[i][c], x[i][c + 4]), half, zz);
            float2 q = ptx::mul2(a, yy);
            q = ptx::fma2(ptx::fma2(q, b, a), yy, q);
            if (!kExactZero) { q.x = fmaxf(q.x, 0.0f); q.y = fmaxf(q.y, 0.0f); }   // (a zero that bf16 rounded up; below an exact one lies no value, and none above 15.1)
            n[c] = ptx::add2(ptx::add2(q, up), down);             // to the nearest integer, ties to even
        }
        // four codes as one number, exactly, above 2^23
        const float2 w = ptx::add2(ptx::fma2(ptx::fma2(ptx::fma2(n[3], by16, n[2]), by16, n[1]), by16, n[0]), make_float2(8388608.0f, 8388608.0f));
        word[i] = __byte_perm(__float_as_uint(w.x), __float_as_uint(w.y), 0x5410);
    }
    return make_uint2(word[0], word[1]);
}

// Tiles of kRows rows of KV head blockIdx.y, taken in turn; a warp requests its next rows before it works on those it has. z of the tile's (head, row) pairs goes
// through shared memory; then a thread per pair forms delta, while the next tile's rows are worked on (two buffers, one barrier per tile).
template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kAppendThreads, sizeof(T) == 2 ? 6 : 4) cache4_append_kernel(const T* K, const T* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld,
                                                                 const int32_t* slot, uint8_t* codes, uint32_t* scales, float* delta, int rows, int Hq, int Hkv, int G,
                                                                 int64_t ks_row, int64_t ks_head, int64_t vs_row, int64_t vs_head, int page_log, int nslots) {
    constexpr int LPR = D / 16, RPW = 32 / LPR, kWarps = kAppendThreads / 32, kPass = kRows / (kWarps * RPW);
    extern __shared__ float smem[];
    float* sW = smem;                     // [G][D]
    float* sZ = smem + G * D;             // [2][G][kRows]
    __shared__ int sSlot[2][kRows];
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(K, V, W, A, delta_new, slot, codes, scales, delta);
    const int place_mask = (1 << page_log) - 1, ntiles = (rows + kRows - 1) / kRows;
    const T* Kh = K + hk * ks_head + sub * 16;
    const T* Vh = V + hk * vs_head + sub * 16;
    Raw16<T> k_next, v_next;
    int at_next;
    auto request = [&](int tile, int pass) {
        const int t = tile * kRows + (pass * kWarps + warp) * RPW + grp;
        k_next = Raw16<T>{};
        v_next = Raw16<T>{};
        at_next = -1;
        if (tile < ntiles && t < rows) {
            k_next = load_raw16(Kh + t * ks_row);
            v_next = load_raw16(Vh + t * vs_row);
            at_next = slot[t];
        }
    };
    request(blockIdx.x, 0);
    if (!delta_new) {
        // (a lane's sixteen weights in four parts, each next to the other lanes' same part: a group's 16-byte reads meet every bank once)
        for (int i = tid; i < G * D; i += kAppendThreads) sW[i / D * D + (i >> 2 & 3) * (D / 4) + i % D / 16 * 4 + (i & 3)] = W[(size_t)hk * G * D + i];
        __syncthreads();
    }
    int buf = 0;
    for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x, buf ^= 1) {
        const int t0 = tile * kRows;
        float* zs = sZ + buf * G * kRows;
        for (int pass = 0; pass < kPass; ++pass) {
            const int r = (pass * kWarps + warp) * RPW + grp, at = at_next;
            const bool in = (unsigned)at < (unsigned)nslots;
            float v[2][8];
            uint32_t kp, vp;
            uint2 kw, vw;
            {
                float k[2][8], lo[2], hi[2];
                group_range(k_next, v_next, lo, hi);
                widen16(k_next, k);
                widen16(v_next, v);
                if (pass + 1 < kPass) request(tile, pass + 1); else request(tile + gridDim.x, 0);
                kw = quantise<sizeof(T) == 2>(k, lo[0], hi[0], in, kp);
                vw = quantise<sizeof(T) == 2>(v, lo[1], hi[1], in, vp);
            }
            if (sub == 0) sSlot[buf][r] = in ? at : -1;
            if (in) {
                const size_t row = key_row(at >> page_log, hk, at & place_mask, Hkv, page_log);
                uint8_t* to = codes + row * D + sub * 8;
                *reinterpret_cast<uint2*>(to) = kw;
                *reinterpret_cast<uint2*>(to + D / 2) = vw;
                if (sub % 4 == 0) {
                    uint32_t* sc = scales + row * (D / 32) + sub / 4;
                    sc[0] = kp;
                    sc[D / 64] = vp;
                }
            }
            if (!delta_new) {
                // Heads in blocks of 4 (then 2, then 1). The sums are those of the other kernels that form delta: a chain over each 8 channels, then neighbours pairwise, the
                // first two of which a lane has itself.
                auto block = [&](int g0, auto nb_tag) {
                    constexpr int NB = decltype(nb_tag)::value;
                    float p[NB];
#pragma unroll
                    for (int q = 0; q < NB; ++q) {
                        float part[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float* wp = sW + (g0 + q) * D + i * (D / 2) + sub * 4;
                            const float4 wa = *reinterpret_cast<const float4*>(wp), wb = *reinterpret_cast<const float4*>(wp + D / 4);
                            const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
                            float a = 0.0f;
#pragma unroll
                            for (int c = 0; c < 8; ++c) a = __fmaf_rn(v[i][c], w[c], a);
                            part[i] = a;
                        }
                        p[q] = __fadd_rn(part[0], part[1]);
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
        for (int i = tid; i < G * kRows; i += kAppendThreads) {
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
    constexpr int LPR = D / 8, RPW = 32 / LPR, kTurns = kRows / (8 * RPW), kTogether = sizeof(T) == 2 ? kTurns : 1;      // (rows of a lane; requested at once)
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(codes, scales, delta, slot, K, V, delta_out);
    const int place_mask = (1 << page_log) - 1, t0 = blockIdx.x * kRows, n = min(kRows, rows - t0);
#pragma unroll 1
    for (int i0 = 0; i0 < kTurns; i0 += kTogether) {
        int at[kTogether];
        uint32_t kw[kTogether], vw[kTogether], kp[kTogether], vp[kTogether];
        auto row_of = [&](int i) { return ((i0 + i) * 8 + warp) * RPW + grp; };
#pragma unroll
        for (int i = 0; i < kTogether; ++i) at[i] = row_of(i) < n ? slot[t0 + row_of(i)] : -1;
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            if ((unsigned)at[i] >= (unsigned)nslots) continue;
            const size_t row = key_row(at[i] >> page_log, hk, at[i] & place_mask, Hkv, page_log);
            kw[i] = *reinterpret_cast<const uint32_t*>(codes + row * D + sub * 4);
            vw[i] = *reinterpret_cast<const uint32_t*>(codes + row * D + D / 2 + sub * 4);
            kp[i] = scales[row * (D / 32) + sub / 8];
            vp[i] = scales[row * (D / 32) + D / 64 + sub / 8];
        }
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            if ((unsigned)at[i] >= (unsigned)nslots) continue;
            const int t = t0 + row_of(i);
            float k[8], v[8];
            expand(kw[i], kp[i], k);
            expand(vw[i], vp[i], v);
            store8(K + t * ks_row + hk * ks_head + sub * 8, k);
            store8(V + t * vs_row + hk * vs_head + sub * 8, v);
        }
    }
    if (!delta_out) return;
    for (int i = tid; i < G * kRows; i += kThreads) {
        const int r = i % kRows, h = hk * G + i / kRows;
        if (r >= n) continue;
        const int at = slot[t0 + r];
        if ((unsigned)at < (unsigned)nslots) delta_out[h * delta_ld + t0 + r] = delta[(((size_t)(at >> page_log) * Hq + h) << page_log) + (at & place_mask)];
    }
}

// What a CTA of the append takes beside its sSlot, and what no opt-in is needed for.
constexpr size_t append_smem(int G, int d, int rows) { return (size_t)G * (d + 2 * rows) * sizeof(float); }
constexpr size_t append_room(int rows) { return 48 * 1024 - 2 * rows * sizeof(int); }

template <typename T, int D, int kRows>
int append_tiles(const Cache& C, int ctas, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
                 uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    const size_t smem = append_smem(C.G, D, kRows);
    if (smem > append_room(kRows) &&
        cudaFuncSetAttribute(cache4_append_kernel<T, D, kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(cache4_append_kernel<T, D, kRows>, dim3(ctas, C.Hkv), dim3(kAppendThreads), smem, st, 1, (const T*)K, (const T*)V, W, A, delta_new, delta_ld, slot, codes,
                             (uint32_t*)scales, delta, C.rows, C.Hq, C.Hkv, C.G, C.ks[0], C.ks[1], C.vs[0], C.vs[1], C.page_log, C.num_pages << C.page_log);
}
// Tiles of 32 rows on six CTAs per SM where there are three per SM (us of 64, 32 and, a pass's, 8 rows, d = 128: 16384 rows of 8 heads 32.1, 30.4 and 32.5, 2048 rows -, 6.5 and 7.0, 1024 rows -, 5.2
// and 4.6); of a pass's rows where there are fewer, or the heads' z need the room.
template <typename T, int D>
int append(const Cache& C, const void* K, const void* V, const float* W, const float* A, const float* delta_new, int64_t delta_ld, const int32_t* slot,
           uint8_t* codes, __nv_bfloat16* scales, float* delta, cudaStream_t st) {
    constexpr int kPassRows = kAppendThreads / (D / 16), kTile = 32;
    const int tiles = (C.rows + kTile - 1) / kTile, most = (6 * 148 + C.Hkv - 1) / C.Hkv;
    if (kTile > kPassRows && (int64_t)tiles * C.Hkv >= 3 * 148 && append_smem(C.G, D, kTile) <= append_room(kTile))
        return append_tiles<T, D, kTile>(C, std::min(tiles, most), K, V, W, A, delta_new, delta_ld, slot, codes, scales, delta, st);
    return append_tiles<T, D, kPassRows>(C, std::min((C.rows + kPassRows - 1) / kPassRows, most), K, V, W, A, delta_new, delta_ld, slot, codes, scales, delta, st);
}

template <typename T, int D, int kRows>
int read_tiles(const Cache& C, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* slot, void* K, void* V, float* delta_out,
               int64_t delta_ld, cudaStream_t st) {
    return launch_overlapped(cache4_read_kernel<T, D, kRows>, dim3((C.rows + kRows - 1) / kRows, C.Hkv), dim3(kThreads), 0, st, 1, codes, (const uint32_t*)scales, delta,
                             slot, (T*)K, (T*)V, delta_out, delta_ld, C.rows, C.Hq, C.Hkv, C.G, C.ks[0], C.ks[1], C.vs[0], C.vs[1], C.page_log,
                             C.num_pages << C.page_log);
}
// A lane has one row where the chip holds all CTAs at once, else two (us of one and of two, 8 heads: d = 128, 64 rows 1.8 and 2.1, 2000 rows 3.3 and 3.5, 32768 rows 38.9 and 34.5; d = 64 22.8 and
// 20.3). bf16 rows are requested together (one after the other 36.4 with d = 128), fp32 ones are not (d = 128: 65.3, together 68.8).
template <typename T, int D>
int read(const Cache& C, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* slot, void* K, void* V, float* delta_out,
         int64_t delta_ld, cudaStream_t st) {
    constexpr int kPass = kThreads / (D / 8);
    if ((int64_t)((C.rows + kPass - 1) / kPass) * C.Hkv > 8 * 148) return read_tiles<T, D, 2 * kPass>(C, codes, scales, delta, slot, K, V, delta_out, delta_ld, st);
    return read_tiles<T, D, kPass>(C, codes, scales, delta, slot, K, V, delta_out, delta_ld, st);
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
