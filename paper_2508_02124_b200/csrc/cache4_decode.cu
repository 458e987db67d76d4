// Decoding over the paged 4-bit cache (include/dma.h, dma_cache4_decode): every (row, query head) keeps the w visible keys with the largest
// dynamic weight delta (ties to the lower index) and attends to them with delta as the bias.
//
// Kernels
//   select_kernel        per (row, query head): the weakest kept key, as a 64-bit order key. A key is kept iff its order key is not below it
//   simt_attn_kernel     per (row, query head, split of the keys), fp32: CUDA cores
//   simt_combine_kernel  the splits' partials -> o, lse
#include <algorithm>

#include "paged.cuh"

namespace dma {
namespace {

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

constexpr int kSelectThreads = 256;

// The weakest of the `keep` best of the row's n keys, by radix passes of eight bits over the row: four over the patterns, then as many as the
// indices take over the keys with the threshold's pattern. Each pass reads the row again (from the L2).
struct RadixShared { int hist[256]; int bin, before, count; };
template <typename Load>
__device__ unsigned long long radix_select(RadixShared& S, Load&& load, int n, int keep) {
    const int tid = threadIdx.x;
    int need = keep;
    uint32_t u_lo = 0u;
    // the bin of the need-th in descending (down) or ascending order
    auto pick = [&](bool down) {
        __syncthreads();
        if (tid < 32) {
            int c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = S.hist[down ? 255 - (8 * tid + i) : 8 * tid + i]; sum += c[i]; }
            int incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (tid >= o) incl += v;
            }
            int before = incl - sum;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < need && need <= before + c[i]) { S.bin = down ? 255 - (8 * tid + i) : 8 * tid + i; S.before = before; S.count = c[i]; }
                before += c[i];
            }
        }
        __syncthreads();
    };
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += blockDim.x) S.hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += blockDim.x) {
            const uint32_t u = load(j);
            if (shift == 24 || (u ^ u_lo) >> (shift + 8) == 0) atomicAdd(&S.hist[u >> shift & 255u], 1);
        }
        pick(true);
        u_lo |= (uint32_t)S.bin << shift;
        need -= S.before;
        if (S.count == need) return order_key(u_lo, INT32_MAX);              // the whole bin is kept
    }
    // the need-th lowest index among the keys with this pattern
    int j_lo = 0;
    for (int shift = (31 - __clz(n)) / 8 * 8; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += blockDim.x) S.hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += blockDim.x)
            if (load(j) == u_lo && (shift == 24 || (j ^ j_lo) >> (shift + 8) == 0)) atomicAdd(&S.hist[j >> shift & 255], 1);
        pick(false);
        j_lo |= S.bin << shift;
        need -= S.before;
    }
    return order_key(u_lo, j_lo);
}

__global__ void __launch_bounds__(kSelectThreads) select_kernel(Rows R, int w, unsigned long long* weakest) {
    __shared__ RadixShared S;
    pdl_enter(R.table, R.seq, R.pos, R.delta, weakest);
    const int t = blockIdx.x / R.Hq, h = blockIdx.x % R.Hq;
    int r;
    const int n = R.visible(t, r);
    unsigned long long k = 0ull;                                  // (every key)
    if (n > w) {
        const int32_t* pages = R.table + r * R.ld;
        k = radix_select(S, [&](int j) {
            const int page = pages[j >> R.page_log];
            if ((unsigned)page >= (unsigned)R.num_pages) return 0u;
            return __float_as_uint(R.delta[(((size_t)page * R.Hq + h) << R.page_log) + (j & R.mask())]) & 0x7FFFFFFFu;
        }, n, w);
    }
    if (threadIdx.x == 0) weakest[blockIdx.x] = k;
}

// CUDA cores, fp32 throughout. A warp looks at 32 keys at a time, a lane per key, and queues the kept ones; eight lanes take one of them, with d / 8
// channels per lane, so that four keys run side by side. Warps and splits take words of 32 keys in turn, each with its own running
// maximum; partials (m, l, o) meet in shared memory and, where a row has several splits, in simt_combine_kernel.
constexpr int kSimtWarps = 4;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kSimtWarps) simt_attn_kernel(Rows R, const T* q, const uint8_t* codes, const uint32_t* scales, const unsigned long long* weakest,
                                                                    T* o, float* lse, float* partial, int Hkv, int G, float scale, int64_t qs_row, int64_t qs_head,
                                                                    int64_t os_row, int64_t os_head) {
    constexpr int C = D / 8;                                      // channels of a lane
    __shared__ size_t sRow[kSimtWarps][32];
    __shared__ float sDelta[kSimtWarps][32];
    __shared__ float sM[kSimtWarps], sL[kSimtWarps], sO[kSimtWarps][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7, grp = lane >> 3;
    const int item = blockIdx.x, t = item / R.Hq, h = item % R.Hq, hk = h / G, split = blockIdx.y, nsplit = gridDim.y;
    pdl_enter(R.table, R.seq, R.pos, R.delta, q, codes, scales, weakest, o, lse, partial);
    int r;
    const int n = R.visible(t, r);
    if (n < 0) return;
    const int32_t* pages = R.table + r * R.ld;
    const unsigned long long least = weakest ? weakest[item] : 0ull;
    float qv[C], qsum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        qv[c] = to_f32(q[t * qs_row + h * qs_head + sub * C + c]) * scale;
        qsum += qv[c];
    }
    float m = -INFINITY, l = 0.0f, acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.0f;
    const int gi = sub * C / kGroup;                              // the lane's group of channels
    for (int word = split * kSimtWarps + warp; word * 32 < n; word += nsplit * kSimtWarps) {
        const int j = word * 32 + lane;
        bool kept = false;
        float dl = 0.0f;
        int page = -1;
        if (j < n) {
            page = pages[j >> R.page_log];
            if ((unsigned)page < (unsigned)R.num_pages) {
                dl = R.delta[(((size_t)page * R.Hq + h) << R.page_log) + (j & R.mask())];
                kept = order_key(__float_as_uint(dl) & 0x7FFFFFFFu, j) >= least;
            }
        }
        const uint32_t b = __ballot_sync(0xffffffffu, kept);
        if (kept) {
            const int at = __popc(b & ((1u << lane) - 1u));
            sRow[warp][at] = key_row(page, hk, j & R.mask(), Hkv, R.page_log);
            sDelta[warp][at] = dl;
        }
        __syncwarp();
        const int count = __popc(b);
        for (int i = 0; i < count; i += 4) {
            const bool real = i + grp < count;
            const size_t row = real ? sRow[warp][i + grp] : 0;
            uint32_t kw[C / 8], vw[C / 8], kp = 0u, vp = 0u;
#pragma unroll
            for (int x = 0; x < C / 8; ++x) kw[x] = vw[x] = 0u;
            if (real) {
#pragma unroll
                for (int x = 0; x < C / 8; ++x) {
                    kw[x] = *reinterpret_cast<const uint32_t*>(codes + row * D + sub * (C / 2) + 4 * x);
                    vw[x] = *reinterpret_cast<const uint32_t*>(codes + row * D + D / 2 + sub * (C / 2) + 4 * x);
                }
                kp = scales[row * (D / 32) + gi];
                vp = scales[row * (D / 32) + D / 64 + gi];
            }
            float s = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) s = fmaf(qv[c], (float)(kw[c / 8] >> (4 * (c % 8)) & 15u), s);
            s = fmaf(s, pair_s(kp), qsum * pair_z(kp));
#pragma unroll
            for (int x = 1; x < 8; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            s = real ? s + sDelta[warp][i + grp] : -INFINITY;
            float top = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(m, top);
            // (a NaN score leaves no maximum and makes the sum NaN; so does one of +inf)
            const float fade = m == -INFINITY ? 0.0f : expf(m - top), p = real ? expf(s - top) : 0.0f;
            m = top;
            l = l * fade + p;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float v = fmaf(pair_s(vp), (float)(vw[c / 8] >> (4 * (c % 8)) & 15u), pair_z(vp));
                acc[c] = acc[c] * fade + (real ? p * v : 0.0f);
            }
        }
        __syncwarp();
    }
    // the four keys side by side, then the warps
#pragma unroll
    for (int x = 8; x < 32; x <<= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, x);
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], x);
    }
    if (lane == 0) { sM[warp] = m; sL[warp] = l; }
    if (grp == 0)
#pragma unroll
        for (int c = 0; c < C; ++c) sO[warp][sub * C + c] = acc[c];
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kSimtWarps; ++x) top = fmaxf(top, sM[x]);
    float sum = 0.0f, f[kSimtWarps];
#pragma unroll
    for (int x = 0; x < kSimtWarps; ++x) {
        f[x] = sM[x] == -INFINITY ? (sL[x] == 0.0f ? 0.0f : 1.0f) : expf(sM[x] - top);
        sum += sL[x] * f[x];
    }
    float* out = partial + ((size_t)item * nsplit + split) * (D + 2);
    for (int c = tid; c < D; c += 32 * kSimtWarps) {
        float a = 0.0f;
#pragma unroll
        for (int x = 0; x < kSimtWarps; ++x) a += sO[x][c] * f[x];
        if (nsplit > 1) out[2 + c] = a;
        else store_as(o + t * os_row + h * os_head + c, sum == 0.0f ? 0.0f : a / sum);
    }
    if (tid == 0) {
        if (nsplit > 1) { out[0] = top; out[1] = sum; }
        else lse[item] = top + logf(sum);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(D) simt_combine_kernel(Rows R, const float* partial, T* o, float* lse, int nsplit, int64_t os_row, int64_t os_head) {
    const int item = blockIdx.x, t = item / R.Hq, h = item % R.Hq, c = threadIdx.x;
    pdl_enter(R.seq, R.pos, partial, o, lse);
    int r;
    if (R.visible(t, r) < 0) return;
    const float* in = partial + (size_t)item * nsplit * (D + 2);
    float top = -INFINITY;
    for (int x = 0; x < nsplit; ++x) top = fmaxf(top, in[x * (D + 2)]);
    float sum = 0.0f, a = 0.0f;
    for (int x = 0; x < nsplit; ++x) {
        const float m = in[x * (D + 2)], l = in[x * (D + 2) + 1], f = m == -INFINITY ? (l == 0.0f ? 0.0f : 1.0f) : expf(m - top);
        sum += l * f;
        a += in[x * (D + 2) + 2 + c] * f;
    }
    store_as(o + t * os_row + h * os_head + c, sum == 0.0f ? 0.0f : a / sum);
    if (c == 0) lse[item] = top + logf(sum);
}

constexpr int kSimtCtas = 148 * 8;
int simt_splits(const Cache& C) {
    const int64_t items = (int64_t)C.rows * C.Hq, keys = (int64_t)C.max_blocks << C.page_log;
    return (int)std::min<int64_t>((kSimtCtas + items - 1) / items, std::min<int64_t>(64, (keys + 255) / 256));
}

size_t weakest_bytes(const Cache& C) { return ((size_t)C.rows * C.Hq * sizeof(unsigned long long) + 255) / 256 * 256; }

template <typename T, int D>
int simt_decode(const Cache& C, const Rows& R, const void* q, const uint8_t* codes, const __nv_bfloat16* scales, const unsigned long long* weakest, void* o, float* lse,
                float* partial, cudaStream_t st) {
    const int items = C.rows * C.Hq, splits = simt_splits(C);
    const int rc = launch_overlapped(simt_attn_kernel<T, D>, dim3(items, splits), dim3(32 * kSimtWarps), 0, st, 1, R, (const T*)q, codes, (const uint32_t*)scales,
                                     weakest, (T*)o, lse, partial, C.Hkv, C.G, C.scale, C.qs[0], C.qs[1], C.os[0], C.os[1]);
    if (rc || splits == 1) return rc;
    return launch_overlapped(simt_combine_kernel<T, D>, dim3(items), dim3(D), 0, st, 1, R, partial, (T*)o, lse, splits, C.os[0], C.os[1]);
}

}  // namespace

size_t cache4_decode_ws_bytes(const Cache& C) {
    return kWsHeaderBytes + weakest_bytes(C) + ((size_t)C.rows * C.Hq + kSimtCtas) * (C.d + 2) * sizeof(float);
}

int launch_cache4_decode(const Cache& C, const void* q, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* table,
                         const int32_t* row_seq, const int32_t* row_pos, void* o, float* lse, void* ws, cudaStream_t st) {
    const Rows R{table, row_seq, row_pos, delta, C.table_ld, C.nseq, C.page_log, C.num_pages, C.max_blocks, C.Hq};
    unsigned long long* weakest = nullptr;
    if (((int64_t)C.max_blocks << C.page_log) > C.w) {            // (no row sees more keys than the table holds)
        weakest = reinterpret_cast<unsigned long long*>((char*)ws + kWsHeaderBytes);
        const int rc = launch_overlapped(select_kernel, dim3(C.rows * C.Hq), dim3(kSelectThreads), 0, st, 1, R, C.w, weakest);
        if (rc) return rc;
    }
    float* partial = reinterpret_cast<float*>((char*)ws + kWsHeaderBytes + weakest_bytes(C));
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? simt_decode<__nv_bfloat16, 128> : simt_decode<__nv_bfloat16, 64>)
                                 : (C.d == 128 ? simt_decode<float, 128> : simt_decode<float, 64>);
    return f(C, R, q, codes, scales, weakest, o, lse, partial, st);
}

}  // namespace dma
