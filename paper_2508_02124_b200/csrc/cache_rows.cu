// A step's rows into the paged cache of the element type (include/dma.h, dma_cache_append): q and K rotated by their positions, V as it is, delta of V.
//
// d / 16 lanes own a row. A lane has the 16 channels of a head whose pairs turn by the same eight angles, whichever of the two pairings is asked for, so that it forms eight
// sines and cosines per row and turns its part of every head with them. Angles: position times frequency in turns, in 64 bits, less the whole turns; fp32 from there on.
#include <algorithm>
#include <type_traits>

#include "delta_fixed.cuh"
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kThreads = 128;

template <typename T> using Raw = typename RawOf<T>::type;

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(ptx::pack_bf16(v[0], v[1]), ptx::pack_bf16(v[2], v[3]), ptx::pack_bf16(v[4], v[5]), ptx::pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store_raw(float* p, const Raw8f& r) {
    *reinterpret_cast<float4*>(p) = r.a;
    *reinterpret_cast<float4*>(p + 4) = r.b;
}
__device__ __forceinline__ void store_raw(__nv_bfloat16* p, const uint4& r) { *reinterpret_cast<uint4*>(p) = r; }

struct Append {
    const void *q, *K, *V;
    const float *W, *A, *delta_new, *inv_freq;
    const int32_t *slot, *pos, *prefix, *prefix_len;
    void *q_out, *kv;
    float* delta;
    int64_t delta_ld, qs_row, qs_head, ks_row, ks_head, vs_row, vs_head, os_row, os_head;
    float rot_scale;
    int rows, Hq, Hkv, G, page_log, nslots, nprefix, rot, interleaved;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) append_kernel(Append P) {
    constexpr int LPR = D / 16, RPW = 32 / LPR, kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter(P.q, P.K, P.V, P.W, P.A, P.delta_new, P.inv_freq, P.slot, P.pos, P.prefix, P.prefix_len, P.q_out, P.kv, P.delta);
    const int t = (blockIdx.x * kWarps + warp) * RPW + grp;
    const bool turning = P.inv_freq != nullptr;
    bool live = t < P.rows;
    int at = -1;
    int64_t m = 0;
    if (live) {
        at = P.slot[t];
        if (turning) {
            m = P.pos[t];
            live = m >= 0;
            if (live && P.prefix) {
                const int g = P.prefix[t];
                if ((unsigned)g < (unsigned)P.nprefix) m += max(P.prefix_len[g], 0);
            }
        }
    }
    const bool in = live && (unsigned)at < (unsigned)P.nslots, ask = live && P.q != nullptr;
    // channels of the lane's two halves: the pairs' first and second ones, or behind `rot` (or with interleaved pairs) neighbours
    const int npair = P.rot / 16;
    const bool turns = sub < npair;
    int c0, c1;
    if (P.interleaved) { c0 = sub * 16; c1 = c0 + 8; }
    else if (turns) { c0 = sub * 8; c1 = c0 + P.rot / 2; }
    else { c0 = P.rot + (sub - npair) * 16; c1 = c0 + 8; }
    float cs[8], sn[8];
    if (turns && live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double turn = (double)m * (double)P.inv_freq[sub * 8 + i] * 0.15915494309189533577;
            sincospif(2.0f * (float)(turn - rint(turn)), &sn[i], &cs[i]);
            cs[i] *= P.rot_scale;
            sn[i] *= P.rot_scale;
        }
    }
    auto rotate_store = [&](const Raw<T>& ra, const Raw<T>& rb, T* to) {
        if (!turns) {
            store_raw(to + c0, ra);
            store_raw(to + c1, rb);
            return;
        }
        float a[8], b[8], x[8], y[8];
        widen8(ra, a);
        widen8(rb, b);
        if (P.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = a[2 * i] * cs[i] - a[2 * i + 1] * sn[i];
                x[2 * i + 1] = a[2 * i] * sn[i] + a[2 * i + 1] * cs[i];
                y[2 * i] = b[2 * i] * cs[4 + i] - b[2 * i + 1] * sn[4 + i];
                y[2 * i + 1] = b[2 * i] * sn[4 + i] + b[2 * i + 1] * cs[4 + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = a[i] * cs[i] - b[i] * sn[i];
                y[i] = a[i] * sn[i] + b[i] * cs[i];
            }
        }
        store8(to + c0, x);
        store8(to + c1, y);
    };
    const int place_mask = (1 << P.page_log) - 1;
    const T *Q = (const T*)P.q + (int64_t)t * P.qs_row, *K = (const T*)P.K + (int64_t)t * P.ks_row, *V = (const T*)P.V + (int64_t)t * P.vs_row;
    T *qo = (T*)P.q_out + (int64_t)t * P.os_row, *kv = (T*)P.kv;
    for (int hk = blockIdx.y; hk < P.Hkv; hk += gridDim.y) {
        Raw<T> k0{}, k1{}, v0{}, v1{};
        if (in) {
            k0 = load_raw8(K + hk * P.ks_head + c0);
            k1 = load_raw8(K + hk * P.ks_head + c1);
            v0 = load_raw8(V + hk * P.vs_head + sub * 16);
            v1 = load_raw8(V + hk * P.vs_head + sub * 16 + 8);
        }
        constexpr int NQ = 4;
        Raw<T> qa[NQ], qb[NQ];
        auto request = [&](int g0) {
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                if (ask && g0 + i < P.G) {
                    const T* x = Q + (int64_t)(hk * P.G + g0 + i) * P.qs_head;
                    qa[i] = load_raw8(x + c0);
                    qb[i] = load_raw8(x + c1);
                }
        };
        request(0);
        if (in) {
            T* to = kv + key_row(at >> P.page_log, hk, at & place_mask, P.Hkv, P.page_log) * (2 * D);
            rotate_store(k0, k1, to);
            store_raw(to + D + sub * 16, v0);
            store_raw(to + D + sub * 16 + 8, v1);
        }
        for (int g0 = 0; g0 < P.G; g0 += NQ) {
            if (g0) request(g0);
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                if (ask && g0 + i < P.G) rotate_store(qa[i], qb[i], qo + (int64_t)(hk * P.G + g0 + i) * P.os_head);
        }
        float* dl = in ? P.delta + (((size_t)(at >> P.page_log) * P.Hq) << P.page_log) + (at & place_mask) : nullptr;
        if (P.delta_new) {
            for (int g = sub; g < P.G; g += LPR)
                if (in) dl[(size_t)(hk * P.G + g) << P.page_log] = P.delta_new[(hk * P.G + g) * P.delta_ld + t];
        } else {
            float v[2][8];
            widen8(v0, v[0]);
            widen8(v1, v[1]);
            // Heads in blocks of 4 (then 2, then 1). The sums are those of the other kernels that form delta: a chain over each 8 channels, then neighbours pairwise, the
            // first two of which a lane has itself.
            auto block = [&](int g0, auto nb_tag) {
                constexpr int NB = decltype(nb_tag)::value;
                float p[NB];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    float part[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float w[8], a = 0.0f;
                        load8(P.W + (size_t)(hk * P.G + g0 + n) * D + sub * 16 + i * 8, w);
#pragma unroll
                        for (int c = 0; c < 8; ++c) a = __fmaf_rn(v[i][c], w[c], a);
                        part[i] = a;
                    }
                    p[n] = __fadd_rn(part[0], part[1]);
                }
                int mine = 0;                 // head of the block this lane ends up with: the low bits of sub, reversed
#pragma unroll
                for (int b = 1, x = NB >> 1; b < NB; b <<= 1, x >>= 1) mine |= (sub & b) ? x : 0;
                block_reduce<NB, LPR>(p, sub);
                const int h = hk * P.G + g0 + mine;
                if (in && sub < NB) dl[(size_t)h << P.page_log] = delta_fixed(p[0], P.A[h]);
            };
            int g0 = 0;
            for (; g0 + 4 <= P.G; g0 += 4) block(g0, std::integral_constant<int, 4>{});
            if (g0 + 2 <= P.G) { block(g0, std::integral_constant<int, 2>{}); g0 += 2; }
            if (g0 < P.G) block(g0, std::integral_constant<int, 1>{});
        }
    }
}

template <typename T, int D>
int append(const Append& P, cudaStream_t st) {
    constexpr int kRows = kThreads / (D / 16);
    const int tiles = (P.rows + kRows - 1) / kRows;
    const int split = std::max(1, std::min(P.Hkv, 8 * 148 / tiles));
    return launch_overlapped(append_kernel<T, D>, dim3(tiles, split), dim3(kThreads), 0, st, 1, P);
}

}  // namespace

int launch_cache_append(const Cache& C, const Rotation& rot, const void* q, const void* K, const void* V, const float* W, const float* A, const float* delta_new,
                        int64_t delta_ld, const int32_t* slot, const int32_t* pos, const int32_t* prefix, const int32_t* prefix_len, int nprefix, void* q_out, void* kv,
                        float* delta, cudaStream_t st) {
    Append P = {q, K, V, W, A, delta_new, rot.inv_freq, slot, pos, prefix, prefix_len, q_out, kv, delta, delta_ld, C.qs[0], C.qs[1], C.ks[0], C.ks[1],
                C.vs[0], C.vs[1], C.os[0], C.os[1], rot.scale, C.rows, C.Hq, C.Hkv, C.G, C.page_log, C.num_pages << C.page_log, nprefix, rot.rot, rot.interleaved};
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? append<__nv_bfloat16, 128> : append<__nv_bfloat16, 64>) : (C.d == 128 ? append<float, 128> : append<float, 64>);
    return f(P, st);
}

}  // namespace dma
