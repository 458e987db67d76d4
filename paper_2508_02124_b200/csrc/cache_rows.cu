// A step's rows into the paged cache of the element type (include/dma.h, dma_cache_append): q and K rotated by their positions, V as it is, delta of V.
//
// d / 16 lanes own a row. A lane has the 16 channels of a head whose pairs turn by the same eight angles, whichever of the two pairings is asked for, so that it forms eight
// sines and cosines per row and turns its part of every head with them. Angles: position times frequency in turns, in 64 bits, less the whole turns; fp32 from there on.
// Bound by memory: a lane copies what it will use into shared memory a stage ahead, without registers or barriers. 16384 rows of 32 and 8 heads, d = 128: 76 us, 5.3 TB/s (bytes alone 62;
// with loads into registers 103 to 88, with the sampling weights read through the L1 94; without forming delta 70). 64 rows 4.7 us: three trips to memory.
#include <algorithm>
#include <type_traits>

#include "delta_fixed.cuh"
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kStages = 2;

template <typename T> using Raw = typename RawOf<T>::type;
template <typename T> constexpr int kQueries = sizeof(T) == 2 ? 4 : 2;            // of a stage
template <typename T> constexpr int stage_bytes = (4 + 2 * kQueries<T>) * ((int)sizeof(T) / 2) * 16;      // of a thread

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

template <typename T, int D, int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) append_kernel(Append P) {
    constexpr int LPR = D / 16, RPW = 32 / LPR, kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR, grp = lane / LPR;
    pdl_enter();
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
    // z of a warp's rows, and delta from it for many heads at once: 100 instructions one behind the other, which every block of heads would wait for
    constexpr int kPending = 32;
    __shared__ float sZ[kWarps][kPending][RPW];
    __shared__ int sHead[kWarps][kPending], sAt[kWarps][RPW];
    int pending = 0;
    if (sub == 0) sAt[warp][grp] = in ? at : -1;
    auto flush = [&]() {
        __syncwarp();
#pragma unroll 2
        for (int i = lane; i < pending * RPW; i += 32) {
            const int h = sHead[warp][i / RPW], to = sAt[warp][i % RPW];
            const float x = delta_fixed(sZ[warp][i / RPW][i % RPW], P.A[h]);
            if (to >= 0) P.delta[(((size_t)(to >> P.page_log) * P.Hq + h) << P.page_log) + (to & place_mask)] = x;
        }
        __syncwarp();
        pending = 0;
    };
    // A stage: a KV head's K and V and NQ of its group's queries, or NQ more of them. A lane copies what it will use to places of its own in shared memory, a stage ahead.
    constexpr int NQ = kQueries<T>, kWide = (int)sizeof(T) / 2, kSlots = (4 + 2 * NQ) * kWide;     // 16-byte places of a lane and stage; of 8 channels
    extern __shared__ uint4 staged[];                             // [kStages][kSlots][kThreads], then the heads' sampling weights
    auto copy = [&](int stage, int c, const T* from) {
#pragma unroll
        for (int i = 0; i < kWide; ++i) ptx::cp_async16_at(ptx::smem_u32(staged + (stage * kSlots + c * kWide + i) * kThreads + tid), from + i * (8 / kWide));
    };
    auto take = [&](int stage, int c) {
        Raw<T> r;
#pragma unroll
        for (int i = 0; i < kWide; ++i) reinterpret_cast<uint4*>(&r)[i] = staged[(stage * kSlots + c * kWide + i) * kThreads + tid];
        return r;
    };
    // KV heads of this CTA: side by side
    const int per = (P.Hkv + gridDim.y - 1) / gridDim.y, first = blockIdx.y * per, heads = min(per, P.Hkv - first), batches = (P.G + NQ - 1) / NQ, units = heads * batches;
    float* sW = reinterpret_cast<float*>(staged + kStages * kSlots * kThreads);
    // (read from global memory they were missed by the L1 between the rows that stream by: 94 us instead of 76. A lane's sixteen in four parts, each next to the other lanes' same part: a
    // group's 16-byte reads meet every bank once)
    if (!P.delta_new)
        for (int i = tid; i < heads * P.G * (D / 4); i += kThreads)
            ptx::cp_async16_at(ptx::smem_u32(sW + i / (D / 4) * D + (i & 3) * (D / 4) + i % (D / 4) / 4 * 4), P.W + (size_t)first * P.G * D + i * 4);
    auto request = [&](int u) {
        if (u < units) {
            const int hk = first + u / batches, g0 = u % batches * NQ, stage = u % kStages;
            if (in && g0 == 0) {
                copy(stage, 0, K + hk * P.ks_head + c0);
                copy(stage, 1, K + hk * P.ks_head + c1);
                copy(stage, 2, V + hk * P.vs_head + sub * 16);
                copy(stage, 3, V + hk * P.vs_head + sub * 16 + 8);
            }
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                if (ask && g0 + i < P.G) {
                    const T* x = Q + (int64_t)(hk * P.G + g0 + i) * P.qs_head;
                    copy(stage, 4 + 2 * i, x + c0);
                    copy(stage, 5 + 2 * i, x + c1);
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) request(i);
    if (turns && live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double turn = (double)m * (double)P.inv_freq[sub * 8 + i] * 0.15915494309189533577;
            sincospif(2.0f * (float)(turn - rint(turn)), &sn[i], &cs[i]);
            cs[i] *= P.rot_scale;
            sn[i] *= P.rot_scale;
        }
    }
#pragma unroll 1
    for (int u = 0; u < units; ++u) {
        const int hk = first + u / batches, q0 = u % batches * NQ, stage = u % kStages;
        request(u + kStages - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        if (u == 0) __syncthreads();                              // (the weights, which others have copied)
#pragma unroll
        for (int i = 0; i < NQ; ++i)
            if (ask && q0 + i < P.G) rotate_store(take(stage, 4 + 2 * i), take(stage, 5 + 2 * i), qo + (int64_t)(hk * P.G + q0 + i) * P.os_head);
        if (q0) continue;
        Raw<T> v0{}, v1{};
        if (in) {
            T* to = kv + key_row(at >> P.page_log, hk, at & place_mask, P.Hkv, P.page_log) * (2 * D);
            rotate_store(take(stage, 0), take(stage, 1), to);
            v0 = take(stage, 2);
            v1 = take(stage, 3);
            store_raw(to + D + sub * 16, v0);
            store_raw(to + D + sub * 16 + 8, v1);
        }
        if (!P.delta_new) {
            float v[2][8];
            widen8(v0, v[0]);
            widen8(v1, v[1]);
            // Heads in blocks of 4 (then 2, then 1). The sums are those of the other kernels that form delta: a chain over each 8 channels, then neighbours pairwise, the
            // first two of which a lane has itself.
            auto block = [&](int g0, auto nb_tag) {
                constexpr int NB = decltype(nb_tag)::value;
                if (pending + NB > kPending) flush();
                float p[NB];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    float part[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float* wp = sW + ((hk - first) * P.G + g0 + n) * D + i * (D / 2) + sub * 4;
                        const float4 wa = *reinterpret_cast<const float4*>(wp), wb = *reinterpret_cast<const float4*>(wp + D / 4);
                        const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
                        float a = 0.0f;
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
                if (sub < NB) {
                    sZ[warp][pending + mine][grp] = p[0];
                    if (grp == 0) sHead[warp][pending + mine] = hk * P.G + g0 + mine;
                }
                pending += NB;
            };
            int g0 = 0;
            for (; g0 + 4 <= P.G; g0 += 4) block(g0, std::integral_constant<int, 4>{});
            if (g0 + 2 <= P.G) { block(g0, std::integral_constant<int, 2>{}); g0 += 2; }
            if (g0 < P.G) block(g0, std::integral_constant<int, 1>{});
        } else if (in) {
            float* to = P.delta + (((size_t)(at >> P.page_log) * P.Hq) << P.page_log) + (at & place_mask);
            for (int h = hk * P.G + sub; h < (hk + 1) * P.G; h += LPR) to[(size_t)h << P.page_log] = P.delta_new[h * P.delta_ld + t];
        }
    }
    if (pending) flush();
}

template <typename T, int D, int kThreads>
int append_rows(const Append& P, cudaStream_t st) {
    constexpr int kRows = kThreads / (D / 16), kWeights = 20 * 1024;
    const int tiles = (P.rows + kRows - 1) / kRows;
    const int64_t group = (int64_t)P.G * D * sizeof(float);       // (weights that are given come for groups of any size)
    // KV heads per CTA: as many as leave eight CTAs per SM (16384 rows of 8: three of them 76 us; eight 84, four 88, two 79, one 92), and so few that their weights take 20 KB, or one
    const int per = std::max(1, std::min({P.Hkv, (int)((int64_t)P.Hkv * tiles / (8 * 148)), (int)std::max<int64_t>(1, kWeights / group)}));
    constexpr int stages = kStages * stage_bytes<T> * kThreads, limit = stages + std::max(kWeights, append_heads(D) * D * (int)sizeof(float));
    const int smem = stages + (P.delta_new ? 0 : per * (int)group);
    // (state of the function, which other threads' calls share: always the limit)
    if (cudaFuncSetAttribute(append_kernel<T, D, kThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, limit) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(append_kernel<T, D, kThreads>, dim3(tiles, (P.Hkv + per - 1) / per), dim3(kThreads), smem, st, 1, P);
}
template <typename T, int D>
int append(const Append& P, cudaStream_t st) {
    // (256 threads share the weights where there are four such CTAs per SM: 16384 rows 76 us against 83 by 128)
    return (int64_t)P.rows * P.Hkv * (D / 16) >= 4 * 148 * 256 ? append_rows<T, D, 256>(P, st) : append_rows<T, D, 128>(P, st);
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
