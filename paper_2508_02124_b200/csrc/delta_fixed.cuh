// The fixed fp32 arithmetic of the dynamic weights (Eq. delta_calc): what every kernel that forms a delta goes through, so that a key's
// weight has the same bits wherever it is computed.
#pragma once

#include "common.cuh"

namespace dma {

// ---- fixed-order fp32 routines: every step is one correctly rounded IEEE operation -----------------------

__device__ __forceinline__ float exp_fixed(float x) {
    x = fminf(fmaxf(x, -87.0f), 88.0f);
    const float magic = 12582912.0f;
    float t = __fmul_rn(x, 0x1.715476p+0f);
    float n = __fadd_rn(__fadd_rn(t, magic), -magic);
    float r = __fmaf_rn(n, -0x1.62e4p-1f, x);
    r = __fmaf_rn(n, -0x1.7f7d1cp-20f, r);
    float q = 0x1.a01a02p-13f;
    q = __fmaf_rn(q, r, 0x1.6c16c2p-10f);
    q = __fmaf_rn(q, r, 0x1.111112p-7f);
    q = __fmaf_rn(q, r, 0x1.555556p-5f);
    q = __fmaf_rn(q, r, 0x1.555556p-3f);
    q = __fmaf_rn(q, r, 0.5f);
    q = __fmaf_rn(q, r, 1.0f);
    q = __fmaf_rn(q, r, 1.0f);
    return __fmul_rn(q, __int_as_float(((int)n + 127) << 23));
}

__device__ __forceinline__ float log1p_fixed(float t) {
    float s = __fdiv_rn(t, __fadd_rn(2.0f, t));
    float u = __fmul_rn(s, s);
    float q = 0x1.111112p-4f;
    q = __fmaf_rn(q, u, 0x1.3b13b2p-4f);
    q = __fmaf_rn(q, u, 0x1.745d18p-4f);
    q = __fmaf_rn(q, u, 0x1.c71c72p-4f);
    q = __fmaf_rn(q, u, 0x1.24924ap-3f);
    q = __fmaf_rn(q, u, 0x1.99999ap-3f);
    q = __fmaf_rn(q, u, 0x1.555556p-2f);
    q = __fmaf_rn(q, u, 1.0f);
    return __fmul_rn(__fmul_rn(2.0f, s), q);
}

__device__ __forceinline__ float delta_fixed(float z, float a) {
    float sp = __fadd_rn(fmaxf(z, 0.0f), log1p_fixed(exp_fixed(-fabsf(z))));
    return exp_fixed(__fmul_rn(a, sp));
}

// eight consecutive channels of one value row as fp32
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
    uint4 a = *reinterpret_cast<const uint4*>(p);
    uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}

// eight consecutive channels of one value row, as loaded (converted to fp32 only when the chain runs)
struct Raw8f { float4 a, b; };
__device__ __forceinline__ Raw8f load_raw8(const float* p) { return {*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)}; }
__device__ __forceinline__ uint4 load_raw8(const __nv_bfloat16* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void widen8(const Raw8f& r, float (&v)[8]) {
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w; v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void widen8(const uint4& a, float (&v)[8]) {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
template <typename T> struct RawOf { using type = uint4; };
template <> struct RawOf<float> { using type = Raw8f; };

// Sum over the LPR lanes of a row group of NB per-lane partials (one per head of a block of NB heads), in the order of the
// xor butterfly (adjacent lanes first: a balanced pairwise tree over the row's 8-channel chunks). The first log2(NB) levels
// are "transposing": a lane keeps half of its values and hands the other half to its partner, so the block costs
// log2(NB) + ... shuffles in all instead of NB log2(LPR) (the additions are the same, and IEEE addition commutes, so the
// bits are those of the plain butterfly). On return p[0] of lane `sub` is the complete sum of head bitrev(sub mod NB) of
// the block (the same value in every lane of the group with those low bits).
template <int NB, int LPR>
__device__ __forceinline__ void block_reduce(float (&p)[NB], int sub) {
    int keep = NB >> 1;
#pragma unroll
    for (int m = 1; m < LPR; m <<= 1) {
        if (keep >= 1) {
            const bool up = (sub & m) != 0;
#pragma unroll
            for (int q = 0; q < NB / 2; ++q) {
                if (q < keep) {
                    const float stay = up ? p[q + keep] : p[q];
                    const float give = up ? p[q] : p[q + keep];
                    p[q] = __fadd_rn(stay, __shfl_xor_sync(0xffffffffu, give, m));
                }
            }
            keep >>= 1;
        } else {
            p[0] = __fadd_rn(p[0], __shfl_xor_sync(0xffffffffu, p[0], m));
        }
    }
}

}  // namespace dma
