// Attention of decoding over the paged 4-bit cache (include/dma.h, dma_cache4_decode): every (row, query head) attends to its kept keys (cache4_select.cu), with delta as
// the bias.
//
// Kernels
//   attn_kernel          bf16, tensor cores: a group's heads together, over the union of their kept keys, the work dealt out by the rows' lengths; the CTA that finishes
//                        a row last adds its pieces
//   simt_attn_kernel     fp32, and bf16 on request, CUDA cores: per (row, query head, split of the keys)
//   simt_combine_kernel  the splits' partials -> o, lse
#include <algorithm>
#include <climits>

#include "cache4_decode.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

// CUDA cores, fp32 throughout. A warp looks at 32 keys at a time, a lane per key, and queues the kept ones; eight lanes take one of them, with d / 8
// channels per lane, so that four keys run side by side. Warps and splits take words of 32 keys in turn, each with its own running
// maximum; partials (m, l, o) meet in shared memory and, where a row has several splits, in simt_combine_kernel.
constexpr int kSimtWarps = 4, kSimtSplits = 64;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kSimtWarps) simt_attn_kernel(Rows R, const T* q, const uint8_t* codes, const uint32_t* scales, const unsigned long long* weakest,
                                                                    T* o, float* lse, float* partial, int32_t* status, int Hkv, int G, float scale, int64_t qs_row, int64_t qs_head,
                                                                    int64_t os_row, int64_t os_head) {
    constexpr int C = D / 8;                                      // channels of a lane
    __shared__ size_t sRow[kSimtWarps][32];
    __shared__ float sDelta[kSimtWarps][32];
    __shared__ float sM[kSimtWarps], sL[kSimtWarps], sO[kSimtWarps][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7, grp = lane >> 3;
    const int item = blockIdx.x, t = item / R.Hq, h = item % R.Hq, hk = h / G, split = blockIdx.y, nsplit = gridDim.y;
    pdl_enter(R.table, R.seq, R.pos, R.delta, q, codes, scales, weakest, o, lse, partial, status);
    if (item == 0 && split == 0 && tid == 0) *status = 0;
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
            s = odd_pair(kp) ? NAN : fmaf(s, pair_s(kp), qsum * pair_z(kp));       // (infinities of both signs, or NaN)
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
    // (the splits' maxima and sums in one go, their values eight at a time: one after the other took 9.8 us for 37 splits, this 6.3)
    __shared__ float sM[kSimtSplits], sL[kSimtSplits];
    static_assert(kSimtSplits <= D && kSimtSplits % 8 == 0, "a thread has a split at most");
    if (c < kSimtSplits) {
        sM[c] = c < nsplit ? in[c * (D + 2)] : -INFINITY;
        sL[c] = c < nsplit ? in[c * (D + 2) + 1] : 0.0f;
    }
    float a = 0.0f, sum = 0.0f, top = -INFINITY;
    __syncthreads();
    for (int x = 0; x < nsplit; ++x) top = fmaxf(top, sM[x]);
    for (int x0 = 0; x0 < nsplit; x0 += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = x0 + k < nsplit ? in[(x0 + k) * (D + 2) + 2 + c] : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float m = sM[x0 + k], l = sL[x0 + k], f = m == -INFINITY ? (l == 0.0f ? 0.0f : 1.0f) : expf(m - top);
            sum += l * f;
            a += v[k] * f;
        }
    }
    store_as(o + t * os_row + h * os_head + c, sum == 0.0f ? 0.0f : a / sum);
    if (c == 0) lse[item] = top + logf(sum);
}

// ---- bf16 on the tensor cores ------------------------------------------------------------------------------------------------------
// A CTA has up to eight query heads of a group (one KV head) and a range of its row's keys; its four warps go through 64 keys in turn, each by itself:
//   scan     a lane per key tests its weight against every head's weakest kept key; keys that some head keeps are queued, with the heads' biases
//            (-inf where a head drops the key), so that a key that several heads keep is read and expanded once
//   gather   32 queued keys at a time, codes and scales, by cp.async into one of the warp's stages while the stage before is used
//   attend   S^T = K q^T and O^T += V^T P^T by mma.m16n8k16 (keys, then channels, by heads). The codes are expanded as little as possible: a code n in the high half of a half's
//            low byte is the subnormal number n 2^-20, exactly, and the eight codes of a word take three shifts and four masks. A group of 64 channels is a chain of four products,
//            whose sum takes the group's scale, and with the query's own sum over the group its zero, in fp32; the query goes in as halves, scaled by a power of two per head and
//            group (its 8 bits survive down to 2^-31 of the largest channel there, and what is lost below that is less than the rounding of the sums). Softmax in registers, with a
//            running maximum per warp and head. Of V the scale goes into the weight, P s in two halves, its rounding and what that leaves, scaled by a power of two per head and
//            group that follows the largest (WarpState): 2^-22 of a weight, and of the small ones 2^-32 of the largest, which is less than the sums' own rounding in fp32. z P is
//            summed in fp32. With up to four heads the operand's columns 4 to 7 hold the same heads again: their lanes take the second 16 keys through the softmax, and in the
//            products of V they hold the low halves (one half per weight was 1.4 % faster; with eight heads per group, whose low halves are products of their own, 7 %).
//            What the products cut: the tensor core adds the 16 addends of an element, and the sum so far, above 2^-25 of the largest one's power of two, and a subnormal operand
//            counts as 2^-14 there whatever it is (both measured). So an addend loses up to 2^-19 of a code's step by the largest weight among its 16 keys, or by the largest
//            channel. With codes in the lowest bits, which take two shifts less, it was 2^-15: 118 us instead of 123, but a key that outweighs 16 others 2^15 times left nothing of
//            them. In the highest bits, a shift more, it is 2^-21, and 126 us. Sums of V begin anew with every 32 keys and are added in fp32, to nearest (125 us): one chain of products
//            over all keys is cut at each of them, always towards zero, and the codes' part and the zeros' nearly cancel (of 64K kept keys' outputs 25 % then rounded elsewhere than
//            the exact ones, now 1.5 %; of 2048 kept of 16K 0.5 and 0.2 %).
// 64 rows of 1 to 16K keys, 32 / 8 heads of 128, w = 2048: 125 us for 414 MB read, 3.3 TB/s, 890 instructions per 32 keys of a union. No unit is at its limit: 55 % of the issue
// slots, 54 % of the integer pipe, 16 % of the tensor pipe. What the time is made of is the chain of test, queue and gather that every warp goes through before it attends, with three
// warps per scheduler to take turns: without the attending 89 us. (Of an earlier form at 113 us: with all pages in the L2 110; sixteen warps per SM instead of twelve, with stages
// that are swizzled to fit, 118; eight with three stages 133 where twelve took 119.) 256 rows of 4096 keys, w = 1024: 247 us, 4.2 TB/s.
// (tcgen05 needs 64 rows of A at least, of which a decoding step has the group's 1 to 8 heads or, turned around, the keys: then the expanded codes would
// have to go through shared memory once more. mma.sync takes them from the registers that the expansion leaves them in, and its rate is not what bounds this kernel.)
constexpr int kBatch = 32, kStages = 2;
constexpr int kRing = 4 * kBatch;           // queue: a batch that is on its way, one that is full, and what a turn's 64 keys may add
// a key's codes and scales in a stage; 32 modulo 128 (or its negative): the rows of a fragment meet every bank once
__host__ __device__ constexpr int key_pitch(int d) { return d == 128 ? 160 : 96; }
template <int D, int kH, int kW>
struct AttnShape {
    static constexpr int kWarps = kW, kThreads = 32 * kW;
    static constexpr int kCols = kH <= 4 ? 4 : 8;                 // heads with a bias slot
    static constexpr int NG = D / kGroup;
    static constexpr int kPitch = key_pitch(D);
    struct alignas(16) Warp {
        uint8_t data[kStages][kBatch * kPitch];
        float bias[kRing][kCols];
        size_t off[kRing];                                        // the key's codes, in bytes from the pool's first
    };
    struct Merge { float o[kWarps][kCols][D]; };
    using Query = uint2[NG][4][32];                               // operand fragments, the same for every warp
    static constexpr size_t kBytes = sizeof(Warp) * kWarps > sizeof(Merge) ? sizeof(Warp) * kWarps : sizeof(Merge);
};
constexpr int kAttnCtas = 3 * 148;

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp8(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t halves(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// a word's codes in four pairs of halves: pair s holds codes s and s + 4, times 2^-20
__device__ __forceinline__ void expand_word(uint32_t x, uint32_t (&d)[4]) {
    d[0] = x << 4 & 0x00f000f0u;
    d[1] = x & 0x00f000f0u;
    d[2] = x >> 4 & 0x00f000f0u;
    d[3] = x >> 8 & 0x00f000f0u;
}
__device__ __forceinline__ float ex2f(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

constexpr float kLog2e = 1.4426950408889634f;

// The heads' softmax state and sums of a warp, in the layout of the accumulators: this lane's columns are heads 2 (lane % 4) and the next one, modulo 4 where there are
// up to four. o is in units of 2^-20 f; f, a power of two, brings the largest weight so far, wref, to 2^7 .. 2^8.
template <int D>
struct WarpState {
    static constexpr int NG = D / kGroup;
    float o[NG][4][4], oz[NG][2], f[NG][2], wref[NG][2], m[2], l[2];
    float qsum[NG][2], scale[NG][2];
};

// 32 keys of a stage. odd (of the warp): some scale is not finite; a head that does not keep the key is to get nothing of it. One instance of this code per kernel:
// with six, a warp waited 4.2 cycles per instruction for the instruction itself (an earlier form, at the 64 rows above: 285 us, with one 210).
template <int D, int kH>
__device__ __forceinline__ void attend(WarpState<D>& W, const uint2 (&q)[D / kGroup][4][32], const uint8_t* data, const float (*bias)[kH <= 4 ? 4 : 8], bool odd) {
    constexpr int NG = D / kGroup, kPitch = key_pitch(D), kCols = kH <= 4 ? 4 : 8, kSets = kH <= 4 ? 1 : 2;       // sets of 16 keys by 8 columns that a lane takes through the softmax
    const int lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3, kr = r ^ (r >> 2 & 1), col = (2 * t) % kCols;
    float c[kSets][NG][4];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float two[2][4];
        uint2 qf[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) qf[s] = q[g][s][lane];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* ka = data + (16 * i + kr) * kPitch + g * 32 + t * 8;
            const uint2 a = *reinterpret_cast<const uint2*>(ka), b = *reinterpret_cast<const uint2*>(ka + 8 * kPitch);
            uint32_t a0[4], a1[4], a2[4], a3[4];
            expand_word(a.x, a0);
            expand_word(b.x, a1);
            expand_word(a.y, a2);
            expand_word(b.y, a3);
            two[i][0] = two[i][1] = two[i][2] = two[i][3] = 0.0f;
#pragma unroll
            for (int s = 0; s < 4; ++s) mma16816(two[i], a0[s], a1[s], a2[s], a3[s], qf[s].x, qf[s].y);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (kSets == 1) c[0][g][e] = t < 2 ? two[0][e] : two[1][e];
            else { c[0][g][e] = two[0][e]; c[1][g][e] = two[1][e]; }
        }
    }
    float x[kSets][4];
    uint32_t sv[kSets][2][NG];                                    // V's pairs of the lane's keys
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
        const int key = 16 * (kSets == 1 ? t >> 1 : i) + kr;
        const uint8_t* ka = data + key * kPitch + D;
        const uint8_t* kb = ka + 8 * kPitch;
        uint32_t pa[2 * NG], pb[2 * NG];
        if constexpr (NG == 2) {
            const uint4 a = *reinterpret_cast<const uint4*>(ka), b = *reinterpret_cast<const uint4*>(kb);
            pa[0] = a.x; pa[1] = a.y; pa[2] = a.z; pa[3] = a.w;
            pb[0] = b.x; pb[1] = b.y; pb[2] = b.z; pb[3] = b.w;
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(ka), b = *reinterpret_cast<const uint2*>(kb);
            pa[0] = a.x; pa[1] = a.y;
            pb[0] = b.x; pb[1] = b.y;
        }
        const float2 ba = *reinterpret_cast<const float2*>(&bias[key][col]), bb = *reinterpret_cast<const float2*>(&bias[key + 8][col]);
        float2 xa = ba, xb = bb;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const float sa = pair_s(pa[g]), za = pair_z(pa[g]), sb = pair_s(pb[g]), zb = pair_z(pb[g]);
            const float2 qs = make_float2(W.qsum[g][0], W.qsum[g][1]), sc = make_float2(W.scale[g][0], W.scale[g][1]);
            xa = ptx::fma2(ptx::fma2(make_float2(sa, sa), make_float2(c[i][g][0], c[i][g][1]), ptx::mul2(make_float2(za, za), qs)), sc, xa);
            xb = ptx::fma2(ptx::fma2(make_float2(sb, sb), make_float2(c[i][g][2], c[i][g][3]), ptx::mul2(make_float2(zb, zb), qs)), sc, xb);
            sv[i][0][g] = pa[NG + g];
            sv[i][1][g] = pb[NG + g];
        }
        x[i][0] = xa.x; x[i][1] = xa.y; x[i][2] = xb.x; x[i][3] = xb.y;
        if (odd) {                                                // (values of a group without finite scale are NaN, or infinities of both signs)
            bool na = false, nb = false;
#pragma unroll
            for (int g = 0; g < NG; ++g) { na = na || odd_pair(pa[g]); nb = nb || odd_pair(pb[g]); }
            x[i][0] = ba.x == -INFINITY ? -INFINITY : na ? NAN : x[i][0];
            x[i][1] = ba.y == -INFINITY ? -INFINITY : na ? NAN : x[i][1];
            x[i][2] = bb.x == -INFINITY ? -INFINITY : nb ? NAN : x[i][2];
            x[i][3] = bb.y == -INFINITY ? -INFINITY : nb ? NAN : x[i][3];
        }
    }
    // Over the lanes that hold the same head's other keys
    auto over_keys = [&](float v) {
#pragma unroll
        for (int o = kSets == 1 ? 2 : 4; o < 32; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    };
    // The maximum that the exponentials refer to moves only when it is passed by more than 5, and the weights' power of two when one of them would pass 2^15: the sums
    // are rescaled rarely.
    float mx[2] = {fmaxf(x[0][0], x[0][2]), fmaxf(x[0][1], x[0][3])};
    if constexpr (kSets == 2) {
        mx[0] = fmaxf(mx[0], fmaxf(x[1][0], x[1][2]));
        mx[1] = fmaxf(mx[1], fmaxf(x[1][1], x[1][3]));
    }
    bool move = __any_sync(0xffffffffu, mx[0] > W.m[0] + 5.0f || mx[1] > W.m[1] + 5.0f);
    float fade[2] = {1.0f, 1.0f};
    if (move) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float top = fmaxf(W.m[e], over_keys(mx[e]));
            fade[e] = ex2f((W.m[e] - top) * kLog2e);
            W.m[e] = top;
            W.l[e] *= fade[e];
#pragma unroll
            for (int g = 0; g < NG; ++g) W.oz[g][e] *= fade[e];
        }
    }
    float w[kSets][NG][4];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = ex2f((x[i][e] - W.m[e & 1]) * kLog2e);
        W.l[0] += p[0] + p[2];
        W.l[1] += p[1] + p[3];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const float sa = pair_s(sv[i][0][g]), za = pair_z(sv[i][0][g]), sb = pair_s(sv[i][1][g]), zb = pair_z(sv[i][1][g]);
            w[i][g][0] = p[0] * sa; w[i][g][1] = p[1] * sa; w[i][g][2] = p[2] * sb; w[i][g][3] = p[3] * sb;
            if (odd) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool kept = x[i][e] != -INFINITY;
                    w[i][g][e] = kept ? w[i][g][e] : 0.0f;
                    W.oz[g][e & 1] += kept ? p[e] * (e < 2 ? za : zb) : 0.0f;
                }
            } else {
                W.oz[g][0] = fmaf(p[0], za, fmaf(p[2], zb, W.oz[g][0]));
                W.oz[g][1] = fmaf(p[1], za, fmaf(p[3], zb, W.oz[g][1]));
            }
            most = fmaxf(most, fmaxf(fmaxf(fabsf(w[i][g][0]), fabsf(w[i][g][2])) * W.f[g][0], fmaxf(fabsf(w[i][g][1]), fabsf(w[i][g][3])) * W.f[g][1]));
        }
    }
    move = move || __any_sync(0xffffffffu, most > 32768.0f);
    if (move) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(fabsf(w[0][g][e]), fabsf(w[0][g][e + 2]));             // (scales of the caller's may be negative)
                if constexpr (kSets == 2) top = fmaxf(top, fmaxf(fabsf(w[1][g][e]), fabsf(w[1][g][e + 2])));
                top = fmaxf(over_keys(top), W.wref[g][e] * fade[e]);
                W.wref[g][e] = top;
                const int up = 7 + 127 - (int)(__float_as_uint(top) >> 23);
                const float f = top > 0.0f ? __uint_as_float((uint32_t)(127 + max(-126, min(up, 126))) << 23) : W.f[g][e];
                // (what fades to nothing has no factor: the ratio of the powers may be any)
                const float by = fade[e] == 0.0f ? 0.0f : fade[e] * (f / W.f[g][e]);
                W.f[g][e] = f;
#pragma unroll
                for (int j = 0; j < 4; ++j) { W.o[g][j][e] *= by; W.o[g][j][e + 2] *= by; }
            }
    }
    const int ra = (2 * t) ^ (t >> 1), other = (t >> 1) ? -kPitch : kPitch;       // the row of operand key 2t; key 2t + 1 lies in the other row of the pair
    const uint8_t* vrow = data + ra * kPitch + D / 2 + 4 * r;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        // hi + lo is the weight to 2^-22 of it
        uint32_t b[2][2], low[2][2];
#pragma unroll
        for (int i = 0; i < kSets; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x0 = w[i][g][2 * e] * W.f[g][0], x1 = w[i][g][2 * e + 1] * W.f[g][1];
                const uint32_t hi = halves(x0, x1);
                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                b[i][e] = turn8x8(hi);
                low[i][e] = turn8x8(halves(x0 - back.x, x1 - back.y));
            }
        if constexpr (kSets == 1) {                               // (columns 0 to 3 hold the first 16 keys' weights, 4 to 7 the others': a product takes its keys' high parts in these, their low parts in those)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t other_low = __shfl_xor_sync(0xffffffffu, low[0][e], 16);
                b[1][e] = lane < 16 ? other_low : b[0][e];
                b[0][e] = lane < 16 ? b[0][e] : other_low;
            }
        }
        float sum[4][4] = {};                                     // of the 32 keys: what the products cut stays relative to these, and fp32 additions round to nearest
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* v = vrow + 16 * i * kPitch + g * 32;
            const uint32_t wa = *reinterpret_cast<const uint32_t*>(v), wb = *reinterpret_cast<const uint32_t*>(v + other);
            const uint32_t wc = *reinterpret_cast<const uint32_t*>(v + 8 * kPitch), wd = *reinterpret_cast<const uint32_t*>(v + 8 * kPitch + other);
            uint32_t a0[4], a1[4], a2[4], a3[4];
            expand_word(__byte_perm(wa, wb, 0x5410), a0);
            expand_word(__byte_perm(wa, wb, 0x7632), a1);
            expand_word(__byte_perm(wc, wd, 0x5410), a2);
            expand_word(__byte_perm(wc, wd, 0x7632), a3);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mma16816(sum[j], a0[j], a1[j], a2[j], a3[j], b[i][0], b[i][1]);
                if constexpr (kSets == 2) mma16816(sum[j], a0[j], a1[j], a2[j], a3[j], low[i][0], low[i][1]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float2 x = ptx::add2(make_float2(W.o[g][j][e], W.o[g][j][e + 1]), make_float2(sum[j][e], sum[j][e + 1]));
                W.o[g][j][e] = x.x; W.o[g][j][e + 1] = x.y;
            }
    }
}

struct AttnArgs {
    Rows R;
    const __nv_bfloat16* q;
    const uint8_t* codes;
    const uint8_t* scales;
    const unsigned long long* weakest;
    __nv_bfloat16* o;
    float *lse, *partial;
    int32_t* status;
    Plan plan;
    int Hkv, G, hb, hpb;                                          // heads of a group, blocks that they come in, heads per block
    float scale;
    int64_t qs_row, qs_head, os_row, os_head;
    int rows;
};

// The last i in [0, n) with first[i] <= x, by a warp: 32 probes per round.
__device__ __forceinline__ int warp_find(const int32_t* first, int n, int x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;                                          // first[lo] <= x; the answer lies in [lo, lo + len)
    while (len > 1) {
        const int step = (len + 31) / 32, at = lo + lane * step;
        const bool in = lane * step < len && first[at] <= x;
        const int last = __popc(__ballot_sync(0xffffffffu, in)) - 1;       // (ascending: a prefix of the lanes)
        const int end = lo + len;
        lo += last * step;
        len = min(step, end - lo);
    }
    return lo;
}

template <int D, int kH, int kW>
__global__ void __launch_bounds__(32 * kW, kW == 4 ? 3 : D == 64 ? 2 : 1) attn_kernel(AttnArgs A) {
    using Sh = AttnShape<D, kH, kW>;
    constexpr int kWarps = kW, kThreads = 32 * kW, NG = Sh::NG, kCols = Sh::kCols, kPitch = Sh::kPitch;
    extern __shared__ __align__(16) uint8_t attn_smem[];
    __shared__ float sM[kWarps][kCols], sL[kWarps][kCols];
    __shared__ typename Sh::Query sQ;
    __shared__ int sTicket;
    auto& M = *reinterpret_cast<typename Sh::Merge*>(attn_smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, t4 = lane & 3;
    auto& S = reinterpret_cast<typename Sh::Warp*>(attn_smem)[warp];
    Rows& R = A.R;
    pdl_enter(R.table, R.seq, R.pos, R.delta, A.q, A.codes, A.scales, A.weakest, A.o, A.lse, A.partial, A.status, A.plan.ustart, A.plan.tickets);
    if (blockIdx.x == 0 && threadIdx.x == 0) *A.status = 0;
    const int per_row = A.Hkv * A.hb;
    int at = 0, until = 1, E = 1, U = 1;                          // units of this CTA; without a plan the CTA's item
    const int cta = blockIdx.x;
    if (A.plan.ustart) {
        U = A.plan.ustart[A.rows];
        E = min((int)gridDim.x, max(U / 2, 1));                   // (two units at least)
        if (cta >= E || U == 0) return;
        at = (int)((int64_t)cta * U / E);
        until = (int)((int64_t)(cta + 1) * U / E);
    }
    const int begin = at;
    while (at < until) {
        int t, i, n, seq, k0 = 0, k1, u0 = 0, u1 = 1;
        if (A.plan.ustart) {
            t = warp_find(A.plan.ustart, A.rows, at);
            const int first = A.plan.ustart[t], units = (A.plan.ustart[t + 1] - first) / per_row;
            i = (at - first) / units;
            u0 = first + i * units;
            u1 = u0 + units;
            n = R.visible(t, seq);
            const int e = min(u1, until);
            // units of 64 keys or a multiple, the last one of the item without any
            const int span = (int)((((uint32_t)n + units - 2) / max(units - 1, 1) + 63) / 64 * 64);
            k0 = min((int64_t)n, (int64_t)(at - u0) * span);
            k1 = min((int64_t)n, (int64_t)(e - u0) * span);
            at = e;
        } else {
            t = cta / per_row;
            i = cta % per_row;
            n = R.visible(t, seq);
            if (n < 0) return;
            k1 = n;
            at = until;
        }
        const int hk = i / A.hb, h0 = hk * A.G + (i % A.hb) * A.hpb, heads = min(A.hpb, (hk + 1) * A.G - h0);
        const int32_t* pages = R.table + seq * R.ld;
        // 64 keys per turn, a lane's two neighbouring keys in every head, requested a turn before they are tested, and their page two
        float2 dl[kH] = {};                                       // (of a lane without a page, or a head that is none: not looked at)
        int page;
        auto page_of = [&](int j) {
            if (j >= k1) return -1;
            const int p = pages[j >> R.page_log];
            return (unsigned)p < (unsigned)R.num_pages ? p : -1;
        };
        const float* plane = R.delta + ((size_t)h0 << R.page_log);
        auto request = [&](int j, int p) {
            page = p;
            const float* src = plane + (size_t)p * ((uint32_t)R.Hq << R.page_log) + (j & R.mask());
#pragma unroll
            for (int h = 0; h < kH; ++h) {
                if (p >= 0 && h < heads) dl[h] = *reinterpret_cast<const float2*>(src + (h << R.page_log));
            }
        };
        int j = k0 + warp * 64;
        request(j + 2 * lane, page_of(j + 2 * lane));
        int after = page_of(j + kWarps * 64 + 2 * lane);
        // A head keeps the patterns above its weakest key's, and those equal to it up to that key's index: least[h], the pattern or, past the index, the next one. The turn
        // that the index lies in (first_mixed and later ones, in turns that are none's) is tested key by key. (delta > 0: 1 keeps every key, and an absent one reads as 0.)
        uint32_t least[kH];
        int first_mixed = INT_MAX;
        auto weakest_of = [&](int h, int& last) {
            const unsigned long long k = A.weakest && h < heads ? A.weakest[t * R.Hq + h0 + h] : 0ull;
            last = k ? (int)(0xFFFFFFFFu - (uint32_t)k) : INT_MAX;
            return h < heads ? max((uint32_t)(k >> 32), 1u) : 0xFFFFFFFFu;
        };
#pragma unroll
        for (int h = 0; h < kH; ++h) {
            int last;
            least[h] = weakest_of(h, last);
            if (least[h] != 0xFFFFFFFFu) {
                least[h] += k0 > last;
                if (k0 <= last) first_mixed = min(first_mixed, last);
            }
        }
        // queries: column r of the operand is head r % kCols; channels in the order that the codes come in
        WarpState<D> W;
        {
            const int h = r % kCols;
            uint4 raw[NG][2];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                raw[g][0] = raw[g][1] = make_uint4(0u, 0u, 0u, 0u);
                if (h < heads) {
                    const uint4* src = reinterpret_cast<const uint4*>(A.q + t * A.qs_row + (h0 + h) * A.qs_head + g * kGroup + t4 * 16);
                    raw[g][0] = src[0];
                    raw[g][1] = src[1];
                }
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                uint32_t big = 0u;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t v[4] = {raw[g][e].x, raw[g][e].y, raw[g][e].z, raw[g][e].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) big = max(big, max(v[k] & 0x7fff0000u, v[k] << 16 & 0x7fff0000u));
                }
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                // the power of two of the head's group brings its largest channel to 2^14 .. 2^15
                const int up = max(-113, min(100, 127 + 14 - (int)(big >> 23)));
                const float k = __uint_as_float((uint32_t)(127 + up) << 23);
                float sum = 0.0f;
                uint32_t frag[4][2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t v[4] = {raw[g][e].x, raw[g][e].y, raw[g][e].z, raw[g][e].w};
                    float ch[8];
#pragma unroll
                    for (int n8 = 0; n8 < 4; ++n8) { ch[2 * n8] = __uint_as_float(v[n8] << 16); ch[2 * n8 + 1] = __uint_as_float(v[n8] & 0xffff0000u); }
#pragma unroll
                    for (int n8 = 0; n8 < 8; ++n8) sum += ch[n8];
#pragma unroll
                    for (int s = 0; s < 4; ++s) frag[s][e] = halves(ch[s] * k, ch[s + 4] * k);
                }
                if (warp == 0)
#pragma unroll
                    for (int s = 0; s < 4; ++s) sQ[g][s][lane] = make_uint2(frag[s][0], frag[s][1]);
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                // (in the products' units: codes 2^-20, queries k)
                sum *= k * 0x1p-20f;
                const float unit = A.scale / k * 0x1p20f;
                W.qsum[g][0] = __shfl_sync(0xffffffffu, sum, 8 * t4);
                W.qsum[g][1] = __shfl_sync(0xffffffffu, sum, 8 * t4 + 4);
                W.scale[g][0] = __shfl_sync(0xffffffffu, unit, 8 * t4);
                W.scale[g][1] = __shfl_sync(0xffffffffu, unit, 8 * t4 + 4);
                W.oz[g][0] = W.oz[g][1] = 0.0f;
                W.f[g][0] = W.f[g][1] = 0x1p126f;                 // (whatever weight comes first passes the half's range by it, and sets the power)
                W.wref[g][0] = W.wref[g][1] = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) W.o[g][j][0] = W.o[g][j][1] = W.o[g][j][2] = W.o[g][j][3] = 0.0f;
            }
            W.m[0] = W.m[1] = -3.4e38f;
            W.l[0] = W.l[1] = 0.0f;
        }
        __syncthreads();                                          // (the queries; the last item's have been used)

        // keys queued, batches requested, batches attended to
        int tail = 0, issued = 0, used = 0;
        const uint32_t page_bytes = (uint32_t)(A.Hkv << R.page_log) * D, head_bytes = (uint32_t)(hk << R.page_log) * D;       // (checked: fewer than 2^32)
        constexpr int kLanes = D / 16, kKeys = 32 / kLanes;       // lanes per key, keys per instruction of a gather
        const uint8_t* codes = A.codes + lane % kLanes * 16;
        auto gather = [&](int batch) {
            const int at = batch * kBatch % kRing, count = min(kBatch, tail - batch * kBatch);
            uint8_t* to = S.data[batch % kStages];
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
            const uint32_t dst_codes = dst + lane / kLanes * kPitch + lane % kLanes * 16;
            if (count < kBatch && lane >= count) {                // places without a key: finite, and of no weight
                S.off[at + lane] = S.off[at];
                uint32_t* p = reinterpret_cast<uint32_t*>(to + lane * kPitch + D);
#pragma unroll
                for (int e = 0; e < D / 32; ++e) p[e] = 0u;
#pragma unroll
                for (int e = 0; e < kCols; ++e) S.bias[at + lane][e] = -INFINITY;
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < kBatch; e += kKeys) cp16(dst_codes + e * kPitch, codes + S.off[at + e + lane / kLanes]);
            if (lane < count) {
                const uint8_t* src = A.scales + (S.off[at + lane] >> 3);          // (an eighth of the codes' bytes)
                if constexpr (D == 128) cp16(dst + lane * kPitch + D, src); else cp8(dst + lane * kPitch + D, src);
            }
        };
        while (true) {
            // keys are queued until a batch is full
            while (j < k1 && tail - issued * kBatch < kBatch) {
                const int key = j + 2 * lane;
                float b[2][kCols];
                bool any[2] = {false, false};
#pragma unroll
                for (int h = 0; h < kCols; ++h) b[0][h] = b[1][h] = -INFINITY;
                auto test = [&](int h, uint32_t least0, uint32_t least1) {
                    const bool k0h = __float_as_uint(dl[h].x) >= least0, k1h = __float_as_uint(dl[h].y) >= least1;
                    b[0][h] = k0h ? dl[h].x : -INFINITY;
                    b[1][h] = k1h ? dl[h].y : -INFINITY;
                    any[0] = any[0] || k0h;
                    any[1] = any[1] || k1h;
                };
                if (j + 63 < first_mixed) {
#pragma unroll
                    for (int h = 0; h < kH; ++h) test(h, least[h], least[h]);
                } else {
                    first_mixed = INT_MAX;
#pragma unroll
                    for (int h = 0; h < kH; ++h) {
                        int last;
                        const uint32_t u = weakest_of(h, last), past = u == 0xFFFFFFFFu ? 0u : 1u;
                        test(h, key > last ? u + past : u, key + 1 > last ? u + past : u);
                        const int next = j + kWarps * 64;
                        least[h] = next > last ? u + past : u;
                        if (next <= last) first_mixed = min(first_mixed, last);
                    }
                }
                any[0] = any[0] && page >= 0;
                any[1] = any[1] && page >= 0 && key + 1 < k1;
                const uint32_t ballot[2] = {__ballot_sync(0xffffffffu, any[0]), __ballot_sync(0xffffffffu, any[1])}, below = (1u << lane) - 1u;
                const size_t off = (size_t)(uint32_t)page * page_bytes + (head_bytes + (uint32_t)(key & R.mask()) * D);
                const int n0 = __popc(ballot[0]);
                auto queue = [&](int to, size_t at, const float (&v)[kCols]) {
                    S.off[to % kRing] = at;
                    float4* dst = reinterpret_cast<float4*>(S.bias[to % kRing]);
                    dst[0] = make_float4(v[0], v[1], v[2], v[3]);
                    if constexpr (kCols == 8) dst[1] = make_float4(v[4], v[5], v[6], v[7]);
                };
                if (any[0]) queue(tail + __popc(ballot[0] & below), off, b[0]);
                if (any[1]) queue(tail + n0 + __popc(ballot[1] & below), off + D, b[1]);
                tail += n0 + __popc(ballot[1]);
                j += kWarps * 64;
                request(j + 2 * lane, after);
                after = page_of(j + kWarps * 64 + 2 * lane);
            }
            // the next batch is requested, the one before it is used; behind the last one an empty group keeps the count
            const bool more = tail > issued * kBatch;
            if (!more && used == issued) break;
            __syncwarp();
            if (more) gather(issued++);
            cp_commit();
            if (issued - used == kStages || !more) {
                cp_wait<kStages - 1>();
                __syncwarp();
                const uint8_t* data = S.data[used % kStages];
                bool odd = false;
                const uint32_t* sc = reinterpret_cast<const uint32_t*>(data + lane * kPitch + D);
#pragma unroll
                for (int e = 0; e < D / 32; ++e) odd |= odd_pair(sc[e]);
                attend<D, kH>(W, sQ, data, &S.bias[used * kBatch % kRing], __any_sync(0xffffffffu, odd));
                __syncwarp();
                ++used;
            }
        }

        // the warp's sums: over the lanes that hold a head's other keys
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int o = kH <= 4 ? 2 : 4; o < 32; o <<= 1) {
                W.l[e] += __shfl_xor_sync(0xffffffffu, W.l[e], o);
#pragma unroll
                for (int g = 0; g < NG; ++g) W.oz[g][e] += __shfl_xor_sync(0xffffffffu, W.oz[g][e], o);
            }
        }
        __syncthreads();                                          // (stages become the merge's memory)
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float unit = 1.0f / W.f[g][e & 1];
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = W.o[g][j][e] * unit * 0x1p20f;
                    if (kH <= 4) v[j] += __shfl_xor_sync(0xffffffffu, v[j], 2);
                    v[j] += W.oz[g][e & 1];
                }
                const int h = 2 * t4 + (e & 1), c = g * kGroup + 8 * r + 4 * (e >> 1);
                if (h < kCols) *reinterpret_cast<float4*>(&M.o[warp][h][c]) = make_float4(v[0], v[1], v[2], v[3]);
            }
        if (r == 0 && 2 * t4 < kCols) {
            sM[warp][2 * t4] = W.m[0]; sM[warp][2 * t4 + 1] = W.m[1];
            sL[warp][2 * t4] = W.l[0]; sL[warp][2 * t4 + 1] = W.l[1];
        }
        __syncthreads();
        const bool whole = !A.plan.ustart || (u0 >= begin && u1 <= until);
        const int item = t * per_row + i;
        float* slot = A.partial + (size_t)(2 * cta + (u0 > begin ? 1 : 0)) * kCols * (D + 2);
        auto write_out = [&](int h, int c, float top, float sum, const float (&v)[4]) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            __nv_bfloat162 lo = __floats2bfloat162_rn(v[0] * inv, v[1] * inv), hi = __floats2bfloat162_rn(v[2] * inv, v[3] * inv);
            *reinterpret_cast<uint2*>(A.o + t * A.os_row + (h0 + h) * A.os_head + c) = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
            if (c == 0) A.lse[t * R.Hq + h0 + h] = sum == 0.0f ? -INFINITY : top + logf(sum);
        };
        // thread: four channels of a head
        for (int e = tid; e < heads * (D / 4); e += kThreads) {
            const int h = e / (D / 4), c = e % (D / 4) * 4;
            float top = sM[0][h];
#pragma unroll
            for (int x = 1; x < kWarps; ++x) top = fmaxf(top, sM[x][h]);
            float sum = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int x = 0; x < kWarps; ++x) {
                const float f = ex2f((sM[x][h] - top) * kLog2e);
                const float4 a = *reinterpret_cast<const float4*>(&M.o[x][h][c]);
                sum = fmaf(sL[x][h], f, sum);
                v[0] = fmaf(a.x, f, v[0]); v[1] = fmaf(a.y, f, v[1]); v[2] = fmaf(a.z, f, v[2]); v[3] = fmaf(a.w, f, v[3]);
            }
            if (whole) {
                write_out(h, c, top, sum, v);
            } else {
                *reinterpret_cast<float4*>(slot + 2 * kCols + h * D + c) = make_float4(v[0], v[1], v[2], v[3]);
                if (c == 0) { slot[2 * h] = top; slot[2 * h + 1] = sum; }
            }
        }
        if (!whole) {
            // the CTA that finishes the item last adds its pieces, in their order
            const int c0 = (int)(((int64_t)(u0 + 1) * E - 1) / U), c1 = (int)(((int64_t)u1 * E - 1) / U), pieces = c1 - c0 + 1;
            __threadfence();
            __syncthreads();
            if (tid == 0) sTicket = atomicAdd(&A.plan.tickets[item], 1);
            __syncthreads();
            if (sTicket == pieces - 1) {
                __threadfence();
                // (only the first piece can lie in its CTA's second place)
                constexpr int kSlot = kCols * (D + 2);
                const float* head_piece = A.partial + (size_t)(2 * c0 + (u0 > (int)((int64_t)c0 * U / E) ? 1 : 0)) * kSlot;
                const float* rest = A.partial + (size_t)2 * c0 * kSlot;
                auto piece = [&](int x) { return x == 0 ? head_piece : rest + (size_t)2 * x * kSlot; };
                // maxima and sums of a chunk of pieces by a thread each, then every piece's values
                constexpr int kChunk = kThreads / kCols;
                float2* sml = reinterpret_cast<float2*>(attn_smem);
                float top[2], sum[2], v[2][4];
                constexpr int kTurns = kCols * D / 4 / kThreads < 1 ? 1 : kCols * D / 4 / kThreads;   // (head, four channels) pairs of a thread
#pragma unroll
                for (int n = 0; n < kTurns; ++n) {
                    top[n] = -3.4e38f;
                    sum[n] = v[n][0] = v[n][1] = v[n][2] = v[n][3] = 0.0f;
                }
                for (int x0 = 0; x0 < pieces; x0 += kChunk) {
                    const int count = min(kChunk, pieces - x0);
                    __syncthreads();
                    if (tid < count * kCols) sml[tid] = __ldcg(reinterpret_cast<const float2*>(piece(x0 + tid / kCols)) + tid % kCols);
                    __syncthreads();
#pragma unroll
                    for (int n = 0; n < kTurns; ++n) {
                        const int e = tid + n * kThreads, h = e / (D / 4), c = e % (D / 4) * 4;
                        if (h >= heads) continue;
                        float most = top[n];
                        for (int x = 0; x < count; ++x) most = fmaxf(most, sml[x * kCols + h].x);
                        const float fade = ex2f((top[n] - most) * kLog2e);
                        top[n] = most;
                        sum[n] *= fade;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[n][k] *= fade;
#pragma unroll 8
                        for (int x = 0; x < count; ++x) {
                            const float2 ml = sml[x * kCols + h];
                            const float f = ex2f((ml.x - most) * kLog2e);
                            const float4 a = __ldcg(reinterpret_cast<const float4*>(piece(x0 + x) + 2 * kCols + h * D + c));
                            sum[n] = fmaf(ml.y, f, sum[n]);
                            v[n][0] = fmaf(a.x, f, v[n][0]); v[n][1] = fmaf(a.y, f, v[n][1]); v[n][2] = fmaf(a.z, f, v[n][2]); v[n][3] = fmaf(a.w, f, v[n][3]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < kTurns; ++n) {
                    const int e = tid + n * kThreads, h = e / (D / 4), c = e % (D / 4) * 4;
                    if (h < heads) write_out(h, c, top[n], sum[n], v[n]);
                }
            }
        }
        __syncthreads();                                          // the merge's memory becomes stages
    }
}

// The keys of few rows are cut into as many splits as give an SM eight CTAs, of 256 keys at least (us, 32 heads; one row of 16K keys in 9 splits 33, 18 23, 37 21; of 2K in 2 splits 18, 8 8.0;
// of 512 in 1 split 11.0, 2 7.0 and 3.0 to join them; joining 8 takes 3.1, 37 6.3).
constexpr int kSimtCtas = 148 * 8;
int simt_splits(const Cache& C) {
    const int64_t items = (int64_t)C.rows * C.Hq, keys = (int64_t)C.max_blocks << C.page_log;
    return (int)std::min<int64_t>((kSimtCtas + items - 1) / items, std::min<int64_t>(kSimtSplits, (keys + 255) / 256));
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t weakest_bytes(const Cache& C) { return round256((size_t)C.rows * C.Hq * sizeof(unsigned long long)); }
// heads of a group: blocks of at most eight, of the same size
int head_blocks(const Cache& C) { return (C.G + 7) / 8; }
size_t plan_bytes(const Cache& C) { return round256(((size_t)C.rows + 1 + (size_t)C.rows * C.Hkv * head_blocks(C)) * sizeof(int32_t)); }

template <typename T, int D>
int simt_decode(const Cache& C, const Rows& R, const void* q, const uint8_t* codes, const __nv_bfloat16* scales, const unsigned long long* weakest, void* o, float* lse,
                float* partial, int32_t* status, cudaStream_t st) {
    const int items = C.rows * C.Hq, splits = simt_splits(C);
    const int rc = launch_overlapped(simt_attn_kernel<T, D>, dim3(items, splits), dim3(32 * kSimtWarps), 0, st, 1, R, (const T*)q, codes, (const uint32_t*)scales,
                                     weakest, (T*)o, lse, partial, status, C.Hkv, C.G, C.scale, C.qs[0], C.qs[1], C.os[0], C.os[1]);
    if (rc || splits == 1) return rc;
    return launch_overlapped(simt_combine_kernel<T, D>, dim3(items), dim3(D), 0, st, 1, R, partial, (T*)o, lse, splits, C.os[0], C.os[1]);
}

template <int D, int kH, int kW>
int attn_launch(const AttnArgs& A, int grid, cudaStream_t st) {
    constexpr size_t bytes = AttnShape<D, kH, kW>::kBytes;
    if (cudaFuncSetAttribute(attn_kernel<D, kH, kW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(attn_kernel<D, kH, kW>, dim3(grid), dim3(32 * kW), bytes, st, 1, A);
}
// Eight warps per CTA where every CTA has one short row and all of them run at once: an SM has one of 128 channels or two of 64 (rows of 1000 keys, 8 KV heads; us of four warps and of eight:
// d = 128, 16 rows 15.1 and 12.3, 20 rows 18.1 and 22.6; d = 64, 16 rows 11.4 and 9.6, 30 rows 13.2 and 12.8, 48 rows of 4 KV heads 13.3 and 12.7).
template <int D, int kH>
int tc_decode(const AttnArgs& A, int grid, cudaStream_t st) {
    return !A.plan.ustart && grid <= (D == 64 ? 2 : 1) * 148 ? attn_launch<D, kH, 8>(A, grid, st) : attn_launch<D, kH, 4>(A, grid, st);
}

}  // namespace

size_t cache4_decode_ws_bytes(const Cache& C) {
    const size_t simt = ((size_t)C.rows * C.Hq + kSimtCtas) * (C.d + 2), pieces = (size_t)2 * kAttnCtas * 8 * (C.d + 2);
    return kWsHeaderBytes + weakest_bytes(C) + plan_bytes(C) + std::max(simt, pieces) * sizeof(float);
}

int launch_cache4_decode(const Cache& C, const void* q, const uint8_t* codes, const __nv_bfloat16* scales, const float* delta, const int32_t* table,
                         const int32_t* row_seq, const int32_t* row_pos, void* o, float* lse, void* ws, cudaStream_t st) {
    const Rows R{table, row_seq, row_pos, delta, C.table_ld, C.nseq, C.page_log, C.num_pages, C.max_blocks, C.Hq};
    const int64_t capacity = (int64_t)C.max_blocks << C.page_log;      // (no row sees more keys than the table holds)
    const bool tensor = C.dtype == DMA_BF16 && !(C.flags & DMA_FLAG_SIMT);
    const int hb = head_blocks(C), per_row = C.Hkv * hb;
    unsigned long long* weakest = nullptr;
    // (units of 256 keys: 64 rows of 16K 174 us, of 512 175; one row of 16K 15.7, of 128 16.5, of 512 19.3)
    Plan plan{nullptr, nullptr, per_row, 8, (C.G + hb - 1) / hb, C.w};
    char* at = (char*)ws + kWsHeaderBytes;
    // The work is dealt out where rows may be long, unless short ones come in numbers that even out by themselves (us dealt out and by a CTA per item, 8 KV heads, w half the row:
    // one row of 1024 keys 14.1 and 11.8, of 1536 13.7 and 15.2; 64 rows of up to 4096 65 and 69, 256 rows of up to 4096 209 and 206, of 4096 338 and 314, of 2048 193 and 174).
    const bool even = capacity <= 1024 || (capacity <= 4096 && (int64_t)C.rows * per_row >= 4 * kAttnCtas);
    if (tensor && !even) {
        plan.ustart = reinterpret_cast<int32_t*>(at + weakest_bytes(C));
        plan.tickets = plan.ustart + C.rows + 1;
        while ((int64_t)C.rows * per_row > INT32_MAX / ((capacity >> plan.unit_log) + 2)) ++plan.unit_log;
    }
    int rc;
    if (capacity > C.w) {
        weakest = reinterpret_cast<unsigned long long*>(at);
        if ((rc = launch_cache4_select(C, R, weakest, plan, st))) return rc;
    } else if (plan.ustart) {
        if ((rc = launch_cache4_plan(C, R, plan, st))) return rc;
    }
    float* partial = reinterpret_cast<float*>(at + weakest_bytes(C) + plan_bytes(C));
    if (!tensor) {
        auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? simt_decode<__nv_bfloat16, 128> : simt_decode<__nv_bfloat16, 64>)
                                     : (C.d == 128 ? simt_decode<float, 128> : simt_decode<float, 64>);
        return f(C, R, q, codes, scales, weakest, o, lse, partial, (int32_t*)ws, st);
    }
    const int hpb = (C.G + hb - 1) / hb, grid = plan.ustart ? kAttnCtas : C.rows * per_row;
    const AttnArgs A{R, (const __nv_bfloat16*)q, codes, (const uint8_t*)scales, weakest, (__nv_bfloat16*)o, lse, partial, (int32_t*)ws, plan, C.Hkv, C.G, hb, hpb, C.scale,
                     C.qs[0], C.qs[1], C.os[0], C.os[1], C.rows};
    if (C.d == 128) return hpb == 1 ? tc_decode<128, 1>(A, grid, st) : hpb == 2 ? tc_decode<128, 2>(A, grid, st) : hpb <= 4 ? tc_decode<128, 4>(A, grid, st) : tc_decode<128, 8>(A, grid, st);
    return hpb == 1 ? tc_decode<64, 1>(A, grid, st) : hpb == 2 ? tc_decode<64, 2>(A, grid, st) : hpb <= 4 ? tc_decode<64, 4>(A, grid, st) : tc_decode<64, 8>(A, grid, st);
}

}  // namespace dma
