// Second step of dma_cache_decode (include/dma.h): the rows' attention over their own keys that they keep.
//
// A warp, or a team of them, per (row, query head): its part of the keys' weights is read again, the kept ones' slots listed, their rows fetched 16 at a time and multiplied. Where a row
// keeps all keys, whatever their weights, a group's heads share the work: every warp takes 16 keys in turn, for all of them.
// FIG
#include <algorithm>

#include "cache4_decode.cuh"
#include "delta_fixed.cuh"
#include "prefix_decode.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kRoom = 640;         // kept keys of a warp: a sweep's 512 more than what waits for the next one

struct OwnShared {
    float m[kWarps], l[kWarps], all_m[kWarps][8], all_l[kWarps][8];
};

__device__ __forceinline__ float warp_max(float x) {              // (NaN only where all are)
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <bool kTrans>
__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (kTrans) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Attention of a warp over keys that lie in shared memory (K's row, V's, kPitch bytes apart), a stage of them at a time; `bias` by key. Maximum and sum in natural units at the end.
template <typename T, int D> struct Attend;

// fp32, on the CUDA cores: eight lanes take a key, 4 channels of every 32 each.
template <int D>
struct Attend<float, D> {
    static constexpr int kStage = 8, kPitch = 2 * D * 4 + 16, C = D / 8;
    float q[C], acc[C], m = -INFINITY, l = 0.0f;
    __device__ __forceinline__ void start(const float* row, float scale, int lane) {
#pragma unroll
        for (int x = 0; x < C; ++x) {
            acc[x] = 0.0f;
            q[x] = row[x / 4 * 32 + (lane & 7) * 4 + x % 4] * scale;
        }
    }
    float s[kStage / 4];                                          // of the keys lane / 8, lane / 8 + 4
    __device__ __forceinline__ void scores(const uint8_t* keys, const uint2* list, int count, int lane) {
#pragma unroll
        for (int i = 0; i < kStage; i += 4) {
            const int e = i + (lane >> 3);
            const float* row = reinterpret_cast<const float*>(keys + e * kPitch) + (lane & 7) * 4;
            float s = 0.0f;
            if (e < count) {
#pragma unroll
                for (int x = 0; x < C; x += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(row + x * 8);
                    s = fmaf(q[x], k.x, s); s = fmaf(q[x + 1], k.y, s); s = fmaf(q[x + 2], k.z, s); s = fmaf(q[x + 3], k.w, s);
                }
            }
#pragma unroll
            for (int x = 1; x < 8; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            this->s[i / 4] = e < count ? s + __uint_as_float(list[e].x) : -INFINITY;
        }
    }
    __device__ __forceinline__ void values(uint8_t* keys, int count, int lane) {
#pragma unroll
        for (int i = 0; i < kStage; i += 4) {
            const int e = i + (lane >> 3);
            const float* row = reinterpret_cast<const float*>(keys + e * kPitch) + (lane & 7) * 4;
            const float s = this->s[i / 4];
            float top = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 8));
            top = fmaxf(m, fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16)));
            // (a NaN score leaves no maximum and makes the sum NaN; so does one of +inf)
            const float ref = top == -INFINITY ? 0.0f : top, fade = m == -INFINITY ? 0.0f : expf(m - ref);
            m = top;
            l *= fade;
#pragma unroll
            for (int x = 0; x < C; ++x) acc[x] = fade == 0.0f ? 0.0f : acc[x] * fade;
            if (e < count) {
                const float w = expf(s - ref);
                l += w;
#pragma unroll
                for (int x = 0; x < C; x += 4) {
                    const float4 v = *reinterpret_cast<const float4*>(row + D + x * 8);
                    acc[x] = fmaf(w, v.x, acc[x]); acc[x + 1] = fmaf(w, v.y, acc[x + 1]); acc[x + 2] = fmaf(w, v.z, acc[x + 2]); acc[x + 3] = fmaf(w, v.w, acc[x + 3]);
                }
            }
        }
    }
    // o to shared memory; (m, l) in every lane
    __device__ __forceinline__ void end(float* o, int lane) {
#pragma unroll
        for (int x = 8; x < 32; x <<= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, x);
#pragma unroll
            for (int y = 0; y < C; ++y) acc[y] += __shfl_xor_sync(0xffffffffu, acc[y], x);
        }
        if (lane < 8)
#pragma unroll
            for (int x = 0; x < C; ++x) o[x / 4 * 32 + lane * 4 + x % 4] = acc[x];
    }
};

// bf16: 16 keys by mma.sync, S = K q with the query as one of the eight columns, o = V^T p with p in two columns, the bf16 number next to it and what that leaves (2^-16 of a weight), for
// nothing: a row of one head has one column to multiply, so that tcgen05's tiles would be empty, and keys go through shared memory once. A sixth of the instructions of FMAs.
template <int D>
struct Attend<__nv_bfloat16, D> {
    static constexpr int kStage = 16, kPitch = 2 * D * 2 + 16;     // (rows 16 bytes off: the eight rows of a matrix lie in different banks)
    uint32_t q[D / 16][2];
    float acc[D / 16][4], m = -INFINITY, l = 0.0f, c1;             // m in log2 units
    __device__ __forceinline__ void start(const __nv_bfloat16* row, float scale, int lane) {
        c1 = scale * 1.4426950408889634f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = 0.0f;
#pragma unroll
            for (int y = 0; y < 2; ++y) q[x][y] = lane < 4 ? *reinterpret_cast<const uint32_t*>(row + x * 16 + y * 8 + lane * 2) : 0u;
        }
    }
    float x0, x1;                                                 // of lane 4 i: the scores of keys i and i + 8, log2 units
    __device__ __forceinline__ void scores(const uint8_t* keys, const uint2* list, int count, int lane) {
        const uint32_t at_k = ptx::smem_u32(keys) + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + (lane >> 4) * 16;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s1[4] = {0.0f, 0.0f, 0.0f, 0.0f};       // (two chains)
#pragma unroll
        for (int x = 0; x < D / 16; x += 2) {
            uint32_t a[4], b[4];
            ldmatrix<false>(a, at_k + x * 32);
            ldmatrix<false>(b, at_k + x * 32 + 32);
            mma_16816(s, a, q[x][0], q[x][1]);
            mma_16816(s1, b, q[x + 1][0], q[x + 1][1]);
        }
        const int e = lane >> 2;
        x0 = (lane & 3) == 0 && e < count ? fmaf(s[0] + s1[0], c1, __uint_as_float(list[e].x) * 1.4426950408889634f) : -INFINITY;
        x1 = (lane & 3) == 0 && e + 8 < count ? fmaf(s[2] + s1[2], c1, __uint_as_float(list[e + 8].x) * 1.4426950408889634f) : -INFINITY;
    }
    __device__ __forceinline__ void values(uint8_t* keys, int count, int lane) {
        if (count < kStage) {                                     // (0 times what lies there must be 0)
            for (int i = count * (D / 8) + lane; i < kStage * (D / 8); i += 32) *reinterpret_cast<uint4*>(keys + i / (D / 8) * kPitch + D * 2 + i % (D / 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
        }
        const uint32_t at_v = ptx::smem_u32(keys) + ((lane & 7) + (lane >> 4) * 8) * kPitch + D * 2 + ((lane >> 3) & 1) * 16;
        const float top = fmaxf(m, warp_max(fmaxf(x0, x1)));
        if (top > m) {                                            // (the same in all lanes)
            if (m != -INFINITY) {
                const float fade = ptx::ex2(m - top);
                l *= fade;
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) acc[x][y] *= fade;
            }
            m = top;
        }
        const float ref = m == -INFINITY ? 0.0f : m, p0 = ptx::ex2(x0 - ref), p1 = ptx::ex2(x1 - ref);
        l += p0 + p1;
        const int from = (lane & 3) * 8;
        float w[4] = {__shfl_sync(0xffffffffu, p0, from), __shfl_sync(0xffffffffu, p0, from + 4), __shfl_sync(0xffffffffu, p1, from), __shfl_sync(0xffffffffu, p1, from + 4)};
        uint32_t b0 = ptx::pack_bf16(w[0], w[1]), b1 = ptx::pack_bf16(w[2], w[3]);
        if (lane >= 4) {
            b0 = ptx::pack_bf16(w[0] - __uint_as_float(b0 << 16), w[1] - __uint_as_float(b0 & 0xffff0000u));
            b1 = ptx::pack_bf16(w[2] - __uint_as_float(b1 << 16), w[3] - __uint_as_float(b1 & 0xffff0000u));
        }
        if (lane >= 8) b0 = b1 = 0u;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            uint32_t a[4];
            ldmatrix<true>(a, at_v + x * 32);
            mma_16816(acc[x], a, b0, b1);
        }
    }
    __device__ __forceinline__ void end(float* o, int lane) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        l = __shfl_sync(0xffffffffu, l, 0);
        m = m == -INFINITY ? m : m * 0.6931471805599453f;
        if ((lane & 3) == 0)
#pragma unroll
            for (int x = 0; x < D / 16; ++x)                      // (an infinite value's second part is not a number)
#pragma unroll
                for (int y = 0; y < 4; y += 2) o[x * 16 + y * 4 + (lane >> 2)] = isfinite(acc[x][y]) ? acc[x][y] + acc[x][y + 1] : acc[x][y];
    }
};

// All of a group's heads, up to eight, over the same keys (bf16): S = Q K^T and O = P V with the heads as the rows 0-7, and in the rows 8-15 what p leaves when it is rounded.
template <int D>
struct AttendAll {
    static constexpr int kStage = 16, kPitch = 2 * D * 2 + 16;
    uint32_t q[D / 16][2];
    float acc[D / 8][4], m = -INFINITY, l = 0.0f, c1;              // of row lane / 4; m in log2 units
    __device__ __forceinline__ void start(const __nv_bfloat16* row, bool real, float scale, int lane) {
        c1 = scale * 1.4426950408889634f;
#pragma unroll
        for (int x = 0; x < D / 8; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = 0.0f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) q[x][y] = real ? *reinterpret_cast<const uint32_t*>(row + x * 16 + y * 8 + (lane & 3) * 2) : 0u;
    }
    float x[4];                                                   // scores of the keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9 with c = lane % 4; bias: of the same
    __device__ __forceinline__ void scores(const uint8_t* keys, const float (&bias)[4], int count, int lane) {
        const uint32_t at_k = ptx::smem_u32(keys) + ((lane & 7) + (lane >> 4) * 8) * kPitch + ((lane >> 3) & 1) * 16;
        float s[2][4] = {};
#pragma unroll
        for (int y = 0; y < D / 16; ++y) {
            uint32_t b[4];
            ldmatrix<false>(b, at_k + y * 32);
            const uint32_t a[4] = {q[y][0], 0u, q[y][1], 0u};
            mma_16816(s[0], a, b[0], b[1]);
            mma_16816(s[1], a, b[2], b[3]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = (lane & 3) * 2 + (i >> 1) * 8 + (i & 1);
            x[i] = e < count ? fmaf(s[i >> 1][i & 1], c1, bias[i] * 1.4426950408889634f) : -INFINITY;
        }
    }
    __device__ __forceinline__ void values(uint8_t* keys, int count, int lane) {
        if (count < kStage) {                                     // (0 times what lies there must be 0)
            for (int i = count * (D / 8) + lane; i < kStage * (D / 8); i += 32) *reinterpret_cast<uint4*>(keys + i / (D / 8) * kPitch + D * 2 + i % (D / 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
        }
        const uint32_t at_v = ptx::smem_u32(keys) + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + D * 2 + (lane >> 4) * 16;
        float top = fmaxf(fmaxf(m, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        if (__any_sync(0xffffffffu, top > m)) {
            const float fade = m == -INFINITY ? 1.0f : ptx::ex2(m - top);
            l *= fade;
#pragma unroll
            for (int y = 0; y < D / 8; ++y)
#pragma unroll
                for (int z = 0; z < 4; ++z) acc[y][z] *= fade;
            m = top;
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = ptx::ex2(x[i] - ref);
            l += p[i];
        }
        const uint32_t h0 = ptx::pack_bf16(p[0], p[1]), h1 = ptx::pack_bf16(p[2], p[3]);
        const uint32_t a[4] = {h0, ptx::pack_bf16(p[0] - __uint_as_float(h0 << 16), p[1] - __uint_as_float(h0 & 0xffff0000u)),
                               h1, ptx::pack_bf16(p[2] - __uint_as_float(h1 << 16), p[3] - __uint_as_float(h1 & 0xffff0000u))};
#pragma unroll
        for (int y = 0; y < D / 16; ++y) {
            uint32_t b[4];
            ldmatrix<true>(b, at_v + y * 32);
            mma_16816(acc[2 * y], a, b[0], b[1]);
            mma_16816(acc[2 * y + 1], a, b[2], b[3]);
        }
    }
    // o [8][D] to shared memory; (m, l) of the lane's head, natural units
    __device__ __forceinline__ void end(float* o, int lane) {
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        m = m == -INFINITY ? m : m * 0.6931471805599453f;
#pragma unroll
        for (int y = 0; y < D / 8; ++y)
#pragma unroll
            for (int z = 0; z < 2; ++z)                           // (an infinite value's second part is not a number)
                o[(lane >> 2) * D + y * 8 + (lane & 3) * 2 + z] = isfinite(acc[y][z]) ? acc[y][z] + acc[y][z + 2] : acc[y][z];
    }
};

// The sums of a row's own keys, D / 32 channels per lane: its piece, or its result where there is no prefix.
template <typename T, int D>
__device__ __forceinline__ void write_own(const DecodeArgs& A, int t, int h, bool behind, float top, float sum, const float (&o)[D / 32], int lane) {
    if (behind) {
        float* out = A.piece_of(t, h, 0, D);
#pragma unroll
        for (int x = 0; x < D / 32; ++x) out[2 + lane + 32 * x] = o[x];
        if (lane == 0) {
            out[0] = top;
            out[1] = sum;
        }
    } else {
        T* out = (T*)A.o + t * A.os_row + h * A.os_head;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) store_as(out + lane + 32 * x, sum == 0.0f ? 0.0f : o[x] / sum);
        if (lane == 0) A.lse[t * A.Hq + h] = sum == 0.0f ? -INFINITY : top + logf(sum);
    }
}

// A CTA per (row, KV head) or part of its heads.
template <typename T, int D, bool kTeams>
__global__ void __launch_bounds__(kThreads, 2) own_kernel(DecodeArgs A, int warps_per_head, int heads) {
    using At = Attend<T, D>;
    constexpr int kStageBytes = At::kStage * At::kPitch;
    extern __shared__ __align__(16) uint8_t dynamic[];            // of each warp [At::kStage][At::kPitch] keys, [kRoom]: (pattern of delta, slot) of kept keys
    __shared__ OwnShared S;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32, team = kTeams ? warps_per_head : 1;
    pdl_enter();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // (the prefixes' attention needs nothing of this kernel before its last step)
    OwnRow R;
    if (!R.find(A, blockIdx.x, heads)) return;
    const int t = R.t, hk = R.hk, n = R.n, listed = R.listed, mask = (1 << A.page_log) - 1;
    const T* kv = (const T*)A.kv;
    uint8_t* keys_at = dynamic + warp * kStageBytes;
    const bool behind = listed > 0;
    constexpr int kRow = D * (int)sizeof(T);                      // bytes of K's row, and of V's

    if constexpr (sizeof(T) == 2) {
        if (R.keeps_all(A)) {
            for (int g0 = R.head0; g0 < R.head1; g0 += 8) {
                const int mine = g0 + (lane >> 2), h = hk * A.G + mine;
                const bool real = mine < R.head1;
                AttendAll<D> at;
                at.start((const T*)A.q + t * A.qs_row + h * A.qs_head, real, A.scale, lane);
                // 16 keys at a time, side by side in one page, turn by turn of the warps
                int next = warp * 16 < n ? R.pages[warp * 16 >> A.page_log] : -1;
#pragma unroll 1
                for (int j = warp * 16; j < n; j += warps * 16) {
                    const int page = next, count = min(n - j, 16);
                    next = j + warps * 16 < n ? R.pages[(j + warps * 16) >> A.page_log] : -1;
                    if ((unsigned)page >= (unsigned)A.num_pages) continue;
                    const uint8_t* from = (const uint8_t*)(kv + key_row(page, hk, j & mask, A.Hkv, A.page_log) * (2 * D));
                    auto copy = [&](int which) {
#pragma unroll
                        for (int i = lane; i < kRow; i += 32) {   // 16 rows of kRow / 16 parts
                            const int e = i / (kRow / 16), x = which * kRow + i % (kRow / 16) * 16;
                            if (e < count) ptx::cp_async16_at(ptx::smem_u32(keys_at) + e * At::kPitch + x, from + e * 2 * kRow + x);
                        }
                        cp_async_commit();
                    };
                    copy(0);
                    copy(1);
                    float bias[4] = {};
                    const float* delta = A.delta + (((size_t)page * A.Hq + h) << A.page_log) + (j & mask) + (lane & 3) * 2;
                    if (real) {
                        const float2 u = *reinterpret_cast<const float2*>(delta), v = *reinterpret_cast<const float2*>(delta + 8);
                        bias[0] = u.x; bias[1] = u.y; bias[2] = v.x; bias[3] = v.y;
                    }
                    cp_async_wait<1>();
                    __syncwarp();
                    at.scores(keys_at, bias, count, lane);
                    cp_async_wait<0>();
                    __syncwarp();
                    at.values(keys_at, count, lane);
                    __syncwarp();
                }
                float* o = reinterpret_cast<float*>(keys_at);     // [8][D]
                at.end(o, lane);
                if ((lane & 3) == 0) {
                    S.all_m[warp][lane >> 2] = at.m;
                    S.all_l[warp][lane >> 2] = at.l;
                }
                __syncthreads();
                for (int y = warp; y < min(8, R.head1 - g0); y += warps) {
                    const int head = hk * A.G + g0 + y;
                    float top = -INFINITY, sum = 0.0f, out[D / 32] = {};
                    for (int w = 0; w < warps; ++w) top = fmaxf(top, S.all_m[w][y]);
                    for (int w = 0; w < warps; ++w) {
                        const float wm = S.all_m[w][y], wl = S.all_l[w][y], f = wm == -INFINITY ? (wl == 0.0f ? 0.0f : 1.0f) : expf(wm - top);
                        if (f == 0.0f) continue;
                        sum += wl * f;
#pragma unroll
                        for (int x = 0; x < D / 32; ++x) out[x] += reinterpret_cast<const float*>(dynamic + w * kStageBytes)[y * D + lane + 32 * x] * f;
                    }
                    write_own<T, D>(A, t, head, behind, top, sum, out, lane);
                }
                __syncthreads();
            }
            return;
        }
    }
    const int in_team = kTeams ? warp % team : 0, bar = 1 + warp / team;
    uint2* mine = reinterpret_cast<uint2*>(dynamic + warps * kStageBytes) + warp * kRoom;
    const int seg = (n + team * 64 - 1) / (team * 64) * 64, j0 = min(n, in_team * seg), j1 = min(n, j0 + seg);
#pragma unroll 1
    for (int head = R.head0 + warp / team; head < R.head1; head += warps / team) {
    const int h = hk * A.G + head;
    const unsigned long long least = A.least[t * A.Hq + h];
    At at;
    at.start((const T*)A.q + t * A.qs_row + h * A.qs_head, A.scale, lane);
    int kept = 0;
    auto attend = [&]() {
        // eight lanes take 128 bytes of a key at a time; K's rows and V's are groups of their own, the next stage's K on its way while this one's V is used
        auto copy = [&](int i, int which) {
            const uint32_t to = ptx::smem_u32(keys_at) + which * kRow + (lane & 7) * 16;
#pragma unroll
            for (int e0 = 0; e0 < At::kStage; e0 += 4) {
                const int e = i + e0 + (lane >> 3);
                if (e < kept) {
                    const int slot = (int)mine[e].y;
                    const uint8_t* from = (const uint8_t*)(kv + key_row(slot >> A.page_log, hk, slot & mask, A.Hkv, A.page_log) * (2 * D)) + which * kRow + (lane & 7) * 16;
#pragma unroll
                    for (int x = 0; x < kRow; x += 128) ptx::cp_async16_at(to + (e0 + (lane >> 3)) * At::kPitch + x, from + x);
                }
            }
            cp_async_commit();
        };
        if (kept) {
            copy(0, 0);
            copy(0, 1);
        }
#pragma unroll 1
        for (int i = 0; i < kept; i += At::kStage) {
            const int count = min(kept - i, At::kStage);
            cp_async_wait<1>();
            __syncwarp();
            at.scores(keys_at, mine + i, count, lane);
            __syncwarp();
            copy(i + At::kStage, 0);
            cp_async_wait<1>();
            __syncwarp();
            at.values(keys_at, count, lane);
            __syncwarp();
            copy(i + At::kStage, 1);
        }
        kept = 0;
    };
    sweep_own(A, R, h, j0, j1, [&](int j, int slot, const int (&u)[16]) {
        if (kept > kRoom - 512) attend();
        uint32_t flags = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) flags |= (uint32_t)(u[i] >= 0 && order_key((uint32_t)u[i], j + i) >= least) << i;
        const int count = __popc(flags);
        int to = count;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, to, o);
            if (lane >= o) to += y;
        }
        const int total = __shfl_sync(0xffffffffu, to, 31);
        to += kept - count;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (flags >> i & 1u) mine[to++] = make_uint2((uint32_t)u[i], (uint32_t)(slot + i));
        kept += total;
        __syncwarp();
    });
    attend();
    at.end(reinterpret_cast<float*>(keys_at), lane);
    if (lane == 0) { S.m[warp] = at.m; S.l[warp] = at.l; }
    team_sync(bar, team * 32);
    if (in_team == 0) {
        float top = -INFINITY, sum = 0.0f, out[D / 32] = {};
        for (int w = warp; w < warp + team; ++w) top = fmaxf(top, S.m[w]);
        for (int w = warp; w < warp + team; ++w) {
            const float f = S.m[w] == -INFINITY ? (S.l[w] == 0.0f ? 0.0f : 1.0f) : expf(S.m[w] - top);
            if (f == 0.0f) continue;
            sum += S.l[w] * f;
#pragma unroll
            for (int x = 0; x < D / 32; ++x) out[x] += reinterpret_cast<const float*>(dynamic + w * kStageBytes)[lane + 32 * x] * f;
        }
        write_own<T, D>(A, t, h, behind, top, sum, out, lane);
    }
    team_sync(bar, team * 32);
    }
}

template <typename T, int D>
int own(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    const Teams W(C, 16, 1024);
    const size_t smem = (size_t)W.warps * (kRoom * sizeof(uint2) + Attend<T, D>::kStage * Attend<T, D>::kPitch);
    auto kernel = W.team > 1 ? own_kernel<T, D, true> : own_kernel<T, D, false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(kernel, dim3((unsigned)W.ctas), dim3(32 * W.warps), smem, st, 1, A, W.team, W.heads);
}

}  // namespace

int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? own<__nv_bfloat16, 128> : own<__nv_bfloat16, 64>) : (C.d == 128 ? own<float, 128> : own<float, 64>);
    return f(C, A, st);
}

}  // namespace dma
