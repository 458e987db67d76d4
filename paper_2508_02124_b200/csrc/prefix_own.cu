// dma_cache_decode (include/dma.h), first kernel: what every row keeps of its prefix' order and of its own keys, and the attention over the latter.
//
// The cut. A row's head keeps k = min(w, listed + own) keys of the merged order. Entry m of the prefix' order has m entries before it and every own key that is greater; so the
// prefix' part ends with the first m for which m + #{own > weight_m} >= k (ties: the prefix' keys come first), and the own part is the k - m best of the row's own keys. Where the list
// has w entries, own keys that do not exceed its last cannot be kept and are left out at once: of n own keys behind a prefix of N about n w / N remain, the candidates. Each of them takes
// at most one entry's place: the i-th best is kept if it is above the i-th entry from the list's end. So
//   - up to 64 candidates, a full list: the first stage's K and V are requested, the lowest candidate is dropped as long as it fails, a minimum of the warp each time, 25 times at most (without both: 16 rows of
//     64 own keys 10.3 us instead of 8.2, 256 of 512 55 instead of 53.5);
//   - else: how many are kept by bisection, #{own keys that are not below entry i from the end} > i, the entries in shared memory; then the weakest between the two entries around it (256 rows
//     of 512 own keys behind 2048, w = 1024: 140 us; by sorting up to 256 of them, and bisecting over the list where it lies beyond, 173);
//   - without room in shared memory for all of them (512 a warp): bisection of the cut over the list where it lies, then of the weakest own key, each count a sweep of the cache by the team. That is
//     slow, and only rows without a full list come to it: 2048 of 16K own keys and no prefix 115 us, of 64K 312 (615 with ten weights only), of 256K 1214; 32 such rows of 64K 1815.
// A row that keeps everything whatever its weights needs no cut: its warps take parts of the keys with all heads together (40 rows of up to 300 own keys: 25 -> 6.5 us).
//
// A CTA takes a (row, KV head), so that K and V of a key that several heads keep come from the L1 or L2. A head has a warp or a team of them: teams where few rows would leave the SMs with
// few warps (8 rows of 4096 own keys: 36 us without them, 19 with), up to 16 warps per SM (asked to make 32 with 64 rows of 1024 own keys: 57 us instead of 33, since every team pays for
// its barriers).
//
// Times (own keys ragged, 32 and 8 heads, d = 128): 64 rows of up to 1024 own keys behind 16K keys, w = 2048: 23 us; 256 rows of up to 512 behind 8K, w = 1024: 54; 8 rows of up to 4096 behind 64K,
// w = 4096: 16. Bound by round trips that few warps hide: pages, weights, the cut, then rows of K and V a stage ahead (64 rows: 10 warps per SM, issue slots 34 % busy; 256 rows: 14 warps, 43 %,
// 186 MB from memory at half the copy's rate). 128 registers (bf16, d = 128: 56 bytes of them spilled, 80 with teams) and 13 KB of shared memory per warp allow no more of them.
#include <algorithm>

#include "cache4_decode.cuh"
#include "delta_fixed.cuh"
#include "prefix_decode.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kRoom = 512;      // kRoom: candidates of a warp at most
constexpr float kLog2e = 1.4426950408889634f;     // of differences of scores: a weight as large as fp32 holds has no value in units of log 2

// A team of 1, 2, 4 or 8 warps has a (row, head), each warp a part of the own keys.
struct OwnShared {
    unsigned long long least[kWarps];
    int part[2][kWarps], cands[kWarps], cut[kWarps];
    float m[kWarps], l[kWarps], all_m[kWarps][8], all_l[kWarps][8];
};

__device__ __forceinline__ void team_sync(int id, int threads) {
    if (threads > 32) asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
    else __syncwarp();
}
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

// Attention of a warp over keys that lie in shared memory (K's row, V's, kPitch bytes apart), a stage of them at a time; use: a bit for each that counts; list: their biases.
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
    __device__ __forceinline__ void scores(const uint8_t* keys, const uint2* list, uint32_t use, int lane) {
#pragma unroll
        for (int i = 0; i < kStage; i += 4) {
            const int e = i + (lane >> 3);
            const float* row = reinterpret_cast<const float*>(keys + e * kPitch) + (lane & 7) * 4;
            float s = 0.0f;
            if (use >> e & 1u) {
#pragma unroll
                for (int x = 0; x < C; x += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(row + x * 8);
                    s = fmaf(q[x], k.x, s); s = fmaf(q[x + 1], k.y, s); s = fmaf(q[x + 2], k.z, s); s = fmaf(q[x + 3], k.w, s);
                }
            }
#pragma unroll
            for (int x = 1; x < 8; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            this->s[i / 4] = use >> e & 1u ? s + __uint_as_float(list[e].x) : -INFINITY;
        }
    }
    __device__ __forceinline__ void values(uint8_t* keys, uint32_t use, int lane) {
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
            if (use >> e & 1u) {
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
    float acc[D / 16][4], m = -INFINITY, l = 0.0f, scale;
    __device__ __forceinline__ void start(const __nv_bfloat16* row, float by, int lane) {
        scale = by;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = 0.0f;
#pragma unroll
            for (int y = 0; y < 2; ++y) q[x][y] = lane < 4 ? *reinterpret_cast<const uint32_t*>(row + x * 16 + y * 8 + lane * 2) : 0u;
        }
    }
    float x0, x1;                                                 // of lane 4 i: the scores of keys i and i + 8
    __device__ __forceinline__ void scores(const uint8_t* keys, const uint2* list, uint32_t use, int lane) {
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
        x0 = (lane & 3) == 0 && (use >> e & 1u) ? fmaf(s[0] + s1[0], scale, __uint_as_float(list[e].x)) : -INFINITY;
        x1 = (lane & 3) == 0 && (use >> (e + 8) & 1u) ? fmaf(s[2] + s1[2], scale, __uint_as_float(list[e + 8].x)) : -INFINITY;
    }
    __device__ __forceinline__ void values(uint8_t* keys, uint32_t use, int lane) {
        if (use != 0xFFFFu) {                                     // (0 times what lies there must be 0)
            for (int i = lane; i < kStage * (D / 8); i += 32)
                if (!(use >> i / (D / 8) & 1u)) *reinterpret_cast<uint4*>(keys + i / (D / 8) * kPitch + D * 2 + i % (D / 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
        }
        const uint32_t at_v = ptx::smem_u32(keys) + ((lane & 7) + (lane >> 4) * 8) * kPitch + D * 2 + ((lane >> 3) & 1) * 16;
        const float top = fmaxf(m, warp_max(fmaxf(x0, x1)));
        if (top > m) {                                            // (the same in all lanes)
            if (m != -INFINITY) {
                const float fade = ptx::ex2((m - top) * kLog2e);
                l *= fade;
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) acc[x][y] *= fade;
            }
            m = top;
        }
        const float ref = m == -INFINITY ? 0.0f : m, p0 = ptx::ex2((x0 - ref) * kLog2e), p1 = ptx::ex2((x1 - ref) * kLog2e);
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
    float acc[D / 8][4], m = -INFINITY, l = 0.0f, scale;           // of row lane / 4
    __device__ __forceinline__ void start(const __nv_bfloat16* row, bool real, float by, int lane) {
        scale = by;
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
            x[i] = e < count ? fmaf(s[i >> 1][i & 1], scale, bias[i]) : -INFINITY;
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
            const float fade = m == -INFINITY ? 1.0f : ptx::ex2((m - top) * kLog2e);
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
            p[i] = ptx::ex2((x[i] - ref) * kLog2e);
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
    // o [8][D] to shared memory; (m, l) of the lane's head
    __device__ __forceinline__ void end(float* o, int lane) {
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
        for (int y = 0; y < D / 8; ++y)
#pragma unroll
            for (int z = 0; z < 2; ++z)                           // (an infinite value's second part is not a number)
                o[(lane >> 2) * D + y * 8 + (lane & 3) * 2 + z] = isfinite(acc[y][z]) ? acc[y][z] + acc[y][z + 2] : acc[y][z];
    }
};

// The rows by prefix, in the order of rows, and tiles of them, by one CTA beside the others. It has the others' width: where thousands of rows have groups of one head, a single warp, whose grouping is
// what the call then waits for (this kernel, 16 own keys behind a prefix and without any: 4096 rows of one head 107 and 19 us, 16384 rows of one 453 and 64, of four 581 and 268).
__device__ void group_rows(const DecodeArgs& A, int* turn) {       // turn: kTogether per thread
    constexpr int kTogether = 4;                                  // rows of a thread requested together
    __shared__ int part[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    if (A.nprefix == 0) {
        if (tid == 0) *A.ntiles = 0;
        return;
    }
    // f(row, its prefix or -1) for kTogether rows at a time, thread by thread
    auto turns = [&](auto f) {
        for (int b = 0; b < A.rows; b += threads * kTogether) {
            int r[kTogether], g[kTogether], n[kTogether];
#pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                const int t = b + i * threads + tid;
                r[i] = g[i] = -1;
                if (t < A.rows) { r[i] = A.seq[t]; g[i] = A.prefix[t]; }
            }
#pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                if ((unsigned)r[i] >= (unsigned)A.nseq || (unsigned)g[i] >= (unsigned)A.nprefix) g[i] = -1;
                n[i] = g[i] >= 0 ? A.order_len[g[i]] : 0;
            }
#pragma unroll
            for (int i = 0; i < kTogether; ++i) g[i] = n[i] > 0 ? g[i] : -1;
            f(b, g);
        }
    };
    for (int i = tid; i <= A.nprefix; i += threads) A.first[i] = 0;
    __syncthreads();
    turns([&](int, const int (&g)[kTogether]) {
#pragma unroll
        for (int i = 0; i < kTogether; ++i)
            if (g[i] >= 0) atomicAdd(&A.first[g[i]], 1);
    });
    __syncthreads();
    int tile_carry = 0;
    for (int b = 0; b < A.nprefix; b += threads) {
        const int g = b + tid, n = g < A.nprefix ? __ldcg(&A.first[g]) : 0, nt = (n + A.tile_rows - 1) / A.tile_rows;
        int y = nt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) y += v;
        }
        if (lane == 31) part[warp] = y;
        __syncthreads();
        int tiles_before = 0, all_tiles = 0;
        for (int i = 0; i < threads / 32; ++i) {
            tiles_before += i < warp ? part[i] : 0;
            all_tiles += part[i];
        }
        if (g < A.nprefix) {
            const int tile = tile_carry + tiles_before + y - nt;
            __stcg(&A.first[g], tile * A.tile_rows);
            const int listed = nt ? (int)min((int64_t)min(A.order_len[g], A.w), A.order_ld) : 0;
            for (int i = 0; i < nt; ++i) A.tiles[tile + i] = make_int4(g, min(A.tile_rows, n - i * A.tile_rows), listed, 0);
        }
        tile_carry += all_tiles;
        __syncthreads();
    }
    if (tid == 0) *A.ntiles = tile_carry;
    // a turn's rows of the same prefix follow one another, the first of them moves the prefix' start on
    turns([&](int b, const int (&g)[kTogether]) {
        const int count = min(A.rows - b, threads * kTogether);
#pragma unroll
        for (int i = 0; i < kTogether; ++i) turn[i * threads + tid] = g[i];
        __syncthreads();
        int rank[kTogether] = {}, same[kTogether] = {}, start[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) start[i] = g[i] >= 0 ? __ldcg(&A.first[g[i]]) : 0;
        for (int e = 0; e < count; ++e) {
            const int x = turn[e];
#pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                same[i] += x == g[i];
                rank[i] += x == g[i] && e < i * threads + tid;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTogether; ++i)
            if (g[i] >= 0) {
                A.members[start[i] + rank[i]] = b + i * threads + tid;
                if (rank[i] == 0) __stcg(&A.first[g[i]], start[i] + same[i]);
            }
        __syncthreads();
    });
}

// The sums of a row's own keys, D / 32 channels per lane: its piece, or its result where there is no prefix.
template <typename T, int D>
__device__ __forceinline__ void write_own(const DecodeArgs& A, int t, int h, bool behind, int cut, float top, float sum, const float (&o)[D / 32], int lane) {
    if (behind) {
        float* out = A.piece_of(t, h, 0, D);
#pragma unroll
        for (int x = 0; x < D / 32; ++x) out[2 + lane + 32 * x] = o[x];
        if (lane == 0) {
            out[0] = top;
            out[1] = sum;
            A.cut[t * A.Hq + h] = cut;
        }
    } else {
        T* out = (T*)A.o + t * A.os_row + h * A.os_head;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) store_as(out + lane + 32 * x, sum == 0.0f ? 0.0f : o[x] / sum);
        if (lane == 0) A.lse[t * A.Hq + h] = sum == 0.0f ? -INFINITY : top + logf(sum);
    }
}

// A CTA per (row, KV head); the first one groups the rows by prefix. The group's heads each have a warp or a team of them (kTeams; else up to eight heads at a time, the others
// in turn). Where a row keeps all keys whatever their weights, the warps share its own keys, all heads together.
template <typename T, int D, bool kTeams>
__global__ void __launch_bounds__(kThreads, 2) own_kernel(DecodeArgs A, int warps_per_head, int room, int heads) {       // heads: of a CTA
    using At = Attend<T, D>;
    extern __shared__ __align__(16) uint8_t dynamic[];            // of each warp [At::kStage][At::kPitch] keys, [room]: (pattern of delta, slot) of candidates by position, then of the kept ones
    __shared__ OwnShared S;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x / 32, team = kTeams ? warps_per_head : 1;
    pdl_enter();
    if (blockIdx.x == 0) {                                        // (first: while the others are at work)
        for (int i = tid; i < kWsHeaderBytes / 4; i += blockDim.x) A.status[i] = 0;      // (a CTA may be one warp)
        group_rows(A, reinterpret_cast<int*>(dynamic));
        return;
    }
    const int parts = (A.G + heads - 1) / heads, item = blockIdx.x - 1, t = item / (A.Hkv * parts), hk = item / parts % A.Hkv, head0 = item % parts * heads, head1 = min(A.G, head0 + heads);
    const int r = A.seq[t], p = A.pos[t], g = A.nprefix ? A.prefix[t] : -1;
    if ((unsigned)r >= (unsigned)A.nseq) return;
    const int n = min(max(p, -1), (A.max_blocks << A.page_log) - 1) + 1;
    const int32_t* pages = A.table + r * A.ld;
    const int mask = (1 << A.page_log) - 1;
    const T* kv = (const T*)A.kv;
    constexpr int kStageBytes = At::kStage * At::kPitch;
    uint8_t* keys_at = dynamic + warp * kStageBytes;
    // what may be asked for at once: the list's length, the first pages
    const int in_team = kTeams ? warp % team : 0, leader = warp - in_team, bar = 1 + warp / team;
    const int seg = (n + team * 64 - 1) / (team * 64) * 64, j0 = min(n, in_team * seg), j1 = min(n, j0 + seg);
    auto page_of = [&](int j, int end) { return j < end ? pages[j >> A.page_log] : -1; };
    const int page_all = sizeof(T) == 2 ? page_of(warp * 16, n) : -1, page_mine = page_of(j0 + 16 * lane, j1);
    int listed = 0;
    if ((unsigned)g < (unsigned)A.nprefix) listed = (int)max((int64_t)0, min((int64_t)min(A.order_len[g], A.w), A.order_ld));
    const bool behind = listed > 0, floored = listed == A.w;      // (as DecodeArgs::listed)
    constexpr int kRow = D * (int)sizeof(T);                      // bytes of K's row, and of V's

    if constexpr (sizeof(T) == 2) {
        if ((int64_t)listed + n <= A.w) {
            for (int g0 = head0; g0 < head1; g0 += 8) {
                const int mine = g0 + (lane >> 2), h = hk * A.G + mine;
                const bool real = mine < head1;
                AttendAll<D> at;
                at.start((const T*)A.q + t * A.qs_row + h * A.qs_head, real, A.scale, lane);
                // 16 keys at a time, side by side in one page, turn by turn of the warps
                int next = page_all;
#pragma unroll 1
                for (int j = warp * 16; j < n; j += warps * 16) {
                    const int page = next, count = min(n - j, 16);
                    next = page_of(j + warps * 16, n);
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
                for (int y = warp; y < min(8, head1 - g0); y += warps) {
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
                    write_own<T, D>(A, t, head, behind, listed, top, sum, out, lane);
                }
                __syncthreads();
            }
            return;
        }
    }
    uint2* found = reinterpret_cast<uint2*>(dynamic + warps * kStageBytes);
    uint2* mine = found + warp * room;
#pragma unroll 1
    for (int head = head0 + warp / team; head < head1; head += warps / team) {
    const int h = hk * A.G + head;
    const float* weight = A.order_weight + ((int64_t)g * A.Hq + h) * A.order_ld;
    // f(position, slot, patterns) for the part's keys, 512 at a time: a lane has 16 of them, side by side in one page (pages have 16 keys and more). Patterns of places without a key: -2
    auto sweep = [&](auto f) {
        int next = page_mine;
#pragma unroll 1
        for (int b = j0; b < j1; b += 512) {
            const int j = b + 16 * lane, page = next, slot = (page << A.page_log) + (j & mask);
            const bool there = (unsigned)page < (unsigned)A.num_pages;
            int u[16];
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                int4 x = make_int4(-2, -2, -2, -2);
                if (there) x = *reinterpret_cast<const int4*>(A.delta + (((size_t)page * A.Hq + h) << A.page_log) + (j & mask) + i);
                u[i] = x.x; u[i + 1] = x.y; u[i + 2] = x.z; u[i + 3] = x.w;
            }
            next = page_of(j + 512, j1);
            if (b + 512 > j1)
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = j + i < j1 ? u[i] : -2;
            f(j, slot, u);
        }
    };
    // what a full list's end asks of the own keys: its entries' patterns plus one, from the last on
    uint32_t asked[2] = {0u, 0u};
    if (floored)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int back = i * 32 + lane;
            asked[i] = back < listed ? (__float_as_uint(weight[listed - 1 - back]) & 0x7FFFFFFFu) + 1u : ~0u;
        }
    At at;
    at.start((const T*)A.q + t * A.qs_row + h * A.qs_head, A.scale, lane);
    // what may be kept: every key that there is, or those above the list's last entry
    const int floor = (int)__shfl_sync(0xffffffffu, asked[0], 0) - 1;
    int c = 0;
    sweep([&](int, int slot, const int (&u)[16]) {
        int count = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) count += u[i] > floor;
        int to = count;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, to, o);
            if (lane >= o) to += y;
        }
        const int total = __shfl_sync(0xffffffffu, to, 31);
        to += c - count;
        if (to + count <= room) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (u[i] > floor) mine[to++] = make_uint2((uint32_t)u[i], (uint32_t)(slot + i));
        }
        c += total;
    });
    if (lane == 0) S.cands[warp] = c;
    __syncwarp();
    // eight lanes take 128 bytes of a key at a time; K's rows and V's are groups of their own
    auto copy = [&](int i, int which, int kept) {
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
    int cands = c, most = c, step = 0;
    if (team > 1) {
        team_sync(bar, team * 32);
        cands = most = 0;
        for (int i = 0; i < team; ++i) {
            cands += S.cands[leader + i];
            most = max(most, S.cands[leader + i]);
        }
    }
    const bool over = most > room;                                // (of the whole team: keys are then told apart by position, else by their place in the list)
    // Few candidates against a full list are kept as a rule: the first of them are on their way while the cut is found, and count or not.
    const bool few = floored && !over && cands <= 64;
    int ahead = few ? min(c, At::kStage) : 0;
    if (ahead) {
        copy(0, 0, ahead);
        copy(0, 1, ahead);
    }
    // keys that the row sees: all own ones are candidates where the list may not be full
    auto team_sum = [&](int x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (kTeams) {
            if (lane == 0) S.part[step & 1][warp] = x;
            team_sync(bar, team * 32);
            x = 0;
            for (int i = 0; i < team; ++i) x += S.part[step & 1][leader + i];
            ++step;
        }
        return x;
    };
    const int k = floored ? listed : (int)min((int64_t)A.w, (int64_t)listed + cands);
    int cut = listed;
    unsigned long long least = 0;                                 // kept: the order keys that are not below
    auto place = [&](int e) { return in_team * (1 << 20) + e; };
    if (k < listed + cands) {
        // the i-th best own key has to be above one of this many entries from the list's end on (the entry's pattern plus one)
        auto rival = [&](int i) {
            const int back = i - (k - listed);
            return back < 0 ? 0u : back < listed ? (__float_as_uint(weight[listed - 1 - back]) & 0x7FFFFFFFu) + 1u : ~0u;
        };
        // of candidates that are equal the first `need` are kept: the last of these
        auto among_equals = [&](uint32_t u, int need) {
            for (int x = 0; x < team; ++x)
                for (int e = 0; e < S.cands[leader + x]; e += 32) {
                    const uint32_t same = __ballot_sync(0xffffffffu, e + lane < S.cands[leader + x] && found[(leader + x) * room + e + lane].x == u);
                    if (__popc(same) >= need) return order_key(u, x * (1 << 20) + e + (int)__fns(same, 0, need));
                    need -= __popc(same);
                }
            return 0ull;
        };
        bool done = false;
        if (few) {
            // The lowest one is dropped as long as it fails. (By a team's first warp. 25 of them at most, else the bisection's twelve counts are fewer steps; 256 rows of 60 own keys behind 512,
            // w = 400: 37.4 us, 39.4 with 9 at most, 37.4 with 64; the same within 1 % where a tenth of the own keys are candidates.)
            if (in_team == 0) {
                unsigned long long keys[2];
                uint32_t last[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int e = 32 * i + lane;
                    last[i] = e < cands ? asked[i] : ~0u;
                    int x = 0, at = e;
                    if (kTeams)
                        while (x < team && at >= S.cands[leader + x]) at -= S.cands[leader + x++];
                    const uint2* of = found + (leader + x) * room;
                    keys[i] = e < cands ? order_key(of[at].x, x * (1 << 20) + at) : ~0ull;
                }
#pragma unroll 1
                for (int kept = cands; kept >= cands - 24 && !done; --kept) {
                    const unsigned long long low = keys[0] < keys[1] ? keys[0] : keys[1];
                    const uint32_t hi = __reduce_min_sync(0xffffffffu, (uint32_t)(low >> 32)), lo = __reduce_min_sync(0xffffffffu, (uint32_t)(low >> 32) == hi ? (uint32_t)low : ~0u);
                    const uint32_t pass = __shfl_sync(0xffffffffu, (kept - 1) >> 5 == 1 ? last[1] : last[0], (kept - 1) & 31);       // what the kept-th best has to be above
                    if (kept <= 0 || hi + 1u > pass) {
                        done = true;
                        least = kept <= 0 ? ~0ull : (unsigned long long)hi << 32 | lo;
                        cut = k - kept;
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) keys[i] = keys[i] == ((unsigned long long)hi << 32 | lo) ? ~0ull : keys[i];
                    }
                }
            }
            if (kTeams) {
                if (in_team == 0 && lane == 0) {
                    S.least[warp] = least;
                    S.cut[warp] = done ? cut : -1;
                }
                team_sync(bar, team * 32);
                least = S.least[leader];
                cut = S.cut[leader];
                done = cut >= 0;
            }
        }
        if (!done && !over) {
            // The best own key is kept if the list's last entry is below it, the second if the last but one is, and so on: how many are, by bisection, i + 1 own keys or more being above
            // the i-th entry from the end; then the weakest of them, between the entries on both sides.
            uint32_t* ask = reinterpret_cast<uint32_t*>(dynamic + leader * kStageBytes);
            if (ahead) cp_async_wait<0>();
            ahead = 0;
            team_sync(bar, team * 32);
            for (int e = in_team * 32 + lane; e < cands; e += team * 32) ask[e] = rival(e);
            team_sync(bar, team * 32);
            auto not_below = [&](uint32_t u) {
                int sum = 0;
#pragma unroll 4
                for (int e = lane; e < c; e += 32) sum += mine[e].x >= u;
                return team_sum(sum);
            };
            int kept = 0, end = cands;
            while (kept < end) {
                const int i = (kept + end) >> 1;
                if (not_below(ask[i]) > i) kept = i + 1; else end = i;
            }
            cut = k - kept;
            least = ~0ull;
            if (kept) {
                uint32_t a = ask[kept - 1], b = kept < cands ? ask[kept] : 1u << 31;     // `kept` or more are not below a, at most so many not below b
                int at_a = not_below(a);
                while (at_a != kept && b - a > 1u) {
                    const uint32_t x = a + (b - a) / 2;
                    const int n_x = not_below(x);
                    if (n_x >= kept) { a = x; at_a = n_x; } else b = x;
                }
                const int need = at_a == kept ? kept : kept - not_below(b);
                if (at_a == kept || need == 0) least = (unsigned long long)(at_a == kept ? a : b) << 32;
                else least = among_equals(a, need);
            }
            team_sync(bar, team * 32);                            // (the entries have been read)
        } else if (!done) {
            // order keys greater than entry m's weight
            auto above = [&](int m) { return (unsigned long long)((__float_as_uint(weight[m]) & 0x7FFFFFFFu) + 1u) << 32; };
            // Entry m of the list has m entries before it and every own key that is greater: the first of which there are k or more is not kept. Each own key takes at most one entry's
            // place, so that it lies among the last `cands` (k >= listed). Bisection of the cut, then of the weakest kept own key between a, which `need` own keys or more are not below, and
            // b, which at most so many are not below.
            int lo = max(0, k - cands), hi = listed, need = 0, at_a = -1;
            unsigned long long a = 0, b = 0;
            bool cutting = true;
            while (true) {
                unsigned long long x;
                if (cutting && lo < hi) x = above((lo + hi) >> 1);
                else if (cutting) {
                    cutting = false;
                    cut = lo;
                    need = k - cut;
                    if (need == 0) { least = ~0ull; break; }
                    a = cut < listed ? above(cut) : 1;
                    b = cut > 0 ? above(cut - 1) : 1ull << 63;
                    x = a;
                } else {
                    if (at_a == need || b - a <= 1) { least = a; break; }
                    x = a + (b - a) / 2;
                }
                // own keys whose order key is not below x (> 0)
                int sum = 0;
                sweep([&](int j, int, const int (&u)[16]) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum += u[i] > floor && order_key((uint32_t)u[i], j + i) >= x;
                });
                sum = team_sum(sum);
                if (cutting) {
                    const int m = (lo + hi) >> 1;
                    if (m + sum >= k) hi = m; else lo = m + 1;
                } else if (sum >= need) {
                    a = x;
                    at_a = sum;
                } else {
                    b = x;
                }
            }
        }
    }
    // attention over the kept ones, a stage of keys at a time
    int b = over ? j0 : 0, front = ahead;
    uint32_t use = ~0u;                                           // of the first stage
    if (front) {
        use = __ballot_sync(0xffffffffu, lane < front && order_key(mine[lane].x, place(lane)) >= least);
        b = front;
    }
    const int end = over ? j1 : c;
    do {
        // as many kept ones as there is room for, at the front of the warp's part; where the candidates did not fit, from the cache again
        int kept = front;
        for (; b < end && (!over || kept + 32 <= room); b += 32) {
            uint2 o = make_uint2(0u, 0u);
            bool keep = false;
            if (over) {
                const int j = b + lane, page = j < j1 ? pages[j >> A.page_log] : -1;
                if ((unsigned)page < (unsigned)A.num_pages) {
                    const int u = __float_as_int(A.delta[(((size_t)page * A.Hq + h) << A.page_log) + (j & mask)]);
                    o = make_uint2((uint32_t)u, (uint32_t)((page << A.page_log) + (j & mask)));
                    keep = u > floor && order_key(o.x, j) >= least;
                }
            } else if (b + lane < c) {
                o = mine[b + lane];
                keep = order_key(o.x, place(b + lane)) >= least;
            }
            const uint32_t bits = __ballot_sync(0xffffffffu, keep);            // (behind every lane's read)
            if (keep) mine[kept + __popc(bits & ((1u << lane) - 1u))] = o;
            kept += __popc(bits);
            __syncwarp();
        }
        if (kept && !front) {
            copy(0, 0, kept);
            copy(0, 1, kept);
        }
        // the next stage's K is on its way while this one's V is used
#pragma unroll 1
        for (int i = 0; i < kept; i += At::kStage) {
            use &= (1u << min(kept - i, At::kStage)) - 1u;
            cp_async_wait<1>();
            __syncwarp();
            at.scores(keys_at, mine + i, use, lane);
            __syncwarp();
            copy(i + At::kStage, 0, kept);
            cp_async_wait<1>();
            __syncwarp();
            at.values(keys_at, use, lane);
            __syncwarp();
            copy(i + At::kStage, 1, kept);
            use = ~0u;
        }
        front = 0;
    } while (b < end);
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
        write_own<T, D>(A, t, h, behind, cut, top, sum, out, lane);
    }
    team_sync(bar, team * 32);
    }
}

// Warps: one per head of a group, eight at most; teams of them, and fewer heads per CTA, where all make fewer than 16 per SM (both sides at the file's head) or where a row's own keys would not
// find room as candidates (up to 1024 of a warp, of which half may be: beyond, every count reads the cache again).
template <typename T, int D>
int own(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    const int64_t capacity = (int64_t)C.max_blocks << C.page_log;
    int heads = 1, team = 1;
    while (heads < C.G && heads < kWarps) heads *= 2;
    const int most = heads;                                       // (more heads take turns)
    auto ctas = [&](int per) { return (int64_t)C.rows * C.Hkv * (per == most ? 1 : (C.G + per - 1) / per); };
    while (team < kWarps && (ctas(heads) * heads * team * 2 <= 16 * 148 || capacity > 1024 * team)) {
        team *= 2;
        if (heads * team > kWarps) heads /= 2;
    }
    const int room = (int)std::min<int64_t>((capacity + team * 64 - 1) / (team * 64) * 64, kRoom), warps = heads * team;
    auto bytes = [](int warps, int room) { return std::max<size_t>((size_t)warps * (room * sizeof(uint2) + Attend<T, D>::kStage * Attend<T, D>::kPitch), 32 * 1024 / kWarps * warps); };
    auto kernel = team > 1 ? own_kernel<T, D, true> : own_kernel<T, D, false>;
    // (state of the function, which other threads' calls share: always the limit)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes(kWarps, kRoom)) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(kernel, dim3((unsigned)(ctas(heads) + 1)), dim3(32 * warps), bytes(warps, room), st, 1, A, team, room, heads == most ? C.G : heads);
}

}  // namespace

int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? own<__nv_bfloat16, 128> : own<__nv_bfloat16, 64>) : (C.d == 128 ? own<float, 128> : own<float, 64>);
    return f(C, A, st);
}

}  // namespace dma
