// dma_cache_decode (include/dma.h), second kernel, on the tensor cores (bf16): up to 128 rows of a prefix together over a head's list, and the sum with the rows' own keys.
//
// The list is sorted, so that a row keeps its first `cut` entries: a dense product whose rows differ in length. A cluster takes a (tile of rows, head); its CTAs take parts of the
// list, 64 keys at a time: rows of K and V gathered by 16-byte asynchronous copies into the swizzled layout, S = Q K^T into tensor memory, softmax by a thread per row, P back over
// S as bf16, O += P V. Then the CTAs' sums meet in distributed shared memory, with each row's piece from its own keys, and o and lse are written.
// The products have 128 rows whatever the tile has. Where it has at most 64 (32), the other lanes take the same rows and other columns: lane group i of n the i-th part of every 64 keys,
// with zeros of P elsewhere, so that a thread walks 32 (16) columns instead of 64 (three tiles of 14 rows 21.4 us instead of 25.8, 16 rows 18.3 instead of 19.7, 64 rows the same).
// Rounding: scores, sums and O are fp32. P goes in as two bf16 numbers, the one next to it and what that leaves (2^-16 of a weight), over the same V: with one, o is a quarter further from
// 64 bits than its own rounding makes it (rms 2.1e-3 and 1.7e-3).
// A value that is not finite would reach rows that do not keep its key, as 0 times infinity. A row whose O is not finite is therefore formed again, by a warp, over the keys it keeps, and in
// natural units: so is one whose weights pass 2^128 / log2 e, which have no value in units of log 2.
//
// Warps: 0-3 softmax and the end, 4 issues the products, 5-8 gather (with two gathering 64 rows 26.7 us instead of 24.1, eight rows with long lists 34 instead of 29). Two CTAs per SM: 97 KB
// of stages, Q and O each. Nine warps twice leave a thread 96 registers, of which softmax and sum want more (132 bytes spilled for 128 channels, 184 for 64).
//
// Times (32 and 8 heads, d = 128): 64 rows behind 16K keys, w = 2048: 23 us; 256 rows in four prefixes of 8K, w = 1024: 32; 8 rows behind 64K, w = 4096: 26.5; 1024 rows behind 16K, w = 2048, 94. On the CUDA
// cores, whose tiles have eight rows (prefix_decode.cu): one row 28 us instead of 17, four 34 instead of 17, 64 rows of a prefix each 520 instead of 281; so bf16 comes here however few its rows are.
// With few rows it is the list's read, a gather of 512 bytes a key from places as the weights fall, that a CTA's tiles wait for (64 rows: four of them, 34 MB asked of the L2, 30 of them of memory; tensor
// pipe 14 % active), and start and end: rows, Q, the cluster's sum (eight rows of a list of 4096 have eight tiles per CTA, twice as many, and take 26.5 us). With many rows it is the softmax' threads (1024 rows: 0.55 PFLOP/s of products, both parts of P counted).
#include <algorithm>
#include <type_traits>

#include "prefix_decode.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

using namespace ptx;

constexpr int kKeys = 64, kGather = 4, kThreads = 32 * (5 + kGather), kIssuer = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRescale = 8.0f;              // log2 units: P stays below 2^8, O is rescaled on larger growth of the maximum only

template <int D>
struct Shared {
    static constexpr int kStages = D == 128 ? 2 : 4;
    static constexpr uint32_t kTile = kKeys * D * 2, kHalfQ = 128 * 128, kHalf = kKeys * 128;      // bytes; halves: 64 channels of all rows
    alignas(1024) uint8_t q[128 * D * 2];
    alignas(1024) uint8_t kv[kStages][2][kTile];              // in the end: O [128][D] fp32, 16-byte parts at (part ^ row)
    alignas(16) float bias[kStages][kKeys];                   // delta log2 e
    float m[128], l[128], joined_m[64], joined_l[64];
    float share[128], own_share[128], over_sum[128];          // of the sum: factors by (row of this CTA, rank), of the rows' own keys, one by the sum
    int row[128], cut[128];
    uint32_t bad[4];                                          // rows to form again, a bit each
    uint64_t q_full, full[kStages], bias_full[kStages], empty[kStages], s_full[2], p_full[2], o_done[2];
    uint32_t tmem;
    int abort_flag;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}

template <int D>
__device__ __forceinline__ uint32_t o_part(int row, int part) { return (uint32_t)(row * D * 4 + ((part ^ (row & (D / 4 - 1))) << 4)); }

// Tiles i0 .. i1 - 1 of 64 keys for a thread's row, W columns of each (part `copy`). Returns false where a wait gave up.
template <int D, int W>
__device__ __forceinline__ bool softmax(Shared<D>& S, int i0, int i1, int copy, int cut, float c1, uint32_t tmem, float& m, float& l) {
    constexpr int kStages = Shared<D>::kStages;
    volatile int* abort_flag = &S.abort_flag;
    for (int i = i0; i < i1; ++i) {
        const int n = i - i0, b = n & 1, st = n % kStages;
        if (!mbar_wait_warp(&S.bias_full[st], (n / kStages) & 1, abort_flag)) return false;
        if (!mbar_wait_warp(&S.s_full[b], (n >> 1) & 1, abort_flag)) return false;
        tc_fence_after();
        const int first = copy * W, keep = cut - i * kKeys - first;           // columns below `keep` are the row's
        float x[W];
#pragma unroll
        for (int c = 0; c < W; c += 16) {
            uint32_t s[16];
            tmem_ld16(tmem + b * kKeys + first + c, s);
            tc_wait_ld();
#pragma unroll
            for (int y = 0; y < 16; ++y) x[c + y] = __uint_as_float(s[y]);
        }
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < W; c += 4) {
            const float4 d = *reinterpret_cast<const float4*>(&S.bias[st][first + c]);
            x[c] = c < keep ? fmaf(x[c], c1, d.x) : -INFINITY;
            x[c + 1] = c + 1 < keep ? fmaf(x[c + 1], c1, d.y) : -INFINITY;
            x[c + 2] = c + 2 < keep ? fmaf(x[c + 2], c1, d.z) : -INFINITY;
            x[c + 3] = c + 3 < keep ? fmaf(x[c + 3], c1, d.w) : -INFINITY;
            top = max3(top, fmaxf(x[c], x[c + 1]), fmaxf(x[c + 2], x[c + 3]));
        }
        const bool grow = top > m + kRescale || (m == -INFINITY && top > m);
        if (__any_sync(0xffffffffu, grow)) {
            const float f = grow && m != -INFINITY ? ex2(m - top) : 1.0f;
            if (grow) m = top;
            l *= f;
            if (n > 0 && __any_sync(0xffffffffu, f != 1.0f)) {
                if (!mbar_wait_warp(&S.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, abort_flag)) return false;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(tmem + 2 * kKeys + c, o);
                    tc_wait_ld();
#pragma unroll
                    for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
                    tmem_st16(tmem + 2 * kKeys + c, o);
                }
            }
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        uint32_t p[W / 2], rest[W / 2];                           // rounded, and what that leaves, rounded
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < W; c += 2) {
            const float u = ex2(x[c] - ref), v = ex2(x[c + 1] - ref);
            sum += u + v;
            p[c / 2] = pack_bf16(u, v);
            rest[c / 2] = pack_bf16(u - __uint_as_float(p[c / 2] << 16), v - __uint_as_float(p[c / 2] & 0xffff0000u));
        }
        l += sum;
        uint32_t r[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) r[c] = W == 64 || c / (W / 2) == copy ? p[c % (W / 2)] : 0u;
        tmem_st32(tmem + b * kKeys, r);
#pragma unroll
        for (int c = 0; c < 32; ++c) r[c] = W == 64 || c / (W / 2) == copy ? rest[c % (W / 2)] : 0u;
        tmem_st32(tmem + b * kKeys + 32, r);
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(&S.p_full[b]);
    }
    return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) prefix_kernel(DecodeArgs A, int nrank) {
    using Sh = Shared<D>;
    constexpr int kStages = Sh::kStages;
    extern __shared__ uint8_t raw[];
    Sh& S = *reinterpret_cast<Sh*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % nrank, item = blockIdx.x / nrank, tile = item / A.Hq, h = item % A.Hq, hk = h / A.G;
    volatile int* abort_flag = &S.abort_flag;
    if (tid == 0) {
        mbar_init(&S.q_full, 128);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&S.full[i], 32 * kGather);
            mbar_init(&S.bias_full[i], kGather);
            mbar_init(&S.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&S.s_full[i], 1);
            mbar_init(&S.p_full[i], 128);
            mbar_init(&S.o_done[i], 1);
        }
        S.abort_flag = 0;
        fence_barrier_init();
    }
    if (tid < 4) S.bad[tid] = 0;
    pdl_enter();
    const int ntiles_all = *A.ntiles, member = tid < 128 ? A.members[tile * 128 + tid] : 0;
    const int4 rows = A.tiles[tile];
    if (warp == kIssuer) {                                        // (while these are on their way)
        tmem_alloc(&S.tmem, 256);
        tmem_relinquish();
    }
    if (tile >= ntiles_all) {                                     // (all CTAs of the cluster)
        __syncwarp();
        if (warp == kIssuer) tmem_dealloc(S.tmem, 256);
        return;
    }
    const int R = rows.y, listed = rows.z, copy_log = R <= 32 ? 2 : R <= 64 ? 1 : 0, copies = 1 << copy_log, lane_log = 7 - copy_log, lanes = 1 << lane_log;
    if (tid < R)
        for (int i = 0; i < copies; ++i) S.row[i * lanes + tid] = member;
    if (tid < lanes && tid >= R)
        for (int i = 0; i < copies; ++i) S.row[i * lanes + tid] = -1;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S.tmem;
    const int ntiles = (listed + kKeys - 1) / kKeys, i0 = (int)((int64_t)ntiles * rank / nrank), i1 = (int)((int64_t)ntiles * (rank + 1) / nrank);
    const __nv_bfloat16 *q = (const __nv_bfloat16*)A.q + h * A.qs_head, *kv = (const __nv_bfloat16*)A.kv;
    const int64_t list = ((int64_t)rows.x * A.Hq + h) * A.order_ld;
    const int32_t* slots = A.order_slot + list;
    const float* weights = A.order_weight + list;
    const int nslots = A.num_pages << A.page_log;
    float m = -INFINITY, l = 0.0f;
    if (warp < 4) {
        int cut = 0;
        if (i0 < i1) {
            // Q: lanes of D / 8 side by side take a row
            constexpr int LPR = D / 8;
            for (int i = lane / LPR; i < 32; i += 32 / LPR) {
                const int r = warp * 32 + i, part = lane % LPR, t = S.row[r];
                cp_async16(S.q + (part >> 3) * Sh::kHalfQ + r * 128 + (((part & 7) ^ (r & 7)) << 4), t >= 0 ? q + t * A.qs_row + part * 8 : q, t >= 0 ? 16 : 0);
            }
            cut = S.row[tid] >= 0 ? A.cut[S.row[tid] * A.Hq + h] : 0;
            cp_async_wait_all();
            fence_proxy_async();
            mbar_arrive(&S.q_full);
            S.cut[tid] = cut;
            const int copy = tid >> lane_log;
            const float c1 = A.scale * kLog2e;
            const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
            bool ok = copies == 4   ? softmax<D, 16>(S, i0, i1, copy, cut, c1, mine, m, l)
                      : copies == 2 ? softmax<D, 32>(S, i0, i1, copy, cut, c1, mine, m, l)
                                    : softmax<D, 64>(S, i0, i1, copy, cut, c1, mine, m, l);
            if (ok) ok = mbar_wait_warp(&S.o_done[(i1 - i0 - 1) & 1], ((i1 - i0 - 1) >> 1) & 1, abort_flag);
            if (ok) {
                tc_fence_after();
                uint8_t* to = &S.kv[0][0][0];
                bool odd = !isfinite(l);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(mine + 2 * kKeys + c, o);
                    tc_wait_ld_dep(o);
#pragma unroll
                    for (int y = 0; y < 32; ++y) odd |= (o[y] & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                    for (int y = 0; y < 32; y += 4) *reinterpret_cast<uint4*>(to + o_part<D>(tid, (c + y) / 4)) = make_uint4(o[y], o[y + 1], o[y + 2], o[y + 3]);
                }
                if (odd && S.row[tid] >= 0) atomicOr(&S.bad[(tid & (lanes - 1)) >> 5], 1u << (tid & (lanes - 1) & 31));
            }
        }
        S.m[tid] = m == -INFINITY ? m : m * kLn2;
        S.l[tid] = l;
    } else if (warp == kIssuer) {
        constexpr uint32_t idesc_s = idesc_bf16(128, kKeys, 0, 0), idesc_pv = idesc_bf16(128, D, 0, 1);
        const uint64_t dq = smem_desc_sw128(smem_u32(S.q), 16, 1024), dk = smem_desc_sw128(smem_u32(S.kv[0][0]), 16, 1024),
                       dv = smem_desc_sw128(smem_u32(S.kv[0][1]), Sh::kHalf, 1024);
        const int n = i1 - i0;
        bool ok = n > 0 && mbar_wait_warp(&S.q_full, 0, abort_flag);
        auto scores = [&](int i) {
            const int st = i % kStages;
            ok = mbar_wait_warp(&S.full[st], (i / kStages) & 1, abort_flag);
            fence_proxy_async();                                  // (the gathered rows were written through the generic proxy)
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(tmem + (i & 1) * kKeys, dq + (uint64_t)(((kk >> 2) * Sh::kHalfQ + (kk & 3) * 32) >> 4),
                           dk + (uint64_t)((st * 2 * Sh::kTile + (kk >> 2) * Sh::kHalf + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
                tc_commit(&S.s_full[i & 1]);
            }
            __syncwarp();
        };
        if (ok) scores(0);
        for (int i = 0; i < n && ok; ++i) {
            const int st = i % kStages;
            if (i + 1 < n) scores(i + 1);
            if (ok) ok = mbar_wait_warp(&S.p_full[i & 1], (i >> 1) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 2 * kKeys / 16; ++kk)
                    mma_ts(tmem + 2 * kKeys, tmem + (i & 1) * kKeys + kk * 8, dv + (uint64_t)((st * 2 * Sh::kTile + kk % (kKeys / 16) * 2048) >> 4), idesc_pv, kk > 0 || i > 0 ? 1u : 0u);
                tc_commit(&S.o_done[i & 1]);      // (the product before the last is done once the last scores are: a wait is never two phases early)
                tc_commit(&S.empty[st]);
            }
            __syncwarp();
        }
    } else {
        // a warp has 16 keys of each tile; eight lanes take 128 bytes of a key at a time
        constexpr int kMine = kKeys / kGather;
        const int w = warp - kIssuer - 1;
        int slot = -1;
        float bias = -INFINITY;
        auto fetch = [&](int i) {
            const int e = i * kKeys + w * kMine + lane;
            slot = -1;
            bias = -INFINITY;
            if (lane < kMine && i < i1 && e < listed) {
                slot = slots[e];
                bias = weights[e] * kLog2e;
                if ((unsigned)slot >= (unsigned)nslots) { slot = -1; bias = -INFINITY; }
            }
        };
        fetch(i0);
        bool ok = true;
        for (int i = i0; i < i1; ++i) {
            const int n = i - i0, st = n % kStages;
            if (n >= kStages) ok = mbar_wait_warp(&S.empty[st], ((n / kStages) - 1) & 1, abort_flag);
            if (!ok) break;
            if (lane < kMine) S.bias[st][w * kMine + lane] = bias;
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.bias_full[st]);
#pragma unroll
            for (int k = 0; k < kMine; k += 4) {
                const int at = __shfl_sync(0xffffffffu, slot, k + (lane >> 3)), r = w * kMine + k + (lane >> 3);
                const __nv_bfloat16* from = kv + (at >= 0 ? key_row(at >> A.page_log, hk, at & ((1 << A.page_log) - 1), A.Hkv, A.page_log) * (2 * D) : 0) + (lane & 7) * 8;
                uint8_t* to = S.kv[st][0] + r * 128 + (((lane & 7) ^ (r & 7)) << 4);
#pragma unroll
                for (int x = 0; x < 2 * D / 64; ++x) cp_async16(to + x / (D / 64) * Sh::kTile + x % (D / 64) * Sh::kHalf, from + x * 64, at >= 0 ? 16 : 0);
            }
            cp_async_arrive(&S.full[st]);
            fetch(i + 1);
        }
        cp_async_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after();
        tmem_dealloc(tmem, 256);
    }
    const uint32_t sO = smem_u32(&S.kv[0][0][0]);
    // rows that are not finite, key by key
    for (int r = (S.bad[0] | S.bad[1] | S.bad[2] | S.bad[3]) ? warp : R; r < R; r += kThreads / 32) {
        if (!(S.bad[r >> 5] >> (r & 31) & 1u)) continue;
        constexpr int C = D / 32;
        const int t = S.row[r], end = min(S.cut[r], i1 * kKeys);
        float qv[C], acc[C] = {}, mm = -INFINITY, ll = 0.0f;
#pragma unroll
        for (int x = 0; x < C; ++x) qv[x] = to_f32(q[t * A.qs_row + lane * C + x]);
        for (int e = i0 * kKeys; e < end; ++e) {
            const int at = slots[e];
            if ((unsigned)at >= (unsigned)nslots) continue;
            const __nv_bfloat16* row = kv + key_row(at >> A.page_log, hk, at & ((1 << A.page_log) - 1), A.Hkv, A.page_log) * (2 * D) + lane * C;
            float s = 0.0f;
#pragma unroll
            for (int x = 0; x < C; ++x) s = fmaf(qv[x], to_f32(row[x]), s);
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            s = fmaf(s, A.scale, weights[e]);
            const float top = fmaxf(mm, s), ref = top == -INFINITY ? 0.0f : top, fade = mm == -INFINITY ? 0.0f : expf(mm - ref), p = expf(s - ref);
            mm = top;
            ll = ll * fade + p;
#pragma unroll
            for (int x = 0; x < C; ++x) acc[x] = (fade == 0.0f ? 0.0f : acc[x] * fade) + p * to_f32(row[D + x]);
        }
#pragma unroll
        for (int x = 0; x < C; ++x) {
            const int c = lane * C + x;
            *reinterpret_cast<float*>(&S.kv[0][0][0] + o_part<D>(r, c / 4) + (c & 3) * 4) = acc[x];
        }
        if (lane < copies) {
            S.m[lane * lanes + r] = lane == 0 ? mm : -INFINITY;
            S.l[lane * lanes + r] = lane == 0 ? ll : 0.0f;
        }
    }
    auto factor = [](float m1, float l1, float top) { return m1 == -INFINITY ? (l1 == 0.0f ? 0.0f : 1.0f) : ex2((m1 - top) * kLog2e); };
    auto add = [](float4& a, const float4& v, float g) { a.x += v.x * g; a.y += v.y * g; a.z += v.z * g; a.w += v.w * g; };
    // a row's lane groups to the first of them: a thread per 16 bytes of O
    if (copies > 1) {
        __syncthreads();
        auto join = [&](auto n_tag) {
            constexpr int N = decltype(n_tag)::value;
#pragma unroll 1
            for (int i = tid; i < R * (D / 4); i += kThreads) {
                const int r = i / (D / 4), part = i % (D / 4);
                float cm[N], top = -INFINITY, sum = 0.0f;
                float4 v[N], acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    cm[c] = S.m[c * (128 / N) + r];
                    v[c] = *reinterpret_cast<const float4*>(&S.kv[0][0][0] + o_part<D>(c * (128 / N) + r, part));
                    top = fmaxf(top, cm[c]);
                }
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const float cl = S.l[c * (128 / N) + r], f = factor(cm[c], cl, top);
                    if (f == 0.0f) continue;                      // (what a part without keys left may be anything)
                    sum += cl * f;
                    add(acc, v[c], f);
                }
                *reinterpret_cast<float4*>(&S.kv[0][0][0] + o_part<D>(r, part)) = acc;
                if (part == 0) { S.joined_m[r] = top; S.joined_l[r] = sum; }
            }
        };
        if (copies == 2) join(std::integral_constant<int, 2>{}); else join(std::integral_constant<int, 4>{});
    }
    const float *sM = copies > 1 ? S.joined_m : S.m, *sL = copies > 1 ? S.joined_l : S.l;
    // The sum: every CTA of the cluster has every nrank-th row. A thread per row for the factors, then one per 16 bytes of O, several of
    // which it has under way at once (a warp per row after row, factors by shuffles: 256 rows 36 us instead of 32, 1024 110 instead of 94).
    const int mine = (R - rank + nrank - 1) / nrank;
    float om = -INFINITY, ol = 0.0f;
    if (tid < mine) {
        const float* own = A.piece_of(S.row[tid * nrank + rank], h, 0, D);
        om = own[0];
        ol = own[1];
    }
    if (nrank > 1) cluster_sync(); else __syncthreads();
    auto sum_up = [&](auto n_tag) {
        constexpr int N = decltype(n_tag)::value, U = N == 1 ? 4 : 8 / N;
        if (tid < mine) {
            const int r = tid * N + rank;
            float pm[N], pl[N], top = om, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                pm[i] = ld_cluster(map_rank(smem_u32(&sM[r]), i));
                pl[i] = ld_cluster(map_rank(smem_u32(&sL[r]), i));
            }
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, pm[i]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float f = factor(pm[i], pl[i], top);
                if (f != 0.0f) sum += pl[i] * f;
                S.share[tid * N + i] = f;
            }
            const float of = factor(om, ol, top);
            if (of != 0.0f) sum += ol * of;
            S.own_share[tid] = of;
            S.over_sum[tid] = sum == 0.0f ? 0.0f : 1.0f / sum;
            A.lse[S.row[r] * A.Hq + h] = sum == 0.0f ? -INFINITY : top + logf(sum);
        }
        __syncthreads();
#pragma unroll 1
        for (int i0 = tid; i0 < mine * (D / 4); i0 += kThreads * U) {
            float4 v[U][N];
            float2 own[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kThreads, r = i / (D / 4) * N + rank, part = i % (D / 4);
                if (i >= mine * (D / 4)) continue;
#pragma unroll
                for (int x = 0; x < N; ++x) v[u][x] = ld_cluster4(map_rank(sO + o_part<D>(r, part), x));
                const float* piece = A.piece_of(S.row[r], h, 0, D) + 2 + part * 4;
                own[u][0] = *reinterpret_cast<const float2*>(piece);
                own[u][1] = *reinterpret_cast<const float2*>(piece + 2);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kThreads, k = i / (D / 4), part = i % (D / 4);
                if (i >= mine * (D / 4)) continue;
                float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float f = S.share[k * N + x];
                    if (f != 0.0f) add(acc, v[u][x], f);          // (what a part without keys left may be anything)
                }
                const float of = S.own_share[k], inv = S.over_sum[k];
                if (of != 0.0f) add(acc, make_float4(own[u][0].x, own[u][0].y, own[u][1].x, own[u][1].y), of);
                uint2 w = make_uint2(0u, 0u);
                if (inv != 0.0f) w = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                *reinterpret_cast<uint2*>((__nv_bfloat16*)A.o + S.row[k * N + rank] * A.os_row + h * A.os_head + part * 4) = w;
            }
        }
    };
    if (nrank == 1) sum_up(std::integral_constant<int, 1>{});
    else if (nrank == 2) sum_up(std::integral_constant<int, 2>{});
    else if (nrank == 4) sum_up(std::integral_constant<int, 4>{});
    else sum_up(std::integral_constant<int, 8>{});
    if (nrank > 1) cluster_sync();                                // (no CTA leaves while another may still read its sums)
    if (tid == 0 && S.abort_flag) atomicExch(A.status, (int32_t)DMA_ERR_DEVICE_TIMEOUT);
}

template <int D>
int launch(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st) {
    const int smem = (int)sizeof(Shared<D>) + 1024;
    if (cudaFuncSetAttribute(prefix_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return DMA_ERR_CUDA;
    // CTAs per (tile, head): as many as make three per SM, so that two are there although not every tile is, with 192 listed keys each at least (us of one rank and of two for 192 items of
    // 1024 keys 46 and 36; of four and of eight for 48 items of 1000 keys 12.8 and 17.7).
    const int64_t items = (int64_t)max_tiles * C.Hq, listed = std::min<int64_t>(C.w, A.order_ld);
    int ranks = 1;
    while (ranks < 8 && items * ranks * 2 <= 3 * 148 && ranks * 2 * 192 <= listed) ranks *= 2;
    return launch_overlapped(prefix_kernel<D>, dim3((unsigned)(items * ranks)), dim3(kThreads), smem, st, ranks, A, ranks);
}

}  // namespace

int launch_prefix_tc(const Cache& C, const DecodeArgs& A, int max_tiles, cudaStream_t st) {
    return C.d == 128 ? launch<128>(C, A, max_tiles, st) : launch<64>(C, A, max_tiles, st);
}

}  // namespace dma
