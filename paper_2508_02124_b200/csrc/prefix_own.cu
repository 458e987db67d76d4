// First half of dma_cache_decode (include/dma.h): what every row keeps of its prefix' order and of its own keys, and the attention over the latter.
//
// The cut. A row's head keeps k = min(w, listed + own) keys of the merged order. Entry m of the prefix' order has m entries before it and every own key that is greater; so the
// prefix' part ends with the first m for which m + #{own > weight_m} >= k, a bisection (ties: the prefix' keys come first), and the own part is the k - m best of the row's own
// keys, a bisection over their order keys between the weights around the cut. Where the list has w entries, own keys that do not exceed its last cannot be kept and are left out
// at once: of n own keys behind a prefix of N about n w / N remain. They lie in shared memory, where every count is a sweep by one warp.
#include <algorithm>

#include "cache4_decode.cuh"
#include "delta_fixed.cuh"
#include "prefix_decode.cuh"
#include "sm100_ptx.cuh"

namespace dma {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// A team of 1, 2, 4 or 8 warps has a (row, head), each warp a part of the own keys.
struct OwnShared {
    uint64_t full[kWarps];
    int part[2][kWarps], seen[kWarps], cands[kWarps];
    float m[kWarps], l[kWarps];
    int abort_flag, drain_flag;
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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(ptx::smem_u32(bar)) : "memory");
}
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
    __device__ __forceinline__ void stage(uint8_t* keys, const uint2* list, int count, int lane) {
#pragma unroll 1
        for (int i = 0; i < count; i += 4) {
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
            s = e < count ? s + __uint_as_float(list[e].x) : -INFINITY;
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
    __device__ __forceinline__ void stage(uint8_t* keys, const uint2* list, int count, int lane) {
        if (count < kStage) {                                     // (0 times what lies there must be 0)
            for (int i = count * (D / 8) + lane; i < kStage * (D / 8); i += 32) *reinterpret_cast<uint4*>(keys + i / (D / 8) * kPitch + D * 2 + i % (D / 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
        }
        const uint32_t base = ptx::smem_u32(keys), at_k = base + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + (lane >> 4) * 16;
        const uint32_t at_v = base + ((lane & 7) + (lane >> 4) * 8) * kPitch + D * 2 + ((lane >> 3) & 1) * 16;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            uint32_t a[4];
            ldmatrix<false>(a, at_k + x * 32);
            mma_16816(s, a, q[x][0], q[x][1]);
        }
        // lane 4 i has the scores of keys i and i + 8
        const int e = lane >> 2;
        const bool real0 = (lane & 3) == 0 && e < count, real1 = (lane & 3) == 0 && e + 8 < count;
        const float x0 = real0 ? fmaf(s[0], c1, __uint_as_float(list[e].x) * 1.4426950408889634f) : -INFINITY;
        const float x1 = real1 ? fmaf(s[2], c1, __uint_as_float(list[e + 8].x) * 1.4426950408889634f) : -INFINITY;
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
        const float ref = m == -INFINITY ? 0.0f : m, p0 = real0 ? ptx::ex2(x0 - ref) : 0.0f, p1 = real1 ? ptx::ex2(x1 - ref) : 0.0f;
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

__device__ void group_rows(const DecodeArgs& A) {
    __shared__ int part[kWarps], tile_part[kWarps], turn[kThreads];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto prefix_of = [&](int t) {
        int r, n;
        return A.own(t, r) < 0 ? -1 : A.listed(t, n);
    };
    if (A.nprefix == 0) {
        if (tid == 0) *A.ntiles = 0;
        return;
    }
    for (int i = tid; i <= A.nprefix; i += kThreads) A.first[i] = 0;
    __syncthreads();
    for (int t = tid; t < A.rows; t += kThreads) {
        const int g = prefix_of(t);
        if (g >= 0) atomicAdd(&A.first[g], 1);
    }
    __syncthreads();
    int row_carry = 0, tile_carry = 0;
    for (int b = 0; b < A.nprefix; b += kThreads) {
        const int g = b + tid, n = g < A.nprefix ? __ldcg(&A.first[g]) : 0, nt = (n + A.tile_rows - 1) / A.tile_rows;
        int x = n, y = nt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) { x += u; y += v; }
        }
        if (lane == 31) { part[warp] = x; tile_part[warp] = y; }
        __syncthreads();
        int before = 0, tiles_before = 0, all = 0, all_tiles = 0;
        for (int i = 0; i < kWarps; ++i) {
            before += i < warp ? part[i] : 0;
            tiles_before += i < warp ? tile_part[i] : 0;
            all += part[i];
            all_tiles += tile_part[i];
        }
        if (g < A.nprefix) {
            const int start = row_carry + before + x - n;
            __stcg(&A.first[g], start);
            for (int i = 0; i < nt; ++i)
                A.tiles[tile_carry + tiles_before + y - nt + i] = make_int4(g, start + i * A.tile_rows, min(A.tile_rows, n - i * A.tile_rows), 0);
        }
        row_carry += all;
        tile_carry += all_tiles;
        __syncthreads();
    }
    if (tid == 0) *A.ntiles = tile_carry;
    // in the order of rows: a turn's rows of the same prefix follow one another, the first of them moves the prefix' start on
    for (int b = 0; b < A.rows; b += kThreads) {
        const int t = b + tid, g = t < A.rows ? prefix_of(t) : -1;
        turn[tid] = g;
        __syncthreads();
        int rank = 0, same = 0;
        if (g >= 0)
            for (int i = 0; i < kThreads; ++i) {
                same += turn[i] == g;
                rank += turn[i] == g && i < tid;
            }
        int start = 0;
        if (g >= 0) start = __ldcg(&A.first[g]);
        __syncthreads();
        if (g >= 0) {
            A.members[start + rank] = t;
            if (rank == 0) __stcg(&A.first[g], start + same);
        }
        __syncthreads();
    }
}

// One CTA per kWarps / team (row, head)s; the last one groups the rows by prefix.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) own_kernel(DecodeArgs A, int team, int room) {
    constexpr int kBatch = 4, kHeld = 4;                          // 128 keys each, requested together; candidates, and entries of the order, that a lane holds
    using At = Attend<T, D>;
    extern __shared__ __align__(16) uint8_t dynamic[];            // [kWarps][At::kStage][At::kPitch] keys, [kWarps][room]: (pattern of delta, position), then (delta, slot) of the kept ones
    __shared__ OwnShared S;
    __shared__ float sO[kWarps][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < kWarps) ptx::mbar_init(&S.full[tid], 1);
    if (tid == 0) S.abort_flag = S.drain_flag = 0;
    ptx::fence_barrier_init();
    pdl_enter(A.q, A.kv, A.delta, A.table, A.seq, A.pos, A.prefix, A.order_slot, A.order_len, A.order_weight, A.o, A.lse, A.status, A.cut, A.piece, A.first, A.members, A.tiles, A.ntiles);
    __syncthreads();
    if (blockIdx.x == gridDim.x - 1) {
        if (tid < kWsHeaderBytes / 4) A.status[tid] = 0;
        group_rows(A);
        return;
    }
    const int in_team = warp % team, leader = warp - in_team, teams = kWarps / team, bar = 1 + warp / team;
    const int64_t item = (int64_t)blockIdx.x * teams + warp / team;
    if (item >= (int64_t)A.rows * A.Hq) return;                   // (a team's barrier counts its own warps only)
    const int t = (int)(item / A.Hq), h = (int)(item % A.Hq), hk = h / A.G;
    const int r = A.seq[t], p = A.pos[t], g = A.nprefix ? A.prefix[t] : -1;
    if ((unsigned)r >= (unsigned)A.nseq) return;
    const int n = min(max(p, -1), (A.max_blocks << A.page_log) - 1) + 1;
    const int32_t* pages = A.table + r * A.ld;
    const int mask = (1 << A.page_log) - 1, seg = (n + team * 128 - 1) / (team * 128) * 128, j0 = min(n, in_team * seg), j1 = min(n, j0 + seg);
    const T* kv = (const T*)A.kv;
    uint8_t* keys_at = dynamic + warp * (At::kStage * At::kPitch);
    uint2* found = reinterpret_cast<uint2*>(dynamic + kWarps * (At::kStage * At::kPitch));
    uint2* mine = found + warp * room;
    auto page_of = [&](int j) {                                   // -1: outside the pool, or no key
        int page = j < j1 ? pages[j >> A.page_log] : -1;
        return (unsigned)page < (unsigned)A.num_pages ? page : -1;
    };
    auto delta_at = [&](int page, int j) { return A.delta + (((size_t)page * A.Hq + h) << A.page_log) + (j & mask); };
    // f(position, page, pattern, is a key) for the part's keys, four side by side per lane (in one page, since pages have 16 keys and more)
    auto sweep = [&](auto f) {
        int page[kBatch], next[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) next[i] = page_of(j0 + 128 * i + 4 * lane);
#pragma unroll 1
        for (int b = j0; b < j1; b += 128 * kBatch) {
            uint4 u[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                page[i] = next[i];
                if (page[i] >= 0) u[i] = *reinterpret_cast<const uint4*>(delta_at(page[i], b + 128 * i + 4 * lane));
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) next[i] = page_of(b + 128 * (kBatch + i) + 4 * lane);
            f(b, page, u);
        }
    };
    int listed = 0;
    if ((unsigned)g < (unsigned)A.nprefix) listed = (int)max((int64_t)0, min((int64_t)min(A.order_len[g], A.w), A.order_ld));
    const bool behind = listed > 0, floored = listed == A.w;      // (as DecodeArgs::listed)
    const float* weight = A.order_weight + ((int64_t)g * A.Hq + h) * A.order_ld;
    // the last entries of the order, from the end on
    uint32_t held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = listed - 1 - 32 * i - lane >= 0 ? __float_as_uint(weight[listed - 1 - 32 * i - lane]) & 0x7FFFFFFFu : 0u;
    const uint32_t floor = __shfl_sync(0xffffffffu, held[0], 0);
    auto word = [](const uint4& u, int x) { return (x == 0 ? u.x : x == 1 ? u.y : x == 2 ? u.z : u.w) & 0x7FFFFFFFu; };
    // what may be kept
    int c = 0, seen = 0;
    sweep([&](int b, const int (&page)[kBatch], const uint4 (&u)[kBatch]) {
        uint32_t flags = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const bool there = page[i] >= 0 && b + 128 * i + 4 * lane + x < j1;
                seen += there;
                flags |= (uint32_t)(there && (!floored || word(u[i], x) > floor)) << (4 * i + x);
            }
        const int mine_count = __popc(flags);
        int at = mine_count;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += y;
        }
        const int total = __shfl_sync(0xffffffffu, at, 31);
        at += c - mine_count;
#pragma unroll
        for (int i = 0; i < 4 * kBatch; ++i)
            if (flags >> i & 1u) {
                if (at < room) mine[at] = make_uint2(word(u[i / 4], i % 4), b + 128 * (i / 4) + 4 * lane + i % 4);
                ++at;
            }
        c += total;
    });
    seen = __reduce_add_sync(0xffffffffu, seen);
    const bool over = c > room;
    __syncwarp();
    int own = seen, cands = c, most = c, step = 0;
    if (team > 1) {
        if (lane == 0) { S.seen[warp] = seen; S.cands[warp] = c; }
        team_sync(bar, team * 32);
        own = cands = most = 0;
        for (int i = 0; i < team; ++i) {
            own += S.seen[leader + i];
            cands += S.cands[leader + i];
            most = max(most, S.cands[leader + i]);
        }
    }
    auto team_sum = [&](int x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (team > 1) {
            if (lane == 0) S.part[step & 1][warp] = x;
            team_sync(bar, team * 32);
            x = 0;
            for (int i = 0; i < team; ++i) x += S.part[step & 1][leader + i];
            ++step;
        }
        return x;
    };
    const int k = (int)min((int64_t)A.w, (int64_t)listed + own);
    int cut = listed;
    unsigned long long least = 0;
    if (k < listed + own) {
        unsigned long long keys[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) keys[i] = !over && 32 * i + lane < c ? order_key(mine[32 * i + lane].x, (int)mine[32 * i + lane].y) : 0ull;
        if (most <= 32 * kHeld && most <= room && cands <= 32 * kHeld) {
            // Few candidates: each against all, and against as many of the last entries. One is kept if fewer than k keys come before it; of the prefix' those that are not below it, and
            // all entries further up are at most another reason to keep it.
            int before[kHeld];
#pragma unroll
            for (int i = 0; i < kHeld; ++i) before[i] = listed;
            for (int w = leader; w < leader + team; ++w) {
                const uint2* f = found + w * room;
                const int count = w == warp ? c : S.cands[w];
                for (int e = 0; e < count; ++e) {
                    const uint2 o = f[e];
                    const unsigned long long x = order_key(o.x, (int)o.y);
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) before[i] += x > keys[i];
                }
            }
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (32 * i < cands) {
                    const int end = min(32, min(cands, listed) - 32 * i);
                    for (int e = 0; e < end; ++e) {
                        const uint32_t x = __shfl_sync(0xffffffffu, held[i], e);
#pragma unroll
                        for (int y = 0; y < kHeld; ++y) before[y] -= x < (uint32_t)(keys[y] >> 32);
                    }
                }
            // the kept ones to the front of the warp's part
            int kept = 0;
            team_sync(bar, team * 32);                            // (all have read)
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                const bool keep = 32 * i + lane < c && before[i] < k;
                const uint32_t bits = __ballot_sync(0xffffffffu, keep);
                const uint2 o = keep ? mine[32 * i + lane] : make_uint2(0u, 0u);
                __syncwarp();
                if (keep) mine[kept + __popc(bits & ((1u << lane) - 1u))] = o;
                kept += __popc(bits);
                __syncwarp();
            }
            c = kept;
            cut = k - team_sum(lane == 0 ? kept : 0);
        } else {
            // order keys greater than entry m's weight
            auto above = [&](int m) {
                const int back = listed - 1 - m;
                uint32_t u = held[0];
#pragma unroll
                for (int i = 1; i < kHeld; ++i) u = back >> 5 == i ? held[i] : u;
                u = back < 32 * kHeld ? __shfl_sync(0xffffffffu, u, back & 31) : __float_as_uint(weight[m]) & 0x7FFFFFFFu;
                return (unsigned long long)(u + 1u) << 32;
            };
            // Each own key takes at most one entry's place, so that the cut lies among the last `cands` entries (k >= listed): bisection of the cut, then of the weakest kept own key between
            // a, which `need` own keys or more are not below, and b, which at most so many are not below.
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
                if (!over) {
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) sum += keys[i] >= x;
                    for (int e = 32 * kHeld + lane; e < c; e += 32) sum += order_key(mine[e].x, (int)mine[e].y) >= x;
                } else {
                    sweep([&](int base, const int (&page)[kBatch], const uint4 (&u)[kBatch]) {
#pragma unroll
                        for (int i = 0; i < kBatch; ++i)
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const int j = base + 128 * i + 4 * lane + y;
                                sum += page[i] >= 0 && j < j1 && order_key(word(u[i], y), j) >= x;
                            }
                    });
                }
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
    if (in_team == 0 && lane == 0) A.cut[item] = cut;
    // attention over the kept ones, a stage of keys at a time: a bulk copy per key
    At at;
    at.start((const T*)A.q + t * A.qs_row + h * A.qs_head, A.scale, lane);
    uint32_t phase = 0;
    bool ok = true;
    for (int b = 0; b < (over ? j1 - j0 : c) && ok;) {
        // as many kept ones as there is room for, at the front of the warp's part; where its candidates did not fit, from the cache again
        int kept = 0;
        const int end = over ? j1 - j0 : c;
        for (; b < end && (!over || kept + 32 <= room); b += 32) {
            uint32_t u = 0;
            int j = -1, page = -1;
            if (over) {
                j = j0 + b + lane;
                page = page_of(j);
                if (page >= 0) u = __float_as_uint(*delta_at(page, j)) & 0x7FFFFFFFu;
            } else if (b + lane < c) {
                u = mine[b + lane].x;
                j = (int)mine[b + lane].y;
                page = pages[j >> A.page_log];
            }
            const bool keep = page >= 0 && order_key(u, j) >= least && (!floored || u > floor);
            const uint32_t bits = __ballot_sync(0xffffffffu, keep);            // (behind every lane's read)
            if (keep) mine[kept + __popc(bits & ((1u << lane) - 1u))] = make_uint2(u, (page << A.page_log) + (j & mask));
            kept += __popc(bits);
            __syncwarp();
        }
#pragma unroll 1
        for (int i = 0; i < kept && ok; i += At::kStage) {
            const int count = min(kept - i, At::kStage);
            ptx::fence_proxy_async();                             // (the stage before has been read)
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_expect_tx(&S.full[warp], count * 2 * D * (uint32_t)sizeof(T));
            __syncwarp();
            if (lane < count) {
                const int slot = (int)mine[i + lane].y;
                bulk_load(ptx::smem_u32(keys_at + lane * At::kPitch), kv + key_row(slot >> A.page_log, hk, slot & mask, A.Hkv, A.page_log) * (2 * D), 2 * D * sizeof(T), &S.full[warp]);
            }
            ok = ptx::mbar_wait_warp(&S.full[warp], phase, &S.abort_flag);
            phase ^= 1u;
            if (ok) at.stage(keys_at, mine + i, count, lane);
            __syncwarp();
        }
    }
    if (!ok) {
        ptx::mbar_wait_warp(&S.full[warp], phase ^ 1u, &S.drain_flag);      // (copies in flight)
        if (lane == 0) atomicExch(A.status, (int32_t)DMA_ERR_DEVICE_TIMEOUT);
    }
    at.end(sO[warp], lane);
    if (lane == 0) { S.m[warp] = at.m; S.l[warp] = at.l; }
    team_sync(bar, team * 32);
    float top = -INFINITY, sum = 0.0f;
    for (int i = 0; i < team; ++i) top = fmaxf(top, S.m[leader + i]);
    auto factor = [&](int w) { return S.m[w] == -INFINITY ? (S.l[w] == 0.0f ? 0.0f : 1.0f) : expf(S.m[w] - top); };
    for (int i = 0; i < team; ++i) sum += S.l[leader + i] * factor(leader + i);
    float* out = A.piece_of(t, h, 0, D);
    for (int x = in_team * 32 + lane; x < D; x += team * 32) {
        float a = 0.0f;
        for (int i = 0; i < team; ++i) {
            const float f = factor(leader + i);
            if (f != 0.0f) a += sO[leader + i][x] * f;
        }
        if (behind) out[2 + x] = a;
        else store_as((T*)A.o + t * A.os_row + h * A.os_head + x, sum == 0.0f ? 0.0f : a / sum);
    }
    if (in_team == 0 && lane == 0) {
        if (behind) { out[0] = top; out[1] = sum; }
        else A.lse[item] = sum == 0.0f ? -INFINITY : top + logf(sum);
    }
}

// Warps per (row, head): as many as make the chip's SMs have 16 of them, and so many that a row's own keys find room as candidates, at most 512 per warp.
template <typename T, int D>
int own(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    const int64_t capacity = (int64_t)C.max_blocks << C.page_log, items = (int64_t)C.rows * C.Hq;
    int team = 1;
    while (team < kWarps && (items * team * 2 <= 16 * 148 || capacity > 1024 * team)) team *= 2;
    const int room = (int)std::min<int64_t>((capacity + team * 128 - 1) / (team * 128) * 128, 512);
    const size_t smem = (size_t)kWarps * (room * sizeof(uint2) + Attend<T, D>::kStage * Attend<T, D>::kPitch);
    if (cudaFuncSetAttribute(own_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return DMA_ERR_CUDA;
    const int64_t per = kWarps / team;
    return launch_overlapped(own_kernel<T, D>, dim3((unsigned)((items + per - 1) / per + 1)), dim3(kThreads), smem, st, 1, A, team, room);
}

}  // namespace

int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? own<__nv_bfloat16, 128> : own<__nv_bfloat16, 64>) : (C.d == 128 ? own<float, 128> : own<float, 64>);
    return f(C, A, st);
}

}  // namespace dma
