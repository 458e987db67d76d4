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

namespace dma {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// One CTA per (row, KV head); the last one groups the rows by prefix.
struct OwnShared {
    int count[kWarps], seen[kWarps];
    unsigned long long least[kWarps];
    float m[kWarps], l[kWarps];
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

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) own_kernel(DecodeArgs A, int room) {
    constexpr int C = D / 8;                                      // channels of a lane: eight lanes take a key
    extern __shared__ uint2 found[];                              // [kWarps][room]: (pattern of delta, position), then (delta, slot) of the kept ones
    __shared__ OwnShared S;
    __shared__ float sO[kWarps][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7, grp = lane >> 3;
    pdl_enter(A.q, A.kv, A.delta, A.table, A.seq, A.pos, A.prefix, A.order_slot, A.order_len, A.order_weight, A.o, A.lse, A.status, A.cut, A.piece, A.first, A.members, A.tiles, A.ntiles);
    if ((int)blockIdx.x == A.rows * A.Hkv) {
        if (tid < kWsHeaderBytes / 4) A.status[tid] = 0;
        group_rows(A);
        return;
    }
    const int t = blockIdx.x / A.Hkv, hk = blockIdx.x % A.Hkv;
    int r, listed;
    const int n = A.own(t, r);
    if (n < 0) return;
    const int pre = A.listed(t, listed);
    const int32_t* pages = A.table + r * A.ld;
    const int mask = (1 << A.page_log) - 1;
    const int team = max(1, kWarps / A.G), heads = kWarps / team, in_team = warp % team;       // warps of a head, heads at a time
    const T* kv = (const T*)A.kv;
    uint2* mine = found + warp * room;
    for (int g0 = 0; g0 < A.G; g0 += heads) {
        const int g = g0 + warp / team, h = hk * A.G + g;
        const bool active = warp / team < heads && g < A.G;
        const int leader = warp / team * team;
        const int seg = (n + team * 32 - 1) / (team * 32) * 32, j0 = min(n, in_team * seg), j1 = min(n, j0 + seg);
        const float* weight = A.order_weight + ((int64_t)pre * A.Hq + h) * A.order_ld;
        const uint32_t floor = active && pre >= 0 && listed == A.w ? __float_as_uint(weight[listed - 1]) & 0x7FFFFFFFu : 0u;
        const bool floored = pre >= 0 && listed == A.w;
        auto load = [&](int j, int& page, uint32_t& u) {
            page = -1;
            u = 0;
            if (j < j1) {
                page = pages[j >> A.page_log];
                if ((unsigned)page < (unsigned)A.num_pages) u = __float_as_uint(A.delta[(((size_t)page * A.Hq + h) << A.page_log) + (j & mask)]) & 0x7FFFFFFFu;
                else page = -1;
            }
        };
        // what may be kept
        int c = 0, seen = 0;
        if (active)
            for (int b = j0; b < j1; b += 32) {
                int page;
                uint32_t u;
                load(b + lane, page, u);
                const bool cand = page >= 0 && (!floored || u > floor);
                const uint32_t m = __ballot_sync(0xffffffffu, cand);
                const int at = c + __popc(m & ((1u << lane) - 1u));
                if (cand && at < room) mine[at] = make_uint2(u, b + lane);
                c += __popc(m);
                seen += __popc(__ballot_sync(0xffffffffu, page >= 0));
            }
        if (lane == 0) { S.count[warp] = c; S.seen[warp] = seen; }
        __syncthreads();
        if (active && in_team == 0) {
            int own = 0;
            bool over = false;
            for (int i = 0; i < team; ++i) {
                own += S.seen[warp + i];
                over |= S.count[warp + i] > room;
            }
            const int k = (int)min((int64_t)A.w, (int64_t)listed + own);
            // own keys whose order key is not below x
            auto at_least = [&](unsigned long long x) {
                int sum = 0;
                if (!over) {
                    for (int i = 0; i < team; ++i) {
                        const uint2* f = found + (warp + i) * room;
                        for (int e = lane; e < S.count[warp + i]; e += 32) sum += order_key(f[e].x, (int)f[e].y) >= x;
                    }
                } else {
                    for (int j = lane; j < n; j += 32) {
                        const int page = pages[j >> A.page_log];
                        if ((unsigned)page < (unsigned)A.num_pages)
                            sum += order_key(__float_as_uint(A.delta[(((size_t)page * A.Hq + h) << A.page_log) + (j & mask)]) & 0x7FFFFFFFu, j) >= x;
                    }
                }
                return __reduce_add_sync(0xffffffffu, sum);
            };
            auto above = [&](int m) { return (unsigned long long)((__float_as_uint(weight[m]) & 0x7FFFFFFFu) + 1u) << 32; };     // order keys greater than entry m's weight
            int cut = listed;
            unsigned long long least = 0;
            if (k < listed + own) {
                int lo = 0, hi = listed;
                while (lo < hi) {
                    const int m = (lo + hi) >> 1;
                    if (m + at_least(above(m)) >= k) hi = m; else lo = m + 1;
                }
                cut = lo;
                const int need = k - cut;
                if (need == 0) least = ~0ull;
                else {
                    // at_least(a) >= need >= at_least(b)
                    unsigned long long a = cut < listed ? above(cut) : 0, b = cut > 0 ? above(cut - 1) : 1ull << 63;
                    int at_a = at_least(a);
                    while (at_a != need && b - a > 1) {
                        const unsigned long long mid = a + (b - a) / 2;
                        const int x = at_least(mid);
                        if (x >= need) { a = mid; at_a = x; } else b = mid;
                    }
                    least = a;
                }
            }
            if (lane == 0) {
                S.least[warp] = least;
                A.cut[t * A.Hq + h] = cut;
            }
        }
        __syncthreads();
        // attention over the kept ones
        float m = -INFINITY, l = 0.0f, acc[C];
#pragma unroll
        for (int x = 0; x < C; ++x) acc[x] = 0.0f;
        if (active) {
            const unsigned long long least = S.least[leader];
            float qv[C];
            const T* q = (const T*)A.q + t * A.qs_row + h * A.qs_head + sub * C;
#pragma unroll
            for (int x = 0; x < C; ++x) qv[x] = to_f32(q[x]) * A.scale;
            const bool over = c > room;
            for (int b = 0; b < (over ? j1 - j0 : c);) {
                // as many kept ones as there is room for, at the front of the warp's part; in a call whose candidates did not fit, from the cache again
                int kept = 0;
                const int end = over ? j1 - j0 : c;
                for (; b < end && (!over || kept + 32 <= room); b += 32) {
                    uint32_t u = 0;
                    int j = -1, page = -1;
                    if (over) {
                        j = j0 + b + lane;
                        load(j, page, u);
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
                for (int i = 0; i < kept; i += 4) {
                    const bool real = i + grp < kept;
                    float s = 0.0f, v[C], bias = 0.0f;
#pragma unroll
                    for (int x = 0; x < C; ++x) v[x] = 0.0f;
                    if (real) {
                        const uint2 e = mine[i + grp];
                        bias = __uint_as_float(e.x);
                        const T* row = kv + key_row((int)e.y >> A.page_log, hk, (int)e.y & mask, A.Hkv, A.page_log) * (2 * D) + sub * C;
                        float kk[C];
#pragma unroll
                        for (int x = 0; x < C; x += 8) {
                            load8(row + x, *reinterpret_cast<float(*)[8]>(kk + x));
                            load8(row + D + x, *reinterpret_cast<float(*)[8]>(v + x));
                        }
#pragma unroll
                        for (int x = 0; x < C; ++x) s = fmaf(qv[x], kk[x], s);
                    }
#pragma unroll
                    for (int x = 1; x < 8; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
                    s = real ? s + bias : -INFINITY;
                    float top = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    top = fmaxf(m, top);
                    // (a NaN score leaves no maximum and makes the sum NaN; so does one of +inf)
                    const float ref = top == -INFINITY ? 0.0f : top, fade = m == -INFINITY ? 0.0f : expf(m - ref), p = real ? expf(s - ref) : 0.0f;
                    m = top;
                    l = l * fade + p;
#pragma unroll
                    for (int x = 0; x < C; ++x) acc[x] = (fade == 0.0f ? 0.0f : acc[x] * fade) + (real ? p * v[x] : 0.0f);
                }
                __syncwarp();
            }
        }
        // the four keys side by side, then the team's warps
#pragma unroll
        for (int x = 8; x < 32; x <<= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, x);
#pragma unroll
            for (int y = 0; y < C; ++y) acc[y] += __shfl_xor_sync(0xffffffffu, acc[y], x);
        }
        if (lane == 0) { S.m[warp] = m; S.l[warp] = l; }
        if (grp == 0)
#pragma unroll
            for (int x = 0; x < C; ++x) sO[warp][sub * C + x] = acc[x];
        __syncthreads();
        if (active) {
            float top = -INFINITY, sum = 0.0f, f[kWarps];
            for (int i = 0; i < team; ++i) top = fmaxf(top, S.m[leader + i]);
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                f[i] = 0.0f;
                if (i < team) {
                    const float mi = S.m[leader + i], li = S.l[leader + i];
                    f[i] = mi == -INFINITY ? (li == 0.0f ? 0.0f : 1.0f) : expf(mi - top);
                    sum += li * f[i];
                }
            }
            float* out = A.piece_of(t, h, 0, D);
            for (int x = in_team * 32 + lane; x < D; x += team * 32) {
                float a = 0.0f;
#pragma unroll
                for (int i = 0; i < kWarps; ++i)
                    if (i < team && f[i] != 0.0f) a += sO[leader + i][x] * f[i];
                if (pre >= 0) out[2 + x] = a;
                else store_as((T*)A.o + t * A.os_row + h * A.os_head + x, sum == 0.0f ? 0.0f : a / sum);
            }
            if (in_team == 0 && lane == 0) {
                if (pre >= 0) { out[0] = top; out[1] = sum; }
                else A.lse[t * A.Hq + h] = sum == 0.0f ? -INFINITY : top + logf(sum);
            }
        }
        __syncthreads();
    }
}

template <typename T, int D>
int own(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    // Room for every own key of the heads that a CTA takes at a time, up to 128 KB.
    const int64_t capacity = (int64_t)C.max_blocks << C.page_log;
    const int team = std::max(1, kWarps / C.G);
    const int room = (int)std::min<int64_t>(std::max<int64_t>((capacity + team * 32 - 1) / (team * 32) * 32, 64), 2048);
    const size_t smem = (size_t)kWarps * room * sizeof(uint2);
    if (smem > 32 * 1024 && cudaFuncSetAttribute(own_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(own_kernel<T, D>, dim3((unsigned)(C.rows * C.Hkv + 1)), dim3(kThreads), smem, st, 1, A, room);
}

}  // namespace

int launch_own_keys(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    auto f = C.dtype == DMA_BF16 ? (C.d == 128 ? own<__nv_bfloat16, 128> : own<__nv_bfloat16, 64>) : (C.d == 128 ? own<float, 128> : own<float, 64>);
    return f(C, A, st);
}

}  // namespace dma
