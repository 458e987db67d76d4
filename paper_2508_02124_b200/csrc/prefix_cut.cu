// First step of dma_cache_decode (include/dma.h): what every row keeps of its prefix' order and of its own keys, and the rows grouped by prefix.
//
// A row's head keeps k = min(w, listed + own) keys of the merged order. Entry m of the prefix' order has m entries before it and every own key that is greater; so the prefix' part ends
// with the first m for which m + #{own > weight_m} >= k (ties: the prefix' keys come first), and the own part is the k - m best of the row's own keys. Put the other way: the best own key
// is kept if the list's last entry is below it, the second if the last but one is, and so on. Where the list has w entries, own keys that do not exceed its last cannot be kept and are
// left out at once: of n own keys behind a prefix of N about n w / N remain. They lie in shared memory, per warp.
// Bound by latency: five dependent trips to memory and some hundred instructions one behind the other. 64 rows of 1 to 1024 own keys, 32 heads: FIG us.
#include <algorithm>
#include <type_traits>

#include "cache4_decode.cuh"
#include "prefix_decode.cuh"

#ifndef CUTFILL
#define CUTFILL 24
#endif
namespace dma {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kRoom = 1024;

struct CutShared {
    unsigned long long least[kWarps];
    int part[2][kWarps], cands[kWarps], cut[kWarps];
    uint32_t low[kWarps], high[kWarps], sorted[kWarps][64];
};

// The rows by prefix, in the order of rows, and tiles of them.
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

// R * 32 numbers of a warp in descending order, number i * 32 + lane in v[i].
template <int R>
__device__ __forceinline__ void sort_down(uint32_t (&v)[R], int lane) {
    auto lanes = [&](int k, int j) {                              // pairs that j < 32 lanes part, in runs of k
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint32_t o = __shfl_xor_sync(0xffffffffu, v[i], j);
            const bool up = ((lane & j) == 0) == (((i * 32 + lane) & k) == 0);
            v[i] = up ? max(v[i], o) : min(v[i], o);
        }
    };
#pragma unroll 1
    for (int k = 2; k <= 32; k *= 2)
#pragma unroll 1
        for (int j = k / 2; j > 0; j /= 2) lanes(k, j);
#pragma unroll
    for (int k = 64; k <= 32 * R; k *= 2) {
#pragma unroll
        for (int j = k / 2; j >= 32; j /= 2)
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (!(i & (j / 32))) {
                    const int o = i | (j / 32);
                    const uint32_t a = v[i], b = v[o];
                    const bool down = ((i * 32) & k) == 0;
                    v[i] = down ? max(a, b) : min(a, b);
                    v[o] = down ? min(a, b) : max(a, b);
                }
#pragma unroll 1
        for (int j = 16; j > 0; j /= 2) lanes(k, j);
    }
}

// A CTA per (row, KV head) or part of its heads; the first one groups the rows by prefix.
template <bool kTeams>
__global__ void __launch_bounds__(kThreads, 3) cut_kernel(DecodeArgs A, int warps_per_head, int room, int heads) {
    extern __shared__ uint2 found[];                              // of each warp [room]: (pattern of delta, position) of candidates
    __shared__ CutShared S;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x / 32, team = kTeams ? warps_per_head : 1;
    pdl_enter();
    if (blockIdx.x == 0) {                                        // (first: it is done while the others are at work)
        if (tid < kWsHeaderBytes / 4) A.status[tid] = 0;
        group_rows(A, reinterpret_cast<int*>(found));
        return;
    }
    OwnRow R;
    if (!R.find(A, blockIdx.x - 1, heads)) return;
    const int t = R.t, n = R.n, listed = R.listed;
    const bool floored = listed == A.w;
    if (R.keeps_all(A)) {
        for (int head = R.head0 + tid; head < R.head1; head += blockDim.x) {
            A.cut[t * A.Hq + R.hk * A.G + head] = listed;
            A.least[t * A.Hq + R.hk * A.G + head] = 0ull;
        }
        return;
    }
    const int in_team = kTeams ? warp % team : 0, leader = warp - in_team, bar = 1 + warp / team;
    uint2* mine = found + warp * room;
    const int seg = (n + team * 64 - 1) / (team * 64) * 64, j0 = min(n, in_team * seg), j1 = min(n, j0 + seg);
    int step = 0;
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
#pragma unroll 1
    for (int head = R.head0 + warp / team; head < R.head1; head += warps / team) {
        const int h = R.hk * A.G + head;
        const float* weight = A.order_weight + ((int64_t)(listed ? A.prefix[t] : 0) * A.Hq + h) * A.order_ld;
        auto pattern = [&](int m) { return __float_as_uint(weight[m]) & 0x7FFFFFFFu; };
        // what may be kept: every key that there is, or those above the list's last entry
        const int floor = floored ? (int)pattern(listed - 1) : -1;
        int c = 0;
        sweep_own(A, R, h, j0, j1, [&](int j, int, const int (&u)[16]) {
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
                    if (u[i] > floor) mine[to++] = make_uint2((uint32_t)u[i], (uint32_t)(j + i));
            }
            c += total;
        });
        if (lane == 0) S.cands[warp] = c;
        team_sync(bar, team * 32);
        int cands = 0, most = 0;
        for (int i = 0; i < team; ++i) {
            cands += S.cands[leader + i];
            most = max(most, S.cands[leader + i]);
        }
        const bool over = most > room;
        // (all own keys are candidates where the list may not be full)
        const int k = floored ? listed : (int)min((int64_t)A.w, (int64_t)listed + cands);
        int cut = listed;
        unsigned long long least = 0;                             // kept: the order keys that are not below
        // the i-th best own key, and one of this many entries from the list's end on, plus one: it has to be above that
        auto rival = [&](int i) {
            const int back = i - (k - listed);
            return back < 0 ? 0u : back < listed ? pattern(listed - 1 - back) + 1u : ~0u;
        };
        // equal ones, of which the first `need` are kept: the last of these
        auto among_equals = [&](uint32_t u, int need) {
            for (int x = leader; x < leader + team; ++x)
                for (int e = 0; e < S.cands[x]; e += 32) {
                    const uint32_t same = __ballot_sync(0xffffffffu, e + lane < S.cands[x] && found[x * room + e + lane].x == u);
                    if (__popc(same) >= need) return order_key(u, (int)found[x * room + e + __fns(same, 0, need)].y);
                    need -= __popc(same);
                }
            return 0ull;
        };
        bool done = k >= listed + cands;
        if (!kTeams && !done && floored && cands <= 128) {
            // Few candidates fail against a full list: the lowest one is dropped as long as it does.
            unsigned long long keys[4];
            uint32_t last[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 32 * i + lane;
                last[i] = e < cands ? rival(e) : ~0u;
                keys[i] = e < c ? order_key(mine[e].x, (int)mine[e].y) : ~0ull;
            }
            for (int kept = cands; kept >= cands - 16 && !done; --kept) {
                unsigned long long low = keys[0] < keys[1] ? keys[0] : keys[1];
                const unsigned long long other = keys[2] < keys[3] ? keys[2] : keys[3];
                low = other < low ? other : low;
                const uint32_t hi = __reduce_min_sync(0xffffffffu, (uint32_t)(low >> 32)), lo = __reduce_min_sync(0xffffffffu, (uint32_t)(low >> 32) == hi ? (uint32_t)low : ~0u);
                const int back = max(kept - 1, 0);
                const uint32_t a = back & 32 ? last[1] : last[0], b = back & 32 ? last[3] : last[2], bar_to_pass = __shfl_sync(0xffffffffu, back & 64 ? b : a, back & 31);
                if (kept == 0 || hi + 1u > bar_to_pass) {
                    done = true;
                    least = kept == 0 ? ~0ull : (unsigned long long)hi << 32 | lo;
                    cut = k - kept;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) keys[i] = keys[i] == ((unsigned long long)hi << 32 | lo) ? ~0ull : keys[i];
                }
            }
        }
        if (!kTeams && !done && !over && cands <= 256) {
            // all of them, sorted, against the list from its end on
            auto match = [&](auto r_tag) {
                constexpr int N = decltype(r_tag)::value;
                uint32_t v[N], w[N];                              // (patterns plus one: 0 is none)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    w[i] = rival(i * 32 + lane);
                    v[i] = i * 32 + lane < c ? mine[i * 32 + lane].x + 1u : 0u;
                }
                sort_down<N>(v, lane);
                int kept = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) kept += __popc(__ballot_sync(0xffffffffu, v[i] > w[i]));       // (the first so many)
                cut = k - kept;
                uint32_t last = 0u, next = 0u;                    // the weakest kept one, and the one behind it
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if ((kept - 1) >> 5 == i) last = v[i];
                    if (kept >> 5 == i) next = v[i];
                }
                last = __shfl_sync(0xffffffffu, last, (kept - 1) & 31);
                next = __shfl_sync(0xffffffffu, next, kept & 31);
                if (kept >= 32 * N) next = 0u;
                least = kept == 0 ? ~0ull : (unsigned long long)(last - 1u) << 32;
                if (kept > 0 && next == last) {
                    int better = 0;
#pragma unroll
                    for (int i = 0; i < N; ++i) better += __popc(__ballot_sync(0xffffffffu, v[i] > last));
                    least = among_equals(last - 1u, kept - better);
                }
            };
            if (cands <= 32) match(std::integral_constant<int, 1>{});
            else if (cands <= 64) match(std::integral_constant<int, 2>{});
            else if (cands <= 128) match(std::integral_constant<int, 4>{});
            else match(std::integral_constant<int, 8>{});
            done = true;
        }
        if (kTeams && !done && most <= 64) {
            // every warp its own, sorted; a key's rank is the sum of its ranks in all of them (equal ones by warp)
            uint32_t v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = i * 32 + lane < c ? mine[i * 32 + lane].x + 1u : 0u;
            sort_down<2>(v, lane);
            S.sorted[warp][lane] = v[0];
            S.sorted[warp][lane + 32] = v[1];
            team_sync(bar, team * 32);
            int rank[2] = {lane, 32 + lane};
            for (int x = leader; x < leader + team; ++x) {
                if (x == warp) continue;
                const uint32_t more = x < warp ? 1u : 0u;         // numbers in front: those not below v + 1 - more
                int lo[2] = {0, 0};
#pragma unroll
                for (int b = 32; b > 0; b /= 2)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (S.sorted[x][lo[i] + b - 1] >= v[i] + 1u - more) lo[i] += b;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (lo[i] == 63 && S.sorted[x][63] >= v[i] + 1u - more) lo[i] = 64;
                    rank[i] += lo[i];
                }
            }
            uint32_t low = ~0u, high = 0u;                        // the weakest kept one, and the best of the others
            int mine_kept = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool keep = v[i] > 0u && v[i] > rival(rank[i]);
                mine_kept += keep;
                if (keep) low = min(low, v[i]); else high = max(high, v[i]);
            }
            const int kept = team_sum(mine_kept);
            low = __reduce_min_sync(0xffffffffu, low);
            high = __reduce_max_sync(0xffffffffu, high);
            if (lane == 0) { S.low[warp] = low; S.high[warp] = high; }
            team_sync(bar, team * 32);
            for (int i = 0; i < team; ++i) {
                low = min(low, S.low[leader + i]);
                high = max(high, S.high[leader + i]);
            }
            cut = k - kept;
            least = kept == 0 ? ~0ull : (unsigned long long)(low - 1u) << 32;
            if (kept > 0 && high == low) least = among_equals(low - 1u, kept - team_sum((v[0] > low) + (v[1] > low)));
            done = true;
        }
        if (!done) {
            // Each own key takes at most one entry's place, so that the cut lies among the last `cands` entries (k >= listed): bisection of the cut, then of the weakest kept own key between
            // a, which `need` own keys or more are not below, and b, which at most so many are not below.
            auto above = [&](int m) { return (unsigned long long)(pattern(m) + 1u) << 32; };          // order keys greater than entry m's weight
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
                    for (int e = lane; e < c; e += 32) sum += order_key(mine[e].x, (int)mine[e].y) >= x;
                } else {                                          // (those that did not fit, from the cache again)
                    sweep_own(A, R, h, j0, j1, [&](int j, int, const int (&u)[16]) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += u[i] > floor && order_key((uint32_t)u[i], j + i) >= x;
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
        if (in_team == 0 && lane == 0) {
            A.cut[t * A.Hq + h] = cut;
            A.least[t * A.Hq + h] = max(least, (unsigned long long)(uint32_t)(floor + 1) << 32);
        }
        team_sync(bar, team * 32);
    }
}

}  // namespace

int launch_cuts(const Cache& C, const DecodeArgs& A, cudaStream_t st) {
    const Teams T(C, CUTFILL, kRoom);
    const int64_t capacity = (int64_t)C.max_blocks << C.page_log;
    const int room = (int)std::min<int64_t>((capacity + T.team * 64 - 1) / (T.team * 64) * 64, kRoom);
    const int smem = std::max(T.warps * room * (int)sizeof(uint2), T.warps * 512);
    auto kernel = T.team > 1 ? cut_kernel<true> : cut_kernel<false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return DMA_ERR_CUDA;
    return launch_overlapped(kernel, dim3((unsigned)(T.ctas + 1)), dim3(32 * T.warps), smem, st, 1, A, T.team, room, T.heads);
}

}  // namespace dma
