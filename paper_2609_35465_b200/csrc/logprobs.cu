// Log probabilities and ranks of given tokens, the entropy and the likeliest tokens of each row of logits (tetra_logprobs).
//
// A row is read once, by a CTA or, where rows are few, by a cluster of CTAs, each a part of it, tile by tile (E logits a thread, read
// 16 bytes at a time; other CTAs of the SM hide the loads):
//   * sums of 2^z and z 2^z, z = (x - m) log2(e) / T, next to a running maximum m that each thread has for itself; a tile's few terms
//     are summed on their own first, and threads' sums in float64;
//   * ranks, by comparing with the given tokens' logits, which are loaded before; a thread whose tile has nothing above one passes it over;
//   * the likeliest tokens: entries (logit, index) above a bound go to a list.  The first tile's bound is the k-th largest of its groups'
//     maxima, which no more than k groups reach.  Then come runs of tiles, each three times as long as all before it: a thread that has
//     something above the bound notes itself and its tile, and behind the run the CTA's warps look at what was noted, put the entries
//     on the list, cut it to its k best and have a new bound.  What was noted of a run may be too much (logits that rise along
//     the row): its tiles are then gone through again, each as the first.
// Entries are 64-bit numbers in the order that ranks them, so all of that is exact.
// The loop over a run's tiles keeps nothing but a tile and the sums in registers, calls nothing, and no warp waits for another in it: 12
// instructions of a thread for a logit, all phases together, which the memory outlasts.  (With the list kept there, the next tile in registers and a barrier a tile it
// were up to 27, and 1024 rows of 151936 took 146 to 226 us.)  1024 rows of 151936 float32 logits take 111 us, 5.6 TB/s, 86 % of a copy's rate; 64
// rows that L2 holds 17.8 us, of which the memory would need 6: a CTA of 1024 threads has 3.7 tiles, and the choice, the cut and the cluster's
// barriers; one row 10 us.  (1 to 4 % of that are for distances beyond float32, taken of parts.)
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <type_traits>

#include "../../include/tetra.h"
#include "../../include/tetra_logprobs.h"
#include "tetra_gemv_common.cuh"

namespace tetra {
namespace {

namespace cg = cooperative_groups;

constexpr int kLpTop = TETRA_LOGPROBS_MAX_TOP, kLpGiven = TETRA_LOGPROBS_MAX_GIVEN;
constexpr int kLpNear = 128;                       // entries of which each is compared with each at once
constexpr int kLpMostCtas = 8;
constexpr int kLpShortRow = 8192, kLpMiddleRow = 16384, kLpWideRow = 131072;  // logits
constexpr float kLpNoRef = -FLT_MAX, kLpLeast = -200.f;  // a weight of 2^-200 is zero

struct LpSums {
    double sum, product;  // of 2^z, of z 2^z
    float top;
};
template <int THREADS, int E>
struct LpShared {
    // Groups whose maxima bound a tile's candidates: of two threads, four of a large CTA, or eight where few entries are looked for (so
    // much less there is to compare: 4.1 us of 17.4 for 20 of 8 rows' entries by groups of two of 1024 threads; no more than kLpTop * kShare E entries
    // reach the bound either way).
    static constexpr int kShare = THREADS >= 1024 ? 4 : 2, kGroups = THREADS / 2, kFewTop = kLpTop * kShare / 8;
    static_assert(THREADS / kShare >= kLpTop && THREADS / 8 >= kFewTop && THREADS <= 1024, "as many groups as candidates");
    static constexpr int kList = kLpTop * kShare * E + kLpTop, kNotes = 1024;
    static constexpr int kNear = kLpTop * kShare * ((kList + THREADS - 1) / THREADS);  // entries of kLpTop groups
    uint64_t list[kList];
    uint64_t best[kLpTop];
    uint64_t near[kNear];
    int32_t note[kNotes];                          // the first element of a thread's tile that has candidates
    uint64_t group[kGroups];
    uint64_t gathered[kLpMostCtas * kLpTop];       // of the cluster's CTAs, at the first
    LpSums sums[kLpMostCtas], warp[THREADS / 32];
    uint64_t least;
    float given[kLpGiven], below[kLpGiven];        // logits of the given tokens, and the next number below
    int32_t token[kLpGiven], count[kLpGiven];
    uint32_t listed, nearby, noted;
};

__device__ __forceinline__ float lp_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t lp_two(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void lp_two(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
// n + 1 where x > y.
__device__ __forceinline__ void lp_count(int& n, float x, float y) {
    asm("{\n.reg .pred p;\nsetp.gt.ftz.f32 p, %1, %2;\n@p add.s32 %0, %0, 1;\n}" : "+r"(n) : "f"(x), "f"(y));
}
__device__ __forceinline__ float lp_clean(float x) { return __fadd_rn(fminf(fmaxf(x, -INFINITY), FLT_MAX), 0.f); }
// In the order of the floats; minus infinity is 0x007FFFFF.
__device__ __forceinline__ uint32_t lp_order(float x) {
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.f));
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float lp_value(uint64_t entry) {
    const uint32_t o = uint32_t(entry >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t lp_entry(float x, uint32_t index) { return uint64_t(lp_order(x)) << 32 | uint32_t(~index); }
__device__ __forceinline__ uint32_t lp_index(uint64_t entry) { return ~uint32_t(entry); }

// Where each of n entries (n > 0, none of them 0; all threads of the CTA come here) stands among them; the k first are put there.
template <int THREADS>
__device__ __forceinline__ void lp_rank(const uint64_t* from, int n, int k, uint64_t* to) {
    int share = 1;
    while (share < 32 && 2 * share * n <= THREADS) share *= 2;
    for (int e0 = 0; e0 < n; e0 += THREADS / share) {
        const int e = e0 + int(threadIdx.x) / share, part = threadIdx.x % share;
        const uint64_t mine = e < n ? from[e] : 0;
        int above = 0;
        for (int i = part; i < n; i += share) above += from[i] > mine;
        for (int o = share >> 1; o >= 1; o >>= 1) above += __shfl_xor_sync(0xFFFFFFFFu, above, o);
        if (mine != 0 && part == 0 && above < k) to[above] = mine;
    }
}

// The `top` first of LISTS lists of so many entries each, which are in order (0: none).  An entry's place is how many of each list are ahead of it.
template <int THREADS, int LISTS>
__device__ __forceinline__ void lp_merge(const uint64_t* from, int top, uint64_t* to) {
    for (int e = threadIdx.x; e < LISTS * top; e += THREADS) {
        const uint64_t mine = from[e];
        int ahead[LISTS] = {}, above = 0;
#pragma unroll
        for (int step = kLpTop; step >= 1; step >>= 1) {
#pragma unroll
            for (int l = 0; l < LISTS; ++l) {
                const int at = ahead[l] + step;
                if (at <= top && from[l * top + at - 1] > mine) ahead[l] = at;
            }
        }
#pragma unroll
        for (int l = 0; l < LISTS; ++l) above += ahead[l];
        if (mine != 0 && above < top) to[above] = mine;
    }
}

// A row, and the part of it that is a CTA's.
struct LpRow {
    const unsigned char* at;  // 16-byte aligned; the row begins `skip` elements on
    int skip, vocab, end;     // the part ends at this 16-byte load
};

template <bool HALF, int THREADS, int E>
struct Reader {
    using Shared = LpShared<THREADS, E>;
    static constexpr int V = HALF ? 8 : 4, LOADS = E / V, TILE = THREADS * LOADS;  // elements of a load; loads of a thread's tile, and of a tile

    // Element j of a thread's tile, the first of which is `first`.
    static __device__ __forceinline__ int place(int first, int j) { return first + j / V * (THREADS * V) + j % V; }
    static __device__ __forceinline__ bool inside(const LpRow& r, int tile, int j, int at) {
        return at >= 0 && at < r.vocab && tile + int(threadIdx.x) + j / V * THREADS < r.end;
    }
    static __device__ __forceinline__ float value(const LpRow& r, int index) {
        return HALF ? __half2float(reinterpret_cast<const __half*>(r.at)[r.skip + index]) : reinterpret_cast<const float*>(r.at)[r.skip + index];
    }
    static __device__ __forceinline__ bool whole(const LpRow& r, int tile) { return tile * V >= r.skip && tile + TILE <= r.end && (tile + TILE) * V - r.skip <= r.vocab; }
    template <bool WHOLE>
    static __device__ __forceinline__ void load(const LpRow& r, int tile, float (&x)[E]) {
        const uint4* from = reinterpret_cast<const uint4*>(r.at) + tile + threadIdx.x;
        const uint32_t least = HALF ? 0xFC00FC00u : 0xFF800000u;  // minus infinity
        uint4 v[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (WHOLE) {
                v[i] = __ldg(from + i * THREADS);
                continue;
            }
            const int vec = tile + int(threadIdx.x) + i * THREADS, first = vec * V - r.skip;
            v[i] = make_uint4(least, least, least, least);
            if (vec >= r.end) continue;
            if (first >= 0 && first + V <= r.vocab) {
                v[i] = __ldg(from + i * THREADS);
            } else {  // where the row begins or ends inside 16 bytes
                uint32_t w[4] = {least, least, least, least};
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (first + j < 0 || first + j >= r.vocab) continue;
                    if (HALF) {
                        const uint32_t h = __ldg(reinterpret_cast<const unsigned short*>(from + i * THREADS) + j);
                        w[j / 2 % 4] = j & 1 ? (w[j / 2 % 4] & 0xFFFFu) | h << 16 : (w[j / 2 % 4] & 0xFFFF0000u) | h;
                    } else {
                        w[j % 4] = __ldg(reinterpret_cast<const uint32_t*>(from + i * THREADS) + j);
                    }
                }
                v[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (HALF) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                    x[i * V + 2 * k] = f.x, x[i * V + 2 * k + 1] = f.y;
                } else {
                    x[i * V + k] = __uint_as_float(w[k]);
                }
            }
        }
    }
    static __device__ __forceinline__ void put(uint64_t entry, Shared* sm) {
        const uint32_t to = atomicAdd(&sm->listed, 1u);
        if (to < uint32_t(Shared::kList)) sm->list[to] = entry;
    }
    // A thread notes its tile.
    static __device__ __forceinline__ void note(const LpRow& r, int tile, Shared* sm) {
        const uint32_t to = atomicAdd(&sm->noted, 1u);
        if (to < uint32_t(Shared::kNotes)) sm->note[to] = (tile + int(threadIdx.x)) * V - r.skip;
    }
    // What was noted, to the list, where it is above the bound and `least` or more (the whole CTA, behind a barrier).
    static __device__ __forceinline__ void look(const LpRow& r, float bound, uint64_t least, Shared* sm) {
        constexpr int AT_ONCE = 4;  // notes a warp looks at side by side, a lane an element
        const int n = int(min(sm->noted, uint32_t(Shared::kNotes))), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        for (int i = warp * AT_ONCE; i < n; i += THREADS / 32 * AT_ONCE) {
            float x[AT_ONCE];
            int at[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                at[k] = -1;
                if (i + k < n && lane < E) at[k] = place(sm->note[i + k], lane);
                const int load = (at[k] + r.skip) / V;
                x[k] = at[k] >= 0 && at[k] < r.vocab && load < r.end ? value(r, at[k]) : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const uint64_t entry = lp_entry(fminf(x[k], FLT_MAX), uint32_t(at[k]));
                if (x[k] > bound && entry >= least) put(entry, sm);
            }
        }
    }
    // The `top`-th largest of groups' maxima, a thread's being `mine`; 0 where there are not so many.  (All of the CTA's threads come here.)
    static __device__ __forceinline__ uint64_t reached(uint64_t mine, int share, int top, Shared* sm) {
        const int groups = THREADS / share, part = threadIdx.x % share;
        for (int o = 1; o < share; o <<= 1) {
            const uint64_t other = __shfl_xor_sync(0xFFFFFFFFu, mine, o);
            mine = mine > other ? mine : other;
        }
        if (part == 0) sm->group[threadIdx.x / share] = mine;
        if (threadIdx.x == 0) sm->least = 0;
        __syncthreads();
        int above = 0;
#pragma unroll 8
        for (int i = part; i < groups; i += share) above += sm->group[i] > mine;
        for (int o = 1; o < share; o <<= 1) above += __shfl_xor_sync(0xFFFFFFFFu, above, o);
        if (above == top - 1 && mine != 0 && part == 0) sm->least = mine;
        __syncthreads();
        return sm->least;
    }
    // The list cut to its `top` best, in order, without entries from index `limit` on (all of the CTA's threads come here, behind a
    // barrier); returns the last one's logit, or minus infinity if there are not so many.
    static __device__ __noinline__ float cut(int top, uint32_t limit, Shared* sm) {
        int n = int(min(sm->listed, uint32_t(Shared::kList)));
        const uint64_t* from = sm->list;
        if (threadIdx.x < kLpTop) sm->best[threadIdx.x] = 0;
        if (threadIdx.x == 0) sm->nearby = sm->noted = 0;
        if (limit != ~0u)
            for (int i = threadIdx.x; i < n; i += THREADS)
                if (lp_index(sm->list[i]) >= limit) sm->list[i] = 0;
        __syncthreads();
        if (n > kLpNear) {
            uint64_t mine = 0;
            for (int i = threadIdx.x; i < n; i += THREADS) mine = sm->list[i] > mine ? sm->list[i] : mine;
            const uint64_t least = reached(mine, Shared::kShare, top, sm);
            for (int i = threadIdx.x; i < n; i += THREADS) {
                const uint64_t entry = sm->list[i];
                if (entry != 0 && entry >= least) sm->near[atomicAdd(&sm->nearby, 1u)] = entry;
            }
            __syncthreads();
            n = int(sm->nearby);
            from = sm->near;
        }
        if (n > 0) lp_rank<THREADS>(from, n, top, sm->best);
        __syncthreads();
        if (threadIdx.x < 32) {
            const bool is = int(threadIdx.x) < top && sm->best[threadIdx.x] != 0;
            if (is) sm->list[threadIdx.x] = sm->best[threadIdx.x];
            const uint32_t kept = __popc(__ballot_sync(0xFFFFFFFFu, is));
            if (threadIdx.x == 0) sm->listed = kept;
        }
        __syncthreads();
        return sm->best[top - 1] ? lp_value(sm->best[top - 1]) : -INFINITY;
    }
    // Which of a thread's tile is its first largest.
    static __device__ __noinline__ int first_most(LpRow r, int tile, float most) {
        int which = 0;
#pragma unroll 1
        for (int j = E - 1; j >= 0; --j) {
            const int at = place((tile + int(threadIdx.x)) * V - r.skip, j);
            if (inside(r, tile, j, at) && value(r, at) >= fminf(most, FLT_MAX)) which = j;
        }
        return which;
    }
    // A tile's candidates by its groups' maxima, of which `which` is the thread's (all of the CTA's threads come here); returns the bound for later tiles.
    static __device__ __forceinline__ float choose(LpRow r, int tile, float most, int which, float bound, int top, Shared* sm) {
        uint64_t mine = most > bound ? lp_entry(fminf(most, FLT_MAX), uint32_t(place((tile + int(threadIdx.x)) * V - r.skip, which))) : 0;
        const uint64_t least = reached(mine, top <= Shared::kFewTop ? 8 : Shared::kShare, top, sm);
        if (most > bound && (least == 0 || most >= lp_value(least))) note(r, tile, sm);
        __syncthreads();
        look(r, bound, least, sm);
        return least ? fmaxf(bound, lp_value(least)) : bound;  // entries that come later, with greater indexes, have to be above it
    }
    // Tiles [from, to) once more, each as if it were the first: the list, without what they left there, is cut behind each.
    static __device__ __noinline__ float again(LpRow r, int from, int to, int top, Shared* sm) {
        float bound = cut(top, uint32_t(max(from * V - r.skip, 0)), sm);
#pragma unroll 1
        for (int tile = from; tile < to; tile += TILE) {
            float most = -INFINITY;
#pragma unroll 1
            for (int j = 0; j < E; ++j) {
                const int at = place((tile + int(threadIdx.x)) * V - r.skip, j);
                if (inside(r, tile, j, at)) most = fmaxf(most, value(r, at));
            }
            choose(r, tile, most, first_most(r, tile, most), bound, top, sm);
            __syncthreads();
            if (threadIdx.x == 0) sm->noted = 0;
            bound = cut(top, ~0u, sm);
        }
        return bound;
    }
};

template <bool HALF, int THREADS, int E, int CTAS>
__device__ __forceinline__ void lp_run(const tetra_logprobs_rows& p, LpShared<THREADS, E>& sm) {
    using R = Reader<HALF, THREADS, E>;
    using Shared = LpShared<THREADS, E>;
    constexpr int V = R::V, WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    const int r = blockIdx.x / CTAS, rank = CTAS == 1 ? 0 : int(cg::this_cluster().block_rank()), top = max(p.top, 1);
    static_assert(THREADS >= kLpGiven, "a thread a counter");
    if (threadIdx.x < kLpGiven) sm.count[threadIdx.x] = 0;
    if (CTAS > 1) cg::this_cluster().barrier_arrive();  // the first CTA is written to when all have begun: what others add to is zero by then
    pdl_wait();
    pdl_release();
    const int size = HALF ? 2 : 4;
    const unsigned char* at = static_cast<const unsigned char*>(p.logits) + int64_t(r) * p.row_stride * size;
    const int skip = int(reinterpret_cast<uintptr_t>(at) & 15u) / size;
    // Loads [begin, end) are this CTA's.
    const int vecs = (p.vocab + skip + V - 1) / V, per = (vecs + CTAS - 1) / CTAS, begin = rank * per, end = min(vecs, begin + per);
    const LpRow row{at - skip * size, skip, p.vocab, end};

    const float T = p.temperature ? __ldg(p.temperature + r) : 1.f;
    const bool greedy = !(T > 0.f);
    // Distances between logits are taken of sixteenths where T is above 1: exact, and float32 holds the largest of them (two logits
    // may lie 2 FLT_MAX apart) and the factor that goes with the largest T.  Where T is not above 1 an infinite distance is no weight.
    const float part = T > 1.f ? 0.0625f : 1.f, c = greedy ? 1.f : fminf(__fdiv_rn(1.4426950408889634f / part, T), FLT_MAX);
    auto distance = [&](float x, float to) { return fmaxf(fmaf(x, part, -to * part) * c, kLpLeast); };  // log2 of a weight
    const double by_temperature = 1. / double(T);
    for (int g = THREADS - 1 - int(threadIdx.x); g < p.given; g += THREADS) {
        const int t = __ldg(p.tokens + int64_t(r) * p.given + g);
        const bool is = t >= 0 && t < p.vocab;
        const float x = lp_clean(is ? R::value(row, t) : 0.f);
        const uint32_t bits = __float_as_uint(x);
        sm.given[g] = x;
        sm.below[g] = x == 0.f ? -1.17549435e-38f : x > 0.f ? __uint_as_float(bits - 1) : __uint_as_float(bits + 1);  // (not used of minus infinity)
        sm.token[g] = is ? t : -1;
    }
    if (threadIdx.x == 0) sm.listed = sm.noted = 0;

    const int ranked = p.rank ? p.given : 0;
    int few = 0;  // of the first given token
    float ref = kLpNoRef, sum = 0.f, product = 0.f, bound = -INFINITY;
    int which = 0;
    // A tile's part in the sums and ranks; returns its largest logit.
    auto step = [&](auto all, int tile) {
        float x[E];
        R::template load<decltype(all)::value>(row, tile, x);
        float most = x[0];
#pragma unroll
        for (int j = 1; j < E; ++j) most = fmaxf(most, x[j]);
        if (most == INFINITY) {
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = x[j] == INFINITY ? FLT_MAX : x[j];
            most = FLT_MAX;
        }
        if (most > ref) {
            const float d = distance(ref, most), f = lp_ex2(d);
            product = f * fmaf(sum, d, product);
            sum *= f;
            ref = most;
        }
        {
            const uint64_t from = lp_two(-ref * part, -ref * part), by = lp_two(c, c), parts = lp_two(part, part);
            uint64_t s2 = 0, w2 = 0;
#pragma unroll
            for (int j = 0; j < E; j += 2) {
                uint64_t z, e;
                float a, b;
                asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(z) : "l"(lp_two(x[j], x[j + 1])), "l"(parts), "l"(from));
                asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(z), "l"(by));
                lp_two(z, a, b);
                a = fmaxf(a, kLpLeast), b = fmaxf(b, kLpLeast);  // infinite distances and NaN: the least
                z = lp_two(a, b);
                e = lp_two(lp_ex2(a), lp_ex2(b));
                asm("add.rn.f32x2 %0, %1, %2;" : "=l"(s2) : "l"(s2), "l"(e));
                asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(w2) : "l"(e), "l"(z), "l"(w2));
            }
            float a, b;
            lp_two(s2, a, b);
            sum += a + b;
            lp_two(w2, a, b);
            product += a + b;
        }
        const int tile_first = tile * V - skip, first = tile_first + int(threadIdx.x) * V;
        if (tile == begin) {
#pragma unroll
            for (int j = E - 1; j >= 0; --j) which = x[j] >= most ? j : which;
            __syncthreads();  // the given tokens
        }
        // Tokens ahead of a given one: before it those that are not below it, behind it those above it.
#pragma unroll 1
        for (int g = 0; g < ranked; ++g) {
            const float mine = sm.given[g], below = sm.below[g];
            const int token = sm.token[g];
            int n = 0;
            if (mine == -INFINITY) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const int at = R::place(first, j);
                    n += x[j] > mine || (at < token && R::inside(row, tile, j, at));
                }
            } else if (most > below) {  // of a likely token hardly ever
                if (tile_first <= token && token < tile_first + R::TILE * V) {
#pragma unroll
                    for (int j = 0; j < E; ++j) lp_count(n, x[j], R::place(first, j) < token ? below : mine);
                } else {
                    const float least = tile_first < token ? below : mine;
#pragma unroll
                    for (int j = 0; j < E; ++j) lp_count(n, x[j], least);
                }
            }
            if (g == 0) {
                few += n;
            } else {
                n = __reduce_add_sync(0xFFFFFFFFu, n);
                if (lane == 0 && n) atomicAdd(&sm.count[g], n);
            }
        }
        return most;
    };
    if (begin < end) {
        const float most = R::whole(row, begin) ? step(std::true_type(), begin) : step(std::false_type(), begin);
        bound = R::choose(row, begin, most, which, bound, top, &sm);
        __syncthreads();
        if (threadIdx.x == 0) sm.noted = 0;
        __syncthreads();
    }
    for (int from = begin + R::TILE; from < end;) {
        const int done = from - begin, to = min(end, from + 3 * done);
        int tile = from;
#pragma unroll 1
        for (; tile < to && R::whole(row, tile); tile += R::TILE) if (step(std::true_type(), tile) > bound) R::note(row, tile, &sm);
        if (tile < to && step(std::false_type(), tile) > bound) R::note(row, tile, &sm);  // the row's, or the part's, last
        __syncthreads();
        if (sm.noted > uint32_t(Shared::kNotes)) {
            __syncthreads();
            bound = R::again(row, from, to, top, &sm);
        } else {
            R::look(row, bound, 0, &sm);
            __syncthreads();
            if (sm.listed > uint32_t(Shared::kList)) {
                __syncthreads();
                bound = R::again(row, from, to, top, &sm);
            } else if (to < end) {
                bound = fmaxf(bound, R::cut(top, ~0u, &sm));
            }
        }
        from = to;
    }
    if (begin >= end) __syncthreads();  // the given tokens
    if (ranked) {
        const int n = __reduce_add_sync(0xFFFFFFFFu, few);
        if (lane == 0 && n) atomicAdd(&sm.count[0], n);
    }
    // The CTA's sums, next to its largest logit, and its best entries.
    auto largest = [&](float x) { return lp_value(uint64_t(__reduce_max_sync(0xFFFFFFFFu, lp_order(x))) << 32); };
    auto add_lanes = [&](double& a, double& b) {
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
            a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
            b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
        }
    };
    LpSums s;
    s.top = largest(ref);
    {
        const float d = distance(ref, s.top), f = lp_ex2(d);
        s.sum = double(sum * f);
        s.product = double(f * fmaf(sum, d, product));
        add_lanes(s.sum, s.product);
    }
    if (lane == 0) sm.warp[warp] = s;
    __syncthreads();
    R::cut(top, ~0u, &sm);
    // Sums of n warps, or CTAs, lane by lane.
    auto join = [&](const LpSums* of, int n) {
        s = lane < n ? of[lane] : LpSums{0., 0., kLpNoRef};
        const float all = largest(s.top), d = distance(s.top, all), f = lp_ex2(d);
        s.product = f * (s.product + s.sum * d);
        s.sum *= f;
        s.top = all;
        add_lanes(s.sum, s.product);
    };
    if (warp == 0) join(sm.warp, WARPS);
    if (CTAS > 1) {
        cg::this_cluster().barrier_wait();
        Shared* to = cg::this_cluster().map_shared_rank(&sm, 0);
        if (warp == 0) {
            if (lane == 0) to->sums[rank] = s;
            if (lane < top) to->gathered[rank * top + lane] = sm.best[lane];
            for (int g = lane; g < ranked; g += 32)
                if (rank > 0 && sm.count[g]) atomicAdd(&to->count[g], sm.count[g]);
        }
        cg::this_cluster().sync();
        if (rank > 0) return;
        if (threadIdx.x < kLpTop) sm.best[threadIdx.x] = 0;
        __syncthreads();
        lp_merge<THREADS, CTAS>(sm.gathered, top, sm.best);
        __syncthreads();
    }
    if (warp > 0) return;
    if (CTAS > 1) join(sm.sums, CTAS);
    const double norm = log(s.sum);
    const uint64_t head = sm.best[0];
    auto logprob = [&](float x, bool likeliest) {
        if (x == -INFINITY || (greedy && !likeliest)) return -INFINITY;
        return greedy ? 0.f : float((double(x) - double(s.top)) * by_temperature - norm);
    };
    if (lane < p.top) {
        const uint64_t entry = sm.best[lane];
        p.top_tokens[int64_t(r) * p.top + lane] = entry ? int32_t(lp_index(entry)) : -1;
        p.top_logprob[int64_t(r) * p.top + lane] = entry ? logprob(lp_value(entry), lane == 0) : -INFINITY;
    }
    for (int g = lane; g < p.given; g += 32) {
        const int t = sm.token[g];
        p.logprob[int64_t(r) * p.given + g] = t >= 0 ? logprob(sm.given[g], head != 0 && uint32_t(t) == lp_index(head)) : -INFINITY;
        if (p.rank) p.rank[int64_t(r) * p.given + g] = t >= 0 ? sm.count[g] : -1;
    }
    if (lane == 0 && p.entropy) p.entropy[r] = greedy || head == 0 ? 0.f : fmaxf(float(norm - 0.693147180559945309417 * (s.product / s.sum)), 0.f);
}

template <bool HALF, int THREADS, int E, int CTAS>
__cluster_dims__(CTAS, 1, 1) __global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprobs(tetra_logprobs_rows p) {
    __shared__ LpShared<THREADS, E> sm;
    lp_run<HALF, THREADS, E, CTAS>(p, sm);
}

// A row's CTAs where each has 1024 threads and an SM of its own.
template <bool HALF, int CTAS>
struct Wide {
    static constexpr int E = HALF ? 24 : 20;
    static cudaError_t launch(const tetra_logprobs_rows& p, cudaStream_t s) { return launch_pdl(k_logprobs<HALF, 1024, E, CTAS>, p.rows * CTAS, 1024, 0, s, p); }
    // Rows whose clusters run at once (a cluster is within a GPC, which leaves some SMs over).
    static cudaError_t rows_at_once(int& rows) {
        static PerDeviceOnce once;
        static int fit[PerDeviceOnce::kMaxDevices];
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        e = once.run([device] {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(CTAS);
            cfg.blockDim = dim3(1024);
            return cudaOccupancyMaxActiveClusters(&fit[device], k_logprobs<HALF, 1024, E, CTAS>, &cfg);
        });
        if (e == cudaSuccess) rows = fit[device];
        return e;
    }
};

// CTAs of 1024 threads: clusters of eight for as many long rows as run at once, then two or one a row that fill the SMs; else of 256, as
// many as fill them four times.  Measured, us with 1024 and 256 threads (1 and 20 likeliest tokens): 151936 logits, 8 rows 10.3 and 11.3 (12.2,
// 12.8), 15 10.9 and 11.5, 16 (in two waves) 18.2 and 12.2, 24 by fours 13.5 and 12.8, 64 17.9 and 19.4 (21.1, 22.8), 74 18.2 and 25.6, 100 25.8 and 23.7 (30.0,
// 30.5), 148 27.3 and 36.3; 100003 logits, 8 rows 10.1 and 9.8 (12.0, 10.9), 64 16.0 and 16.5; 20011 logits, 36 rows 9.7 and 10.6 (11.5, 13.3), 148 10.2 and 15.4.
template <bool HALF>
cudaError_t launch_logprobs(const tetra_logprobs_rows& p, int sms, cudaStream_t s) {
    if (p.vocab <= kLpShortRow) return launch_pdl(k_logprobs<HALF, 128, 16, 1>, p.rows, 128, 0, s, p);
    if (p.vocab > kLpWideRow && p.rows * 8 <= sms) {
        int rows = 0;
        const cudaError_t e = Wide<HALF, 8>::rows_at_once(rows);
        if (e != cudaSuccess) return e;
        if (p.rows <= rows) return Wide<HALF, 8>::launch(p, s);
    }
    if (p.vocab > kLpMiddleRow && p.rows * 4 >= sms && p.rows <= sms) return p.rows * 2 <= sms ? Wide<HALF, 2>::launch(p, s) : Wide<HALF, 1>::launch(p, s);
    const int at_once = 4 * sms + sms / 2;  // CTAs of 256 threads, and some that come behind them
    return p.rows * 8 <= at_once ? launch_pdl(k_logprobs<HALF, 256, 32, 8>, p.rows * 8, 256, 0, s, p)
         : p.rows * 4 <= at_once ? launch_pdl(k_logprobs<HALF, 256, 32, 4>, p.rows * 4, 256, 0, s, p)
         : p.rows * 2 <= at_once ? launch_pdl(k_logprobs<HALF, 256, 32, 2>, p.rows * 2, 256, 0, s, p)
                                 : launch_pdl(k_logprobs<HALF, 256, 32, 1>, p.rows, 256, 0, s, p);
}

bool lp_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" int tetra_logprobs(const tetra_logprobs_rows* rows, void* stream) {
    if (!rows) return TETRA_ERR_NULL;
    const tetra_logprobs_rows& p = *rows;
    if (p.rows < 0 || p.rows > TETRA_LOGPROBS_MAX_ROWS || p.vocab < 1 || p.vocab > TETRA_LOGPROBS_MAX_VOCAB || p.row_stride < p.vocab || p.half_type < 0 || p.half_type > 1 ||
        p.given < 0 || p.given > TETRA_LOGPROBS_MAX_GIVEN || p.top < 0 || p.top > TETRA_LOGPROBS_MAX_TOP)
        return TETRA_ERR_SHAPE;
    if (!p.logits || (p.given > 0 && (!p.tokens || !p.logprob)) || (p.top > 0 && (!p.top_tokens || !p.top_logprob))) return TETRA_ERR_NULL;
    if (!lp_aligned(p.logits, p.half_type ? 2 : 4)) return TETRA_ERR_ALIGN;
    for (const void* at : {static_cast<const void*>(p.temperature), static_cast<const void*>(p.tokens), static_cast<const void*>(p.logprob), static_cast<const void*>(p.rank),
                           static_cast<const void*>(p.entropy), static_cast<const void*>(p.top_tokens), static_cast<const void*>(p.top_logprob)})
        if (!lp_aligned(at, 4)) return TETRA_ERR_ALIGN;
    if (p.rows == 0) return TETRA_OK;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) return TETRA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return (p.half_type ? launch_logprobs<true>(p, sms, s) : launch_logprobs<false>(p, sms, s)) == cudaSuccess ? TETRA_OK : TETRA_ERR_CUDA;
}
