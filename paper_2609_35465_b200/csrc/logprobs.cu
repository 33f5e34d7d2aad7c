// Log probabilities and ranks of given tokens, the entropy and the likeliest tokens of each row of logits (tetra_logprobs).
//
// A row is read once, by a CTA or, where rows are few, by a cluster of CTAs, each a part of it, tile by tile; the next tile is on its way
// while one is worked on.  Everything comes out of that pass:
//   * sums of 2^z and z 2^z, z = (x - m) log2(e) / T, next to a running maximum m that each thread has for itself; a tile's few terms
//     are summed on their own first, and threads' sums in float64;
//   * ranks, by comparing with the given tokens' logits, which are loaded before;
//   * the likeliest tokens: entries (logit, index) above a bound go to a list.  The first tile's bound is the k-th largest of 256 groups'
//     maxima, which no more than k groups reach; later ones pass the k-th best entry so far, which few do.  The list is cut to its k best
//     when it has grown; a tile with more entries than the list takes (logits that rise along the row) is treated as the first.
// Entries are 64-bit numbers in the order that ranks them, so all of that is exact.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <cfloat>

#include "../../include/tetra.h"
#include "../../include/tetra_logprobs.h"
#include "tetra_gemv_common.cuh"

namespace tetra {
namespace {

namespace cg = cooperative_groups;

constexpr int kLpLong = 512, kLpShort = 128;       // threads of a CTA
constexpr int kLpEach = 16;                        // elements of a thread's tile
constexpr int kLpTop = TETRA_LOGPROBS_MAX_TOP, kLpGiven = TETRA_LOGPROBS_MAX_GIVEN;
constexpr int kLpSoft = 192;                       // entries after which the list is cut
constexpr int kLpMostCtas = 8;
constexpr int kLpShortRow = 8192;                  // logits
constexpr float kLpNoRef = -FLT_MAX, kLpLeast = -200.f;  // a weight of 2^-200 is zero

struct LpSums {
    double sum, product;  // of 2^z, of z 2^z
    float top;
};
template <int THREADS>
struct LpShared {
    static constexpr int kGroups = THREADS / 2;    // whose maxima bound a tile's candidates: two threads each
    static_assert(kGroups >= kLpTop, "as many groups as candidates");
    // the tile's candidates: those of kLpTop groups at most, and what was there
    static constexpr int kList = kLpTop * 2 * kLpEach + kLpSoft + kLpTop;
    uint64_t list[kList];
    uint64_t best[kLpTop];                         // the list's, while it is cut
    uint64_t group[kGroups];
    uint64_t gathered[kLpMostCtas * kLpTop];       // of the cluster's CTAs, at the first
    LpSums sums[kLpMostCtas], warp[THREADS / 32];
    uint64_t bound;
    float given[kLpGiven], below[kLpGiven];        // logits of the given tokens, and the next number below
    int32_t token[kLpGiven], count[kLpGiven];
    uint32_t listed, kept;
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

// How many of n entries (n > 0, all threads of the CTA come here) are above each, for entry e the threads e P .. e P + P - 1; each of the
// k first is put where it belongs.  Entries of 0 are none.
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

template <bool HALF, int THREADS, int CTAS>
struct Scorer {
    using Shared = LpShared<THREADS>;
    static constexpr int V = HALF ? 8 : 4, E = kLpEach, LOADS = E / V, TILE = THREADS * LOADS;  // elements of a load, of a thread's tile; loads of a tile

    const unsigned char* row;  // 16-byte aligned; the row begins `skip` elements on
    int skip, vocab;
    Shared& sm;
    int top;                   // entries that are looked for, one at least

    __device__ __forceinline__ uint4 load(int vec, int end) const {
        const int first = vec * V - skip;
        if (vec >= end) return none();
        if (first >= 0 && first + V <= vocab) return __ldg(reinterpret_cast<const uint4*>(row) + vec);
        uint4 v = none();
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
        if (HALF) {
            const unsigned short* p = reinterpret_cast<const unsigned short*>(row);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (first + i >= 0 && first + i < vocab) w[i / 2] = i & 1 ? (w[i / 2] & 0xFFFFu) | uint32_t(__ldg(p + vec * V + i)) << 16 : (w[i / 2] & 0xFFFF0000u) | __ldg(p + vec * V + i);
        } else {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(row);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (first + i >= 0 && first + i < vocab) w[i % 4] = __ldg(p + vec * V + i);
        }
        return v;
    }
    static __device__ __forceinline__ uint4 none() { return HALF ? make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u) : make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
    static __device__ __forceinline__ void values(const uint4& v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (HALF) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[2 * i] = f.x, x[2 * i + 1] = f.y;
            } else {
                x[i] = __uint_as_float(w[i]);
            }
        }
    }

    // Of a thread's tile, how many are ahead of given token g.
    __device__ __forceinline__ int ahead(const float (&x)[E], int first, int g) const {
        const float mine = sm.given[g], below = sm.below[g];
        const int token = sm.token[g];
        int n = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = first + i * (THREADS * V);
            if (mine == -INFINITY || (at <= token && token < at + V)) {
#pragma unroll
                for (int j = 0; j < V; ++j) n += x[i * V + j] > mine || (at + j >= 0 && at + j < token && (x[i * V + j] == mine || mine == -INFINITY));
            } else {
                const float least = at < token ? below : mine;
#pragma unroll
                for (int j = 0; j < V; ++j) n += x[i * V + j] > least;
            }
        }
        return n;
    }

    // The list cut to its best, without entries from index `limit` on.
    __device__ __forceinline__ void cut(uint32_t limit, float& bound) {
        const int n = int(min(sm.listed, uint32_t(Shared::kList)));
        for (int i = threadIdx.x; i < kLpTop; i += THREADS) sm.best[i] = 0;
        if (limit != ~0u)
            for (int i = threadIdx.x; i < n; i += THREADS)
                if (lp_index(sm.list[i]) >= limit) sm.list[i] = 0;
        __syncthreads();
        if (n > 0) lp_rank<THREADS>(sm.list, n, top, sm.best);
        __syncthreads();
        if (threadIdx.x < 32) {
            const bool is = int(threadIdx.x) < top && sm.best[threadIdx.x] != 0;
            sm.list[threadIdx.x] = is ? sm.best[threadIdx.x] : 0;
            const uint32_t kept = __popc(__ballot_sync(0xFFFFFFFFu, is));
            if (threadIdx.x == 0) sm.listed = sm.kept = kept;
        }
        __syncthreads();
        bound = int(sm.kept) == top ? lp_value(sm.list[top - 1]) : -INFINITY;
    }
    // A tile's candidates by its groups' maxima.
    __device__ __forceinline__ void choose(const float (&x)[E], int first, float most, float& bound) {
        uint64_t mine = 0;
        if (most > bound) {
#pragma unroll
            for (int j = E - 1; j >= 0; --j)
                if (x[j] == most) mine = lp_entry(x[j], uint32_t(first + j / V * (THREADS * V) + j % V));
        }
        const uint64_t other = __shfl_xor_sync(0xFFFFFFFFu, mine, 1);
        if ((threadIdx.x & 1) == 0) sm.group[threadIdx.x >> 1] = mine > other ? mine : other;
        if (threadIdx.x == 0) sm.bound = 0;
        __syncthreads();
        {
            const int g = threadIdx.x >> 1;
            const uint64_t key = sm.group[g];
            int above = 0;
#pragma unroll 8
            for (int i = threadIdx.x & 1; i < Shared::kGroups; i += 2) above += sm.group[i] > key;
            above += __shfl_xor_sync(0xFFFFFFFFu, above, 1);
            if (above == top - 1 && key != 0 && (threadIdx.x & 1) == 0) sm.bound = key;
        }
        __syncthreads();
        const uint64_t least = sm.bound;
        if (most > bound && (least == 0 || most >= lp_value(least))) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (!(x[j] > bound)) continue;
                const uint64_t entry = lp_entry(x[j], uint32_t(first + j / V * (THREADS * V) + j % V));
                if (entry >= least) sm.list[atomicAdd(&sm.listed, 1u)] = entry;
            }
        }
        if (least != 0) bound = fmaxf(bound, lp_value(least));  // entries that come later, with greater indexes, have to be above it
    }
};

template <bool HALF, int THREADS, int CTAS>
__device__ __forceinline__ void lp_run(const tetra_logprobs_rows& p, LpShared<THREADS>& sm) {
    using S = Scorer<HALF, THREADS, CTAS>;
    constexpr int V = S::V, E = S::E, LOADS = S::LOADS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = blockIdx.x / CTAS, rank = CTAS == 1 ? 0 : int(cg::this_cluster().block_rank());
    if (CTAS > 1) cg::this_cluster().barrier_arrive();  // the first CTA is written to when all have begun
    pdl_wait();
    pdl_release();
    const int size = HALF ? 2 : 4;
    const unsigned char* at = static_cast<const unsigned char*>(p.logits) + int64_t(r) * p.row_stride * size;
    const int skip = int(reinterpret_cast<uintptr_t>(at) & 15u) / size;
    S sc{at - skip * size, skip, p.vocab, sm, max(p.top, 1)};
    // Loads [begin, end) are this CTA's.
    const int vecs = (p.vocab + skip + V - 1) / V, per = (vecs + CTAS - 1) / CTAS, begin = rank * per, end = min(vecs, begin + per);
    uint4 next[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) next[i] = sc.load(begin + i * THREADS + threadIdx.x, end);

    const float T = p.temperature ? __ldg(p.temperature + r) : 1.f;
    const bool greedy = !(T > 0.f);
    const float c = greedy ? 1.f : fminf(__fdiv_rn(1.4426950408889634f, T), FLT_MAX);
    for (int g = threadIdx.x; g < p.given; g += THREADS) {
        const int t = __ldg(p.tokens + int64_t(r) * p.given + g);
        const bool is = t >= 0 && t < p.vocab;
        float x = 0.f;
        if (is) x = HALF ? __half2float(static_cast<const __half*>(p.logits)[int64_t(r) * p.row_stride + t]) : static_cast<const float*>(p.logits)[int64_t(r) * p.row_stride + t];
        x = lp_clean(x);
        sm.given[g] = x;
        const uint32_t bits = __float_as_uint(x);
        sm.below[g] = x == 0.f ? -1.17549435e-38f : x > 0.f ? __uint_as_float(bits - 1) : __uint_as_float(bits + 1);  // (not used of minus infinity)
        sm.token[g] = is ? t : -1;
        sm.count[g] = 0;
    }
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();

    constexpr int kFew = 4;  // given tokens whose counts a thread keeps
    int few[kFew] = {0, 0, 0, 0};
    const int ranked = p.rank ? p.given : 0;
    float ref = kLpNoRef, sum = 0.f, product = 0.f, bound = -INFINITY;
    bool fresh = true;
    for (int tile = begin; tile < end; tile += S::TILE) {
        float x[E];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) S::values(next[i], x + i * V);
        if (tile + S::TILE < end) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) next[i] = sc.load(tile + S::TILE + i * THREADS + threadIdx.x, end);
        }
        const int first = (tile + int(threadIdx.x)) * V - skip;  // element j: first + j / V * (THREADS * V) + j % V
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < E; ++j) most = fmaxf(most, x[j]);
        if (most == INFINITY) {
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = x[j] == INFINITY ? FLT_MAX : x[j];
            most = FLT_MAX;
        }
        if (most > ref) {
            const float d = fmaxf((ref - most) * c, kLpLeast), f = lp_ex2(d);
            product = f * fmaf(sum, d, product);
            sum *= f;
            ref = most;
        }
        float part, part_product;
        {
            const uint64_t from = lp_two(-ref, -ref), by = lp_two(c, c);
            uint64_t s2 = 0, w2 = 0;
#pragma unroll
            for (int j = 0; j < E; j += 2) {
                uint64_t z, e;
                float a, b;
                asm("add.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(lp_two(x[j], x[j + 1])), "l"(from));
                asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(z), "l"(by));
                lp_two(z, a, b);
                e = lp_two(lp_ex2(a), lp_ex2(b));
                asm("add.rn.f32x2 %0, %1, %2;" : "=l"(s2) : "l"(s2), "l"(e));
                asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(w2) : "l"(e), "l"(z), "l"(w2));
            }
            float a, b;
            lp_two(s2, a, b);
            part = a + b;
            lp_two(w2, a, b);
            part_product = a + b;
            if (!(part_product == part_product)) {  // infinite distances, or NaN, among them
                part = part_product = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const float z = fmaxf((x[j] - ref) * c, kLpLeast), e = lp_ex2(z);  // NaN: the least
                    part += e;
                    part_product = fmaf(e, z, part_product);
                }
            }
        }
        sum += part;
        product += part_product;
        // Tokens ahead of a given one: before it those that are not below it, behind it those above it.
#pragma unroll
        for (int g = 0; g < kFew; ++g)
            if (g < ranked) few[g] += sc.ahead(x, first, g);
        for (int g = kFew; g < ranked; ++g) {
            const int ahead = __reduce_add_sync(0xFFFFFFFFu, sc.ahead(x, first, g));
            if (lane == 0 && ahead) atomicAdd(&sm.count[g], ahead);
        }
        if (fresh) {
            sc.choose(x, first, most, bound);
            fresh = false;
            if (__syncthreads_or(sm.listed >= kLpSoft)) sc.cut(~0u, bound);  // read behind a barrier by those that add last: one of them sees it
        } else {
            uint32_t last = 0;
            if (most > bound) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (!(x[j] > bound)) continue;
                    last = atomicAdd(&sm.listed, 1u);
                    if (last < uint32_t(LpShared<THREADS>::kList)) sm.list[last] = lp_entry(x[j], uint32_t(first + j / V * (THREADS * V) + j % V));
                }
            }
            if (__syncthreads_or(last >= kLpSoft)) {
                const bool lost = sm.listed > uint32_t(LpShared<THREADS>::kList);
                const int tile_first = tile * V - skip;
                __syncthreads();
                sc.cut(lost ? uint32_t(max(tile_first, 0)) : ~0u, bound);
                if (lost) {
                    sc.choose(x, first, most, bound);
                    __syncthreads();
                    sc.cut(~0u, bound);
                }
            }
        }
    }
    __syncthreads();
    if (sm.listed > 0 && end > begin) sc.cut(~0u, bound);

#pragma unroll
    for (int g = 0; g < kFew; ++g) {
        if (g >= ranked) break;
        const int ahead = __reduce_add_sync(0xFFFFFFFFu, few[g]);
        if (lane == 0 && ahead) atomicAdd(&sm.count[g], ahead);
    }
    // The CTA's sums.
    {
        LpSums s{double(sum), double(product), ref};
        auto join = [&](LpSums& a, const LpSums& b) {
            const float now = fmaxf(a.top, b.top);
            const float da = fmaxf((a.top - now) * c, kLpLeast), db = fmaxf((b.top - now) * c, kLpLeast), fa = lp_ex2(da), fb = lp_ex2(db);
            a.product = fa * (a.product + a.sum * da) + fb * (b.product + b.sum * db);
            a.sum = fa * a.sum + fb * b.sum;
            a.top = now;
        };
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
            LpSums b{__shfl_xor_sync(0xFFFFFFFFu, s.sum, o), __shfl_xor_sync(0xFFFFFFFFu, s.product, o), __shfl_xor_sync(0xFFFFFFFFu, s.top, o)};
            join(s, b);
        }
        if (lane == 0) sm.warp[warp] = s;
        __syncthreads();
        if (warp == 0) {
            s = sm.warp[lane % (THREADS / 32)];
#pragma unroll
            for (int o = (THREADS / 32) / 2; o >= 1; o >>= 1) {
                LpSums b{__shfl_xor_sync(0xFFFFFFFFu, s.sum, o), __shfl_xor_sync(0xFFFFFFFFu, s.product, o), __shfl_xor_sync(0xFFFFFFFFu, s.top, o)};
                join(s, b);
            }
            if (CTAS > 1) {
                cg::this_cluster().barrier_wait();
                LpShared<THREADS>* to = cg::this_cluster().map_shared_rank(&sm, 0);
                if (lane == 0) to->sums[rank] = s;
                if (lane < sc.top) to->gathered[rank * sc.top + lane] = lane < int(sm.listed) ? sm.list[lane] : 0;
                for (int g = lane; g < ranked; g += 32)
                    if (rank > 0 && sm.count[g]) atomicAdd(&to->count[g], sm.count[g]);
            } else if (lane == 0) {
                sm.sums[0] = s;
            }
        } else if (CTAS > 1) {
            cg::this_cluster().barrier_wait();
        }
        if (CTAS > 1) {
            cg::this_cluster().sync();
            if (rank > 0) return;
        } else {
            __syncthreads();
        }
        s = sm.sums[0];
        for (int i = 1; i < CTAS; ++i) join(s, sm.sums[i]);
        if (CTAS > 1) {
            for (int i = threadIdx.x; i < kLpTop; i += THREADS) sm.best[i] = 0;
            __syncthreads();
            lp_rank<THREADS>(sm.gathered, CTAS * sc.top, sc.top, sm.best);
            __syncthreads();
        }
        const uint64_t* best = CTAS > 1 ? sm.best : sm.list;
        const int found = CTAS > 1 ? sc.top : int(sm.listed);
        const double norm = log(s.sum);
        auto logprob = [&](float x, bool likeliest) {
            if (x == -INFINITY || (greedy && !likeliest)) return -INFINITY;
            return greedy ? 0.f : float((double(x) - double(s.top)) / double(T) - norm);
        };
        const uint64_t head = found > 0 ? best[0] : 0;
        for (int i = threadIdx.x; i < p.top; i += THREADS) {
            const uint64_t entry = i < found ? best[i] : 0;
            p.top_tokens[int64_t(r) * p.top + i] = entry ? int32_t(lp_index(entry)) : -1;
            p.top_logprob[int64_t(r) * p.top + i] = entry ? logprob(lp_value(entry), i == 0) : -INFINITY;
        }
        for (int g = threadIdx.x; g < p.given; g += THREADS) {
            const int t = sm.token[g];
            p.logprob[int64_t(r) * p.given + g] = t >= 0 ? logprob(sm.given[g], head != 0 && uint32_t(t) == lp_index(head)) : -INFINITY;
            if (p.rank) p.rank[int64_t(r) * p.given + g] = t >= 0 ? sm.count[g] : -1;
        }
        if (threadIdx.x == 0 && p.entropy) p.entropy[r] = greedy || head == 0 ? 0.f : float(norm - 0.693147180559945309417 * (s.product / s.sum));
    }
}

template <bool HALF, int THREADS, int CTAS>
__cluster_dims__(CTAS, 1, 1) __global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprobs(tetra_logprobs_rows p) {
    __shared__ LpShared<THREADS> sm;
    lp_run<HALF, THREADS, CTAS>(p, sm);
}

template <bool HALF>
cudaError_t launch_logprobs(const tetra_logprobs_rows& p, int sms, cudaStream_t s) {
    const int many = p.rows * 8;
    if (p.vocab <= kLpShortRow) return launch_pdl(k_logprobs<HALF, kLpShort, 1>, p.rows, kLpShort, 0, s, p);
    return many <= sms ? launch_pdl(k_logprobs<HALF, kLpLong, 8>, p.rows * 8, kLpLong, 0, s, p)
         : many <= 2 * sms ? launch_pdl(k_logprobs<HALF, kLpLong, 4>, p.rows * 4, kLpLong, 0, s, p)
         : many <= 8 * sms ? launch_pdl(k_logprobs<HALF, kLpLong, 2>, p.rows * 2, kLpLong, 0, s, p)
                           : launch_pdl(k_logprobs<HALF, kLpLong, 1>, p.rows, kLpLong, 0, s, p);
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
