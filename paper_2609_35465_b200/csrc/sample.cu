// The next token of each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers (tetra_sample).
//
// A cluster of four to eight CTAs takes a row, or one CTA a short one.  Each CTA reads its part of it once into shared memory; everything after
// that happens there and in the cluster's distributed shared memory.
//   * Weights are fixed-point numbers (units of 2^-44 of the largest), so sums are exact in whatever order, and what
//     is found by a histogram here, by counting there and by a scan at the end agrees to the last bit.
//   * The three filters all keep a prefix of the order (logit down, index up), so they come to one cut: the last entry
//     (logit, index) that stays.  A histogram over the distance from the largest logit, of counts for top-k and of masses
//     for top-p alone, finds the bin that the cut is in.  Where the bins up to it hold no more than 2048 entries, these
//     go to the first CTA, which does all the rest.  Otherwise the entries of that bin go there, a second histogram among
//     them finds the cut, and the cluster draws.  A bin with too many entries (equal logits, outliers) is cut by bisection
//     over the entries instead: any input is right, the usual ones are fast.
//   * The draw goes through the kept weights in the order of the indexes.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <cfloat>

#include "../../include/tetra.h"
#include "../../include/tetra_sample.h"
#include "tetra_gemv_common.cuh"

namespace tetra {
namespace {

namespace cg = cooperative_groups;

constexpr int kSmpMostCtas = 8, kSmpMaxWarps = 32;
constexpr int kSmpBins = 1024;
constexpr int kSmpCounted = kSmpBins / 4;                       // bins of masses whose entries are counted too: few are so near
constexpr int kSmpList = 2048;                                  // entries that one CTA takes
constexpr int kSmpFew = 256;                                    // ... and compares each with each
constexpr int kSmpNear = 128;                                   // ... and does so at once to find a cut: 256 such take as long as a histogram
constexpr int kSmpAlone = 8192, kSmpAloneMany = 32768;           // logits that one CTA takes; of more rows than clusters run at once
constexpr int kSmpBits = 44;                                    // a weight of 1 is 2^44

static_assert(TETRA_SAMPLE_MAX_VOCAB <= 1 << 19, "sums of weights stay below 2^63");

struct Tally {  // so many entries with so much mass
    uint64_t mass;
    uint64_t count;
};

struct alignas(16) SmpShared {
    uint64_t list[kSmpList];
    uint64_t weight[kSmpFew];
    uint32_t ahead_of[kSmpFew];
    double powers[64];                    // 2^(44 + j / 64)
    uint32_t count[kSmpBins], lo[kSmpBins], hi[kSmpBins];  // of the bins: entries, mass in two words
    Tally slots[2][kSmpMostCtas];           // what the CTAs tell each other
    Tally warp[kSmpMaxWarps], whole;
    uint64_t bin, ahead, need, entries;   // a crossing: its bin, the sum before it, what is needed, entries up to its end
    uint64_t cut;
    uint32_t listed, sub, few, least_key;
};

// Logits are compared as integers in the order of the floats; NaN is minus infinity, plus infinity the largest float32, zeros
// (and what is below 2^-126) are equal.
__device__ __forceinline__ float clean(float x) { return __fadd_rn(fminf(fmaxf(x, -INFINITY), FLT_MAX), 0.f); }
__device__ __forceinline__ float distance_up(float a, float b) { return __fsub_ru(a, b); }
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// Weight of a logit in units of 2^-44: 2^t, t = (x - max) log2(e) / T = k / 64 + f / 64 with |f| <= 1/2, as 2^(k / 64) from a table
// times a polynomial of the fourth degree for e^(f ln 2 / 64), rounded once; in float64, whose multiply-adds run at half the rate
// of float32's here.  The exponential series cut behind the fourth power is off by up to 3.9e-14, 0.68 units of 2^-44, which with the
// rounding is more than a unit; so its fifth power is not left out but economised (Lanczos): f^5 is 5/16 f^3 - 5/256 f but for
// T_5(2 f) / 512, a sixteenth of its largest.  That takes no operation more, and a weight is off by 0.55 units at most (0.544 over 30 million arguments).
// Adding 1.5 * 2^52 leaves a whole number in the low bits.
struct Weigh {
    double top, by;         // largest logit; 64 log2(e) / T
    float reach;            // distance from the largest to which there is mass: e^-31.25 is less than half a unit
    const double* powers;
    __device__ __forceinline__ bool has(float x) const { return float(top) - x <= reach; }
    __device__ __forceinline__ uint64_t any(float x) const { return has(x) ? (*this)(x) : 0; }
    // ... of one that has mass.
    __device__ __forceinline__ uint64_t operator()(float x) const {
        constexpr double magic = 6755399441055744.;
        const double d = double(x) - top, m = fma(d, by, magic), f = fma(d, by, magic - m);
        const int k = __double2loint(m);
        constexpr double c = 0.693147180559945309417 / 64., fifth = c * c * c * c * c / 120.;
        double e = fma(c * c * c * c / 24., f, c * c * c / 6. + fifth * 5. / 16.);
        e = fma(e, f, c * c / 2.);
        e = fma(e, f, c - fifth * 5. / 256.);
        e = fma(e, f, 1.);
        const double power = powers[k & 63];
        const double w = e * __hiloint2double(__double2hiint(power) + (k >> 6) * (1 << 20), __double2loint(power)) + 4503599627370496.;  // 2^52
        return uint64_t(__double_as_longlong(w)) & 0xFFFFFFFFFFFFFull;
    }
};

__device__ __forceinline__ Tally operator+(const Tally& a, const Tally& b) { return {a.mass + b.mass, a.count + b.count}; }

// Sum over the warp's lanes up to this one.
__device__ __forceinline__ Tally warp_scan(Tally v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Tally u{__shfl_up_sync(0xFFFFFFFFu, v.mass, o), __shfl_up_sync(0xFFFFFFFFu, v.count, o)};
        if (lane >= o) v = v + u;
    }
    return v;
}
struct Settings {
    uint64_t k;       // entries that stay
    float p;          // 1 and above: off
    uint64_t floor_w; // least weight
    float u;
};

// What a CTA of so many threads does.
template <int kSmpThreads, int kSmpCtas>
struct Sampler {

static constexpr int kSmpWarps = kSmpThreads / 32;
static constexpr int kSmpRegion = kSmpList / kSmpCtas;  // entries of a CTA, in equal shares

// The cluster, which may be a CTA alone.
static __device__ __forceinline__ void sync() {
    if (kSmpCtas == 1) __syncthreads();
    else cg::this_cluster().sync();
}
// Nothing may be written to a CTA that has not begun: each tells so at its first instruction, and before the first such
// write waits for the others' word, which is long there by then.
static __device__ __forceinline__ void begun() {
    if (kSmpCtas > 1) cg::this_cluster().barrier_arrive();
}
static __device__ __forceinline__ void all_begun() {
    if (kSmpCtas > 1) cg::this_cluster().barrier_wait();
}
template <typename P>
static __device__ __forceinline__ P* of(P* mine, int rank) { return kSmpCtas == 1 ? mine : cg::this_cluster().map_shared_rank(mine, rank); }

// ... over the CTA's threads up to this one; `total` is the CTA's.  The warps' sums are added by one warp: each thread adding them
// for itself takes more cycles than all the rest.
static __device__ __forceinline__ Tally block_scan(SmpShared& sm, Tally v, Tally& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_scan(v, lane);
    if (lane == 31) sm.warp[warp] = v;
    __syncthreads();
    if (warp == 0) {
        const Tally own = lane < kSmpWarps ? sm.warp[lane] : Tally{0, 0}, upto = warp_scan(own, lane);
        if (lane < kSmpWarps) sm.warp[lane] = {upto.mass - own.mass, upto.count - own.count};
        if (lane == 31) sm.whole = upto;
    }
    __syncthreads();
    total = sm.whole;
    const Tally before = sm.warp[warp];
    __syncthreads();
    return before + v;
}

// Largest mass and least count of N lanes next to each other.
template <int N>
static __device__ __forceinline__ Tally extremes(Tally v) {
#pragma unroll
    for (int o = N / 2; o >= 1; o >>= 1) {
        v.mass = max(v.mass, __shfl_xor_sync(0xFFFFFFFFu, v.mass, o));
        v.count = min(v.count, __shfl_xor_sync(0xFFFFFFFFu, v.count, o));
    }
    return v;
}

// Sorts list[0 .. size), a power of two, the largest first.
static __device__ __forceinline__ void sort_list(uint64_t* list, uint32_t size) {
#pragma unroll 1
    for (uint32_t k = 2; k <= size; k <<= 1)
#pragma unroll 1
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            for (uint32_t i = threadIdx.x; i < size / 2; i += kSmpThreads) {
                const uint32_t a = (i & ~(j - 1)) << 1 | (i & (j - 1)), b = a | j;
                const uint64_t u = list[a], v = list[b];
                if ((u < v) == !(a & k)) list[a] = v, list[b] = u;
            }
            __syncthreads();
        }
}
static __device__ __forceinline__ uint32_t power_of_two(uint32_t n) {
    uint32_t size = 2;
    while (size < n) size <<= 1;
    return size;
}

// How far from the largest logit there is mass.
static __device__ __forceinline__ float reach_of(float T) { return fminf(31.25f * T, FLT_MAX); }

// Distance bins: logit -> bin, the largest in bin 0; kSmpBins for one without mass.
struct Bins {
    float top, range, by;
    // Rounded up, so that neither `least` nor top - range leaves the least logit out.
    __device__ __forceinline__ Bins(float top_, float least, float T) : top(top_), range(fminf(distance_up(top_, least), reach_of(T))) {
        by = range > 1e-30f ? float(kSmpBins) / range : 0.f;
    }
    __device__ __forceinline__ bool has(float x) const { return top - x <= range; }
    __device__ __forceinline__ uint32_t operator()(float x) const { return min(uint32_t((top - x) * by), uint32_t(kSmpBins - 1)); }  // of one that has mass
    __device__ __forceinline__ uint32_t any(float x) const { return has(x) ? (*this)(x) : uint32_t(kSmpBins); }
};

struct Row {
    SmpShared& sm;
    const float* x;   // this CTA's part, minus infinity up to a multiple of four
    int count;
    uint32_t index;   // of its first token
    int rank, turn;

    // Every CTA's value for every CTA, in the order of their ranks.  The first warp's lanes bring the CTA's.
    __device__ __forceinline__ const Tally* tell(Tally mine) {
        Tally* slots = sm.slots[turn & 1];
        ++turn;
        if (threadIdx.x < kSmpCtas) of(slots, threadIdx.x)[rank] = mine;
        sync();
        return slots;
    }
    __device__ __forceinline__ uint64_t entry(int i, float v) const { return uint64_t(key_of(v)) << 32 | uint32_t(~(index + uint32_t(i))); }
    // body(i, x_i) for all of the part's tokens, four of a thread at a time (what is behind the part is minus infinity).
    template <typename F>
    __device__ __forceinline__ void each(F&& body) const {
#pragma unroll 2
        for (int i = 4 * threadIdx.x; i < count; i += 4 * kSmpThreads) {
            const float4 v = *reinterpret_cast<const float4*>(x + i);
            body(i, v.x);
            body(i + 1, v.y);
            body(i + 2, v.z);
            body(i + 3, v.w);
        }
    }
};

// A mass to a bin's: 64 bits in two words, the carry by hand.
static __device__ __forceinline__ void add_mass(uint32_t* lo, uint32_t* hi, uint64_t w) {
    const uint32_t low = uint32_t(w), old = atomicAdd(lo, low), high = uint32_t(w >> 32) + (old + low < old);
    if (high) atomicAdd(hi, high);
}

static __device__ __forceinline__ uint64_t needed(float p, uint64_t mass) {
    const uint64_t need = uint64_t(ceil(double(p) * double(mass)));
    return need < 1 ? 1 : need > mass ? mass : need;
}
static __device__ __forceinline__ uint64_t aimed(float u, uint64_t mass) {
    const uint64_t aim = uint64_t(fmin(fmax(double(u), 0.), 1.) * double(mass));  // NaN: 0
    return aim >= mass ? mass - 1 : aim;
}

// The bin in which this CTA's counts reach k; kSmpBins where they do not.
static __device__ __forceinline__ uint32_t local_bin(SmpShared& sm, uint64_t k) {
    constexpr int PER = kSmpBins / kSmpThreads;
    if (threadIdx.x == 0) sm.sub = kSmpBins, sm.least_key = 0xFFFFFFFFu;
    __syncthreads();
    uint64_t sum = 0;
    uint32_t own[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += own[i] = sm.count[threadIdx.x * PER + i];
    Tally total;
    uint64_t upto = block_scan(sm, {sum, 0}, total).mass - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (upto < k && k <= upto + own[i]) sm.sub = threadIdx.x * PER + i;
        upto += own[i];
    }
    __syncthreads();
    return sm.sub;
}

// The cluster's histogram in the first CTA, which finds the bin in which the sums (entries, or mass) reach k entries, or p of the
// whole mass, and tells all.  Every CTA's histogram is complete but for a barrier.
template <bool MASS>
static __device__ __forceinline__ void find_bin(Row& row, uint64_t k, float p) {
    SmpShared& sm = row.sm;
    __syncthreads();
    if (row.rank != 0) {
        SmpShared* first = of(&sm, 0);
#pragma unroll
        for (int i = 0; i < kSmpBins / kSmpThreads; ++i) {
            const int b = threadIdx.x + i * kSmpThreads;
            if (!MASS || b < kSmpCounted) {
                if (sm.count[b]) atomicAdd(first->count + b, sm.count[b]);
            }
            if (MASS && (sm.lo[b] | sm.hi[b])) add_mass(first->lo + b, first->hi + b, (uint64_t(sm.hi[b]) << 32) + sm.lo[b]);
        }
    }
    sync();
    if (row.rank == 0) {
        constexpr int PER = kSmpBins / kSmpThreads;
        Tally own[PER], sum{0, 0}, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = threadIdx.x * PER + i;
            own[i] = {MASS ? (uint64_t(sm.hi[b]) << 32) + sm.lo[b] : 0ull, sm.count[b]};
            sum = sum + own[i];
        }
        Tally upto = block_scan(sm, sum, total);
        upto = {upto.mass - sum.mass, upto.count - sum.count};
        // With fewer entries than k all stay: the last bin, and no cut.
        const uint64_t need = MASS ? needed(p, total.mass) : k, whole = total.count;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Tally from = upto;
            upto = upto + own[i];
            const uint64_t a = MASS ? from.mass : from.count, b = MASS ? upto.mass : upto.count;
            const bool all = !MASS && need >= whole && threadIdx.x == kSmpThreads - 1 && i == PER - 1;
            if (all || ((MASS || need < whole) && a < need && need <= b))
                for (int r = 0; r < kSmpCtas; ++r) {
                    SmpShared* other = of(&sm, r);
                    other->bin = all ? kSmpBins : uint64_t(threadIdx.x * PER + i);
                    other->ahead = a;
                    other->need = need;
                    other->entries = upto.count;
                }
        }
    }
    sync();
}

// Entries of the bins [low, high] that are not below `cut`: how many there are in the cluster, and all of them in the list of
// the first CTA where they are kSmpList at most.  Collected at home first: a counter in another CTA takes a thousand cycles.
static __device__ __forceinline__ uint32_t gather(Row& row, const Bins& bins, uint32_t low, uint32_t high, uint64_t cut) {
    SmpShared& sm = row.sm;
    row.each([&](int i, float v) {
        const uint32_t bin = bins.any(v);
        if (bin >= low && bin <= high && row.entry(i, v) >= cut) {
            const uint32_t at = atomicAdd(&sm.listed, 1u);
            if (at < kSmpList) sm.list[at] = row.entry(i, v);
        }
    });
    __syncthreads();
    const uint32_t mine = sm.listed;
    const Tally* all = row.tell({0, mine});
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int c = 0; c < kSmpCtas; ++c) {
        if (c == row.rank) before = total;
        total += uint32_t(all[c].count);
    }
    if (threadIdx.x == 0) sm.listed = 0;
    if (total <= kSmpList) {
        if (row.rank != 0) {
            uint64_t* list = of(sm.list, 0) + before;
            for (uint32_t i = threadIdx.x; i < mine; i += kSmpThreads) list[i] = sm.list[i];
        }
        sync();
    }
    return total;
}

// Among sm.list[0 .. n), n >= 1, the entry with which `need` is reached from `ahead` on: into *cut.  scale (distance * bins.by - bin)
// is where an entry lies in a histogram of their own.  One CTA.
template <bool MASS>
static __device__ __noinline__ void cut_list(SmpShared& sm, const Bins bins, const Weigh weigh, uint32_t n, float bin, float scale, uint64_t ahead, uint64_t need, uint64_t* cut) {
    constexpr int PER = kSmpBins / kSmpThreads;
    auto weight = [&](uint64_t entry) { return MASS ? weigh.any(value_of(uint32_t(entry >> 32))) : 1ull; };
    if (n > kSmpNear) {  // a histogram of their own
        for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.count[i] = sm.lo[i] = sm.hi[i] = 0;
        if (threadIdx.x == 0) sm.few = 0;
        __syncthreads();
        auto inside = [&](uint64_t entry) {
            const float f = ((bins.top - value_of(uint32_t(entry >> 32))) * bins.by - bin) * scale;
            return uint32_t(fminf(fmaxf(f, 0.f), float(kSmpBins - 1)));
        };
        for (uint32_t i = threadIdx.x; i < n; i += kSmpThreads) {
            const uint32_t b = inside(sm.list[i]);
            atomicAdd(sm.count + b, 1u);
            if (MASS) add_mass(sm.lo + b, sm.hi + b, weight(sm.list[i]));
        }
        __syncthreads();
        uint64_t own[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = threadIdx.x * PER + i;
            own[i] = MASS ? (uint64_t(sm.hi[b]) << 32) + sm.lo[b] : sm.count[b];
            sum += own[i];
        }
        Tally total;
        uint64_t upto = ahead + block_scan(sm, {sum, 0}, total).mass - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (upto < need && need <= upto + own[i]) sm.sub = threadIdx.x * PER + i, sm.need = need - upto;
            upto += own[i];
        }
        __syncthreads();
        if (sm.count[sm.sub] <= kSmpFew) {  // its entries, to be counted
            uint64_t keep[kSmpList / kSmpThreads];
#pragma unroll
            for (int i = 0; i < kSmpList / kSmpThreads; ++i) {
                const uint32_t at = threadIdx.x + i * kSmpThreads;
                keep[i] = at < n && inside(sm.list[at]) == sm.sub ? sm.list[at] : 0;
            }
            n = sm.count[sm.sub];
            need = sm.need;
            ahead = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kSmpList / kSmpThreads; ++i)
                if (keep[i]) sm.list[atomicAdd(&sm.few, 1u)] = keep[i];
            __syncthreads();
        }
    }
    if (n <= kSmpFew) {  // an entry counts what is ahead of it
        const uint64_t entry = threadIdx.x < n ? sm.list[threadIdx.x] : 0, own = entry ? weight(entry) : 0;
        if (threadIdx.x < n) sm.weight[threadIdx.x] = own;
        __syncthreads();
        if (entry) {
            uint64_t from = ahead;
            for (uint32_t j = 0; j < n; ++j) from += sm.list[j] > entry ? sm.weight[j] : 0;
            if (from < need && need <= from + own) *cut = entry;
        }
    } else {  // many equal logits
        const uint32_t size = power_of_two(n);
        for (uint32_t i = n + threadIdx.x; i < size; i += kSmpThreads) sm.list[i] = 0;
        __syncthreads();
        sort_list(sm.list, size);
        constexpr int EACH = kSmpList / kSmpThreads;
        uint64_t own[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint32_t at = threadIdx.x * EACH + i;
            own[i] = at < n ? weight(sm.list[at]) : 0ull;
            sum += own[i];
        }
        Tally total;
        uint64_t upto = ahead + block_scan(sm, {sum, 0}, total).mass - sum;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (upto < need && need <= upto + own[i]) *cut = sm.list[threadIdx.x * EACH + i];
            upto += own[i];
        }
    }
    __syncthreads();
}

// The entry in bin sm.bin with which sm.need (entries, or mass, counted from the largest logit, of the entries not below `least`)
// is reached.
template <bool MASS>
static __device__ __forceinline__ uint64_t find_cut(Row& row, const Bins& bins, const Weigh& weigh, uint64_t least) {
    SmpShared& sm = row.sm;
    const uint32_t bin = uint32_t(sm.bin);
    const uint64_t ahead = sm.ahead, need = sm.need;
    const uint32_t entries = gather(row, bins, bin, bin, least);
    if (entries <= kSmpList) {
        if (row.rank == 0) {
            cut_list<MASS>(sm, bins, weigh, entries, float(bin), float(kSmpBins), ahead, need, &sm.cut);
            if (threadIdx.x < kSmpCtas) *of(&sm.cut, threadIdx.x) = sm.cut;
        }
        sync();
        // What is read here is written again behind a barrier of the cluster that follows.
        return sm.cut;
    }
    // The largest c with enough in the entries >= c: one bit after another.
    uint64_t c = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t mid = c | 1ull << bit;
        Tally v{0, 0}, total;
        row.each([&](int i, float x) {
            const uint64_t entry = row.entry(i, x);
            if (entry >= mid && entry >= least && bins.any(x) == bin) v.mass += MASS ? weigh(x) : 1ull;
        });
        block_scan(sm, v, total);
        const Tally* all = row.tell(total);
        uint64_t sum = ahead;
        for (int r = 0; r < kSmpCtas; ++r) sum += all[r].mass;
        if (sum >= need) c = mid;
    }
    return c;
}

// All of the filters and the draw among sm.list[0 .. n), which holds the first n entries in the order, 1 <= n <= kSmpFew: one CTA.
// `need`: the mass that top-p wants where that is known, or 0: then the list holds all that top-k leaves.  An entry counts
// what is ahead of it in the order, then what stays of smaller index.
static __device__ __forceinline__ void finish(SmpShared& sm, const Weigh& weigh, uint32_t n, const Settings& set, uint64_t need, int32_t* token, float* prob) {
    constexpr int SIDE = kSmpThreads / kSmpFew;  // threads of an entry
    const uint32_t i = threadIdx.x % kSmpFew, side = threadIdx.x / kSmpFew;
    uint64_t entry = i < n ? sm.list[i] : 0;
    if (threadIdx.x < kSmpFew) sm.ahead_of[threadIdx.x] = 0;
    __syncthreads();
    if (entry) {
        uint32_t ahead = 0;
#pragma unroll 4
        for (uint32_t j = side; j < n; j += SIDE) ahead += sm.list[j] > entry;
        if (ahead) atomicAdd(&sm.ahead_of[i], ahead);
    }
    __syncthreads();
    if (side == 0 && entry) sm.list[kSmpFew + sm.ahead_of[i]] = entry;  // in the order
    if (set.k < n) n = uint32_t(set.k);
    __syncthreads();
    const uint64_t* order = sm.list + kSmpFew;
    entry = threadIdx.x < n ? order[threadIdx.x] : 0;
    const uint64_t own = entry ? weigh.any(value_of(uint32_t(entry >> 32))) : 0;
    if (threadIdx.x < n) sm.weight[threadIdx.x] = own;
    Tally total;
    const uint64_t from = block_scan(sm, {own, 0}, total).mass - own;
    if (need == 0) need = set.p < 1.f ? needed(set.p, total.mass) : ~0ull;
    const bool stays = own && from < need && own >= set.floor_w;
    n = __syncthreads_count(stays);  // the first so many
    if (stays) {
        uint64_t base = 0, mass = 0;
#pragma unroll 4
        for (uint32_t j = 0; j < n; ++j) {
            const uint64_t w = sm.weight[j];
            mass += w;
            base += uint32_t(order[j]) > uint32_t(entry) ? w : 0;
        }
        const uint64_t aim = aimed(set.u, mass);
        if (base <= aim && aim < base + own) {
            *token = int(~uint32_t(entry));
            if (prob) *prob = float(double(own) / double(mass));
        }
    }
}

// The same from the CTAs' parts, top-k being on: all[c].count has how many entries lie at sm.list + c * kSmpRegion, and above that
// the key below which the CTA has k entries at least (so have all: the largest of these keys is a bound for all); all[c].mass
// is the CTA's largest.
static __device__ __forceinline__ void finish_parts(SmpShared& sm, const Tally* all, double by, float T, const Settings& set, int32_t* token, float* prob) {
    constexpr int ALL = kSmpCtas * kSmpRegion, PER = (ALL + kSmpThreads - 1) / kSmpThreads;
    const int lane = threadIdx.x & 31;
    uint64_t best = 0, entry[PER];
    uint32_t bound = 0;
#pragma unroll
    for (int c = 0; c < kSmpCtas; ++c) best = max(best, all[c].mass), bound = max(bound, uint32_t(all[c].count >> 32));
    const float top = value_of(uint32_t(best >> 32));
    const Weigh weigh{double(top), by, reach_of(T), sm.powers};
    if (top == -INFINITY) {
        if (threadIdx.x == 0) {
            *token = -1;
            if (prob) *prob = 0.f;
        }
        return;
    }
    uint32_t own = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t at = threadIdx.x + i * kSmpThreads;
        entry[i] = at < ALL && at % kSmpRegion < uint32_t(all[at / kSmpRegion].count) ? sm.list[at] : 0;
        if (entry[i] >> 32 < bound) entry[i] = 0;
        own += entry[i] != 0;
    }
    if (threadIdx.x == 0) sm.few = 0;
    __syncthreads();
    uint32_t place = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, place, o);
        if (lane >= o) place += v;
    }
    const uint32_t before = place - own;
    if (lane == 31) place = atomicAdd(&sm.few, place);
    place = __shfl_sync(0xFFFFFFFFu, place, 31) + before;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (entry[i]) sm.list[place++] = entry[i];
    __syncthreads();
    uint32_t n = sm.few;
    __syncthreads();
    if (n > kSmpFew) {
        cut_list<false>(sm, Bins(top, -INFINITY, T), weigh, n, 0.f, 1.f, 0, set.k, &sm.cut);
        const uint64_t cut = sm.cut;
        if (threadIdx.x == 0) sm.few = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (entry[i] >= cut) sm.list[atomicAdd(&sm.few, 1u)] = entry[i];
        __syncthreads();
        n = uint32_t(set.k);
    }
    finish(sm, weigh, n, set, 0, token, prob);
}

template <typename T>
static __device__ __forceinline__ void run(const tetra_sample_rows& p, int part) {
    extern __shared__ __align__(16) unsigned char smem[];
    SmpShared& sm = *reinterpret_cast<SmpShared*>(smem);
    float* held = reinterpret_cast<float*>(smem + sizeof(SmpShared));
    static_assert(sizeof(SmpShared) % 16 == 0, "the part lies behind it");
    const int r = blockIdx.x / kSmpCtas, rank = blockIdx.x % kSmpCtas, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int begin = min(part * rank, p.vocab), count = min(part, p.vocab - begin);
    Row row{sm, held, count, uint32_t(begin), rank, 0};
    begun();
    if (threadIdx.x == 0) sm.listed = 0;
    if (threadIdx.x < 64) sm.powers[threadIdx.x] = exp2(kSmpBits + threadIdx.x / 64.);
    for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.count[i] = sm.lo[i] = sm.hi[i] = 0;
    if (threadIdx.x < 3 && count + threadIdx.x < ((count + 3) & ~3)) held[count + threadIdx.x] = -INFINITY;
    pdl_wait();
    pdl_release();

    int32_t* token = p.tokens + r;
    float* prob = p.prob ? p.prob + r : nullptr;
    const float T_row = p.temperature ? p.temperature[r] : 1.f, p_row = p.top_p ? p.top_p[r] : 1.f, m_row = p.min_p ? p.min_p[r] : 0.f;
    const int k_row = p.top_k ? p.top_k[r] : 0;

    // The part; its largest entry, its least logit above minus infinity.
    const T* x = static_cast<const T*>(p.logits) + r * p.row_stride + begin;
    float most = -INFINITY, least = INFINITY;
    int most_at = 0;
    auto take = [&](int i, float v) {
        if (v > most) most = v, most_at = i;  // a thread's tokens come in order: the first of equal ones
        if (v > -INFINITY) least = fminf(least, v);
    };
    constexpr int VEC = 16 / sizeof(T);
    if ((reinterpret_cast<uintptr_t>(x) & 15) == 0) {
        constexpr int AHEAD = 5;
        const int n = count / VEC;
        for (int i = threadIdx.x; i < n; i += AHEAD * kSmpThreads) {
            uint4 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * kSmpThreads < n) v[k] = __ldg(reinterpret_cast<const uint4*>(x) + i + k * kSmpThreads);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int at = (i + k * kSmpThreads) * VEC;
                if (at < n * VEC) {
                    const T* e = reinterpret_cast<const T*>(&v[k]);
                    float f[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        f[j] = clean(float(e[j]));
                        take(at + j, f[j]);
                    }
#pragma unroll
                    for (int j = 0; j < VEC; j += 4) *reinterpret_cast<float4*>(held + at + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                }
            }
        }
        for (int i = n * VEC + threadIdx.x; i < count; i += kSmpThreads) {
            const float v = clean(float(x[i]));
            held[i] = v;
            take(i, v);
        }
    } else {
        constexpr int AHEAD = 8;
        for (int i = threadIdx.x; i < count; i += AHEAD * kSmpThreads) {
            T v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * kSmpThreads < count) v[k] = x[i + k * kSmpThreads];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * kSmpThreads < count) {
                    const float f = clean(float(v[k]));
                    held[i + k * kSmpThreads] = f;
                    take(i + k * kSmpThreads, f);
                }
        }
    }
    const uint32_t most_key = __reduce_max_sync(0xFFFFFFFFu, key_of(most));
    const uint32_t at = __reduce_min_sync(0xFFFFFFFFu, key_of(most) == most_key ? uint32_t(begin + most_at) : 0x7FFFFFFFu);
    const uint32_t least_key = __reduce_min_sync(0xFFFFFFFFu, key_of(least));
    if (lane == 0) sm.warp[warp] = {uint64_t(most_key) << 32 | uint32_t(~at), least_key};
    __syncthreads();
    Tally first{0, 0xFFFFFFFFu};
    if (warp == 0) {
        if (lane < kSmpWarps) first = sm.warp[lane];
        first = extremes<32>(first);
    }
    all_begun();
    const Settings set{k_row > 0 ? uint64_t(k_row) : ~0ull, p_row, m_row > 0.f ? uint64_t(ceil(double(m_row) * double(1ull << kSmpBits))) : 0ull, p.u[r]};
    const double by = 64. * 1.4426950408889634074 / double(T_row);
    const bool one = p_row <= 0.f || m_row > 1.f || k_row == 1;  // the first alone stays

    // Few of many: each CTA sends what may be among its own first k to the first CTA, and that is all they tell each other.  The
    // bin that holds the k-th of its threads' largest logits is not before that of the k-th of its part, and hardly behind it.
    if (T_row > 0.f && !one && k_row > 0 && k_row <= kSmpFew / 2) {
        if (threadIdx.x == 0) sm.whole = first;
        __syncthreads();
        const uint64_t own_best = sm.whole.mass;
        const float own_top = value_of(uint32_t(own_best >> 32));
        const Bins bins(own_top, value_of(uint32_t(sm.whole.count)), T_row);
        const uint32_t bin = most > -INFINITY ? bins.any(most) : uint32_t(kSmpBins);
        if (bin < kSmpBins) atomicAdd(sm.count + bin, 1u);
        const uint32_t last = local_bin(sm, set.k);
        if (bin <= last && bin < kSmpBins) atomicMin(&sm.least_key, key_of(most));
        __syncthreads();
        // Below k threads' largest there is nothing to find; where there are not so many, all that have mass are sent.
        const float least_sent = sm.sub < kSmpBins ? value_of(sm.least_key) : fmaxf(own_top - bins.range, -FLT_MAX);
        uint64_t* list = of(sm.list, 0) + rank * kSmpRegion;
        row.each([&](int i, float v) {
            if (v >= least_sent) {
                const uint32_t at = atomicAdd(&sm.listed, 1u);
                if (at < kSmpRegion) list[at] = row.entry(i, v);
            }
        });
        __syncthreads();
        const Tally* all = row.tell({own_best, uint64_t(sm.sub < kSmpBins ? sm.least_key : 0u) << 32 | sm.listed});
        const bool fits = __all_sync(0xFFFFFFFFu, uint32_t(all[lane % kSmpCtas].count) <= kSmpRegion);
        if (fits) {
            // A quarter of the threads is enough, and fewer warps meet sooner at a barrier.
            if (rank == 0 && threadIdx.x < kSmpFew) Sampler<kSmpFew, kSmpCtas>::finish_parts(sm, all, by, T_row, set, token, prob);
            return;
        }
        for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.count[i] = 0;
        if (threadIdx.x == 0) sm.listed = 0;
    }
    const Tally* all = row.tell(first);
    first = extremes<kSmpMostCtas>(all[min(lane % kSmpMostCtas, kSmpCtas - 1)]);
    const uint64_t best = first.mass;
    const uint32_t low = uint32_t(first.count);
    const float top = value_of(uint32_t(best >> 32));

    const bool none = top == -INFINITY;
    if (none || !(T_row > 0.f) || one) {
        if (rank == 0 && threadIdx.x == 0) {
            *token = none ? -1 : int(~uint32_t(best));
            if (prob) *prob = none ? 0.f : 1.f;
        }
        return;
    }
    const Weigh weigh{double(top), by, reach_of(T_row), sm.powers};
    const bool nucleus = p_row < 1.f, top_k = k_row > 0 && k_row < p.vocab;

    uint64_t cut = 0;
    if (top_k || nucleus) {
        const Bins bins(top, value_of(low), T_row);
        auto add = [&](float v) {
            if (bins.has(v)) {
                const uint32_t bin = bins(v);
                if (bin < kSmpCounted) atomicAdd(sm.count + bin, 1u);
                add_mass(sm.lo + bin, sm.hi + bin, weigh(v));
            }
        };
        if (top_k) {
            row.each([&](int, float v) {
                if (bins.has(v)) atomicAdd(sm.count + bins(v), 1u);
            });
            find_bin<false>(row, set.k, 1.f);
        } else {
            row.each([&](int, float v) { add(v); });
            find_bin<true>(row, 0, p_row);
        }
        if (sm.entries <= kSmpFew && (top_k || sm.bin < kSmpCounted)) {
            const uint32_t n = gather(row, bins, 0, min(uint32_t(sm.bin), uint32_t(kSmpBins - 1)), 0);
            if (rank == 0 && threadIdx.x < kSmpFew) Sampler<kSmpFew, kSmpCtas>::finish(sm, weigh, n, set, top_k ? 0 : sm.need, token, prob);
            return;
        }
        if (top_k) {
            if (sm.bin < kSmpBins) cut = find_cut<false>(row, bins, weigh, 0);
            if (nucleus) {  // again, of masses and of what is left
                for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.count[i] = sm.lo[i] = sm.hi[i] = 0;
                sync();
                row.each([&](int i, float v) {
                    if (row.entry(i, v) >= cut) add(v);
                });
                find_bin<true>(row, 0, p_row);
            }
        }
        if (nucleus) cut = find_cut<true>(row, bins, weigh, cut);
    }

    // The draw, in the order of the indexes: a warp takes so many consecutive fours.
    const int fours = (count + 3) / 4, each = (fours + kSmpWarps - 1) / kSmpWarps, from = min(each * warp, fours), to = min(from + each, fours);
    const float cut_at = cut ? value_of(uint32_t(cut >> 32)) : -INFINITY;
    const uint32_t cut_index = ~uint32_t(cut);  // of the logits that equal the cut's, those up to here stay
    auto stays = [&](int i, float v) { return v > cut_at || (v == cut_at && row.index + uint32_t(i) <= cut_index); };
    auto kept = [&](float v) -> uint64_t {
        const uint64_t w = weigh.any(v);
        return w >= set.floor_w ? w : 0;
    };
    uint64_t sum = 0;
    if (cut) {  // few stay: they are put next to each other before they are weighed
        float* queue = reinterpret_cast<float*>(sm.list) + warp * 64;
        static_assert(kSmpWarps * 64 * sizeof(float) <= sizeof(sm.list), "a queue for each warp");
        int queued = 0;
        for (int i = from; i < to; i += 32) {
            const int four = 4 * (i + lane);
            const float4 v = i + lane < to ? *reinterpret_cast<const float4*>(held + four) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool in = stays(four + k, f[k]);
                const uint32_t who = __ballot_sync(0xFFFFFFFFu, in);
                if (in) queue[queued + __popc(who & ((1u << lane) - 1))] = f[k];
                queued += __popc(who);
                if (queued >= 32) {
                    __syncwarp();
                    const uint64_t w = weigh(queue[lane]);
                    sum += w >= set.floor_w ? w : 0;
                    const float rest = queue[32 + lane];
                    queued -= 32;
                    __syncwarp();
                    if (lane < queued) queue[lane] = rest;  // the places from there on are the next ones', filled without a barrier in between
                }
            }
        }
        __syncwarp();
        const uint64_t w = lane < queued ? weigh(queue[lane]) : 0;
        sum += w >= set.floor_w ? w : 0;
    } else {
#pragma unroll 2
        for (int i = from + lane; i < to; i += 32) {
            const float4 v = *reinterpret_cast<const float4*>(held + 4 * i);
            sum += (kept(v.x) + kept(v.y)) + (kept(v.z) + kept(v.w));
        }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    Tally total;
    uint64_t base = block_scan(sm, {lane == 31 ? sum : 0, 0}, total).mass, mass = 0;
    base = __shfl_sync(0xFFFFFFFFu, base, 31) - sum;  // of the warps before
    all = row.tell(total);
#pragma unroll
    for (int c = 0; c < kSmpCtas; ++c) {
        if (c == rank) base += mass;
        mass += all[c].mass;
    }
    const uint64_t aim = aimed(set.u, mass);
    if (base <= aim && aim < base + sum) {  // this warp's
        for (int i = from; i < to; i += 32) {
            uint64_t w[4] = {0, 0, 0, 0};
            const int four = 4 * (i + lane);
            if (i + lane < to) {
                const float4 v = *reinterpret_cast<const float4*>(held + four);
                const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = stays(four + k, f[k]) ? kept(f[k]) : 0;
            }
            const uint64_t own = w[0] + w[1] + w[2] + w[3];
            if (!__any_sync(0xFFFFFFFFu, own != 0)) continue;
            uint64_t end = base + warp_scan({own, 0}, lane).mass, at = end - own;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (at <= aim && aim < at + w[k]) {
                    *token = int(row.index) + four + k;
                    if (prob) *prob = float(double(w[k]) / double(mass));
                }
                at += w[k];
            }
            base = __shfl_sync(0xFFFFFFFFu, end, 31);
            if (base > aim) break;
        }
    }
}

};  // Sampler

template <typename T, int THREADS, int CTAS>
__cluster_dims__(CTAS, 1, 1) __global__ void __launch_bounds__(THREADS) k_sample(tetra_sample_rows p, int part) {
    Sampler<THREADS, CTAS>::template run<T>(p, part);
}

using SampleKernel = void (*)(tetra_sample_rows, int);
// ctas: of a row.  wide: a CTA has its SM for itself; otherwise two of 512 threads share its registers, 64 a thread either way (the
// narrow ones spill 28 bytes).
template <typename T>
SampleKernel sample_kernel(int ctas, bool wide) {
    switch (ctas) {
        case 1: return k_sample<T, 1024, 1>;
        case 4: return k_sample<T, 1024, 4>;
        case 5: return k_sample<T, 1024, 5>;
        case 6: return k_sample<T, 1024, 6>;
        default: return wide ? k_sample<T, 1024, kSmpMostCtas> : k_sample<T, 512, kSmpMostCtas>;
    }
}
constexpr int kSmpClusters[] = {kSmpMostCtas, 6, 5, 4};  // of seven no more run at once than of eight
constexpr int kSmpMostBytes = 232448;  // a CTA's shared memory
static_assert(sizeof(SmpShared) + 4 * (size_t(TETRA_SAMPLE_MAX_VOCAB) / kSmpMostCtas) <= kSmpMostBytes, "a row of the largest vocabulary fits a cluster");

// How many clusters, each CTA with an SM for itself, the current device runs at once: by the number of CTAs.
cudaError_t wide_clusters(const int** found) {
    static int counts[64][kSmpMostCtas + 1];
    static PerDeviceOnce once;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = once.run([dev] {
        for (int c : {1, 4, 5, 6, kSmpMostCtas})
            for (bool wide : {false, true})
                for (SampleKernel kernel : {sample_kernel<float>(c, wide), sample_kernel<__half>(c, wide)}) {
                    const cudaError_t got = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmpMostBytes);
                    if (got != cudaSuccess) return got;
                }
        for (int c : kSmpClusters) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(unsigned(c));
            cfg.blockDim = dim3(1024);
            cfg.dynamicSmemBytes = kSmpMostBytes;
            const cudaError_t got = cudaOccupancyMaxActiveClusters(&counts[dev][c], sample_kernel<float>(c, true), &cfg);
            if (got != cudaSuccess) return got;
        }
        return cudaSuccess;
    });
    *found = e == cudaSuccess ? counts[dev] : nullptr;
    return e;
}

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" {

int tetra_sample(const tetra_sample_rows* p, void* stream) {
    if (!p) return TETRA_ERR_NULL;
    if (p->rows < 0 || p->rows > TETRA_SAMPLE_MAX_ROWS || p->vocab < 1 || p->vocab > TETRA_SAMPLE_MAX_VOCAB || p->row_stride < p->vocab ||
        (p->half_type != 0 && p->half_type != 1))
        return TETRA_ERR_SHAPE;
    if (p->rows == 0) return TETRA_OK;
    if (!p->logits || !p->u || !p->tokens) return TETRA_ERR_NULL;
    auto off = [](const void* q, size_t a) { return (reinterpret_cast<uintptr_t>(q) & (a - 1)) != 0; };
    if (off(p->logits, p->half_type ? 2 : 4) || off(p->u, 4) || off(p->temperature, 4) || off(p->top_k, 4) || off(p->top_p, 4) || off(p->min_p, 4) ||
        off(p->tokens, 4) || off(p->prob, 4))
        return TETRA_ERR_ALIGN;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) return TETRA_ERR_CUDA;
    // A barrier of a cluster takes ten times as long as a CTA's: a short row is one CTA's.  Measured, a cluster against one CTA,
    // us for top-k 50 with top-p 0.9 / for top-p alone / for neither: 1 row of 8000 9.0 and 6.4 / 8.5 and 8.4 / 6.6 and
    // 8.0, of 16000 9.0 and 7.2 / 8.5 and 10.8 / 6.7 and 11.2; 64 rows of 32000 19 and 9 / 30 and 29 / 19 and 20.
    const bool alone = p->vocab <= (p->rows * kSmpMostCtas > 2 * sms ? kSmpAloneMany : kSmpAlone);
    auto part_of = [&](int ctas) { return ((p->vocab + ctas - 1) / ctas + 7) / 8 * 8; };
    auto bytes_of = [&](int ctas) { return sizeof(SmpShared) + 4 * size_t(part_of(ctas)); };
    // A CTA on an SM of its own has twice the warps to hide its latencies and all of the SM's units, so of the clusters that
    // leave each CTA its SM the largest is taken; where none does, two CTAs of clusters of eight share an SM.  Clusters do not cross the
    // boundaries of the SMs' groups, so the device says how many run at once (15, 22, 26 and 33 of eight, six, five and four
    // on one).  Measured, two CTAs of eight to an SM against so, 151936 logits, us for top-k 40 with top-p 0.9 / for top-p alone /
    // for neither: 16 rows 13.2 and 11.7 / 36.7 and 32.6 / 21.5 and 17.9 (six), 24 rows 14.4 and 12.1 / 40.5 and 37.2 / 24.7
    // and 21.6 (five), 32 rows 19.9 and 13.2 / 43.0 and 43.7 / 26.4 and 25.3 (four); 40 rows in two rounds of four 24.6 and 22.1 /
    // 61.4 and 66.5 / 36.3 and 41.2.
    int ctas = alone ? 1 : kSmpMostCtas;
    bool wide = alone;
    const int* at_once = nullptr;
    if (wide_clusters(&at_once) != cudaSuccess) return TETRA_ERR_CUDA;
    for (int c : kSmpClusters)
        if (!wide && bytes_of(c) <= kSmpMostBytes && p->rows <= at_once[c]) ctas = c, wide = true;
    auto kernel = p->half_type ? sample_kernel<__half>(ctas, wide) : sample_kernel<float>(ctas, wide);
    return launch_pdl(kernel, p->rows * ctas, wide ? 1024 : 512, bytes_of(ctas), static_cast<cudaStream_t>(stream), *p, part_of(ctas)) == cudaSuccess
               ? TETRA_OK : TETRA_ERR_CUDA;
}

}  // extern "C"
