// The next token of each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers (tetra_sample).
//
// A cluster of eight CTAs takes a row.  Each CTA reads an eighth of it once, as integer keys in the order of the floats, into
// shared memory; everything after that happens there and in the cluster's distributed shared memory.
//   * Weights are fixed-point numbers (units of 2^-44 of the largest), so sums are exact in whatever order, and what
//     is found by a histogram here, by a sort there and by a scan at the end agrees to the last bit.
//   * The three filters all keep a prefix of the order (logit down, index up), so they come to one cut: the last entry
//     (key, index) that stays.  Top-k: a histogram of counts over the distance from the largest logit finds the bin of the
//     k-th; where the bins up to it hold no more than 2048 entries these go to one CTA, which sorts them and does all the
//     rest.  Otherwise, and for top-p without top-k, a histogram of masses finds the bin that the cut is in, and the one CTA
//     sorts that bin.  A bin with too many entries (equal logits, outliers) is cut by bisection over the entries instead:
//     any input is right, the usual ones are fast.
//   * The draw scans the kept weights in the order of the indexes.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "../../include/tetra.h"
#include "../../include/tetra_sample.h"
#include "tetra_gemv_common.cuh"

namespace tetra {
namespace {

namespace cg = cooperative_groups;

constexpr int kSmpThreads = 512, kSmpWarps = kSmpThreads / 32, kSmpCtas = 8;
constexpr int kSmpBins = 1024, kSmpMine = kSmpBins / kSmpCtas;  // bins of the cluster, and those that a CTA adds up
constexpr int kSmpList = 2048;                                  // entries of a bin that are sorted
constexpr int kSmpBits = 44;                                    // a weight of 1 is 2^44
constexpr uint32_t kMinusInf = 0x007FFFFFu;                     // its key

static_assert(kSmpCtas * kSmpThreads > 0 && TETRA_SAMPLE_MAX_VOCAB <= 1 << 19, "sums of weights stay below 2^63");

struct Tally {  // so many entries with so much mass
    uint64_t mass;
    uint64_t count;
};

struct SmpShared {
    uint64_t list[kSmpList];
    double powers[64];          // 2^(44 + j / 64)
    uint32_t lo[kSmpBins], hi[kSmpBins];  // counts (lo), or masses
    Tally mine[kSmpMine];       // inclusive sums over this CTA's bins
    Tally slots[2][kSmpCtas];   // what the CTAs tell each other
    Tally warp[kSmpWarps];
    uint64_t bin[3];            // a crossing: its bin, sum before it, sum in it
    uint64_t found[2];          // a cut, and the mass up to it
    uint32_t listed[2];         // by the first gathering, by the second
};

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return kMinusInf;  // NaN
    if (b == 0x80000000u) return 0x80000000u;               // -0 equals 0
    return b ^ (b & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// Weight of a key in units of 2^-44: 2^t, t = (x - max) log2(e) / T = k / 64 + f / 64 with |f| <= 1/2, as 2^(k / 64) from a table
// times the exponential series of f ln 2 / 64 up to the fourth power (the next is 4e-14, 2^-44), rounded once; in float64, whose
// multiply-adds run at half the rate of float32's here.  Adding 1.5 * 2^52 leaves a whole number in the low bits.
struct Weigh {
    uint32_t top;           // largest key
    double max, by;         // its value; 64 log2(e) / T
    const double* powers;
    __device__ __forceinline__ uint64_t operator()(uint32_t key) const {
        constexpr double magic = 6755399441055744.;
        if (key == top) return 1ull << kSmpBits;
        const double d = double(value_of(key)) - max, t = d * by;
        if (!(t > -46. * 64.) || key <= kMinusInf) return 0;  // not where the largest is infinite
        const double m = t + magic, f = t - (m - magic);
        const int k = __double2loint(m);
        constexpr double c = 0.693147180559945309417 / 64.;
        double e = fma(c * c * c * c / 24., f, c * c * c / 6.);
        e = fma(e, f, c * c / 2.);
        e = fma(e, f, c);
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
// ... over the CTA's threads up to this one; `total` is the CTA's.
__device__ __forceinline__ Tally block_scan(SmpShared& sm, Tally v, Tally& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_scan(v, lane);
    __syncthreads();
    if (lane == 31) sm.warp[warp] = v;
    __syncthreads();
    total = {0, 0};
    Tally before{0, 0};
#pragma unroll
    for (int w = 0; w < kSmpWarps; ++w) {
        if (w == warp) before = total;
        total = total + sm.warp[w];
    }
    return before + v;
}

// Sorts list[0 .. size), a power of two, the largest first.  Up to 64 entries are the first warp's own work.
__device__ __forceinline__ void sort_list(uint64_t* list, uint32_t size) {
    const bool small = size <= 64;
    for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            if (small) __syncwarp();
            else __syncthreads();
            for (uint32_t i = threadIdx.x; i < size / 2; i += kSmpThreads) {
                const uint32_t a = (i & ~(j - 1)) << 1 | (i & (j - 1)), b = a | j;
                const uint64_t u = list[a], v = list[b];
                if ((u < v) == !(a & k)) list[a] = v, list[b] = u;
            }
        }
    __syncthreads();
}
__device__ __forceinline__ uint32_t power_of_two(uint32_t n) {
    uint32_t size = 2;
    while (size < n) size <<= 1;
    return size;
}

struct Row {
    SmpShared& sm;
    const uint32_t* keys;
    int count;      // of this CTA's part
    uint32_t index; // of its first token
    cg::cluster_group cluster;
    int rank, turn;

    // Every CTA's value for every CTA, in the order of their ranks.
    __device__ __forceinline__ const Tally* tell(Tally mine) {
        Tally* slots = sm.slots[turn & 1];
        ++turn;
        if (threadIdx.x < kSmpCtas) cluster.map_shared_rank(slots, threadIdx.x)[rank] = mine;
        cluster.sync();
        return slots;
    }
    __device__ __forceinline__ uint64_t entry(int i) const { return uint64_t(keys[i]) << 32 | uint32_t(~(index + uint32_t(i))); }
};

// Distance bins: key -> bin, the largest logit in bin 0; kSmpBins for a key without mass.
struct Bins {
    uint32_t top;
    float max, range, by;
    __device__ __forceinline__ uint32_t operator()(uint32_t key) const {
        if (key == top) return 0;
        const float d = max - value_of(key);
        if (!(d <= range) || key <= kMinusInf) return kSmpBins;
        return min(uint32_t(kSmpBins - 1), uint32_t(d * by));
    }
};

// The histogram's sums (counts, or masses: as Tally.mass) over the cluster: an eighth of the bins to each CTA, whose inclusive sums
// are left in sm.mine; what is before them, and the whole.
__device__ __forceinline__ void add_bins(Row& row, uint64_t& before, uint64_t& whole) {
    SmpShared& sm = row.sm;
    row.cluster.sync();
    uint64_t v = 0;
    if (threadIdx.x < kSmpMine) {
        const int b = row.rank * kSmpMine + threadIdx.x;
#pragma unroll
        for (int c = 0; c < kSmpCtas; ++c) {
            const SmpShared* other = row.cluster.map_shared_rank(&sm, c);
            v += (uint64_t(other->hi[b]) << 32) + other->lo[b];
        }
    }
    Tally total;
    const Tally upto = block_scan(sm, {v, 0}, total);
    if (threadIdx.x < kSmpMine) sm.mine[threadIdx.x] = upto;
    const Tally* all = row.tell(total);
    before = whole = 0;
    for (int c = 0; c < kSmpCtas; ++c) {
        if (c == row.rank) before = whole;
        whole += all[c].mass;
    }
}

// The bin in which the sums reach `need`, 0 < need <= whole: told to all CTAs in sm.bin.
__device__ __forceinline__ void find_bin(Row& row, uint64_t before, uint64_t need) {
    SmpShared& sm = row.sm;
    if (threadIdx.x < kSmpMine) {
        const uint64_t upto = before + sm.mine[threadIdx.x].mass, from = threadIdx.x ? before + sm.mine[threadIdx.x - 1].mass : before;
        if (from < need && need <= upto)
            for (int r = 0; r < kSmpCtas; ++r) {
                uint64_t* bin = row.cluster.map_shared_rank(sm.bin, r);
                bin[0] = uint64_t(row.rank * kSmpMine) + threadIdx.x;
                bin[1] = from;
                bin[2] = upto - from;
            }
    }
    row.cluster.sync();
}

// Entries of the bins [low, high] that are not below `cut` into the list of the first CTA, whose sm.listed[which] says how
// many there are (more than kSmpList: the list is not whole).  A row gathers at most twice.
__device__ __forceinline__ void gather(Row& row, const Bins& bins, uint32_t low, uint32_t high, uint64_t cut, int which) {
    uint64_t* list = row.cluster.map_shared_rank(row.sm.list, 0);
    uint32_t* listed = row.cluster.map_shared_rank(row.sm.listed + which, 0);
    for (int i = threadIdx.x; i < row.count; i += kSmpThreads) {
        const uint32_t bin = bins(row.keys[i]);
        if (bin >= low && bin <= high && row.entry(i) >= cut) {
            const uint32_t at = atomicAdd(listed, 1u);
            if (at < kSmpList) list[at] = row.entry(i);
        }
    }
    row.cluster.sync();
}

// The entry in bin sm.bin[0] with which `need` (entries, or mass, counted from the largest logit, of the entries not below
// `least`) is reached, and the mass in the bin up to it.
template <bool MASS>
__device__ __forceinline__ uint64_t find_cut(Row& row, const Bins& bins, const Weigh& weigh, uint64_t need, uint64_t least) {
    SmpShared& sm = row.sm;
    const uint32_t bin = uint32_t(sm.bin[0]);
    const uint64_t ahead = sm.bin[1];
    gather(row, bins, bin, bin, least, MASS);
    const uint32_t entries = *row.cluster.map_shared_rank(row.sm.listed + MASS, 0);  // that CTA passes another barrier before it ends
    if (entries <= kSmpList) {
        if (row.rank == 0) {
            const uint32_t size = power_of_two(entries);
            for (uint32_t i = entries + threadIdx.x; i < size; i += kSmpThreads) sm.list[i] = 0;
            __syncthreads();
            sort_list(sm.list, size);
            constexpr int PER = kSmpList / kSmpThreads;
            uint64_t own[PER], sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t at = threadIdx.x * PER + i;
                own[i] = at < entries ? MASS ? weigh(uint32_t(sm.list[at] >> 32)) : 1ull : 0ull;
                sum += own[i];
            }
            Tally total;
            uint64_t upto = ahead + block_scan(sm, {sum, 0}, total).mass - sum;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint64_t from = upto;
                upto += own[i];
                if (from < need && need <= upto)
                    for (int r = 0; r < kSmpCtas; ++r) *row.cluster.map_shared_rank(sm.found, r) = sm.list[threadIdx.x * PER + i];
            }
        }
        row.cluster.sync();
        // sm.bin and sm.found are written again behind a barrier of the cluster that follows these reads.
        return sm.found[0];
    }
    // The largest c with enough in the entries >= c: one bit after another.
    uint64_t c = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t mid = c | 1ull << bit;
        Tally v{0, 0}, total;
        for (int i = threadIdx.x; i < row.count; i += kSmpThreads) {
            const uint64_t entry = row.entry(i);
            if (entry >= mid && entry >= least && bins(row.keys[i]) == bin) v.mass += MASS ? weigh(row.keys[i]) : 1ull;
        }
        block_scan(sm, v, total);
        const Tally* all = row.tell(total);
        uint64_t sum = ahead;
        for (int r = 0; r < kSmpCtas; ++r) sum += all[r].mass;
        if (sum >= need) c = mid;
    }
    return c;
}

struct Settings {
    uint64_t k;       // entries that stay
    float p;          // 1 and above: off
    uint64_t floor_w; // least weight
    float u;
};

__device__ __forceinline__ uint64_t needed(float p, uint64_t mass) {
    const uint64_t need = uint64_t(ceil(double(p) * double(mass)));
    return need < 1 ? 1 : need > mass ? mass : need;
}
__device__ __forceinline__ uint64_t aimed(float u, uint64_t mass) {
    const uint64_t aim = uint64_t(fmin(fmax(double(u), 0.), 1.) * double(mass));  // NaN: 0
    return aim >= mass ? mass - 1 : aim;
}

// All of the filters and the draw among sm.list[0 .. n), which holds the first n entries in the order, n >= 1: one CTA.
__device__ __forceinline__ void finish(SmpShared& sm, const Weigh& weigh, uint32_t n, const Settings& set, int32_t* token, float* prob) {
    constexpr int PER = kSmpList / kSmpThreads;
    uint32_t size = power_of_two(n);
    for (uint32_t i = n + threadIdx.x; i < size; i += kSmpThreads) sm.list[i] = 0;
    __syncthreads();
    sort_list(sm.list, size);
    if (set.k < n) n = uint32_t(set.k);
    uint64_t entry[PER], own[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t at = threadIdx.x * PER + i;
        entry[i] = at < n ? sm.list[at] : 0;
        own[i] = at < n ? weigh(uint32_t(entry[i] >> 32)) : 0;
        sum += own[i];
    }
    Tally total;
    uint64_t from = block_scan(sm, {sum, 0}, total).mass - sum;
    const uint64_t need = set.p < 1.f ? needed(set.p, total.mass) : ~0ull;
    // What stays, in the order of the indexes: (~index, key) sorted the same way.
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t at = threadIdx.x * PER + i;
        const bool stays = at < n && from < need && own[i] >= set.floor_w;
        if (at < size) sm.list[at] = stays ? entry[i] << 32 | entry[i] >> 32 : 0;
        from += own[i];
    }
    size = power_of_two(n);
    __syncthreads();
    sort_list(sm.list, size);
    sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t at = threadIdx.x * PER + i;
        entry[i] = at < n ? sm.list[at] : 0;
        own[i] = entry[i] ? weigh(uint32_t(entry[i])) : 0;
        sum += own[i];
    }
    from = block_scan(sm, {sum, 0}, total).mass - sum;
    const uint64_t aim = aimed(set.u, total.mass);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (from <= aim && aim < from + own[i]) {
            *token = int(~uint32_t(entry[i] >> 32));
            if (prob) *prob = float(double(own[i]) / double(total.mass));
        }
        from += own[i];
    }
}

// Adds a mass to a bin's: 64 bits in two words, the carry by hand.
__device__ __forceinline__ void add_mass(SmpShared& sm, uint32_t bin, uint64_t w) {
    const uint32_t lo = uint32_t(w), old = atomicAdd(&sm.lo[bin], lo), hi = uint32_t(w >> 32) + (old + lo < old);
    if (hi) atomicAdd(&sm.hi[bin], hi);
}

template <typename T>
__cluster_dims__(kSmpCtas, 1, 1) __global__ void __launch_bounds__(kSmpThreads) k_sample(tetra_sample_rows p, int part) {
    extern __shared__ __align__(16) unsigned char smem[];
    SmpShared& sm = *reinterpret_cast<SmpShared*>(smem);
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem + sizeof(SmpShared));
    const int r = blockIdx.x / kSmpCtas, rank = blockIdx.x % kSmpCtas, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int begin = min(part * rank, p.vocab), count = min(part, p.vocab - begin);
    Row row{sm, keys, count, uint32_t(begin), cg::this_cluster(), rank, 0};
    if (threadIdx.x < 2) sm.listed[threadIdx.x] = 0;
    if (threadIdx.x < 64) sm.powers[threadIdx.x] = exp2(kSmpBits + threadIdx.x / 64.);
    for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.lo[i] = sm.hi[i] = 0;
    pdl_wait();
    pdl_release();

    // The part, as keys; its largest entry, its least finite key.
    const T* x = static_cast<const T*>(p.logits) + r * p.row_stride + begin;
    uint32_t most = 0, most_at = 0, least = 0xFFFFFFFFu;
    auto take = [&](int i, float v) {
        const uint32_t key = key_of(v);
        keys[i] = key;
        if (key > most) most = key, most_at = uint32_t(i);  // a thread's tokens come in order: the first of equal ones
        if (key > kMinusInf) least = min(least, key);
    };
    constexpr int VEC = 16 / sizeof(T);
    if ((reinterpret_cast<uintptr_t>(x) & 15) == 0) {
#pragma unroll 4
        for (int i = threadIdx.x; i < count / VEC; i += kSmpThreads) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(x) + i);
            const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) take(i * VEC + k, float(e[k]));
        }
        for (int i = count / VEC * VEC + threadIdx.x; i < count; i += kSmpThreads) take(i, float(x[i]));
    } else {
#pragma unroll 8
        for (int i = threadIdx.x; i < count; i += kSmpThreads) take(i, float(x[i]));
    }
    uint64_t best = most ? uint64_t(most) << 32 | uint32_t(~(uint32_t(begin) + most_at)) : 0;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    if (lane == 0) sm.warp[warp] = {best, least};
    __syncthreads();
    for (int w = 0; w < kSmpWarps; ++w) best = max(best, sm.warp[w].mass), least = min(least, uint32_t(sm.warp[w].count));
    const Tally* all = row.tell({best, least});
    for (int c = 0; c < kSmpCtas; ++c) best = max(best, all[c].mass), least = min(least, uint32_t(all[c].count));
    const uint32_t top = uint32_t(best >> 32);

    int32_t* token = p.tokens + r;
    float* prob = p.prob ? p.prob + r : nullptr;
    const float T_row = p.temperature ? p.temperature[r] : 1.f, p_row = p.top_p ? p.top_p[r] : 1.f, m_row = p.min_p ? p.min_p[r] : 0.f;
    const int k_row = p.top_k ? p.top_k[r] : 0;
    const bool one = p_row <= 0.f || m_row > 1.f || k_row == 1;  // the first alone stays
    if (top <= kMinusInf || !(T_row > 0.f) || one) {
        if (rank == 0 && threadIdx.x == 0) {
            *token = top <= kMinusInf ? -1 : int(~uint32_t(best));
            if (prob) *prob = top <= kMinusInf ? 0.f : 1.f;
        }
        return;
    }
    const Weigh weigh{top, double(value_of(top)), 64. * 1.4426950408889634074 / double(T_row), sm.powers};
    const Settings set{k_row > 0 ? uint64_t(k_row) : ~0ull, p_row, m_row > 0.f ? uint64_t(ceil(double(m_row) * double(1ull << kSmpBits))) : 0ull, p.u[r]};
    const bool nucleus = p_row < 1.f, top_k = k_row > 0 && k_row < p.vocab;

    uint64_t cut = 0;
    if (top_k || nucleus) {
        // e^-31.25 is less than half a unit
        const float max = value_of(top), range = fminf(fminf(max - value_of(least), 31.25f * T_row), 3.0e38f);
        const Bins bins{top, max, range, range > 1e-30f ? float(kSmpBins) / range : 0.f};
        uint64_t before, whole;
        if (top_k) {
            for (int i = threadIdx.x; i < count; i += kSmpThreads) {
                const uint32_t bin = bins(keys[i]);
                if (bin < kSmpBins) atomicAdd(&sm.lo[bin], 1u);
            }
            add_bins(row, before, whole);
            uint32_t last = kSmpBins - 1;
            uint64_t entries = whole;
            if (set.k < whole) {
                find_bin(row, before, set.k);
                last = uint32_t(sm.bin[0]);
                entries = sm.bin[1] + sm.bin[2];
            }
            if (entries <= kSmpList) {
                gather(row, bins, 0, last, 0, 0);
                if (rank == 0) finish(sm, weigh, uint32_t(entries), set, token, prob);
                return;
            }
            if (set.k < whole) cut = find_cut<false>(row, bins, weigh, set.k, 0);
            if (nucleus) {  // the other CTAs have read these counts: add_bins told the sums behind them
                for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.lo[i] = 0;
                __syncthreads();
            }
        }
        if (nucleus) {
            for (int i = threadIdx.x; i < count; i += kSmpThreads) {
                const uint32_t bin = bins(keys[i]);
                if (bin < kSmpBins && row.entry(i) >= cut) add_mass(sm, bin, weigh(keys[i]));
            }
            add_bins(row, before, whole);
            const uint64_t need = needed(p_row, whole);
            find_bin(row, before, need);
            cut = find_cut<true>(row, bins, weigh, need, cut);
        }
    }

    // The draw: kept weights in the order of the indexes, so many consecutive ones a thread.
    const int per = (part + kSmpThreads - 1) / kSmpThreads | 1;  // odd: no bank conflicts
    const int from = min(int(threadIdx.x) * per, count), to = min(from + per, count);
    auto kept = [&](int i) -> uint64_t {
        if (row.entry(i) < cut) return 0;
        const uint64_t w = weigh(keys[i]);
        return w >= set.floor_w ? w : 0;
    };
    uint64_t sum = 0;
    for (int i = from; i < to; ++i) sum += kept(i);
    Tally total;
    const uint64_t upto = block_scan(sm, {sum, 0}, total).mass;
    all = row.tell(total);
    uint64_t base = 0, mass = 0;
    for (int c = 0; c < kSmpCtas; ++c) {
        if (c == rank) base = mass;
        mass += all[c].mass;
    }
    const uint64_t aim = aimed(set.u, mass);
    const bool mine = base + upto - sum <= aim && aim < base + upto;
    const uint32_t who = __ballot_sync(0xFFFFFFFFu, mine);
    if (who) {  // the warp walks through the thread's tokens together
        const int l = __ffs(who) - 1, a = __shfl_sync(0xFFFFFFFFu, from, l), b = __shfl_sync(0xFFFFFFFFu, to, l);
        uint64_t at = __shfl_sync(0xFFFFFFFFu, base + upto - sum, l);
        for (int i = a; i < b; i += 32) {
            const uint64_t w = i + lane < b ? kept(i + lane) : 0;
            const uint64_t end = at + warp_scan({w, 0}, lane).mass;
            if (end - w <= aim && aim < end) {
                *token = int(row.index) + i + lane;
                if (prob) *prob = float(double(w) / double(mass));
            }
            at = __shfl_sync(0xFFFFFFFFu, end, 31);
        }
    }
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
    const int part = ((p->vocab + kSmpCtas - 1) / kSmpCtas + 7) / 8 * 8;
    const size_t smem = sizeof(SmpShared) + 4 * size_t(part);
    constexpr size_t most = sizeof(SmpShared) + 4 * (size_t(TETRA_SAMPLE_MAX_VOCAB) / kSmpCtas);
    static_assert(most <= 232448, "a CTA's shared memory");
    static PerDeviceOnce once;
    const cudaError_t e = once.run([] {
        const cudaError_t first = cudaFuncSetAttribute(k_sample<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(most));
        return first != cudaSuccess ? first : cudaFuncSetAttribute(k_sample<__half>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(most));
    });
    if (e != cudaSuccess) return TETRA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int grid = p->rows * kSmpCtas;
    return launch_pdl(p->half_type ? k_sample<__half> : k_sample<float>, grid, kSmpThreads, smem, s, *p, part) == cudaSuccess ? TETRA_OK : TETRA_ERR_CUDA;
}

}  // extern "C"
