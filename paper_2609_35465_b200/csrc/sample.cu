// The next token of each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers (tetra_sample).
//
// A cluster of eight CTAs takes a row.  Each CTA reads an eighth of it once, as integer keys in the order of the floats, into
// shared memory; everything after that happens there and in the cluster's distributed shared memory.
//   * Weights are fixed-point numbers (units of 2^-44 of the largest), so sums are exact in whatever order, and what
//     is found by a histogram here, by a sort there and by a scan at the end agrees to the last bit.
//   * The three filters all keep a prefix of the order (logit down, index up), so they come to one cut: the last entry
//     (key, index) that stays.  A histogram over the distance from the largest logit finds the bin that the cut is in; the
//     bin's few entries go to one CTA, which sorts them and finds it.  A bin with too many entries (equal logits,
//     outliers) is cut by bisection over the entries instead: any input is right, the usual ones are fast.
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
    uint32_t count[kSmpBins], lo[kSmpBins], hi[kSmpBins];
    Tally mine[kSmpMine];       // inclusive sums over this CTA's bins
    Tally slots[2][kSmpCtas];   // what the CTAs tell each other
    Tally warp[kSmpWarps];
    uint64_t bin[4];            // a crossing: its bin, entries and mass before it, entries in it
    uint64_t found[2];          // a cut, and the mass up to it
    uint32_t listed;
};

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return kMinusInf;  // NaN
    if (b == 0x80000000u) return 0x80000000u;               // -0 equals 0
    return b ^ (b & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// Weight of a key in units of 2^-44: 2^t, t = (x - max) log2(e) / T, by the exponential series over half a binade to either
// side (degree 11: the remainder is 6e-15).
struct Weigh {
    uint32_t top;   // largest key
    double max, by; // its value; log2(e) / T
    __device__ __forceinline__ uint64_t operator()(uint32_t key) const {
        if (key == top) return 1ull << kSmpBits;
        const double t = (double(value_of(key)) - max) * by;
        if (!(t > -46.) || key <= kMinusInf) return 0;  // not where the largest is infinite
        const double n = rint(t), f = (t - n) * 0.693147180559945309417;
        double e = 1. / 39916800.;
        e = fma(e, f, 1. / 3628800.);
        e = fma(e, f, 1. / 362880.);
        e = fma(e, f, 1. / 40320.);
        e = fma(e, f, 1. / 5040.);
        e = fma(e, f, 1. / 720.);
        e = fma(e, f, 1. / 120.);
        e = fma(e, f, 1. / 24.);
        e = fma(e, f, 1. / 6.);
        e = fma(e, f, .5);
        e = fma(e, f, 1.);
        e = fma(e, f, 1.);
        return __double2ull_rn(__longlong_as_double(__double_as_longlong(e) + (int64_t(n) + kSmpBits) * (1ll << 52)));
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

// The crossing of a bin's inclusive sums with `need` (entries, or mass): told to all CTAs in sm.bin.
template <bool MASS>
__device__ __forceinline__ void find_bin(Row& row, Tally before, uint64_t need) {
    SmpShared& sm = row.sm;
    if (threadIdx.x < kSmpMine) {
        const Tally upto = before + sm.mine[threadIdx.x], from = threadIdx.x ? before + sm.mine[threadIdx.x - 1] : before;
        const uint64_t a = MASS ? from.mass : from.count, b = MASS ? upto.mass : upto.count;
        if (a < need && need <= b) {
            for (int r = 0; r < kSmpCtas; ++r) {
                uint64_t* found = row.cluster.map_shared_rank(sm.bin, r);
                found[0] = uint64_t(row.rank * kSmpMine) + threadIdx.x;
                found[1] = from.count;
                found[2] = from.mass;
                found[3] = upto.count - from.count;
            }
        }
    }
    row.cluster.sync();
}

// The entry with which `need` (entries, or mass, counted from the largest logit) is reached, and the mass up to it.
template <bool MASS>
__device__ __forceinline__ void find_cut(Row& row, const Bins& bins, const Weigh& weigh, Tally before, uint64_t need, uint64_t& cut, uint64_t& mass) {
    SmpShared& sm = row.sm;
    find_bin<MASS>(row, before, need);
    const uint32_t bin = uint32_t(sm.bin[0]), entries = uint32_t(sm.bin[3]);
    const Tally ahead{sm.bin[2], sm.bin[1]};
    if (entries <= kSmpList) {
        uint64_t* list = row.cluster.map_shared_rank(sm.list, 0);
        uint32_t* listed = row.cluster.map_shared_rank(&sm.listed, 0);
        for (int i = threadIdx.x; i < row.count; i += kSmpThreads)
            if (bins(row.keys[i]) == bin) list[atomicAdd(listed, 1u)] = row.entry(i);
        row.cluster.sync();
        if (row.rank == 0) {
            uint32_t size = 2;
            while (size < entries) size <<= 1;
            for (uint32_t i = entries + threadIdx.x; i < size; i += kSmpThreads) sm.list[i] = 0;
            for (uint32_t k = 2; k <= size; k <<= 1)
                for (uint32_t j = k >> 1; j > 0; j >>= 1) {  // bitonic, the largest first
                    __syncthreads();
                    for (uint32_t i = threadIdx.x; i < size / 2; i += kSmpThreads) {
                        const uint32_t a = (i & ~(j - 1)) << 1 | (i & (j - 1)), b = a | j;
                        const uint64_t u = sm.list[a], v = sm.list[b];
                        if ((u < v) == !(a & k)) sm.list[a] = v, sm.list[b] = u;
                    }
                }
            __syncthreads();
            constexpr int PER = kSmpList / kSmpThreads;
            Tally own[PER], sum{0, 0}, total;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t at = threadIdx.x * PER + i;
                own[i] = at < entries ? Tally{weigh(uint32_t(sm.list[at] >> 32)), 1} : Tally{0, 0};
                sum = sum + own[i];
            }
            Tally upto = ahead + block_scan(sm, sum, total);
            upto = {upto.mass - sum.mass, upto.count - sum.count};
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const Tally from = upto;
                upto = upto + own[i];
                if (own[i].count && (MASS ? from.mass < need && need <= upto.mass : from.count < need && need <= upto.count)) {
                    for (int r = 0; r < kSmpCtas; ++r) {
                        uint64_t* found = row.cluster.map_shared_rank(sm.found, r);
                        found[0] = sm.list[threadIdx.x * PER + i];
                        found[1] = upto.mass;
                    }
                }
            }
            if (threadIdx.x == 0) sm.listed = 0;
        }
        row.cluster.sync();
        cut = sm.found[0];
        mass = sm.found[1];
    } else {
        // The largest c with enough in the entries >= c: one bit after another.
        uint64_t c = 0, upto = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t mid = c | 1ull << bit;
            Tally v{0, 0}, total;
            for (int i = threadIdx.x; i < row.count; i += kSmpThreads)
                if (row.entry(i) >= mid && bins(row.keys[i]) == bin) v = v + Tally{weigh(row.keys[i]), 1};
            block_scan(sm, v, total);
            const Tally* all = row.tell(total);
            total = ahead;
            for (int r = 0; r < kSmpCtas; ++r) total = total + all[r];
            if ((MASS ? total.mass : total.count) >= need) c = mid, upto = total.mass;
        }
        cut = c;
        mass = upto;
    }
    // sm.bin and sm.found are written again behind a barrier of the cluster that follows these reads.
}

template <typename T>
__cluster_dims__(kSmpCtas, 1, 1) __global__ void __launch_bounds__(kSmpThreads) k_sample(tetra_sample_rows p, int part) {
    extern __shared__ __align__(16) unsigned char smem[];
    SmpShared& sm = *reinterpret_cast<SmpShared*>(smem);
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem + sizeof(SmpShared));
    pdl_wait();
    pdl_release();
    const int r = blockIdx.x / kSmpCtas, rank = blockIdx.x % kSmpCtas, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int begin = min(part * rank, p.vocab), count = min(part, p.vocab - begin);
    Row row{sm, keys, count, uint32_t(begin), cg::this_cluster(), rank, 0};
    if (threadIdx.x == 0) sm.listed = 0;

    // The part, as keys; its largest entry, its least finite key.
    const T* x = static_cast<const T*>(p.logits) + r * p.row_stride + begin;
    uint64_t best = 0;
    uint32_t least = 0xFFFFFFFFu;
    for (int i = threadIdx.x; i < count; i += kSmpThreads) {
        const uint32_t key = key_of(float(x[i]));
        keys[i] = key;
        best = max(best, row.entry(i));
        if (key > kMinusInf) least = min(least, key);
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    if (lane == 0) sm.warp[warp] = {best, least};
    for (int i = threadIdx.x; i < kSmpBins; i += kSmpThreads) sm.count[i] = sm.lo[i] = sm.hi[i] = 0;
    __syncthreads();
    for (int w = 0; w < kSmpWarps; ++w) best = max(best, sm.warp[w].mass), least = min(least, uint32_t(sm.warp[w].count));
    const Tally* all = row.tell({best, least});
    for (int c = 0; c < kSmpCtas; ++c) best = max(best, all[c].mass), least = min(least, uint32_t(all[c].count));
    const uint32_t top = uint32_t(best >> 32);

    const float T_row = p.temperature ? p.temperature[r] : 1.f;
    if (top <= kMinusInf || !(T_row > 0.f)) {
        if (rank == 0 && threadIdx.x == 0) {
            p.tokens[r] = top <= kMinusInf ? -1 : int(~uint32_t(best));
            if (p.prob) p.prob[r] = top <= kMinusInf ? 0.f : 1.f;
        }
        return;
    }
    const Weigh weigh{top, double(value_of(top)), 1.4426950408889634074 / double(T_row)};
    float p_row = p.top_p ? p.top_p[r] : 1.f, m_row = p.min_p ? p.min_p[r] : 0.f;
    int64_t k_row = p.top_k ? p.top_k[r] : 0;
    if (k_row <= 0) k_row = INT32_MAX;
    if (p_row <= 0.f || m_row > 1.f) k_row = 1;
    const bool nucleus = p_row < 1.f && k_row > 1;
    const uint64_t floor_w = m_row > 0.f && m_row <= 1.f ? uint64_t(ceil(double(m_row) * double(1ull << kSmpBits))) : 0;

    uint64_t cut = 0;
    if (k_row < p.vocab || nucleus) {
        // e^-31.25 is less than half a unit
        const float max = value_of(top), range = fminf(fminf(max - value_of(least), 31.25f * T_row), 3.0e38f);
        const Bins bins{top, max, range, range > 1e-30f ? float(kSmpBins) / range : 0.f};
        for (int i = threadIdx.x; i < count; i += kSmpThreads) {
            const uint32_t bin = bins(keys[i]);
            if (bin < kSmpBins) {
                const uint64_t w = weigh(keys[i]);
                const uint32_t lo = uint32_t(w), old = atomicAdd(&sm.lo[bin], lo);
                atomicAdd(&sm.hi[bin], uint32_t(w >> 32) + (old + lo < old));  // with the carry: a 64-bit sum
                atomicAdd(&sm.count[bin], 1u);
            }
        }
        row.cluster.sync();
        Tally v{0, 0}, total;
        if (threadIdx.x < kSmpMine)
            for (int c = 0; c < kSmpCtas; ++c) {
                const SmpShared* other = row.cluster.map_shared_rank(&sm, c);
                const int b = rank * kSmpMine + threadIdx.x;
                v = v + Tally{(uint64_t(other->hi[b]) << 32) + other->lo[b], other->count[b]};
            }
        v = block_scan(sm, v, total);
        if (threadIdx.x < kSmpMine) sm.mine[threadIdx.x] = v;
        all = row.tell(total);
        Tally before{0, 0}, whole{0, 0};
        for (int c = 0; c < kSmpCtas; ++c) {
            if (c == rank) before = whole;
            whole = whole + all[c];
        }
        uint64_t mass = whole.mass;
        if (uint64_t(k_row) < whole.count) find_cut<false>(row, bins, weigh, before, uint64_t(k_row), cut, mass);
        if (nucleus) {
            uint64_t need = uint64_t(ceil(double(p_row) * double(mass))), got;
            need = need < 1 ? 1 : need > mass ? mass : need;
            find_cut<true>(row, bins, weigh, before, need, cut, got);
        }
    }

    // The draw: kept weights in the order of the indexes, so many consecutive ones a thread.
    const int per = (part + kSmpThreads - 1) / kSmpThreads | 1;  // odd: no bank conflicts
    const int from = min(int(threadIdx.x) * per, count), to = min(from + per, count);
    auto kept = [&](int i) -> uint64_t {
        if (row.entry(i) < cut) return 0;
        const uint64_t w = weigh(keys[i]);
        return w >= floor_w ? w : 0;
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
    const double u = fmin(fmax(double(p.u[r]), 0.), 1.);  // NaN: 0
    uint64_t aim = uint64_t(u * double(mass));
    if (aim >= mass) aim = mass - 1;
    const bool mine = base + upto - sum <= aim && aim < base + upto;
    const uint32_t who = __ballot_sync(0xFFFFFFFFu, mine);
    if (who) {  // the warp walks through the thread's tokens together
        const int l = __ffs(who) - 1, a = __shfl_sync(0xFFFFFFFFu, from, l), b = __shfl_sync(0xFFFFFFFFu, to, l);
        uint64_t at = __shfl_sync(0xFFFFFFFFu, base + upto - sum, l);
        for (int i = a; i < b; i += 32) {
            const uint64_t w = i + lane < b ? kept(i + lane) : 0;
            const uint64_t end = at + warp_scan({w, 0}, lane).mass;
            if (end - w <= aim && aim < end) {
                p.tokens[r] = int(row.index) + i + lane;
                if (p.prob) p.prob[r] = float(double(w) / double(mass));
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
