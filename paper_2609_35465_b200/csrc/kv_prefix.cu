// Attention of a group's rows to the tokens that its sequences share (the first kernel of tetra_kv_attend_shared).
//
// S answers behind one prompt are S times the query heads of a group as columns for the same keys: 256 columns a kv head for 64
// answers of a model with four query heads to a kv head.  2 D bytes a token and kv head stand against 4 D multiply-adds a column, so
// from about 100 columns on the tensor cores bound it, not HBM, and tcgen05 pays: a tile of 128 columns is one operand's 128 rows.
//
// Work.  An item is (group, kv head, tile of 256 columns; 128 with heads of 256), its tokens come in steps of 64 (four records)
// and are cut into parts; what a CTA does is found by each CTA from the lengths, which are on the device.  A part leaves its sums
// in the workspace; k_kv_attend does the sequences' own tokens meanwhile, and k_kv_join adds both.  No atomics on memory:
// bit-identical from run to run.
//
// A CTA.  One warp copies records by cp.async.bulk into a ring.  Four warps turn their bytes into float16 (exact: codes are small
// integers) and lay them out for the tensor cores: keys as [token][dim], values as [dim][token], rows of 128 bytes, swizzled; the
// order of the tokens inside a block is that in which a lane's bytes lie, the same for both.  One thread a slot issues the
// products: S = Q K^T and O += P V (P from tensor memory, over S).  Two groups of four warps ("slots"), a thread a column, turn S
// into weights: no value of a column is in another thread, so there are no exchanges.  The slots take the two halves of a tile's
// columns, or, where a tile has no more than 128, every other step, so that the products of one run beside the exponentials of the
// other.  A slot has two places for scores, so that those of its next step are there when the weights of this one are, and a warp
// of its own that issues its products.
//
// What bounds it: for 64 tokens of 256 columns the exponentials alone take 1024 cycles (four a scheduler and cycle), what else the
// warps of the weights issue beside them makes it 1570, the products 1280; a step takes about 2100.  With one place for scores it
// was 3300 to 3500, with one warp for both slots' products, which waits for one slot while the other could go on, 2700.  64 answers
// with 32/8 heads of 128 behind 16384 tokens: 31 us, 4300 cycles of which find out how work is cut and 4000 are the first step's
// loads, 3 times the time of the bytes (34 MB) or of the products; with k_kv_attend's 15 and k_kv_join's 6 behind it 60 us, where
// each sequence for itself takes 243.
//
// Arithmetic is that of k_kv_attend: scores are exact products summed in float32, times s_K (not rounded before the reference is
// taken off, where that is small: kPreLargeRef); weights enter as float16(2^(score - m) s_V) with m a running reference, a whole
// number, that moves only when a block's weights together would pass 2^15, an s_V below 2^-60 counting as that; the denominator
// sums 2^(score - m) in float32.
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "kv_shared.cuh"

namespace tetra {
namespace {

constexpr int kPreStep = 64;                              // tokens
constexpr int kPreBlocks = kPreStep / kKvBlock;
constexpr int kPreSoft = 8, kPreConvert = 4;              // warps
constexpr int kPreConvertAt = kPreSoft, kPreCopyWarp = kPreSoft + kPreConvert, kPreMmaWarp = kPreCopyWarp + 1;
constexpr int kPreThreads = (kPreMmaWarp + 2) * 32;       // a warp a slot issues products
constexpr int kPreScales = 8;                             // steps whose scales are kept
constexpr uint32_t kPrePartCost = 8;                      // steps that a part's beginning and end take
constexpr uint32_t kPreTries = 1u << 22;                  // of a wait: then the call's results are NaN
constexpr int kPreSmem = 227 * 1024 - 2304;               // what a CTA may have, but for the barriers
constexpr float kPreNoRef = -FLT_MAX, kPreLeastLog = -60.f, kPreHigh = 15.f, kPreBase = 7.f;  // as in k_kv_attend
// Next to a reference up to this a score is not rounded before the reference is taken off (one fma for two scores).  From 2^27 on
// a score that is not rounded is powers of two beside the one that is, which is what the reference was found from: next to larger
// references a score is rounded first, as in k_kv_attend.  That goes by the column's own reference: what its weights are made from
// does not depend on the other columns.  (A packed product and a packed sum with .rn become one fma all the same: measured.)
constexpr float kPreLargeRef = 65536.f;

template <int D>
struct PreCfg {
    static constexpr int SLOTS = pre_slots(D);
    static constexpr bool QTENSOR = D == 256;             // queries in tensor memory, else in shared memory
    static constexpr int REC = kv_record_bytes(D), STAGE = kPreBlocks * REC;
    static constexpr int TILE = kPreStep * D * 2, TILES = D == 256 ? 4 : 6;  // bytes of a step's keys, or values, in float16; tiles
    static constexpr int QTILE = QTENSOR ? 0 : kPreColumns * D * 2;
    static constexpr int RING = TILES * TILE + SLOTS * QTILE;  // the ring of records is behind the tiles and the queries
    static constexpr int smem(int stages) { return RING + stages * STAGE + 1024; }  // 1024: alignment; and the plan
    // Columns of tensor memory of a slot: queries, scores (weights over them) twice, sums.
    static constexpr int QCOLS = QTENSOR ? D / 2 : 0, SLOT = QCOLS + 2 * kPreStep + D;
    static_assert(SLOTS * SLOT <= 512, "tensor memory");
};

using PreParams = SharedCall;

// The plan, in shared memory, by group.
struct PrePlan {
    int32_t *part0, *leader, *row0, *rows_end, *blocks, *parts, *each;  // each: steps of a part
    static __host__ __device__ size_t bytes(int groups) { return (size_t(groups) * 7 + 1) * 4; }
};

struct PrePart {
    int32_t leader, head, col0, cols;  // the sequence whose pages are read; first column of the tile, and columns of it
    int32_t row0;
    uint32_t begin, end, blocks;       // steps; blocks that are shared
    bool both;                         // the slots share the columns
};

__device__ __forceinline__ float pre_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pre_lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Bytes 0, 1 (HIGH: 2, 3) of w as float16 codes: 1024 + byte, minus 1152.
template <bool HIGH>
__device__ __forceinline__ uint32_t pre_codes(uint32_t w) {
    const uint32_t u = prmt(w, 0x64646464u, HIGH ? 0x4342u : 0x4140u);
    uint32_t h;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h) : "r"(u), "r"(0x64806480u));
    return h;
}
__device__ __forceinline__ uint4 pre_lds(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ void pre_sts(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void pre_sts(uint32_t at, uint32_t a, uint32_t b) {
    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(a), "r"(b) : "memory");
}

// ---- barriers --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Every wait ends: after so many tries, or when another one has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
#pragma unroll 1
    for (uint32_t i = 0; i < kPreTries; ++i) {
        uint32_t done;
        asm volatile(
            "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (done) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}
__device__ __forceinline__ void copy_record(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

// ---- tensor cores ------------------------------------------------------------------------------------------------------
// Rows of 128 bytes in groups of eight (1024 bytes), 16-byte pieces of a row exchanged by the row's place in its group.
// `at`: the address in shared memory, in units of 16 bytes.
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t at) {
    return uint64_t(at | 1u << 16) | uint64_t(1024 >> 4 | 1u << 14 | 2u << 29) << 32;
}
// float16 x float16 -> float32, 128 rows, n columns, both operands with k running fastest.
__host__ __device__ constexpr uint32_t product_kind(int n) { return 1u << 4 | uint32_t(n / 8) << 17 | uint32_t(128 / 16) << 24; }
__device__ __forceinline__ void tensor_product(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"(uint32_t(add))
        : "memory");
}
__device__ __forceinline__ void tensor_product(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"(uint32_t(add))
        : "memory");
}
__device__ __forceinline__ void tensor_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// One lane of a whole warp, always the same.  (The compiler knows it to be one: with `lane == 0` in its place each product is issued
// in a loop over the lanes that may be active, 140 cycles a product where it takes 45.)
__device__ __forceinline__ bool elected() {
    uint32_t is;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define TETRA_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define TETRA_W8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of the lane's row.
__device__ __forceinline__ void tensor_load(uint32_t at, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : TETRA_R8(r, 0), TETRA_R8(r, 8), TETRA_R8(r, 16), TETRA_R8(r, 24)
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::TETRA_W8(r, 0),
        TETRA_W8(r, 8), TETRA_W8(r, 16), TETRA_W8(r, 24), "r"(at)
        : "memory");
}
// 16 columns.
__device__ __forceinline__ void tensor_load16(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : TETRA_R8(r, 0), TETRA_R8(r, 8) : "r"(at) : "memory");
}
// 8 columns.
__device__ __forceinline__ void tensor_store8(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::TETRA_W8(r, 0), "r"(at) : "memory");
}
#undef TETRA_R8
#undef TETRA_W8

// ---- the plan ------------------------------------------------------------------------------------------------------------
struct PreGroup {
    uint32_t items, steps;
};
template <int D>
__device__ __forceinline__ PreGroup group_work(const PreParams& p, const PrePlan& plan, int g) {
    PreGroup w{0, 1};
    if (g < p.g.groups && plan.rows_end[g] > 0) {
        const uint32_t cols = uint32_t(plan.rows_end[g] - plan.row0[g]) * p.group;
        w.items = min((cols + pre_tile(D) - 1) / pre_tile(D) * p.c.kv_heads, 1u << 20);  // (that many have no place: no sum wraps)
        w.steps = (uint32_t(plan.blocks[g]) * kKvBlock + kPreStep - 1) / kPreStep;
    }
    return w;
}
// Parts of an item when none has more than `share` steps, all but the last of `each`.
__device__ __forceinline__ uint32_t pre_parts(uint32_t steps, uint32_t share, uint32_t& each) {
    each = steps;
    if (steps <= share) return 1;
    const uint32_t parts = (steps + share - 1) / share;
    each = (steps + parts - 1) / parts;
    return (steps + each - 1) / each;
}

// Every CTA finds out for itself how the work is cut.  The longest part decides, so the share of a part is the least with which
// there are no more parts than CTAs, or twice as many, whichever takes less: 32 shares are looked at at a time.  Returns the number of parts.
template <int D>
__device__ __forceinline__ uint32_t make_plan(const PreParams& p, const PrePlan& plan, uint32_t* total) {
    const int groups = p.g.groups, seqs = p.c.seqs, tid = threadIdx.x, lane = tid & 31;
    for (int g = tid; g < groups; g += kPreThreads) {
        plan.leader[g] = plan.row0[g] = INT_MAX;
        plan.rows_end[g] = plan.blocks[g] = 0;
    }
    // A sequence's rows and its group, 0 blocks if it does not take part.
    auto look = [&](int s, int& group, int& a, int& b) {
        const int before = __ldg(p.c.lengths + s);
        int first, last, which;
        group = group_of(p.g, seqs, s, first, last, which);
        const int blocks = shared_blocks(p.c, p.g, which);  // (loaded beside the others, whatever they say)
        p.c.rows_of(s, a, b);
        return group >= 0 && takes_part(first, last, blocks, a, b, before) ? blocks : 0;
    };
    int group = -1, a = 0, b = 0, blocks = 0;
    if (tid < seqs) blocks = look(tid, group, a, b);
    __syncthreads();
#pragma unroll 1
    for (int s = tid; s < seqs; s += kPreThreads) {
        if (s != tid) blocks = look(s, group, a, b);
        if (blocks > 0) {
            plan.blocks[group] = blocks;
            atomicMin(plan.leader + group, s);
            atomicMin(plan.row0 + group, a);
            atomicMax(plan.rows_end + group, b);
        }
    }
    __syncthreads();
    if (tid < 32) {
        const uint32_t G = gridDim.x;
        const PreGroup mine = group_work<D>(p, plan, lane);
        auto work_of = [&](int g) { return g == lane ? mine : group_work<D>(p, plan, g); };
        uint32_t items = 0, work = 0, longest = 1;
        for (int g = lane; g < groups; g += 32) {
            const PreGroup w = work_of(g);
            items += w.items;
            work += w.items * min(w.steps, 1u << 22);  // (looked at where items are few)
            longest = max(longest, w.steps);
        }
        items = __reduce_add_sync(0xFFFFFFFFu, items);
        work = __reduce_add_sync(0xFFFFFFFFu, work);
        longest = __reduce_max_sync(0xFFFFFFFFu, longest);
        uint32_t share = longest, cost = ~0u;
#pragma unroll 1
        for (uint32_t k = 1; k <= kPreWaves && items; ++k) {
            const uint32_t may = min(k * G, p.most);
            if (items > may || (k > 1 && (2 * items <= G || k * (1 + kPrePartCost) >= cost))) continue;
            uint32_t from = max(1u, (work + may - 1) / may), tried, fits;
            do {
                const uint32_t by = max(1u, from >> 4);
                tried = min(from + lane * by, longest);
                uint32_t need = 0;
                for (int g0 = 0; g0 < groups; g0 += 32) {
                    const PreGroup w = work_of(g0 + lane);
#pragma unroll 1
                    for (int g = 0; g < min(groups - g0, 32); ++g)
                        need += __shfl_sync(0xFFFFFFFFu, w.items, g) * ((__shfl_sync(0xFFFFFFFFu, w.steps, g) + tried - 1) / tried);
                }
                fits = __ballot_sync(0xFFFFFFFFu, need <= may);  // some does: an item in one part
                from += 32 * by;
            } while (fits == 0);
            tried = __shfl_sync(0xFFFFFFFFu, tried, __ffs(fits) - 1);
            if (k * (tried + kPrePartCost) < cost) cost = k * (tried + kPrePartCost), share = tried;
        }
        // A group whose parts have no place (which takes sequences that have rows in common) has no parts.
        uint32_t at = 0;
        for (int g0 = 0; g0 < groups; g0 += 32) {
            const int g = g0 + lane;
            const PreGroup w = work_of(g);
            uint32_t each = 1;
            const uint32_t parts = w.items ? pre_parts(w.steps, share, each) : 0u;
            uint32_t own = w.items * parts, sum = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= o) sum += v;
            }
            if (g < groups) {
                plan.part0[g] = int(min(at + sum - own, p.most));
                plan.parts[g] = at + sum <= p.most ? int(parts) : 0;
                plan.each[g] = int(each);
            }
            at += __shfl_sync(0xFFFFFFFFu, sum, 31);
        }
        if (lane == 0) *total = plan.part0[groups] = int(min(at, p.most));
    }
    __syncthreads();
    if (blockIdx.x == 0) {
#pragma unroll 1
        for (int s = tid; s < seqs; s += kPreThreads) {
            SharedSeq out = {};
            const int blocks = look(s, group, a, b);
            if (blocks > 0) {
                out.first = blocks;
                out.part0 = plan.part0[group];
                out.parts = plan.parts[group];
                out.row0 = plan.row0[group];
                out.cols = (plan.rows_end[group] - plan.row0[group]) * p.group;
                out.tiles = (out.cols + pre_tile(D) - 1) / pre_tile(D);
            }
            p.seqs[s] = out;
        }
    }
    return *total;
}

// Part number n of the plan; false: of a group that has none.
template <int D>
__device__ __forceinline__ bool part_of(const PreParams& p, const PrePlan& plan, uint32_t n, PrePart& q) {
    int lo = 0, hi = p.g.groups;
    while (hi - lo > 1) {  // the last group whose parts begin at or before n
        const int mid = (lo + hi) >> 1;
        if (uint32_t(plan.part0[mid]) <= n) lo = mid;
        else hi = mid;
    }
    const uint32_t parts = uint32_t(plan.parts[lo]);
    if (parts == 0) return false;
    const uint32_t local = n - uint32_t(plan.part0[lo]), item = parts == 1 ? local : local / parts, part = local - item * parts;
    const uint32_t cols = uint32_t(plan.rows_end[lo] - plan.row0[lo]) * p.group, tiles = (cols + pre_tile(D) - 1) / pre_tile(D);
    const uint32_t head = tiles == 1 ? item : item / tiles, steps = (uint32_t(plan.blocks[lo]) * kKvBlock + kPreStep - 1) / kPreStep, each = uint32_t(plan.each[lo]);
    q.leader = plan.leader[lo];
    q.head = int(head);
    q.col0 = int(item - head * tiles) * pre_tile(D);
    q.cols = min(int(cols) - q.col0, pre_tile(D));
    q.row0 = plan.row0[lo];
    q.blocks = uint32_t(plan.blocks[lo]);
    q.begin = part * each;
    q.end = min(steps, q.begin + each);
    q.both = pre_slots(D) == 2 && q.cols <= kPreColumns;
    return int(head) < p.c.kv_heads;
}

__device__ __forceinline__ uint64_t two_floats(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void two_floats(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
// Weights of a block of 16 tokens, two and two as float16; returns the sum of 2^(score - ref).  scale: s_K times the call's, s_V, log2 s_V, the
// most that the sum may come to; 0: no such block.
__device__ __forceinline__ float block_weights(const uint32_t* scores, const float4& scale, float ref, uint32_t* weights) {
    if (scale.w == 0.f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) weights[k] = 0u;
        return 0.f;
    }
    const uint64_t by = two_floats(scale.x, scale.x), from = two_floats(-ref, -ref), times = two_floats(scale.y, scale.y);
    uint64_t sum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        uint64_t x, e, w;
        float a, b;
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(two_floats(__uint_as_float(scores[2 * k]), __uint_as_float(scores[2 * k + 1]))), "l"(by), "l"(from));
        two_floats(x, a, b);
        e = two_floats(pre_ex2(a), pre_ex2(b));
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(sum) : "l"(sum), "l"(e));
        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(w) : "l"(e), "l"(times));
        two_floats(w, a, b);
        const __half2 h = __floats2half2_rn(a, b);
        weights[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    float a, b;
    two_floats(sum, a, b);
    return a + b;
}

template <int D>
__global__ void __launch_bounds__(kPreThreads, 1) k_kv_prefix(PreParams p) {
    using C = PreCfg<D>;
    constexpr int SLOTS = C::SLOTS, TILES = C::TILES, CHUNKS = D / 32;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t raw_full[8], raw_empty[8], tile_full[TILES], tile_empty[TILES], q_ready, q_seen, s_full[4], p_ready[4], o_done[4], scales_full[kPreScales],
        other_ready, other_free, drained;
    __shared__ __align__(16) float4 scales[kPreScales][kPreBlocks];  // s_K times the call's, s_V, log2 s_V (-60 at least), the most that weights may come to; 0: no such block
    __shared__ float2 other[kPreColumns];                            // of the slots that share columns: the second one's references and denominators
    __shared__ uint32_t placed[8], total, tensor_base;
    __shared__ int failed;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    const uint32_t stages = uint32_t(p.stages);
    if (threadIdx.x == 0) {
        failed = 0;
        for (uint32_t i = 0; i < stages; ++i) bar_init(smem_u32(raw_full + i), 1), bar_init(smem_u32(raw_empty + i), kPreConvert);
        for (int i = 0; i < TILES; ++i) bar_init(smem_u32(tile_full + i), kPreConvert), bar_init(smem_u32(tile_empty + i), SLOTS);
        bar_init(smem_u32(&q_ready), 4 * SLOTS), bar_init(smem_u32(&q_seen), SLOTS);
        for (int i = 0; i < 4; ++i) bar_init(smem_u32(p_ready + i), 4), bar_init(smem_u32(s_full + i), 1), bar_init(smem_u32(o_done + i), 1);
        for (int i = 0; i < kPreScales; ++i) bar_init(smem_u32(scales_full + i), 1);
        bar_init(smem_u32(&other_ready), 4), bar_init(smem_u32(&other_free), 4);
        bar_init(smem_u32(&drained), SLOTS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_release();
    // (Not ahead of the wait: what is waited for may want tensor memory itself.)
    if (warp == kPreMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tensor_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();

    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    PrePlan plan;
    {
        int32_t* at = reinterpret_cast<int32_t*>(raw + (base - smem_u32(raw)) + C::RING + p.stages * C::STAGE);
        const int n = p.g.groups;
        plan = PrePlan{at, at + n + 1, at + 2 * n + 1, at + 3 * n + 1, at + 4 * n + 1, at + 5 * n + 1, at + 6 * n + 1};
    }
    const uint32_t parts = make_plan<D>(p, plan, &total);  // (its barriers are also those behind what is above)
    fence_after();
    if (parts <= blockIdx.x) {
        if (warp == kPreMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tensor_base) : "memory");
        return;
    }

    const uint32_t tensor = tensor_base;
    volatile int* gave_up = &failed;
    const uint32_t queries = base + TILES * C::TILE, ring = base + C::RING;
    uint32_t n0 = 0;  // steps before the part

    if (warp == kPreCopyWarp) {
        // ---- records into the ring: lane l looks up the place of the l-th of the next 32, a batch ahead
        bool ok = true;
        uint32_t stage = 0, turn = 0, issued = 0;
        for (uint32_t at = blockIdx.x; ok && at < parts; at += gridDim.x) {
            PrePart q;
            if (!part_of<D>(p, plan, at, q)) continue;
            const uint32_t begin = q.begin, last = q.end, end = min(last * kPreBlocks, q.blocks);
            auto look = [&](uint32_t first) { return first + lane < end ? p.c.template record<D>(q.leader, first + lane, q.head) : nullptr; };
            const unsigned char *now = look(begin * kPreBlocks), *next = look(begin * kPreBlocks + 32);
            for (uint32_t half = begin; half < last; ++half) {
                const uint32_t k = (half - begin) * kPreBlocks & 31u;
                if (k == 0 && half > begin) now = next, next = look(half * kPreBlocks + 32);
                ok = bar_wait(smem_u32(raw_empty + stage), (turn & 1u) ^ 1u, gave_up);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                const unsigned char* from = reinterpret_cast<const unsigned char*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<uint64_t>(now), k + (lane & 3)));
                const uint32_t there = __ballot_sync(0xFFFFFFFFu, lane < kPreBlocks && from != nullptr);
                const uint32_t bar = smem_u32(raw_full + stage);
                if (lane == 0) {
                    placed[stage] = there;
                    if (there) bar_expect(bar, __popc(there) * C::REC);
                    else bar_arrive(bar);
                }
                __syncwarp();
                if (there >> lane & 1u) copy_record(ring + stage * C::STAGE + lane * C::REC, from, C::REC, bar);
                ++issued;
                if (++stage == stages) stage = 0, ++turn;
            }
        }
        // Nothing is in flight when the CTA ends, whoever gave up: the last copies into each stage have arrived.
        int none = 0;
        for (uint32_t back = 0; back < stages && back < issued; ++back) {
            if (stage == 0) stage = stages, --turn;
            bar_wait(smem_u32(raw_full + --stage), turn & 1u, &none);
        }
    } else if (warp >= kPreConvertAt && warp < kPreCopyWarp) {
        // ---- bytes to operands
        const int w = warp - kPreConvertAt;
        bool ok = true;
        uint32_t stage = 0, turn = 0, tile = 0, tile_turn = 0, n = 0;
        // Keys: a unit of 16 bytes is 8 dims (tt of a chunk of 32) of tokens g and g + 8.  A quarter of the warp takes tokens g, g ^ 1 of
        // two chunks, which no two lanes read or write through the same bank.
        const int odd = lane >> 2 & 1, tt = lane & 3;
        // Values: a unit is dims 4 dq .. + 3 of tokens 2 tq, 2 tq + 1, and 8 on; half a warp takes two blocks.
        const int vblock = (w >> 1) * 2 + (lane >> 3 & 1), e = lane >> 2 & 1, tq = lane & 3;
        for (uint32_t at = blockIdx.x; ok && at < parts; at += gridDim.x) {
            PrePart q;
            if (!part_of<D>(p, plan, at, q)) continue;
            for (uint32_t step = q.begin; ok && step < q.end; ++step) {
                const uint32_t key_tile = tile, key_turn = tile_turn;
                if (++tile == TILES) tile = 0, ++tile_turn;
                const uint32_t value_tile = tile, value_turn = tile_turn;
                if (++tile == TILES) tile = 0, ++tile_turn;
                const uint32_t from = ring + stage * C::STAGE;
                ok = bar_wait(smem_u32(raw_full + stage), turn & 1u, gave_up) && bar_wait(smem_u32(tile_empty + key_tile), (key_turn & 1u) ^ 1u, gave_up);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                if (w == 0) {
                    if (lane < kPreBlocks) {
                        const bool is = placed[stage] >> lane & 1u;
                        const uint4 raw4 = pre_lds(from + lane * C::REC + 32 * D);
                        const float vs = __uint_as_float(raw4.y);
                        float lv = pre_lg2(vs);
                        lv = lv < kPreLeastLog ? kPreLeastLog : lv;  // NaN stays
                        // The most that a block's 2^(score - reference) may come to, by the same logarithm as the reference; never zero.
                        const float most = fmaxf(pre_ex2(kPreHigh - lv), FLT_MIN);
                        scales[n % kPreScales][lane] = is ? make_float4(__uint_as_float(raw4.x) * p.scale, vs, lv, most) : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(scales_full + n % kPreScales));
                }
                {
                    const uint32_t to = base + key_tile * C::TILE;
#pragma unroll
                    for (int pair = 0; pair < CHUNKS / 2; ++pair) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int g = (2 * (lane >> 3) + h) ^ odd, row = w * kKvBlock + (g >> 1) * 4 + (g & 1);
                            const uint4 u = pre_lds(from + w * C::REC + (2 * pair + odd) * 512 + (g * 4 + tt) * 16);
                            const uint32_t chunk = odd * 4 + tt, line = to + pair * (kPreStep * 128) + row * 128;
                            pre_sts(line + ((chunk ^ (row & 7)) << 4), pre_codes<false>(u.x), pre_codes<true>(u.x), pre_codes<false>(u.y), pre_codes<true>(u.y));
                            pre_sts(line + 256 + ((chunk ^ ((row + 2) & 7)) << 4), pre_codes<false>(u.z), pre_codes<true>(u.z), pre_codes<false>(u.w), pre_codes<true>(u.w));
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(tile_full + key_tile));
                ok = bar_wait(smem_u32(tile_empty + value_tile), (value_turn & 1u) ^ 1u, gave_up);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                {
                    const uint32_t to = base + value_tile * C::TILE;
#pragma unroll
                    for (int it = 0; it < D / 32; ++it) {
                        const int chunk = (w & 1) + 2 * (it >> 1), dq = ((it & 1) * 2 + (lane >> 4)) * 2 + e;
                        const uint4 u = pre_lds(from + vblock * C::REC + 16 * D + chunk * 512 + (dq * 4 + tq) * 16);
                        const uint32_t word[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int d = chunk * 32 + dq * 4 + i;
                            pre_sts(to + d * 128 + (((2 * vblock + (tq >> 1)) ^ (d & 7)) << 4) + (tq & 1) * 8, pre_codes<false>(word[i]), pre_codes<true>(word[i]));
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    bar_arrive(smem_u32(tile_full + value_tile));
                    bar_arrive(smem_u32(raw_empty + stage));
                }
                if (++stage == stages) stage = 0, ++turn;
                ++n;
            }
        }
    } else if (warp >= kPreMmaWarp && warp < kPreMmaWarp + SLOTS) {
        // ---- products, issued by one thread a slot.  A job is a step of the slot's.  Its scores are issued one job ahead of its weights'
        // products, into the place that the last job but one had, whose products are waited for (products with different results are in no
        // order).  Each place has barriers of its own: a barrier tells of its last phase only, and the products of two jobs may both be
        // on their way.  For the same reason each slot waits for every step's tiles, its own or not, and for every part's queries,
        // which are announced by all warps of the weights, whoever brings them, and not again before both slots have said that they
        // have seen them: a part of one step that the slots share is no work for the second one's weights, which would be two parts
        // ahead otherwise.
        const uint32_t slot = warp - kPreMmaWarp;
        bool ok = true;
        uint32_t own = 0, q_parts = 0;  // jobs so far
        const uint32_t tiles = (base & 0x3FFFFu) >> 4, to_slot = tensor + slot * C::SLOT;
        constexpr uint32_t PAIRS = TILES / 2;  // a step's keys are tile 2 (step % PAIRS), its values the next one
        auto full = [&](uint32_t step, uint32_t value) { ok = ok && bar_wait(smem_u32(tile_full + 2 * (step % PAIRS) + value), step / PAIRS & 1u, gave_up); };
        for (uint32_t at = blockIdx.x; ok && at < parts; at += gridDim.x) {
            PrePart q;
            if (!part_of<D>(p, plan, at, q)) continue;
            const uint32_t steps = q.end - q.begin, by = q.both ? 2u : 1u, first = q.both ? slot : 0u;
            const uint32_t queries_at = ((queries & 0x3FFFFu) + (q.both ? 0u : slot * C::QTILE)) >> 4;
            ok = bar_wait(smem_u32(&q_ready), q_parts & 1u, gave_up);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            if (lane == 0) bar_arrive(smem_u32(&q_seen));
            auto scores = [&](uint32_t i, uint32_t job) {
                const uint32_t step = n0 + i, pair = step % PAIRS, place = job & 1u;
                if (job >= 2) ok = ok && bar_wait(smem_u32(o_done + slot * 2) + place * 8, (job >> 1) + 1 & 1u, gave_up);
                full(step, 0);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) return;
                fence_after();
                const uint32_t to = to_slot + C::QCOLS + place * kPreStep, keys = tiles + (2 * pair * C::TILE >> 4);
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t b = tile_descriptor(keys + ((k / 4 * (kPreStep * 128) + k % 4 * 32) >> 4));
                        if constexpr (C::QTENSOR) tensor_product(to, to_slot + k * 8, b, product_kind(kPreStep), k > 0);
                        else tensor_product(to, tile_descriptor(queries_at + ((k / 4 * (kPreColumns * 128) + k % 4 * 32) >> 4)), b, product_kind(kPreStep), k > 0);
                    }
                    tensor_commit(smem_u32(s_full + slot * 2) + place * 8);
                    tensor_commit(smem_u32(tile_empty) + 16 * pair);
                }
                __syncwarp();
            };
            auto sums = [&](uint32_t i, uint32_t job) {
                const uint32_t step = n0 + i, pair = step % PAIRS, place = job & 1u;
                full(step, 1);
                ok = ok && bar_wait(smem_u32(p_ready + slot * 2) + place * 8, job >> 1 & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) return;
                fence_after();
                const uint32_t to = to_slot + C::QCOLS + 2 * kPreStep, a = to_slot + C::QCOLS + place * kPreStep, values = tiles + ((2 * pair + 1) * C::TILE >> 4);
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < kPreStep / 16; ++k) tensor_product(to, a + k * 8, tile_descriptor(values + (k * 32 >> 4)), product_kind(D), i > first || k > 0);
                    tensor_commit(smem_u32(o_done + slot * 2) + place * 8);
                    tensor_commit(smem_u32(tile_empty + 1) + 16 * pair);
                }
                __syncwarp();
            };
            auto others = [&](uint32_t i) {  // a step that is the other slot's
                for (uint32_t value = 0; value < 2; ++value) {
                    full(n0 + i, value);
                    if (ok && lane == 0) bar_arrive(smem_u32(tile_empty + 2 * ((n0 + i) % PAIRS) + value));
                }
                ok = __all_sync(0xFFFFFFFFu, ok);
            };
            if (q.both && slot == 1) others(0);
            if (ok && first < steps) scores(first, own);
            for (uint32_t i = first; ok && i < steps; i += by, ++own) {
                if (q.both && i + 1 < steps) others(i + 1);
                if (ok && i + by < steps) scores(i + by, own + 1);
                if (ok) sums(i, own);
            }
            n0 += steps;
            ++q_parts;
        }
        // What was issued has ended when the tensor memory is given back.
        if (elected()) tensor_commit(smem_u32(&drained));
        int none = 0;
        bar_wait(smem_u32(&drained), 0, &none);
        __syncwarp();
    } else if (warp < 4 * SLOTS) {
        // ---- weights: a thread a column
        const uint32_t slot = warp >> 2, column = threadIdx.x & 127;
        const uint32_t at_q = tensor + slot * C::SLOT + ((warp & 3u) << 21), at_scores = at_q + C::QCOLS, at_o = at_scores + 2 * kPreStep;  // lanes from bit 16 on
        uint32_t jobs = 0, shared_parts = 0, freed = 0, q_parts = 0;
        bool ok = true;
        for (uint32_t at = blockIdx.x; ok && at < parts; at += gridDim.x) {
            PrePart q;
            if (!part_of<D>(p, plan, at, q)) continue;
            const uint32_t steps = q.end - q.begin, first = q.both ? slot : 0u, by = q.both ? 2u : 1u;
            const int col = q.col0 + (q.both || SLOTS == 1 ? 0 : int(slot) * kPreColumns) + int(column);
            const bool live = col < q.col0 + q.cols, mine = !q.both || slot == 0;  // whose queries these are, and who leaves the piece
            float ref = kPreNoRef, sum = 0.f;
            if (mine) {
                const uint32_t row = live ? uint32_t(col) / uint32_t(p.group) : 0u, h = live ? uint32_t(col) - row * p.group : 0u;
                const uint4* src = reinterpret_cast<const uint4*>(p.q + int64_t(q.row0 + row) * p.q_stride + (int64_t(q.head) * p.group + h) * D);
                if constexpr (C::QTENSOR) {
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        uint32_t r[32];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint4 v = live ? __ldg(src + j * 8 + i) : make_uint4(0, 0, 0, 0);
                            r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
                        }
                        tensor_store(at_q + j * 32, r);
                    }
                } else {
                    // Lanes read a column's 16 bytes side by side, several columns at a time.
                    constexpr int LANES = D / 8, COLS = 32 / LANES, LOADS = 32 / COLS;
                    const uint32_t chunk = lane % LANES;
                    const uint64_t mine_at = live ? reinterpret_cast<uint64_t>(src) : 0;
                    uint4 v[LOADS];
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) {
                        const uint64_t from = __shfl_sync(0xFFFFFFFFu, mine_at, i * COLS + lane / LANES);
                        v[i] = from ? __ldg(reinterpret_cast<const uint4*>(from) + chunk) : make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) {
                        const uint32_t to = (warp & 3) * 32 + i * COLS + lane / LANES;
                        pre_sts(queries + slot * C::QTILE + chunk / 8 * (kPreColumns * 128) + to * 128 + ((chunk % 8 ^ to % 8) << 4), v[i].x, v[i].y, v[i].z, v[i].w);
                    }
                }
                if constexpr (C::QTENSOR) {
                    wait_stores();
                    fence_before();
                } else {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
            }
            if (q_parts > 0) {  // the last part's have been seen
                ok = bar_wait(smem_u32(&q_seen), (q_parts - 1) & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
            }
            ++q_parts;
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&q_ready));
            if (slot == 1 && freed < shared_parts) {  // the first slot has yet to read the sums of the last part that they shared
                ok = bar_wait(smem_u32(&other_free), (shared_parts - 1) & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                freed = shared_parts;
            }
            for (uint32_t i = first; ok && i < steps; i += by, ++jobs) {
                const uint32_t which = jobs & 1u, at_s = at_scores + which * kPreStep, n = n0 + i;
                ok = bar_wait(smem_u32(scales_full + n % kPreScales), n / kPreScales & 1u, gave_up) && bar_wait(smem_u32(s_full + slot * 2 + which), jobs >> 1 & 1u, gave_up);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                fence_after();
                uint32_t r[kPreStep], w[kPreStep / 2];
                tensor_load(at_s, r);
                tensor_load(at_s + 32, r + 32);
                const float4* c = scales[n % kPreScales];
                wait_loads();
                // Weights next to the reference so far.  A block's weights that with s_V are more than 2^15 together (or infinite ones:
                // the first of a column) call for a new one; as long as none does, no maximum is looked for.  An s_V below 2^-60
                // counts as that: the weights of values that are zero, or next to it, stay within what the denominator holds, 2^75 a
                // block.
                float now = 0.f;
                bool over = !(fabsf(ref) <= kPreLargeRef);  // a column that has seen nothing, too
                if (!__all_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                    for (int b = 0; b < kPreBlocks; ++b) {
                        const float4 by = c[b];
                        const float one = block_weights(r + 16 * b, by, ref, w + 8 * b);
                        over |= !(one <= by.w);
                        now += one;
                    }
                }
                if (__any_sync(0xFFFFFFFFu, over)) {  // from tensor memory again, a block at a time: little code, which is cold the first time
                    float next = ref;
#pragma unroll 1
                    for (int b = 0; b < kPreBlocks; ++b) {
                        uint32_t x[16];
                        tensor_load16(at_s + 16 * b, x);
                        wait_loads();
                        const float4 by = c[b];
                        float top = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 16; ++k) top = fmaxf(top, __uint_as_float(x[k]) * by.x);
                        if (by.w == 0.f) top = -INFINITY;
                        float want = rintf(top + by.z - kPreBase);
                        if (top - want > kPreHigh - by.z) want = top;  // a step of so large scores is more than the room there is
                        if (over && want > next) next = want;
                    }
                    const float f = pre_ex2(ref - next);  // a power of two
                    ref = next;
                    sum *= f;
                    now = 0.f;
#pragma unroll 1
                    for (int b = 0; b < kPreBlocks; ++b) {  // (weights are behind or over the scores of their block)
                        uint32_t x[16];
                        tensor_load16(at_s + 16 * b, x);
                        wait_loads();
                        float4 by = c[b];
                        const bool large = !(fabsf(ref) <= kPreLargeRef);
                        const float first_by = large ? by.x : 1.f;
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__fmul_rn(__uint_as_float(x[k]), first_by));
                        by.x = large ? 1.f : by.x;
                        now += block_weights(x, by, ref, w);
                        tensor_store8(at_s + 8 * b, w);
                    }
                    if (i > first) {
                        ok = ok && bar_wait(smem_u32(o_done + slot * 2 + (which ^ 1u)), (jobs - 1) >> 1 & 1u, gave_up);
                        fence_after();
#pragma unroll 1
                        for (int j = 0; j < D; j += 32) {
                            tensor_load(at_o + j, r);
                            wait_loads();
#pragma unroll
                            for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * f);
                            tensor_store(at_o + j, r);
                        }
                    }
                } else {
                    tensor_store(at_s, w);
                }
                sum += now;
                wait_stores();
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(p_ready + slot * 2 + which));
            }
            // The piece: sums, then references and denominators.
            float* piece = p.pieces + (size_t(at) * SLOTS + (mine ? slot : 0u)) * pre_piece(D);
            if (ok && first < steps) {
                ok = bar_wait(smem_u32(o_done + slot * 2 + ((jobs - 1) & 1u)), (jobs - 1) >> 1 & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (ok) fence_after();
            }
            if (!mine) {
                other[column] = make_float2(ref, ok ? sum : __uint_as_float(0x7FC00000u));
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&other_ready));
            } else if (ok) {
                float2 end{kPreNoRef, 0.f};
                if (q.both) {
                    ok = bar_wait(smem_u32(&other_ready), shared_parts & 1u, gave_up);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    fence_after();
                    end = other[column];
                }
                const float top = fmaxf(ref, end.x), f0 = pre_ex2(ref - top), f1 = pre_ex2(end.x - top);
                const bool two = q.both && steps > 1;  // else the other slot has nothing
                sum = two ? fmaf(sum, f0, end.y * f1) : sum;
                ref = two ? top : ref;
                uint32_t o[2][16], u[2][16];  // 16 dims are on their way while the 16 before are stored
                auto load = [&](int which, int j) {
                    tensor_load16(at_o + j, o[which]);
                    if (two) tensor_load16(at_o + C::SLOT + j, u[which]);
                };
                auto store = [&](int which, int j) {
                    if (two) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[which][k] = __float_as_uint(fmaf(__uint_as_float(o[which][k]), f0, __uint_as_float(u[which][k]) * f1));
                    }
                    if (live) {
#pragma unroll
                        for (int k = 0; k < 16; k += 8)
                            asm volatile("st.global.cg.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(piece + column * D + j + k), "r"(o[which][k]), "r"(o[which][k + 1]),
                                         "r"(o[which][k + 2]), "r"(o[which][k + 3]), "r"(o[which][k + 4]), "r"(o[which][k + 5]), "r"(o[which][k + 6]), "r"(o[which][k + 7])
                                         : "memory");
                    }
                };
                if (ok) load(0, 0);
#pragma unroll 1
                for (int j = 0; ok && j < D; j += 32) {
                    wait_loads();
                    load(1, j + 16);
                    store(0, j);
                    wait_loads();
                    if (j + 32 < D) load(0, j + 32);
                    store(1, j + 16);
                }
                fence_before();
                if (q.both) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&other_free));
                }
            }
            if (mine && live) __stcg(reinterpret_cast<float2*>(piece + kPreColumns * D) + column, make_float2(ref, ok ? sum : __uint_as_float(0x7FC00000u)));
            n0 += steps;
            shared_parts += q.both;
        }
        // A wait that gave up: all that the CTA had still to do becomes NaN.
        if (!ok) {
            for (uint32_t at = blockIdx.x; at < parts; at += gridDim.x) {
                float* piece = p.pieces + (size_t(at) * SLOTS + slot) * pre_piece(D);
                __stcg(reinterpret_cast<float2*>(piece + kPreColumns * D) + column, make_float2(0.f, __uint_as_float(0x7FC00000u)));
            }
        }
    }
    __syncthreads();
    if (warp == kPreMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tensor) : "memory");
}

// A column's sums: of its own tokens and of its pieces, in this order.  A CTA has four columns of a row, two warps a column, which take every
// other piece and have all of theirs on the way at once (one warp and eight at a time: 14 us where 18 pieces of 2048 columns take 6).
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinColumns = kJoinWarps / 2;

// Four floats, or the two that there are.  (Volatile: these loads stay where they are, side by side.)
template <int E>
__device__ __forceinline__ void load_four(const float* from, float* to) {
    if constexpr (E == 2) asm volatile("ld.global.cg.v2.f32 {%0,%1}, [%2];" : "=f"(to[0]), "=f"(to[1]) : "l"(from));
    else asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(to[0]), "=f"(to[1]), "=f"(to[2]), "=f"(to[3]) : "l"(from));
}
template <int D>
__global__ void __launch_bounds__(kJoinThreads) k_kv_join(PreParams p) {
    constexpr int E = D / 32, BATCH = D == 256 ? 8 : 12;  // dims a lane; pieces of a warp that are on the way
    __shared__ float halves[kJoinColumns][D + 2];
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0), column = warp >> 1, second = warp & 1;
    const int heads = p.c.kv_heads * p.group, h = blockIdx.y * kJoinColumns + column, r = blockIdx.x;
    // What came before the three kernels is complete (each starts behind the one before it has waited).
    int a = 0, b = 0;
    const int s = sequence_of(p.c, r, lane, a, b);
    pdl_wait();
    pdl_release();
    if (s < 0) return;
    const uint4 s0 = __ldcg(reinterpret_cast<const uint4*>(p.seqs + s)), s1 = __ldcg(reinterpret_cast<const uint4*>(p.seqs + s) + 1);
    const uint4 o = p.runs ? __ldcg(reinterpret_cast<const uint4*>(p.owns + s)) : make_uint4(0, 1, 0, 0);
    if (!p.runs && s0.x == 0) return;  // stored already
    const bool is = h < heads;
    float v[E], ref = kPreNoRef, sum = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = 0.f;
    const int64_t row = int64_t(r) * heads + h;
    if (is) {
        // Its own pieces, then those of the tokens that it shares.
        constexpr uint32_t TILE = pre_tile(D);
        const uint32_t head = uint32_t(h) / uint32_t(p.group), in_group = uint32_t(h) - head * p.group;
        const uint32_t mine_at = uint32_t(r - a) * p.group + in_group, own_count = o.y;
        const int64_t first_own = p.runs ? (int64_t(o.x) + (int64_t(head) * o.z + mine_at / 8) * own_count) * 8 + mine_at % 8 : row;
        const float *own = p.own + first_own * D + lane * E, *own_ends = p.own + p.own_ends + first_own * 2;
        const uint32_t at = uint32_t(r - int(s1.x)) * p.group + in_group, tile = at / TILE, in = at % TILE;
        const bool both = pre_slots(D) == 2 && s1.y - tile * TILE <= kPreColumns;
        const size_t piece = size_t(pre_piece(D)), step = piece * pre_slots(D);
        const float* from = p.pieces + (size_t(s0.y) + (size_t(head) * s0.w + tile) * s0.z) * step + (both ? 0 : in / kPreColumns) * piece;
        const float* ends = from + kPreColumns * D + in % kPreColumns * 2;
        from += in % kPreColumns * D + lane * E;
        const int count = int(own_count + (s0.x ? s0.z : 0u));
        auto sums_at = [&](int i) { return i < int(own_count) ? own + size_t(i) * 8 * D : from + size_t(i - int(own_count)) * step; };
        auto ends_at = [&](int i) { return i < int(own_count) ? own_ends + size_t(i) * 16 : ends + size_t(i - int(own_count)) * step; };
#pragma unroll 1
        for (int i = second; i < count; i += 2 * BATCH) {
            float x[BATCH][E];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float* to = sums_at(min(i + 2 * k, count - 1));
#pragma unroll
                for (int j = 0; j < E; j += 4) load_four<E>(to + j, x[k] + j);
            }
            const bool mine = lane < BATCH && i + 2 * lane < count;
            const float2 end = mine ? __ldcg(reinterpret_cast<const float2*>(ends_at(i + 2 * lane))) : make_float2(kPreNoRef, 0.f);
            // A denominator of zero: nothing seen.
            const float own_ref = end.y != 0.f ? end.x : kPreNoRef;
            const uint32_t order = __float_as_uint(own_ref) ^ (uint32_t(int32_t(__float_as_uint(own_ref)) >> 31) | 0x80000000u);
            const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, order);
            const float now = fmaxf(ref, __uint_as_float(most & 0x80000000u ? most ^ 0x80000000u : ~most));
            const float f = pre_ex2(ref - now), g = end.y != 0.f ? pre_ex2(end.x - now) : 0.f;
            sum *= f;
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] *= f;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float by = __shfl_sync(0xFFFFFFFFu, g, k), d = __shfl_sync(0xFFFFFFFFu, end.y, k);
                sum = d != 0.f ? fmaf(d, by, sum) : sum;
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = d != 0.f ? fmaf(x[k][j], by, v[j]) : v[j];
            }
            ref = now;
        }
        if (second) {
#pragma unroll
            for (int k = 0; k < E; ++k) halves[column][lane * E + k] = v[k];
            if (lane == 0) halves[column][D] = ref, halves[column][D + 1] = sum;
        }
    }
    __syncthreads();
    if (!is || second) return;
    const float r1 = halves[column][D], u1 = halves[column][D + 1];
    if (u1 != 0.f) {
        const float now = fmaxf(ref, r1), f0 = pre_ex2(ref - now), f1 = pre_ex2(r1 - now);
        sum = fmaf(u1, f1, sum * f0);
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = fmaf(halves[column][lane * E + k], f1, v[k] * f0);
    }
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    __half* out = p.out + row * D + lane * E;
#pragma unroll
    for (int k = 0; k < E; k += 2) *reinterpret_cast<__half2*>(out + k) = __floats2half2_rn(v[k] * by, v[k + 1] * by);
}

template <int D>
cudaError_t launch_prefix_for(PreParams& p, int sms, cudaStream_t s) {
    using C = PreCfg<D>;
    static PerDeviceOnce once;  // per instantiation
    const cudaError_t e = once.run([] { return cudaFuncSetAttribute(k_kv_prefix<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPreSmem); });
    if (e != cudaSuccess) return e;
    const size_t plan = PrePlan::bytes(p.g.groups);
    static_assert(C::smem(2) + (TETRA_KV_MAX_SEQS * 7 + 1) * 4 <= kPreSmem, "two stages and the largest plan");
    p.stages = 2;
    while (p.stages < 6 && C::smem(p.stages + 1) + plan <= size_t(kPreSmem)) ++p.stages;
    return launch_pdl(k_kv_prefix<D>, sms < kPreMostCtas ? sms : kPreMostCtas, kPreThreads, C::smem(p.stages) + plan, s, p);
}
template <int D>
cudaError_t launch_join_for(const PreParams& p, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(p.c.rows), unsigned((p.c.kv_heads * p.group + kJoinColumns - 1) / kJoinColumns));
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_kv_join<D>, p);
}

}  // namespace

cudaError_t launch_prefix(SharedCall& p, int head_dim, int sms, cudaStream_t s) {
    return head_dim == 64 ? launch_prefix_for<64>(p, sms, s) : head_dim == 128 ? launch_prefix_for<128>(p, sms, s) : launch_prefix_for<256>(p, sms, s);
}
cudaError_t launch_join(const SharedCall& p, int head_dim, cudaStream_t s) {
    return head_dim == 64 ? launch_join_for<64>(p, s) : head_dim == 128 ? launch_join_for<128>(p, s) : launch_join_for<256>(p, s);
}

}  // namespace tetra
