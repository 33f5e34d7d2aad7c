// Attention of a step's rows over the 8-bit paged cache (tetra_kv_attend).
//
// A step has one or a few rows a sequence and reads each sequence's keys and values once: 2 D bytes a token and kv head
// against 4 D multiply-adds for each query head of the group, so HBM bounds it and the arrangement serves the stream.
//
// Work.  An item is (sequence, kv head, chunk of 8 NT columns); a column is one (row, query head of the group).  The lengths are
// on the device and change from step to step of a captured graph, so every CTA of a persistent grid finds its work from
// them: one part of one item where items are few, so many parts each that all are of about the same size; a contiguous
// range of the blocks of all items where they are many; and where they are many and very short, a warp takes an item.  Of a
// CTA's part of an item the eight warps take every eighth record; each warp streams its records through a cp.async ring of its
// own that goes on over the ends of items.  A lane copies the very bytes that it will use, so nothing but a warp-wide fence
// stands between a copy and its use.  The warps' sums meet in shared memory; of an item that several CTAs share each leaves a piece in
// the workspace, and the CTA that finds the others there adds them in order of the CTAs.  Nothing waits for another CTA.
//
// Arithmetic.  S^T = K Q^T and O^T = V^T P^T by mma.sync m16n8k16: tokens, then dims, fill the 16 rows and up to eight
// columns of a group the 8 columns, where Q K^T would leave 12 of 16 rows empty.  (tcgen05 wants 64 or 128 rows of one
// operand from shared memory as they are; these are bytes that have to become float16 in registers first, and the tensor
// pipe is mostly idle as it is.)  A byte u becomes the float16 1024 + u by a permutation and code = u - 128 by one
// subtraction, both exact, so scores are exact products summed in float32 times s_K.  The weights enter as
// float16(2^(score + log2 s_V - m)), m a running reference such that the largest lies between 2^7 and 2^15: relative to the
// largest weight TIMES SCALE of V, not the largest weight, so that a block of large values keeps no block of small ones
// that is attended to from its bits, and 2^-32 of the largest is still seen.  The denominator sums 2^(score - m) in float32.
// m moves only when a weight would pass 2^15: a vote per block, a reduction when it does.
//
// SHARED: the second kernel of tetra_kv_attend_shared.  The first blocks of a sequence that shares them with others are k_kv_prefix's:
// here they are not read, and the columns' sums are left for k_kv_join.  As that adds pieces anyway, items of eight columns are cut
// into runs of blocks, a warp's each, and no warp waits for another (64 sequences of 100 to 1024 tokens of their own: 15 us, 10 of
// them for 85 MB that come from L2; 33 where CTAs have ranges of units and merge at the end of each item).
#include <cfloat>
#include <cmath>

#include "kv_shared.cuh"

namespace tetra {
namespace {

constexpr int kAttThreads = 256, kAttWarps = kAttThreads / 32;
constexpr uint32_t kAttLeastUnits = 4;     // of a CTA: what sharing an item costs is worth some work
constexpr int kAttSegs = 32;              // parts of items that a CTA looks up at a time
constexpr int kAttMaxCtas = 384;          // of a launch: pieces in the workspace
constexpr int kAttBatch = 8;               // pieces that are loaded at a time
constexpr float kNoRef = -FLT_MAX;        // reference of a column that has seen nothing: below every finite score
constexpr float kLeastLog = -60.f;        // log2 of the least s_V that counts: 127 * 2^-60 is zero in float16
constexpr float kHigh = 15.f, kBase = 7.f; // a weight reaches 2^kHigh at most, a new reference puts the largest at 2^kBase

template <int D, int NT>
struct AttCfg {
    static constexpr int REC = kv_record_bytes(D);
    static constexpr int CHUNKS = D / 32;                      // 512-byte chunks of the keys, and of the values
    static constexpr int FRAGS = NT * D / 16;                  // accumulators, four floats a lane each
    static constexpr int CTAS = D == 256 || (D == 128 && NT == 4) ? 1 : 2;  // of an SM
    static constexpr int EACH = CTAS == 1 ? 2 : 1;             // of them that a warp adds at a time
    static constexpr int ROUND = FRAGS < EACH * kAttWarps ? FRAGS : EACH * kAttWarps;
    static constexpr int TURNS = (FRAGS + kAttWarps - 1) / kAttWarps;  // of them that are a warp's
    static constexpr int STAGES = D == 64 || CTAS == 1 && D == 128 ? 3 : 2;
    static constexpr int RING = kAttWarps * STAGES * REC;
    static constexpr int MERGE = kAttWarps * 512 * (ROUND + NT);
    static constexpr int QBYTES = NT > 1 ? NT * CHUNKS * 512 : 0;
    static constexpr int PIECE = 32 * FRAGS * 4 + NT * 16;     // floats of a piece in the workspace: accumulators; references and sums
    static constexpr int SMEM = RING + MERGE + QBYTES;          // and 4 bytes a sequence
};

// A CTA's part of an item.
struct Seg {
    int32_t seq, head;
    int32_t row0;          // first row of the sequence
    int32_t col0, cols;    // the item's first column, and the sequence's columns
    uint32_t r0, r1;       // blocks, of those that the item's last row sees (SHARED: behind the shared ones)
    int32_t first, last;   // CTAs that the item begins and ends in
    int32_t before;        // tokens before the step
    bool joined;           // SHARED: what is stored are sums, which others are added to
};

struct AttParams {
    KvCache c;
    const __half* q;
    __half* out;
    int64_t q_stride;
    float scale;           // times log2 e
    int32_t group;
    int32_t unit_shift;    // blocks of a unit: 8 << unit_shift
    // A CTA may be an item's last and the next one's first: what it keeps for either is apart (second: of the item that begins in it).
    float* pieces;         // [CTA][4][PIECE]: pieces, then groups' sums, two each
    uint32_t* arrived;     // [3][CTA]: pieces of the groups that begin in this CTA, two; groups of the item that begins in it
    SharedGroups shared;      // SHARED
    float* own;               // SHARED: [row][head][D] sums and, behind them, [row][head][2] references and denominators
    int64_t own_ends;         // where these begin
    OwnSeq* owns;             // SHARED, of eight columns: by sequence, which runs it has; then `own` is [run][8][D]
    uint32_t runs_most;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Bytes 0, 1 (HIGH: 2, 3) of w as float16 codes.
template <bool HIGH>
__device__ __forceinline__ uint32_t codes_of(uint32_t w) {
    const uint32_t u = prmt(w, 0x64646464u, HIGH ? 0x4342u : 0x4140u);  // 1024 + byte
    uint32_t h;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h) : "r"(u), "r"(0x64806480u));  // 1152 = 1024 + 128
    return h;
}
__device__ __forceinline__ uint4 lds_uint4(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// a / b, without a division where the quotient is plain (which it mostly is: one row, one chunk, one part).
__device__ __forceinline__ uint32_t quotient(uint32_t a, uint32_t b) { return a < b ? 0u : b == 1u ? a : a / b; }

// What a sequence asks for: its items, and units an item (one at least, so that an item without a token is somebody's
// work: its rows are zero).
struct Work {
    int32_t row0, rows, before;
    uint32_t chunks, blocks, units;
    uint32_t first;  // SHARED: blocks that are not read here
    bool joined;
};
template <int NT, bool SHARED>
__device__ __forceinline__ Work sequence_work(const AttParams& p, int s) {
    Work w;
    int b;
    p.c.rows_of(s, w.row0, b);
    w.rows = b - w.row0;
    w.before = __ldg(p.c.lengths + s);
    w.chunks = (uint32_t(w.rows) * p.group + 8 * NT - 1) / (8 * NT);
    const uint32_t most = uint32_t(p.c.width) * uint32_t(p.c.blocks_per_page);
    const int64_t seen = int64_t(w.before) + w.rows;
    const uint32_t n = seen <= 0 ? 0u : uint32_t((seen + kKvBlock - 1) / kKvBlock);
    w.blocks = min(n, most);
    w.first = 0;
    w.joined = false;
    if (SHARED) {
        const uint32_t first = uint32_t(shared_of(p.c, p.shared, s, w.row0, b, w.before));
        w.joined = first > 0;
        w.first = min(first, w.blocks);
        w.blocks -= w.first;
    }
    w.units = max(1u, (w.blocks + (kAttWarps << p.unit_shift) - 1) / (kAttWarps << p.unit_shift));
    return w;
}
// Behind the blocks that an item's last row sees.
template <int NT, bool SHARED>
__device__ __forceinline__ uint32_t last_block(const AttParams& p, const Work& w, const Seg& q) {
    const uint32_t rows = q.col0 + 8 * NT >= q.cols ? w.rows : (q.col0 + 8 * NT - 1) / uint32_t(p.group) + 1;  // up to the item's last
    const int64_t seen = int64_t(w.before) + rows;
    return seen <= 0 ? 0u : min(SHARED ? w.first + w.blocks : w.blocks, uint32_t((seen + kKvBlock - 1) / kKvBlock));
}
// The part of units [u0, u1) of an item.
template <int NT, bool SHARED>
__device__ __forceinline__ void set_seg(const AttParams& p, const Work& w, int s, uint32_t item, uint32_t u0, uint32_t u1, int first, int last, Seg& q) {
    q.seq = s;
    const uint32_t head = quotient(item, w.chunks);
    q.head = int(head);
    q.row0 = w.row0;
    q.col0 = int(item - head * w.chunks) * 8 * NT;
    q.cols = w.rows * p.group;
    q.before = w.before;
    q.joined = w.joined;
    q.first = first;
    q.last = last;
    const uint32_t n = last_block<NT, SHARED>(p, w, q);
    q.r0 = (SHARED ? w.first : 0u) + u0 * (kAttWarps << p.unit_shift);
    q.r1 = min(n, (SHARED ? w.first : 0u) + u1 * (kAttWarps << p.unit_shift));
}

// Parts of an item of so many units when a CTA takes `share` at most, and units of a part.
__device__ __forceinline__ uint32_t parts_of(uint32_t units, uint32_t share, uint32_t& each) {
    if (units <= share) {
        each = units;
        return 1;
    }
    const uint32_t parts = (units + share - 1) / share;
    each = (units + parts - 1) / parts;
    return (units + each - 1) / each;
}

// Units of a part that may do for so many items on G CTAs, items <= G: a quarter or half of the items' last parts are thought to be
// short, then all: that one does.
__device__ __forceinline__ uint32_t tried_share(uint32_t G, uint32_t items, uint32_t units, int j) {
    const uint32_t over = max(1u, G - (j == 0 ? items >> 2 : j == 1 ? items >> 1 : items));
    return max(kAttLeastUnits, (units + over - 1) / over);
}
// A CTA with one part of one item has neither to look up its items one after another nor to begin anew, which takes as long as
// about five units (16 sequences of 2048: 19.4 us so, 22.5 us with even ranges of 7 units instead of 8).
__device__ __forceinline__ bool worth_it(uint32_t share, uint32_t even) { return share <= even + even / 8 + 5; }

// Whether a warp for each item is faster than parts or ranges of units, items being of so many blocks at most.  In hundreds of
// cycles: a part of an item takes a CTA 45 and 22 for each of its units, an item a warp 5 and 13 for each block.  Measured, 8
// heads, without against with: 40 sequences of 3 tokens 8.9 and 5.3 us, of 250 13.9 and 13.1, of 500 18.2 and 23.4; 128 of 700 41.6
// and 36.5; 500 of 3 tokens 42 and 12 us, of 700 133 and 120.
__device__ __forceinline__ bool short_items(uint32_t G, uint32_t items, uint32_t blocks) {
    const uint32_t rounds = (items + kAttWarps * G - 1) / (kAttWarps * G), parts = (items + G - 1) / G;
    return blocks < 64 && rounds * (5 + 13 * blocks) < parts * (45 + 22 * ((blocks + kAttWarps - 1) / kAttWarps));
}

template <int N>
__device__ __forceinline__ void block_sums(uint32_t (&v)[N], uint32_t (*warp_sums)[kAttWarps]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = __reduce_add_sync(0xFFFFFFFFu, v[i]);
        if (lane == 0) warp_sums[i][warp] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0;
#pragma unroll
        for (int w = 0; w < kAttWarps; ++w) v[i] += warp_sums[i][w];
    }
    __syncthreads();
}

template <int D, int NT, bool SHARED>
__device__ __forceinline__ void attend(const AttParams& p) {
    using C = AttCfg<D, NT>;
    constexpr int CHUNKS = C::CHUNKS, STAGES = C::STAGES, REC = C::REC, FRAGS = C::FRAGS, ROUND = C::ROUND;
    constexpr bool RUNS = SHARED && NT == 1;  // of an item, a warp's each
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* ring = smem;
    float4* merge = reinterpret_cast<float4*>(smem + C::RING);                             // [warps][ROUND + NT][32]
    unsigned char* qs = smem + C::RING + C::MERGE;                                         // [NT][CHUNKS][32][16 bytes]
    uint32_t* prefix = reinterpret_cast<uint32_t*>(smem + C::RING + C::MERGE + C::QBYTES); // [seqs + 1]
    __shared__ Seg segs[kAttSegs];
    __shared__ int nsegs, cursor_seq;
    __shared__ int64_t places[2][8 * NT];  // of an item's columns in the output, or -1; the next item's apart
    __shared__ uint32_t cursor_unit, is_last, the_share, are_few, are_tiny, warp_sums[4][kAttWarps];

    // (What all lanes of a warp have alike is taken from lane 0 here and below: branches on it need no reconvergence.)
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0), g = lane >> 2, t = lane & 3;
    const int heads = p.c.kv_heads, heads_all = heads * p.group;
    // The first lines of the page table, which is wanted as soon as it is known whose it is.
    {
        const int64_t entries = (p.c.seqs - 1) * p.c.table_stride + p.c.width, at = int64_t(threadIdx.x) * 32;
        if (at < entries) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.c.table + at));
    }
    // How the work is cut.  Every CTA finds out for itself.  With few items each gets CTAs of its own, as many parts as leave the
    // longest part short: part sizes are tried from one that may need too many CTAs to one that cannot.  With many, or where
    // that would leave CTAs idle for long, a CTA takes a range of the sequence of all units; but of very short items each is a
    // warp's own.  Up to 32 sequences are one warp's work to cut, without a barrier.
    const uint32_t G = gridDim.x;
    bool few = false, tiny = RUNS;
    uint32_t share = 0, run = 1;  // blocks of a run
    if (RUNS) {
        // Runs as long as leave every warp of the grid one, but of eight blocks at least (what a warp begins and ends with takes as long).
        const int per = (p.c.seqs + kAttThreads - 1) / kAttThreads, s0 = threadIdx.x * per, s1 = min(s0 + per, p.c.seqs);
        uint64_t read = 0;
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            const Work w = sequence_work<NT, SHARED>(p, s);
            read += uint64_t(w.chunks * heads) * w.blocks;
        }
        uint32_t total[2] = {uint32_t(read) & 0xFFFFFFu, uint32_t(read >> 24)};  // 256 threads' sums do not wrap
        block_sums(total, warp_sums);
        const uint32_t warps = G * kAttWarps;
        run = max(8u, total[1] ? uint32_t(((uint64_t(total[1]) << 24) + total[0]) / warps) + 1u : (total[0] + warps - 1) / warps);
        auto wanted = [&](const Work& w) { return w.chunks * heads * max(1u, (w.blocks + run - 1) / run); };
        uint32_t mine = 0;
#pragma unroll 1
        for (int s = s0; s < s1; ++s) mine += wanted(sequence_work<NT, SHARED>(p, s));
        uint32_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) warp_sums[0][warp] = sum;
        __syncthreads();
        uint32_t at = sum - mine;
        for (int w = 0; w < warp; ++w) at += warp_sums[0][w];
        if (threadIdx.x == kAttThreads - 1) prefix[p.c.seqs] = min(at + mine, p.runs_most);
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            const Work w = sequence_work<NT, SHARED>(p, s);
            prefix[s] = min(at, p.runs_most);
            if (blockIdx.x == 0) p.owns[s] = OwnSeq{int32_t(at), int32_t(at + wanted(w) <= p.runs_most ? max(1u, (w.blocks + run - 1) / run) : 0u), int32_t(w.chunks), 0};
            at += wanted(w);
        }
        if (threadIdx.x == 0) cursor_seq = 0;
        __syncthreads();
    } else if (p.c.seqs <= 32) {
        if (warp == 0) {
            const bool is = lane < p.c.seqs;
            Work w = is ? sequence_work<NT, SHARED>(p, lane) : Work{0, 0, 0, 0, 0, 1, 0, false};
            const uint32_t items = w.chunks * heads, all_items = __reduce_add_sync(0xFFFFFFFFu, items), all_units = __reduce_add_sync(0xFFFFFFFFu, items * w.units);
            const uint32_t even = (all_units + G - 1) / G;
            if (all_items <= G) {
#pragma unroll 1
                for (int j = 0; j < 3; ++j) {
                    share = tried_share(G, all_items, all_units, j);
                    if (__reduce_add_sync(0xFFFFFFFFu, items * ((w.units + share - 1) / share)) <= G) break;
                }
            }
            few = all_items <= G && worth_it(share, even);
            if (!few) share = even;
            if (NT == 1 && !few) tiny = short_items(G, all_items, __reduce_max_sync(0xFFFFFFFFu, items ? w.blocks : 0u));
            uint32_t each = 0, parts = 1;
            if (few) parts = parts_of(w.units, share, each);
            const uint32_t own = items * (few ? parts : tiny ? 1u : w.units);
            uint32_t at = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, at, o);
                if (lane >= o) at += v;
            }
            const uint32_t want = few || tiny ? blockIdx.x : share * blockIdx.x;
            if (lane == 31) {
                prefix[p.c.seqs] = at;
                if (want >= at) cursor_seq = -1;  // nothing left for this CTA
                the_share = share;
                are_few = few;
                are_tiny = tiny;
            }
            at -= own;
            if (is) prefix[lane] = at;
            if (at <= want && want < at + own) {
                cursor_seq = lane;
                cursor_unit = want;
                if (few) {
                    const uint32_t local = want - at, item = quotient(local, parts), part = local - item * parts;
                    set_seg<NT, SHARED>(p, w, lane, item, part * each, (part + 1) * each, int(blockIdx.x - part), int(blockIdx.x - part + parts - 1), segs[0]);
                    nsegs = 1;
                }
            }
        }
        __syncthreads();
        few = are_few;
        tiny = are_tiny;
        share = the_share;
    } else {
        // ... otherwise all threads', in loops that have one turn for up to 256 sequences (kept as loops: instructions that
        // run once a launch cost their fetch).
        const int per = (p.c.seqs + kAttThreads - 1) / kAttThreads, s0 = threadIdx.x * per, s1 = min(s0 + per, p.c.seqs);
        uint32_t total[2] = {0, 0}, longest = 0;
        if (threadIdx.x == 0) cursor_unit = 0;
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            const Work w = sequence_work<NT, SHARED>(p, s);
            total[0] += w.chunks * heads;
            total[1] += w.chunks * heads * w.units;
            if (w.chunks) longest = max(longest, w.blocks);
        }
        block_sums(total, warp_sums);
        const uint32_t even = (total[1] + G - 1) / G;
        share = even;
        few = total[0] <= G;
        if (few) {
            uint32_t tried[3], need[3] = {0, 0, 0};
#pragma unroll
            for (int j = 0; j < 3; ++j) tried[j] = tried_share(G, total[0], total[1], j);
#pragma unroll 1
            for (int s = s0; s < s1; ++s) {
                const Work w = sequence_work<NT, SHARED>(p, s);
#pragma unroll
                for (int j = 0; j < 3; ++j) need[j] += w.chunks * heads * ((w.units + tried[j] - 1) / tried[j]);
            }
            block_sums(need, warp_sums);
            share = need[0] <= G ? tried[0] : need[1] <= G ? tried[1] : tried[2];
            few = worth_it(share, even);
            if (!few) share = even;
        }
        if (NT == 1 && !few) {
            longest = __reduce_max_sync(0xFFFFFFFFu, longest);
            if (lane == 0) atomicMax(&cursor_unit, longest);
            __syncthreads();
            tiny = short_items(G, total[0], cursor_unit);
            __syncthreads();
        }
        // Prefix sum over the sequences: of CTAs, of items, or of units.
        {
            auto wanted = [&](const Work& w) {
                uint32_t each;
                return w.chunks * heads * (few ? parts_of(w.units, share, each) : tiny ? 1u : w.units);
            };
            uint32_t mine = 0;
#pragma unroll 1
            for (int s = s0; s < s1; ++s) {
                const Work w = sequence_work<NT, SHARED>(p, s);
                if (w.chunks) mine += wanted(w);
            }
            uint32_t sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= o) sum += v;
            }
            if (lane == 31) warp_sums[0][warp] = sum;
            __syncthreads();
            uint32_t at = sum - mine;
            for (int w = 0; w < warp; ++w) at += warp_sums[0][w];
            const uint32_t want = few || tiny ? blockIdx.x : share * blockIdx.x;
            if (threadIdx.x == kAttThreads - 1) {
                prefix[p.c.seqs] = at + mine;
                if (want >= at + mine) cursor_seq = -1;  // nothing left for this CTA
            }
            if (!few || (at <= want && want < at + mine)) {
#pragma unroll 1
                for (int s = s0; s < s1; ++s) {
                    const Work w = sequence_work<NT, SHARED>(p, s);
                    const uint32_t own = w.chunks ? wanted(w) : 0u;
                    prefix[s] = at;
                    if (at <= want && want < at + own) {
                        cursor_seq = s;
                        cursor_unit = want;
                        if (few) {
                            uint32_t each;
                            const uint32_t parts = parts_of(w.units, share, each), local = want - at, item = quotient(local, parts), part = local - item * parts;
                            set_seg<NT, SHARED>(p, w, s, item, part * each, (part + 1) * each, int(blockIdx.x - part), int(blockIdx.x - part + parts - 1), segs[0]);
                            nsegs = 1;
                        }
                    }
                    at += own;
                }
            }
            __syncthreads();
        }
    }
    if (cursor_seq < 0) return;

    const uint32_t my_ring = smem_u32(ring) + warp * STAGES * REC, lane16 = lane * 16;
    // A warp's records of a part: every eighth, or all.
    const uint32_t offset = tiny ? 0 : warp, step = tiny ? 1 : kAttWarps;
    const Seg* list = tiny ? segs + warp : segs;
    for (uint32_t item = warp * G + blockIdx.x;; item += kAttWarps * G) {
        if (tiny) {  // the warp's next item
            if (item >= prefix[p.c.seqs]) return;
            int s = 0;
            for (uint32_t who = 0; !who; s += 32) {
                const int at = s + lane;
                who = __ballot_sync(0xFFFFFFFFu, at < p.c.seqs && prefix[at] <= item && item < prefix[at + 1]);
                if (who) s += __ffs(who) - 33;
            }
            const Work w = sequence_work<NT, SHARED>(p, s);
            __syncwarp();
            if (RUNS) {
                const uint32_t runs = max(1u, (w.blocks + run - 1) / run), local = item - prefix[s], it = quotient(local, runs), u = local - it * runs;
                if (lane == 0) {
                    set_seg<NT, SHARED>(p, w, s, it, 0, 0, 0, 0, segs[warp]);
                    const uint32_t end = last_block<NT, SHARED>(p, w, segs[warp]);
                    segs[warp].r0 = w.first + u * run;
                    segs[warp].r1 = min(end, w.first + (u + 1) * run);
                }
            } else {
                if (lane == 0) set_seg<NT, SHARED>(p, w, s, item - prefix[s], 0, w.units, 0, 0, segs[warp]);
            }
            __syncwarp();
        } else if (!few) {  // the next parts of items of this CTA's range
            if (threadIdx.x == 0) {
                int n = 0, s = cursor_seq;
                uint32_t u = cursor_unit;
                const uint32_t end = min(prefix[p.c.seqs], share * (blockIdx.x + 1));
                while (n < kAttSegs && u < end) {
                    while (u >= prefix[s + 1]) ++s;
                    const Work w = sequence_work<NT, SHARED>(p, s);
                    uint32_t item = (u - prefix[s]) / w.units;
                    while (n < kAttSegs && u < end && u < prefix[s + 1]) {
                        const uint32_t at = prefix[s] + item * w.units, stop = min(at + w.units, end);
                        set_seg<NT, SHARED>(p, w, s, item, u - at, stop - at, int(at / share), int((at + w.units - 1) / share), segs[n++]);
                        u = stop;
                        ++item;
                    }
                }
                nsegs = n;
                cursor_seq = s;
                cursor_unit = u;
            }
            __syncthreads();
        }
        const int count = tiny ? 1 : __shfl_sync(0xFFFFFFFFu, nsegs, 0);
        if (count == 0) return;

        // The warp's stream of records over these parts: lane l looks up the place of the l-th of the next 32.
        int ahead_seg = -1, ahead_lane = 31;
        uint32_t ahead_rec = 0, ahead_end = 0;
        const unsigned char* ahead_at = nullptr;  // of the lane's record
        auto advance = [&] {
            ahead_rec += step;
            if (++ahead_lane < 32 && ahead_rec < ahead_end) return;
            while (ahead_rec >= ahead_end) {
                if (++ahead_seg >= count) return;
                ahead_rec = __shfl_sync(0xFFFFFFFFu, list[ahead_seg].r0, 0) + offset;
                ahead_end = __shfl_sync(0xFFFFFFFFu, list[ahead_seg].r1, 0);
            }
            ahead_lane = 0;
            const uint32_t mine = ahead_rec + lane * step;
            ahead_at = mine < ahead_end ? p.c.template record<D>(list[ahead_seg].seq, mine, list[ahead_seg].head) : nullptr;
        };
        uint32_t placed = 0;  // bit per stage: its record has a place
        int stage = 0;
        auto issue = [&](int to) {
            placed &= ~(1u << to);
            if (ahead_seg < count) {
                const unsigned char* from = reinterpret_cast<const unsigned char*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<uint64_t>(ahead_at), ahead_lane));
                if (__ballot_sync(0xFFFFFFFFu, ahead_at != nullptr) >> ahead_lane & 1u) {
                    placed |= 1u << to;
                    const uint32_t dst = my_ring + to * REC;
#pragma unroll
                    for (int j = 0; j < 2 * CHUNKS; ++j) copy16(dst + j * 512 + lane16, from + j * 512 + lane16);
                    if (lane == 0) copy16(dst + 2 * CHUNKS * 512, from + 2 * CHUNKS * 512);
                }
                advance();
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        advance();

        for (int i = 0; i < count; ++i) {
            const Seg& sg = list[i];
            // Queries: lane (g, t) holds column g's dims 32 j + 8 t .. + 7 of every chunk j.
            uint4 qr[NT == 1 ? CHUNKS : 1];
            if (NT == 1) {
                const uint32_t col = sg.col0 + g;
                const bool live = int(col) < sg.cols;
                const uint32_t row = live ? quotient(col, p.group) : 0, h = live ? col - row * p.group : 0;
                const __half* src = p.q + int64_t(sg.row0 + row) * p.q_stride + (sg.head * p.group + h) * D + 8 * t;
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) qr[j] = live ? __ldg(reinterpret_cast<const uint4*>(src + 32 * j)) : make_uint4(0, 0, 0, 0);
                if (i == 0) {  // behind the queries' loads: the first copies wait for a page number
#pragma unroll
                    for (int k = 0; k < STAGES; ++k) issue(k);
                }
            } else {
                constexpr int EACH = (NT * CHUNKS * 32 + kAttThreads - 1) / kAttThreads;
                uint4 v[EACH];
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    const int k = threadIdx.x + e * kAttThreads, l = k & 31, j = k / 32 % CHUNKS;
                    const uint32_t col = sg.col0 + k / (32 * CHUNKS) * 8 + (l >> 2);
                    v[e] = make_uint4(0, 0, 0, 0);
                    if (k < NT * CHUNKS * 32 && int(col) < sg.cols) {
                        const uint32_t row = quotient(col, p.group), h = col - row * p.group;
                        v[e] = __ldg(reinterpret_cast<const uint4*>(p.q + int64_t(sg.row0 + row) * p.q_stride + (sg.head * p.group + h) * D + 32 * j + 8 * (l & 3)));
                    }
                }
                if (i == 0) {
#pragma unroll
                    for (int k = 0; k < STAGES; ++k) issue(k);
                }
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    if (int(threadIdx.x) + e * kAttThreads < NT * CHUNKS * 32) reinterpret_cast<uint4*>(qs)[threadIdx.x + e * kAttThreads] = v[e];
                __syncthreads();
            }
            if (!tiny && threadIdx.x < 8 * NT) {  // read behind the merge's barrier
                const uint32_t col = sg.col0 + threadIdx.x;
                int64_t at = -1;
                if (int(col) < sg.cols) {
                    const uint32_t row = quotient(col, p.group), h = col - row * p.group;
                    at = (int64_t(sg.row0 + row) * heads_all + sg.head * p.group + h) * D;
                }
                places[i & 1][threadIdx.x] = at;
            }
            // Last position of the lane's columns (2 t, 2 t + 1 of each eight), and of the item's first.
            int sees[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int col = sg.col0 + nt * 8 + 2 * t + k;
                    sees[nt][k] = int(min(int64_t(INT32_MAX), int64_t(sg.before) + (col < sg.cols ? quotient(col, p.group) : 0u)));
                }
            const int all_see = int(min(int64_t(INT32_MAX), int64_t(sg.before) + quotient(sg.col0, p.group)));

            float o[FRAGS][4], ref[NT][2], sum[NT][2];
#pragma unroll
            for (int f = 0; f < FRAGS; ++f)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[f][k] = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) ref[nt][0] = ref[nt][1] = kNoRef, sum[nt][0] = sum[nt][1] = 0.f;

            const uint32_t end = __shfl_sync(0xFFFFFFFFu, sg.r1, 0);
            for (uint32_t rec = __shfl_sync(0xFFFFFFFFu, sg.r0, 0) + offset; rec < end; rec += step) {
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
                __syncwarp();  // the scales were copied by lane 0
                if (placed >> stage & 1u) {
                    const uint32_t at = my_ring + stage * REC;
                    const uint4 scales = lds_uint4(at + 2 * CHUNKS * 512);
                    const float by = __uint_as_float(scales.x) * p.scale, vs = __uint_as_float(scales.y);
                    float lv = lg2(vs);
                    lv = lv < kLeastLog ? kLeastLog : lv;  // NaN stays
                    // A score of 2^24 or more has no fractions, and what is added to it is rounded away: it is its difference from the
                    // reference, which is exact where it matters, that is held against the room for a weight.
                    const float room = kHigh - lv;
                    float x[NT][4], y[NT][4];  // two chains: a product waits for the one before it
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[nt][k] = y[nt][k] = 0.f;
#pragma unroll
                    for (int j = 0; j < CHUNKS; ++j) {
                        const uint4 w = lds_uint4(at + j * 512 + lane16);
                        const uint32_t a0 = codes_of<false>(w.x), a2 = codes_of<true>(w.x), a1 = codes_of<false>(w.z), a3 = codes_of<true>(w.z);
                        const uint32_t c0 = codes_of<false>(w.y), c2 = codes_of<true>(w.y), c1 = codes_of<false>(w.w), c3 = codes_of<true>(w.w);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint4 b = NT == 1 ? qr[j] : reinterpret_cast<const uint4*>(qs)[(nt * CHUNKS + j) * 32 + lane];
                            mma16816(x[nt], a0, a1, a2, a3, b.x, b.y);
                            mma16816(NT < 4 ? y[nt] : x[nt], c0, c1, c2, c3, b.z, b.w);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[nt][k] = (NT < 4 ? x[nt][k] + y[nt][k] : x[nt][k]) * by;
                    const int token = int(rec * kKvBlock) + g;  // and 8 on
                    bool over = false;
                    if (int(rec * kKvBlock) + kKvBlock - 1 > all_see) {  // the last blocks: some column does not see all of it
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (token + (k >> 1) * 8 > sees[nt][k & 1]) x[nt][k] = -INFINITY;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        over |= fmaxf(x[nt][0], x[nt][2]) - ref[nt][0] > room || fmaxf(x[nt][1], x[nt][3]) - ref[nt][1] > room;
                    if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                float top = fmaxf(x[nt][k], x[nt][k + 2]);
#pragma unroll
                                for (int m = 4; m <= 16; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
                                float now = top + lv - kBase;
                                if (top - now > room) now = top;  // a step of so large scores is more than the room there is
                                if (now > ref[nt][k]) {
                                    const float f = ex2(ref[nt][k] - now);
                                    ref[nt][k] = now;
                                    sum[nt][k] *= f;
#pragma unroll
                                    for (int m = 0; m < D / 16; ++m) {
                                        o[nt * (D / 16) + m][k] *= f;
                                        o[nt * (D / 16) + m][k + 2] *= f;
                                    }
                                }
                            }
                    }
                    uint32_t b0[NT], b1[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float e = ex2(x[nt][k] - ref[nt][k & 1]);
                            sum[nt][k & 1] += e;
                            w[k] = x[nt][k] == -INFINITY ? 0.f : e * vs;  // nothing of a block whose scale is NaN where it is not seen
                        }
                        const __half2 lo = __floats2half2_rn(w[0], w[1]), hi = __floats2half2_rn(w[2], w[3]);
                        b0[nt] = transpose8x8(*reinterpret_cast<const uint32_t*>(&lo));
                        b1[nt] = transpose8x8(*reinterpret_cast<const uint32_t*>(&hi));
                    }
#pragma unroll
                    for (int j = 0; j < CHUNKS; ++j) {
                        const uint4 w = lds_uint4(at + (CHUNKS + j) * 512 + lane16);
                        const uint32_t a0 = codes_of<false>(w.x), a2 = codes_of<true>(w.x), a1 = codes_of<false>(w.y), a3 = codes_of<true>(w.y);
                        const uint32_t c0 = codes_of<false>(w.z), c2 = codes_of<true>(w.z), c1 = codes_of<false>(w.w), c3 = codes_of<true>(w.w);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma16816(o[nt * (D / 16) + 2 * j], a0, a1, a2, a3, b0[nt], b1[nt]);
                            mma16816(o[nt * (D / 16) + 2 * j + 1], c0, c1, c2, c3, b0[nt], b1[nt]);
                        }
                    }
                }
                __syncwarp();  // all lanes have read the scales before lane 0 copies over them
                issue(stage);
                stage = stage + 1 == STAGES ? 0 : stage + 1;
            }

            // Two of a fragment's values belong to column 2 t (2 t + 1) and dims d, d + 1.
            auto store = [&](int f, const float (&v)[4], float r_even, float r_odd, float s_even, float s_odd) {
                const int nt = f / (D / 16), m = f % (D / 16), d = m / 2 * 32 + 4 * g + (m & 1) * 2;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int64_t at = places[i & 1][nt * 8 + 2 * t + k];
                    const float s = k ? s_odd : s_even, by = s == 0.f ? 0.f : 1.f / s;  // nothing seen: zero
                    if (SHARED && sg.joined && at >= 0) {
                        __stcg(reinterpret_cast<float2*>(p.own + at + d), make_float2(v[k], v[k + 2]));
                        if (d == 0) __stcg(reinterpret_cast<float2*>(p.own + p.own_ends) + at / D, make_float2(k ? r_odd : r_even, s));
                        continue;
                    }
                    if (at >= 0) *reinterpret_cast<__half2*>(p.out + at + d) = __floats2half2_rn(v[k] * by, v[k + 2] * by);
                }
            };

            // The warps' sums become one: as many fragments as there are warps at a time, each warp adds one over all of them.
            // Of an item that several CTAs share, each leaves a piece: place 1 of the CTA that the item begins in, place 0 of the others.
            const int me = blockIdx.x, shared_by = sg.last - sg.first + 1;
            auto piece_at = [&](int cta, int place) { return reinterpret_cast<float4*>(p.pieces + (size_t(cta) * 4 + place) * C::PIECE); };
            auto leave = [&](float4* piece, int f, const float (&v)[4], float r0, float r1, float u0, float u1) {
                __stcg(piece + f * 32 + lane, make_float4(v[0], v[1], v[2], v[3]));
                if (f % (D / 16) == 0 && g == 0) __stcg(piece + FRAGS * 32 + f / (D / 16) * 4 + t, make_float4(r0, r1, u0, u1));
            };
            constexpr int SLOT = (ROUND + NT) * 32;
            float4* mine = merge + warp * SLOT + lane;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int m = 4; m <= 16; m <<= 1) sum[nt][k] += __shfl_xor_sync(0xFFFFFFFFu, sum[nt][k], m);
            }
            if (tiny) {  // all of a column's dims that the lane has, four at a time
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t col = sg.col0 + 2 * t + k, row = quotient(col, p.group), h = col - row * p.group;
                    const float s = sum[0][k], by = s == 0.f ? 0.f : 1.f / s;  // nothing seen: zero
                    if (int(col) >= sg.cols) continue;
                    const int64_t at = int64_t(sg.row0 + row) * heads_all + sg.head * p.group + h;
                    if (RUNS) {
                        const int64_t piece = int64_t(item) * 8 + 2 * t + k;
#pragma unroll
                        for (int j = 0; j < CHUNKS; ++j)
                            __stcg(reinterpret_cast<float4*>(p.own + piece * D + 4 * g + 32 * j), make_float4(o[2 * j][k], o[2 * j][k + 2], o[2 * j + 1][k], o[2 * j + 1][k + 2]));
                        if (g == 0) __stcg(reinterpret_cast<float2*>(p.own + p.own_ends) + piece, make_float2(ref[0][k], s));
                        continue;
                    }
                    __half* out = p.out + at * D + 4 * g;
#pragma unroll
                    for (int j = 0; j < CHUNKS; ++j) {
                        const __half2 lo = __floats2half2_rn(o[2 * j][k] * by, o[2 * j][k + 2] * by), hi = __floats2half2_rn(o[2 * j + 1][k] * by, o[2 * j + 1][k + 2] * by);
                        *reinterpret_cast<uint2*>(out + 32 * j) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
                    }
                }
                break;  // count is one
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mine[(ROUND + nt) * 32] = make_float4(ref[nt][0], ref[nt][1], sum[nt][0], sum[nt][1]);
#pragma unroll
            for (int at = 0; at < FRAGS; at += ROUND) {
#pragma unroll
                for (int f = 0; f < ROUND; ++f) mine[f * 32] = make_float4(o[at + f][0], o[at + f][1], o[at + f][2], o[at + f][3]);
                __syncthreads();
#pragma unroll
                for (int turn = 0; turn < C::EACH; ++turn) {
                    const int slot = warp + turn * kAttWarps, f = at + slot, nt = f / (D / 16);
                    if (slot < ROUND) {
                        const float4* all = merge + lane;
                        float4 m[kAttWarps];
                        float r0 = kNoRef, r1 = kNoRef, u0 = 0.f, u1 = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int w = 0; w < kAttWarps; ++w) {
                            m[w] = all[w * SLOT + (ROUND + nt) * 32];
                            r0 = fmaxf(r0, m[w].x);
                            r1 = fmaxf(r1, m[w].y);
                        }
#pragma unroll
                        for (int w = 0; w < kAttWarps; ++w) {
                            const float4 x = all[w * SLOT + slot * 32];
                            const float f0 = ex2(m[w].x - r0), f1 = ex2(m[w].y - r1);
                            u0 = fmaf(m[w].z, f0, u0);
                            u1 = fmaf(m[w].w, f1, u1);
                            v[0] = fmaf(x.x, f0, v[0]);
                            v[1] = fmaf(x.y, f1, v[1]);
                            v[2] = fmaf(x.z, f0, v[2]);
                            v[3] = fmaf(x.w, f1, v[3]);
                        }
                        if (shared_by == 1) store(f, v, r0, r1, u0, u1);
                        else leave(piece_at(me, me == sg.first), f, v, r0, r1, u0, u1);
                    }
                }
                __syncthreads();
            }
            if (shared_by > 1) {
                // The CTA that finds all of a group's pieces there adds them, in order; of many, the square root at a time, and then the
                // groups' sums (places 2 and 3 of a group's first CTA): a load of what another CTA has just written takes long, and
                // one after another so many of them.
                int group = shared_by;
                if (group > kAttBatch) {
                    group = 3;
                    while (group * group < shared_by) ++group;
                }
                const int groups = (shared_by + group - 1) / group, begin = sg.first + (me - sg.first) / group * group;
#pragma unroll 1
                for (int level = 0; level < 2; ++level) {
                    const int from = level ? sg.first : begin, step = level ? group : 1, n = level ? groups : min(group, sg.last + 1 - begin);
                    if (threadIdx.x == 0) {
                        uint32_t* counter = p.arrived + (level ? 2 : from == sg.first) * kAttMaxCtas + from;
                        uint32_t had;  // behind the barrier: releases the whole CTA's stores, and acquires the others'
                        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(had) : "l"(counter) : "memory");
                        is_last = had + 1 == uint32_t(n);
                        if (is_last) *counter = 0u;  // for the next call
                    }
                    __syncthreads();
                    const bool go_on = is_last;
                    __syncthreads();
                    if (!go_on) break;
                    const bool final = level == 1 || groups == 1;
                    constexpr int TURNS = C::TURNS, BATCH = kAttBatch / TURNS;
                    float r0[TURNS], r1[TURNS], u0[TURNS], u1[TURNS], v[TURNS][4];
#pragma unroll
                    for (int k = 0; k < TURNS; ++k) r0[k] = r1[k] = kNoRef, u0[k] = u1[k] = v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0.f;
#pragma unroll 1
                    for (int at = 0; at < n; at += BATCH) {
                        float4 u[TURNS][BATCH], m[TURNS][BATCH];
#pragma unroll
                        for (int k = 0; k < BATCH; ++k) {
                            const int cta = from + min(at + k, n - 1) * step;
                            const float4* piece = piece_at(cta, 2 * level + (cta == sg.first));
#pragma unroll
                            for (int i = 0; i < TURNS; ++i) {
                                const int f = warp + i * kAttWarps;
                                const bool is = at + k < n && f < FRAGS;
                                u[i][k] = is ? __ldcg(piece + f * 32 + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
                                m[i][k] = is ? __ldcg(piece + FRAGS * 32 + f / (D / 16) * 4 + t) : make_float4(kNoRef, kNoRef, 0.f, 0.f);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < TURNS; ++i) {
                            float q0 = r0[i], q1 = r1[i];
#pragma unroll
                            for (int k = 0; k < BATCH; ++k) q0 = fmaxf(q0, m[i][k].x), q1 = fmaxf(q1, m[i][k].y);
                            const float f0 = ex2(r0[i] - q0), f1 = ex2(r1[i] - q1);
                            u0[i] *= f0, u1[i] *= f1, v[i][0] *= f0, v[i][1] *= f1, v[i][2] *= f0, v[i][3] *= f1;
#pragma unroll
                            for (int k = 0; k < BATCH; ++k) {
                                const float n0 = ex2(m[i][k].x - q0), n1 = ex2(m[i][k].y - q1);
                                u0[i] = fmaf(m[i][k].z, n0, u0[i]);
                                u1[i] = fmaf(m[i][k].w, n1, u1[i]);
                                v[i][0] = fmaf(u[i][k].x, n0, v[i][0]);
                                v[i][1] = fmaf(u[i][k].y, n1, v[i][1]);
                                v[i][2] = fmaf(u[i][k].z, n0, v[i][2]);
                                v[i][3] = fmaf(u[i][k].w, n1, v[i][3]);
                            }
                            r0[i] = q0;
                            r1[i] = q1;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < TURNS; ++i) {
                        const int f = warp + i * kAttWarps;
                        if (f >= FRAGS) break;
                        if (final) store(f, v[i], r0[i], r1[i], u0[i], u1[i]);
                        else leave(piece_at(begin, 2 + (begin == sg.first)), f, v[i], r0[i], r1[i], u0[i], u1[i]);
                    }
                    if (final) break;
                    __syncthreads();  // the stores are all before the next arrival
                }
            }
        }
        if (few) return;
        if (!tiny) __syncthreads();  // segs
    }
}

template <int D, int NT, bool SHARED>
__global__ void __launch_bounds__(kAttThreads, AttCfg<D, NT>::CTAS) k_kv_attend(AttParams p) {
    if (!SHARED) {
        pdl_wait();
        pdl_release();
    }
    attend<D, NT, SHARED>(p);
    if (SHARED) end_behind_prefix();
}

constexpr int kAttCounters = kAttMaxCtas * 3 * 4;  // bytes
template <int D>
constexpr int att_most_columns() { return D == 256 ? 2 : 4; }
template <int D>
constexpr size_t att_workspace() { return size_t(kAttCounters) + size_t(kAttMaxCtas) * 4 * AttCfg<D, att_most_columns<D>()>::PIECE * 4; }

template <int D, int NT, bool SHARED>
cudaError_t launch_attend(AttParams p, int sms, cudaStream_t s) {
    using C = AttCfg<D, NT>;
    constexpr int most = C::SMEM + 4 * (TETRA_KV_MAX_SEQS + 1);
    static PerDeviceOnce once;  // per instantiation
    cudaError_t e = once.run([] { return cudaFuncSetAttribute(k_kv_attend<D, NT, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize, most); });
    if (e != cudaSuccess) return e;
    const int grid = C::CTAS * sms < kAttMaxCtas ? C::CTAS * sms : kAttMaxCtas;
    // Units are counted in 32 bits, a grid's rounding with them: larger ones where all sequences, as long as the table and with
    // all of the rows (row_start is not known here), could pass that.
    const int64_t items = (int64_t(p.c.rows) * p.group / (8 * NT) + 1) * p.c.seqs * p.c.kv_heads, blocks = int64_t(p.c.width) * p.c.blocks_per_page;
    while (items * (blocks / (kAttWarps << p.unit_shift) + 1) > (1ll << 30) && blocks > (kAttWarps << p.unit_shift)) ++p.unit_shift;
    return launch_pdl(k_kv_attend<D, NT, SHARED>, grid, kAttThreads, size_t(C::SMEM) + 4 * (p.c.seqs + 1), s, p);
}

// Columns of an item by what a sequence has on average: more of them read a block's codes once for more rows, but an
// item with empty columns pays for all.  One kernel serves all of a step's sequences, so a piece of a prompt among single tokens is cut
// into items of eight columns that each read its context (mostly from L2).  Measured, 63 single tokens and one piece of 16 rows, 32/8
// heads of 128, us with 8 / 16 / 32 columns: tokens behind 100 and the piece behind 2000 25 / 26 / 42, behind 100 and 8000 61 / 55 / 74,
// 1000 and 8000 47 / 57 / 78, 2000 and 8000 64 / 76 / 101; one row in the piece's place 15, 20, 33 and 57 with 8.
// (At the cap of 128 registers two CTAs to an SM leave 16 columns of 128 dims with 100 bytes spilt a thread, 32 of 64 with 12:
// 64 sequences of 4 rows behind 4000 tokens, 16 columns of 128, take 106 us, 5.0 TB/s.)
int64_t attend_columns(const AttParams& p) { return (int64_t(p.c.rows) * p.group + p.c.seqs - 1) / p.c.seqs; }
template <int D, bool SHARED>
cudaError_t launch_attend_for(const AttParams& p, int sms, cudaStream_t s) {
    const int64_t columns = attend_columns(p);
    if (columns <= 8) return launch_attend<D, 1, SHARED>(p, sms, s);
    if (D == 256 || columns <= 24) return launch_attend<D, 2, SHARED>(p, sms, s);
    return launch_attend<D, att_most_columns<D>(), SHARED>(p, sms, s);
}
template <bool SHARED>
cudaError_t launch_attend_all(const AttParams& p, int D, int sms, cudaStream_t s) {
    return D == 64 ? launch_attend_for<64, SHARED>(p, sms, s) : D == 128 ? launch_attend_for<128, SHARED>(p, sms, s) : launch_attend_for<256, SHARED>(p, sms, s);
}

// Whether one launch in which each sequence reads all of its tokens may take longer than three that read shared ones once, if the table is full
// and shared by all: in bytes at 7.9 TB/s, a token and kv head are 2 D of them for an item of 8 columns, 1.75 times that of 16 and 2.7 of 32 (whose
// products bound it), and for a tile of k_kv_prefix what its steps take; two more launches are 63 MB, a row's pieces 40 times its queries.
// Measured with 32/8 heads, us apart and shared: heads of 128, 16 single tokens behind 1024 13.3 and 16.8, 2048 17.8 and 17.5, 4096 26.5 and 19.3; 64
// behind 512 23.2 and 25.3, 1024 30.8 and 26.2; 64 times 5 rows behind 512 39 and 50, 1024 55.5 and 53.2; 2 tokens behind 65536 41 and 62, 4 behind
// 16384 26.2 and 26.7; heads of 64, 4 behind 32768 27 and 34; heads of 256, 2 behind 32768 44 and 50.  Of 312 calls the better one is missed by
// 1.2 % on average, 23 % at worst.
bool worth_sharing(const AttParams& p, int D) {
    const int64_t columns = attend_columns(p), item = columns <= 8 ? 8 : D == 256 || columns <= 24 ? 16 : 32, all = int64_t(p.c.rows) * p.group;
    const double apart = double(p.c.seqs * ((columns + item - 1) / item)) * (item == 8 ? 1. : item == 16 ? 1.75 : 2.7) * (2 * D);
    const double shared = D < 256 && all <= kPreColumns ? (D == 64 ? 576. : 712.) : (D == 64 ? 800. : 1040.) * double((all + pre_tile(D) - 1) / pre_tile(D));
    const double tokens = double(p.c.kv_heads) * p.c.width * p.c.blocks_per_page * kKvBlock, queries = double(all) * p.c.kv_heads * D * 2;
    return (apart - shared) * tokens >= 63e6 + 40. * queries;
}

// What both calls check, in the order in which they say so.
int attend_params(const tetra_kv_cache* cache, const void* q, int64_t q_stride, void* out, int rows, int q_heads, float scale, void* workspace, size_t workspace_bytes,
                  size_t wanted_bytes, AttParams& p) {
    const int rc = kv_check(cache, rows, p.c);
    if (rc != TETRA_OK) return rc;
    const int D = cache->head_dim;
    if (!q || !out || !workspace) return TETRA_ERR_NULL;
    if (q_heads < 1 || q_heads % p.c.kv_heads || q_heads > 4096 || q_stride < int64_t(q_heads) * D) return TETRA_ERR_SHAPE;
    p.scale = scale * 1.4426950408889634f;  // times log2 e
    if (!std::isfinite(p.scale) || int64_t(cache->seqs) * rows * q_heads > (1ll << 32)) return TETRA_ERR_SHAPE;
    if (!kv_aligned(q, 16) || q_stride % 8 || !kv_aligned(out, 16) || !kv_aligned(workspace, 256)) return TETRA_ERR_ALIGN;
    if (workspace_bytes < wanted_bytes) return TETRA_ERR_SIZE;
    p.q = static_cast<const __half*>(q);
    p.out = static_cast<__half*>(out);
    p.q_stride = q_stride;
    p.group = q_heads / p.c.kv_heads;
    p.unit_shift = 0;
    p.arrived = static_cast<uint32_t*>(workspace);
    p.pieces = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + kAttCounters);
    p.shared = SharedGroups{nullptr, nullptr, 0};
    p.own = nullptr;
    p.own_ends = 0;
    p.owns = nullptr;
    p.runs_most = 0;
    return TETRA_OK;
}

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" {

size_t tetra_kv_workspace_bytes(int head_dim) {
    return head_dim == 64 ? att_workspace<64>() : head_dim == 128 ? att_workspace<128>() : head_dim == 256 ? att_workspace<256>() : 0;
}

int tetra_kv_attend(const tetra_kv_cache* cache, const void* q, int64_t q_stride, void* out, int rows, int q_heads, float scale, void* workspace,
                    size_t workspace_bytes, void* stream) {
    AttParams p;
    const int rc = attend_params(cache, q, q_stride, out, rows, q_heads, scale, workspace, workspace_bytes, cache ? tetra_kv_workspace_bytes(cache->head_dim) : 0, p);
    if (rc != TETRA_OK || rows == 0) return rc;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) return TETRA_ERR_CUDA;
    return kv_status(launch_attend_all<false>(p, cache->head_dim, sms, static_cast<cudaStream_t>(stream)));
}

size_t tetra_kv_shared_workspace_bytes(int head_dim, int rows, int q_heads, int kv_heads, int groups) {
    if (tetra_kv_workspace_bytes(head_dim) == 0 || rows < 0 || rows > TETRA_KV_MAX_ROWS || kv_heads < 1 || kv_heads > 1024 || q_heads < 1 || q_heads > 4096 ||
        q_heads % kv_heads || groups < 0 || groups > TETRA_KV_MAX_SEQS)
        return 0;
    return SharedPlaces(head_dim, rows, q_heads, kv_heads, groups).end;
}

int tetra_kv_attend_shared(const tetra_kv_cache* cache, const tetra_kv_groups* groups, const void* q, int64_t q_stride, void* out, int rows, int q_heads, float scale,
                           void* workspace, size_t workspace_bytes, void* stream) {
    AttParams p;
    if (!groups || (groups->groups > 0 && (!groups->group_start || !groups->shared))) return TETRA_ERR_NULL;
    if (groups->groups < 0 || groups->groups > TETRA_KV_MAX_SEQS) return TETRA_ERR_SHAPE;
    if (!kv_aligned(groups->group_start, 4) || !kv_aligned(groups->shared, 4)) return TETRA_ERR_ALIGN;
    const size_t wanted = cache ? tetra_kv_shared_workspace_bytes(cache->head_dim, rows, q_heads, cache->kv_heads, groups->groups) : 0;
    const int rc = attend_params(cache, q, q_stride, out, rows, q_heads, scale, workspace, workspace_bytes, wanted, p);
    if (rc != TETRA_OK || rows == 0) return rc;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) return TETRA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int D = cache->head_dim;
    if (groups->groups == 0 || !worth_sharing(p, D)) return kv_status(launch_attend_all<false>(p, D, sms, s));
    const SharedPlaces at(D, rows, q_heads, cache->kv_heads, groups->groups);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    SharedCall call;
    call.c = p.c;
    call.g = SharedGroups{groups->group_start, groups->shared, groups->groups};
    call.q = p.q;
    call.out = p.out;
    call.q_stride = q_stride;
    call.scale = p.scale;
    call.group = p.group;
    call.seqs = reinterpret_cast<SharedSeq*>(ws + at.seqs);
    call.own = reinterpret_cast<float*>(ws + at.own);
    call.runs = attend_columns(p) <= 8;
    call.own_ends = (call.runs ? int64_t(at.runs) * 8 : int64_t(rows) * q_heads) * D;
    call.owns = reinterpret_cast<OwnSeq*>(ws + at.owns);
    call.pieces = reinterpret_cast<float*>(ws + at.pieces);
    call.most = uint32_t(at.parts);
    p.shared = call.g;
    p.own = call.own;
    p.own_ends = call.own_ends;
    p.owns = call.owns;
    p.runs_most = uint32_t(at.runs);
    cudaError_t e = launch_prefix(call, D, sms, s);
    if (e == cudaSuccess) e = launch_attend_all<true>(p, D, sms, s);
    if (e == cudaSuccess) e = launch_join(call, D, s);
    return kv_status(e);
}

}  // extern "C"
