// Attention of a step's rows over the 8-bit paged cache (tetra_kv_attend).
//
// A step has one or a few rows a sequence and reads each sequence's keys and values once: 2 D bytes a token and kv head
// against 4 D multiply-adds for each query head of the group, so HBM bounds it and the arrangement serves the stream.
//
// Work.  An item is (sequence, kv head, chunk of 8 NT columns); a column is one (row, query head of the group).  The
// blocks of 16 tokens of all items form one sequence of units that the CTAs of a persistent grid cut into equal
// contiguous ranges, whatever the lengths: a CTA finds its range from a prefix sum over the sequences that each CTA makes for
// itself (lengths are on the device and change from step to step of a captured graph).  Of its part of an item the eight
// warps take every eighth record; each warp streams its records through a cp.async ring of its own that goes on over the
// ends of items.  A lane copies the very bytes that it will use, so nothing but a warp-wide fence stands between
// a copy and its use.  The warps' sums meet in shared memory; an item cut by ranges leaves a piece per CTA in the
// workspace, and the CTA that finds the others there adds them in order of the CTAs.  Nothing waits for another CTA.
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
#include <cmath>

#include "kv_common.cuh"

namespace tetra {
namespace {

constexpr int kAttThreads = 256, kAttWarps = kAttThreads / 32;
constexpr int kAttSegs = 32;              // parts of items that a CTA looks up at a time
constexpr int kAttMaxCtas = 512;          // of a launch: pieces in the workspace
constexpr float kNoRef = -1e30f;          // reference of a column that has seen nothing
constexpr float kLeastLog = -60.f;        // log2 of the least s_V that counts: 127 * 2^-60 is zero in float16
constexpr float kHigh = 15.f, kBase = 7.f; // a weight reaches 2^kHigh at most, a new reference puts the largest at 2^kBase

template <int D, int NT>
struct AttCfg {
    static constexpr int REC = kv_record_bytes(D);
    static constexpr int CHUNKS = D / 32;                      // 512-byte chunks of the keys, and of the values
    static constexpr int FRAGS = NT * D / 16;                  // accumulators, four floats a lane each
    static constexpr int STAGES = D == 64 ? 4 : 2;
    static constexpr int CTAS = D == 256 || (D == 128 && NT == 4) ? 1 : 2;  // of an SM
    static constexpr int RING = kAttWarps * STAGES * REC;
    static constexpr int MERGE = kAttWarps / 2 * 32 * (FRAGS * 16 + NT * 16);
    static constexpr int QBYTES = NT > 1 ? NT * CHUNKS * 512 : 0;
    static constexpr int PIECE = 32 * (FRAGS * 4 + NT * 4);    // floats of a piece in the workspace
    static constexpr int SMEM = RING + MERGE + QBYTES;          // and 8 bytes a sequence
};

// A CTA's part of an item.
struct Seg {
    int32_t seq, head;
    int32_t row0;          // first row of the sequence
    int32_t col0, cols;    // the item's first column, and the sequence's columns
    uint32_t r0, r1;       // blocks, of those that the item's last row sees
    int32_t first, last;   // CTAs that the item begins and ends in
    int64_t before;        // tokens before the step
};

struct AttParams {
    KvCache c;
    const __half* q;
    __half* out;
    int64_t q_stride;
    float scale;           // times log2 e
    int32_t group;
    float* pieces;         // [CTA][2][PIECE]
    uint32_t* arrived;     // [CTA]: pieces of the item that begins in this CTA and ends beyond it
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

// The sequence's columns, chunks of them, and blocks that its last row sees (one at least, so that an item without a
// token is somebody's work: its rows are zero).
template <int NT>
__device__ __forceinline__ void sequence_work(const AttParams& p, int s, int& a, int& rows, int64_t& before, uint32_t& chunks, uint32_t& blocks) {
    int b;
    p.c.rows_of(s, a, b);
    rows = b - a;
    before = __ldg(p.c.lengths + s);
    chunks = (uint32_t(rows) * p.group + 8 * NT - 1) / (8 * NT);
    const int64_t most = int64_t(p.c.width) * p.c.blocks_per_page, seen = before + rows;
    const int64_t n = seen <= 0 ? 0 : (seen + kKvBlock - 1) / kKvBlock;
    blocks = uint32_t(n < 1 ? 1 : n > most ? most : n);
}

// Column (of the sequence) -> row of the step and query head; its last position.
__device__ __forceinline__ int64_t column_at(const AttParams& p, const Seg& g, int col, int heads_all, int D) {
    const int row = col / p.group, h = col % p.group;
    return (int64_t(g.row0 + row) * heads_all + g.head * p.group + h) * D;
}

template <int D, int NT>
__global__ void __launch_bounds__(kAttThreads, AttCfg<D, NT>::CTAS) k_kv_attend(AttParams p) {
    using C = AttCfg<D, NT>;
    constexpr int CHUNKS = C::CHUNKS, STAGES = C::STAGES, REC = C::REC, FRAGS = C::FRAGS;
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* ring = smem;
    float4* merge = reinterpret_cast<float4*>(smem + C::RING);                             // [warps / 2][FRAGS + NT][32]
    unsigned char* qs = smem + C::RING + C::MERGE;                                         // [NT][CHUNKS][32][16 bytes]
    uint64_t* prefix = reinterpret_cast<uint64_t*>(smem + C::RING + C::MERGE + C::QBYTES); // [seqs + 1]
    __shared__ Seg segs[kAttSegs];
    __shared__ int nsegs, cursor_seq;
    __shared__ uint64_t cursor_unit, range_end, share_units, warp_sums[kAttWarps];
    __shared__ uint32_t is_last;

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int heads = p.c.kv_heads, heads_all = heads * p.group;
    pdl_wait();
    pdl_release();

    // Prefix sum of the sequences' units.
    {
        const int per = (p.c.seqs + kAttThreads - 1) / kAttThreads, s0 = threadIdx.x * per;
        uint64_t mine = 0;
        uint64_t own[TETRA_KV_MAX_SEQS / kAttThreads];
#pragma unroll
        for (int i = 0; i < TETRA_KV_MAX_SEQS / kAttThreads; ++i) {
            own[i] = 0;
            if (i < per && s0 + i < p.c.seqs) {
                int a, rows;
                int64_t before;
                uint32_t chunks, blocks;
                sequence_work<NT>(p, s0 + i, a, rows, before, chunks, blocks);
                own[i] = uint64_t(chunks) * heads * blocks;
            }
            mine += own[i];
        }
        uint64_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) warp_sums[warp] = sum;
        __syncthreads();
        uint64_t at = sum - mine;
        for (int w = 0; w < warp; ++w) at += warp_sums[w];
#pragma unroll
        for (int i = 0; i < TETRA_KV_MAX_SEQS / kAttThreads; ++i) {
            if (i < per && s0 + i < p.c.seqs) prefix[s0 + i] = at;
            at += own[i];
        }
        if (threadIdx.x == kAttThreads - 1) prefix[p.c.seqs] = at;
        __syncthreads();
    }
    const uint64_t units = prefix[p.c.seqs];
    const uint64_t share = max(uint64_t(2 * kAttWarps), (units + gridDim.x - 1) / gridDim.x);
    const uint64_t begin = share * blockIdx.x;
    if (begin >= units) return;
    for (int s = threadIdx.x; s < p.c.seqs; s += kAttThreads)
        if (prefix[s] <= begin && begin < prefix[s + 1]) cursor_seq = s;
    if (threadIdx.x == 0) {
        cursor_unit = begin;
        range_end = min(units, begin + share);
        share_units = share;
    }
    __syncthreads();

    const uint32_t my_ring = smem_u32(ring) + warp * STAGES * REC, lane16 = lane * 16;
    for (;;) {
        // The next parts of items of this CTA's range.
        if (threadIdx.x == 0) {
            int n = 0, s = cursor_seq;
            uint64_t u = cursor_unit;
            const uint64_t end = range_end;
            while (n < kAttSegs && u < end) {
                while (u >= prefix[s + 1]) ++s;
                int a, rows;
                int64_t before;
                uint32_t chunks, blocks;
                sequence_work<NT>(p, s, a, rows, before, chunks, blocks);
                uint64_t item = (u - prefix[s]) / blocks;
                while (n < kAttSegs && u < end && u < prefix[s + 1]) {
                    const uint64_t at = prefix[s] + item * blocks;
                    Seg& q = segs[n++];
                    q.seq = s;
                    q.head = int(item / chunks);
                    q.row0 = a;
                    q.col0 = int(item % chunks) * 8 * NT;
                    q.cols = rows * p.group;
                    q.before = before;
                    q.first = int(at / share);
                    q.last = int((at + blocks - 1) / share);
                    const uint32_t r0 = uint32_t(u - at), r1 = uint32_t(min(uint64_t(blocks), end - at));
                    const int64_t seen = before + (min(q.col0 + 8 * NT, q.cols) - 1) / p.group + 1;  // of the item's last row
                    const int64_t nb = seen <= 0 ? 0 : (seen + kKvBlock - 1) / kKvBlock;
                    q.r0 = r0;
                    q.r1 = nb < r1 ? uint32_t(nb) : r1;
                    u = at + r1;
                    ++item;
                }
            }
            nsegs = n;
            cursor_seq = s;
            cursor_unit = u;
        }
        __syncthreads();
        const int count = nsegs;
        if (count == 0) return;

        // The warp's stream of records over these parts: what is copied next (its page number is loaded a record ahead).
        int ahead_seg = -1;
        uint32_t ahead_rec = 0, ahead_end = 0;
        const unsigned char* ahead_at = nullptr;
        auto advance = [&] {
            ahead_rec += kAttWarps;
            while (ahead_rec >= ahead_end) {
                if (++ahead_seg >= count) {
                    ahead_seg = count;
                    ahead_at = nullptr;
                    return;
                }
                ahead_rec = segs[ahead_seg].r0 + warp;
                ahead_end = segs[ahead_seg].r1;
            }
            ahead_at = p.c.template record<D>(segs[ahead_seg].seq, ahead_rec, segs[ahead_seg].head);
        };
        uint32_t placed = 0;  // bit per stage: its record has a place
        int stage = 0;
        auto issue = [&](int to) {
            placed &= ~(1u << to);
            if (ahead_seg < count) {
                if (ahead_at) {
                    placed |= 1u << to;
                    const uint32_t dst = my_ring + to * REC;
#pragma unroll
                    for (int j = 0; j < 2 * CHUNKS; ++j) copy16(dst + j * 512 + lane16, ahead_at + j * 512 + lane16);
                    if (lane == 0) copy16(dst + 2 * CHUNKS * 512, ahead_at + 2 * CHUNKS * 512);
                }
                advance();
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        advance();
#pragma unroll
        for (int i = 0; i < STAGES; ++i) issue(i);

        for (int i = 0; i < count; ++i) {
            const Seg& sg = segs[i];
            // Queries: lane (g, t) holds column g's dims 32 j + 8 t .. + 7 of every chunk j.
            uint4 qr[NT == 1 ? CHUNKS : 1];
            if (NT == 1) {
                const int col = sg.col0 + g;
                const bool live = col < sg.cols;
                const __half* src = p.q + int64_t(sg.row0 + (live ? col : 0) / p.group) * p.q_stride + (sg.head * p.group + (live ? col : 0) % p.group) * D + 8 * t;
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) qr[j] = live ? __ldg(reinterpret_cast<const uint4*>(src + 32 * j)) : make_uint4(0, 0, 0, 0);
            } else {
                for (int k = threadIdx.x; k < NT * CHUNKS * 32; k += kAttThreads) {
                    const int l = k & 31, j = k / 32 % CHUNKS, col = sg.col0 + k / (32 * CHUNKS) * 8 + (l >> 2);
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (col < sg.cols)
                        v = __ldg(reinterpret_cast<const uint4*>(p.q + int64_t(sg.row0 + col / p.group) * p.q_stride + (sg.head * p.group + col % p.group) * D + 32 * j + 8 * (l & 3)));
                    reinterpret_cast<uint4*>(qs)[k] = v;
                }
                __syncthreads();
            }
            // Last position of the lane's columns (2 t, 2 t + 1 of each eight).
            int64_t sees[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k) sees[nt][k] = sg.before + (sg.col0 + nt * 8 + 2 * t + k) / p.group;
            const int64_t all_see = sg.before + sg.col0 / p.group;  // the item's first row

            float o[FRAGS][4], ref[NT][2], sum[NT][2];
#pragma unroll
            for (int f = 0; f < FRAGS; ++f)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[f][k] = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) ref[nt][0] = ref[nt][1] = kNoRef, sum[nt][0] = sum[nt][1] = 0.f;

            for (uint32_t rec = sg.r0 + warp; rec < sg.r1; rec += kAttWarps) {
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
                __syncwarp();  // the scales were copied by lane 0
                if (placed >> stage & 1u) {
                    const uint32_t at = my_ring + stage * REC;
                    const uint4 scales = lds_uint4(at + 2 * CHUNKS * 512);
                    const float by = __uint_as_float(scales.x) * p.scale, vs = __uint_as_float(scales.y);
                    float lv = lg2(vs);
                    lv = lv < kLeastLog ? kLeastLog : lv;  // NaN stays
                    float x[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[nt][k] = 0.f;
#pragma unroll
                    for (int j = 0; j < CHUNKS; ++j) {
                        const uint4 w = lds_uint4(at + j * 512 + lane16);
                        const uint32_t a0 = codes_of<false>(w.x), a2 = codes_of<true>(w.x), a1 = codes_of<false>(w.z), a3 = codes_of<true>(w.z);
                        const uint32_t c0 = codes_of<false>(w.y), c2 = codes_of<true>(w.y), c1 = codes_of<false>(w.w), c3 = codes_of<true>(w.w);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint4 b = NT == 1 ? qr[j] : reinterpret_cast<const uint4*>(qs)[(nt * CHUNKS + j) * 32 + lane];
                            mma16816(x[nt], a0, a1, a2, a3, b.x, b.y);
                            mma16816(x[nt], c0, c1, c2, c3, b.z, b.w);
                        }
                    }
                    const int64_t token = int64_t(rec) * kKvBlock + g;  // and 8 on
                    bool over = false;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[nt][k] *= by;
                    if (int64_t(rec) * kKvBlock + kKvBlock - 1 > all_see) {  // the last blocks: some column does not see all of it
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (token + (k >> 1) * 8 > sees[nt][k & 1]) x[nt][k] = -INFINITY;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        over |= fmaxf(x[nt][0], x[nt][2]) + lv > ref[nt][0] + kHigh || fmaxf(x[nt][1], x[nt][3]) + lv > ref[nt][1] + kHigh;
                    if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                float top = fmaxf(x[nt][k], x[nt][k + 2]);
#pragma unroll
                                for (int m = 4; m <= 16; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
                                const float now = top + lv - kBase;
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

            // The warps' sums become one, halving the number of warps at a time, in a fixed order.
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int m = 4; m <= 16; m <<= 1) sum[nt][k] += __shfl_xor_sync(0xFFFFFFFFu, sum[nt][k], m);
#pragma unroll 1
            for (int half = kAttWarps / 2; half >= 1; half >>= 1) {
                float4* slot = merge + (warp & (half - 1)) * (FRAGS + NT) * 32 + lane;
                if (warp >= half && warp < 2 * half) {
#pragma unroll
                    for (int f = 0; f < FRAGS; ++f) slot[f * 32] = make_float4(o[f][0], o[f][1], o[f][2], o[f][3]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) slot[(FRAGS + nt) * 32] = make_float4(ref[nt][0], ref[nt][1], sum[nt][0], sum[nt][1]);
                }
                __syncthreads();
                if (warp < half) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float4 v = slot[(FRAGS + nt) * 32];
                        const float r0 = fmaxf(ref[nt][0], v.x), r1 = fmaxf(ref[nt][1], v.y);
                        const float m0 = ex2(ref[nt][0] - r0), m1 = ex2(ref[nt][1] - r1), n0 = ex2(v.x - r0), n1 = ex2(v.y - r1);
                        ref[nt][0] = r0;
                        ref[nt][1] = r1;
                        sum[nt][0] = sum[nt][0] * m0 + v.z * n0;
                        sum[nt][1] = sum[nt][1] * m1 + v.w * n1;
#pragma unroll
                        for (int m = 0; m < D / 16; ++m) {
                            const int f = nt * (D / 16) + m;
                            const float4 u = slot[f * 32];
                            o[f][0] = o[f][0] * m0 + u.x * n0;
                            o[f][1] = o[f][1] * m1 + u.y * n1;
                            o[f][2] = o[f][2] * m0 + u.z * n0;
                            o[f][3] = o[f][3] * m1 + u.w * n1;
                        }
                    }
                }
                __syncthreads();
            }

            // Two of a fragment's values belong to column 2 t (2 t + 1) and dims d, d + 1.
            auto store = [&](int f, const float (&v)[4], float s0, float s1) {
                const int nt = f / (D / 16), m = f % (D / 16), d = m / 2 * 32 + 4 * g + (m & 1) * 2;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int col = sg.col0 + nt * 8 + 2 * t + k;
                    const float s = k ? s1 : s0, by = s == 0.f ? 0.f : 1.f / s;  // nothing seen: zero
                    if (col < sg.cols)
                        *reinterpret_cast<__half2*>(p.out + column_at(p, sg, col, heads_all, D) + d) = __floats2half2_rn(v[k] * by, v[k + 2] * by);
                }
            };
            if (sg.first == sg.last) {
                if (warp == 0) {
#pragma unroll
                    for (int f = 0; f < FRAGS; ++f) store(f, o[f], sum[f / (D / 16)][0], sum[f / (D / 16)][1]);
                }
            } else {
                // A piece of an item that several CTAs share: place 1 of the CTA that it begins in, place 0 of the others.
                const int me = blockIdx.x;
                if (warp == 0) {
                    float4* piece = reinterpret_cast<float4*>(p.pieces + (size_t(me) * 2 + (me == sg.first)) * C::PIECE) + lane;
#pragma unroll
                    for (int f = 0; f < FRAGS; ++f) __stcg(piece + f * 32, make_float4(o[f][0], o[f][1], o[f][2], o[f][3]));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) __stcg(piece + (FRAGS + nt) * 32, make_float4(ref[nt][0], ref[nt][1], sum[nt][0], sum[nt][1]));
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) {
                        const uint32_t others = uint32_t(sg.last - sg.first);
                        const uint32_t had = atomicAdd(p.arrived + sg.first, 1u);
                        is_last = had == others;
                        if (had == others) p.arrived[sg.first] = 0u;  // for the next call
                        __threadfence();
                    }
                }
                __syncthreads();
                if (is_last) {
                    const float4* pieces = reinterpret_cast<const float4*>(p.pieces) + lane;
                    constexpr int P4 = C::PIECE / 4;
                    for (int f = warp; f < FRAGS; f += kAttWarps) {
                        const int nt = f / (D / 16);
                        float r0 = kNoRef, r1 = kNoRef, s0 = 0.f, s1 = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                        for (int b = sg.first; b <= sg.last; ++b) {
                            const float4* at = pieces + (size_t(b) * 2 + (b == sg.first)) * P4;
                            const float4 u = __ldcg(at + f * 32), m = __ldcg(at + (FRAGS + nt) * 32);
                            const float q0 = fmaxf(r0, m.x), q1 = fmaxf(r1, m.y);
                            const float f0 = ex2(r0 - q0), f1 = ex2(r1 - q1), n0 = ex2(m.x - q0), n1 = ex2(m.y - q1);
                            r0 = q0;
                            r1 = q1;
                            s0 = s0 * f0 + m.z * n0;
                            s1 = s1 * f1 + m.w * n1;
                            v[0] = v[0] * f0 + u.x * n0;
                            v[1] = v[1] * f1 + u.y * n1;
                            v[2] = v[2] * f0 + u.z * n0;
                            v[3] = v[3] * f1 + u.w * n1;
                        }
                        store(f, v, s0, s1);
                    }
                }
                __syncthreads();  // is_last
            }
        }
        __syncthreads();  // segs
    }
}

constexpr int kAttCounters = kAttMaxCtas * 4;  // bytes
template <int D>
constexpr int att_most_columns() { return D == 256 ? 2 : 4; }
template <int D>
constexpr size_t att_workspace() { return size_t(kAttCounters) + size_t(kAttMaxCtas) * 2 * AttCfg<D, att_most_columns<D>()>::PIECE * 4; }

template <int D, int NT>
cudaError_t launch_attend(const AttParams& p, int sms, cudaStream_t s) {
    using C = AttCfg<D, NT>;
    constexpr int most = C::SMEM + 8 * (TETRA_KV_MAX_SEQS + 1);
    static PerDeviceOnce once;  // per instantiation
    cudaError_t e = once.run([] { return cudaFuncSetAttribute(k_kv_attend<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, most); });
    if (e != cudaSuccess) return e;
    const int grid = C::CTAS * sms < kAttMaxCtas ? C::CTAS * sms : kAttMaxCtas;
    return launch_pdl(k_kv_attend<D, NT>, grid, kAttThreads, size_t(C::SMEM) + 8 * (p.c.seqs + 1), s, p);
}

// Columns of an item by what a sequence has on average: more of them read a block's codes once for more rows, but an
// item with empty columns pays for all.
template <int D>
cudaError_t launch_attend_for(const AttParams& p, int sms, cudaStream_t s) {
    const int64_t columns = (int64_t(p.c.rows) * p.group + p.c.seqs - 1) / p.c.seqs;
    if (columns <= 8) return launch_attend<D, 1>(p, sms, s);
    if (D == 256 || columns <= 16) return launch_attend<D, 2>(p, sms, s);
    return launch_attend<D, att_most_columns<D>()>(p, sms, s);
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
    const int rc = kv_check(cache, rows, p.c);
    if (rc != TETRA_OK) return rc;
    const int D = cache->head_dim;
    if (!q || !out || !workspace) return TETRA_ERR_NULL;
    if (q_heads < 1 || q_heads % p.c.kv_heads || q_heads > 4096 || q_stride < int64_t(q_heads) * D) return TETRA_ERR_SHAPE;
    if (!std::isfinite(scale)) return TETRA_ERR_SHAPE;
    if (!kv_aligned(q, 16) || q_stride % 8 || !kv_aligned(out, 16) || !kv_aligned(workspace, 256)) return TETRA_ERR_ALIGN;
    if (workspace_bytes < tetra_kv_workspace_bytes(D)) return TETRA_ERR_SIZE;
    if (rows == 0) return TETRA_OK;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) return TETRA_ERR_CUDA;
    p.q = static_cast<const __half*>(q);
    p.out = static_cast<__half*>(out);
    p.q_stride = q_stride;
    p.scale = scale * 1.4426950408889634f;
    p.group = q_heads / p.c.kv_heads;
    p.arrived = static_cast<uint32_t*>(workspace);
    p.pieces = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + kAttCounters);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return kv_status(D == 64 ? launch_attend_for<64>(p, sms, s) : D == 128 ? launch_attend_for<128>(p, sms, s) : launch_attend_for<256>(p, sms, s));
}

}  // extern "C"
