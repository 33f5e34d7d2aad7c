// New rows of a step into the key/value cache (tetra_kv_append), and the cache's decoder (tetra_kv_read).
//
// Append.  One CTA per (row, kv head).  It makes that head group's queries, and where its row is the first that falls into
// a block of 16 tokens (the sequence's first row of the call, or a position that is a multiple of 16) it also brings
// all of the call's rows of that block into the block's record: a block has one writer, so its scale is found once and nothing
// depends on the order of CTAs.  A warp takes a head's row at a time, lane l its dims l, l + 32, ..: the two halves of
// a rotated pair lie in one lane.
// Norm and rotation are in 64 bits: a key next to the border of two codes, or of two scales, then goes where the
// formulas put it whatever the order of the sum of squares, and the angle of a far position (10^5 rad) keeps its fraction.
// A CTA makes its row's D / 2 float64 sines once for its queries and its key; each kv head's CTA makes them anew (32768 for 64 rows of
// 128 and 8 kv heads, where 4096 differ), and a block's first row makes those of the call's other rows of the block as well.
// That is cheap: the float64 pipe is 6 % busy.  Latency bounds the kernel: the row's sequence, its length, its page and the
// block's scales are loads that depend on one another (3.3 us for one row, 4.2 us for 64, 8 kv heads of 128).
#include "kv_rows.cuh"

namespace tetra {
namespace {

template <int D, typename T>
__global__ void __launch_bounds__(kAppendThreads) k_kv_append(KvCache c, KvRows p) {
    constexpr int E = D / 32, TASKS = kAppendTasks;
    extern __shared__ __align__(16) unsigned char smem[];
    double2* turns = reinterpret_cast<double2*>(smem);  // [rows of the block][D / 2]
    __shared__ uint32_t amax[2];                        // keys, values
    pdl_wait();
    pdl_release();
    const int r = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    // The first query of the warp: nothing that is looked up below decides where it lies.
    const int own = kAppendWarps - 1 - warp;
    float xq[E];
    if (own < p.group) load_row<T>(p.q, r * p.q_stride + int64_t(head * p.group + own) * D, lane, xq);
    if (threadIdx.x < 2) amax[threadIdx.x] = 0u;
    int a, b;
    const int s = sequence_of(c, r, lane, a, b);
    if (s < 0) return;
    const int64_t pos = int64_t(__ldg(c.lengths + s)) + (r - a);
    const int first = int(pos & (kKvBlock - 1));
    const bool leader = r == a || first == 0;
    unsigned char* rec = leader ? c.record<D>(s, pos >> 4, head) : nullptr;
    const int n = rec ? min(kKvBlock - first, b - r) : 0;  // rows of the call in this block
    if (p.inv_freq) {
        for (int i = threadIdx.x; i < max(n, 1) * (D / 2); i += kAppendThreads) {
            double sn, cs;
            sincospi(double(pos + i / (D / 2)) * __ldg(p.inv_freq + i % (D / 2)) * 0.318309886183790671538, &sn, &cs);  // 1 / pi
            turns[i] = make_double2(cs, sn);
        }
    }
    __syncthreads();

    // Tasks: the block's keys, then its values, a warp each; the queries from the other end of the warps.
    float x[TASKS][E];
#pragma unroll
    for (int k = 0; k < TASKS; ++k) {
        const int task = warp + kAppendWarps * k;
        if (task >= 2 * n) break;
        const bool key = task < n;
        const int row = key ? task : task - n;
        if (key) {
            double z[E];
            load_row<T>(p.k, (r + row) * p.k_stride + head * D, lane, x[k]);
            turn<E>(x[k], p.k_weight, p.eps, p.inv_freq ? turns + row * (D / 2) : nullptr, lane, z);
#pragma unroll
            for (int i = 0; i < E; ++i) x[k][i] = float(z[i]);
        } else {
            load_row<T>(p.v, (r + row) * p.v_stride + head * D, lane, x[k]);
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(x[k][i]) & 0x7FFFFFFFu);  // NaN is above infinity
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (lane == 0) atomicMax(&amax[key ? 0 : 1], top);
    }
    for (int j = own; j < p.group; j += kAppendWarps) {  // none without q
        const int h = head * p.group + j;
        if (j > own) load_row<T>(p.q, r * p.q_stride + int64_t(h) * D, lane, xq);
        double z[E];
        turn<E>(xq, p.q_weight, p.eps, p.inv_freq ? turns : nullptr, lane, z);
        __half* out = p.q_out + (int64_t(r) * c.kv_heads * p.group + h) * D;
#pragma unroll
        for (int i = 0; i < E; ++i) out[lane + 32 * i] = __double2half(z[i]);
    }
    if (!rec) return;

    finish_block<D>(rec, first, n, amax, x, lane, warp);
}

// Two warps per (row, kv head), or, where rows are many, per (block, kv head): those of the first row of a block write all of the call's rows of it, each half of the dims.
// A lane turns the bytes that it loads into the values that it stores: eight dims of two tokens, or four of four.
constexpr int kReadRows = 4;  // of a CTA

template <int D, bool BLOCKS>
__global__ void __launch_bounds__(64 * kReadRows) k_kv_read(KvCache c, __half* k_out, __half* v_out) {
    pdl_wait();
    pdl_release();
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0), g = lane >> 2, t = lane & 3;
    const int head = blockIdx.y, half = warp & 1;
    int r = blockIdx.x * kReadRows + (warp >> 1), a = 0, b = 0, s;
    int64_t before = 0;
    if (BLOCKS) {
        s = block_of(c, r, lane, r, a, b, before);
    } else {
        s = r < c.rows ? sequence_of(c, r, lane, a, b) : -1;
        if (s >= 0) before = __ldg(c.lengths + s);
    }
    if (s < 0) return;
    const int64_t pos = before + (r - a);
    const int first = int(pos & (kKvBlock - 1));
    if (!BLOCKS && r != a && first != 0) return;
    const int n = min(kKvBlock - first, b - r);
    const unsigned char* rec = c.record<D>(s, pos >> 4, head);
    constexpr int MINE = D / 64;  // chunks of 32 dims
    uint4 kw[MINE], vw[MINE];
    float ks = 0.f, vs = 0.f;
    if (rec) {
        const uint4* at = reinterpret_cast<const uint4*>(rec) + half * MINE * 32 + lane;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            kw[j] = at[j * 32];
            vw[j] = at[j * 32 + D];
        }
        const float2 scales = *reinterpret_cast<const float2*>(rec + 2 * kKvBlock * D);
        ks = scales.x;
        vs = scales.y;
    } else {
#pragma unroll
        for (int j = 0; j < MINE; ++j) kw[j] = vw[j] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
    }
    auto value = [](uint32_t word, int k, float scale) { return float(int(word >> (8 * k) & 255u) - 128) * scale; };
    auto pair = [](float x, float y) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    };
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
        const int d = (half * MINE + j) * 32;
        const uint32_t kb[4] = {kw[j].x, kw[j].y, kw[j].z, kw[j].w}, vb[4] = {vw[j].x, vw[j].y, vw[j].z, vw[j].w};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = g + 8 * i - first;
            if (row >= 0 && row < n)
                *reinterpret_cast<uint4*>(k_out + (size_t(r + row) * c.kv_heads + head) * D + d + 8 * t) =
                    make_uint4(pair(value(kb[2 * i], 0, ks), value(kb[2 * i], 1, ks)), pair(value(kb[2 * i], 2, ks), value(kb[2 * i], 3, ks)),
                               pair(value(kb[2 * i + 1], 0, ks), value(kb[2 * i + 1], 1, ks)), pair(value(kb[2 * i + 1], 2, ks), value(kb[2 * i + 1], 3, ks)));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 2 * t + (i & 1) + 8 * (i >> 1) - first;
            if (row >= 0 && row < n)
                *reinterpret_cast<uint2*>(v_out + (size_t(r + row) * c.kv_heads + head) * D + d + 4 * g) =
                    make_uint2(pair(value(vb[0], i, vs), value(vb[1], i, vs)), pair(value(vb[2], i, vs), value(vb[3], i, vs)));
        }
    }
}

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" {

size_t tetra_kv_cache_bytes(int pages, int page_tokens, int kv_heads, int head_dim) {
    if (!kv_shape_ok(pages, page_tokens, kv_heads, head_dim)) return 0;
    return size_t(pages) * kv_heads * (page_tokens / kKvBlock) * kv_record_bytes(head_dim);
}

int tetra_kv_append(const tetra_kv_cache* cache, const tetra_kv_rows* rows, void* stream) {
    KvCache c;
    if (!rows) return TETRA_ERR_NULL;
    int rc = kv_check(cache, rows->rows, c);
    if (rc != TETRA_OK) return rc;
    const int D = cache->head_dim;
    KvRows p;
    rc = kv_check_rows(*rows, c, D, p);
    if (rc != TETRA_OK || c.rows == 0) return rc;
    auto launch = [&](auto kernel) { return launch_rows(kernel, c.rows, c.kv_heads, kAppendThreads, p.inv_freq ? size_t(kKvBlock) * D / 2 * sizeof(double2) : 0, stream, c, p); };
    if (rows->half_type) return launch(D == 64 ? k_kv_append<64, __half> : D == 128 ? k_kv_append<128, __half> : k_kv_append<256, __half>);
    return launch(D == 64 ? k_kv_append<64, float> : D == 128 ? k_kv_append<128, float> : k_kv_append<256, float>);
}

int tetra_kv_read(const tetra_kv_cache* cache, void* k_out, void* v_out, int rows, void* stream) {
    KvCache c;
    const int rc = kv_check(cache, rows, c);
    if (rc != TETRA_OK) return rc;
    if (!k_out || !v_out) return TETRA_ERR_NULL;
    if (!kv_aligned(k_out, 16) || !kv_aligned(v_out, 16)) return TETRA_ERR_ALIGN;
    if (rows == 0) return TETRA_OK;
    const int D = cache->head_dim;
    // Many rows a sequence: by blocks (2949 rows of one, 8 kv heads: 21 us by rows).
    const int64_t blocks = kv_most_blocks(c);
    const bool by_blocks = 32 * int64_t(c.seqs) <= c.rows;
    const int items = by_blocks ? int(blocks) : c.rows;
    auto launch = [&](auto kernel) {
        return launch_rows(kernel, (items + kReadRows - 1) / kReadRows, c.kv_heads, 64 * kReadRows, 0, stream, c, static_cast<__half*>(k_out), static_cast<__half*>(v_out));
    };
    if (by_blocks) return launch(D == 64 ? k_kv_read<64, true> : D == 128 ? k_kv_read<128, true> : k_kv_read<256, true>);
    return launch(D == 64 ? k_kv_read<64, false> : D == 128 ? k_kv_read<128, false> : k_kv_read<256, false>);
}

}  // extern "C"
