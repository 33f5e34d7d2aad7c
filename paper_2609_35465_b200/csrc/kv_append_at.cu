// New rows into the key/value cache at given positions of several axes (tetra_kv_append_at).
//
// As tetra_kv_append, but a pair is turned by the row's position on the pair's axis, and that has nothing to do with the row's slot.
// A picture comes as one call of some thousand rows, so work is cut by blocks, not rows: a CTA per (block of 16 slots, kv head) makes
// its rows' sines once for the block's keys and all queries of the head group.  Rows of a chat's step are a block each.
#include <type_traits>

#include "kv_rows.cuh"

namespace tetra {
namespace {

struct KvAxes {
    const int32_t* positions;  // [row][axes]
    const uint8_t* axis;       // [D / 2]
    int64_t stride;
    int32_t axes;
};

// Block number `at` among the blocks that the call's rows fall in, sequence after sequence: its sequence and the first of its rows.  A
// warp looks at 32 sequences at a time.
__device__ __forceinline__ int block_of(const KvCache& c, int at, int lane, int& r, int& a, int& b, int64_t& before) {
    for (int s0 = 0; s0 < c.seqs; s0 += 32) {
        const int s = s0 + lane;
        int x = 0, y = 0, own = 0;
        int64_t len = 0;
        if (s < c.seqs) {
            c.rows_of(s, x, y);
            len = __ldg(c.lengths + s);
            if (y > x) own = int(((len + (y - x - 1)) >> 4) - (len >> 4)) + 1;
        }
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, at < sum);
        if (who) {
            const int l = __ffs(who) - 1;
            a = __shfl_sync(0xFFFFFFFFu, x, l);
            b = __shfl_sync(0xFFFFFFFFu, y, l);
            before = __shfl_sync(0xFFFFFFFFu, len, l);
            const int local = at - (__shfl_sync(0xFFFFFFFFu, sum, l) - __shfl_sync(0xFFFFFFFFu, own, l));
            r = local == 0 ? a : a + int((((before >> 4) + local) << 4) - before);
            return s0 + l;
        }
        at -= __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    return -1;
}

// BLOCKS: a CTA for each block; else one for each row, of which the first of a block does its work.
template <int D, typename T, bool BLOCKS>
__global__ void __launch_bounds__(kAppendThreads) k_kv_append_at(KvCache c, KvRows p, KvAxes t) {
    constexpr int E = D / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    double2* turns = reinterpret_cast<double2*>(smem);  // [rows of the block][D / 2]
    __shared__ uint32_t amax[2];                        // keys, values
    pdl_wait();
    pdl_release();
    const int head = blockIdx.y, lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    if (threadIdx.x < 2) amax[threadIdx.x] = 0u;
    int r = blockIdx.x, a = 0, b = 0, s;
    int64_t before = 0;
    if (BLOCKS) {
        s = block_of(c, blockIdx.x, lane, r, a, b, before);
    } else {
        s = sequence_of(c, r, lane, a, b);
        if (s >= 0) before = __ldg(c.lengths + s);
    }
    if (s < 0) return;
    const int64_t slot = before + (r - a);
    const int first = int(slot & (kKvBlock - 1));
    if (!BLOCKS && r != a && first != 0) return;
    unsigned char* rec = c.record<D>(s, slot >> 4, head);
    const int rows = min(kKvBlock - first, b - r), n = rec ? rows : 0;
    for (int i = threadIdx.x; i < rows * (D / 2); i += kAppendThreads) {
        const int row = i / (D / 2), pair = i % (D / 2);
        const int axis = __ldg(t.axis + pair);
        const int at = axis < t.axes ? __ldg(t.positions + int64_t(r + row) * t.stride + axis) : 0;
        double sn, cs;
        sincospi(double(at) * __ldg(p.inv_freq + pair) * 0.318309886183790671538, &sn, &cs);  // 1 / pi
        turns[i] = make_double2(cs, sn);
    }
    __syncthreads();

    // Tasks: the block's keys, then its values, a warp each; the queries from the other end of the warps.
    float x[kAppendTasks][E];
#pragma unroll
    for (int k = 0; k < kAppendTasks; ++k) {
        const int task = warp + kAppendWarps * k;
        if (task >= 2 * n) break;
        const bool key = task < n;
        const int row = key ? task : task - n;
        if (key) {
            double z[E];
            load_row<T>(p.k, (r + row) * p.k_stride + head * D, lane, x[k]);
            turn<E>(x[k], p.k_weight, p.eps, turns + row * (D / 2), lane, z);
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
    for (int j = kAppendWarps - 1 - warp; j < rows * p.group; j += kAppendWarps) {  // none without q
        const int row = j / p.group, h = head * p.group + j - row * p.group;
        float xq[E];
        double z[E];
        load_row<T>(p.q, (r + row) * p.q_stride + int64_t(h) * D, lane, xq);
        turn<E>(xq, p.q_weight, p.eps, turns + row * (D / 2), lane, z);
        __half* out = p.q_out + (int64_t(r + row) * c.kv_heads * p.group + h) * D;
#pragma unroll
        for (int i = 0; i < E; ++i) out[lane + 32 * i] = __double2half(z[i]);
    }
    if (!rec) return;
    finish_block<D>(rec, first, n, amax, x, lane, warp);
}

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" int tetra_kv_append_at(const tetra_kv_cache* cache, const tetra_kv_rows* rows, const tetra_kv_axes* axes, void* stream) {
    KvCache c;
    if (!rows || !axes) return TETRA_ERR_NULL;
    int rc = kv_check(cache, rows->rows, c);
    if (rc != TETRA_OK) return rc;
    const int D = cache->head_dim;
    KvRows p;
    rc = kv_check_rows(*rows, c, D, p);
    if (rc != TETRA_OK) return rc;
    if (!rows->inv_freq || !axes->positions || !axes->axis) return TETRA_ERR_NULL;
    if (axes->axes < 1 || axes->axes > TETRA_KV_MAX_AXES || axes->stride < axes->axes) return TETRA_ERR_SHAPE;
    if (!kv_aligned(axes->positions, 4)) return TETRA_ERR_ALIGN;
    if (c.rows == 0) return TETRA_OK;
    const KvAxes t{axes->positions, axes->axis, axes->stride, axes->axes};
    // Blocks that the rows may fall in: each sequence's, and one more where it begins inside one.
    const int64_t blocks = int64_t(c.rows) / kKvBlock + 2 * int64_t(c.seqs);
    const bool by_blocks = blocks < c.rows;
    auto launch = [&](auto kernel) {
        return launch_rows(kernel, by_blocks ? int(blocks) : c.rows, c.kv_heads, kAppendThreads, size_t(kKvBlock) * D / 2 * sizeof(double2), stream, c, p, t);
    };
    auto pick = [&](auto half, auto blocks_too) {
        using T = decltype(half);
        constexpr bool B = decltype(blocks_too)::value;
        return launch(D == 64 ? k_kv_append_at<64, T, B> : D == 128 ? k_kv_append_at<128, T, B> : k_kv_append_at<256, T, B>);
    };
    if (rows->half_type) return by_blocks ? pick(__half(), std::true_type()) : pick(__half(), std::false_type());
    return by_blocks ? pick(0.f, std::true_type()) : pick(0.f, std::false_type());
}
