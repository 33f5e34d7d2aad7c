// Pieces shared by the kernels of the key/value cache (include/tetra_kv.h): its geometry, checks of arguments, and which
// sequence a row belongs to.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/tetra.h"
#include "../../include/tetra_kv.h"
#include "tetra_gemv_common.cuh"

namespace tetra {
namespace {

constexpr int kKvBlock = TETRA_KV_BLOCK;
__host__ __device__ constexpr int kv_record_bytes(int D) { return 2 * kKvBlock * D + 16; }

struct KvCache {
    unsigned char* cache;
    const int32_t* table;
    const int32_t* row_start;
    const int32_t* lengths;
    int64_t table_stride;
    int32_t pages, blocks_per_page, kv_heads, seqs, width, rows;

    // The record of (sequence, block of tokens, head); nullptr where the block has no place.
    template <int D>
    __device__ __forceinline__ unsigned char* record(int s, int64_t block, int head) const {
        if (block < 0 || block >= int64_t(width) * blocks_per_page) return nullptr;
        const int page = __ldg(table + s * table_stride + uint32_t(block) / uint32_t(blocks_per_page));
        if (page < 0 || page >= pages) return nullptr;
        return cache + ((size_t(page) * kv_heads + head) * blocks_per_page + uint32_t(block) % uint32_t(blocks_per_page)) * kv_record_bytes(D);
    }
    // Rows [a, b) of a sequence; none where the ranges make no sense.
    __device__ __forceinline__ void rows_of(int s, int& a, int& b) const {
        a = __ldg(row_start + s);
        b = __ldg(row_start + s + 1);
        if (a < 0 || b > rows || b < a) b = a = 0;
    }
};

// The sequence of row r, or -1; its rows [a, b).  row_start does not decrease: a warp finds the place in two steps, among every
// so many entries and then among those between two of them.
static_assert(TETRA_KV_MAX_SEQS < 32 * 33, "two steps of 32 lanes");
__device__ __forceinline__ int sequence_of(const KvCache& c, int r, int lane, int& a, int& b) {
    const int entries = c.seqs + 1, stride = (entries + 31) / 32;
    int at = lane * stride;
    int s = __popc(__ballot_sync(0xFFFFFFFFu, at < entries && __ldg(c.row_start + at) <= r));
    if (s == 0) return -1;
    s = (s - 1) * stride;
    if (stride > 1) {
        at = s + 1 + lane;
        s += __popc(__ballot_sync(0xFFFFFFFFu, lane < stride - 1 && at < entries && __ldg(c.row_start + at) <= r));
    }
    if (s >= c.seqs) return -1;
    c.rows_of(s, a, b);
    return a <= r && r < b ? s : -1;
}

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

inline bool kv_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool kv_shape_ok(int pages, int page_tokens, int kv_heads, int D) {
    return pages > 0 && page_tokens > 0 && page_tokens % kKvBlock == 0 && page_tokens <= (1 << 20) && kv_heads > 0 && kv_heads <= 1024 &&
           (D == 64 || D == 128 || D == 256);
}

inline int kv_check(const tetra_kv_cache* c, int rows, KvCache& k) {
    if (!c || !c->cache || !c->page_table || !c->row_start || !c->lengths) return TETRA_ERR_NULL;
    if (!kv_shape_ok(c->pages, c->page_tokens, c->kv_heads, c->head_dim)) return TETRA_ERR_SHAPE;
    if (c->seqs < 1 || c->seqs > TETRA_KV_MAX_SEQS || c->width < 1 || c->table_stride < c->width) return TETRA_ERR_SHAPE;
    if (int64_t(c->width) * c->page_tokens > INT32_MAX) return TETRA_ERR_SHAPE;  // positions are 32-bit
    if (rows < 0 || rows > TETRA_KV_MAX_ROWS) return TETRA_ERR_SHAPE;
    if (!kv_aligned(c->cache, 16) || !kv_aligned(c->page_table, 4) || !kv_aligned(c->row_start, 4) || !kv_aligned(c->lengths, 4))
        return TETRA_ERR_ALIGN;
    k = KvCache{static_cast<unsigned char*>(c->cache), c->page_table, c->row_start, c->lengths, c->table_stride, c->pages,
                c->page_tokens / kKvBlock, c->kv_heads, c->seqs, c->width, rows};
    return TETRA_OK;
}

// Blocks that a call's rows may fall in: each sequence's, and one more where it begins inside one.
inline int64_t kv_most_blocks(const KvCache& c) { return int64_t(c.rows) / kKvBlock + 2 * int64_t(c.seqs); }

inline int kv_status(cudaError_t e) { return e == cudaSuccess ? TETRA_OK : TETRA_ERR_CUDA; }

}  // namespace
}  // namespace tetra
