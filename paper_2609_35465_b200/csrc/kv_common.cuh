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

inline int kv_status(cudaError_t e) { return e == cudaSuccess ? TETRA_OK : TETRA_ERR_CUDA; }

}  // namespace
}  // namespace tetra
