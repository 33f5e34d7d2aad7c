/*
 * tetra_kv.h -- C ABI of the keys and values of a served model: a paged cache in 8 bits and the attention over it.
 *
 * Between the products of a decode step (tetra.h, tetra_q4.h) stand the attention and its cache.  New rows of the
 * projections (float32, as the products write them) are normalised per head, rotated and appended; the attention of
 * the step's rows over everything before them gives float16 activations for the next product.
 *
 * Conventions are those of tetra.h (status codes, device/host pointers, stream, validation before launch; a rejected
 * call launches nothing).  All of these kernels wait for the end of the kernels before them on the stream before
 * they read or write anything, so their operands may come from any call; what they write may be used as activations
 * as it is.  No result depends on the order in which threads run: every output is bit-identical from run to run.
 *
 * Cache.  Tokens are kept in blocks of 16; a page is page_tokens / 16 blocks; cache[pages][kv_heads][page_tokens/16]
 * holds one record of 32 D + 16 bytes for each page, head and block:
 *   keys    16 D bytes   token t, dim d at (d/32) 512 + ((t%8) 4 + d%32/8) 16 + (t/8) 8 + d%8
 *   values  16 D bytes   token t, dim d at (d/32) 512 + ((d%32/4) 4 + t%8/2) 16 + (d%4) 4 + (t/8) 2 + t%2
 *   scales  2 float32    s_K, s_V, and 8 bytes that are not used
 * A byte holds code + 128, code in [-127, 127]; the value it stands for is code * scale.  (The orders are those in
 * which the lanes of a warp hold the operands of a tensor-core product: a lane's bytes are contiguous.)
 * tetra_kv_append writes powers of two as scales, the attention takes any finite scale that is not
 * negative.
 *
 * Rows.  A step has `rows` rows of q, k and v.  Those of sequence s are row_start[s] .. row_start[s+1] - 1, its
 * next tokens in order; lengths[s] tokens of it are in the cache before this step, so row row_start[s] + i is at
 * position lengths[s] + i, and position p is in page page_table[s][p / page_tokens].  A sequence may have no rows.
 * Rows behind row_start[seqs] belong to nobody: what they would produce is left as it is.  row_start does not decrease;
 * a sequence whose range is not 0 <= row_start[s] <= row_start[s+1] <= rows counts as one without rows.  A position below zero (lengths
 * below zero: a slot without a sequence), a position at or behind width * page_tokens, and one whose page number is
 * not in [0, pages) has no place: nothing is stored there, nothing is read from there, and it has no part in an
 * attention.  None of that is an error the host can see without a copy.  Sequences may share pages for reading, and a
 * page may stand in a sequence twice; a block that rows are appended to must stand at one place of one sequence.
 */
#ifndef TETRA_KV_H
#define TETRA_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    TETRA_KV_BLOCK = 16,      /* tokens that share a scale */
    TETRA_KV_MAX_SEQS = 1024, /* sequences of one call */
    TETRA_KV_MAX_ROWS = 65536 /* rows of one call */
};

/* A cache and the step's sequences.  cache: 16-byte aligned; page_table int32 [seqs][table_stride], of which `width`
 * entries a row are used; row_start int32 [seqs + 1]; lengths int32 [seqs]; all device memory.  page_tokens: a
 * multiple of 16; kv_heads: up to 1024 (query heads: up to 4096); head_dim: 64, 128 or 256; 1 <= seqs <=
 * TETRA_KV_MAX_SEQS; width * page_tokens below 2^31. */
typedef struct {
    void *cache;
    const int32_t *page_table;
    const int32_t *row_start;
    const int32_t *lengths;
    int64_t table_stride;
    int32_t pages, page_tokens, kv_heads, head_dim, seqs, width;
} tetra_kv_cache;

/* New rows.  q [rows][q_heads][head_dim], k and v [rows][kv_heads][head_dim], float32 (half_type 0) or float16
 * (half_type 1); rows lie *_stride elements apart (they may be slices of one buffer), a row's heads are contiguous.
 * q and q_out may be NULL together: then only the cache is written.  q_out: float16 [rows][q_heads][head_dim].
 * q_weight, k_weight: float32 [head_dim] or NULL; inv_freq: float64 [head_dim / 2] or NULL. */
typedef struct {
    const void *q, *k, *v;
    void *q_out;
    const double *inv_freq;
    const float *q_weight, *k_weight;
    int64_t q_stride, k_stride, v_stride;
    double eps;
    int32_t rows, q_heads, half_type;
} tetra_kv_rows;

/* Bytes of a cache; 0 for a shape that is rejected. */
size_t tetra_kv_cache_bytes(int pages, int page_tokens, int kv_heads, int head_dim);

/* Appends the rows' keys and values and makes the queries of the attention, in one launch.  For a head's row x at
 * position p, in 64 bits:
 *   x <- x / sqrt(mean x^2 + eps) * weight         q and k, where q_weight / k_weight is given
 *   (x_i, x_{i+D/2}) <- turned by p * inv_freq[i]   q and k, where inv_freq is given
 * q is rounded to float16 once; k to float32.  A block's scale becomes s = max(its scale so far, the smallest power of
 * two >= 2^-126 with |x| <= 127 s for all its new elements) -- so far: 0 where no token of the block is in the cache
 * yet --, new codes are rint(x / s), and where the scale grew the codes before become rint(code * s_old / s)
 * (ties to even).  So a cache does not depend on how its tokens were cut into calls, but for the rounding of that
 * last step.  Magnitudes below 2^-126 count as zero.  A block that gets an infinite or NaN element has the scale NaN from then on, and codes of zero: what
 * attends to it is NaN, other blocks are untouched. */
int tetra_kv_append(const tetra_kv_cache *cache, const tetra_kv_rows *rows, void *stream);

/* What the cache holds for the rows' positions, as values: k_out, v_out float16 [rows][kv_heads][head_dim] (16-byte
 * aligned), code * scale rounded once; zero for a position without a place.  The rows are given by row_start and
 * lengths alone: reading a whole sequence takes lengths 0 and as many rows as it has tokens. */
int tetra_kv_read(const tetra_kv_cache *cache, void *k_out, void *v_out, int rows, void *stream);

/* Bytes of the workspace of tetra_kv_attend; 0 for a head_dim that is rejected.  The caller zeroes it once; every call
 * leaves its counters zero again.  Calls that share it must not overlap on the GPU. */
size_t tetra_kv_workspace_bytes(int head_dim);

/* out[r][n] = sum_p softmax_p(scale * q[r][n] . k[p][n / (q_heads / kv_heads)]) v[p][...] over the positions
 * p <= lengths[s] + i that have a place, for row r = row_start[s] + i; zero for a row that has none.  The rows' own
 * keys and values are in the cache already (tetra_kv_append with the same row_start and lengths).  out may be q, where
 * its rows are contiguous.
 * q: float16, rows q_stride elements apart, 16-byte aligned, q_stride a multiple of 8; out: float16
 * [rows][q_heads][head_dim], 16-byte aligned; q_heads a multiple of kv_heads; seqs * rows * q_heads up to 2^32; scale below
 * 2^127 in size.  One launch.  Products are of float16 values that are exact but for the weights, which are rounded to float16 next to a
 * running maximum of weight times scale; sums are float32, scores of any size that it holds among them (scale * s_K has to be a
 * float32 number too).  Any number of rows a sequence is right; the kernel is made for up to 16 (a step's mixture of such and of
 * single tokens is right too, but has one kernel for all, by the average). */
int tetra_kv_attend(const tetra_kv_cache *cache, const void *q, int64_t q_stride, void *out, int rows, int q_heads,
                    float scale, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
