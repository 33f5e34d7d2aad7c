/*
 * tetra_kv.h -- C ABI of the keys and values of a served model: a paged cache in 8 bits and the attention over it.
 *
 * Between the products of a decode step (tetra.h, tetra_q4.h) stand the attention and its cache.  New rows of the
 * projections (float32, as the products write them) are normalised per head, rotated and appended; the attention of
 * the step's rows over everything before them gives float16 activations for the next product.
 *
 * Conventions are those of tetra.h (status codes, device/host pointers, stream, validation before launch; a rejected
 * call launches nothing).  Every call waits for the end of the kernels before it on the stream before it reads or writes
 * anything, so its operands may come from any call; what it writes may be used as activations as it is.  (Of the three
 * kernels of tetra_kv_attend_shared the first one waits; the others start behind that wait, and the second one
 * reads, the third one looks up its rows, without one of their own.)  No result depends on the order in which threads run:
 * every output is bit-identical from run to run.
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
    TETRA_KV_MAX_ROWS = 65536, /* rows of one call */
    TETRA_KV_MAX_AXES = 8      /* axes of a row's position */
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

/* Positions apart from slots, on several axes (time, height and width of pictures): positions int32 [rows][axes], rows `stride`
 * elements apart; axis uint8 [head_dim / 2], below axes; device memory.  axes: 1 to TETRA_KV_MAX_AXES. */
typedef struct {
    const int32_t *positions;
    const uint8_t *axis;
    int64_t stride;
    int32_t axes;
} tetra_kv_axes;

/* tetra_kv_append, but for the angle: row r turns pair i by positions[r][axis[i]] * inv_freq[i], in 64 bits.  Positions may be
 * negative; an axis that is not below axes does not turn its pairs.  Where a row's key and value go is, as there, the next
 * slot of its sequence (row_start, lengths).  inv_freq is required.  One launch.
 * Queries of calls with more than two rows a sequence or so (rows - rows / 16 > 2 seqs) are turned in 32 bits, with sines that were made in 64 and
 * rounded: beside the rounding to float16, 2^-11 of a result, that moves each of a pair by 2^-20 of the two's sizes together at most.  Norms
 * hold for rows of any size, as there. */
int tetra_kv_append_at(const tetra_kv_cache *cache, const tetra_kv_rows *rows, const tetra_kv_axes *axes, void *stream);

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

/* Groups of sequences that begin with the same tokens (several answers to one prompt).  Group g is the sequences
 * group_start[g] .. group_start[g+1] - 1; their first shared[g] tokens have the same pages, that is, equal entries of
 * page_table.  group_start int32 [groups + 1], shared int32 [groups], device memory; groups up to TETRA_KV_MAX_SEQS, or none
 * (then both may be NULL).  group_start does not decrease; a group whose range is not 0 <= a <= b <= seqs counts as empty.  Sequences
 * may be in no group. */
typedef struct {
    const int32_t *group_start, *shared;
    int32_t groups;
} tetra_kv_groups;

/* Bytes of the workspace of tetra_kv_attend_shared for so many rows, heads and groups at most (more rows, groups or
 * query heads take no less); 0 for what is rejected.  As with tetra_kv_attend, the caller zeroes it once, and calls that share it must not overlap. */
size_t tetra_kv_shared_workspace_bytes(int head_dim, int rows, int q_heads, int kv_heads, int groups);

/* What tetra_kv_attend gives, with the same arguments and limits, but for the rounding: tokens that a group shares are read once for
 * all of its rows, through the page table of the first of its sequences that take part.  Whole blocks are shared, where there are
 * eight at least; the tokens behind them are read by each sequence.  A sequence takes part where its group has two sequences at least, it has
 * rows, and lengths[s] is not below the shared tokens of whole blocks; others read all of their tokens themselves.  Three launches; where
 * the table has no room for as many tokens as make up for that (width * page_tokens, for all sequences), tetra_kv_attend's
 * one. */
int tetra_kv_attend_shared(const tetra_kv_cache *cache, const tetra_kv_groups *groups, const void *q, int64_t q_stride,
                           void *out, int rows, int q_heads, float scale, void *workspace, size_t workspace_bytes,
                           void *stream);

#ifdef __cplusplus
}
#endif
#endif
