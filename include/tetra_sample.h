/*
 * tetra_sample.h -- C ABI of the choice of the next token from the output head's logits.
 *
 * Conventions are those of tetra.h (status codes, device/host pointers, stream, validation before launch; a rejected
 * call launches nothing).  The kernel waits for the end of the kernels before it on the stream before it reads anything.
 */
#ifndef TETRA_SAMPLE_H
#define TETRA_SAMPLE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { TETRA_SAMPLE_MAX_VOCAB = 393216, TETRA_SAMPLE_MAX_ROWS = 65535 };

/* Rows of logits [rows][vocab], float32 (half_type 0, as tetra_q4_gemv writes them) or float16 (half_type 1), row_stride
 * elements apart.  Per row, device memory: u float32 (required), temperature float32, top_k int32, top_p float32, min_p
 * float32; NULL stands for temperature 1, or for a filter that is off.  tokens int32 [rows]; prob float32 [rows] or NULL. */
typedef struct {
    const void *logits;
    const float *u, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *tokens;
    float *prob;
    int64_t row_stride;
    int32_t rows, vocab, half_type;
} tetra_sample_rows;

/* For each row x, with temperature T > 0 and w_i = exp((x_i - max x) / T):
 *   tokens are ordered by logit, the largest first, equal ones by index;
 *   top_k   k > 0: the first k stay;
 *   top_p   p < 1: of these the fewest first ones whose mass is at least p times the mass of these, one at least;
 *   min_p   m > 0: of these the ones with w_i >= m, the first at least;
 *   token   the smallest index i, among those that are left, with the sum of w_j over j <= i above u times their
 *           whole mass M; prob = w_i / M.
 * u lies in [0, 1) (values outside are taken as the nearest inside, NaN as 0).  T that is not above zero takes the first
 * of the largest logits, with prob 1.  NaN counts as minus infinity, which is never taken, plus infinity as float32's largest
 * number; magnitudes below 2^-126 count as zero, and a distance from the largest logit that float32 cannot hold as infinite.
 * A row without a logit above minus infinity gives token -1 and prob 0.
 * The weights are whole multiples of 2^-44, off by no more than that (the least have none), and every sum of them is exact:
 * the result does not depend on any order of summation and is the same from run to run.  One launch, no scratch memory. */
int tetra_sample(const tetra_sample_rows *rows, void *stream);

#ifdef __cplusplus
}
#endif
#endif
