/*
 * tetra_logprobs.h -- C ABI of what tokens are worth under the output head's logits: the log probabilities and ranks of given
 * tokens, the entropy of the distribution, and the likeliest tokens.
 *
 * Conventions are those of tetra.h (status codes, device/host pointers, stream, validation before launch; a rejected
 * call launches nothing).  The kernel waits for the end of the kernels before it on the stream before it reads anything.
 */
#ifndef TETRA_LOGPROBS_H
#define TETRA_LOGPROBS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    TETRA_LOGPROBS_MAX_VOCAB = 1 << 24,
    TETRA_LOGPROBS_MAX_ROWS = 65535,
    TETRA_LOGPROBS_MAX_GIVEN = 64,
    TETRA_LOGPROBS_MAX_TOP = 32
};

/* Rows of logits [rows][vocab], float32 (half_type 0) or float16 (half_type 1), row_stride elements apart; temperature float32
 * [rows] or NULL (1).  Per row, all tightly packed: tokens int32 [given] with logprob float32 [given] and rank int32 [given] or
 * NULL; entropy float32 or NULL; top_tokens int32 [top] with top_logprob float32 [top].  given or top may be 0: what
 * belongs to it may be NULL then. */
typedef struct {
    const void *logits;
    const float *temperature;
    const int32_t *tokens;
    float *logprob;
    int32_t *rank;
    float *entropy;
    int32_t *top_tokens;
    float *top_logprob;
    int64_t row_stride;
    int32_t rows, vocab, half_type, given, top;
} tetra_logprobs_rows;

/* For each row x, with temperature T > 0, p_i = exp(x_i / T) / sum_j exp(x_j / T):
 *   logprob     log p of each given token;
 *   rank        how many tokens are ahead of it in the order (logit, the largest first; equal ones by index): 0 is the likeliest;
 *   entropy     - sum p log p, over the tokens with p > 0;
 *   top_tokens  the first `top` tokens of that order, and log p of each.
 * Natural logarithms.  T that is not above zero puts all of the probability on the first of the largest logits: its log
 * probability is 0, any other's minus infinity, the entropy 0.  NaN counts as minus infinity, plus infinity as float32's largest
 * number; magnitudes below 2^-126 count as zero.  A token with a logit of minus infinity has log probability minus
 * infinity and is not among the top tokens; where there are fewer than `top` others, -1 and minus infinity fill the rest.  A row without a
 * logit above minus infinity has entropy 0.  A given token outside [0, vocab) has log probability minus infinity and rank -1.
 * A thread's sums are float32, its tiles' added one after another, threads' sums float64; nothing depends on the order in which threads run: every output
 * is bit-identical from run to run.  One launch, no scratch memory. */
int tetra_logprobs(const tetra_logprobs_rows *rows, void *stream);

#ifdef __cplusplus
}
#endif
#endif
