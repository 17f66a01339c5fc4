/*
 * cllm_verify.h -- verification of drafted tokens against the target's probabilities, for
 * decoding with a temperature: what the greedy fixed-point test of a Jacobi block is to
 * greedy decoding.
 *
 * Request b's rows are row_start[b] .. row_start[b+1]-1, as a page plan counts them
 * (cllm_paged.h): its first token is known, the tokens after it are drafted.  Row i's
 * logits are the target's after its token, p_i = softmax(logits_i / temperature).  Token i + 1, drawn
 * from a draft's distribution q_i, stands when  u_i q_i(x) < p_i(x);  the first that does
 * not is replaced by a token drawn from max(p_i - q_i, 0), normalised, and if all stand the next
 * one is drawn from the last row's p.  Then the tokens are distributed as if they had been
 * drawn from the target one by one.  The random numbers are inputs: u uniform in [0, 1), and a race
 * e_v > 0 of independent exponentially distributed numbers, one per token of the vocabulary:
 * the v with the largest w_v / e_v is drawn in proportion to the weights w.
 *
 * Conventions: as in cllm_paged.h (device memory of the caller, work queued on the stream,
 * lengths on the device, nothing allocated by a call).
 */
#ifndef CLLM_VERIFY_H
#define CLLM_VERIFY_H

#include <stdint.h>

#include "cllm_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cllm_verifier cllm_verifier;

/* A verifier owns the scratch of calls of up to max_rows rows and max_batch requests on the current
 * device (28 bytes a row, 12 a request and 40 KB).  Calls on one verifier must not overlap in time.
 * Errors: EINVAL (sizes < 1, null), EUNSUPPORTED (not an sm_103 device), ENOMEM, ECUDA. */
int cllm_verifier_create(int max_rows, int max_batch, cllm_verifier **out);

/* Wait for the device, then release what the verifier owns.  NULL is a no-op. */
void cllm_verifier_destroy(cllm_verifier *v);

/*
 * accepted[b] = 1 + the drafts that stand (1 .. rows of the request), next[b] = the token that
 * follows them.
 * Greedy requests (all, without a race; else those whose temperature is below 2^-60): a
 * draft stands when it is the row's largest logit (the lowest index of equal ones), which is also
 * the next token.
 * Without draft_probs the drafts are certain, q_i = 1 at the draft (a Jacobi block, an n-gram).
 * A draft outside [0, vocab) is none: it does not stand, and the next token is drawn from p_i
 * itself.  Where max(p_i - q_i, 0) is nothing, too.
 * A request without rows, or with more rows than tokens (seq_len[b], as a plan leaves a refused one), or
 * with rows outside the arrays has accepted 0 and next -1.  A row without a distribution (a logit that is NaN or,
 * unless greedy, +inf; none above -inf; a temperature that is negative, NaN or above 2^40) ends its
 * request: no draft stands against it, and next is -1 if it decides.
 * Logits of -inf are tokens that are never drawn.
 * In fp32: probabilities to about 2^-20 of themselves.
 */
typedef struct {
  int batch, rows, vocab, dtype;        /* rows: of the logits; dtype: CLLM_F32 | CLLM_BF16 | CLLM_F16, of the logits */
  const void *logits;                   /* [rows][vocab] */
  int64_t logits_stride;                /* elements between rows */
  const int32_t *tokens;                /* [rows] */
  const int32_t *row_start, *seq_len;   /* [batch + 1], [batch] */
  const float *temperature;             /* [batch], or NULL: 1 */
  const float *uniforms;                /* [rows], or NULL with race */
  const float *race;                    /* [batch][vocab], or NULL: greedy */
  int64_t race_stride;
  const float *draft_probs;             /* [rows][vocab]: row i's are the distribution that token i + 1 was drawn from; or NULL */
  int64_t probs_stride;
  int32_t *accepted, *next;             /* [batch] */
  float *target_probs;                  /* [rows], or NULL: p_i(token i + 1) (greedy: 1 or 0); 0 where a row has no
                                         * draft or distribution; rows behind the last request's are not written */
} cllm_verify_args;

/* Errors: EINVAL (null or misaligned pointers, sizes or strides outside their ranges or past the
 * verifier's, a race without uniforms or the reverse, a temperature or draft_probs without a race), ECUDA. */
int cllm_verify(cllm_verifier *v, const cllm_verify_args *a, void *cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* CLLM_VERIFY_H */
