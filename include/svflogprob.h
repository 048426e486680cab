/*
 * svflogprob.h -- what the tokens of an answer are worth: log probabilities of
 * given tokens, with entropies and the best alternatives, from logits.
 *
 * Part of libsvfsim.so.  Where a simulated step is carried out (svfkv.h), this is
 * its end: every running request has a row of logits, and the token that
 * it answers with a probability.
 *
 * With the logits x of a row and p = softmax(scale x):
 *   logprob      ln p[token]
 *   entropy      - sum_i p_i ln p_i  (0 ln 0 = 0)
 *   rank         how many indices come before the token
 *   top_logprob, top_index   the first ``top`` indices, and their ln p
 * in the order of falling logits and, among equal ones, rising indices (-0 equals 0, NaN comes last).
 * Sums are held in 32 bits.
 *   - A row with a NaN or a logit of +infinity has no distribution: logprob, entropy and
 *     top_logprob are NaN; rank and top_index are still those of the order.
 *   - A row with only logits of -infinity (nothing is allowed) has logprob and top_logprob
 *     -infinity and entropy 0.
 *   - A token outside [0, vocab) has logprob NaN and rank -1.
 *
 * Conventions are those of svfkv.h: device memory inside a host struct, asynchronous on
 * hip_stream, nothing allocated or kept, may be recorded into a graph; sizes are checked before anything is
 * enqueued, with the text from svf_logprob_last_error; return codes of svfsim.h.
 */
#ifndef SVFLOGPROB_H
#define SVFLOGPROB_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of logits. */
enum {
    SVF_LOGITS_BF16 = 0,
    SVF_LOGITS_F16 = 1,
    SVF_LOGITS_F32 = 2
};

enum { SVF_LOGPROB_MOST_TOP = 64, SVF_LOGPROB_MOST_VOCAB = 1 << 21 };

/*
 *   logits       [rows][vocab], row_stride elements from row to row (0 and up), vocab contiguous; any
 *                alignment that the type has
 *   token        [rows], int32 or int64 as token_bytes says (4 or 8)
 *   vocab        1 .. 2^21;  top 0 .. 64, no more than vocab;  scale (1 / temperature) > 0, below 2^126
 *   logprob, entropy   float [rows];  rank int32 [rows]
 *   top_logprob, top_index   float and int32 [rows][top]
 *   workspace    svf_logprob_workspace bytes, 256-byte aligned, nothing kept in it
 * rows * top below 2^31, rows (some 2^23) such that a launch has fewer than 2^32 threads.
 */
typedef struct svf_logprob_args {
    const void *logits;
    const void *token;
    float *logprob;
    float *entropy;
    int32_t *rank;
    float *top_logprob;
    int32_t *top_index;
    void *workspace;
    int64_t workspace_bytes;
    int64_t row_stride;
    float scale;
    int32_t rows, vocab, top, dtype, token_bytes;
} svf_logprob_args;

int svf_logprob(const svf_logprob_args *args, void *hip_stream);

/* Bytes of workspace that svf_logprob needs (rows, vocab, top and dtype are read); negative: the code of an error. */
int64_t svf_logprob_workspace(const svf_logprob_args *args);

/* Text of the calling thread's last error in one of these calls. */
const char *svf_logprob_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* SVFLOGPROB_H */
