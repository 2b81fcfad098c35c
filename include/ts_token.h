/*
 * ts_token.h -- C ABI of the calls on rows of token logits (libtschain.so, MI355X / gfx950):
 * what a chain needs beside a large model.
 *   - the K largest logits of every row and its log-sum-exp: what a teacher leaves behind;
 *   - the divergence of a student's rows from a teacher's top logits, and its gradient;
 *   - the log-probabilities of given tokens, rows' entropies and most likely tokens, and the
 *     gradient of the first two;
 *   - the verification of drafted tokens (a chain's samples, for instance) against the
 *     target's probabilities, from given random numbers.
 * Status codes, errors, ownership, streams and reproducibility are those of ts_chain.h: every
 * pointer is a device pointer owned by the caller, nothing is allocated, work is enqueued on
 * `stream`, and results are bitwise the same for the same inputs.
 *
 * Common arguments
 *   logits   [B, N, V] of one of the types below.  The V logits of a row are contiguous; rows
 *            lie stride_n elements apart and sequences stride_b (both >= 0, so that a padded
 *            vocabulary or an expanded batch needs no copy).  Rows need no alignment beyond
 *            their element's.  Finite values and -inf (a token that cannot follow) are
 *            allowed; +inf and NaN are not.
 *   lengths  int32 [B]: rows of each sequence, 0 <= lengths[b] <= N, or NULL (every length is
 *            N).  Rows n >= lengths[b] are padding: they are never read, and each call says
 *            what it writes there.  Values are clamped on the device; with TS_CHECK=1 in the
 *            environment the call copies them to the host and returns TS_ERR_LENGTHS.
 *   B, N, V  B >= 1, N >= 1, 1 <= V <= ts_token_max_vocab(), B * N <= 2^29.
 *   K        logits kept of a row: 1 <= K <= min(V, ts_token_max_top()).
 *   temperature  T > 0: a row's probabilities are softmax(logits / T).
 *   ws       device workspace of at least ts_token_workspace_bytes(op, B, N, V, K) bytes,
 *            aligned to 256 bytes; NULL when that is 0.  Its contents on entry are ignored.
 */
#ifndef TS_TOKEN_H
#define TS_TOKEN_H

#include "ts_chain.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TS_ERR_BAD_ARG -7 /* an element type, a temperature or a stride out of range */

/* element types */
#define TS_FLOAT32 0
#define TS_BFLOAT16 1
#define TS_FLOAT16 2

/* operation codes for ts_token_workspace_bytes */
#define TS_TOKEN_TOP 0
#define TS_TOKEN_DISTILL 1
#define TS_TOKEN_DISTILL_GRAD 2
#define TS_TOKEN_VERIFY 3 /* N: the most drafts of a sequence; K is ignored */
#define TS_TOKEN_SCORE 4 /* K may be 0 */
#define TS_TOKEN_SCORE_GRAD 5 /* K is ignored */

/* Largest V and largest K. */
int ts_token_max_vocab(void);
int ts_token_max_top(void);

/* Workspace bytes that operation `op` needs; 0 for invalid arguments (check with the call
 * itself, which reports why). */
size_t ts_token_workspace_bytes(int op, int64_t B, int64_t N, int64_t V, int64_t K);

/*
 * The K largest logits of every row, largest first, equal ones by the lowest index (-0 equals
 * 0), and the row's log-sum-exp.
 *   values   [B, N, K] of the logits' type: the logits themselves (not divided by T).
 *   indices  int32 [B, N, K].
 *   lse      float32 [B, N] or NULL: log sum_v exp(logits_v / T); -inf for a row without a
 *            finite logit.
 * Padding: values -inf, indices -1, lse -inf.
 */
ts_status ts_token_top(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                       const int32_t* lengths, int64_t B, int64_t N, int64_t V, int64_t K,
                       float temperature, void* values, int32_t* indices, float* lse, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * Distillation from a teacher's top logits: the Kullback-Leibler divergence of the student's
 * q = softmax(logits / T) from the teacher's p, of every row.
 *   top_values   [B, N, K], any of the element types (top_dtype): the teacher's logits t_k.
 *   top_indices  int32 [B, N, K]: their tokens i_k, all different within a row.  An index
 *                outside [0, V) is an empty slot, whose value is never used: -1 where a row has
 *                fewer than K.  TS_CHECK=1 returns TS_ERR_LABELS for an index below -1, above
 *                V - 1, or twice in a row.
 *   top_lse      float32 [B, N] or NULL.
 * Without top_lse the teacher is normalised over its slots, p = softmax(t / T), and
 *   loss = sum_k p_k (log p_k - log q[i_k]).
 * With it (the teacher's log sum_v exp(t_v / T) over its whole vocabulary) p_k =
 * exp(t_k / T - top_lse), and what the slots leave, p_r = 1 - sum_k p_k, is one class of its
 * own that the student gives q_r, its probability outside the slots:
 *   loss = sum_k p_k (log p_k - log q[i_k]) + p_r (log p_r - log q_r).
 * p_r below 2^-22 (8 + |top_lse|) counts as 0: that is the rounding of the p_k and of top_lse in 32
 * bits.  It is 0 too where the slots hold every token of the vocabulary.
 *   loss     float32 [B, N]: +inf where q is 0 and p is not; 0 for padding and for rows with no
 *            teacher probability at all.
 */
ts_status ts_token_distill(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                           const void* top_values, int top_dtype, const int32_t* top_indices,
                           const float* top_lse, const int32_t* lengths, int64_t B, int64_t N,
                           int64_t V, int64_t K, float temperature, float* loss, void* ws,
                           size_t ws_bytes, void* stream);

/*
 * The same with its gradient.
 *   weights  float32 [B, N] or NULL (all 1): the derivative of what is minimised by each row's
 *            loss (1 / rows for a mean; T^2 / rows to keep the scale of T = 1).
 *   loss     float32 [B, N] or NULL: as above, not weighted.
 *   grad     [B, N, V], contiguous, of the logits' type, not overlapping them:
 *            weights * d loss / d logits,
 *              weights / T * (q_v sum_k p_k - p_v)      without top_lse,
 *              weights / T * (q_v - p_v)                with it, at the slots' tokens,
 *              weights / T * q_v (1 - p_r / q_r)        with it, elsewhere,
 *            rounded once.  Exactly 0 for padding, for rows with no teacher probability and for
 *            rows without a finite logit.
 */
ts_status ts_token_distill_grad(const void* logits, int dtype, int64_t stride_b,
                                int64_t stride_n, const void* top_values, int top_dtype,
                                const int32_t* top_indices, const float* top_lse,
                                const float* weights, const int32_t* lengths, int64_t B,
                                int64_t N, int64_t V, int64_t K, float temperature, float* loss,
                                void* grad, void* ws, size_t ws_bytes, void* stream);

/*
 * Scores of given tokens, with p = softmax(logits / T) of every row.
 *   tokens   int32 [B, N].  One outside [0, V) has no score.
 *   K        >= 0: alternatives asked for.
 *   logp     float32 [B, N]: log p(token); 0 where there is none.
 *   entropy  float32 [B, N]: - sum_v p_v log p_v.
 *   alternatives      int32 [B, N, K]: the K most likely tokens, the most likely first, equal ones by the
 *                     lowest index (the given token among them where it is one).  May be NULL when K == 0.
 *   alternative_logp  float32 [B, N, K]: log p of these.  May be NULL when K == 0.
 * Padding: logp and entropy 0, alternatives -1, alternative_logp -inf.  A row without a finite logit
 * has log p = -inf throughout, and entropy 0.
 */
ts_status ts_token_score(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                         const int32_t* tokens, const int32_t* lengths, int64_t B, int64_t N,
                         int64_t V, int64_t K, float temperature, float* logp, float* entropy,
                         int32_t* alternatives, float* alternative_logp, void* ws,
                         size_t ws_bytes, void* stream);

/*
 * The first two with a gradient.
 *   weights, entropy_weights  float32 [B, N] or NULL (all 1; all 0): the derivatives of what is
 *            maximised by each row's log p(token) and by its entropy (-1 / rows and 0 for a mean
 *            negative log-likelihood that is minimised).
 *   logp, entropy  float32 [B, N] or NULL: as above, not weighted.
 *   grad     [B, N, V], contiguous, of the logits' type, not overlapping them:
 *            (weights ([v = token] - p_v) - entropy_weights p_v (log p_v + entropy)) / T,
 *            rounded once; without the first term where the row's token has no score.  Exactly 0 for
 *            padding and for rows without a finite logit.
 */
ts_status ts_token_score_grad(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                              const int32_t* tokens, const float* weights,
                              const float* entropy_weights, const int32_t* lengths, int64_t B,
                              int64_t N, int64_t V, float temperature, float* logp,
                              float* entropy, void* grad, void* ws, size_t ws_bytes,
                              void* stream);

/*
 * Verification of drafted tokens (speculative sampling): what is emitted is distributed as the
 * target's own samples are, whatever the drafts.
 *   target   [B, G+1, V] logits of the model that answers: row t is its distribution p_t after
 *            the first t drafts.
 *   draft    [B, G, V] logits that the drafts were drawn from, q_t, at draft_temperature (a
 *            chain's rows of log-probabilities are such logits).  May be NULL only when G == 0.
 *   draft_lse float32 [B, G] or NULL: log sum_v exp(draft_v / draft_temperature), where the
 *            caller has it (0 for normalised rows); it saves the sum over the drafts' rows.  -inf:
 *            q_t is 0 throughout.
 *   tokens   int32 [B, G]: the drafts z_t.  One outside [0, V) is never accepted; TS_CHECK=1 returns
 *            TS_ERR_LABELS for one among a sequence's lengths[b] drafts.
 *   uniforms float32 [B, G] in [0, 1), noise float32 [B, V], positive, independent standard
 *            exponentials: the caller's random numbers.
 *   lengths  int32 [B] or NULL: drafts of each sequence, 0 <= lengths[b] <= G.
 *   G        >= 0, B * (G + 1) <= 2^29.
 * Draft t is accepted when all before it are and uniforms_t * q_t(z_t) < p_t(z_t); a p below
 * 2^-1074 of its row's largest counts as 0.  After a accepted drafts one more token is drawn: from
 * max(p_a - q_a, 0), normalised, where draft a was refused, and from p_a where there was none (or
 * where max(p_a - q_a, 0) is 0 throughout).
 * The draw is argmax_v r_v / noise_v, the lowest index of equal ones: the first of
 * exponential clocks of rates r_v rings at v with probability r_v / sum r.  It needs no sum
 * of r and its outcome does not depend on how a row is divided.  A target's row without a
 * finite logit has p = 0: it refuses its draft and draws token 0.
 *   out      int32 [B, G+1]: the accepted drafts, the drawn token, then -1.
 *   accepted int32 [B]: a.
 *   logp     float32 [B, G+1] or NULL: log p_t(out_t); 0 where out is -1.
 */
ts_status ts_token_verify(const void* target, int target_dtype, int64_t target_stride_b,
                          int64_t target_stride_n, const void* draft, int draft_dtype,
                          int64_t draft_stride_b, int64_t draft_stride_n, const float* draft_lse,
                          const int32_t* tokens, const float* uniforms, const float* noise,
                          const int32_t* lengths, int64_t B, int64_t G, int64_t V,
                          float temperature, float draft_temperature, int32_t* out,
                          int32_t* accepted, float* logp, void* ws, size_t ws_bytes,
                          void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TS_TOKEN_H */
