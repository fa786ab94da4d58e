/*
 * mv_lm.h -- C ABI of the operators that stand between a language model and the sparse step of
 * mv_sparse.h: the two ends of the model, whose gradients fill a worker's row, and the norm that bounds
 * a worker's gradient before error feedback.
 *
 *   embedding    out_t = s W[id_t]                  and its gradient  dW_v = s sum_{t: id_t = v} dout_t
 *   layer norm   y = (x - mean) / sqrt(variance + eps) w + b row by row, and its gradients
 *   token loss   z = c x, lse = log sum_v exp z_v, log p = z - lse:  log p of given tokens, the entropy
 *                H = -sum_v p_v log p_v, the k largest log p, and the gradient with respect to x
 *   distillation the divergence of softmax(c x) from a teacher that is known by its largest log probabilities, and its gradient
 *   sampling     one token per row from softmax(c x), cut to the top k, the top p and the min p, by given random numbers
 *   clipping     n_g = sqrt(sum of squares over the tensors of group g), every tensor of the group times
 *                min(1, max_norm / n_g): in place, or laid end to end as the fp32 rows that
 *                mv_sparse_step takes (one group per worker)
 *
 * Types.  MV_F32 / MV_BF16 / MV_F16 for values, MV_I32 / MV_I64 for token ids.  Whatever the inputs'
 * type, products, sums, exponentials and norms are formed in 32 bits or more and rounded once to the
 * output's type.
 *
 * Memory and errors follow mv_sparse.h: DEVICE pointers owned by the caller unless said otherwise,
 * nothing is allocated on the device, work is enqueued on `stream` (a cudaStream_t, NULL = default
 * stream) without synchronising the host, on the current device, which is the one of the pointers and of
 * the stream; status codes are MV_OK / MV_ERR_*, and arguments are checked before anything is enqueued.
 * Pointers need the alignment of their element type only (a table may start anywhere in a worker's row);
 * rows are contiguous and `ld...` elements apart.  Results do not depend
 * on the order in which the GPU runs things: the same call on the same inputs gives the same bytes.  Where
 * the inputs lie can change the order of the sums in mv_token_logprob, mv_layer_norm*, mv_distill and mv_clip_* (rows and tensors are
 * cut at their own 16- or 32-byte boundaries), and so can the number of rows; the other calls' bytes do not depend on it.
 */
#ifndef MV_LM_H
#define MV_LM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { MV_F32 = 0, MV_BF16 = 1, MV_F16 = 2, MV_I32 = 3, MV_I64 = 4 };

#define MV_TOP_MAX 64        /* most alternatives per position that mv_token_logprob finds */
#define MV_TEACHER_MAX 1024  /* most alternatives per position that mv_distill takes */

/* Embedding lookup.  out[t, :] = scale * weight[ids[t], :], the product rounded once to 32 bits and once to
 * out's type.  A token id outside [0, V) gives a row of zeros.  weight and out share no bytes.
 *   weight [V, D] w_type in, rows ldw >= D apart;  ids [T] id_type in;  out [T, D] out_type out, rows ldo >= D apart
 * Limits: 1 <= V < 2^31, 1 <= D < 2^31, 0 <= T < 2^31. */
int mv_embed(void* stream, const void* weight, int w_type, int64_t V, int64_t D, int64_t ldw, const void* ids, int id_type,
             int64_t T, float scale, void* out, int out_type, int64_t ldo);

/* Bytes of scratch mv_embed_grad needs (host arithmetic only); 0 if out of range. */
size_t mv_embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D);

/* Gradient of the lookup with respect to the table, dense.  The tokens are grouped by id, and each row is summed
 * in 32 bits in an order that only the ids fix, then multiplied by scale.
 *   dout    [T, D] dout_type in, rows ldd >= D apart, no bytes of dweight;  ids [T] id_type in
 *   dweight [V, D] float, rows ldw >= D apart.  accumulate = 0: overwritten (rows without a token become +0);
 *           accumulate = 1: added to, rows without a token are not touched
 *   pad_id  tokens with this id, like ids outside [0, V), have no gradient; -1 for none
 *   workspace  mv_embed_grad_workspace_bytes(T, V, D) bytes, 16-byte aligned
 * Limits: as mv_embed. */
int mv_embed_grad(void* stream, const void* dout, int dout_type, int64_t ldd, const void* ids, int id_type, int64_t T, int64_t V,
                  int64_t D, float scale, int64_t pad_id, int accumulate, float* dweight, int64_t ldw, void* workspace,
                  size_t workspace_bytes);

/* Layer norm of rows.  mu = mean of x[t, :], v = mean of (x - mu)^2, r = 1 / sqrt(v + eps), y[t, i] = (x[t, i] - mu) r w[i] + b[i],
 * in 32 bits (sums of D terms, the squares' after the mean is known, and what that is off by taken out of mu, v and y again, so that rows
 * far from zero keep their digits), rounded once to y's type.
 *   x [T, D] type in, rows ldx >= D apart;  y [T, D] out, of the same type, rows ldy >= D apart; may be x itself (then ldy = ldx)
 *   weight, bias [D] w_type in: MV_F32 or x's type; each may be NULL (1 and 0)
 *   mean, rstd [T] float out (mu and r), what the gradient needs; each may be NULL
 * What is written shares no bytes with anything else, y with x excepted.
 * eps >= 0, finite.  A row that holds an inf or a NaN, or whose sums pass the range of 32 bits, has no other meaning than the
 * formula's in 32 bits.  Limits: 0 <= T < 2^31, 1 <= D < 2^31. */
int mv_layer_norm(void* stream, const void* x, int type, int64_t T, int64_t D, int64_t ldx, const void* weight, const void* bias, int w_type,
                  float eps, void* y, int64_t ldy, float* mean, float* rstd);

/* Bytes of scratch mv_layer_norm_grad needs (host arithmetic only); 0 if out of range. */
size_t mv_layer_norm_grad_workspace_bytes(int64_t T, int64_t D);

/* Its gradients, given dy.  With n = (x - mu) r and h = dy w:
 *   dx[t, i] = r (h_i - mean(h) - n_i mean(h n)),  dweight[i] = sum_t dy[t, i] n[t, i],  dbias[i] = sum_t dy[t, i]
 *   dy, x [T, D] type in, rows lddy and ldx apart;  weight as in mv_layer_norm;  mean, rstd [T] float in, as mv_layer_norm left them
 *   dx [T, D] out, of the same type, rows lddx apart; may be dy or x itself (of the same pitch); NULL: not wanted
 *   dweight, dbias [D] float out, each may be NULL.  accumulate = 0: overwritten (T = 0: zeros); accumulate = 1: added to
 *   workspace  mv_layer_norm_grad_workspace_bytes(T, D) bytes, 16-byte aligned (unused, and may be NULL, without dweight and dbias)
 * dx, dweight, dbias and the workspace share no bytes with one another or with an input, dx with dy or x excepted.
 * The sums over rows are in 32 bits, in an order that the sizes, the type and the rows' places within 16 bytes fix. */
int mv_layer_norm_grad(void* stream, const void* dy, int64_t lddy, const void* x, int64_t ldx, int type, int64_t T, int64_t D,
                       const void* weight, int w_type, const float* mean, const float* rstd, void* dx, int64_t lddx, float* dweight,
                       float* dbias, int accumulate, void* workspace, size_t workspace_bytes);

/* Log probabilities of given tokens under softmax(scale * logits), row by row, with entropy and alternatives.
 *   logits  [T, V] type in, rows ld >= V apart;  scale > 0 (an inverse temperature)
 *   targets [T] id_type in (NULL if logprob is NULL).  A target outside [0, V) marks a position without one:
 *           its logprob is 0
 *   logprob, entropy, lse [T] float out, each may be NULL
 *   top_logprob, top_id [T, k] float / int32 out, 0 <= k <= MV_TOP_MAX, each may be NULL: the k largest logits in
 *           descending order, equal ones (+0 and -0 are equal) by ascending index
 * -inf marks a masked logit: p = 0, no share in the entropy.  A row with nothing else has lse = -inf, entropy 0 and
 * logprob -inf.  A row with a NaN or +inf has NaN for lse, entropy, logprob and top_logprob; NaN is no alternative.
 * Where a row has fewer than k alternatives the rest are id -1 and -inf.  An lse below the range of 32 bits (a row of the
 * type's lowest value, scaled up) is -inf, though the row's other outputs are finite.
 * Limits: 0 <= T < 2^31, 1 <= V < 2^31. */
int mv_token_logprob(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const void* targets, int id_type,
                     float scale, int k, float* logprob, float* entropy, float* lse, float* top_logprob, int32_t* top_id);

/* Gradient of sum_t (g_logprob[t] logprob[t] + g_entropy[t] entropy[t]) with respect to the logits:
 *   dlogits[t, v] = scale ( g_logprob[t] (1[v = target] - p_v) - g_entropy[t] p_v (log p_v + entropy[t]) )
 * with log p_v = min(0, scale logits[t, v] - lse[t]): p is as exact as the 32-bit lse is, and never above 1.
 *   lse, entropy [T] float in, as mv_token_logprob left them (entropy only with g_entropy)
 *   g_logprob [T] float in (NULL: zero; then targets may be NULL);  g_entropy [T] float in (NULL: zero)
 *   dlogits [T, V] out, of the logits' type, rows ldg >= V apart; may be the logits themselves (then ldg = ld)
 * A position without a target has no logprob term.  Where neither term is left (no target or g_logprob 0, and
 * g_entropy 0) the row is +0 whatever its logits hold; so is a row whose lse is -inf.  In a row of finite logits whose
 * lse is +inf (beyond the range of 32 bits once scaled) every p is 0. */
int mv_token_logprob_grad(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const void* targets,
                          int id_type, float scale, const float* lse, const float* entropy, const float* g_logprob,
                          const float* g_entropy, void* dlogits, int64_t ldg);

/* Divergence of the student p = softmax(scale * logits) from a teacher that is known by k alternatives per row, a_j = top_logprob[t, j]
 * of token top_id[t, j] (what mv_token_logprob leaves for the teacher's logits, at the same scale).
 *   rest = 0: the alternatives stand for the whole teacher, q = softmax(a) over them:  kl = sum_j q_j (log q_j - log p_j)
 *   rest = 1: q_j = exp(a_j) are the teacher's probabilities; what is missing to one, r = max(0, 1 - sum_j q_j), is one more class, beside
 *             the student's mass outside the list P = 1 - sum of p over the listed tokens:  kl = ... + r (log r - log P)
 *   logits [T, V] type in, rows ld >= V apart;  top_logprob, top_id [T, k] float / id_type in, contiguous, 1 <= k <= MV_TEACHER_MAX
 *   kl, lse, log_rest [T] float out, each may be NULL: the divergence, log sum exp of the scaled logits, and log P (rest = 1 only)
 *           They share no bytes with the inputs or one another.
 * An id outside [0, V) is no alternative, nor is a_j = -inf with rest = 0.  A row without one has no teacher: kl 0 whatever its
 * logits hold, log_rest as if the list were empty.  The same id twice is two terms of the sums, but one token.  q_j = 0 adds
 * nothing; q_j > 0 where p_j = 0 (a masked logit, a row that is all -inf) makes kl +inf.  P is summed without the listed tokens,
 * not taken as a difference; terms below 2^-126 of the row's largest count as 0.  A row of logits with a NaN or +inf has NaN in all
 * three; a NaN or +inf among a row's a_j makes kl NaN.
 * Limits as mv_token_logprob. */
int mv_distill(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* top_logprob, const void* top_id,
               int id_type, int k, int rest, float scale, float* kl, float* lse, float* log_rest);

/* Gradient of sum_t g[t] kl[t] with respect to the logits, M = sum_j q_j + r (1 without rest):
 *   dlogits[t, v] = scale g[t] (M p_v - sum_{j: id_j = v} q_j) for a listed token v,  scale g[t] p_v (M - r / P) for the others
 * with log p_v = min(0, scale logits[t, v] - lse[t]).
 *   lse, log_rest [T] float in, as mv_distill left them (log_rest NULL: rest = 0);  g [T] float in
 *   dlogits [T, V] out, of the logits' type, rows ldg >= V apart; may be the logits themselves (then ldg = ld), else no bytes of any input
 * A row without a teacher, with g[t] = 0 or with lse = -inf is +0 whatever its logits hold; where log_rest is -inf, the others are 0. */
int mv_distill_grad(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* top_logprob,
                    const void* top_id, int id_type, int k, float scale, const float* lse, const float* log_rest, const float* g,
                    void* dlogits, int64_t ldg);

/* Draws a token per row.  w_v = exp(scale (x_v - max x)); the tokens in descending order of x, equal ones (+0 and -0 are equal) by
 * ascending index, are cut to the first top_k, those to the shortest start whose sum is at least top_p times theirs, those to w_v >=
 * min_p; the first always stays.  token[t] is the first index at which the sum of the kept w, in ascending order of the index, exceeds u[t] times their
 * sum, and logprob[t] the log of its share of that sum.  Weights are formed in 64 bits and added as whole multiples of n / 2^61 of the largest,
 * n the smallest power of two that is not below V and at least 1024: a token with less than half of that (3e-14 for V = 10^5) is
 * never drawn.
 *   logits [T, V] type in, rows ld >= V apart;  u [T] float in, in [0, 1) (below: 0; from 1 on: the last kept token that has a weight)
 *   scale, top_p, min_p [T] float in, top_k [T] int32 in, on the device, each may be NULL: 1, 1 (all), 0 (all), 0 (all).
 *           scale > 0, an inverse temperature; top_k <= 0 or >= V, top_p >= 1, min_p <= 0: nothing is cut
 *   token [T] id_type out;  logprob [T] float out, may be NULL.  They share no bytes with the inputs or one another, but each may
 *           take the very place of u or a setting, element for element of 4 bytes
 * -inf marks a masked logit, which is never drawn.  A row with nothing else has token -1 and logprob -inf.  A row with a NaN or
 * +inf, with a NaN among its settings, or whose scale is not positive and finite, has token -1 and logprob NaN.
 * Limits as mv_token_logprob. */
int mv_sample(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* u, const float* scale,
              const int32_t* top_k, const float* top_p, const float* min_p, void* token, int id_type, float* logprob);

/* Norms and clipping over a fixed list of tensors.  The plan holds the list (the tensors' addresses, types and
 * sizes), not their values; it stays valid as long as the tensors stay where they are. */
typedef struct mv_clip mv_clip;

/* Bytes of device scratch for a plan (host arithmetic only); 0 if out of range. */
size_t mv_clip_workspace_bytes(const int64_t* numel, int n_tensors, int n_groups);

/* Creates a plan.  All arrays are HOST arrays, read before the call returns.
 *   tensors [n_tensors] device pointers, contiguous tensors (a plan whose tensors share bytes, as tied weights do, has no
 *           mv_clip_scale);  types MV_F32 / MV_BF16 / MV_F16;
 *           numel >= 0, below 2^40
 *   groups  [n_tensors] ascending, 0 <= groups[i] < n_groups: the tensors that share a norm (NULL: all in group 0)
 *   workspace  mv_clip_workspace_bytes() bytes, 256-byte aligned, owned by the caller, must outlive the plan and every call enqueued on it
 * The list is copied to the workspace on `stream`, and the call waits for that copy: not inside a stream capture.
 * A plan serves one call at a time (calls on several streams must be ordered).  n_tensors >= 0, 1 <= n_groups < 2^20. */
int mv_clip_create(mv_clip** out, void* stream, void* const* tensors, const int* types, const int64_t* numel, const int* groups,
                   int n_tensors, int n_groups, void* workspace, size_t workspace_bytes);
int mv_clip_destroy(mv_clip* plan);

/* Waits for the stream (not inside a stream capture) and returns MV_ERR_TIMEOUT if a wait between the CTAs of a call on the
 * plan has run out since the last time it was asked, MV_OK if none has.  Later calls on the plan are not affected. */
int mv_clip_status(mv_clip* plan, void* stream);

/* How often a CTA polls its group's factor before it gives up, in later calls: polls >= 0; -1: the default (a second or more). */
int mv_clip_set_polls(mv_clip* plan, int polls);

/* The calls on a plan.  A short list (up to 14 MB) is clipped by one cooperative kernel whose CTAs wait, with a limit, for
 * their group's factor; should a wait ever run out (never expected), what the CTA writes is NaN, and mv_clip_status says so.
 *
 * norms [n_groups] float out: sqrt of the sum of squares, added in 64 bits and rounded once (0 for an empty group; finite values
 *       whose norm passes the range of 32 bits: inf). */
int mv_clip_norm(mv_clip* plan, void* stream, float* norms);

/* In place: every tensor of group g is multiplied by c_g = min(1, max_norm / n_g), max_norm >= 0 (+inf: no clipping).
 * MV_ERR_INVALID_ARG where tensors of the plan share bytes, which would be multiplied twice.
 * A group that holds an inf or a NaN is left as it is (its norm is inf or NaN).  One of finite values is scaled by its norm in
 * 64 bits, even where the norm that is reported passes the range of 32.  norms may be NULL. */
int mv_clip_scale(mv_clip* plan, void* stream, float max_norm, float* norms);

/* Out of place: row g of `rows` receives the tensors of group g, end to end in list order, times c_g, in fp32.
 *   rows [n_groups] rows of ld floats, ld >= the elements of every group; what a row holds beyond its group stays.
 *   rows may not overlap the tensors.  norms may be NULL. */
int mv_clip_pack(mv_clip* plan, void* stream, float max_norm, float* rows, int64_t ld, float* norms);

#ifdef __cplusplus
}
#endif
#endif /* MV_LM_H */
