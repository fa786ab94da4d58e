/*
 * mv_lm.h -- C ABI of the operators that stand between a language model and the sparse step of
 * mv_sparse.h: the two ends of the model, whose gradients fill a worker's row, and the norm that bounds
 * a worker's gradient before error feedback.
 *
 *   embedding    out_t = s W[id_t]                  and its gradient  dW_v = s sum_{t: id_t = v} dout_t
 *   token loss   z = c x, lse = log sum_v exp z_v, log p = z - lse:  log p of given tokens, the entropy
 *                H = -sum_v p_v log p_v, the k largest log p, and the gradient with respect to x
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
 * stream) without synchronising the host, status codes are MV_OK / MV_ERR_*, and arguments are checked
 * before anything is enqueued.  Pointers need the alignment of their element type only (a table may start
 * anywhere in a worker's row); rows are contiguous and `ld...` elements apart.  Results do not depend
 * on the order in which the GPU runs things: the same call on the same inputs gives the same bytes.  Where
 * the inputs lie can change the order of the sums in mv_token_logprob and mv_clip_* (rows and tensors are cut at
 * their own 16- or 32-byte boundaries), and so can the number of rows; the other calls' bytes do not depend on it.
 */
#ifndef MV_LM_H
#define MV_LM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { MV_F32 = 0, MV_BF16 = 1, MV_F16 = 2, MV_I32 = 3, MV_I64 = 4 };

#define MV_TOP_MAX 64 /* most alternatives per position */

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
