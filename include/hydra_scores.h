/*
 * hydra_scores.h -- one rank's attention share with modified scores, on AMD MI355X (gfx950).
 *
 * The calls of hydra_attn.h for attention whose scores are capped, biased by distance, or seen
 * through a prefix mask.  For a visible pair of query i and key j of head h, at global positions
 * p_i and p_j:
 *
 *   s_ij = softmax_scale <q_i, k_j>
 *   s_ij = c tanh(s_ij / c)                  with a cap c
 *   s_ij = s_ij - slope_h |p_i - p_j|        with slopes
 *
 * and query i sees key j iff both lie in one document d and
 *
 *   p_j <= p_i  or  p_j < cu_seqlens[d] + prefix_len[d]
 *
 * (a document's first prefix_len[d] tokens are seen by all of its tokens, themselves included; the
 * others as in hydra_attn.h).  LSE, O, the merge of ring steps and D are those of hydra_attn.h for these
 * scores.  Backward, with P = exp(s - LSE) and t = tanh(softmax_scale <q_i, k_j> / c):
 *
 *   dV = P^T dO,  dS = P o (dO V^T - D) o (1 - t^2),  dQ = softmax_scale dS K,  dK = softmax_scale dS^T Q
 *
 * The slopes and the cap are constants: they get no gradient.
 *
 * Scores are formed in 32 bits.  With A = softmax_scale sum_c |q_ic k_jc|, s the (capped) score before its bias and
 * B = |slope_h (p_i - p_j)|, one is off by at most 2^-16 A + 2^-21 (|s| + B), with a cap by 2^-19 |s| besides, and its
 * weight by that much of itself; the factor 1 - t^2 is off by up to 2^-20.  tanh is a polynomial whose length is
 * chosen for a block of scores (32 x 32, in dK/dV 96 x 32) by its largest, masked ones included: within these bounds
 * a capped row's results depend on the rows and keys beside it in the window, and are not the same bits in another.
 * A row's largest score must stay below 2^20 in magnitude (a zigzag step may see far keys alone: 2^17 rows away under
 * a slope of 1/2 they have scores of -2^16, and weights to 2^-5); others may be lower.
 *
 * Every convention, status code and limit is that of hydra_attn.h.  q, k and v must be finite in every
 * row, also in rows that no query sees: a masked score's weight is 0, and 0 times a value that is not
 * finite is not 0.  hydra_lse_merge merges partials of these calls too; the no-allocation call has no
 * such form.
 */
#ifndef HYDRA_SCORES_H
#define HYDRA_SCORES_H

#include "hydra_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How the scores are modified.  All fields 0 or NULL, or a NULL hydra_scores_t*: not at all, and
 * the calls below are those of hydra_attn.h, on plans of either. */
typedef struct {
  float softcap;              /* c: 0 for none, else from 2^-10 to 2^10, with a softmax_scale of at least 2^-8
                                 and from 2^-14 to 2^10 times c                                */
  const float* slopes;        /* NULL for none, or DEVICE float[n_heads], finite, 4-byte aligned; read when
                                 the kernels run                                               */
  const int32_t* prefix_len;  /* NULL for none, or HOST int32[n_docs], 0 .. the document's
                                 length; read only during the call, part of the plan           */
} hydra_scores_t;

/* hydra_workspace_size, hydra_split_scratch_size, hydra_bwd_ds_bytes, hydra_visible_pairs and
 * hydra_plan_items of `p` with scores `sc` (host only). */
size_t hydra_scores_workspace_size(const hydra_problem_t* p, const hydra_scores_t* sc);
size_t hydra_scores_scratch_size(const hydra_problem_t* p, const hydra_scores_t* sc);
size_t hydra_scores_ds_bytes(const hydra_problem_t* p, const hydra_scores_t* sc, int32_t kv_heads_per_pass);
int64_t hydra_scores_visible_pairs(const hydra_problem_t* p, const hydra_scores_t* sc);
int64_t hydra_scores_plan_items(const hydra_problem_t* p, const hydra_scores_t* sc, int32_t which, int32_t* out,
                                int64_t cap);

/* hydra_attn_plan: the plan, and the workspace's size, depend on the prefixes (NULL is 0 for every document) and on
 * whether the scores are modified at all, not on the cap or the slopes: planned calls may turn either on, off or to
 * another value on one plan, but not the last modification off or the first one on (HYDRA_ERR_WORKSPACE). */
int hydra_scores_plan(const hydra_problem_t* p, const hydra_scores_t* sc, void* workspace, size_t workspace_bytes,
                      void* stream);

/* hydra_attn_fwd_split: partial O and LSE of one ring step, merged into o and lse with merge != 0, on
 * the plan in the workspace with planned != 0; scratch may be NULL.  The slopes must not overlap an
 * output. */
int hydra_scores_fwd(const hydra_problem_t* p, const hydra_scores_t* sc, const void* q, const void* k, const void* v,
                     float* o, float* lse, void* o_bf16, void* workspace, size_t workspace_bytes, void* scratch,
                     size_t scratch_bytes, int32_t merge, int32_t planned, void* stream);

/* hydra_attn_bwd_split: dQ, dK and dV of one ring step, added to the accumulators; with ds_buf the
 * stored-dS form where it applies (planned must then be 0).  o_final is bf16 (o_bytes = 2) or the merged
 * fp32 O itself (4): dQ and dK then do not carry its rounding, which where a few keys take a row's weight
 * is more than all others together. */
int hydra_scores_bwd(const hydra_problem_t* p, const hydra_scores_t* sc, const void* q, const void* k, const void* v,
                     const void* o_final, int32_t o_bytes, const float* lse_final, const void* d_o, float* dq_acc,
                     float* dk_acc, float* dv_acc, void* ds_buf, size_t ds_bytes, void* workspace, size_t workspace_bytes,
                     void* scratch, size_t scratch_bytes, int32_t planned, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HYDRA_SCORES_H */
