/*
 * hydra_linear.h -- linear attention with a decay for each head, on AMD MI355X (gfx950).
 *
 * For a sequence (a document, or a rank's piece of one) with rows 0 .. n - 1 and a head with log decay g:
 *
 *   S_t = e^g S_{t-1} + k_t v_t^T            S_{-1}: the state that the sequence starts from
 *   o_t = scale q_t S_t
 *
 * that is, o_i = scale (sum over j <= i of e^(g (i - j)) <q_i, k_j> v_j + e^(g (i + 1)) q_i S_{-1}), and the sequence
 * ends with the state S_{n-1}.  Work grows with the rows, not with their square.  A context-parallel rank computes
 * its rows of a document from the state of the rank before and hands its own to the next; what a rank adds to a state
 * is the last state of its rows from zero (a call without o), so that ranks need not wait for each other's outputs:
 * with rank r's A_r and n_r rows, the state behind it is e^(g n_r) S + A_r.  A zigzag chunk's two pieces are two
 * sequences.
 *
 * Backward, with dO and the gradient D of the last state, G_t the gradient of S_t:
 *
 *   G_t = scale q_t^T dO_t + e^g G_{t+1}     e^g G_n = D
 *   dq_t = scale dO_t S_t^T,  dk_t = G_t v_t,  dv_t = G_t^T k_t,  dS_{-1} = e^g G_0
 *
 * The decays are constants: they get no gradient.
 *
 * Conventions: those of hydra_attn.h (device pointers unless marked HOST, 16-byte aligned; token-major bf16 tensors;
 * host checks before any HIP call, status codes, streams).  States are fp32 [n_seqs][n_heads][d_k][d_v].  Sums and
 * states are held in 32 bits; the products take weighted scores and states as bf16 values, in the forward as sums of two,
 * and what is added to a state as a sum of three where the state is an output, of two elsewhere.  q, k, v, d_o and the
 * states must be finite: a value that is not reaches rows of its sequence that do not depend on it.  Rows of the tensors
 * from cu_seqlens[n_seqs] on are neither read nor written.
 */
#ifndef HYDRA_LINEAR_H
#define HYDRA_LINEAR_H

#include "hydra_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t n_heads;                  /* 1 .. 4096                                         */
  int32_t n_kv_heads;               /* 0 for n_heads; divides n_heads: query head i uses K/V
                                       head i / (n_heads / n_kv_heads), with a state of its own */
  int32_t d_k;                      /* 64, 128 or 192                                    */
  int32_t d_v;                      /* 64 or 128                                         */
  float   scale;                    /* <= 0 selects 1/sqrt(d_k)                          */
  const int32_t* cu_seqlens;        /* HOST int32[n_seqs+1]: the sequences' boundaries in the
                                       rows, cu[0] = 0, nondecreasing; read only during the call */
  int32_t n_seqs;                   /* >= 1                                              */
  int32_t q_tok_stride;             /* elements from one token row to the next, as in      */
  int32_t k_tok_stride;             /* hydra_problem_t: 0 = dense, else at least that, a   */
  int32_t v_tok_stride;             /* multiple of 8 and below 2^22                        */
} hydra_linear_t;

/* Bytes of device workspace that the calls below need for `p` (host only; 0: `p` is invalid).  The calls write it:
 * two that overlap need one each. */
size_t hydra_linear_workspace_size(const hydra_linear_t* p);

/* Uploads the work plan of `p` into `workspace`, for calls with planned != 0, which only launch kernels (and can be
 * recorded into a graph): they return HYDRA_ERR_WORKSPACE where the workspace does not hold the plan of `p` (strides,
 * scale and d_k, d_v may differ within what the workspace holds), as in hydra_attn.h.  While the stream is recorded this
 * call, and the ones below without `planned`, return it too: the upload's source does not outlive them. */
int hydra_linear_plan(const hydra_linear_t* p, void* workspace, size_t workspace_bytes, void* stream);

/* q [T][H][d_k], k [T][Hkv][d_k], v [T][Hkv][d_v] bf16 with T = cu_seqlens[n_seqs] rows; decay: float[n_heads] log
 * decays, 4-byte aligned, read when the kernels run (-infinity forgets at once; above 0 states grow, and
 * e^(g n) over the n rows of a sequence has to fit 32 bits, n = 1 in hydra_linear_step).
 *   o          [T][H][d_v] bf16, or NULL: only the last states are computed
 *   state_in   NULL (zero), or the states that the sequences start from
 *   state_out  NULL, or receives their last states; may be state_in itself
 * A sequence without rows ends with the state that it starts from.  Outputs and the workspace must otherwise not overlap
 * each other or an input. */
int hydra_linear_fwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
                     const float* state_in, void* o, float* state_out, void* workspace, size_t workspace_bytes,
                     int32_t planned, void* stream);

/* d_o [T][H][d_v] bf16, d_state_out NULL (zero) or the gradients of the last states.  Writes dq [T][H][d_k],
 * dk [T][Hkv][d_k] and dv [T][Hkv][d_v] bf16 (dk and dv summed in 32 bits over the query heads of a K/V head) and, where it is
 * not NULL, d_state_in. */
int hydra_linear_bwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
                     const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
                     float* d_state_in, void* workspace, size_t workspace_bytes, int32_t planned, void* stream);

/* One token of each of n_rows sequences whose states lie in a pool: q [n_rows][H][d_k], k, v, o as above (dense),
 *   state      [n_slots][H][d_k][d_v] fp32
 *   state_out  the pool that receives the new states, state itself for in place; slots of no row keep what they hold
 *   slots      DEVICE int32[n_rows], 4-byte aligned, or NULL for row i's slot i (n_slots >= n_rows)
 * Rows whose slot is not in [0, n_slots) are padding: neither their o nor any state is written.  Rows of one slot are
 * taken in their order, as consecutive tokens of its sequence.  n_rows up to 65536, and
 * n_rows * n_heads * (d_v / 32) below 2^25. */
int hydra_linear_step(int32_t n_rows, int32_t n_slots, int32_t n_heads, int32_t n_kv_heads, int32_t d_k, int32_t d_v,
                      float scale, const void* q, const void* k, const void* v, const float* decay,
                      const float* state, float* state_out, const int32_t* slots, void* o, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HYDRA_LINEAR_H */
