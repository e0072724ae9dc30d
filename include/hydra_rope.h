/*
 * hydra_rope.h -- rotary positions with several axes, between an attention layer's projections and its
 * attention share on AMD MI355X (gfx950).
 *
 * What enters the exchange of an MLA layer is q after its rotation, v after the split, and k after the
 * rotation and the concatenation (Sec. 5.2.2).  These calls make them, in one pass over the projections'
 * outputs and in the layout that the exchange sends (hydra_layout.h), and turn the gradients that
 * come back into the gradients of the projections' outputs:
 *
 *   hydra_rope_q       q [T][H][d]                          -> q rotated
 *   hydra_rope_kv      kv [T][H][d_nope + d_v], k_pe [T][r] -> k [d_nope | k_pe rotated] per head, and v
 *   hydra_rope_q_bwd   dq                                   -> gradient of q
 *   hydra_rope_kv_bwd  dk, dv                               -> gradients of kv and of k_pe (summed over heads)
 *
 * The last r = 2 * (sum of pairs) columns of each query head, and the r columns of k_pe, which all heads
 * share, are rotated in pairs.  Pair j takes the position p of its axis and the frequency f_j:
 *
 *   a' = a cos(p f_j) - b sin(p f_j),   b' = b cos(p f_j) + a sin(p f_j)
 *
 * The angle is exact to 2^-24 of a turn for every int32 position (p f_j / 2 pi is formed modulo one turn in
 * 64-bit fixed point).  Rotations and the sum over heads are computed in 32 bits and rounded once.
 *
 * Conventions: device pointers unless marked HOST, 16-byte aligned (positions: 4); bf16 tensors as raw
 * 16-bit patterns; token rows of inputs from projections and of their gradients are tok_stride elements
 * apart (0: dense, else at least the row's width and a multiple of 8, below 2^30), every other tensor is dense.
 * [G] stands for send buffers [cp_u][T][H/cp_u][*] (cp_u = 1: [T][H][*]).  Arguments are checked on the host before any
 * HIP call (status codes and hydra_strerror are those of hydra_attn.h); outputs must not overlap each other
 * or an input (strided rows of one stride may be columns of one buffer).  A call enqueues one kernel on
 * `stream`, allocates nothing and writes every element of its outputs; what lies between token rows of a strided
 * output stays as it is.  n_tokens = 0 is a no-op.
 */
#ifndef HYDRA_ROPE_H
#define HYDRA_ROPE_H

#include <stdint.h>

#include "hydra_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HYDRA_ROPE_MAX_AXES 4
#define HYDRA_ROPE_MAX_PAIRS 128

/* Which columns (of the r) pair j rotates; axis a's pairs are j0 .. j0 + pairs[a] - 1. */
#define HYDRA_ROPE_INTERLEAVED 0  /* 2 j and 2 j + 1                                              */
#define HYDRA_ROPE_HALVES      1  /* j and j + r / 2                                              */
#define HYDRA_ROPE_AXIS_HALVES 2  /* j0 + j and j0 + j + pairs[a]: each axis has columns of its own */

typedef struct {
  int32_t n_axes;                        /* 1 .. 4: text 1, images 2, video (time, height, width) 3 */
  int32_t pairs[HYDRA_ROPE_MAX_AXES];    /* pairs of each axis, at least 1; their sum is a multiple of 4
                                            and at most 128                                        */
  int32_t pairing;                       /* HYDRA_ROPE_*                                           */
  int32_t per_axis;                      /* 0: f_j = base^(-j / sum of pairs); 1: each axis anew,
                                            f_j = base^(-(j - j0) / pairs[a])                      */
  double base;                           /* >= 1, finite; not read with inv_freq                    */
  const double* inv_freq;                /* NULL, or HOST double[sum of pairs]: f_j in radians per
                                            position, finite, |f_j| <= 2^20 (scaled frequencies)   */
} hydra_rope_t;

/* Limits: n_tokens <= 2^30, n_heads <= 4096 and a multiple of cp_u, d_head, d_nope and d_v multiples of 8,
 * r <= d_head <= 512, d_nope + d_v <= 512, positions int32 [n_axes][n_tokens]. */

/* q [T][H][d_head] bf16 -> dst [G][d_head] bf16.  dst == src (with cp_u = 1): in place, in src's rows; the
 * columns that are not rotated are then not touched. */
int hydra_rope_q(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_head, int32_t cp_u,
                 const void* src, int64_t src_tok_stride, const int32_t* positions, void* dst, void* stream);

/* kv [T][H][d_nope + d_v] bf16 (a head's keys, then its values), k_pe [T][r] bf16
 * -> k [G][d_nope + r] bf16, v [G][d_v] bf16 (NULL when d_v = 0). */
int hydra_rope_kv(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_nope, int32_t d_v, int32_t cp_u,
                  const void* kv, int64_t kv_tok_stride, const void* k_pe, int64_t pe_tok_stride,
                  const int32_t* positions, void* k, void* v, void* stream);

/* dq [G][d_head], fp32 (grad_bytes = 4: the attention's accumulator) or bf16 (2) -> d_src [T][H][d_head] bf16. */
int hydra_rope_q_bwd(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_head, int32_t cp_u,
                     int32_t grad_bytes, const void* dq, const int32_t* positions, void* d_src, int64_t src_tok_stride,
                     void* stream);

/* dk [G][d_nope + r] and dv [G][d_v] (NULL when d_v = 0), fp32 or bf16 -> d_kv [T][H][d_nope + d_v] bf16 and
 * d_k_pe [T][r] bf16, the sum over the n_heads heads, in one order whatever the launch. */
int hydra_rope_kv_bwd(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_nope, int32_t d_v,
                      int32_t cp_u, int32_t grad_bytes, const void* dk, const void* dv, const int32_t* positions,
                      void* d_kv, int64_t kv_tok_stride, void* d_k_pe, int64_t pe_tok_stride, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HYDRA_ROPE_H */
