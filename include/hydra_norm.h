/*
 * hydra_norm.h -- the norm of every head with an activation or a gate, fused with the rank-local half of the reverse
 * Ulysses exchange, on AMD MI355X.
 *
 * What follows linear attention (hydra_linear.h) before the output projection, whose rows have no softmax to keep their
 * size: a group norm whose groups are the heads, channels last.  For one token and head with channels x[0 .. d):
 *
 *   m = mean(x) with center, else 0        r = 1 / sqrt(mean((x - m)^2) + eps)
 *   z = (x - m) r weight + bias            weight, bias per head and channel; without them 1 and 0
 *   y = z act(gate)                        with gate logits per head and channel, or
 *   y = act(z)                             without
 *
 * act is the logistic sigmoid, s(t) = 1 / (1 + exp(-t)), or silu, t s(t).  Backward, with dz = dY act(gate) or
 * dY act'(z), x' = (x - m) r and u = dz weight:
 *
 *   d_gate = dY z act'(gate),  d_weight = sum over tokens of dz x',  d_bias = sum over tokens of dz,
 *   d_x = r (u - mean(u) [with center] - x' mean(u x'))
 *
 * As in hydra_gate.h, x arrives from the reverse (head -> sequence) exchange and d_x leaves for the backward one, and
 * with cp_u = 1 the calls are the plain norm.
 *
 * Conventions: those of hydra_gate.h; weight, bias and their gradients are fp32.  Sums are in 32 bits, each bf16 output
 * is rounded once; results are deterministic.  x is finite and at most 2^58 in size: the sum of its squares, of up to 512
 * channels, has to fit 32 bits.  A value that is not finite reaches no other token and head than its own but through the
 * sums over tokens: d_weight, and d_bias, in which x has no part where there is a gate.
 */
#ifndef HYDRA_NORM_H
#define HYDRA_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "hydra_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HYDRA_ACT_SIGMOID 0
#define HYDRA_ACT_SILU    1

typedef struct {
  int64_t n_tokens;    /* T, 0 .. 2^31                                                   */
  int32_t n_heads;     /* H, 1 .. 65536, a multiple of cp_u                              */
  int32_t d;           /* channels of a head, a power of two from 8 to 512               */
  int32_t cp_u;
  int32_t center;      /* 0: m = 0 (root mean square norm)                               */
  int32_t activation;  /* HYDRA_ACT_*                                                    */
  float   eps;         /* at least 2^-126                                                */
} hydra_norm_t;

/* x [cp_u][T][H/cp_u][d] bf16 (buffer j: this rank's tokens of head group j), weight, bias [H][d] fp32 or NULL,
 * gate [T][H][d] bf16 or NULL -> y [T][H][d] bf16.  n_tokens = 0 is a no-op.
 * Errors: HYDRA_ERR_INVALID (sizes, NULL, overlap), HYDRA_ERR_ALIGN, HYDRA_ERR_HIP. */
int hydra_unpack_heads_normed(const hydra_norm_t* p, const void* x, const float* weight, const float* bias,
                              const void* gate, void* y, void* stream);

/* Bytes of device workspace that the backward needs for d_weight and d_bias (host only; 0: invalid sizes). */
size_t hydra_norm_workspace_size(int64_t n_tokens, int32_t n_heads, int32_t d);

/* Writes d_x [cp_u][T][H/cp_u][d] bf16, d_gate [T][H][d] bf16 (NULL without a gate), and where they are not NULL
 * d_weight and d_bias [H][d] fp32 (d_weight needs weight, d_bias bias).  workspace, which the call writes (two that
 * overlap need one each), may be NULL where neither is asked for.  With n_tokens = 0 these two are zero. */
int hydra_pack_heads_normed_bwd(const hydra_norm_t* p, const void* x, const float* weight, const float* bias,
                                const void* gate, const void* d_y, void* d_x, void* d_gate, float* d_weight,
                                float* d_bias, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HYDRA_NORM_H */
