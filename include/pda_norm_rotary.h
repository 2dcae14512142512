/*
 * pda_norm_rotary.h -- norms of query and key heads, rotary positions with several
 * axes, and the append through a slot map: what a layer does with its fused
 * projection's rows before attention (pda.h), and the gradient of it.
 *
 * A head row x of D values of one token, with the norm's weight w (one for all query
 * heads, one for all key heads), becomes
 *   u = x / sqrt(mean_d x_d^2 + eps),  z = u * (w + weight_offset),  y = R z
 * where R turns the first rotary_dim elements in pairs as pda_rotary says
 * (pda_fp8.h).  Everything is computed in fp32 and rounded once; an angle is formed in 64 bits, whole
 * turns are taken off it, and what is left is fp32, within 2^-25 turns however far the position.
 * Either step may be left out: `norm` NULL, `rotary` NULL.
 *
 * Several axes.  With pda_rotary_axes a token has a position on each axis (time,
 * height and width of an image's patches; all the same for text), and pair i is
 * turned by position[axis_of_pair[i]] * inv_freq[i].  Any arrangement is one such
 * map: contiguous sections, or axes in turn.
 *
 * Rows.  q is [T][num_q_heads][D], k [T][num_kv_heads][D]; the strides are the
 * elements from one token to the next (at least heads * D), the heads of a token are
 * contiguous: the parts of a fused projection's rows can be used where they lie.
 * num_kv_heads 0: no keys.  dtype PDA_DTYPE_BF16 or PDA_DTYPE_F32, the same for all rows of a
 * call.  D is a multiple of 8, at most 512; pointers and rows are 16-byte aligned.
 * Elements are below 2^59 in magnitude (their squares are summed in fp32); with eps below 2^-118 a
 * row's largest is above 2^-59, or all are zero.
 * `positions` is device int32 [T], or [num_axes] rows of T.  A token whose position
 * (on the first axis) is negative is padding: its rows are neither read nor
 * written.  Positions on further axes may have either sign.
 *
 * Errors, ownership and streams are as in pda.h: host checks first, nothing
 * allocated, no state kept, every launch on `stream` (so a caller may capture the
 * calls into a graph).  All pointers belong to the device that `stream` does.
 */
#ifndef PDA_NORM_ROTARY_H
#define PDA_NORM_ROTARY_H

#include "pda_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The norms of query and key heads. */
typedef struct pda_head_norm {
  float eps;             /* >= 0, finite (0: a row of zeros becomes NaN) */
  float weight_offset;   /* added to the weights: 1 where they are stored about zero; finite */
  int32_t weight_dtype;  /* PDA_DTYPE_BF16 or PDA_DTYPE_F32 */
  const void *q_weight;  /* DEVICE [D], 16-byte aligned; NULL: no weights (all ones, without the offset) */
  const void *k_weight;
} pda_head_norm;

/* Positions on several axes. */
typedef struct pda_rotary_axes {
  int32_t num_axes;             /* 1 .. 4 */
  const uint8_t *axis_of_pair;  /* DEVICE [rotary_dim / 2]: each pair's axis (num_axes or more is taken for 0) */
  int64_t position_stride;      /* elements of `positions` from one axis to the next, at least T */
} pda_rotary_axes;

/* y of q into q_out and of k into k_out.  An output may be its own input (same
 * pointer and stride); otherwise it overlaps no other buffer of the call.  `axes` NULL: one.
 * (The rotation alone on one axis is pda_rotary_apply, the faster call for it; the two agree but for the last
 * rounding.)
 * Without `norm`, rotary->backward 1 turns back (the gradient of the rotation);
 * with it, backward must be 0.  `norm` and `rotary` may not both be NULL. */
int pda_norm_rotary(const pda_head_norm *norm, const pda_rotary *rotary, const pda_rotary_axes *axes,
                    int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t dtype,
                    const int32_t *positions, const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride,
                    const void *k, int64_t k_stride, void *k_out, int64_t k_out_stride, hipStream_t stream);

/* The gradient of pda_norm_rotary with norms.  q and k are its inputs, q_grad and
 * k_grad the gradients of a loss with respect to its outputs, dq and dk receive those
 * with respect to its inputs, dq_weight and dk_weight (fp32 [D], either may be NULL: left
 * out) those with respect to the weights, overwritten.  With h = R^T g,
 * u = x / s, s = sqrt(mean x^2 + eps), f = h * (w + weight_offset):
 *   dx = (f - u mean(f u)) / s,   dw = sum over tokens and heads of h u
 * `rotary` is the forward's (backward 0).  dq may be q_grad or q, dk k_grad or k (same pointer and
 * stride).  Padding rows of dq and dk are left as they were, and add nothing to the
 * weights' gradients.  The sums run in a fixed order: results are reproducible.
 * `workspace`: pda_norm_rotary_workspace_bytes() bytes, any contents, 16-byte aligned; calls
 * that overlap on the GPU need separate ones. */
int pda_norm_rotary_workspace_bytes(int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                    size_t *bytes);
int pda_norm_rotary_backward(const pda_head_norm *norm, const pda_rotary *rotary, const pda_rotary_axes *axes,
                             int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                             int32_t dtype, const int32_t *positions, const void *q, int64_t q_stride,
                             const void *q_grad, int64_t q_grad_stride, void *dq, int64_t dq_stride, const void *k,
                             int64_t k_stride, const void *k_grad, int64_t k_grad_stride, void *dk,
                             int64_t dk_stride, float *dq_weight, float *dk_weight, void *workspace,
                             size_t workspace_bytes, hipStream_t stream);

/* pda_norm_rotary over bf16 rows of packed tokens, with the keys, and the values v
 * [T][num_kv_heads][D] as they are, stored in the paged cache of pda.h: token t's in slot
 * slots[t] = 16 * block + place in the block (pda_blocks.h makes such maps).  A slot
 * outside [0, 16 num_blocks) stores nothing; a padding token neither stores nor
 * writes its row of q_out.  num_q_heads 0: no queries (q and q_out NULL).  `norm`
 * and `rotary` may both be NULL: the keys are stored as they are, and the queries must be left
 * out.  D is 64 or 128.  Two tokens of the same slot must hold the same bytes.
 * Nothing else in the cache changes. */
int pda_norm_rotary_append(const pda_head_norm *norm, const pda_rotary *rotary, const pda_rotary_axes *axes,
                           int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                           int32_t num_blocks, const int32_t *positions, const int32_t *slots, const void *q,
                           int64_t q_stride, void *q_out, int64_t q_out_stride, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, void *k_cache, void *v_cache, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDA_NORM_ROTARY_H */
