/*
 * pda_fp8.h -- an 8-bit paged KV cache and rotary positions for the decode step
 * of pda.h.
 *
 * A decode step is bound by the bytes of the cache it reads.  Here the cache
 * holds 8-bit floating-point codes with one scale byte per token and KV head:
 * 2 D + 2 bytes per token and KV head instead of 4 D.  Four operations:
 *   pda_append_kv_fp8   the new tokens' keys rotated, keys and values quantised
 *                       and stored (and the queries rotated), in one launch
 *   pda_decode_fp8      attention of one or several new tokens per sequence
 *   pda_read_kv_fp8     rows of the cache back as contiguous bf16
 *   pda_rotary_apply    rotary positions of query and key rows by themselves
 *
 * The stored row.  A row x of D values (one token, one KV head, keys or
 * values) is kept as D e4m3 codes c_d (4 significant bits, largest 448) and a
 * scale byte s; it stands for c_d * 2^(s - 127).
 *   s = the smallest integer >= 1 with max|x_d| <= 448 * 2^(s - 127)
 *   c_d = x_d * 2^(127 - s) rounded to the nearest e4m3 value, ties to even
 * A row of zeros has s = 0.  A row that holds a NaN or an infinity has s = 255
 * and NaN codes: it reads as NaN, and the attention's result is NaN in the rows that
 * see it, and in no others.  A value of 2^128 or more is an infinity (an element of
 * 1.9375 * 2^127 or more rounds to one: code 256 under s = 247): it reads as one, and
 * the attention's rows that see it hold what it makes of them, or NaN; no others
 * change.  A power of two as the scale loses nothing
 * (the codes are floating point: whatever the scale, a value within 2^-15 of
 * the row's largest keeps its 4 bits), and both it and the codes' conversion
 * to bf16 are exact (under s = 1 and 2 values are rounded to the nearest multiple of
 * 2^-133, bf16's smallest).  Elements below 2^-6 / 448 of the row's largest lose bits
 * to e4m3's subnormals; a key's strong channels take nothing from the others
 * before that.
 *
 * Layouts (row-major, DEVICE pointers; q, k_new, v_new, block_table,
 * context_lens and out are those of pda.h):
 *   k_cache   e4m3  [num_blocks][num_kv_heads][D/64][4][16][2][8]
 *                    element d of slot o at [d/64][(d/8)%4][o][(d/32)%2][d%8]: the
 *                    16 bytes of (c, kg, o) are the two 8-element MFMA fragments
 *                    that lane 16 kg + o needs in k-steps 2c and 2c + 1
 *   v_cache   e4m3  [num_blocks][num_kv_heads][2][4][D/8][2][8]
 *                    element d of slot o at [(o/2)%2][o/4][d/8][o%2][d%8]: 16 bytes
 *                    are 8 columns of two neighbouring tokens
 *   kv_scale  uint8 [num_blocks][num_kv_heads][2][16]: the slots' bytes of K, then of V
 * All three 16-byte aligned.  A cache that a caller fills by itself follows the
 * same rules; larger scale bytes mean c_d * 2^(s - 127) too, and s = 0 zeros
 * whatever the codes (the attention takes them for c_d * 2^-127: below 2^-118).
 * NaN codes belong under s = 255 (under a byte below 247 they may also reach rows of
 * the same step that do not see them).
 * Slots past a context and blocks no sequence references are never
 * used, whatever they hold.
 *
 * Errors, ownership, streams and device contents are as in pda.h: host checks
 * first, nothing allocated, no state kept, every launch on `stream` (so a caller
 * may capture the calls into a graph), lengths clamped, block ids outside the pool
 * never dereferenced.  All pointers must belong to the device that `stream`
 * does.
 */
#ifndef PDA_FP8_H
#define PDA_FP8_H

#include "pda.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotary positions.  The first `rotary_dim` elements of a head row are
 * rotary_dim / 2 pairs; pair i of a token at position t is turned by the angle
 * t * inv_freq[i] and multiplied by `magnitude`:
 *   x' = m (x cos a - y sin a),  y' = m (y cos a + x sin a)
 * (interleaved 0: the pair is elements i and i + rotary_dim / 2; 1: elements 2i
 * and 2i + 1); the other elements are unchanged.  Angles are formed and
 * reduced in 64 bits, so far positions lose nothing.  `backward` 1 turns by
 * -a: the adjoint, i.e. the gradient with respect to x, y of a loss whose
 * gradient with respect to x', y' is given. */
typedef struct pda_rotary {
  int32_t rotary_dim;     /* a multiple of 16, 16 <= rotary_dim <= head_dim */
  int32_t interleaved;
  int32_t backward;
  float magnitude;        /* 1 unless the positions are scaled with PDA_ROTARY_RAMP; finite */
  const double *inv_freq; /* DEVICE fp64 [rotary_dim / 2], 8-byte aligned: radians per position */
} pda_rotary;

/* Scaling of the frequencies f_i = base^(-2i / rotary_dim) for contexts longer
 * than those a model was trained on (original_len), by published methods, to the letter
 * (a model trained with one needs exactly its frequencies): position interpolation
 * (arXiv 2306.15595), the "NTK-aware" change of the base, the wavelength bands of the
 * Llama-3 family's long-context versions, and YaRN (arXiv 2309.00071):
 *   PLAIN   none
 *   LINEAR  f / factor: positions interpolated
 *   BASE    base * factor^(R / (R - 2)): the lowest frequency is divided by factor,
 *           the highest stays (R = rotary_dim > 2)
 *   BANDS   wavelengths below original_len / high keep f, those above
 *           original_len / low take f / factor, between them the two are mixed
 *           linearly in original_len / wavelength
 *   RAMP    dimensions that turn more than `high` times over original_len keep f, those that
 *           turn less than `low` times take f / factor, between them a linear ramp in i
 *           (its ends rounded outwards to whole i); magnitude = 1 + ln(factor) / 10 */
enum pda_rotary_kind {
  PDA_ROTARY_PLAIN = 0, PDA_ROTARY_LINEAR = 1, PDA_ROTARY_BASE = 2, PDA_ROTARY_BANDS = 3, PDA_ROTARY_RAMP = 4
};
typedef struct pda_rotary_scaling {
  int32_t kind;
  double factor;       /* >= 1 */
  double original_len; /* > 0 (BANDS, RAMP) */
  double low, high;    /* 0 < low < high (BANDS, RAMP) */
} pda_rotary_scaling;

/* The frequencies, in HOST memory (rotary_dim / 2 doubles), and the magnitude
 * (may be NULL) for a pda_rotary; `scaling` NULL means PLAIN.  base > 1. */
int pda_rotary_inv_freq(int32_t rotary_dim, double base, const pda_rotary_scaling *scaling, double *inv_freq,
                        float *magnitude);

/* Rotate the rows of num_tokens tokens: q [T][num_q_heads][head_dim] into
 * q_out, and k [T][num_kv_heads][head_dim] into k_out (num_kv_heads 0: no
 * keys).  dtype PDA_DTYPE_BF16 or PDA_DTYPE_F32, the same for all; computed in
 * fp32, rounded once.  The strides are the elements from one token to the next
 * (at least heads * head_dim, so a projection's fused rows can be used where
 * they lie); the heads of a token are contiguous.  An output may be its own input
 * (same pointer and stride: in place); otherwise it overlaps no other buffer of the
 * call.  head_dim is a multiple of 8, at most 512; 16-byte aligned pointers and rows.
 * A token at a negative position is padding: its rows are neither read nor written.
 * `positions` is device int32 [T]. */
int pda_rotary_apply(const pda_rotary *rotary, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                     int32_t head_dim, int32_t dtype, const int32_t *positions, const void *q, int64_t q_stride,
                     void *q_out, int64_t q_out_stride, const void *k, int64_t k_stride, void *k_out,
                     int64_t k_out_stride, hipStream_t stream);

/* pda_append_kv for this cache: the keys and values of the n new tokens of every
 * sequence, quantised (and, with `rotary`, the keys rotated in fp32 before), stored
 * at positions L - n .. L - 1.  With `rotary`, q (bf16 [B][n][Hq][D]) is rotated
 * into q_out (which may be q) for the same positions in the same launch; q and
 * q_out NULL leave the queries out, `rotary` NULL stores the keys as they are (q
 * must then be NULL).  New tokens at negative positions are skipped (their rows of
 * q_out stay as they are), and so is the store of a token whose block id is outside
 * the pool.  rotary->backward must be 0.  Two new tokens of the same slot (block
 * tables that share a block that is written) must be the same bytes. */
int pda_append_kv_fp8(const pda_problem *prob, const pda_rotary *rotary, const void *q, void *q_out,
                      const void *k_new, const void *v_new, const int32_t *block_table, const int32_t *context_lens,
                      void *k_cache, void *v_cache, uint8_t *kv_scale, hipStream_t stream);

/* Plan of pda_decode_fp8 (its workspace differs from pda_decode's).  PDA_ERR_SHAPE also
 * for what its launches cannot hold: 2^24 or more work items (partitions x sequences x KV
 * heads x groups of up to 128 query rows), or more than 2^26 - 4 output rows where
 * contexts are split. */
int pda_plan_fp8(const pda_problem *prob, pda_plan_info *plan);

/* pda_decode over this cache: the softmax attention of pda.h with
 *   K[t][d] = k code * 2^(s_K - 127),  V[t][d] = v code * 2^(s_V - 127).
 * Both products run on exactly converted values with fp32 sums, so the result is
 * that of a bf16 cache holding the stored values: to fp32 accuracy (3e-7 of its norm)
 * where n Hq / Hkv is at most 32, and 2.5e-6 of its norm beyond, where the probabilities
 * are kept to 16 bits or more.  Scores (scale * q . K * log2 e) are below 2^30 in
 * magnitude: past that the references that probabilities are taken against are too coarse.
 * out is fp32 [B][n][Hq][D]; rows that see nothing are zero.  `workspace`: any contents,
 * pda_plan_fp8()'s workspace_bytes, 16-byte aligned; calls that overlap on the GPU
 * need separate ones. */
int pda_decode_fp8(const pda_problem *prob, const void *q, const void *k_cache, const void *v_cache,
                   const uint8_t *kv_scale, const int32_t *block_table, const int32_t *context_lens, float scale,
                   float *out, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Rows of the cache as bf16 (exact, as said above: a stored value has 4 significant bits).  Of
 * sequence b the tokens first_token[b], first_token[b] + 1, ... go to the rows
 * row_start[b] .. row_start[b + 1] - 1 of k_out and v_out
 * (bf16 [num_rows][num_kv_heads][D]), up to the end of its context; rows beyond that,
 * rows of no sequence and rows past num_rows are left as they were.  first_token
 * NULL means 0 everywhere; tokens before 0 are skipped (their rows left).  The rows of
 * a block whose id is outside the pool are NaN.  row_start is device int32 [B + 1],
 * non-decreasing; sequences whose row ranges overlap leave either's rows. */
int pda_read_kv_fp8(const pda_problem *prob, const void *k_cache, const void *v_cache, const uint8_t *kv_scale,
                    const int32_t *block_table, const int32_t *context_lens, const int32_t *first_token,
                    const int32_t *row_start, int32_t num_rows, void *k_out, void *v_out, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDA_FP8_H */
