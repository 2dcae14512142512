/*
 * pda_window.h -- paged attention with a sliding window and a few first tokens that
 * stay visible (sinks), over the cache of pda.h: layers that look at the last `window`
 * tokens only, and long generations that keep the first ones beside them.
 *
 * The step is pda_decode's (one or several new tokens per sequence, its layouts,
 * descriptor, clamping and errors) with another mask: new token i of a sequence of length L
 * sits at position p = L - n + i and sees the tokens t <= p with
 *   t > p - window   or   t < num_sinks
 * so itself and the window - 1 tokens before it, and the sinks.  A window of
 * max_context_len or more is pda_decode's mask.
 *
 * Only the table entries and cache blocks that some new token of a sequence sees are
 * read: entries of blocks that lie behind every window and past the sinks may hold
 * anything, so a caller may give those blocks to other sequences.  Tokens that a row does
 * not see never reach its result, whatever their slots hold (NaN included; its rounding
 * may depend on the other rows of its work item).  Of the tokens that it sees, one whose score is NaN
 * or plus infinity makes the row non-finite, and a NaN or infinite element of a value the row's
 * element there; one whose score is minus infinity counts nothing, and a row that sees no others is zero,
 * as if it saw nothing.  A block id outside the pool among those read
 * makes the rows of the work item that meets it NaN.
 */
#ifndef PDA_WINDOW_H
#define PDA_WINDOW_H

#include "pda.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pda_window {
  int32_t window;     /* >= 1 */
  int32_t num_sinks;  /* >= 0 */
} pda_window;

/* Plan of pda_decode_window; prob->partition_tokens counts the tokens that are
 * read (a multiple of 16, rounded up to one of 32 for more than 32 query rows per KV head).
 * PDA_ERR_SHAPE also for what its launches cannot hold: more than 2^24 - 1 work items
 * (partitions x sequences x KV heads x groups of up to 128 query rows; with more than 32 rows per KV
 * head, sequences x KV heads count as the next multiple of 8) or 2^26 - 4 output rows where
 * contexts are split. */
int pda_plan_window(const pda_problem *prob, const pda_window *window, pda_plan_info *plan);

/* The attention of one step; out is fp32 [B][n][Hq][D], rows that see nothing are
 * zero.  Everything is computed to fp32 accuracy: with scores of the order of 1 (in units of log2) an
 * output is off by less than 1e-6 of its norm; what larger scores add is fp32's rounding of them.
 * `workspace`: any contents, pda_plan_window()'s workspace_bytes, 16-byte
 * aligned (NULL where that is 0); calls that overlap on the GPU need separate ones.  Results are bit-for-bit
 * reproducible for a descriptor. */
int pda_decode_window(const pda_problem *prob, const pda_window *window, const void *q, const void *k_cache,
                      const void *v_cache, const int32_t *block_table, const int32_t *context_lens, float scale,
                      float *out, void *workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDA_WINDOW_H */
