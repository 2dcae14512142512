/*
 * pda_blocks.h -- the block tables of a running batch, and the slot maps of its new
 * tokens, kept on the GPU (the KV-cache management of the rollout stage: paging,
 * Section 3.2 and Appendix C of the paper): a step's lengths are all that the host, or a kernel
 * before, has to provide, and nothing comes back to the host.
 *
 * A block pool is a block table int32 [num_seqs][max_blocks_per_seq] (pda.h), the
 * number of entries of each row that hold a block, `held` int32 [num_seqs], and a
 * stack of the free blocks' ids, free_blocks int32 [num_blocks], of which the first
 * counts[0] are the stack, its top last.  All are DEVICE buffers of the caller; a
 * block id is in one row or on the stack, once.  Entries of a row past its `held` and
 * of the stack past its size hold anything.
 *
 * pda_blocks_resize makes every row hold ceil(L / 16) blocks, L = context_lens[b]
 * clamped to [0, 16 max_blocks_per_seq]:
 *  1. rows that hold more put the entries past it back: with all of these entries in
 *     the order of the sequences, and in each of its entries, the first ends on top of the
 *     stack;
 *  2. rows that hold less are granted what is missing from the top of the stack, in the order of
 *     the sequences, their entries in order.  A row whose blocks, with those of
 *     all rows before it, are more than the stack holds is not granted: it keeps
 *     what it has, and so does every row after it that needs any.  counts[1]
 *     becomes the number of blocks that are missing for all to be granted (0: all were).
 * So a length of 0 releases a sequence, growing and then shrinking to the old lengths
 * restores table, `held` and stack, and the outcome depends on the contents alone.
 * Past its `held`, a row that was not granted may name blocks that it gave back and other rows own by
 * now: given that row's length, attention would read their tokens.  A caller whose blocks may run short
 * gives attention a length of 0 where 16 held[b] < L, formed from `held` on the GPU: the row is left out.
 *
 * Slot maps.  Row r of a packed batch of new tokens, row_start[b] <= r <
 * row_start[b + 1], is new token i = r - row_start[b] of sequence b, whose last new
 * token is at position L - 1: it gets
 *   positions[r] = L - (row_start[b + 1] - row_start[b]) + i
 *   slots[r] = 16 * (id of its block) + position % 16
 * A negative position (more new tokens than L: padding in front) and rows of no sequence get -1 for
 * both; a position whose entry is not held (a row that was not granted its blocks), or holds an id outside the
 * pool, gets its position and slot -1.
 *
 * Errors, ownership and streams are as in pda.h: host checks first, nothing allocated,
 * no state kept beside the caller's buffers, every launch on `stream` (so a caller may capture the
 * calls into a graph).  Calls on one pool must not overlap on the GPU.  Device contents are the
 * caller's contract; whatever they are, no access leaves the buffers.
 */
#ifndef PDA_BLOCKS_H
#define PDA_BLOCKS_H

#include "pda.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pda_block_pool {
  int32_t num_seqs;            /* rows of the table, 0 .. 2^20 */
  int32_t num_blocks;          /* 1 .. 2^27 */
  int32_t max_blocks_per_seq;  /* 1 .. 2^24 */
  int32_t *block_table;        /* DEVICE int32 [num_seqs][max_blocks_per_seq] */
  int32_t *held;               /* DEVICE int32 [num_seqs] */
  int32_t *free_blocks;        /* DEVICE int32 [num_blocks] */
  int32_t *counts;             /* DEVICE int32 [2]: free blocks; blocks the last resize lacked */
} pda_block_pool;

/* The rows of a batch of new tokens. */
typedef struct pda_token_rows {
  int32_t num_rows;           /* >= 0 */
  const int32_t *row_start;   /* DEVICE int32 [num_seqs + 1], non-decreasing, within [0, num_rows]; NULL: num_rows /
                                 num_seqs rows to each sequence (then num_rows is a multiple of num_seqs) */
  int32_t *positions;         /* DEVICE int32 [num_rows], written; NULL: left out */
  int32_t *slots;             /* DEVICE int32 [num_rows], written; NULL: left out */
} pda_token_rows;

/* Workspace of pda_blocks_resize (0 for no sequences). */
int pda_blocks_workspace_bytes(const pda_block_pool *pool, size_t *bytes);

/* Resize every row for context_lens (device int32 [num_seqs]) and, with `rows` (may be
 * NULL), write the slot map of its rows.  `workspace`: pda_blocks_workspace_bytes() bytes,
 * 16-byte aligned, filled with ZEROS before its first use; a call leaves it ready for the
 * next one (of any pool), and calls that overlap on the GPU need separate ones.
 * context_lens, row_start, positions and slots overlap no buffer of the pool; positions and slots
 * overlap no other buffer of the call at all (PDA_ERR_VALUE). */
int pda_blocks_resize(const pda_block_pool *pool, const int32_t *context_lens, const pda_token_rows *rows,
                      void *workspace, size_t workspace_bytes, hipStream_t stream);

/* The slot map alone, for a block table however it was made (every entry counts as
 * held).  positions and slots may not both be NULL unless num_rows is 0, and overlap no other
 * buffer of the call (PDA_ERR_VALUE). */
int pda_slot_map(int32_t num_seqs, int32_t num_blocks, int32_t max_blocks_per_seq, const int32_t *block_table,
                 const int32_t *context_lens, const pda_token_rows *rows, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDA_BLOCKS_H */
