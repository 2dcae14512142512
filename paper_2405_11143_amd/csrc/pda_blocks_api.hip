// Host side of the block tables and slot maps (declared in include/pda_blocks.h):
// validation and the launches.  Nothing here allocates memory or keeps state between calls.
#include <stdint.h>

#include "pda_blocks_internal.h"

namespace {

constexpr int32_t kMaxSeqs = 1 << 20;
constexpr int32_t kMaxBlocks = 1 << 27;     // 16 * num_blocks fits the slots' int32
constexpr int32_t kMaxRowBlocks = 1 << 24;  // (positions of up to 2^28)

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

int check_pool(int32_t num_seqs, int32_t num_blocks, int32_t max_blocks_per_seq) {
  if (num_seqs < 0 || num_seqs > kMaxSeqs || num_blocks < 1 || num_blocks > kMaxBlocks || max_blocks_per_seq < 1 ||
      max_blocks_per_seq > kMaxRowBlocks)
    return PDA_ERR_SHAPE;
  return PDA_OK;
}

int check_rows(const pda_token_rows* rows, int32_t num_seqs, pda::BlocksArgs* a) {
  a->rows = pda_token_rows{};
  a->uniform_rows = 0;
  if (!rows) return PDA_OK;
  if (rows->num_rows < 0) return PDA_ERR_SHAPE;
  if (!rows->row_start && rows->num_rows > 0 && (num_seqs == 0 || rows->num_rows % num_seqs != 0)) return PDA_ERR_SHAPE;
  if (!aligned(rows->row_start, 4) || !aligned(rows->positions, 4) || !aligned(rows->slots, 4)) return PDA_ERR_ALIGNMENT;
  a->rows = *rows;
  if (!rows->positions && !rows->slots) a->rows.num_rows = 0;
  if (!rows->row_start && num_seqs > 0) a->uniform_rows = a->rows.num_rows / num_seqs;
  return PDA_OK;
}

size_t workspace_of(int32_t num_seqs) {
  return num_seqs == 0 ? 0 : 4 * sizeof(int32_t) + (size_t)num_seqs * sizeof(pda::BlockMove);
}

bool overlap(const void* p, size_t bytes, const void* q, size_t more) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return p && q && bytes > 0 && more > 0 && (a < b ? b - a < bytes : a - b < more);
}

// Workgroups read lengths, row starts and ids while others write the map.
int check_apart(const pda::BlocksArgs& a, size_t workspace_bytes) {
  const size_t n = 4 * (size_t)a.rows.num_rows, seqs = 4 * (size_t)a.pool.num_seqs;
  for (const int32_t* out : {a.rows.positions, a.rows.slots}) {
    if (overlap(out, n, a.lens, seqs) || overlap(out, n, a.rows.row_start, seqs + 4) ||
        overlap(out, n, a.table, seqs * (size_t)a.pool.max_blocks_per_seq) || overlap(out, n, a.pool.held, seqs) ||
        overlap(out, n, a.pool.free_blocks, 4 * (size_t)a.pool.num_blocks) || overlap(out, n, a.pool.counts, 8) ||
        overlap(out, n, a.arrived, workspace_bytes))
      return PDA_ERR_VALUE;
  }
  return overlap(a.rows.positions, n, a.rows.slots, n) ? PDA_ERR_VALUE : PDA_OK;
}

}  // namespace

extern "C" {

int pda_blocks_workspace_bytes(const pda_block_pool* pool, size_t* bytes) {
  if (!pool || !bytes) return PDA_ERR_NULL;
  const int rc = check_pool(pool->num_seqs, pool->num_blocks, pool->max_blocks_per_seq);
  if (rc != PDA_OK) return rc;
  *bytes = workspace_of(pool->num_seqs);
  return PDA_OK;
}

int pda_blocks_resize(const pda_block_pool* pool, const int32_t* context_lens, const pda_token_rows* rows,
                      void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!pool) return PDA_ERR_NULL;
  int rc = check_pool(pool->num_seqs, pool->num_blocks, pool->max_blocks_per_seq);
  if (rc != PDA_OK) return rc;
  pda::BlocksArgs a;
  rc = check_rows(rows, pool->num_seqs, &a);
  if (rc != PDA_OK) return rc;
  if (pool->num_seqs > 0) {
    if (!pool->block_table || !pool->held || !pool->free_blocks || !pool->counts || !context_lens) return PDA_ERR_NULL;
    if (!aligned(pool->block_table, 4) || !aligned(pool->held, 4) || !aligned(pool->free_blocks, 4) ||
        !aligned(pool->counts, 4) || !aligned(context_lens, 4))
      return PDA_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < workspace_of(pool->num_seqs)) return PDA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return PDA_ERR_ALIGNMENT;
  } else if (a.rows.num_rows == 0) {
    return PDA_OK;
  }
  a.pool = *pool;
  a.lens = context_lens;
  a.table = pool->block_table;
  a.arrived = static_cast<int32_t*>(workspace);
  a.totals = a.arrived + 2;
  a.moves = reinterpret_cast<pda::BlockMove*>(a.totals + 2);
  rc = check_apart(a, workspace_of(pool->num_seqs));
  if (rc != PDA_OK) return rc;
  const hipError_t e = pool->num_seqs > 0 ? pda::launch_blocks_resize(a, stream) : pda::launch_slot_map(a, stream);
  return e == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

int pda_slot_map(int32_t num_seqs, int32_t num_blocks, int32_t max_blocks_per_seq, const int32_t* block_table,
                 const int32_t* context_lens, const pda_token_rows* rows, hipStream_t stream) {
  if (!rows) return PDA_ERR_NULL;
  int rc = check_pool(num_seqs, num_blocks, max_blocks_per_seq);
  if (rc != PDA_OK) return rc;
  pda::BlocksArgs a;
  rc = check_rows(rows, num_seqs, &a);
  if (rc != PDA_OK) return rc;
  if (rows->num_rows == 0) return PDA_OK;
  if (!rows->positions && !rows->slots) return PDA_ERR_NULL;
  if (num_seqs > 0 && (!block_table || !context_lens)) return PDA_ERR_NULL;
  if (!aligned(block_table, 4) || !aligned(context_lens, 4)) return PDA_ERR_ALIGNMENT;
  a.pool = pda_block_pool{num_seqs, num_blocks, max_blocks_per_seq, nullptr, nullptr, nullptr, nullptr};
  a.lens = context_lens;
  a.table = block_table;
  a.moves = nullptr;
  a.totals = a.arrived = nullptr;
  rc = check_apart(a, 0);
  if (rc != PDA_OK) return rc;
  return pda::launch_slot_map(a, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

}  // extern "C"
