// Internal interface of the block tables and slot maps (include/pda_blocks.h), between
// their host layer and their gfx950 kernels.
#pragma once

#include "pda_blocks.h"
#include "pda_internal.h"

namespace pda {

// What the plan of a resize leaves for the kernel that moves the ids: per sequence the
// entries held before, the rank of its first entry put back and that of its
// first entry granted.
struct BlockMove {
  int32_t held, back, grant;
};

struct BlocksArgs {
  pda_block_pool pool;
  const int32_t* lens;
  const int32_t* table;  // (of the pool, or the slot map's own)
  pda_token_rows rows;
  int32_t uniform_rows;  // rows per sequence where row_start is null
  int32_t* arrived;      // (workspace) workgroups that have read the held counts; 0 between calls
  BlockMove* moves;      // [num_seqs] (workspace)
  int32_t* totals;       // [2] (workspace): free blocks before, blocks put back
};

hipError_t launch_blocks_resize(const BlocksArgs& a, hipStream_t stream);
hipError_t launch_slot_map(const BlocksArgs& a, hipStream_t stream);

}  // namespace pda
