// Internal interface of attention with a sliding window and sinks
// (include/pda_window.h), between its host layer and its gfx950 kernels.
#pragma once

#include "pda_window.h"
#include "pda_internal.h"

namespace pda {

// Arguments of a step (passed by value).  `step` holds the buffers and sizes of
// pda_decode; of its plan only the fields named here are used: partition_tokens
// (whole blocks, an even number of them in the wide kernel), num_partitions and slots_per_row (the most that a
// row has), part_o / part_m / part_l, query_chunk and num_regular_items.
struct WindowArgs {
  StepArgs step;
  int32_t window, sinks;
  int32_t group_tokens;  // new tokens of a work item (they share its tiles)
  int32_t num_groups;    // ceil(n / group_tokens)
};

constexpr int kWindowTileRows = 16;     // query rows of an MFMA tile of the narrow kernel
constexpr int kWindowNarrowRows = 32;   // most query rows of a work item there: two tiles
constexpr int kWindowWideRows = 128;    // and of the wide kernel: 4 wavefronts of 32
constexpr int kWindowUnit = kBlockTokens;
constexpr int kWindowXcds = 8;          // the wide kernel launches a (sequence, KV head) for each, in turn

// The blocks that new tokens [i0, i1) of a sequence of length L see something of, as a list: the
// sinks' blocks [0, sinks), then [first, end).
struct WindowSpan {
  int sinks, first, end;
  __host__ __device__ int count() const { return sinks + (end - first); }
  // Entry v of the list, and its first token.
  __host__ __device__ int block(int v) const { return v < sinks ? v : v - sinks + first; }
  __host__ __device__ int token(int v) const { return block(v) * kWindowUnit; }
};

// First token of the window of a row that sees tokens below `up`.
__host__ __device__ inline int window_start(int up, int window) { return up > window ? up - window : 0; }

__host__ __device__ inline WindowSpan window_span(int L, int n, int i0, int i1, int window, int sinks) {
  const int end = L - n + i1;  // of the last row
  if (end <= 0) return WindowSpan{0, 0, 0};
  const int lo = window_start(L - n + i0 + 1, window);
  const int s = ((sinks < lo ? sinks : lo) + kWindowUnit - 1) / kWindowUnit;
  const int first = lo / kWindowUnit, last = (end - 1) / kWindowUnit + 1;
  if (first <= s) return WindowSpan{0, 0, last};  // nothing left out between
  return WindowSpan{s, first, last};
}

// Partitions of the list of group `gr` of new tokens (0: it sees nothing).
__host__ __device__ inline int window_partitions(const WindowArgs& a, int L, int gr) {
  const int n = a.step.num_query_tokens, i0 = gr * a.group_tokens;
  const int i1 = i0 + a.group_tokens < n ? i0 + a.group_tokens : n;
  const int blocks = a.step.partition_tokens / kWindowUnit;
  return (window_span(L, n, i0, i1, a.window, a.sinks).count() + blocks - 1) / blocks;
}

hipError_t launch_window(const WindowArgs& a, int head_dim, hipStream_t stream);        // up to kWindowNarrowRows rows
hipError_t launch_window_wide(const WindowArgs& a, int head_dim, hipStream_t stream);   // more
hipError_t launch_window_merge(const WindowArgs& a, int head_dim, hipStream_t stream);

}  // namespace pda
