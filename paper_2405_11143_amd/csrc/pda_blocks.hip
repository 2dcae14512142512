// Block tables and slot maps on the GPU (include/pda_blocks.h).
//
// A resize moves few bytes; what it costs is a chain of latencies.  The ranks of the
// entries that move are prefix sums over the sequences:
//   back_b  = sum over a < b of max(0, held_a - need_a)   entries put back before b's
//   want_b  = sum over a < b of max(0, need_a - held_a)   entries wanted before b's
// With F entries put back onto a stack of C, entry r of them goes to place C + F - 1 - r, and
// entry x granted comes from place C + F - 1 - x: it is entry x put back where x < F
// (read from its row, not from the stack, so nothing here waits for another
// workgroup's store), else the old stack's place C - 1 - (x - F).
//
// One workgroup forms the sums and the new counts (plan_kernel); then a workgroup for every
// kSpan entries of every row moves that row's ids and writes the slots of the tokens in those
// blocks (move_kernel).
#include "pda_blocks_internal.h"

namespace pda {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWaveSize;
constexpr int kMoveThreads = 256;
constexpr int kSpan = 256;  // entries of a row per workgroup
constexpr unsigned kMaxGridY = 65535;

__device__ __forceinline__ int clamp_to(int x, int most) { return min(max(x, 0), most); }

__device__ __forceinline__ int blocks_for(const BlocksArgs& a, int len) {
  return clamp_to((int)(((int64_t)max(len, 0) + kBlockTokens - 1) / kBlockTokens), a.pool.max_blocks_per_seq);
}

// Inclusive sum of x over the workgroup's threads below and with this one, plus `carry`;
// the carry becomes the sum of all.  64-bit: held counts are the caller's.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t& carry, int64_t* lds) {
  const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == kWaveSize - 1) lds[wave] = x;
  __syncthreads();
  int64_t before = carry, all = carry;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? lds[w] : 0;
    all += lds[w];
  }
  __syncthreads();
  carry = all;
  return x + before;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const BlocksArgs a) {
  __shared__ int64_t lds[kPlanWaves];
  const int B = a.pool.num_seqs, most = a.pool.max_blocks_per_seq;
  const int count = clamp_to(a.pool.counts[0], a.pool.num_blocks);
  int64_t back = 0, want = 0, granted = 0;
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {  // what is put back
    const int b = b0 + threadIdx.x;
    const int held = b < B ? clamp_to(a.pool.held[b], most) : 0;
    const int need = b < B ? blocks_for(a, a.lens[b]) : 0;
    const int mine = max(held - need, 0);
    const int64_t upto = scan(mine, back, lds);
    if (b < B) {
      a.moves[b].held = held;
      a.moves[b].back = (int)min<int64_t>(upto - mine, a.pool.num_blocks);
    }
  }
  // (a stack cannot hold more than all blocks: the rest of what rows claim to hold is dropped)
  const int stack = (int)min<int64_t>(count + back, a.pool.num_blocks);
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {  // what is granted
    const int b = b0 + threadIdx.x;
    const int held = b < B ? clamp_to(a.pool.held[b], most) : 0;
    const int need = b < B ? blocks_for(a, a.lens[b]) : 0;
    const int mine = max(need - held, 0);
    const int64_t upto = scan(mine, want, lds);
    const bool fits = upto <= stack;
    if (b < B) {
      a.moves[b].grant = fits && mine > 0 ? (int)(upto - mine) : -1;
      a.pool.held[b] = need <= held || fits ? need : held;
    }
    int64_t dummy = 0;
    scan(fits ? mine : 0, dummy, lds);
    granted += dummy;
  }
  if (threadIdx.x == 0) {
    a.totals[0] = count;
    a.totals[1] = stack - count;
    a.pool.counts[0] = stack - (int)granted;
    a.pool.counts[1] = (int)min<int64_t>(max<int64_t>(want - stack, 0), 0x7fffffff);
  }
}

// The row of the first entry put back whose rank is at most r.
__device__ __forceinline__ int row_of_rank(const BlocksArgs& a, int r) {
  int lo = 0, hi = a.pool.num_seqs - 1;  // the last row with back <= r
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.moves[mid].back <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Entry x granted: the id of its block.
__device__ __forceinline__ int granted_id(const BlocksArgs& a, int count, int back, int x) {
  if (x >= back) return a.pool.free_blocks[clamp_to(count - 1 - (x - back), a.pool.num_blocks - 1)];
  const int b = row_of_rank(a, x);
  const int j = blocks_for(a, a.lens[b]) + x - a.moves[b].back;
  return a.table[(size_t)b * a.pool.max_blocks_per_seq + clamp_to(j, a.pool.max_blocks_per_seq - 1)];
}

__device__ __forceinline__ void write_row(const BlocksArgs& a, int64_t r, int position, int slot) {
  if (a.rows.positions) a.rows.positions[r] = position;
  if (a.rows.slots) a.rows.slots[r] = slot;
}

// MOVE: a resize's moves and its slot map; otherwise the slot map of a table as it is.
template <bool MOVE>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const BlocksArgs a) {
  const int B = a.pool.num_seqs;
  const int n = a.rows.num_rows;
  const int b = blockIdx.x;
  const int width = a.pool.max_blocks_per_seq;
  if (b == B) {  // rows of no sequence
    const int first = B > 0 ? (a.rows.row_start ? clamp_to(a.rows.row_start[0], n) : 0) : n;
    const int last = B > 0 ? (a.rows.row_start ? clamp_to(a.rows.row_start[B], n) : n) : n;
    const int64_t step = (int64_t)gridDim.y * kMoveThreads, mine = (int64_t)blockIdx.y * kMoveThreads + threadIdx.x;
    for (int64_t r = mine; r < first; r += step) write_row(a, r, -1, -1);
    for (int64_t r = max(first, last) + mine; r < n; r += step) write_row(a, r, -1, -1);
    return;
  }
  int* const row = MOVE ? a.pool.block_table + (size_t)b * width : nullptr;
  const int L = (int)min<int64_t>(max(a.lens[b], 0), (int64_t)kBlockTokens * width);
  const int held_new = MOVE ? clamp_to(a.pool.held[b], width) : width;
  const int start = a.rows.row_start ? clamp_to(a.rows.row_start[b], n) : b * a.uniform_rows;
  const int end = a.rows.row_start ? clamp_to(a.rows.row_start[b + 1], n) : start + a.uniform_rows;
  const int64_t first = (int64_t)L - (end - start);  // position of row `start`
  for (int64_t j0 = (int64_t)blockIdx.y * kSpan; j0 < width; j0 += (int64_t)gridDim.y * kSpan) {
    if (MOVE) {
      const BlockMove m = a.moves[b];
      const int count = a.totals[0], back = a.totals[1];
      for (int j = (int)j0 + threadIdx.x; j < min<int64_t>(j0 + kSpan, width); j += kMoveThreads) {
        if (j >= m.held && j < held_new && m.grant >= 0) row[j] = granted_id(a, count, back, m.grant + j - m.held);
        if (j >= held_new && j < m.held) {
          const int rank = m.back + j - held_new;
          if (rank < back) a.pool.free_blocks[clamp_to(count + back - 1 - rank, a.pool.num_blocks - 1)] = row[j];
        }
      }
      __syncthreads();  // the slots below read what was granted
    }
    const int64_t t0 = max<int64_t>(j0 * kBlockTokens, max<int64_t>(first, 0));
    const int64_t t1 = min<int64_t>((j0 + kSpan) * kBlockTokens, L);
    for (int64_t t = t0 + threadIdx.x; t < t1; t += kMoveThreads) {
      const int j = (int)(t / kBlockTokens);
      const int id = j < held_new ? a.table[(size_t)b * width + j] : -1;
      const int slot = (unsigned)id < (unsigned)a.pool.num_blocks ? id * kBlockTokens + (int)(t % kBlockTokens) : -1;
      write_row(a, start + (t - first), (int)t, slot);
    }
  }
  if (blockIdx.y == 0)
    for (int64_t r = start + threadIdx.x; r < end && r - start + first < 0; r += kMoveThreads) write_row(a, r, -1, -1);
}

template <bool MOVE>
hipError_t launch_moves(const BlocksArgs& a, hipStream_t stream) {
  const unsigned spans = (unsigned)((a.pool.max_blocks_per_seq + kSpan - 1) / kSpan);
  hipLaunchKernelGGL((move_kernel<MOVE>), dim3(a.pool.num_seqs + (a.rows.num_rows > 0 ? 1 : 0), min(spans, kMaxGridY)),
                     dim3(kMoveThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_blocks_resize(const BlocksArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_moves<true>(a, stream) : e;
}

hipError_t launch_slot_map(const BlocksArgs& a, hipStream_t stream) { return launch_moves<false>(a, stream); }

}  // namespace pda
