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
// Up to kOneSeqs sequences it is one launch (resize_kernel): every workgroup forms all the sums,
// a thread to a sequence, and takes its share of the ids and of the slot map; the last one to
// have read the held counts writes the new ones.  For more, one workgroup forms the sums and
// the new counts (plan_kernel); then a workgroup for every kSpan entries of every row moves
// that row's ids and writes the slots of the tokens in those blocks (move_kernel).  5 new tokens of
// every sequence and back, two calls: 1024 sequences 13.6 us, 1025 24, 4096 49, 16384 169, most of it in the one workgroup.
// A slot map alone is move_kernel's second half, whose grid follows the table's width: a decode step's of 256
// sequences 3.9 us over tables of 4096 entries, 30 over tables of 65536, of whose 65792 workgroups 256 have work;
// of 48 prompts, 92000 rows, 5.1.
#include <algorithm>

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

// The whole resize, every workgroup with all the sums: the first workgroup moves up to kOwn of each
// row's ids, a row to a thread; what is left is shared out, a row to a wavefront or several, and the slot map
// a token row to a thread.  An id is read from where it was before the call, so no workgroup reads
// what another has written.  Two calls, us, against the two kernels: 256 sequences of up to 4096
// tokens, 5 new ones each and back, 11.8 / 16.1 (of which 4.4 a call are the calls themselves);
// all of their 33000 blocks granted and put back 16.3 / 16.1.  With one workgroup for everything the
// first took 9.8 and the second 32.  Two rows of 3750 blocks 19, with a wavefront to a row 29.
constexpr int kOneSeqs = kPlanThreads;
constexpr int kOwn = 4;
constexpr int64_t kEntriesEach = 4096, kRowsEach = 1024;  // of a workgroup
// With more token rows than this the two kernels take over, whose threads need not find
// their row's sequence.  Admitted and released in two calls, us, one launch each / two: 32000
// rows of 8 sequences 14.9 / 19.0, 25600 of 256 14.9 / 16.6, 64000 of 64 15.8 / 16.7, 115200
// of 128 17.4 / 17.2, 1 million of 512 24.5 / 20.4.
constexpr int kOneRows = 65536;
constexpr int64_t kMostGroups = 128;
constexpr int kAhead = 4;  // entries of a row that a lane has in flight
__global__ void __launch_bounds__(kPlanThreads) resize_kernel(const BlocksArgs a) {
  const int group = blockIdx.x, groups = gridDim.x;
  __shared__ int64_t sums[2][kPlanWaves];
  __shared__ int most_granted[kPlanWaves];
  __shared__ int back_at[kOneSeqs], need_of[kOneSeqs], held_of[kOneSeqs], grant_at[kOneSeqs], start_of[kOneSeqs + 1];
  __shared__ bool last;
  struct Rest {
    int row, from, count, rank;  // count below 0: put back
  };
  __shared__ Rest rest[kOneSeqs];
  __shared__ int rests[kPlanWaves];
  const int B = a.pool.num_seqs, width = a.pool.max_blocks_per_seq, n = a.rows.num_rows;
  const int b = threadIdx.x, lane = b % kWaveSize, wave = b / kWaveSize;
  const bool mine = b < B;
  const int held = mine ? clamp_to(a.pool.held[b], width) : 0;
  const int need = mine ? blocks_for(a, a.lens[b]) : 0;
  const int count = clamp_to(a.pool.counts[0], a.pool.num_blocks);
  if (n > 0 && a.rows.row_start) {
    if (b <= B) start_of[b] = clamp_to(a.rows.row_start[b], n);
    if (b == 0) start_of[B] = clamp_to(a.rows.row_start[B], n);
  }
  // both sums at once
  const int back = max(held - need, 0), want = max(need - held, 0);
  int64_t x = back, y = want;
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) {
    const int64_t p = __shfl_up(x, o), q = __shfl_up(y, o);
    if (lane >= o) x += p, y += q;
  }
  if (lane == kWaveSize - 1) sums[0][wave] = x, sums[1][wave] = y;
  __syncthreads();
  int64_t all_back = 0, all_want = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) x += sums[0][w], y += sums[1][w];
    all_back += sums[0][w], all_want += sums[1][w];
  }
  const int stack = (int)min<int64_t>(count + all_back, a.pool.num_blocks), put = stack - count;
  const bool fits = y <= stack;
  const int first_back = (int)min<int64_t>(x - back, a.pool.num_blocks), first_grant = fits ? (int)(y - want) : 0;
  const int held_new = need <= held || fits ? need : held;
  back_at[b] = mine ? first_back : 0x7fffffff, need_of[b] = need, held_of[b] = held;
  grant_at[b] = want > 0 && fits ? first_grant : -1;
  int g = fits ? (int)y : 0;  // (sums do not fall: the largest that fits is all that is granted)
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) g = max(g, __shfl_xor(g, o));
  if (lane == 0) most_granted[wave] = g;
  __syncthreads();
  if (groups > 1 && b == 0) last = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
  if (groups > 1) __syncthreads();
  if (groups == 1 || last) {  // every workgroup has read the counts (its sums are formed)
    if (mine) a.pool.held[b] = held_new;
    if (b == 0) {
#pragma unroll
      for (int w = 0; w < kPlanWaves; ++w) g = max(g, most_granted[w]);
      a.pool.counts[0] = stack - g;
      a.pool.counts[1] = (int)min<int64_t>(max<int64_t>(all_want - stack, 0), 0x7fffffff);
      if (groups > 1) *a.arrived = 0;  // for the next call
    }
  }
  // A row's moves: entries from, from + 1, ... (`grant`: granted, otherwise put back), of these ranks on.
  struct Moves {
    int row, from, count, rank;
    bool grant;
  };
  auto source = [&](const Moves& m, int e) -> const int32_t* {
    if (!m.grant) return a.pool.block_table + (size_t)m.row * width + m.from + e;
    const int r = m.rank + e;
    if (r >= put) return a.pool.free_blocks + clamp_to(count - 1 - (r - put), a.pool.num_blocks - 1);
    int lo = 0, hi = B - 1;  // an entry put back in this call: the last row whose ranks begin at or below it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (back_at[mid] <= r)
        lo = mid;
      else
        hi = mid - 1;
    }
    return a.pool.block_table + (size_t)lo * width + clamp_to(need_of[lo] + r - back_at[lo], width - 1);
  };
  auto store = [&](const Moves& m, int e, int id) {
    if (m.grant)
      a.pool.block_table[(size_t)m.row * width + m.from + e] = id;
    else if (m.rank + e < put)
      a.pool.free_blocks[clamp_to(stack - 1 - (m.rank + e), a.pool.num_blocks - 1)] = id;
  };
  const bool grows = want > 0 && fits;
  const Moves my{b, grows ? held : need, grows ? want : back, grows ? first_grant : first_back, grows};
  const int own = group == 0 ? min(my.count, kOwn) : 0;
  int ids[kOwn];
#pragma unroll
  for (int e = 0; e < kOwn; ++e)
    if (e < own) ids[e] = *source(my, e);
#pragma unroll
  for (int e = 0; e < kOwn; ++e)
    if (e < own) store(my, e, ids[e]);
  const bool more = my.count > kOwn;
  const uint64_t mask = __builtin_amdgcn_ballot_w64(more);
  if (lane == 0) rests[wave] = __builtin_popcountll(mask);
  __syncthreads();
  int place = __builtin_popcountll(mask & ((1ull << lane) - 1)), all_rests = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) place += w < wave ? rests[w] : 0, all_rests += rests[w];
  if (all_rests > 0) {  // (the same for all threads)
    if (more) rest[place] = Rest{b, my.from, grows ? my.count : -my.count, my.rank};
    __syncthreads();
    const int waves = groups * kPlanWaves;
    const int share = max(__builtin_clz(all_rests) - __builtin_clz(waves) - 1, 0);  // 2^share wavefronts to a row
    for (int i = group * kPlanWaves + wave; i < all_rests << share; i += waves) {
      const Rest x = rest[i >> share];
      const Moves m{x.row, x.from, abs(x.count), x.rank, x.count > 0};
      const int part = i & ((1 << share) - 1);
      for (int e0 = kOwn + part * kAhead * kWaveSize + lane; e0 < m.count; e0 += kAhead * kWaveSize << share) {
        int id[kAhead];
#pragma unroll
        for (int h = 0; h < kAhead; ++h)
          if (e0 + h * kWaveSize < m.count) id[h] = *source(m, e0 + h * kWaveSize);
#pragma unroll
        for (int h = 0; h < kAhead; ++h)
          if (e0 + h * kWaveSize < m.count) store(m, e0 + h * kWaveSize, id[h]);
      }
    }
  }
  // the slot map
  for (int64_t r = (int64_t)group * kPlanThreads + b; r < n; r += (int64_t)groups * kPlanThreads) {
    int row;
    int64_t t;
    if (a.rows.row_start) {
      int lo = 0, hi = B - 1;  // the last row that starts at or before r
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start_of[mid] <= r)
          lo = mid;
        else
          hi = mid - 1;
      }
      row = r >= start_of[lo] && r < start_of[lo + 1] ? lo : -1;
      t = r - start_of[lo + 1];
    } else {
      row = (int)r / a.uniform_rows;
      t = r - (int64_t)(row + 1) * a.uniform_rows;
    }
    if (row >= 0) t += (int)min<int64_t>(max(a.lens[row], 0), (int64_t)kBlockTokens * width);
    if (row < 0 || t < 0) {
      write_row(a, r, -1, -1);
      continue;
    }
    const int j = (int)(t / kBlockTokens);
    const int32_t* at = nullptr;  // where the block's id was before the call
    if (j < min(held_of[row], need_of[row]))
      at = a.pool.block_table + (size_t)row * width + j;
    else if (grant_at[row] >= 0 && j < need_of[row])
      at = source(Moves{row, held_of[row], 0, grant_at[row], true}, j - held_of[row]);
    const int id = at ? *at : -1;
    write_row(a, r, (int)t, (unsigned)id < (unsigned)a.pool.num_blocks ? id * kBlockTokens + (int)(t % kBlockTokens) : -1);
  }
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
  if (a.pool.num_seqs <= kOneSeqs && a.rows.num_rows <= kOneRows) {
    const int64_t entries = (int64_t)a.pool.num_seqs * a.pool.max_blocks_per_seq;
    const int64_t groups = std::max((entries + kEntriesEach - 1) / kEntriesEach, (a.rows.num_rows + kRowsEach - 1) / kRowsEach);
    hipLaunchKernelGGL(resize_kernel, dim3((unsigned)std::min(groups, kMostGroups)), dim3(kPlanThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_moves<true>(a, stream) : e;
}

hipError_t launch_slot_map(const BlocksArgs& a, hipStream_t stream) { return launch_moves<false>(a, stream); }

}  // namespace pda
