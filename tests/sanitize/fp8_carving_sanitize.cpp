// Sanitizer driver for what pda_decode_fp8 hands to its kernels (test
// infrastructure): pda_api.hip and pda_fp8_api.hip under AddressSanitizer and
// UndefinedBehaviorSanitizer, with launchers that check the pointers they get against
// the workspace of the plan (no memory is behind it, and none is touched) and the
// sizes against each other and against a launch's limits.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "pda_fp8_internal.h"

static int fails = 0;
#define EXPECT(c)                                            \
  do {                                                       \
    if (!(c)) {                                              \
      fprintf(stderr, "line %d: %s failed\n", __LINE__, #c); \
      ++fails;                                               \
    }                                                        \
  } while (0)

static const uintptr_t kWorkspace = (uintptr_t)1 << 44;
static pda_problem prob;
static pda_plan_info info;
static int ordered, attended, merged, picked;

static int64_t new_tokens() { return prob.num_query_tokens > 0 ? prob.num_query_tokens : 1; }
static int64_t rows() { return prob.num_seqs * new_tokens() * prob.num_q_heads; }
static bool inside(const void* p, uint64_t bytes) {
  const uintptr_t at = (uintptr_t)p;
  return at >= kWorkspace && at % 4 == 0 && at - kWorkspace + bytes <= info.workspace_bytes;
}

static void check_step(const pda::StepArgs& s) {
  const uint64_t slots = info.num_partitions > 1 ? (uint64_t)rows() * info.num_partitions : 0;
  EXPECT(s.num_partitions == info.num_partitions && s.partition_tokens == info.partition_tokens);
  EXPECT(s.slots_per_row == s.num_partitions && s.num_groups == 0 && s.query_chunk == 1);
  EXPECT(s.num_query_chunks == s.num_query_tokens && s.num_query_tokens == new_tokens());
  EXPECT((int64_t)s.num_partitions * s.num_seqs * s.num_kv_heads * s.num_chunk_groups == s.num_regular_items);
  EXPECT(s.num_regular_items > 0 && s.num_regular_items < (1 << 24));  // workgroups of 256: fewer than 2^32 threads
  EXPECT(s.group * s.num_kv_heads == s.num_q_heads);
  if (slots > 0) {
    const uint64_t o = slots * prob.head_dim * 4, m = slots * 4;
    EXPECT(inside(s.part_o, o) && inside(s.part_m, m) && inside(s.part_l, m));
    EXPECT((uintptr_t)s.part_o % 16 == 0);  // stored 16 bytes at a time
    EXPECT((uintptr_t)s.part_m >= (uintptr_t)s.part_o + o && (uintptr_t)s.part_l >= (uintptr_t)s.part_m + m);
  } else {
    EXPECT(!s.part_o && !s.part_m && !s.part_l);
  }
  if (s.order) {
    EXPECT(inside(s.order, (uint64_t)s.num_regular_items * 4));
    EXPECT((uintptr_t)s.order >= (slots > 0 ? (uintptr_t)s.part_l + slots * 4 : kWorkspace));
  }
}

namespace pda {
hipError_t launch_logprob(const LogprobArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_append(const StepArgs&, const uint16_t*, const uint16_t*, uint16_t*, uint16_t*, int, hipStream_t) {
  return hipErrorInvalidValue;
}
hipError_t launch_partition(const StepArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_rotary(const RotaryApplyArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_append_fp8(const AppendFp8Args&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_read_fp8(const ReadFp8Args&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_order(const StepArgs& s, hipStream_t) {
  check_step(s);
  EXPECT(s.order && attended == 0);
  ++ordered;
  return hipSuccess;
}
hipError_t launch_decode_fp8(const DecodeFp8Args& a, int head_dim, hipStream_t) {
  const StepArgs& s = a.step;
  check_step(s);
  EXPECT(head_dim == prob.head_dim);
  const int64_t per_head = new_tokens() * s.group;
  EXPECT((int64_t)s.num_chunk_groups * fp8_item_rows(per_head) >= per_head);
  EXPECT(!(a.picks && s.order) && (s.order != nullptr) == (ordered == 1));
  if (a.picks) EXPECT(per_head <= 2 * kFp8TileRows && (int64_t)s.num_seqs * s.num_partitions <= kPickPairs);
  if (!a.picks && !s.order && per_head <= 2 * kFp8TileRows)  // a grid of three dimensions
    EXPECT(s.num_seqs <= 65535 && s.num_partitions <= 65535);
  picked += a.picks;
  ++attended;
  return hipSuccess;
}
hipError_t launch_merge(const StepArgs& s, int, hipStream_t) {
  check_step(s);
  EXPECT(attended == 1 && s.part_o);
  EXPECT((rows() + 3) / 4 * 256 < (int64_t)1 << 32);  // its threads: a wavefront per row, 4 to a workgroup
  ++merged;
  return hipSuccess;
}
}  // namespace pda

static uint64_t state = 1951;
static uint32_t next_u32() {  // xorshift64*
  state ^= state >> 12;
  state ^= state << 25;
  state ^= state >> 27;
  return (uint32_t)((state * 2685821657736338717ull) >> 32);
}
static int32_t pick(const std::vector<int32_t>& v) { return v[next_u32() % v.size()]; }

int main() {
  alignas(16) static char dummy[256];
  const int32_t* ints = (const int32_t*)dummy;
  int planned = 0, with_order = 0, with_merge = 0, with_picks = 0;
  for (int it = 0; it < 200000; ++it) {
    prob.num_seqs = pick({1, 2, 3, 8, 16, 33, 64, 255, 256, 257, 512, 4096, 65536, 1 << 20, 1 << 24, 0x7fffffff});
    prob.num_kv_heads = pick({1, 2, 3, 5, 8, 8, 16, 40, 1 << 16});
    prob.num_q_heads = prob.num_kv_heads * pick({1, 2, 3, 4, 7, 8, 16});
    prob.head_dim = next_u32() % 2 ? 64 : 128;
    prob.block_size = 16;
    prob.num_blocks = pick({1, 100, 0x7fffffff});
    prob.max_context_len = pick({0, 1, 16, 257, 512, 2048, 2049, 4096, 16384, 100000, 1 << 20, 1 << 28});
    prob.max_blocks_per_seq = prob.max_context_len / 16 + 1 + pick({0, 0, 3});
    prob.partition_tokens = pick({0, 0, 0, 16, 48, 256, 4096, 1 << 28});
    prob.num_query_tokens = pick({0, 1, 1, 2, 4, 5, 8, 17, 64, 512, 8192, 1 << 20, 1 << 28});
    if (pda_plan_fp8(&prob, &info) != PDA_OK) continue;
    ++planned;
    ordered = attended = merged = picked = 0;
    const int rc = pda_decode_fp8(&prob, dummy, dummy, dummy, (const uint8_t*)dummy, ints, ints, 0.125f, (float*)dummy,
                                  (void*)kWorkspace, info.workspace_bytes, nullptr);
    EXPECT(rc == PDA_OK && attended == 1);
    EXPECT(merged == (info.num_partitions > 1 ? 1 : 0));
    EXPECT(pda_decode_fp8(&prob, dummy, dummy, dummy, (const uint8_t*)dummy, ints, ints, 0.125f, (float*)dummy,
                          (void*)kWorkspace, info.workspace_bytes - 1, nullptr) == PDA_ERR_WORKSPACE);
    with_order += ordered, with_merge += merged, with_picks += picked;
    if (fails > 20) break;
  }
  EXPECT(planned > 10000 && with_order > 1000 && with_merge > 1000 && with_picks > 100);
  if (fails) {
    fprintf(stderr, "%d check(s) failed\n", fails);
    return 1;
  }
  printf("8-bit cache launches: %d plans, %d ordered, %d picked, %d merged: all checks passed\n", planned, with_order, with_picks,
         with_merge);
  return 0;
}
