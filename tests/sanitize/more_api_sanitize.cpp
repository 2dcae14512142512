// Sanitizer driver for the host side of the head norms, the windowed attention and the block
// tables (test infrastructure): their host layers under AddressSanitizer and
// UndefinedBehaviorSanitizer, with launchers that report a failed launch, and the list of
// blocks that a window's rows see against a search token by token.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <vector>

#include "pda_blocks_internal.h"
#include "pda_norm_rotary_internal.h"
#include "pda_window_internal.h"

namespace {
bool wide_seen = false;
pda::WindowArgs seen;
}  // namespace

namespace pda {  // no GPU here: every launch reports failure
hipError_t launch_logprob(const LogprobArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_append(const StepArgs&, const uint16_t*, const uint16_t*, uint16_t*, uint16_t*, int, hipStream_t) {
  return hipErrorInvalidValue;
}
hipError_t launch_order(const StepArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_partition(const StepArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_merge(const StepArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_norm_rotary(const NormRotaryArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_norm_rotary_append(const NormRotaryArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_norm_rotary_backward(const NormRotaryArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_window(const WindowArgs& a, int, hipStream_t) {
  seen = a, wide_seen = false;
  return hipErrorInvalidValue;
}
hipError_t launch_window_wide(const WindowArgs& a, int, hipStream_t) {
  seen = a, wide_seen = true;
  return hipErrorInvalidValue;
}
hipError_t launch_window_merge(const WindowArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_blocks_resize(const BlocksArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_slot_map(const BlocksArgs&, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace pda

static uint64_t state = 405;
static uint32_t next_u32() {  // xorshift64*
  state ^= state >> 12;
  state ^= state << 25;
  state ^= state >> 27;
  return (uint32_t)((state * 2685821657736338717ull) >> 32);
}
static int32_t pick(const std::vector<int32_t>& v) { return v[next_u32() % v.size()]; }

static int fails = 0;
#define EXPECT(c)                                            \
  do {                                                       \
    if (!(c)) {                                              \
      fprintf(stderr, "line %d: %s failed\n", __LINE__, #c); \
      if (++fails > 20) return 1;                            \
    }                                                        \
  } while (0)

// The list of a group of new tokens: every block with a token that some row sees, once, in order, and none other.
static int check_span(int L, int n, int i0, int i1, int window, int sinks) {
  const pda::WindowSpan s = pda::window_span(L, n, i0, i1, window, sinks);
  std::vector<int> want;
  for (int j = 0; j * 16 < L; ++j) {
    bool any = false;
    for (int t = 16 * j; t < 16 * j + 16 && !any; ++t)
      for (int i = i0; i < i1 && !any; ++i) {
        const int p = L - n + i;
        any = t <= p && (t > (int64_t)p - window || t < sinks);
      }
    if (any) want.push_back(j);
  }
  EXPECT(s.count() == (int)want.size());
  for (int v = 0; v < s.count(); ++v) {
    EXPECT(s.block(v) == want[v]);
    EXPECT(s.token(v) == 16 * want[v]);
  }
  return 0;
}

int main() {
  const std::vector<int32_t> sizes = {-1, 0, 1, 2, 3, 7, 8, 16, 17, 64, 255, 256, 4096, 65536, 1 << 20, 1 << 30,
                                      0x7fffffff, (int32_t)0x80000000};
  for (int it = 0; it < 20000; ++it) {
    const int L = next_u32() % 400, n = 1 + next_u32() % 40;
    const int i0 = next_u32() % n, i1 = i0 + 1 + next_u32() % (n - i0);
    const int window = next_u32() % 8 ? 1 + next_u32() % 200 : (next_u32() % 2 ? 0x7fffffff : 1);
    const int sinks = next_u32() % 8 ? next_u32() % 100 : (next_u32() % 2 ? 0x7fffffff : 0);
    if (check_span(L, n, i0, i1, window, sinks)) return 1;
  }
  alignas(16) static char dummy[256];
  int32_t* ints = (int32_t*)dummy;
  int planned = 0;
  for (int it = 0; it < 30000; ++it) {
    pda_problem p;
    p.num_seqs = pick(sizes);
    p.num_kv_heads = next_u32() % 2 ? 1 + (int32_t)(next_u32() % 8) : pick(sizes);
    p.num_q_heads = next_u32() % 2 && p.num_kv_heads > 0 && p.num_kv_heads < 100
                        ? p.num_kv_heads * (1 + (int32_t)(next_u32() % 17))
                        : pick(sizes);
    p.head_dim = next_u32() % 4 ? (next_u32() % 2 ? 64 : 128) : pick(sizes);
    p.block_size = next_u32() % 8 ? 16 : pick(sizes);
    p.num_blocks = pick(sizes);
    p.max_blocks_per_seq = pick(sizes);
    p.max_context_len = next_u32() % 2 ? (int32_t)(next_u32() % 70000) : pick(sizes);
    p.partition_tokens = next_u32() % 2 ? 0 : (next_u32() % 3 ? 16 * (int32_t)(next_u32() % 300) : pick(sizes));
    p.num_query_tokens = next_u32() % 2 ? 1 : pick(sizes);
    pda_window w = {pick(sizes), pick(sizes)};
    if (next_u32() % 2) w = pda_window{1 + (int32_t)(next_u32() % 5000), (int32_t)(next_u32() % 200)};
    pda_plan_info info;
    const int rc = pda_plan_window(&p, &w, &info);
    if (rc == PDA_OK) {
      ++planned;
      EXPECT(info.partition_tokens > 0 && info.partition_tokens % 16 == 0 && info.num_partitions >= 1);
      EXPECT((info.workspace_bytes > 0) == (info.num_partitions > 1 && p.num_seqs > 0));
      const int drc = pda_decode_window(&p, &w, dummy, dummy, dummy, ints, ints, 0.125f, (float*)dummy, dummy,
                                        info.workspace_bytes, nullptr);
      EXPECT(drc == (p.num_seqs == 0 ? PDA_OK : PDA_ERR_HIP));
      if (p.num_seqs > 0) {
        // every row's list fits the partitions that the plan has room for, at any length
        const pda::StepArgs& s = seen.step;
        const int n = s.num_query_tokens;
        EXPECT((int64_t)seen.group_tokens * seen.num_groups >= n && (int64_t)seen.group_tokens * (seen.num_groups - 1) < n);
        EXPECT((int64_t)seen.group_tokens * s.group <= (wide_seen ? pda::kWindowWideRows : pda::kWindowNarrowRows));
        EXPECT(!wide_seen || s.partition_tokens % 32 == 0);
        EXPECT(s.num_regular_items < (1 << 24));  // (workgroups of 256 threads, less than 2^32)
        const int64_t pairs = (int64_t)s.num_seqs * s.num_kv_heads;
        EXPECT(!wide_seen || (pairs + 7) / 8 * 8 * seen.num_groups * s.num_partitions < (1 << 24));
        for (int k = 0; k < 8; ++k) {
          const int L = k == 0 ? p.max_context_len : (int)(next_u32() % ((uint32_t)p.max_context_len + 1));
          const int gr = k < 2 ? seen.num_groups - 1 : (int)(next_u32() % seen.num_groups);
          EXPECT(pda::window_partitions(seen, L, gr) <= s.num_partitions);
        }
      }
    } else {
      EXPECT(pda_decode_window(&p, &w, dummy, dummy, dummy, ints, ints, 0.125f, (float*)dummy, dummy, ~(size_t)0, nullptr) == rc);
    }
    // ---- norms ----
    pda_rotary r = {next_u32() % 2 ? 16 * (int32_t)(next_u32() % 10) : pick(sizes), (int32_t)(next_u32() % 2),
                    (int32_t)(next_u32() % 2), 1.f, (const double*)dummy};
    pda_head_norm h = {next_u32() % 4 ? 1e-6f : -1.f, 0.f, (int32_t)(next_u32() % 3), dummy, next_u32() % 2 ? dummy : nullptr};
    pda_rotary_axes x = {(int32_t)(next_u32() % 7) - 1, (const uint8_t*)dummy, pick(sizes)};
    const int32_t T = pick(sizes), hq = next_u32() % 2 ? 1 + (int32_t)(next_u32() % 64) : pick(sizes);
    const int32_t hkv = next_u32() % 2 ? (int32_t)(next_u32() % 16) : pick(sizes), d = next_u32() % 2 ? 8 * (int32_t)(next_u32() % 70) : pick(sizes);
    const int64_t stride = (int64_t)pick(sizes) * pick(sizes);
    const pda_head_norm* hp = next_u32() % 3 ? &h : nullptr;
    const pda_rotary* rp = next_u32() % 3 ? &r : nullptr;
    const pda_rotary_axes* xp = next_u32() % 3 ? nullptr : &x;
    EXPECT(pda_norm_rotary(hp, rp, xp, T, hq, hkv, d, (int32_t)(next_u32() % 3), ints, dummy, stride, dummy, stride, dummy, stride,
                           dummy, stride, nullptr) != PDA_OK || T == 0);
    size_t ws = 0;
    const int wrc = pda_norm_rotary_workspace_bytes(T, hq, hkv, d, &ws);
    EXPECT(wrc != PDA_OK || ws <= ((size_t)1 << 22));
    const int brc = pda_norm_rotary_backward(hp, rp, xp, T, hq, hkv, d, (int32_t)(next_u32() % 3), ints, dummy, stride, dummy, stride,
                                             dummy, stride, dummy, stride, dummy, stride, dummy, stride, (float*)dummy, nullptr,
                                             dummy, ws, nullptr);
    EXPECT(brc != PDA_OK);  // (the weights' gradient is written without tokens too)
    EXPECT(pda_norm_rotary_append(hp, rp, xp, T, hq, hkv, d, pick(sizes), ints, ints, dummy, stride, dummy, stride, dummy,
                                  stride, dummy, stride, dummy, dummy, nullptr) != PDA_OK || T == 0);
    // ---- block tables ----
    pda_block_pool pool = {pick(sizes), pick(sizes), pick(sizes), ints, ints, ints, ints};
    pda_token_rows rows = {pick(sizes), next_u32() % 2 ? ints : nullptr, next_u32() % 2 ? ints : nullptr, next_u32() % 2 ? ints : nullptr};
    size_t bytes = 0;
    const int prc = pda_blocks_workspace_bytes(&pool, &bytes);
    EXPECT(prc != PDA_OK || bytes <= ((size_t)1 << 24));
    const int rrc = pda_blocks_resize(&pool, ints, next_u32() % 2 ? &rows : nullptr, dummy, ~(size_t)0, nullptr);
    EXPECT(rrc != PDA_OK || pool.num_seqs == 0);
    const int src = pda_slot_map(pool.num_seqs, pool.num_blocks, pool.max_blocks_per_seq, ints, ints, &rows, nullptr);
    EXPECT(src != PDA_OK || rows.num_rows == 0);
  }
  EXPECT(planned > 1000);
  if (fails) {
    fprintf(stderr, "%d check(s) failed\n", fails);
    return 1;
  }
  printf("norms, windows and block tables: all checks passed\n");
  return 0;
}
