// Sanitizer driver for the host side of the 8-bit cache and the rotary positions
// (test infrastructure): pda_api.hip and pda_fp8_api.hip under AddressSanitizer and
// UndefinedBehaviorSanitizer, with launchers that report a failed launch.  Seeded
// random and extreme descriptors go through the checks, the plan and every entry
// point; any out-of-bounds access or undefined operation aborts the run.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "pda_fp8_internal.h"

namespace pda {  // no GPU here: every launch reports failure
hipError_t launch_logprob(const LogprobArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_append(const StepArgs&, const uint16_t*, const uint16_t*, uint16_t*, uint16_t*, int, hipStream_t) {
  return hipErrorInvalidValue;
}
hipError_t launch_order(const StepArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_partition(const StepArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_merge(const StepArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_rotary(const RotaryApplyArgs&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_append_fp8(const AppendFp8Args&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_decode_fp8(const DecodeFp8Args&, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_read_fp8(const ReadFp8Args&, int, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace pda

static uint64_t state = 950;
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
      ++fails;                                               \
    }                                                        \
  } while (0)

int main() {
  const std::vector<int32_t> sizes = {-1, 0, 1, 2, 3, 7, 8, 16, 17, 64, 255, 256, 4096, 65536, 1 << 20, 1 << 30,
                                      0x7fffffff, (int32_t)0x80000000};
  alignas(16) static char dummy[256];
  const int32_t* ints = (const int32_t*)dummy;
  uint8_t* bytes = (uint8_t*)dummy;
  int planned = 0;
  for (int it = 0; it < 20000; ++it) {
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
    pda_plan_info info;
    const int rc = pda_plan_fp8(&p, &info);
    if (rc == PDA_OK) {
      ++planned;
      EXPECT(info.partition_tokens > 0 && info.partition_tokens % 16 == 0 && info.num_partitions >= 1);
      EXPECT((int64_t)info.num_partitions * info.partition_tokens >= p.max_context_len);
      EXPECT(p.num_seqs == 0 || info.workspace_bytes > 0);
      // a valid step reaches its first launch, which fails here
      const int drc = pda_decode_fp8(&p, dummy, dummy, dummy, bytes, ints, ints, 0.125f, (float*)dummy, dummy,
                                     info.workspace_bytes, nullptr);
      EXPECT(drc == (p.num_seqs == 0 ? PDA_OK : PDA_ERR_HIP));
    } else {
      EXPECT(pda_decode_fp8(&p, dummy, dummy, dummy, bytes, ints, ints, 0.125f, (float*)dummy, dummy, ~(size_t)0,
                            nullptr) == rc);
    }
    pda_rotary r = {next_u32() % 2 ? 16 * (int32_t)(next_u32() % 10) : pick(sizes), (int32_t)(next_u32() % 2),
                    (int32_t)(next_u32() % 2), 1.f, (const double*)dummy};
    const int arc = pda_append_kv_fp8(&p, next_u32() % 2 ? &r : nullptr, nullptr, nullptr, dummy, dummy, ints, ints, dummy,
                                      dummy, bytes, nullptr);
    EXPECT(arc != PDA_OK || p.num_seqs == 0);
    const int32_t rows = pick(sizes);
    const int rrc = pda_read_kv_fp8(&p, dummy, dummy, bytes, ints, ints, nullptr, ints, rows, dummy, dummy, nullptr);
    EXPECT(rrc != PDA_OK || p.num_seqs == 0 || rows == 0);
    const int32_t T = pick(sizes), hq = pick(sizes), hkv = pick(sizes), d = pick(sizes);
    const int64_t stride = (int64_t)pick(sizes) * pick(sizes);
    const int trc = pda_rotary_apply(&r, T, hq, hkv, d, (int32_t)(next_u32() % 3), ints, dummy, stride, dummy, stride, dummy,
                                     stride, dummy, stride, nullptr);
    EXPECT(trc != PDA_OK || T == 0);
  }
  EXPECT(planned > 1000);
  // the frequencies, over random and extreme scalings
  std::vector<double> f(1 << 16);
  for (int it = 0; it < 5000; ++it) {
    const double xs[] = {0.0, 1.0, -1.0, 1e-300, 1e300, 10000.0, 5e5, 4.0, 32.0, __builtin_nan(""), __builtin_inf(), 8192.0};
    auto x = [&] { return xs[next_u32() % 12]; };
    pda_rotary_scaling s = {(int32_t)(next_u32() % 7) - 1, x(), x(), x(), x()};
    const int32_t dim = next_u32() % 2 ? 2 * (int32_t)(next_u32() % 300) : pick(sizes);
    if (dim > (1 << 16)) continue;
    float m = 0.f;
    if (pda_rotary_inv_freq(dim, x(), next_u32() % 2 ? &s : nullptr, f.data(), &m) == PDA_OK)
      EXPECT(f[0] > 0.0 && m >= 1.f);
  }
  if (fails) {
    fprintf(stderr, "%d check(s) failed\n", fails);
    return 1;
  }
  printf("8-bit cache host layer: all checks passed\n");
  return 0;
}
