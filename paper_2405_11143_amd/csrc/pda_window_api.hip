// Host side of attention with a sliding window and sinks (declared in
// include/pda_window.h): validation, the plan, the launches.  Nothing here
// allocates memory or keeps state between calls.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "pda_window_internal.h"

namespace {

constexpr int64_t kMostItems = (1 << 24) - 1;        // workgroups of 256: a launch has less than 2^32 threads
constexpr int64_t kMostMergeRows = 4 * kMostItems;   // the merge: workgroups of 256 for 4 rows
// Narrow items are split into as many as make one for every compute unit, of at least
// kNarrowLeast tokens, where that shortens an item by kNarrowGain.  Wide ones into up to two for
// every unit, of at least kWideLeast tokens, or one for every unit of at least kWideFew;
// two from one would share a unit that one has to itself.  Decode steps of 32 / 8 heads of
// 128, us, this rule / whole / the best of partitions of 128 to 2064: 1 sequence with a window of 512 7.9
// / 7.9 / 9.3, of 1024 10.3 / 12.9 / 10.4, of 4096 13.1 / - / 12.7; 4: 8.9 / 8.9 / 10.1, 11.2 /
// 13.5 / 11.1, 17.9 / - / 18.0; 8: 9.2 / 9.2 / 10.7, 12.8 / 14.1 / 13.0, 26.9 / - / 27.0; 16 of 1024
// 15.7 / 15.7 / 17.7, of 4096 45.8 / - / 46.0; 24 of 1024 18.5 / 18.5 / 22.2.  64 new tokens over a window
// of 1024, this rule / whole / in 288s / in 128s: 1 sequence 18.6 / 46.2 / 22.0 / 18.7; 2 21.7 / 46.6 / 23.9 / 25.3;
// 4 28.9 / 46.7 / 27.9 / 40.4; 8 43.4 / 48.1 / 42.9 / 63.6; 512 new ones of 2 (256 items) 51 whole, 69 in 512s.
constexpr int64_t kNarrowAtOnce = 256, kNarrowLeast = 176, kNarrowGain = 600;
constexpr int64_t kWideAtOnce = 512, kWideLeast = 256, kWideFew = 128, kWideGain = 400;

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

int query_tokens(const pda_problem* p) { return p->num_query_tokens > 0 ? p->num_query_tokens : 1; }

struct Plan {
  pda_plan_info info;
  bool narrow;
  int group_tokens, num_groups, query_chunk;
  int64_t items;
  size_t slots;  // partial states, 0 when nothing is split
};

// The most tokens that a work item's list holds.
int64_t longest_list(const pda_problem* p, const pda_window* w, const Plan& plan) {
  constexpr int64_t u = pda::kWindowUnit;
  auto units = [&](int64_t tokens) { return (tokens + u - 1) / u; };
  const int64_t whole = units(p->max_context_len);
  // (a window starts anywhere in its first block)
  const int64_t apart = units(w->num_sinks) + units((int64_t)w->window + plan.group_tokens - 1) + 1;
  return std::min(whole, apart) * u;
}

// Tokens per partition when the caller leaves them to the library.  Lists are as long as
// the window wherever contexts are longer, so there is nothing to balance, and splitting pays only
// where it fills compute units that would be idle, by more than the merge costs.  Windows that cover
// the contexts give lists as unequal as those, which run in launch order all the same: 256 contexts of 512 to 4096 (32 / 8
// heads of 128) under a window of 2048 289 us, of 4096 or 8192 388, where a gather takes 270 and 362
// and pda_decode, whose items start with the longest, 372.
int64_t partition_rule(const pda_problem* p, const Plan& plan, int64_t len) {
  const int64_t units = (int64_t)p->num_seqs * p->num_kv_heads * plan.num_groups;
  if (units == 0) return len;
  int64_t pieces, gain;
  if (plan.narrow) {
    pieces = std::min(kNarrowAtOnce / units, len / kNarrowLeast);
    gain = kNarrowGain;
  } else {
    const int64_t room = kWideAtOnce / units;
    pieces = room < 3 ? 1 : std::min(room, std::max(len / kWideLeast, std::min(room / 2, len / kWideFew)));
    gain = kWideGain;
  }
  return pieces < 2 || len - len / pieces < gain ? len : (len + pieces - 1) / pieces;
}

int make_plan(const pda_problem* p, const pda_window* w, Plan* plan) {
  if (!w) return PDA_ERR_NULL;
  int rc = pda_plan(p, &plan->info);
  if (rc != PDA_OK) return rc;
  if (w->window < 1 || w->num_sinks < 0) return PDA_ERR_SHAPE;
  const int n = query_tokens(p), G = p->num_q_heads / p->num_kv_heads;
  plan->query_chunk = std::min(n, pda::kMaxGroup / G);
  plan->narrow = (int64_t)n * G <= pda::kWindowNarrowRows;
  const int64_t quantum = plan->narrow ? pda::kWindowUnit : 2 * pda::kWindowUnit;  // (the wide kernel takes two blocks at a time)
  plan->group_tokens = plan->narrow ? n : std::min(n, plan->query_chunk * (pda::kWindowWideRows / pda::kMaxGroup));
  plan->num_groups = (n + plan->group_tokens - 1) / plan->group_tokens;
  const int64_t len = longest_list(p, w, *plan);
  int64_t tokens = p->partition_tokens > 0 ? p->partition_tokens : partition_rule(p, *plan, len);
  tokens = std::max(quantum, (std::min(tokens, len) + quantum - 1) / quantum * quantum);
  const int64_t parts = std::max<int64_t>(1, (len + tokens - 1) / tokens);
  // (each factor below 2^31, and rows of the whole batch too: two factors at a time)
  int64_t pairs = (int64_t)p->num_seqs * p->num_kv_heads;
  if (!plan->narrow) pairs = (pairs + pda::kWindowXcds - 1) / pda::kWindowXcds * pda::kWindowXcds;  // as launched
  if (pairs > kMostItems || pairs * plan->num_groups > kMostItems || parts * pairs * plan->num_groups > kMostItems)
    return PDA_ERR_SHAPE;
  if (parts > 1 && (int64_t)p->num_seqs * n * p->num_q_heads > kMostMergeRows) return PDA_ERR_SHAPE;
  plan->items = parts * pairs * plan->num_groups;
  plan->slots = parts > 1 ? (size_t)p->num_seqs * n * p->num_q_heads * (size_t)parts : 0;
  plan->info.partition_tokens = (int32_t)tokens;
  plan->info.num_partitions = (int32_t)parts;
  plan->info.workspace_bytes = plan->slots * (p->head_dim + 2) * sizeof(float);
  return PDA_OK;
}

}  // namespace

extern "C" {

int pda_plan_window(const pda_problem* prob, const pda_window* window, pda_plan_info* info) {
  if (!prob || !info) return PDA_ERR_NULL;
  Plan plan;
  const int rc = make_plan(prob, window, &plan);
  if (rc != PDA_OK) return rc;
  *info = plan.info;
  return PDA_OK;
}

int pda_decode_window(const pda_problem* prob, const pda_window* window, const void* q, const void* k_cache,
                      const void* v_cache, const int32_t* block_table, const int32_t* context_lens, float scale,
                      float* out, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!prob) return PDA_ERR_NULL;
  Plan plan;
  const int rc = make_plan(prob, window, &plan);
  if (rc != PDA_OK) return rc;
  if (prob->num_seqs > 0 && (!q || !k_cache || !v_cache || !block_table || !context_lens || !out)) return PDA_ERR_NULL;
  if (!isfinite(scale)) return PDA_ERR_VALUE;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16)) return PDA_ERR_ALIGNMENT;
  if (prob->num_seqs == 0) return PDA_OK;
  if (plan.info.workspace_bytes > 0) {
    if (!workspace || workspace_bytes < plan.info.workspace_bytes) return PDA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return PDA_ERR_ALIGNMENT;
  }
  pda::WindowArgs a{};
  pda::StepArgs& s = a.step;
  if (plan.slots > 0) {
    float* ws = static_cast<float*>(workspace);
    s.part_o = ws;
    s.part_m = ws + plan.slots * prob->head_dim;
    s.part_l = ws + plan.slots * (prob->head_dim + 1);
  }
  s.q = static_cast<const uint16_t*>(q);
  s.k = static_cast<const uint16_t*>(k_cache);
  s.v = static_cast<const uint16_t*>(v_cache);
  s.table = block_table;
  s.lens = context_lens;
  s.out = out;
  s.scale_log2 = scale * 1.4426950408889634f;
  s.num_seqs = prob->num_seqs;
  s.num_q_heads = prob->num_q_heads;
  s.num_kv_heads = prob->num_kv_heads;
  s.group = prob->num_q_heads / prob->num_kv_heads;
  s.group_inverse = (65536 + s.group - 1) / s.group;
  s.num_blocks = prob->num_blocks;
  s.max_blocks_per_seq = prob->max_blocks_per_seq;
  s.max_context_len = prob->max_context_len;
  s.num_query_tokens = query_tokens(prob);
  s.query_chunk = plan.query_chunk;
  s.partition_tokens = plan.info.partition_tokens;
  s.num_partitions = plan.info.num_partitions;
  s.slots_per_row = plan.info.num_partitions;
  s.num_regular_items = (int32_t)plan.items;
  // (past every context they say the same, and the kernels' sums of positions stay inside int32)
  a.window = std::min(window->window, prob->max_context_len + 1);
  a.sinks = std::min(window->num_sinks, prob->max_context_len);
  a.group_tokens = plan.group_tokens;
  a.num_groups = plan.num_groups;
  const hipError_t e = plan.narrow ? pda::launch_window(a, prob->head_dim, stream)
                                                     : pda::launch_window_wide(a, prob->head_dim, stream);
  if (e != hipSuccess) return PDA_ERR_HIP;
  if (plan.slots > 0 && pda::launch_window_merge(a, prob->head_dim, stream) != hipSuccess) return PDA_ERR_HIP;
  return PDA_OK;
}

}  // extern "C"
