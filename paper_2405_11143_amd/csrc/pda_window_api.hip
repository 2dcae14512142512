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

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

int query_tokens(const pda_problem* p) { return p->num_query_tokens > 0 ? p->num_query_tokens : 1; }

struct Plan {
  pda_plan_info info;
  int unit, group_tokens, num_groups, query_chunk;
  int64_t items;
  size_t slots;  // partial states, 0 when nothing is split
};

// The most tokens that a work item's list holds.
int64_t longest_list(const pda_problem* p, const pda_window* w, const Plan& plan) {
  const int64_t u = plan.unit;
  auto units = [&](int64_t tokens) { return (tokens + u - 1) / u; };
  const int64_t whole = units(p->max_context_len);
  // (a window starts anywhere in its first unit)
  const int64_t apart = units(w->num_sinks) + units((int64_t)w->window + plan.group_tokens - 1) + 1;
  return std::min(whole, apart) * u;
}

int make_plan(const pda_problem* p, const pda_window* w, Plan* plan) {
  if (!w) return PDA_ERR_NULL;
  int rc = pda_plan(p, &plan->info);
  if (rc != PDA_OK) return rc;
  if (w->window < 1 || w->num_sinks < 0) return PDA_ERR_SHAPE;
  const int n = query_tokens(p), G = p->num_q_heads / p->num_kv_heads;
  plan->query_chunk = std::min(n, pda::kMaxGroup / G);
  const bool narrow = (int64_t)n * G <= pda::kWindowNarrowRows;
  plan->unit = narrow ? pda::kWindowUnit : pda::kWindowWideUnit;
  plan->group_tokens = narrow ? n : std::min(n, plan->query_chunk * (pda::kWindowWideRows / pda::kMaxGroup));
  plan->num_groups = (n + plan->group_tokens - 1) / plan->group_tokens;
  const int64_t len = longest_list(p, w, *plan);
  // the partitions of pda_decode's plan for contexts as long as what is read here
  pda_problem like = *p;
  like.max_context_len = (int32_t)std::min<int64_t>(len, p->max_context_len);
  rc = pda_plan(&like, &plan->info);
  if (rc != PDA_OK) return rc;
  int64_t tokens = (plan->info.partition_tokens + plan->unit - 1) / plan->unit * plan->unit;
  const int64_t parts = std::max<int64_t>(1, (len + tokens - 1) / tokens);
  // (each factor below 2^31, and rows of the whole batch too: two factors at a time)
  const int64_t pairs = (int64_t)p->num_seqs * p->num_kv_heads;
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
  a.window = window->window;
  a.sinks = window->num_sinks;
  a.group_tokens = plan.group_tokens;
  a.num_groups = plan.num_groups;
  a.unit = plan.unit;
  const hipError_t e = plan.unit == pda::kWindowUnit ? pda::launch_window(a, prob->head_dim, stream)
                                                     : pda::launch_window_wide(a, prob->head_dim, stream);
  if (e != hipSuccess) return PDA_ERR_HIP;
  if (plan.slots > 0 && pda::launch_window_merge(a, prob->head_dim, stream) != hipSuccess) return PDA_ERR_HIP;
  return PDA_OK;
}

}  // extern "C"
