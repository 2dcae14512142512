// Host side of the 8-bit KV cache and the rotary positions (declared in
// include/pda_fp8.h): validation, the plan, the launches.  Nothing here
// allocates memory or keeps state between calls.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "pda_fp8_internal.h"

namespace {

// Steps of more items than this run them sorted by size.  It is what the one-tile decode
// kernel at head_dim 128 runs at once, 3 workgroups per compute unit; at 128 the two-tile
// and the four-wavefront kernels run 512 and the two-wavefront one 1024 (at 64: one tile
// 1024, two 768, four wavefronts 768, two 1536), where this line was not measured.
constexpr int64_t kAtOnce = 768;
// Sorted steps of at most this many items, and of pda::kPickPairs pairs, find their
// items without the order kernel (one tile): a step of 256 sequences of 512-4096 tokens (2048 items)
// takes 194.7 us instead of 197.7, 8 of up to 16384 (1152) 21.4 instead of 23.3.  Ranking costs
// every workgroup about a microsecond: 16 of up to 16384 in 512s (3328 items) took
// 42.5 instead of 36.7.
constexpr int64_t kPickItems = 3 * kAtOnce;
// Contexts of one-tile steps up to this length stay whole where they all run at once and
// there are kWholePairs (sequence, KV head) pairs for every kWholeOf tokens: a workgroup alone on a
// compute unit reads 2048 tokens in 13 us, and splitting costs a merge of 5, which
// pays where most compute units would be idle.  Whole / the best of 256, 512 and 1024 in
// us, 8 KV heads, contexts uniform up to the maximum: 24 sequences of 2048 16.6 / 17.8, 16
// 16.8 / 13.9, 16 of 1500 13.6 / 13.4, 24 13.8 / 15.8, 16 of 1024 10.5 / 11.1, 8 10.5 /
// 9.5.  The rule has no line above, where whole contexts are a little slower: 48 of 2048
// 26.4 / 25.7, 64 31.8 / 30.0.  Other numbers of KV heads and head_dim 64 were not measured.
constexpr int kWholeTokens = 2048;
constexpr int64_t kWholePairs = 1, kWholeOf = 12;
constexpr int64_t kMostItems = (1 << 24) - 1;  // workgroups of 256: a launch has less than 2^32 threads
constexpr int64_t kMostMergeRows = 4 * kMostItems;  // the merge: workgroups of 256 for 4 rows
constexpr int kMaxHeadDim = 512;  // of pda_rotary_apply

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

int query_tokens(const pda_problem* p) { return p->num_query_tokens > 0 ? p->num_query_tokens : 1; }

using pda::check_rotary;
using pda::rotary_args;

// The descriptor's own errors (those of pda_plan).
int check_problem(const pda_problem* p) {
  pda_plan_info info;
  return pda_plan(p, &info);
}

struct Plan {
  pda_plan_info info;
  int tiles;      // row tiles of a sequence and KV head
  int64_t items;  // partitions x sequences x KV heads x tiles
  size_t slots;   // partial states, 0 when nothing is split
  bool narrow;    // few query rows: the decode kernel
};

int make_plan(const pda_problem* p, Plan* plan) {
  int rc = pda_plan(p, &plan->info);
  if (rc != PDA_OK) return rc;
  const int n = query_tokens(p);
  if (p->partition_tokens == 0 && (int64_t)n * (p->num_q_heads / p->num_kv_heads) <= pda::kFp8TileRows &&
      p->max_context_len <= kWholeTokens && (int64_t)p->num_seqs * p->num_kv_heads <= kAtOnce &&
      (int64_t)p->num_seqs * p->num_kv_heads * kWholeOf >= kWholePairs * p->max_context_len) {
    pda_problem whole = *p;
    whole.partition_tokens = kWholeTokens;
    rc = pda_plan(&whole, &plan->info);
    if (rc != PDA_OK) return rc;
  }
  const int64_t rows = (int64_t)n * (p->num_q_heads / p->num_kv_heads);
  const int item_rows = pda::fp8_item_rows(rows);
  plan->tiles = (int)((rows + item_rows - 1) / item_rows);
  plan->narrow = item_rows <= 2 * pda::kFp8TileRows;
  const int64_t parts = plan->info.num_partitions;
  // (each factor below 2^31, and rows of the whole batch too: two factors at a time)
  const int64_t pairs = (int64_t)p->num_seqs * p->num_kv_heads * plan->tiles;
  if (pairs > kMostItems || parts * pairs > kMostItems) return PDA_ERR_SHAPE;
  if (parts > 1 && (int64_t)p->num_seqs * n * p->num_q_heads > kMostMergeRows) return PDA_ERR_SHAPE;
  plan->items = parts * pairs;
  plan->slots = parts > 1 ? (size_t)p->num_seqs * n * p->num_q_heads * (size_t)parts : 0;
  plan->info.workspace_bytes = plan->slots * (p->head_dim + 2) * sizeof(float) + (size_t)plan->items * sizeof(int32_t);
  return PDA_OK;
}

}  // namespace

extern "C" {

int pda_rotary_inv_freq(int32_t rotary_dim, double base, const pda_rotary_scaling* scaling, double* inv_freq,
                        float* magnitude) {
  if (!inv_freq) return PDA_ERR_NULL;
  if (rotary_dim < 2 || rotary_dim % 2 != 0) return PDA_ERR_SHAPE;
  const int kind = scaling ? scaling->kind : PDA_ROTARY_PLAIN;
  if (kind < PDA_ROTARY_PLAIN || kind > PDA_ROTARY_RAMP) return PDA_ERR_UNSUPPORTED;
  if (!(base > 1.0) || !isfinite(base)) return PDA_ERR_VALUE;
  if (kind != PDA_ROTARY_PLAIN && !(scaling->factor >= 1.0 && isfinite(scaling->factor))) return PDA_ERR_VALUE;
  const bool ranged = kind == PDA_ROTARY_BANDS || kind == PDA_ROTARY_RAMP;
  if (ranged && !(scaling->original_len > 0.0 && isfinite(scaling->original_len) && scaling->low > 0.0 &&
                  scaling->high > scaling->low && isfinite(scaling->high)))
    return PDA_ERR_VALUE;
  if (kind == PDA_ROTARY_BASE && rotary_dim <= 2) return PDA_ERR_SHAPE;
  const double two_pi = 6.283185307179586477, R = rotary_dim;
  if (kind == PDA_ROTARY_BASE) base *= pow(scaling->factor, R / (R - 2));
  double i_low = 0, i_high = 0;
  if (kind == PDA_ROTARY_RAMP) {
    // the (real) index of the pair that turns x times over original_len tokens
    auto index_of = [&](double x) { return R * log(scaling->original_len / (x * two_pi)) / (2 * log(base)); };
    i_low = std::min(std::max(floor(index_of(scaling->high)), 0.0), R - 1);
    i_high = std::min(std::max(ceil(index_of(scaling->low)), 0.0), R - 1);
    if (i_high <= i_low) i_high = i_low + 0.001;
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / R);
    if (kind == PDA_ROTARY_LINEAR) f /= scaling->factor;
    if (kind == PDA_ROTARY_BANDS) {
      const double turns = scaling->original_len * f / two_pi;
      const double keep = std::min(std::max((turns - scaling->low) / (scaling->high - scaling->low), 0.0), 1.0);
      f = keep * f + (1 - keep) * f / scaling->factor;
    }
    if (kind == PDA_ROTARY_RAMP) {
      const double keep = 1 - std::min(std::max((i - i_low) / (i_high - i_low), 0.0), 1.0);
      f = keep * f + (1 - keep) * f / scaling->factor;
    }
    inv_freq[i] = f;
  }
  if (magnitude) *magnitude = kind == PDA_ROTARY_RAMP ? (float)(1 + 0.1 * log(scaling->factor)) : 1.f;
  return PDA_OK;
}

int pda_rotary_apply(const pda_rotary* rotary, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                     int32_t head_dim, int32_t dtype, const int32_t* positions, const void* q, int64_t q_stride,
                     void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out,
                     int64_t k_out_stride, hipStream_t stream) {
  if (!rotary) return PDA_ERR_NULL;
  if (num_tokens < 0 || num_q_heads < 1 || num_kv_heads < 0 || head_dim < 1) return PDA_ERR_SHAPE;
  if (dtype != PDA_DTYPE_BF16 && dtype != PDA_DTYPE_F32) return PDA_ERR_UNSUPPORTED;
  if (head_dim % 8 != 0 || head_dim > kMaxHeadDim) return PDA_ERR_UNSUPPORTED;
  if (((int64_t)num_q_heads + num_kv_heads) * head_dim > (1 << 24)) return PDA_ERR_SHAPE;  // a token's rows
  int rc = check_rotary(rotary, head_dim);
  if (rc != PDA_OK) return rc;
  const int64_t qw = (int64_t)num_q_heads * head_dim, kw = (int64_t)num_kv_heads * head_dim;
  if (q_stride < qw || q_out_stride < qw) return PDA_ERR_SHAPE;
  if (num_kv_heads > 0 && (k_stride < kw || k_out_stride < kw)) return PDA_ERR_SHAPE;
  if (num_tokens == 0) return PDA_OK;
  if (!positions || !q || !q_out || (num_kv_heads > 0 && (!k || !k_out))) return PDA_ERR_NULL;
  const int per16 = dtype == PDA_DTYPE_BF16 ? 8 : 4;
  if (!aligned(q, 16) || !aligned(q_out, 16) || q_stride % per16 || q_out_stride % per16) return PDA_ERR_ALIGNMENT;
  if (num_kv_heads > 0 && (!aligned(k, 16) || !aligned(k_out, 16) || k_stride % per16 || k_out_stride % per16))
    return PDA_ERR_ALIGNMENT;
  // an output that starts where its input does has the input's rows
  if ((q == q_out && q_stride != q_out_stride && num_tokens > 1) ||
      (num_kv_heads > 0 && k == k_out && k_stride != k_out_stride && num_tokens > 1))
    return PDA_ERR_SHAPE;
  pda::RotaryApplyArgs a;
  a.rot = rotary_args(rotary);
  a.q = pda::RotaryRows{q, q_out, q_stride, q_out_stride, num_q_heads};
  a.k = pda::RotaryRows{k, k_out, k_stride, k_out_stride, num_kv_heads};
  a.positions = positions;
  a.num_tokens = num_tokens;
  a.head_dim = head_dim;
  return pda::launch_rotary(a, dtype, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

int pda_append_kv_fp8(const pda_problem* prob, const pda_rotary* rotary, const void* q, void* q_out,
                      const void* k_new, const void* v_new, const int32_t* block_table, const int32_t* context_lens,
                      void* k_cache, void* v_cache, uint8_t* kv_scale, hipStream_t stream) {
  int rc = check_problem(prob);
  if (rc != PDA_OK) return rc;
  if (rotary) {
    rc = check_rotary(rotary, prob->head_dim);
    if (rc != PDA_OK) return rc;
    if (rotary->backward) return PDA_ERR_VALUE;
  }
  if ((q != nullptr) != (q_out != nullptr) || (q && !rotary)) return PDA_ERR_NULL;
  if (prob->num_seqs == 0) return PDA_OK;
  if (!k_new || !v_new || !block_table || !context_lens || !k_cache || !v_cache || !kv_scale) return PDA_ERR_NULL;
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_cache, 16) ||
      !aligned(v_cache, 16) || !aligned(kv_scale, 16))
    return PDA_ERR_ALIGNMENT;
  pda::AppendFp8Args a;
  a.rot = rotary_args(rotary);
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.table = block_table;
  a.lens = context_lens;
  a.k = static_cast<uint8_t*>(k_cache);
  a.v = static_cast<uint8_t*>(v_cache);
  a.scale = kv_scale;
  a.num_seqs = prob->num_seqs;
  a.num_query_tokens = query_tokens(prob);
  a.num_q_heads = prob->num_q_heads;
  a.num_kv_heads = prob->num_kv_heads;
  a.num_blocks = prob->num_blocks;
  a.max_blocks_per_seq = prob->max_blocks_per_seq;
  a.max_context_len = prob->max_context_len;
  return pda::launch_append_fp8(a, prob->head_dim, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

int pda_plan_fp8(const pda_problem* prob, pda_plan_info* info) {
  if (!info) return PDA_ERR_NULL;
  Plan plan;
  int rc = make_plan(prob, &plan);
  if (rc != PDA_OK) return rc;
  *info = plan.info;
  return PDA_OK;
}

int pda_decode_fp8(const pda_problem* prob, const void* q, const void* k_cache, const void* v_cache,
                   const uint8_t* kv_scale, const int32_t* block_table, const int32_t* context_lens, float scale,
                   float* out, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Plan plan;
  int rc = make_plan(prob, &plan);
  if (rc != PDA_OK) return rc;
  if (prob->num_seqs > 0 && (!q || !k_cache || !v_cache || !kv_scale || !block_table || !context_lens || !out))
    return PDA_ERR_NULL;
  if (!isfinite(scale)) return PDA_ERR_VALUE;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(kv_scale, 16) || !aligned(out, 16))
    return PDA_ERR_ALIGNMENT;
  if (prob->num_seqs == 0) return PDA_OK;
  if (!workspace || workspace_bytes < plan.info.workspace_bytes) return PDA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return PDA_ERR_ALIGNMENT;
  pda::DecodeFp8Args a;
  a.step = pda::StepArgs{};
  pda::StepArgs& s = a.step;
  float* ws = static_cast<float*>(workspace);
  if (plan.slots > 0) {
    s.part_o = ws;
    s.part_m = ws + plan.slots * prob->head_dim;
    s.part_l = ws + plan.slots * (prob->head_dim + 1);
  }
  // (unsorted items are a grid of three dimensions, whose y and z must hold them)
  const bool ordered = plan.items > kAtOnce;
  a.picks = ordered && plan.narrow && plan.items <= kPickItems &&
            (int64_t)prob->num_seqs * plan.info.num_partitions <= pda::kPickPairs;
  if (ordered && !a.picks) s.order = reinterpret_cast<int32_t*>(ws + plan.slots * (prob->head_dim + 2));
  s.q = static_cast<const uint16_t*>(q);
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
  s.query_chunk = 1;
  s.num_query_chunks = s.num_query_tokens;
  s.chunks_per_group = 1;
  s.num_chunk_groups = plan.tiles;
  s.partition_tokens = plan.info.partition_tokens;
  s.num_partitions = plan.info.num_partitions;
  s.slots_per_row = plan.info.num_partitions;
  s.num_regular_items = (int32_t)plan.items;
  a.k = static_cast<const uint8_t*>(k_cache);
  a.v = static_cast<const uint8_t*>(v_cache);
  a.scale = kv_scale;
  if (s.order && pda::launch_order(s, stream) != hipSuccess) return PDA_ERR_HIP;
  if (pda::launch_decode_fp8(a, prob->head_dim, stream) != hipSuccess) return PDA_ERR_HIP;
  if (plan.slots > 0 && pda::launch_merge(s, prob->head_dim, stream) != hipSuccess) return PDA_ERR_HIP;
  return PDA_OK;
}

int pda_read_kv_fp8(const pda_problem* prob, const void* k_cache, const void* v_cache, const uint8_t* kv_scale,
                    const int32_t* block_table, const int32_t* context_lens, const int32_t* first_token,
                    const int32_t* row_start, int32_t num_rows, void* k_out, void* v_out, hipStream_t stream) {
  int rc = check_problem(prob);
  if (rc != PDA_OK) return rc;
  if (num_rows < 0) return PDA_ERR_SHAPE;
  const int64_t blocks = ((int64_t)prob->max_context_len + pda::kBlockTokens - 1) / pda::kBlockTokens;
  if (blocks * prob->num_seqs > 0x7fffffff) return PDA_ERR_SHAPE;  // the grid
  if (prob->num_seqs == 0 || num_rows == 0) return PDA_OK;
  if (!k_cache || !v_cache || !kv_scale || !block_table || !context_lens || !row_start || !k_out || !v_out)
    return PDA_ERR_NULL;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(kv_scale, 16) || !aligned(k_out, 16) ||
      !aligned(v_out, 16))
    return PDA_ERR_ALIGNMENT;
  pda::ReadFp8Args a;
  a.k = static_cast<const uint8_t*>(k_cache);
  a.v = static_cast<const uint8_t*>(v_cache);
  a.scale = kv_scale;
  a.table = block_table;
  a.lens = context_lens;
  a.first = first_token;
  a.row_start = row_start;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.num_rows = num_rows;
  a.num_seqs = prob->num_seqs;
  a.num_kv_heads = prob->num_kv_heads;
  a.num_blocks = prob->num_blocks;
  a.max_blocks_per_seq = prob->max_blocks_per_seq;
  a.max_context_len = prob->max_context_len;
  return pda::launch_read_fp8(a, prob->head_dim, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

}  // extern "C"
