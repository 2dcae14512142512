// Host side of the head norms and several-axis rotary positions (declared in
// include/pda_norm_rotary.h): validation and the launches.  Nothing here allocates
// memory or keeps state between calls.
#include <math.h>
#include <stdint.h>

#include "pda_norm_rotary_internal.h"

namespace {

constexpr int kMaxHeadDim = 512;
constexpr int kMaxAxes = 4;
constexpr int32_t kMaxSlotBlocks = 1 << 27;  // 16 * num_blocks fits the slots' int32

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

// The norm, the rotation and the axes, and the kernels' arguments for them.
int check_heads(const pda_head_norm* norm, const pda_rotary* rotary, const pda_rotary_axes* axes, int32_t num_tokens,
                int32_t head_dim, pda::NormRotaryArgs* a) {
  if (head_dim < 1 || num_tokens < 0) return PDA_ERR_SHAPE;
  if (head_dim % 8 != 0 || head_dim > kMaxHeadDim) return PDA_ERR_UNSUPPORTED;
  if (norm) {
    if (norm->weight_dtype != PDA_DTYPE_BF16 && norm->weight_dtype != PDA_DTYPE_F32) return PDA_ERR_UNSUPPORTED;
    if (!isfinite(norm->eps) || norm->eps < 0.f || !isfinite(norm->weight_offset)) return PDA_ERR_VALUE;
    if (!aligned(norm->q_weight, 16) || !aligned(norm->k_weight, 16)) return PDA_ERR_ALIGNMENT;
  }
  if (rotary) {
    const int rc = pda::check_rotary(rotary, head_dim);
    if (rc != PDA_OK) return rc;
    if (norm && rotary->backward) return PDA_ERR_VALUE;
  }
  if (axes) {
    if (!rotary || !axes->axis_of_pair) return PDA_ERR_NULL;
    if (axes->num_axes < 1 || (axes->num_axes > 1 && axes->position_stride < num_tokens)) return PDA_ERR_SHAPE;
    if (axes->num_axes > kMaxAxes) return PDA_ERR_UNSUPPORTED;
  }
  *a = pda::NormRotaryArgs{};
  a->rot = pda::rotary_args(rotary);
  a->num_axes = axes ? axes->num_axes : 1;
  a->axis = a->num_axes > 1 ? axes->axis_of_pair : nullptr;
  a->position_stride = axes ? axes->position_stride : 0;
  if (norm) {
    a->normed = 1;
    a->eps = norm->eps;
    a->offset = norm->weight_offset;
    a->weight_f32 = norm->weight_dtype == PDA_DTYPE_F32;
    a->weight[0] = norm->q_weight;
    a->weight[1] = norm->k_weight;
  }
  a->num_tokens = num_tokens;
  a->head_dim = head_dim;
  return PDA_OK;
}

int check_sizes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t dtype) {
  if (num_q_heads < 0 || num_kv_heads < 0) return PDA_ERR_SHAPE;
  if (dtype != PDA_DTYPE_BF16 && dtype != PDA_DTYPE_F32) return PDA_ERR_UNSUPPORTED;
  if (((int64_t)num_q_heads + 2 * (int64_t)num_kv_heads) * head_dim > (1 << 24)) return PDA_ERR_SHAPE;  // a token's rows
  return PDA_OK;
}

int check_stride(int64_t stride, int32_t heads, int32_t head_dim) {
  return stride < (int64_t)heads * head_dim ? PDA_ERR_SHAPE : PDA_OK;
}

// One operand's pointer and stride (heads > 0).
int check_rows(const void* p, int64_t stride, int32_t dtype) {
  if (!p) return PDA_ERR_NULL;
  return aligned(p, 16) && stride % (dtype == PDA_DTYPE_BF16 ? 8 : 4) == 0 ? PDA_OK : PDA_ERR_ALIGNMENT;
}

// An output that starts where an input does has the input's rows.
int check_in_place(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int32_t num_tokens) {
  return in == out && in_stride != out_stride && num_tokens > 1 ? PDA_ERR_SHAPE : PDA_OK;
}

#define PDA_CHECK(expr)                 \
  do {                                  \
    const int rc_ = (expr);             \
    if (rc_ != PDA_OK) return rc_;      \
  } while (0)

}  // namespace

extern "C" {

int pda_norm_rotary(const pda_head_norm* norm, const pda_rotary* rotary, const pda_rotary_axes* axes,
                    int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t dtype,
                    const int32_t* positions, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                    const void* k, int64_t k_stride, void* k_out, int64_t k_out_stride, hipStream_t stream) {
  if (!norm && !rotary) return PDA_ERR_NULL;
  pda::NormRotaryArgs a;
  PDA_CHECK(check_heads(norm, rotary, axes, num_tokens, head_dim, &a));
  if (num_q_heads < 1) return PDA_ERR_SHAPE;
  PDA_CHECK(check_sizes(num_q_heads, num_kv_heads, head_dim, dtype));
  PDA_CHECK(check_stride(q_stride, num_q_heads, head_dim));
  PDA_CHECK(check_stride(q_out_stride, num_q_heads, head_dim));
  if (num_kv_heads > 0) {
    PDA_CHECK(check_stride(k_stride, num_kv_heads, head_dim));
    PDA_CHECK(check_stride(k_out_stride, num_kv_heads, head_dim));
  }
  if (num_tokens == 0) return PDA_OK;
  if (!positions) return PDA_ERR_NULL;
  PDA_CHECK(check_rows(q, q_stride, dtype));
  PDA_CHECK(check_rows(q_out, q_out_stride, dtype));
  PDA_CHECK(check_in_place(q, q_stride, q_out, q_out_stride, num_tokens));
  if (num_kv_heads > 0) {
    PDA_CHECK(check_rows(k, k_stride, dtype));
    PDA_CHECK(check_rows(k_out, k_out_stride, dtype));
    PDA_CHECK(check_in_place(k, k_stride, k_out, k_out_stride, num_tokens));
  }
  a.q = pda::RotaryRows{q, q_out, q_stride, q_out_stride, num_q_heads};
  a.k = pda::RotaryRows{k, k_out, k_stride, k_out_stride, num_kv_heads};
  a.positions = positions;
  return pda::launch_norm_rotary(a, dtype, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

int pda_norm_rotary_workspace_bytes(int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                    size_t* bytes) {
  if (!bytes) return PDA_ERR_NULL;
  if (num_tokens < 0 || head_dim < 1 || num_q_heads < 1) return PDA_ERR_SHAPE;
  if (head_dim % 8 != 0 || head_dim > kMaxHeadDim) return PDA_ERR_UNSUPPORTED;
  PDA_CHECK(check_sizes(num_q_heads, num_kv_heads, head_dim, PDA_DTYPE_F32));
  const int parts = pda::grad_parts(num_tokens, num_q_heads, head_dim);
  *bytes = (size_t)pda::grad_groups(num_tokens, parts) * 2 * head_dim * sizeof(float);
  return PDA_OK;
}

int pda_norm_rotary_backward(const pda_head_norm* norm, const pda_rotary* rotary, const pda_rotary_axes* axes,
                             int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                             int32_t dtype, const int32_t* positions, const void* q, int64_t q_stride,
                             const void* q_grad, int64_t q_grad_stride, void* dq, int64_t dq_stride, const void* k,
                             int64_t k_stride, const void* k_grad, int64_t k_grad_stride, void* dk,
                             int64_t dk_stride, float* dq_weight, float* dk_weight, void* workspace,
                             size_t workspace_bytes, hipStream_t stream) {
  if (!norm) return PDA_ERR_NULL;
  pda::NormRotaryArgs a;
  PDA_CHECK(check_heads(norm, rotary, axes, num_tokens, head_dim, &a));
  size_t need;
  PDA_CHECK(pda_norm_rotary_workspace_bytes(num_tokens, num_q_heads, num_kv_heads, head_dim, &need));
  PDA_CHECK(check_sizes(num_q_heads, num_kv_heads, head_dim, dtype));
  PDA_CHECK(check_stride(q_stride, num_q_heads, head_dim));
  PDA_CHECK(check_stride(q_grad_stride, num_q_heads, head_dim));
  PDA_CHECK(check_stride(dq_stride, num_q_heads, head_dim));
  if (num_kv_heads > 0) {
    PDA_CHECK(check_stride(k_stride, num_kv_heads, head_dim));
    PDA_CHECK(check_stride(k_grad_stride, num_kv_heads, head_dim));
    PDA_CHECK(check_stride(dk_stride, num_kv_heads, head_dim));
  } else if (dk_weight) {
    return PDA_ERR_SHAPE;
  }
  if (num_tokens > 0) {
    if (!positions) return PDA_ERR_NULL;
    PDA_CHECK(check_rows(q, q_stride, dtype));
    PDA_CHECK(check_rows(q_grad, q_grad_stride, dtype));
    PDA_CHECK(check_rows(dq, dq_stride, dtype));
    PDA_CHECK(check_in_place(q, q_stride, dq, dq_stride, num_tokens));
    PDA_CHECK(check_in_place(q_grad, q_grad_stride, dq, dq_stride, num_tokens));
    if (num_kv_heads > 0) {
      PDA_CHECK(check_rows(k, k_stride, dtype));
      PDA_CHECK(check_rows(k_grad, k_grad_stride, dtype));
      PDA_CHECK(check_rows(dk, dk_stride, dtype));
      PDA_CHECK(check_in_place(k, k_stride, dk, dk_stride, num_tokens));
      PDA_CHECK(check_in_place(k_grad, k_grad_stride, dk, dk_stride, num_tokens));
    }
  }
  if (!aligned(dq_weight, 16) || !aligned(dk_weight, 16)) return PDA_ERR_ALIGNMENT;
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return PDA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return PDA_ERR_ALIGNMENT;
  }
  a.rot.sign = -1.f;  // the transpose turns back
  a.q = pda::RotaryRows{q, dq, q_stride, dq_stride, num_q_heads};
  a.k = pda::RotaryRows{k, dk, k_stride, dk_stride, num_kv_heads};
  a.q_grad = pda::RotaryRows{q_grad, nullptr, q_grad_stride, 0, num_q_heads};
  a.k_grad = pda::RotaryRows{k_grad, nullptr, k_grad_stride, 0, num_kv_heads};
  a.d_weight[0] = dq_weight;
  a.d_weight[1] = dk_weight;
  a.part = static_cast<float*>(workspace);
  a.positions = positions;
  if (num_tokens == 0 && !dq_weight && !dk_weight) return PDA_OK;
  return pda::launch_norm_rotary_backward(a, dtype, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

int pda_norm_rotary_append(const pda_head_norm* norm, const pda_rotary* rotary, const pda_rotary_axes* axes,
                           int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                           int32_t num_blocks, const int32_t* positions, const int32_t* slots, const void* q,
                           int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride,
                           const void* v, int64_t v_stride, void* k_cache, void* v_cache, hipStream_t stream) {
  pda::NormRotaryArgs a;
  PDA_CHECK(check_heads(norm, rotary, axes, num_tokens, head_dim, &a));
  if (head_dim != 64 && head_dim != 128) return PDA_ERR_UNSUPPORTED;
  if (num_kv_heads < 1 || num_blocks < 1 || num_blocks > kMaxSlotBlocks) return PDA_ERR_SHAPE;
  PDA_CHECK(check_sizes(num_q_heads, num_kv_heads, head_dim, PDA_DTYPE_BF16));
  if (rotary && rotary->backward) return PDA_ERR_VALUE;
  if (!norm && !rotary && num_q_heads > 0) return PDA_ERR_NULL;
  if (num_q_heads > 0) {
    PDA_CHECK(check_stride(q_stride, num_q_heads, head_dim));
    PDA_CHECK(check_stride(q_out_stride, num_q_heads, head_dim));
  }
  PDA_CHECK(check_stride(k_stride, num_kv_heads, head_dim));
  PDA_CHECK(check_stride(v_stride, num_kv_heads, head_dim));
  if (num_tokens == 0) return PDA_OK;
  if (!positions || !slots || !k_cache || !v_cache) return PDA_ERR_NULL;
  if (num_q_heads > 0) {
    PDA_CHECK(check_rows(q, q_stride, PDA_DTYPE_BF16));
    PDA_CHECK(check_rows(q_out, q_out_stride, PDA_DTYPE_BF16));
    PDA_CHECK(check_in_place(q, q_stride, q_out, q_out_stride, num_tokens));
  }
  PDA_CHECK(check_rows(k, k_stride, PDA_DTYPE_BF16));
  PDA_CHECK(check_rows(v, v_stride, PDA_DTYPE_BF16));
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return PDA_ERR_ALIGNMENT;
  a.q = pda::RotaryRows{q, q_out, q_stride, q_out_stride, num_q_heads};
  a.k = pda::RotaryRows{k, nullptr, k_stride, 0, num_kv_heads};
  a.v = static_cast<const uint16_t*>(v);
  a.v_stride = v_stride;
  a.positions = positions;
  a.slots = slots;
  a.k_cache = static_cast<uint16_t*>(k_cache);
  a.v_cache = static_cast<uint16_t*>(v_cache);
  a.num_blocks = num_blocks;
  return pda::launch_norm_rotary_append(a, stream) == hipSuccess ? PDA_OK : PDA_ERR_HIP;
}

}  // extern "C"
