// Internal interface of the head norms and several-axis rotary positions
// (include/pda_norm_rotary.h), between their host layer and their gfx950 kernels.
#pragma once

#include "pda_fp8_internal.h"
#include "pda_norm_rotary.h"

namespace pda {

struct NormRotaryArgs {
  RotaryArgs rot;           // (its inv_freq null: no rotation)
  const uint8_t* axis;      // [rotary_dim / 2], or null: one axis
  int64_t position_stride;  // elements from axis to axis
  int32_t num_axes;
  int32_t normed;           // 0: rotation alone
  float eps, offset;
  int32_t weight_f32;       // else bf16
  const void* weight[2];    // of queries and keys, or null
  RotaryRows q, k;          // a backward pass: x in, dx out
  const int32_t* positions;
  int32_t num_tokens;
  int32_t head_dim;
  // the append
  const uint16_t* v;        // bf16 [T][heads of k][D]
  int64_t v_stride;
  const int32_t* slots;
  uint16_t* k_cache;        // bf16 [num_blocks][Hkv][D/8][16][8]
  uint16_t* v_cache;        // bf16 [num_blocks][Hkv][16][D]
  int32_t num_blocks;
  // the backward pass
  RotaryRows q_grad, k_grad;  // in: the gradients of the outputs
  float* d_weight[2];         // fp32 [D], or null
  float* part;                // [grad_groups()][2][D]
};

// Workgroups of a backward pass (4 wavefronts, a token each at a time); each leaves one
// partial sum of the weights' gradients.
inline int grad_groups(int64_t num_tokens) { return (int)(num_tokens < 4 * 768 ? (num_tokens + 3) / 4 : 768); }

hipError_t launch_norm_rotary(const NormRotaryArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_rotary_append(const NormRotaryArgs& a, hipStream_t stream);
hipError_t launch_norm_rotary_backward(const NormRotaryArgs& a, int dtype, hipStream_t stream);

}  // namespace pda
