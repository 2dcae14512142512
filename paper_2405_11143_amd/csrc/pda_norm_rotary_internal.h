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

// Lanes of a wavefront that share a row.
inline int row_lanes(int head_dim) {
  const int shares = row_shares(head_dim);
  return shares <= 4 ? 4 : shares <= 8 ? 8 : shares <= 16 ? 16 : 32;
}

// Steps of a wavefront that rows of several kinds take, and wavefronts of at most `ways` that share them: as many
// as make the last trip a full one, nearly.
inline int row_steps(int heads, int lanes) { return (heads * lanes + kWaveSize - 1) / kWaveSize; }
inline int wave_parts(int steps, int64_t ways) {
  const int most = (int)(ways < 1 ? 1 : ways < steps ? ways : steps);
  const int trips = (steps + most - 1) / most;
  return (steps + trips - 1) / trips;
}

// A backward pass: wavefronts that share a token, and workgroups (4 wavefronts, each a token or its part
// of one at a time); each workgroup leaves one partial sum of the weights' gradients.  By the queries alone: their
// results are the same bits with and without keys.  32 + 8 heads of 128, us, whole / up to 2048 wavefronts / up to
// half as many again or half: 4 tokens 14.1 / 11.2, 300 15.1 / 13.4, 700 15.3 / 14.6 / 15.8 or 15.1, 1500 18.2 / 18.1 / 18.8 or 18.1.
constexpr int kGradGroups = 768;  // three wavefronts to every SIMD
constexpr int kGradWaves = 2048;
inline int grad_parts(int64_t num_tokens, int q_heads, int head_dim) {
  return num_tokens < 1 ? 1 : wave_parts(row_steps(q_heads, row_lanes(head_dim)), kGradWaves / num_tokens);
}
inline int grad_groups(int64_t num_tokens, int parts) {
  const int64_t groups = (num_tokens * parts + 3) / 4;
  return (int)(groups < kGradGroups ? groups : kGradGroups);
}

hipError_t launch_norm_rotary(const NormRotaryArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_rotary_append(const NormRotaryArgs& a, hipStream_t stream);
hipError_t launch_norm_rotary_backward(const NormRotaryArgs& a, int dtype, hipStream_t stream);

}  // namespace pda
