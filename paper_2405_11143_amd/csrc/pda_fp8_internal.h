// Internal interface of the 8-bit KV cache and the rotary positions
// (include/pda_fp8.h), between their host layer and their gfx950 kernels.
#pragma once

#include "pda_fp8.h"
#include "pda_internal.h"

namespace pda {

// A rotary embedding as the kernels take it.
struct RotaryArgs {
  const double* inv_freq;  // [rotary_dim / 2], or null: no rotation
  float magnitude;
  float sign;              // of the angle: -1 in the backward direction
  int32_t rotary_dim;
  int32_t interleaved;
};

struct RotaryRows {        // rows of one operand
  const void* in;
  void* out;
  int64_t in_stride, out_stride;  // elements from token to token
  int32_t heads;
};

struct RotaryApplyArgs {
  RotaryArgs rot;
  RotaryRows q, k;
  const int32_t* positions;
  int32_t num_tokens;
  int32_t head_dim;
};

// The quantised append.
struct AppendFp8Args {
  RotaryArgs rot;
  const uint16_t* q;       // bf16 [B][n][Hq][D], or null
  uint16_t* q_out;
  const uint16_t* k_new;   // bf16 [B][n][Hkv][D]
  const uint16_t* v_new;
  const int32_t* table;
  const int32_t* lens;
  uint8_t* k;              // the cache
  uint8_t* v;
  uint8_t* scale;
  int32_t num_seqs, num_query_tokens, num_q_heads, num_kv_heads, num_blocks, max_blocks_per_seq, max_context_len;
};

// Attention over the 8-bit cache.  `step` is what the order and merge kernels
// read (query_chunk is 1 there: every row has its own number of partitions,
// and num_chunk_groups counts the row tiles of a work item's sequence and KV
// head); its k and v are null.
struct DecodeFp8Args {
  StepArgs step;
  const uint8_t* k;        // e4m3 [num_blocks][Hkv][D/64][4][16][2][8]
  const uint8_t* v;        // e4m3 [num_blocks][Hkv][2][4][D/8][2][8]
  const uint8_t* scale;    // [num_blocks][Hkv][2][16]
};

struct ReadFp8Args {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* scale;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* first;      // [B], or null
  const int32_t* row_start;  // [B + 1]
  uint16_t* k_out;           // bf16 [num_rows][Hkv][D]
  uint16_t* v_out;
  int32_t num_rows;
  int32_t num_seqs, num_kv_heads, num_blocks, max_blocks_per_seq, max_context_len;
};

hipError_t launch_rotary(const RotaryApplyArgs& a, int dtype, hipStream_t stream);
hipError_t launch_append_fp8(const AppendFp8Args& a, int head_dim, hipStream_t stream);
hipError_t launch_decode_fp8(const DecodeFp8Args& a, int head_dim, hipStream_t stream);
hipError_t launch_wide_fp8(const DecodeFp8Args& a, int head_dim, hipStream_t stream);  // more than 32 rows
hipError_t launch_read_fp8(const ReadFp8Args& a, int head_dim, hipStream_t stream);

constexpr int kFp8TileRows = 16;  // query rows of an MFMA tile of the decode kernel

// Query rows of a work item whose sequence and KV head has `rows` of them: one or
// two tiles of the decode kernel, or the rows of a workgroup of the wide one.
inline int fp8_item_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

// ---- device helpers ----

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int clamped(int L, int most) { return L < 0 ? 0 : (L > most ? most : L); }

// The factor 2^(s - 127) of scale byte `which` (0 .. 3) of a dword (0 for byte 0).
template <int WHICH>
__device__ __forceinline__ float scale_of(unsigned bytes) {
  constexpr int up = 23 - 8 * WHICH;
  return __uint_as_float((up >= 0 ? bytes << (up & 31) : bytes >> (-up & 31)) & 0x7f800000u);
}

// 8 codes (two dwords) times a power of two, as 8 bf16: exact, and one
// instruction for two of them.
__device__ __forceinline__ uint4 to_bf16(unsigned lo, unsigned hi, float factor) {
  auto two = [&](unsigned w, bool upper) {
    const bf16x2_t x = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, factor, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, factor, false);
    return __builtin_bit_cast(unsigned, x);
  };
  return make_uint4(two(lo, false), two(lo, true), two(hi, false), two(hi, true));
}

// cos and sin of position * frequency (times sign), the angle in 64 bits:
// whole turns are taken off before it is rounded to 32.
__device__ __forceinline__ float2 turn(const RotaryArgs& r, int position, int pair) {
  const double turns = (double)position * r.inv_freq[pair] * 0.15915494309189533577;  // 1 / (2 pi)
  float s, c;
  sincospif(2.f * (float)(turns - __builtin_rint(turns)), &s, &c);
  return make_float2(c * r.magnitude, r.sign * s * r.magnitude);
}

}  // namespace pda
