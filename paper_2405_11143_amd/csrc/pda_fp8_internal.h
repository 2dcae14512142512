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
  bool picks;              // every workgroup finds its item in the work order by itself (no step.order)
};

constexpr int kPickPairs = 256;  // (sequence, partition) pairs of a step that does: one per thread

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

// 8 codes (two dwords) times a power of two, as 8 bf16, one instruction for two of them:
// exact down to bf16's smallest, 2^-133 (values that are no multiples of it are rounded), and
// infinite from 2^128 on.
__device__ __forceinline__ uint4 to_bf16(unsigned lo, unsigned hi, float factor) {
  auto two = [&](unsigned w, bool upper) {
    const bf16x2_t x = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, factor, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, factor, false);
    return __builtin_bit_cast(unsigned, x);
  };
  return make_uint4(two(lo, false), two(lo, true), two(hi, false), two(hi, true));
}

// Whether any of 4 codes stands for 2^128 or more under scale byte s (247 .. 254: codes
// above that of 240 under 247, 120 under 248, ..; 255 is a row of NaN): an infinity as bf16.
constexpr unsigned kLargeScale = 247;
__device__ __forceinline__ bool infinite(unsigned codes, unsigned s) {
  const unsigned top = 0x77u - 8u * (s - kLargeScale);
  const unsigned m = codes & 0x7f7f7f7fu;
  return s >= kLargeScale && ((m + (0x7fu - top) * 0x01010101u) & 0x80808080u) != 0;
}

// cos and sin of position * frequency (times sign), the angle in 64 bits:
// whole turns are taken off before it is rounded to 32.
__device__ __forceinline__ float2 turn(const RotaryArgs& r, int position, int pair) {
  const double turns = (double)position * r.inv_freq[pair] * 0.15915494309189533577;  // 1 / (2 pi)
  float s, c;
  sincospif(2.f * (float)(turns - __builtin_rint(turns)), &s, &c);
  return make_float2(c * r.magnitude, r.sign * s * r.magnitude);
}

// A thread's share of a head row: two vectors of 8 elements, d0 and d1 (from D on:
// there is none), of which the first `turned` are rotated.  In the half layout a
// rotated share is 8 pairs; interleaved, each vector is 4 pairs by itself.  Shares of
// neighbouring threads are neighbouring vectors, so that a store of the
// wavefront covers whole cache lines where the row allows it.
struct RowShare {
  int d0, d1, turned;
};
__host__ __device__ constexpr int row_shares(int head_dim) { return (head_dim + 15) / 16; }
__device__ __forceinline__ RowShare row_share(const RotaryArgs& r, int rotary_dim, int head_dim, int u) {
  const int shares = row_shares(head_dim);
  if (r.interleaved || rotary_dim == 0) {
    const int d0 = 8 * u, d1 = 8 * (u + shares);
    return RowShare{d0, d1, d1 < rotary_dim ? 2 : d0 < rotary_dim ? 1 : 0};
  }
  const int pairs8 = rotary_dim / 16;
  if (u < pairs8) return RowShare{8 * u, rotary_dim / 2 + 8 * u, 2};
  const int d0 = rotary_dim + 8 * (u - pairs8);
  return RowShare{d0, d0 + 8 * (shares - pairs8), 0};
}

// Rotates a share's vectors by the cosines and sines of the row's pairs.
__device__ __forceinline__ void rotate_share(const float2* turns, bool interleaved, const RowShare& w, float (&p)[8],
                                             float (&q)[8]) {
  auto four = [](const float2* cs, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float2 c = cs[e / 2];
      const float a = x[e], b = x[e + 1];
      x[e] = a * c.x - b * c.y, x[e + 1] = b * c.x + a * c.y;
    }
  };
  if (w.turned == 0) return;
  if (interleaved) {
    four(turns + w.d0 / 2, p);
    if (w.turned == 2) four(turns + w.d1 / 2, q);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 c = turns[w.d0 + e];
      const float a = p[e], b = q[e];
      p[e] = a * c.x - b * c.y, q[e] = b * c.x + a * c.y;
    }
  }
}

// Whether the stores of the rotated rows (bf16) cover whole cache lines of 128 bytes:
// then, with many tokens, they go out with the non-temporal hint (16384 tokens of
// 32 + 8 heads of 128: 64 -> 59 us); lines written in halves would be written
// twice (neighbouring pairs in shares of 16 neighbouring elements took 30% longer).
inline bool whole_lines(const RotaryArgs& r, int head_dim) {
  const int copied = r.interleaved ? head_dim : head_dim - r.rotary_dim;  // elements in vectors of their own
  return copied % 128 == 0 && (r.interleaved || r.rotary_dim % 128 == 0);
}
constexpr int64_t kManyTokens = 2048;

}  // namespace pda
