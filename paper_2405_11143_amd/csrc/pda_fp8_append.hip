// The quantised KV append (include/pda_fp8.h): each new token's key row rotated
// and, like its value row, stored as e4m3 codes and a power-of-two scale; its
// query rows rotated beside.
//
// A workgroup takes one new token: the cosines and sines of its position go
// to LDS once, then D / 16 threads take each row, 16 elements each (for a
// rotated row 8 pairs), and form the row's largest magnitude by shuffles.
#include "pda_fp8_internal.h"

namespace pda {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups (a launch has less than 2^32 threads); they loop over the rest

typedef __bf16 bf16v8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const bf16v8_t a = *reinterpret_cast<const bf16v8_t*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
}

// The scale byte of a row whose largest magnitude has the bits `top` (of the
// absolute value: a NaN's are the largest).  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(unsigned top) {
  const int e = top >> 23;
  if (top == 0) return 0;
  if (e == 255) return 255;
  return max(e - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
}

// 8 values times 2^(127 - s) as codes, rounded to nearest even; at most 448
// in magnitude, so nothing saturates.
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], int s) {
  if (s == 255) return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);  // NaN
  const float f = __uint_as_float((unsigned)(254 - max(s, 1)) << 23);
  unsigned w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h] * f, x[4 * h + 1] * f, 0, false);
    w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2] * f, x[4 * h + 3] * f, c, true);
  }
  return make_uint2(w[0], w[1]);
}

template <int D>
__global__ void __launch_bounds__(kThreads) append_fp8_kernel(const AppendFp8Args a) {
  constexpr int U = D / 16;  // threads per row
  __shared__ float2 turns[D / 2];
  const int n = a.num_query_tokens;
  for (int64_t token = blockIdx.x; token < (int64_t)a.num_seqs * n; token += gridDim.x) {
  const int b = (int)(token / n), i = (int)(token % n);
  const int L = clamped(a.lens[b], a.max_context_len);
  const int t = L - n + i;
  if (t < 0) continue;  // (the whole workgroup)
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  if ((int)threadIdx.x < R / 2) turns[threadIdx.x] = turn(a.rot, t, threadIdx.x);
  const int page = a.table[(size_t)b * a.max_blocks_per_seq + t / kBlockTokens];
  const bool stored = (unsigned)page < (unsigned)a.num_blocks;
  const int o = t % kBlockTokens;
  __syncthreads();
  const int nq = a.q ? a.num_q_heads : 0;
  const int rows = nq + 2 * a.num_kv_heads;  // queries, keys, values
  const int u = threadIdx.x % U;
  for (int row0 = 0; row0 < rows; row0 += kThreads / U) {  // (the same trips for all threads: they shuffle)
    const int row = row0 + threadIdx.x / U;
    const bool live = row < rows;
    const int which = row < nq ? 0 : row < nq + a.num_kv_heads ? 1 : 2;
    const int h = !live ? 0 : which == 0 ? row : which == 1 ? row - nq : row - nq - a.num_kv_heads;
    const uint16_t* src = which == 0 ? a.q : which == 1 ? a.k_new : a.v_new;
    src += (token * (which == 0 ? a.num_q_heads : a.num_kv_heads) + h) * D;
    const bool turned = which < 2 && 16 * u < R;
    int d0 = 16 * u, d1 = 16 * u + 8;
    if (turned && !a.rot.interleaved) d0 = 8 * u, d1 = 8 * u + R / 2;
    float x[8], y[8];
    if (live) {
      load8(src + d0, x);
      load8(src + d1, y);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
    }
    if (turned) {
      const float2* cs = &turns[8 * u];
      if (a.rot.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 c0 = cs[e / 2], c1 = cs[4 + e / 2];
          const float x0 = x[e], x1 = x[e + 1], y0 = y[e], y1 = y[e + 1];
          x[e] = x0 * c0.x - x1 * c0.y, x[e + 1] = x1 * c0.x + x0 * c0.y;
          y[e] = y0 * c1.x - y1 * c1.y, y[e + 1] = y1 * c1.x + y0 * c1.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 c = cs[e];
          const float x0 = x[e], y0 = y[e];
          x[e] = x0 * c.x - y0 * c.y, y[e] = y0 * c.x + x0 * c.y;
        }
      }
    }
    if (which == 0) {
      bf16v8_t p, q;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (__bf16)x[e], q[e] = (__bf16)y[e];
      uint16_t* dst = a.q_out + (token * a.num_q_heads + h) * D;
      if (live) {
        *reinterpret_cast<bf16v8_t*>(dst + d0) = p;
        *reinterpret_cast<bf16v8_t*>(dst + d1) = q;
      }
    }
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      top = max(top, max(__float_as_uint(x[e]) & 0x7fffffffu, __float_as_uint(y[e]) & 0x7fffffffu));
#pragma unroll
    for (int m = 1; m < U; m <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, m));
    if (which == 0 || !live || !stored) continue;
    const int s = scale_byte(top);
    const uint2 cx = codes_of(x, s), cy = codes_of(y, s);
    const size_t tile = (size_t)page * a.num_kv_heads + h;
    auto at = [&](int d) {
      return which == 1 ? ((d / 64 * 4 + d / 8 % 4) * 16 + o) * 16 + d / 32 % 2 * 8
                        : (((o / 2 % 2) * 4 + o / 4) * (D / 8) + d / 8) * 16 + o % 2 * 8;
    };
    uint8_t* dst = (which == 1 ? a.k : a.v) + tile * (16 * D);
    *reinterpret_cast<uint2*>(dst + at(d0)) = cx;
    *reinterpret_cast<uint2*>(dst + at(d1)) = cy;
    if (u == 0) a.scale[tile * 32 + (which == 1 ? 0 : 16) + o] = (uint8_t)s;
  }
  __syncthreads();  // the next token's turns take the same place
  }
}

}  // namespace

hipError_t launch_append_fp8(const AppendFp8Args& a, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)min((int64_t)a.num_seqs * a.num_query_tokens, kMaxGrid));
  if (head_dim == 64)
    hipLaunchKernelGGL((append_fp8_kernel<64>), grid, dim3(kThreads), 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((append_fp8_kernel<128>), grid, dim3(kThreads), 0, stream, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pda
