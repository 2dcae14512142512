// Rotary positions of query and key rows (include/pda_fp8.h).
//
// Bound by memory: every row is read and written once, and a pair costs 4
// multiply-adds.  The angles are what is expensive (a 64-bit product and
// reduction, then sine and cosine), and the same for all heads of a token: a
// workgroup takes one token, forms its cosines and sines in LDS, a thread each,
// and then its rows, 16 elements per thread.  16384 tokens of 32 + 8 heads of 128, bf16:
// 59 us, 5.6 TB/s (a large copy 4.9); neighbouring pairs in half of 28 + 4 heads'
// elements, the others copied: 47 us, 5.6 TB/s; in fp32, without the hint, 125 and 99 us, 5.3
// TB/s.  Four tokens to a workgroup (its loop
// goes from row to row and from token to token) took 8% longer than one, two 10%.
#include "pda_fp8_internal.h"

namespace pda {
namespace {

constexpr int kMaxThreads = 256;
constexpr int kMaxGrid = 1 << 20;  // workgroups (a launch has less than 2^32 threads); they loop over the rest
constexpr int kMaxPairs = 256;  // head_dim <= 512

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  const v8 a = *reinterpret_cast<const v8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
}
template <bool NT>
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  static_assert(!NT, "bf16 rows only");
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <bool NT>
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  v8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
  if (NT)
    __builtin_nontemporal_store(a, reinterpret_cast<v8*>(p));
  else
    *reinterpret_cast<v8*>(p) = a;
}

// NT: stores with the non-temporal hint (bf16).
template <typename T, bool NT>
__global__ void __launch_bounds__(kMaxThreads) rotary_kernel(const RotaryApplyArgs a) {
  __shared__ float2 turns[kMaxPairs];
  const int D = a.head_dim;
  const int pairs = a.rot.rotary_dim / 2;
  const int shares = row_shares(D);
  const int first_row = threadIdx.x / shares;
  const int rows_at_once = blockDim.x / shares;
  const RowShare w = row_share(a.rot, a.rot.rotary_dim, D, threadIdx.x % shares);
  const int heads = a.q.heads + a.k.heads;
  for (int64_t t = blockIdx.x; t < a.num_tokens; t += gridDim.x) {
    const int pos = a.positions[t];
    if (pos < 0) continue;  // padding (the whole workgroup)
    for (int x = threadIdx.x; x < pairs; x += blockDim.x) turns[x] = turn(a.rot, pos, x);
    __syncthreads();
    for (int h = first_row < rows_at_once ? first_row : heads; h < heads; h += rows_at_once) {
      const bool is_q = h < a.q.heads;
      const RotaryRows& r = is_q ? a.q : a.k;
      const int64_t at = (int64_t)(is_q ? h : h - a.q.heads) * D;
      const T* in = static_cast<const T*>(r.in) + t * r.in_stride + at;
      T* out = static_cast<T*>(r.out) + t * r.out_stride + at;
      const bool copies = r.in != r.out;
      const bool one = copies || w.turned > 0, two = w.d1 < D && (copies || w.turned > 1);
      float p[8], q[8];
      if (one) load8(in + w.d0, p);
      if (two) load8(in + w.d1, q);
      rotate_share(turns, a.rot.interleaved, w, p, q);
      if (one) store8<NT>(out + w.d0, p);
      if (two) store8<NT>(out + w.d1, q);
    }
    __syncthreads();  // the next token's turns take the same place
  }
}

// A workgroup has as many threads as make its last trip through the rows a full
// one, nearly (up to 512 of them for a single trip took 12% longer).
template <typename T>
hipError_t launch_t(const RotaryApplyArgs& a, hipStream_t stream) {
  const int units = (a.q.heads + a.k.heads) * row_shares(a.head_dim);
  const int trips = (units + kMaxThreads - 1) / kMaxThreads;
  const int threads = min(kMaxThreads, ((units + trips - 1) / trips + kWaveSize - 1) / kWaveSize * kWaveSize);
  const dim3 grid(min(a.num_tokens, kMaxGrid));
  if constexpr (sizeof(T) == 2) {
    if (a.num_tokens >= kManyTokens && whole_lines(a.rot, a.head_dim)) {
      hipLaunchKernelGGL((rotary_kernel<T, true>), grid, dim3(threads), 0, stream, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((rotary_kernel<T, false>), grid, dim3(threads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryApplyArgs& a, int dtype, hipStream_t stream) {
  return dtype == PDA_DTYPE_BF16 ? launch_t<__bf16>(a, stream) : launch_t<float>(a, stream);
}

}  // namespace pda
