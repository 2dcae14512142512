// Rotary positions of query and key rows (include/pda_fp8.h).
//
// Bound by memory: every row is read and written once, and a pair costs 4
// multiply-adds.  The angles are what is expensive (a 64-bit product and
// reduction, then sine and cosine), and the same for all heads of a token: a
// workgroup takes one or a few tokens, forms their cosines and sines in LDS
// first, one thread each, and then streams the tokens' rows, 16 elements per
// thread: 8 pairs, as two vectors of 8 in either layout.
#include "pda_fp8_internal.h"

namespace pda {
namespace {

constexpr int kThreads = 256;
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
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  v8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
  *reinterpret_cast<v8*>(p) = a;
}

// TOKENS: tokens of a workgroup.
template <typename T, int TOKENS>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryApplyArgs a) {
  __shared__ float2 turns[TOKENS][kMaxPairs];
  const int R = a.rot.rotary_dim;
  const int pairs = R / 2;
  for (int64_t t0 = (int64_t)blockIdx.x * TOKENS; t0 < a.num_tokens; t0 += (int64_t)gridDim.x * TOKENS) {
  const int nt = (int)min((int64_t)TOKENS, a.num_tokens - t0);
  for (int x = threadIdx.x; x < nt * pairs; x += kThreads) {
    const int pos = a.positions[t0 + x / pairs];
    if (pos >= 0) turns[x / pairs][x % pairs] = turn(a.rot, pos, x % pairs);
  }
  __syncthreads();
  const int units = R / 16;                           // of 8 pairs
  const int per_head = units + (a.head_dim - R) / 8;  // and vectors of 8 that are copied
  const int heads = a.q.heads + a.k.heads;
  for (int x = threadIdx.x; x < nt * heads * per_head; x += kThreads) {
    const int u = x % per_head;
    const int hx = x / per_head % heads;
    const int t = x / per_head / heads;
    if (a.positions[t0 + t] < 0) continue;
    const bool is_q = hx < a.q.heads;
    const RotaryRows& r = is_q ? a.q : a.k;
    const int h = is_q ? hx : hx - a.q.heads;
    const T* in = static_cast<const T*>(r.in) + (int64_t)(t0 + t) * r.in_stride + (int64_t)h * a.head_dim;
    T* out = static_cast<T*>(r.out) + (int64_t)(t0 + t) * r.out_stride + (int64_t)h * a.head_dim;
    float p[8], q[8];
    if (u >= units) {
      const int d = R + 8 * (u - units);
      if (r.in == r.out) continue;
      load8(in + d, p);
      store8(out + d, p);
      continue;
    }
    const int d0 = a.rot.interleaved ? 16 * u : 8 * u;
    const int d1 = a.rot.interleaved ? d0 + 8 : d0 + pairs;
    load8(in + d0, p);
    load8(in + d1, q);
    const float2* cs = &turns[t][8 * u];
    if (a.rot.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 c0 = cs[i / 2], c1 = cs[4 + i / 2];
        const float x0 = p[i], y0 = p[i + 1], x1 = q[i], y1 = q[i + 1];
        p[i] = x0 * c0.x - y0 * c0.y, p[i + 1] = y0 * c0.x + x0 * c0.y;
        q[i] = x1 * c1.x - y1 * c1.y, q[i + 1] = y1 * c1.x + x1 * c1.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 c = cs[i];
        const float x0 = p[i], y0 = q[i];
        p[i] = x0 * c.x - y0 * c.y, q[i] = y0 * c.x + x0 * c.y;
      }
    }
    store8(out + d0, p);
    store8(out + d1, q);
  }
  __syncthreads();  // the next tokens' turns take the same place
  }
}

template <typename T>
hipError_t launch_t(const RotaryApplyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((rotary_kernel<T, 1>), dim3(min(a.num_tokens, kMaxGrid)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryApplyArgs& a, int dtype, hipStream_t stream) {
  return dtype == PDA_DTYPE_BF16 ? launch_t<__bf16>(a, stream) : launch_t<float>(a, stream);
}

}  // namespace pda
