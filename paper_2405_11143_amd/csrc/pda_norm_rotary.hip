// Head norms, rotary positions with several axes, the append through a slot map and the
// gradient of the norms (include/pda_norm_rotary.h).
//
// All bound by memory: a row is read and written once (the gradient reads two).  As in
// pda_rotary.hip a workgroup takes a token, forms the cosines and sines of its
// positions in LDS, and then its rows, 16 elements per thread; a row's U threads are
// neighbouring lanes, so its sum of squares is a few DPP steps.  A thread has two rows
// in flight, loaded before the angles are formed.
#include "pda_norm_rotary_internal.h"

namespace pda {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesHere = kThreads / kWaveSize;
constexpr int kMaxGrid = 1 << 20;  // workgroups (a launch has less than 2^32 threads); they loop over the rest
constexpr int kMaxDim = 512;
constexpr int kXcds = 8;

// 8 elements as they lie in memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<__bf16> {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  v8 x;
  __device__ __forceinline__ void load(const __bf16* p) { x = *reinterpret_cast<const v8*>(p); }
  __device__ __forceinline__ void floats(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)x[i];
  }
};
template <>
struct Raw8<float> {
  f32x4_t x[2];
  __device__ __forceinline__ void load(const float* p) {
    x[0] = reinterpret_cast<const f32x4_t*>(p)[0], x[1] = reinterpret_cast<const f32x4_t*>(p)[1];
  }
  __device__ __forceinline__ void floats(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i / 4][i % 4];
  }
};

// The sum over the U neighbouring lanes of a row, the same bits in each.
template <int U>
__device__ __forceinline__ float row_sum(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x += dpp(x, std::integral_constant<int, 0xb1>());              // quad_perm [1, 0, 3, 2]
  x += dpp(x, std::integral_constant<int, 0x4e>());              // quad_perm [2, 3, 0, 1]
  if (U >= 8) x += dpp(x, std::integral_constant<int, 0x141>()); // the other four of 8
  if (U >= 16) x += dpp(x, std::integral_constant<int, 0x140>());// the other eight of 16
  if (U >= 32) x += __shfl_xor(x, 16);
  return x;
}

// A thread's share of every row: as in pda_rotary.hip, or none at all for the lanes that fill
// U up.
__device__ __forceinline__ RowShare share_of(const RotaryArgs& r, int rotary_dim, int D, int u) {
  return u < row_shares(D) ? row_share(r, rotary_dim, D, u) : RowShare{D, D, 0};
}

template <typename T>
struct RawShare {
  Raw8<T> p, q;
  __device__ __forceinline__ void load(const T* row, const RowShare& w, int D) {
    if (w.d0 < D) p.load(row + w.d0);
    if (w.d1 < D) q.load(row + w.d1);
  }
  // (what the lane does not have counts as zeros)
  __device__ __forceinline__ void floats(const RowShare& w, int D, float (&x)[8], float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.f;
    if (w.d0 < D) p.floats(x);
    if (w.d1 < D) q.floats(y);
  }
};

// The lane's 16 weights of a norm, the offset added.
__device__ __forceinline__ void load_weights(const NormRotaryArgs& a, int which, const RowShare& w, float (&x)[16]) {
  const int D = a.head_dim;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 1.f;
  const void* p = a.weight[which];
  if (!p) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int d = h ? w.d1 : w.d0;
    if (d >= D) continue;
    float y[8];
    if (a.weight_f32)
      load8(static_cast<const float*>(p) + d, y);
    else
      load8(static_cast<const __bf16*>(p) + d, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[8 * h + i] = y[i] + a.offset;
  }
}

// cos and sin of pair x of token t, whose position on the first axis is pos.
__device__ __forceinline__ float2 turn_of(const NormRotaryArgs& a, int64_t t, int pos, int x) {
  if (a.axis) {
    const int axis = a.axis[x];
    if (axis > 0 && axis < a.num_axes) pos = a.positions[axis * a.position_stride + t];
  }
  return turn(a.rot, pos, x);
}

// What a row of the launch is.
enum RowKind { kQuery = 0, kKey = 1, kValue = 2 };

// U: lanes per row.  NORM: the rows are normed.  STORE: keys and values go to the cache.  NT: the
// queries go out with the non-temporal hint (and, without STORE, the keys).
template <typename T, int U, bool NORM, bool STORE, bool NT>
__global__ void __launch_bounds__(kThreads) norm_rotary_kernel(const NormRotaryArgs a) {
  __shared__ float2 turns[kMaxDim / 2];
  const int D = a.head_dim;
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  const int u = threadIdx.x % U;
  const int rows_at_once = blockDim.x / U;
  const RowShare rotated = share_of(a.rot, R, D, u), plain = share_of(a.rot, 0, D, u);
  const int nq = a.q.heads, nk = a.k.heads;
  const int rows = nq + (STORE ? 2 : 1) * nk;
  auto kind = [&](int h) { return h < nq ? kQuery : !STORE || h < nq + nk ? kKey : kValue; };
  auto share = [&](int h) { return STORE && kind(h) == kValue ? plain : rotated; };
  float wq[16], wk[16];
  if (NORM) {
    load_weights(a, 0, rotated, wq);
    load_weights(a, 1, rotated, wk);
  }
  const float inv_d = 1.f / (float)D;
  for (int64_t x = blockIdx.x; x < a.num_tokens; x += gridDim.x) {
    int64_t t = x;
    if (STORE) {
      // 16 neighbouring tokens, which fill whole lines of a block's keys together, on one XCD
      const int64_t whole = a.num_tokens / (16 * kXcds) * (16 * kXcds);
      if (x < whole) t = ((x / kXcds) / 16 * kXcds + x % kXcds) * 16 + (x / kXcds) % 16;
    }
    const int pos = a.positions[t];
    if (pos < 0) continue;  // padding (the whole workgroup)
    const int slot = STORE ? a.slots[t] : 0;
    const bool stores = (unsigned)slot < 16u * (unsigned)a.num_blocks;
    auto load = [&](int h, RawShare<T>& raw) {
      const int which = kind(h);
      const T* in = which == kQuery ? static_cast<const T*>(a.q.in) + t * a.q.in_stride + (int64_t)h * D
                    : which == kKey ? static_cast<const T*>(a.k.in) + t * a.k.in_stride + (int64_t)(h - nq) * D
                                    : reinterpret_cast<const T*>(a.v) + t * a.v_stride + (int64_t)(h - nq - nk) * D;
      raw.load(in, share(h), D);
    };
    auto finish = [&](int h, const RawShare<T>& raw) {
      const int which = kind(h);
      const RowShare w = share(h);
      float p[8], q[8];
      raw.floats(w, D, p, q);
      if (NORM) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(p[e], p[e], fmaf(q[e], q[e], s));
        const float r = rsqrtf(fmaf(row_sum<U>(s), inv_d, a.eps));
        if (!STORE || which != kValue) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] *= r * (which == kQuery ? wq[e] : wk[e]);
            q[e] *= r * (which == kQuery ? wq[8 + e] : wk[8 + e]);
          }
        }
      }
      rotate_share(turns, a.rot.interleaved, w, p, q);
      if (STORE && which != kQuery) {
        if (!stores) return;
        const size_t tile = (size_t)(slot / kBlockTokens) * nk;
        const int o = slot % kBlockTokens;
        const size_t g = tile + (which == kKey ? h - nq : h - nq - nk);
        __bf16* dst = reinterpret_cast<__bf16*>(which == kKey ? a.k_cache : a.v_cache);
        auto at = [&](int d) { return which == kKey ? ((g * (D / 8) + d / 8) * kBlockTokens + o) * 8 : (g * kBlockTokens + o) * D + d; };
        if (w.d0 < D) store8<false>(dst + at(w.d0), p);
        if (w.d1 < D) store8<false>(dst + at(w.d1), q);
        return;
      }
      T* out = which == kQuery ? static_cast<T*>(a.q.out) + t * a.q.out_stride + (int64_t)h * D
                               : static_cast<T*>(a.k.out) + t * a.k.out_stride + (int64_t)(h - nq) * D;
      if (w.d0 < D) store8<NT>(out + w.d0, p);
      if (w.d1 < D) store8<NT>(out + w.d1, q);
    };
    RawShare<T> first, second;
    int h = threadIdx.x / U;
    if (h >= rows_at_once) h = rows;
    if (h < rows) load(h, first);
    if (h + rows_at_once < rows) load(h + rows_at_once, second);
    for (int i = threadIdx.x; i < R / 2; i += blockDim.x) turns[i] = turn_of(a, t, pos, i);
    __syncthreads();
    while (h < rows) {  // (all lanes of a row together)
      finish(h, first);
      if (h + rows_at_once < rows) finish(h + rows_at_once, second);
      h += 2 * rows_at_once;
      if (h < rows) load(h, first);
      if (h + rows_at_once < rows) load(h + rows_at_once, second);
    }
    __syncthreads();  // the next token's turns take the same place
  }
}

// The gradient.  Every thread sums its elements' h u over its rows and tokens; at the end
// the wavefronts' rows are summed by shuffles, the wavefronts through LDS.
template <typename T, int U>
__global__ void __launch_bounds__(kThreads) norm_rotary_grad_kernel(const NormRotaryArgs a) {
  __shared__ float2 turns[kMaxDim / 2];
  __shared__ float sums[kWavesHere][2][kMaxDim];
  const int D = a.head_dim;
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  const int u = threadIdx.x % U;
  const int rows_at_once = blockDim.x / U;
  const RowShare w = share_of(a.rot, R, D, u);
  const int nq = a.q.heads, rows = nq + a.k.heads;
  float wq[16], wk[16], dwq[16], dwk[16];
  load_weights(a, 0, w, wq);
  load_weights(a, 1, w, wk);
#pragma unroll
  for (int e = 0; e < 16; ++e) dwq[e] = dwk[e] = 0.f;
  const float inv_d = 1.f / (float)D;
  for (int64_t t = blockIdx.x; t < a.num_tokens; t += gridDim.x) {
    const int pos = a.positions[t];
    if (pos < 0) continue;  // padding (the whole workgroup)
    for (int i = threadIdx.x; i < R / 2; i += blockDim.x) turns[i] = turn_of(a, t, pos, i);
    __syncthreads();
    for (int h = threadIdx.x / U; h < rows; h += rows_at_once) {  // (all lanes of a row together)
      const bool is_q = h < nq;
      const RotaryRows& xr = is_q ? a.q : a.k;
      const RotaryRows& gr = is_q ? a.q_grad : a.k_grad;
      const int64_t at = (int64_t)(is_q ? h : h - nq) * D;
      RawShare<T> xs, gs;
      xs.load(static_cast<const T*>(xr.in) + t * xr.in_stride + at, w, D);
      gs.load(static_cast<const T*>(gr.in) + t * gr.in_stride + at, w, D);
      float p[8], q[8], gp[8], gq[8];
      xs.floats(w, D, p, q);
      gs.floats(w, D, gp, gq);
      rotate_share(turns, a.rot.interleaved, w, gp, gq);
      float ss = 0.f, gx = 0.f;  // sums of x^2 and of f x
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss = fmaf(p[e], p[e], fmaf(q[e], q[e], ss));
        gx = fmaf(gp[e] * (is_q ? wq[e] : wk[e]), p[e], fmaf(gq[e] * (is_q ? wq[8 + e] : wk[8 + e]), q[e], gx));
      }
      const float r = rsqrtf(fmaf(row_sum<U>(ss), inv_d, a.eps));
      const float c = row_sum<U>(gx) * r * inv_d;  // mean of f u
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float up = p[e] * r, uq = q[e] * r;
        const float hp = gp[e] * up, hq = gq[e] * uq;
        dwq[e] += is_q ? hp : 0.f, dwq[8 + e] += is_q ? hq : 0.f;
        dwk[e] += is_q ? 0.f : hp, dwk[8 + e] += is_q ? 0.f : hq;
        p[e] = r * fmaf(-up, c, gp[e] * (is_q ? wq[e] : wk[e]));
        q[e] = r * fmaf(-uq, c, gq[e] * (is_q ? wq[8 + e] : wk[8 + e]));
      }
      T* out = static_cast<T*>(xr.out) + t * xr.out_stride + at;
      if (w.d0 < D) store8<false>(out + w.d0, p);
      if (w.d1 < D) store8<false>(out + w.d1, q);
    }
    __syncthreads();  // the next token's turns take the same place
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int m = U; m < kWaveSize; m <<= 1) {
      dwq[e] += __shfl_xor(dwq[e], m);
      dwk[e] += __shfl_xor(dwk[e], m);
    }
  const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
  if (lane < U) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int d = (e < 8 ? w.d0 : w.d1) + e % 8;
      if (d < D) sums[wave][0][d] = dwq[e], sums[wave][1][d] = dwk[e];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += blockDim.x) {
    float s = 0.f;
    for (int x = 0; x < (int)blockDim.x / kWaveSize; ++x) s += sums[x][i / D][i % D];
    a.part[(size_t)blockIdx.x * 2 * D + i] = s;
  }
}

// The weights' gradients from the workgroups' partial sums, in a fixed order: 8 columns to a
// workgroup, 32 runs of partial sums beside each other.
constexpr int kSumColumns = 8;
__global__ void __launch_bounds__(kThreads) weight_grad_kernel(const float* part, int groups, int D, float* dq, float* dk) {
  __shared__ float s[kThreads / kSumColumns][kSumColumns];
  const int c = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns, run = threadIdx.x / kSumColumns;
  float x = 0.f;
  for (int i = run; i < groups; i += kThreads / kSumColumns) x += part[(size_t)i * 2 * D + c];
  s[run][threadIdx.x % kSumColumns] = x;
  __syncthreads();
  if (run == 0) {
    for (int i = 1; i < kThreads / kSumColumns; ++i) x += s[i][threadIdx.x];
    float* out = c < D ? dq : dk;
    if (out) out[c < D ? c : c - D] = x;
  }
}

// A workgroup has as many threads as make its last trip through the rows a full one, nearly.
int threads_for(int rows, int U) {
  const int64_t units = (int64_t)rows * U;
  const int64_t trips = (units + kThreads - 1) / kThreads;
  return (int)min((int64_t)kThreads, ((units + trips - 1) / trips + kWaveSize - 1) / kWaveSize * kWaveSize);
}

// f(integral_constant U): the lanes that a row of head_dim elements takes.
template <typename F>
void with_lanes(int head_dim, F&& f) {
  const int shares = row_shares(head_dim);
  if (shares <= 4)
    f(std::integral_constant<int, 4>());
  else if (shares <= 8)
    f(std::integral_constant<int, 8>());
  else if (shares <= 16)
    f(std::integral_constant<int, 16>());
  else
    f(std::integral_constant<int, 32>());
}

template <typename T, bool NORM>
void launch_apply(const NormRotaryArgs& a, hipStream_t stream) {
  const dim3 grid(min(a.num_tokens, kMaxGrid));
  with_lanes(a.head_dim, [&](auto lanes) {
    constexpr int U = decltype(lanes)::value;
    const dim3 threads(threads_for(a.q.heads + a.k.heads, U));
    if constexpr (sizeof(T) == 2) {
      if (a.num_tokens >= kManyTokens && whole_lines(a.rot, a.head_dim)) {
        hipLaunchKernelGGL((norm_rotary_kernel<T, U, NORM, false, true>), grid, threads, 0, stream, a);
        return;
      }
    }
    hipLaunchKernelGGL((norm_rotary_kernel<T, U, NORM, false, false>), grid, threads, 0, stream, a);
  });
}

}  // namespace

hipError_t launch_norm_rotary(const NormRotaryArgs& a, int dtype, hipStream_t stream) {
  if (dtype == PDA_DTYPE_BF16)
    a.normed ? launch_apply<__bf16, true>(a, stream) : launch_apply<__bf16, false>(a, stream);
  else
    a.normed ? launch_apply<float, true>(a, stream) : launch_apply<float, false>(a, stream);
  return hipGetLastError();
}

hipError_t launch_norm_rotary_append(const NormRotaryArgs& a, hipStream_t stream) {
  const dim3 grid(min(a.num_tokens, kMaxGrid));
  const bool nt = a.num_tokens >= kManyTokens && whole_lines(a.rot, a.head_dim);
  with_lanes(a.head_dim, [&](auto lanes) {
    constexpr int U = decltype(lanes)::value;
    if constexpr (U <= 8) {  // head_dim 64 and 128
      const dim3 threads(threads_for(a.q.heads + 2 * a.k.heads, U));
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a); };
      if (a.normed)
        nt ? launch(norm_rotary_kernel<__bf16, U, true, true, true>) : launch(norm_rotary_kernel<__bf16, U, true, true, false>);
      else
        nt ? launch(norm_rotary_kernel<__bf16, U, false, true, true>) : launch(norm_rotary_kernel<__bf16, U, false, true, false>);
    }
  });
  return hipGetLastError();
}

hipError_t launch_norm_rotary_backward(const NormRotaryArgs& a, int dtype, hipStream_t stream) {
  const int groups = grad_groups(a.num_tokens);
  if (groups > 0)
    with_lanes(a.head_dim, [&](auto lanes) {
      constexpr int U = decltype(lanes)::value;
      const dim3 threads(threads_for(a.q.heads + a.k.heads, U));
      if (dtype == PDA_DTYPE_BF16)
        hipLaunchKernelGGL((norm_rotary_grad_kernel<__bf16, U>), dim3(groups), threads, 0, stream, a);
      else
        hipLaunchKernelGGL((norm_rotary_grad_kernel<float, U>), dim3(groups), threads, 0, stream, a);
    });
  if (a.d_weight[0] || a.d_weight[1])
    hipLaunchKernelGGL(weight_grad_kernel, dim3(2 * a.head_dim / kSumColumns), dim3(kThreads), 0, stream, a.part, groups,
                       a.head_dim, a.d_weight[0], a.d_weight[1]);
  return hipGetLastError();
}

}  // namespace pda
