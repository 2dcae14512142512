// Head norms, rotary positions with several axes, the append through a slot map and the
// gradient of the norms (include/pda_norm_rotary.h).
//
// All bound by memory: a row is read and written once (the gradient reads two).  A
// wavefront takes a token, or with few tokens a part of one: it forms the cosines and sines of its
// positions in its own corner of LDS, and then takes the rows, 64 / U at a time, 16 elements
// per lane; a row's U lanes are neighbours, so its sum of squares is a few DPP steps.  The rows
// of two steps are in flight, the first two loaded before the angles are formed.
// Nothing waits for another wavefront.
//
// Measured, bf16 (a copy of 1 GiB runs at 5.1 TB/s here): 16384 tokens of 32 + 8 heads of 128, with
// norms, 59 us, 5.6 TB/s; their gradient 100 us, 4.9 TB/s; 26000 tokens of 28 + 4 heads with their
// values into the cache 96 us, 5.0 TB/s; 6000 tokens of 28 + 4 heads, three axes, rotation alone, 22.3 us
// (17.8 with rows that the last-level cache holds); 4097 of 16 + 16 heads of 64 in fp32, two axes,
// turned back, 18.8 us (16.1); 256 tokens of a decode step into the cache 5.1 us, of which the launch is 4.4.
// The gradient in fp32, 16384 of 32 + 8, 199 us, 5.1 TB/s; of 16 + 16 heads of 80 116 us (floor 99), in bf16 80 (49),
// the forward 44 (33): 5 of a row's 8 lanes have elements.
//
// Tokens of few heads are furthest from the bytes: a step's rows are of one kind and one token, so 8 + 2 heads
// of 64 fill 10 of 32 places, with values 12 of 48.  60000 tokens of them 53 us (floor 30), 54000 into the cache 77 (32);
// of 4 + 1 heads of 128 51 and 76.
//
// The rotation alone on one axis is what rotary_kernel (pda_rotary.hip) does, and that is the faster there:
// 16384 tokens of 32 + 8 heads 61 us here and 60 there, 6000 of 28 + 4 17.5 and 16.7, 60000 of 8 + 2 of 64 49 and 36.
#include <algorithm>
#include <type_traits>

#include "pda_norm_rotary_internal.h"

namespace pda {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesHere = kThreads / kWaveSize;
constexpr int kMaxGrid = 1 << 20;  // workgroups (a launch has less than 2^32 threads); they loop over the rest
constexpr int kMaxDim = 512;
constexpr int kXcds = 8;
constexpr int kComputeUnits = 256;
constexpr int kFewWaves = 4096;  // wavefronts that fewer tokens are split into
// From so many tokens on, rows of whole cache lines go out with the non-temporal hint.  32 + 8 heads of 128,
// us, without / with: 256 tokens 5.0 / 5.0, 512 5.4 / 4.9, 1024 7.2 / 6.2, 1500 9.1 / 7.6, 2500 13.8 / 10.6, 16384 65.2
// / 59.2; into the cache 26000 of 28 + 4 101.7 / 96.0.  The line is that of the call alone: a kernel behind it that
// reads the rows finds fewer of them in the caches, and from about 2000 tokens on loses what the hint gains, or more.
// With one that reads the queries, the two take 9.0 / 8.9 for 512, 13.0 / 11.7 for 1024, 18.2 / 18.4 for 2048,
// 20.5 / 22.0 for 3000, 53.2 / 55.4 for 8192, 107 / 110 for 16384; the append with attention over a window of 64
// behind it 25.7 / 25.2 for 1024, 45.0 / 47.3 for 3000, 104 / 109 for 8192, 208 / 212 for 16384; the gradient with a
// product over its rows 27.0 / 26.8 for 1024, 47.6 / 50.5 for 3000, 98 / 104 for 8192, 199 / 205 for 16384.
constexpr int kHintTokens = 512;

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

// What a lane has of every row: 16 elements as in pda_rotary.hip, or nothing (lanes that fill U up);
// with the cosines and sines of the token at hand for them.
struct Share {
  int d0, d1, turned, D;
  bool interleaved;
  float c[8], s[8];  // half layout: of pair d0 + e; neighbouring pairs: of d0 / 2 + e and of d1 / 2 + e - 4

  __device__ __forceinline__ Share(const RotaryArgs& r, int R, int D_, int u) : D(D_), interleaved(r.interleaved) {
    const RowShare w = u < row_shares(D) ? row_share(r, R, D, u) : RowShare{D, D, 0};
    d0 = w.d0, d1 = w.d1, turned = w.turned;
  }
  __device__ __forceinline__ void read(const float2* turns) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (turned == 0) continue;
      if (interleaved && e >= 4 && turned < 2) continue;
      const float2 t = turns[interleaved ? (e < 4 ? d0 / 2 + e : d1 / 2 + e - 4) : d0 + e];
      c[e] = t.x, s[e] = t.y;
    }
  }
  // Turns the lane's elements.
  __device__ __forceinline__ void turn(float (&x)[8], float (&y)[8]) const {
    if (turned == 0) return;
    auto pair = [&](float& a, float& b, int e) {
      const float t = a;
      a = t * c[e] - b * s[e], b = b * c[e] + t * s[e];
    };
    if (interleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e) pair(x[2 * e], x[2 * e + 1], e);
      if (turned == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) pair(y[2 * e], y[2 * e + 1], 4 + e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) pair(x[e], y[e], e);
    }
  }
};

// A lane's elements of a row, as they lie in memory.  FULL: every lane has both vectors.
template <typename T, bool FULL>
struct RawShare {
  Raw8<T> p, q;
  // (`at` is the wavefront's, the byte offsets the lane's)
  __device__ __forceinline__ void load(const char* at, bool has0, unsigned o0, bool has1, unsigned o1) {
    if (FULL || has0) p.load(reinterpret_cast<const T*>(at + o0));
    if (FULL || has1) q.load(reinterpret_cast<const T*>(at + o1));
  }
  // (what the lane does not have counts as zeros)
  __device__ __forceinline__ void floats(bool has0, bool has1, float (&x)[8], float (&y)[8]) const {
    if (!FULL) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.f;
    }
    if (FULL || has0) p.floats(x);
    if (FULL || has1) q.floats(y);
  }
};

// The norms' weights of queries and of keys, the offset added, as fp32 in LDS.
__device__ __forceinline__ void load_weights(const NormRotaryArgs& a, float (*weights)[kMaxDim]) {
  for (int i = threadIdx.x; i < 2 * a.head_dim; i += blockDim.x) {
    const int k = i < a.head_dim ? 0 : 1, d = i - k * a.head_dim;
    const void* p = k == 0 ? a.weight[0] : a.weight[1];
    float x = 1.f;
    if (p) x = (a.weight_f32 ? static_cast<const float*>(p)[d] : (float)static_cast<const __bf16*>(p)[d]) + a.offset;
    weights[k][d] = x;
  }
  __syncthreads();
}

// LDS that the wavefront's lanes have written is theirs to read, and the other way round.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The cosine and sine of every pair of token t, whose position on the first axis is pos, into the
// wavefront's corner of LDS.
__device__ __forceinline__ void form_turns(const NormRotaryArgs& a, int R, int64_t t, int pos, float2* turns) {
  for (int i = threadIdx.x % kWaveSize; i < R / 2; i += kWaveSize) {
    int p = pos;
    if (a.axis) {
      const int axis = a.axis[i];
      if (axis > 0 && axis < a.num_axes) p = a.positions[axis * a.position_stride + t];
    }
    turns[i] = turn(a.rot, p, i);
  }
  wave_sync();
}

// A token's rows are taken by wavefronts, 64 / U of one kind at a time, so that what kind they
// are, and where they lie, is the same for the wavefront.
enum RowKind { kQuery = 0, kKey = 1, kValue = 2 };
struct RowStep {
  int kind, first;  // first head
};
__device__ __forceinline__ RowStep row_step(int i, int q_steps, int k_steps) {
  const int kind = i < q_steps ? kQuery : i < q_steps + k_steps ? kKey : kValue;
  return RowStep{kind, i - (kind == kQuery ? 0 : kind == kKey ? q_steps : q_steps + k_steps)};
}

// U: lanes per row.  FULL: head_dim is 16 U.  NORM: the rows are normed.  STORE: keys and values go to the cache.  NT: the
// queries go out with the non-temporal hint (and, without STORE, the keys).  `parts` wavefronts
// share a token.
template <typename T, int U, bool FULL, bool NORM, bool STORE, bool NT>
__global__ void __launch_bounds__(kThreads) norm_rotary_kernel(const NormRotaryArgs a, int parts) {
  constexpr int RPW = kWaveSize / U;  // rows of a step
  __shared__ float2 all_turns[kWavesHere][kMaxDim / 2];
  __shared__ __align__(16) float weights[NORM ? 2 : 1][kMaxDim];
  if constexpr (NORM) load_weights(a, weights);
  const int D = FULL ? 16 * U : a.head_dim;
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  const int lane = threadIdx.x % kWaveSize, u = lane % U, row = lane / U;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
  float2* const turns = all_turns[wave];
  Share w(a.rot, R, D, u);
  const int shares = row_shares(D);
  const int v0 = 8 * u, v1 = 8 * (u + shares);  // of a row of values (STORE: every lane has both)
  const int nq = a.q.heads, nk = a.k.heads;
  const int q_steps = (nq + RPW - 1) / RPW, k_steps = (nk + RPW - 1) / RPW;
  const int steps = q_steps + (STORE ? 2 : 1) * k_steps;
  const float inv_d = 1.f / (float)D;
  const int d0 = w.d0, d1 = w.d1;
  const bool has0 = d0 < D, has1 = d1 < D;
  const unsigned row_at = row * D * (unsigned)sizeof(T);
  for (int64_t x = (int64_t)blockIdx.x * kWavesHere + wave; x < (int64_t)a.num_tokens * parts;
       x += (int64_t)gridDim.x * kWavesHere) {
    int64_t t = x;
    int part = 0;
    if (parts > 1) {
      t = (uint64_t)x >> 32 ? x / parts : (uint32_t)x / (uint32_t)parts;
      part = (int)(x - t * parts);
    } else if (STORE) {
      // 16 neighbouring tokens, which fill whole lines of a block's keys together, on one XCD: 4
      // workgroups, 8 numbers apart
      constexpr int kRun = 16 * kXcds;
      if (x < a.num_tokens / kRun * kRun) {
        const int in = (int)(x % kRun), group = in / kWavesHere;
        t = x - in + group % kXcds * 16 + group / kXcds * kWavesHere + in % kWavesHere;
      }
    }
    const int pos = a.positions[t];
    if (pos < 0) continue;  // padding
    const int slot = STORE ? a.slots[t] : 0;
    const uint64_t q_at = (uint64_t)(static_cast<const T*>(a.q.in) + t * a.q.in_stride);
    const uint64_t k_at = (uint64_t)(static_cast<const T*>(a.k.in) + t * a.k.in_stride);
    const uint64_t v_at = STORE ? (uint64_t)(reinterpret_cast<const T*>(a.v) + t * a.v_stride) : 0;
    auto load = [=](int i, RawShare<T, FULL>& raw) __attribute__((always_inline)) {
      if (i >= steps) return;
      const RowStep s = row_step(i, q_steps, k_steps);
      const int h = s.first * RPW + row;
      const bool is_v = STORE && s.kind == kValue;
      // (by arithmetic: selects of captured values would keep them in memory)
      const int k = s.kind != kQuery, v = is_v;
      const uint64_t at = q_at + k * (k_at - q_at) + v * (v_at - k_at) + s.first * (RPW * D * (int)sizeof(T));
      if (h < nq + k * (nk - nq))
        raw.load(reinterpret_cast<const char*>(at), has0, row_at + (d0 + v * (v0 - d0)) * (unsigned)sizeof(T), has1,
                 row_at + (d1 + v * (v1 - d1)) * (unsigned)sizeof(T));
    };
    // A step's rows; `next` is loaded into its place.  Loads go out before the stores: waiting for a load waits
    // for every store before it, too (16384 tokens of 32 + 8 heads 80 us with the loads behind, 63 so).
    auto finish = [&](int i, RawShare<T, FULL>& raw, int next) __attribute__((always_inline)) {
      if (i >= steps) return;
      const RowStep s = row_step(i, q_steps, k_steps);
      const int h = s.first * RPW + row;
      const bool is_v = STORE && s.kind == kValue, is_q = s.kind == kQuery;
      const RawShare<T, FULL> now = raw;
      float p[8], q[8];
      now.floats(has0, has1, p, q);
      load(next, raw);
      __builtin_amdgcn_sched_barrier(0);
      if (h >= (is_q ? nq : nk)) return;  // (all lanes of a row together)
      if constexpr (STORE) {
        if (is_v) {
          if ((unsigned)slot >= 16u * (unsigned)a.num_blocks) return;
          char* at = reinterpret_cast<char*>(a.v_cache) +
                     (((size_t)(slot / kBlockTokens) * nk + s.first * RPW) * kBlockTokens + slot % kBlockTokens) * (D * 2);
          *reinterpret_cast<decltype(raw.p.x)*>(at + (row_at * kBlockTokens + v0 * 2u)) = now.p.x;
          *reinterpret_cast<decltype(raw.q.x)*>(at + (row_at * kBlockTokens + v1 * 2u)) = now.q.x;
          return;
        }
      }
      if constexpr (NORM) {
        const float* wt = weights[is_q ? 0 : 1];
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(p[e], p[e], fmaf(q[e], q[e], ss));
        const float r = rsqrtf(fmaf(row_sum<U>(ss), inv_d, a.eps));
        const int w0 = FULL ? d0 : min(d0, D - 8), w1 = FULL ? d1 : min(d1, D - 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] *= r * wt[w0 + e], q[e] *= r * wt[w1 + e];
      }
      w.turn(p, q);
      if (STORE && !is_q) {
        if ((unsigned)slot >= 16u * (unsigned)a.num_blocks) return;
        char* at = reinterpret_cast<char*>(a.k_cache) +
                   ((size_t)(slot / kBlockTokens) * nk + s.first * RPW) * (D * kBlockTokens * 2) + slot % kBlockTokens * 16;
        store8<false>(reinterpret_cast<__bf16*>(at + (row_at + d0 * 2u) * kBlockTokens), p);
        store8<false>(reinterpret_cast<__bf16*>(at + (row_at + d1 * 2u) * kBlockTokens), q);
        return;
      }
      char* out = reinterpret_cast<char*>(is_q ? static_cast<T*>(a.q.out) + t * a.q.out_stride : static_cast<T*>(a.k.out) + t * a.k.out_stride) +
                  s.first * (RPW * D * (int)sizeof(T));
      if (FULL || has0) store8<NT>(reinterpret_cast<T*>(out + (row_at + d0 * (unsigned)sizeof(T))), p);
      if (FULL || has1) store8<NT>(reinterpret_cast<T*>(out + (row_at + d1 * (unsigned)sizeof(T))), q);
    };
    RawShare<T, FULL> first, second;
    load(part, first);
    load(part + parts, second);
    form_turns(a, R, t, pos, turns);
    w.read(turns);
    for (int i = part; i < steps; i += 2 * parts) {
      finish(i, first, i + 2 * parts);
      finish(i + parts, second, i + 3 * parts);
    }
    wave_sync();  // the next token's turns take the same place
  }
}

// The gradient.  Every lane sums its elements' h u over its rows and tokens; at the end
// the wavefront's rows are summed by shuffles, the wavefronts through LDS.  One step's rows are in flight
// and three wavefronts share a SIMD: 104 us for 16384 tokens of 32 + 8 heads of 128; with two steps in
// flight 116, with four wavefronts 139.  NT: the rows go out with the non-temporal hint: 100, 1500 tokens 19.9 -> 18.1.
template <typename T, int U, bool FULL, bool NT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3)))
norm_rotary_grad_kernel(const NormRotaryArgs a, int parts) {
  constexpr int RPW = kWaveSize / U;
  __shared__ union {
    float2 turns[kWavesHere][kMaxDim / 2];
    float sums[kWavesHere][2][kMaxDim];
  } lds;
  __shared__ __align__(16) float weights[2][kMaxDim];
  __shared__ f32x4_t key_sums[kWavesHere][4][kWaveSize];
  load_weights(a, weights);
  const int D = FULL ? 16 * U : a.head_dim;
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  const int lane = threadIdx.x % kWaveSize, u = lane % U, row = lane / U;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
  float2* const turns = lds.turns[wave];
  Share w(a.rot, R, D, u);
  const int nq = a.q.heads, nk = a.k.heads;
  const int q_steps = (nq + RPW - 1) / RPW, steps = q_steps + (nk + RPW - 1) / RPW;
  float dw[16];  // of queries; of keys, in LDS: with both in registers the kernel spills
#pragma unroll
  for (int e = 0; e < 16; ++e) dw[e] = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) key_sums[wave][x][lane] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const float inv_d = 1.f / (float)D;
  const int d0 = w.d0, d1 = w.d1;
  const bool has0 = d0 < D, has1 = d1 < D;
  const unsigned row_at = row * D * (unsigned)sizeof(T);
  for (int64_t x = (int64_t)blockIdx.x * kWavesHere + wave; x < a.num_tokens * (int64_t)parts;
       x += (int64_t)gridDim.x * kWavesHere) {
    int64_t t = x;
    int part = 0;
    if (parts > 1) {
      t = (uint32_t)x / (uint32_t)parts;  // (few tokens)
      part = (int)(x - t * parts);
    }
    const int pos = a.positions[t];
    if (pos < 0) continue;  // padding
    const uint64_t q_at = (uint64_t)(static_cast<const T*>(a.q.in) + t * a.q.in_stride);
    const uint64_t k_at = (uint64_t)(static_cast<const T*>(a.k.in) + t * a.k.in_stride);
    const uint64_t qg_at = (uint64_t)(static_cast<const T*>(a.q_grad.in) + t * a.q_grad.in_stride);
    const uint64_t kg_at = (uint64_t)(static_cast<const T*>(a.k_grad.in) + t * a.k_grad.in_stride);
    auto load = [=](int i, RawShare<T, FULL>& xs, RawShare<T, FULL>& gs) __attribute__((always_inline)) {
      if (i >= steps) return;
      const int k = i >= q_steps, first = i - k * q_steps;
      if (first * RPW + row >= nq + k * (nk - nq)) return;
      const int skip = first * (RPW * D * (int)sizeof(T));
      const unsigned o0 = row_at + d0 * (unsigned)sizeof(T), o1 = row_at + d1 * (unsigned)sizeof(T);
      xs.load(reinterpret_cast<const char*>(q_at + k * (k_at - q_at) + skip), has0, o0, has1, o1);
      gs.load(reinterpret_cast<const char*>(qg_at + k * (kg_at - qg_at) + skip), has0, o0, has1, o1);
    };
    auto finish = [&](int i, RawShare<T, FULL>& xs, RawShare<T, FULL>& gs, int next) __attribute__((always_inline)) {  // (as above)
      if (i >= steps) return;
      const bool is_q = i < q_steps;
      const int h = (is_q ? i : i - q_steps) * RPW + row;
      float p[8], q[8], gp[8], gq[8];
      xs.floats(has0, has1, p, q);
      gs.floats(has0, has1, gp, gq);
      load(next, xs, gs);
      __builtin_amdgcn_sched_barrier(0);
      if (h >= (is_q ? nq : nk)) return;  // (all lanes of a row together)
      float wp[8], wq[8];
      int which = is_q ? 0 : 1;
      asm volatile("" : "+v"(which));  // (read for every step: kept, the weights of both kinds would take 32 registers)
      const float* wt = weights[which];
      const int w0 = FULL ? d0 : min(d0, D - 8), w1 = FULL ? d1 : min(d1, D - 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) wp[e] = wt[w0 + e], wq[e] = wt[w1 + e];
      w.turn(gp, gq);
      float ss = 0.f, gx = 0.f;  // sums of x^2 and of f x
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        wp[e] *= gp[e], wq[e] *= gq[e];  // f
        ss = fmaf(p[e], p[e], fmaf(q[e], q[e], ss));
        gx = fmaf(wp[e], p[e], fmaf(wq[e], q[e], gx));
      }
      const float r = rsqrtf(fmaf(row_sum<U>(ss), inv_d, a.eps));
      const float c = row_sum<U>(gx) * r * inv_d;  // mean of f u
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] *= r, q[e] *= r;  // u
        gp[e] *= p[e], gq[e] *= q[e];
        p[e] = r * fmaf(-p[e], c, wp[e]), q[e] = r * fmaf(-q[e], c, wq[e]);
      }
      if (is_q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[e] += gp[e], dw[8 + e] += gq[e];
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float* y = x < 2 ? gp + 4 * x : gq + 4 * (x - 2);
          key_sums[wave][x][lane] += f32x4_t{y[0], y[1], y[2], y[3]};
        }
      }
      char* out = reinterpret_cast<char*>(is_q ? static_cast<T*>(a.q.out) + t * a.q.out_stride : static_cast<T*>(a.k.out) + t * a.k.out_stride) +
                  (is_q ? i : i - q_steps) * (RPW * D * (int)sizeof(T));
      if (FULL || has0) store8<NT>(reinterpret_cast<T*>(out + (row_at + d0 * (unsigned)sizeof(T))), p);
      if (FULL || has1) store8<NT>(reinterpret_cast<T*>(out + (row_at + d1 * (unsigned)sizeof(T))), q);
    };
    RawShare<T, FULL> xs, gs;
    load(part, xs, gs);
    form_turns(a, R, t, pos, turns);
    w.read(turns);
    for (int i = part; i < steps; i += parts) finish(i, xs, gs, i + parts);
    wave_sync();  // the next token's turns take the same place
  }
  __syncthreads();  // (the sums take the turns' place)
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float x = k == 0 ? dw[e] : key_sums[wave][e / 4][lane][e % 4];
#pragma unroll
      for (int m = U; m < kWaveSize; m <<= 1) x += __shfl_xor(x, m);
      const int d = (e < 8 ? d0 : d1) + e % 8;
      if (lane < U && d < D) lds.sums[wave][k][d] = x;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < kWavesHere; ++x) s += lds.sums[x][i / D][i % D];
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
  constexpr int kRuns = kThreads / kSumColumns, kAhead = 16;
  for (int i = run; i < groups; i += kRuns * kAhead) {
    float y[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) y[k] = i + k * kRuns < groups ? part[(size_t)(i + k * kRuns) * 2 * D + c] : 0.f;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x += y[k];
  }
  s[run][threadIdx.x % kSumColumns] = x;
  __syncthreads();
  if (run == 0) {
    for (int i = 1; i < kThreads / kSumColumns; ++i) x += s[i][threadIdx.x];
    float* out = c < D ? dq : dk;
    if (out) out[c < D ? c : c - D] = x;
  }
}

// Wavefronts that share a token: one where tokens are many, up to one for each of its steps where
// they are few; as many as make the last trip a full one, nearly.  Two for many tokens too where
// they are normed, rows are of up to 8 lanes and a token has 5 steps or more.  us, one / two, bf16: 16384
// tokens of 32 + 8 heads of 128 (5 steps) 61.0 / 58.9, 50000 180 / 165, 8000 33.8 / 32.9; in fp32 128.1 /
// 124.5; 20000 of 40 + 8 88.1 / 82.3; 6000 of 64 + 8 44.6 / 41.9; but 30000 of 12 + 2 (3 steps) 48.6 /
// 61.9, 12000 of 16 + 4 of 256 48.9 / 51.2, rotation alone of 14000 of 28 + 4 43.1 / 45.7, 26000 of
// 28 + 4 into the cache, whose neighbours then do not fill lines together, 96 / 112.
int parts_of(int U, bool halved, int64_t tokens, int steps) {
  const bool two = halved && U <= 8 && steps >= 5 && tokens > kFewWaves;
  return wave_parts(steps, two ? 2 : kFewWaves / tokens);
}

// Workgroups: one for every 4 wavefronts' turns; where rows fill less than three quarters of their steps, so that
// instructions bound the kernel, only as many as run at once (4 or 5 wavefronts on a SIMD), which loop over the rest.
// us, so / in rounds: 30000 tokens of 12 + 2 heads of 128 43.4 / 49.0, 60000 of 8 + 2 of 64 52.7 / 64.4, 20000 of 16 + 1
// of 128 36.8 / 38.1; into the cache 22000 of 12 + 2 45.6 / 51.2, 54000 of 8 + 2 of 64 80 / 91; but 16384 of 32 + 8
// of 128, all full, 62.4 / 59.1, 20000 of 24 + 8 60.3 / 58.3, into the cache 22000 of 16 + 16 of 64 68.2 / 62.8.
unsigned grid_of(int64_t tokens, int parts, int U, int rows, int steps, int waves_at_once) {
  const bool sparse = rows * U * 4 < kWaveSize * steps * 3;
  const int64_t most = sparse ? kComputeUnits * 4 * waves_at_once / kWavesHere : kMaxGrid;
  return (unsigned)std::min<int64_t>(most, (tokens * parts + kWavesHere - 1) / kWavesHere);
}

// f(U, FULL) as integral constants: the lanes that a row of head_dim elements takes.
template <typename F>
void with_lanes(int head_dim, F&& f) {
  auto with = [&](auto lanes) {
    head_dim == 16 * decltype(lanes)::value ? f(lanes, std::true_type()) : f(lanes, std::false_type());
  };
  const int lanes = row_lanes(head_dim);
  if (lanes == 4)
    with(std::integral_constant<int, 4>());
  else if (lanes == 8)
    with(std::integral_constant<int, 8>());
  else if (lanes == 16)
    with(std::integral_constant<int, 16>());
  else
    with(std::integral_constant<int, 32>());
}

template <typename T, bool NORM>
void launch_apply(const NormRotaryArgs& a, hipStream_t stream) {
  with_lanes(a.head_dim, [&](auto lanes, auto full) {
    constexpr int U = decltype(lanes)::value;
    constexpr bool FULL = decltype(full)::value;
    const int steps = row_steps(a.q.heads, U) + row_steps(a.k.heads, U), parts = parts_of(U, NORM, a.num_tokens, steps);
    const dim3 grid(grid_of(a.num_tokens, parts, U, a.q.heads + a.k.heads, steps, sizeof(T) == 2 ? 5 : 4)), threads(kThreads);
    if constexpr (sizeof(T) == 2 && FULL && U >= 8) {
      if (a.num_tokens >= kHintTokens && whole_lines(a.rot, a.head_dim)) {
        hipLaunchKernelGGL((norm_rotary_kernel<T, U, FULL, NORM, false, true>), grid, threads, 0, stream, a, parts);
        return;
      }
    }
    hipLaunchKernelGGL((norm_rotary_kernel<T, U, FULL, NORM, false, false>), grid, threads, 0, stream, a, parts);
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
  const bool nt = a.num_tokens >= kHintTokens && whole_lines(a.rot, a.head_dim);
  with_lanes(a.head_dim, [&](auto lanes, auto full) {
    constexpr int U = decltype(lanes)::value;
    if constexpr (U <= 8 && decltype(full)::value) {  // head_dim 64 and 128
      const int steps = row_steps(a.q.heads, U) + 2 * row_steps(a.k.heads, U), parts = parts_of(U, false, a.num_tokens, steps);
      const dim3 grid(grid_of(a.num_tokens, parts, U, a.q.heads + 2 * a.k.heads, steps, 4)), threads(kThreads);
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a, parts); };
      auto launch_kind = [&](auto normed) {
        constexpr bool NORM = decltype(normed)::value;
        if constexpr (U == 8) {
          if (nt) return launch(norm_rotary_kernel<__bf16, U, true, NORM, true, true>);
        }
        launch(norm_rotary_kernel<__bf16, U, true, NORM, true, false>);
      };
      a.normed ? launch_kind(std::true_type()) : launch_kind(std::false_type());
    }
  });
  return hipGetLastError();
}

hipError_t launch_norm_rotary_backward(const NormRotaryArgs& a, int dtype, hipStream_t stream) {
  const int parts = grad_parts(a.num_tokens, a.q.heads, a.head_dim), groups = grad_groups(a.num_tokens, parts);
  if (groups > 0)
    with_lanes(a.head_dim, [&](auto lanes, auto full) {
      constexpr int U = decltype(lanes)::value;
      constexpr bool FULL = decltype(full)::value;
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, stream, a, parts); };
      if (dtype != PDA_DTYPE_BF16) return launch(norm_rotary_grad_kernel<float, U, FULL, false>);
      if constexpr (FULL && U >= 8) {
        if (a.num_tokens >= kHintTokens && whole_lines(a.rot, a.head_dim)) return launch(norm_rotary_grad_kernel<__bf16, U, FULL, true>);
      }
      launch(norm_rotary_grad_kernel<__bf16, U, FULL, false>);
    });
  if (a.d_weight[0] || a.d_weight[1])
    hipLaunchKernelGGL(weight_grad_kernel, dim3(2 * a.head_dim / kSumColumns), dim3(kThreads), 0, stream, a.part, groups,
                       a.head_dim, a.d_weight[0], a.d_weight[1]);
  return hipGetLastError();
}

}  // namespace pda
