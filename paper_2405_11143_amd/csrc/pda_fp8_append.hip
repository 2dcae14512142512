// The quantised KV append (include/pda_fp8.h): each new token's key row rotated
// and, like its value row, stored as e4m3 codes and a power-of-two scale; its
// query rows rotated beside.
//
// Bound by memory: per token 4 Hq D + 4 Hkv D bytes of bf16 rows and 2 Hkv (D + 1)
// of cache, and by latency in a decode step, which is one launch of one token
// per workgroup.  A workgroup forms the cosines and sines of its tokens' positions
// in LDS, then D / 16 threads take each row, 16 elements each (for a rotated row 8
// pairs), and form the row's largest magnitude by shuffles.  A row of K goes out 8
// codes at a time, to pieces 16 bytes apart from its neighbours in the block.
// Workgroups of one block of 16 tokens, which write whole cache lines, took longer
// (87 us against 71 for 32 x 512 tokens): their 24 trips wait for each other.
#include "pda_fp8_internal.h"

namespace pda {
namespace {

constexpr int kMaxThreads = 256;  // (512: the prompts below took 131 us instead of 95)
constexpr int kFewUnits = 200;
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

template <bool NT>
__device__ __forceinline__ void store_query(uint16_t* dst, const float (&x)[8]) {
  bf16v8_t p;
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = (__bf16)x[e];
  if (NT)
    __builtin_nontemporal_store(p, reinterpret_cast<bf16v8_t*>(dst));
  else
    *reinterpret_cast<bf16v8_t*>(dst) = p;
}

// The bits of the largest magnitude of a row that U neighbouring lanes hold.
template <int U>
__device__ __forceinline__ unsigned row_top(const float (&x)[8], const float (&y)[8]) {
  unsigned top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    top = max(top, max(__float_as_uint(x[e]) & 0x7fffffffu, __float_as_uint(y[e]) & 0x7fffffffu));
#pragma unroll
  for (int m = 1; m < U; m <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, m));
  return top;
}

// A lane's two vectors (elements d0 .. and d1 ..) of the row of slot o, tile
// `tile` (block and KV head), K (which 1) or V (2); lane u 0 stores the scale byte.
template <int D>
__device__ __forceinline__ void store_codes(const AppendFp8Args& a, int which, size_t tile, int o, int u, int d0, int d1,
                                            const float (&x)[8], const float (&y)[8], int s) {
  auto at = [&](int d) {
    return which == 1 ? ((d / 64 * 4 + d / 8 % 4) * 16 + o) * 16 + d / 32 % 2 * 8
                      : (((o / 2 % 2) * 4 + o / 4) * (D / 8) + d / 8) * 16 + o % 2 * 8;
  };
  uint8_t* dst = (which == 1 ? a.k : a.v) + tile * (16 * D);
  *reinterpret_cast<uint2*>(dst + at(d0)) = codes_of(x, s);
  *reinterpret_cast<uint2*>(dst + at(d1)) = codes_of(y, s);
  if (u == 0) a.scale[tile * 32 + (which == 1 ? 0 : 16) + o] = (uint8_t)s;
}

// TOKENS: neighbouring new tokens of one sequence that a workgroup takes.  NT: the
// queries go out with the non-temporal hint.
template <int D, int TOKENS, bool NT>
__global__ void __launch_bounds__(kMaxThreads) append_fp8_kernel(const AppendFp8Args a, int groups) {
  constexpr int U = D / 16;  // threads per row
  __shared__ float2 turns[TOKENS][D / 2];
  const int n = a.num_query_tokens;
  const int R = a.rot.inv_freq ? a.rot.rotary_dim : 0;
  const int nq = a.q ? a.num_q_heads : 0;
  const int rows = nq + 2 * a.num_kv_heads;  // of a token: queries, keys, values
  const int u = threadIdx.x % U;
  const int rows_at_once = blockDim.x / U;
  const RowShare rotated = row_share(a.rot, R, D, u), plain = row_share(a.rot, 0, D, u);
  for (int64_t x = blockIdx.x; x < (int64_t)a.num_seqs * groups; x += gridDim.x) {
    const int b = (int)(x / groups), i0 = (int)(x % groups) * TOKENS;
    const int L = clamped(a.lens[b], a.max_context_len);
    const int t0 = L - n + i0;  // the first token's position
    const int first = max(-t0, 0), end = min(TOKENS, n - i0);
    if (first >= end) continue;  // (the whole workgroup)
    for (int e = threadIdx.x; e < end * (R / 2); e += blockDim.x) {
      const int i = TOKENS == 1 ? 0 : e / (R / 2);
      turns[i][e - i * (R / 2)] = turn(a.rot, t0 + i, e - i * (R / 2));
    }
    __syncthreads();
    int i = first, row = threadIdx.x / U;
    for (; row >= rows; row -= rows) ++i;
    while (i < end) {  // (all threads of a row together: they shuffle)
      const int which = row < nq ? 0 : row < nq + a.num_kv_heads ? 1 : 2;
      const int h = which == 0 ? row : which == 1 ? row - nq : row - nq - a.num_kv_heads;
      const size_t token = (size_t)b * n + i0 + i;
      const uint16_t* src = which == 0 ? a.q : which == 1 ? a.k_new : a.v_new;
      src += (token * (which == 0 ? a.num_q_heads : a.num_kv_heads) + h) * D;
      const RowShare w = which < 2 ? rotated : plain;
      const int t = t0 + i;
      const float2* cs = turns[i];
      float xs[8], ys[8];
      load8(src + w.d0, xs);
      load8(src + w.d1, ys);
      for (row += rows_at_once; row >= rows; row -= rows) ++i;
      rotate_share(cs, a.rot.interleaved, w, xs, ys);
      if (which == 0) {
        uint16_t* dst = a.q_out + (token * a.num_q_heads + h) * D;
        store_query<NT>(dst + w.d0, xs);
        store_query<NT>(dst + w.d1, ys);
        continue;
      }
      const int page = a.table[(size_t)b * a.max_blocks_per_seq + t / kBlockTokens];
      const int s = scale_byte(row_top<U>(xs, ys));
      if ((unsigned)page < (unsigned)a.num_blocks)
        store_codes<D>(a, which, (size_t)page * a.num_kv_heads + h, t % kBlockTokens, u, w.d0, w.d1, xs, ys, s);
    }
    __syncthreads();  // the next tokens' turns take the same place
  }
}

// Two new tokens of a sequence to a workgroup, four where many tokens have few rows
// (at most kFewUnits threads' worth), one in a decode step.  Time in us with one, two
// and four, the same inputs again and again: 48 prompts of up to 1024 tokens, 28 / 4 heads of 128, 99 / 95 / 101; 32 x
// 512 tokens of 32 / 8 72 / 71 / 73; 128 x 16 10.3 / 9.5 / 10.4; 48 x 300 tokens of 16 /
// 16 heads of 64 38 / 33 / 30; a few tokens 5.2 / 5.3 / 7.0.  With whole lines of
// queries stored past the caches (whole_lines) the prompts take 83, and 92 where the
// inputs change from call to call: 4.9 TB/s, the rate of a large copy.
template <int D>
hipError_t launch_d(const AppendFp8Args& a, hipStream_t stream) {
  const int units = ((a.q ? a.num_q_heads : 0) + 2 * a.num_kv_heads) * (D / 16);
  auto launch = [&](auto kernel, int tokens) {
    const int groups = (a.num_query_tokens - 1) / tokens + 1;
    const unsigned grid = (unsigned)min((int64_t)a.num_seqs * groups, kMaxGrid);
    // as many threads as make the last trip through the rows a full one, nearly
    const int64_t all = (int64_t)tokens * units;
    const int64_t trips = (all + kMaxThreads - 1) / kMaxThreads;
    const int threads = (int)min((int64_t)kMaxThreads, ((all + trips - 1) / trips + kWaveSize - 1) / kWaveSize * kWaveSize);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, stream, a, groups);
    return hipGetLastError();
  };
  const bool many = (int64_t)a.num_seqs * a.num_query_tokens >= kManyTokens;
  if (a.num_query_tokens == 1) return launch(append_fp8_kernel<D, 1, false>, 1);
  if (many && units <= kFewUnits && a.num_query_tokens >= 4) return launch(append_fp8_kernel<D, 4, false>, 4);
  if (many && D == 128 && whole_lines(a.rot, D)) return launch(append_fp8_kernel<D, 2, D == 128>, 2);
  return launch(append_fp8_kernel<D, 2, false>, 2);
}

}  // namespace

hipError_t launch_append_fp8(const AppendFp8Args& a, int head_dim, hipStream_t stream) {
  if (head_dim == 64) return launch_d<64>(a, stream);
  if (head_dim == 128) return launch_d<128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace pda
