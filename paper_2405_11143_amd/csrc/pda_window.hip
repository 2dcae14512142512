// Attention with a sliding window and sinks (include/pda_window.h) for up to 32 query rows of a
// (sequence, KV head): decode steps and short drafts.
//
// Bound by the cache it reads.  As in pda_partition.hip a work item is (partition,
// sequence, KV head); its 4 wavefronts take contiguous runs of the item's blocks, tiles
// straight into registers (pda_wave.h), and their states are merged in LDS.  What
// differs: the blocks are those of a list (the sinks', then the window's), rows have a lower limit
// beside the upper one, and the rows are one or two 16-row tiles that share the block's
// V fragments.  Probabilities go through the second product in three bf16 parts,
// 24 bits: the products are far from the bound here (in two parts the time is the same).
//
// Measured: 256 sequences of 32 / 8 heads of 128 past a window of 1024 167 us, 6.3 TB/s, 94% of
// what a bare gather of such tiles reaches; four wavefronts to a SIMD, whose registers hold one
// tile less in flight, 184; 5 new tokens of each 190; 8 long samples, a window of 4096, 19.4 with the merge, whose launch
// is 3.4 of them.  For two tiles at D = 128 set_apart, inlined though it hardly ever runs, makes the kernel spill (36
// bytes of scratch a lane).
#include "pda_wave.h"
#include "pda_window_internal.h"

namespace pda {
namespace {

constexpr int kRows = kWindowTileRows;

// What the rows of a wavefront's tiles see, of the tokens: a row sees t if t < up and (t <
// sinks or t >= low); up and low lie between these.
struct Limits {
  int up_min, up_max, low_min, low_max, sinks;
  __device__ __forceinline__ bool all(int t) const { return t < up_min && (t < sinks || t >= low_max); }
  __device__ __forceinline__ bool some(int t) const { return t < up_max && (t < sinks || t >= low_min); }
  // every token of [t0, t1) is seen by every row
  __device__ __forceinline__ bool whole(int t0, int t1) const {
    return t1 <= up_min && (t1 <= sinks || t0 >= low_max);
  }
};

// One 16-row tile of a wavefront.
template <int D>
struct WindowTile : WaveAttention<D> {
  using Base = WaveAttention<D>;
  int up, low;  // this lane's row
  int token;    // its new token

  __device__ __forceinline__ WindowTile() : Base(0.f) {}

  __device__ __forceinline__ bool sees(int t, int sinks) const { return t < up && (t < sinks || t >= low); }

  // P^T as three bf16 B fragments, high part first.
  struct Parts {
    shortx4_t part[3];
  };

  // The probabilities of a block's scaled scores (tokens tok0 .. tok0 + 15).
  __device__ __forceinline__ Parts probabilities(float (&sc)[1][4], int tok0, bool masked, int sinks) {
    if (masked) {
      asm volatile("");  // a branch: as selects the masking would run on every block
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!sees(tok0 + 4 * this->kg + i, sinks)) sc[0][i] = Base::kNegInf;
    }
    const float top = max3(sc[0][0], sc[0][1], max3(sc[0][2], sc[0][3], Base::kNegInf));
    if (__builtin_amdgcn_ballot_w64(top > this->m_run + Base::kRescaleSlack) != 0) this->rescale(top);
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = exp2_fast(sc[0][i] - this->m_run);
    this->l_run += (p[0] + p[1]) + (p[2] + p[3]);
    Parts f;
#pragma unroll
    for (int x = 0; x < 3; ++x) {
      const uint2 w = make_uint2(pack_halves(__float_as_uint(p[0]), __float_as_uint(p[1]), true),
                                 pack_halves(__float_as_uint(p[2]), __float_as_uint(p[3]), true));
      f.part[x] = __builtin_bit_cast(shortx4_t, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] -= __uint_as_float(__float_as_uint(p[i]) & 0xffff0000u);  // exact
    }
    return f;
  }
};

// A wavefront's fold of one block into its tiles.  MULTI: their rows are of several new tokens.
template <int D, int TILES, bool MULTI>
struct WindowFold {
  using WT = WindowTile<D>;
  static constexpr int NC = WT::NC, VT = WT::VT;

  // V fragment t of the block: 4 tokens of one column.
  static __device__ __forceinline__ shortx4_t v_part(const WT& w, const uint4 (&vr)[4], int t) {
    const bool hi = t & 1;
    return __builtin_bit_cast(shortx4_t, make_uint2(pack_halves(w.col_dword(vr, 0, t), w.col_dword(vr, 1, t), hi),
                                                    pack_halves(w.col_dword(vr, 2, t), w.col_dword(vr, 3, t), hi)));
  }

  // 0xffff for every half of x that is an infinity or NaN, as bf16.
  static __device__ __forceinline__ unsigned odd_halves(unsigned x) {
    return ((x & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
  }

  // Tokens that only some rows see hold infinities or NaN: the rows that do see them become NaN in those
  // columns (counted by a product of ones), and the elements are zeroed for the others.
  static __device__ __forceinline__ void set_apart(WT (&w)[TILES], uint4 (&vr)[4], int tok0, const Limits& lim) {
    constexpr unsigned kOnes = 0x3f803f80u;
    unsigned partly[2] = {0u, 0u}, seen[TILES][2];  // of a fragment's two dwords: tokens 4 kg .. 4 kg + 3
#pragma unroll
    for (int x = 0; x < TILES; ++x) seen[x][0] = seen[x][1] = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = tok0 + 4 * w[0].kg + e;
      const unsigned half = e % 2 ? 0xffff0000u : 0x0000ffffu;
      if (!lim.all(t)) partly[e / 2] |= half;
#pragma unroll
      for (int x = 0; x < TILES; ++x)
        if (w[x].sees(t, lim.sinks)) seen[x][e / 2] |= half & kOnes;
    }
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const uint2 u = __builtin_bit_cast(uint2, v_part(w[0], vr, t));
      const shortx4_t ones = __builtin_bit_cast(
          shortx4_t, make_uint2(odd_halves(u.x) & partly[0] & kOnes, odd_halves(u.y) & partly[1] & kOnes));
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        const floatx4_t zero = {0.f, 0.f, 0.f, 0.f};
        const floatx4_t count = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            ones, __builtin_bit_cast(shortx4_t, make_uint2(seen[x][0], seen[x][1])), zero, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[x].o[t][e] = count[e] > 0.f ? __builtin_nanf("") : w[x].o[t][e];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (lim.all(tok0 + 4 * w[0].kg + e)) continue;
      vr[e].x &= ~odd_halves(vr[e].x), vr[e].y &= ~odd_halves(vr[e].y);
      vr[e].z &= ~odd_halves(vr[e].z), vr[e].w &= ~odd_halves(vr[e].w);
    }
  }

  static __device__ __forceinline__ void block(WT (&w)[TILES], const uint4 (&kr)[NC], uint4 (&vr)[4], int tok0,
                                               const Limits& lim) {
    uint4 k1[1][NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) k1[0][c] = kr[c];
    const bool masked = !lim.whole(tok0, tok0 + kBlockTokens);  // wavefront-uniform
    float sc[TILES][1][4];
#pragma unroll
    for (int x = 0; x < TILES; ++x) w[x].template scores<1>(k1, sc[x]);
    typename WT::Parts f[TILES];
#pragma unroll
    for (int x = 0; x < TILES; ++x) f[x] = w[x].probabilities(sc[x], tok0, masked, lim.sinks);
    if (masked) {
      asm volatile("");  // a branch, as above
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = tok0 + 4 * w[0].kg + e;
        if (!lim.some(t)) vr[e] = make_uint4(0u, 0u, 0u, 0u);  // nobody sees it: whatever it holds
        odd |= MULTI && !lim.all(t) && (odd_halves(vr[e].x) | odd_halves(vr[e].y) | odd_halves(vr[e].z) | odd_halves(vr[e].w)) != 0;
      }
      if (MULTI && __builtin_amdgcn_ballot_w64(odd) != 0) set_apart(w, vr, tok0, lim);
    }
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const shortx4_t a = v_part(w[0], vr, t);
#pragma unroll
      for (int x = 0; x < TILES; ++x)
#pragma unroll
        for (int part = 0; part < 3; ++part)
          w[x].o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, f[x].part[part], w[x].o[t], 0, 0, 0);
    }
  }
};

template <int D>
struct WindowLds {
  float o[kWaves][kRows][D];
  float m[kWaves][kRows];
  float l[kWaves][kRows];
  int bad[kWaves];
};

// One finished output row's columns d0 .. d0 + 3.
__device__ __forceinline__ void store_row4(float* p, const float (&acc)[4], float lsum) {
  const bool pos = lsum > 0.f || lsum != lsum;
  store_nt4(p, pos ? acc[0] / lsum : acc[0], pos ? acc[1] / lsum : acc[1], pos ? acc[2] / lsum : acc[2],
            pos ? acc[3] / lsum : acc[3]);
}

template <int D, int TILES, bool MULTI>
__global__ void __launch_bounds__(kWaves * kWaveSize) __attribute__((amdgpu_waves_per_eu(TILES == 1 ? 3 : 2)))
window_kernel(const WindowArgs a) {
  using WT = WindowTile<D>;
  using Fold = WindowFold<D, TILES, MULTI>;
  __shared__ __align__(16) WindowLds<D> sh;
  const StepArgs& s = a.step;
  const int Hq = s.num_q_heads, Hkv = s.num_kv_heads, G = s.group, n = s.num_query_tokens;
  const int item = blockIdx.x;  // (p * B + b) * Hkv + g
  const int g = item % Hkv;
  const int b = (item / Hkv) % s.num_seqs;
  const int p = item / (Hkv * s.num_seqs);
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = n * G;
  int L = s.lens[b];
  L = L < 0 ? 0 : (L > s.max_context_len ? s.max_context_len : L);
  const WindowSpan span = window_span(L, n, 0, n, a.window, a.sinks);
  const int per_part = s.partition_tokens / kWindowUnit;
  const int parts = (span.count() + per_part - 1) / per_part;
  auto out_row = [&](int r) {  // output row of the item's row r (token-major, then the G heads)
    const int i = r * s.group_inverse >> 16;  // r / G
    return ((size_t)b * n + i) * Hq + (size_t)g * G + (r - i * G);
  };
  if (p >= parts) {
    if (parts == 0 && p == 0)  // nothing to see
      for (int x = tid; x < rows * (D / 4); x += kWaves * kWaveSize)
        store_nt4(s.out + out_row(x / (D / 4)) * D + 4 * (x % (D / 4)), 0.f, 0.f, 0.f, 0.f);
    return;
  }

  WT w[TILES];
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    w[x].scale_log2 = s.scale_log2;
    const int r = min(x * kRows + (lane & 15), rows - 1);  // lane rows past the last one repeat it
    w[x].token = r * s.group_inverse >> 16;
    w[x].up = L - n + 1 + w[x].token;
    w[x].low = window_start(w[x].up, a.window);
    w[x].start(s.q + out_row(r) * D, 0);
  }
  const int first_up = L - n + 1;
  const Limits lim{first_up, L, window_start(first_up, a.window), window_start(L, a.window), a.sinks};

  const char* kpool = reinterpret_cast<const char*>(s.k) + (size_t)g * WT::kTileBytes;
  const char* vpool = reinterpret_cast<const char*>(s.v) + (size_t)g * WT::kTileBytes;
  const int32_t* table_row = s.table + (size_t)b * s.max_blocks_per_seq;
  const size_t block_bytes = (size_t)Hkv * WT::kTileBytes;
  // this wavefront's run of the item's blocks
  const int v_end = min(span.count(), (p + 1) * per_part);
  const int per_wave = (v_end - p * per_part + kWaves - 1) / kWaves;
  const int v0 = min(v_end, p * per_part + wave * per_wave), v1 = min(v_end, v0 + per_wave);
  uint4 ka[WT::NC], va[4], kb[WT::NC], vb[4];
  for (int c0 = v0; c0 < v1; c0 += kWaveSize) {
    const int cn = min(kWaveSize, v1 - c0);
    const int ids = lane < cn ? table_row[span.block(c0 + lane)] : 0;
    auto load = [&](uint4(&k)[WT::NC], uint4(&v)[4], int i) {
      w[0].load_tiles(k, v, kpool, vpool, block_bytes, s.num_blocks, __builtin_amdgcn_readlane(ids, min(i, cn - 1)), i < cn);
    };
    auto fold = [&](const uint4(&k)[WT::NC], uint4(&v)[4], int i) {
      Fold::block(w, k, v, span.token(c0 + i), lim);
    };
    load(ka, va, 0);
    for (int i = 0; i < cn; i += 2) {
      load(kb, vb, i + 1);
      __builtin_amdgcn_sched_barrier(0);
      fold(ka, va, i);
      if (i + 1 >= cn) break;
      load(ka, va, i + 2);
      __builtin_amdgcn_sched_barrier(0);
      fold(kb, vb, i + 1);
    }
  }

  // ---- merge the wavefronts' states in a fixed order, a tile at a time ----
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    const int tile_rows = min(kRows, rows - x * kRows);
    if (tile_rows <= 0) break;
    if (x > 0) __syncthreads();  // the first tile's states have been read
    w[x].finish();
    const int row = lane & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d0 = w[x].d_of(i, 0);  // D = 128: 8 consecutive columns; D = 64: 4
      *reinterpret_cast<f32x4_t*>(&sh.o[wave][row][d0]) = f32x4_t{w[x].o[0][i], w[x].o[1][i], w[x].o[2][i], w[x].o[3][i]};
      if constexpr (D == 128)
        *reinterpret_cast<f32x4_t*>(&sh.o[wave][row][d0 + 4]) = f32x4_t{w[x].o[4][i], w[x].o[5][i], w[x].o[6][i], w[x].o[7][i]};
    }
    if (lane < 16) {
      sh.m[wave][row] = w[x].m_run;
      sh.l[wave][row] = w[x].l_run;
    }
    if (lane == 0) sh.bad[wave] = w[0].bad ? 1 : 0;
    __syncthreads();
    int bad = 0;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) bad |= sh.bad[y];
    for (int idx = tid; idx < tile_rows * (D / 4); idx += kWaves * kWaveSize) {  // 4 columns per thread
      const int h = idx / (D / 4), d0 = 4 * (idx % (D / 4));
      float M = WT::kFloor, lsum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < kWaves; ++y) M = fmaxf(M, sh.m[y][h]);
#pragma unroll
      for (int y = 0; y < kWaves; ++y) {
        const float sc = exp2_fast(sh.m[y][h] - M);
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(&sh.o[y][h][d0]);
        lsum = fmaf(sc, sh.l[y][h], lsum);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(sc, o[e], acc[e]);
      }
      if (bad) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_nanf("");
      }
      const size_t row_out = out_row(x * kRows + h);
      if (parts == 1) {
        store_row4(s.out + row_out * D + d0, acc, lsum);
      } else {
        const size_t slot = row_out * s.slots_per_row + p;
        *reinterpret_cast<f32x4_t*>(s.part_o + slot * D + d0) = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
        if (d0 == 0) {
          s.part_m[slot] = M;
          s.part_l[slot] = lsum;
        }
      }
    }
  }
}

// Pass 2: a wavefront per output row joins its partitions' states in a fixed order.  A chain of
// latencies: 1 us less where the first states are loaded before the row's length is known.
constexpr int kMergeRows = 4, kMergeAhead = 8;
template <int D>
__global__ void __launch_bounds__(kMergeRows * kWaveSize) window_merge_kernel(const WindowArgs a) {
  constexpr int C = D / kWaveSize;  // columns of a lane
  const StepArgs& s = a.step;
  const int row = blockIdx.x * kMergeRows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & (kWaveSize - 1);
  if ((size_t)row >= (size_t)s.num_seqs * s.num_query_tokens * s.num_q_heads) return;
  const int i = (row / s.num_q_heads) % s.num_query_tokens, b = row / (s.num_q_heads * s.num_query_tokens);
  const size_t first = (size_t)row * s.slots_per_row;
  // The first slots are loaded before it is known how many the row has: the rest is one chain of
  // latencies less.
  float m[kMergeAhead], l[kMergeAhead], v[kMergeAhead][C];
  auto load = [&](int x0, int count) {
#pragma unroll
    for (int x = 0; x < kMergeAhead; ++x) {
      const size_t slot = first + min(x0 + x, count - 1);
      m[x] = s.part_m[slot], l[x] = s.part_l[slot];
#pragma unroll
      for (int c = 0; c < C; ++c) v[x][c] = s.part_o[slot * D + lane * C + c];
    }
  };
  load(0, s.slots_per_row);
  int L = s.lens[b];
  L = L < 0 ? 0 : (L > s.max_context_len ? s.max_context_len : L);
  const int parts = window_partitions(a, L, i / a.group_tokens);
  if (parts <= 1) return;  // pass 1 wrote the row
  float M = -__builtin_huge_valf();
#pragma unroll
  for (int x = 0; x < kMergeAhead; ++x) M = x < parts ? fmaxf(M, m[x]) : M;
  if (parts > kMergeAhead) {
    for (int x = kMergeAhead + lane; x < parts; x += kWaveSize) M = fmaxf(M, s.part_m[first + x]);
#pragma unroll
    for (int o = 1; o < kWaveSize; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  }
  float lsum = 0.f, acc[C];
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = 0.f;
  for (int x0 = 0; x0 < parts; x0 += kMergeAhead) {
    if (x0 > 0) load(x0, parts);
#pragma unroll
    for (int x = 0; x < kMergeAhead; ++x) {
      if (x0 + x >= parts) break;
      const float wgt = exp2_fast(m[x] - M);
      lsum = fmaf(wgt, l[x], lsum);
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = fmaf(wgt, v[x][c], acc[c]);
    }
  }
  const bool pos = lsum > 0.f || lsum != lsum;  // 0: the row sees nothing
  float* p = s.out + (size_t)row * D + lane * C;
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = pos ? acc[c] / lsum : acc[c];
  if constexpr (C == 2)
    store_nt2(p, acc[0], acc[1]);
  else
    __builtin_nontemporal_store(acc[0], p);
}

}  // namespace

hipError_t launch_window(const WindowArgs& a, int head_dim, hipStream_t stream) {
  const dim3 grid(a.step.num_regular_items), threads(kWaves * kWaveSize);
  const int n = a.step.num_query_tokens;
  if (head_dim != 64 && head_dim != 128) return hipErrorInvalidValue;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a); };
  auto launch_d = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (n == 1)
      launch(window_kernel<D, 1, false>);
    else if (n * a.step.group <= kWindowTileRows)
      launch(window_kernel<D, 1, true>);
    else
      launch(window_kernel<D, 2, true>);
  };
  head_dim == 64 ? launch_d(std::integral_constant<int, 64>()) : launch_d(std::integral_constant<int, 128>());
  return hipGetLastError();
}

hipError_t launch_window_merge(const WindowArgs& a, int head_dim, hipStream_t stream) {
  const unsigned rows = (unsigned)a.step.num_seqs * (unsigned)a.step.num_query_tokens * (unsigned)a.step.num_q_heads;
  const dim3 grid((rows + kMergeRows - 1) / kMergeRows), threads(kMergeRows * kWaveSize);
  if (head_dim == 64)
    hipLaunchKernelGGL(window_merge_kernel<64>, grid, threads, 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL(window_merge_kernel<128>, grid, threads, 0, stream, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pda
