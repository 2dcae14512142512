// Pass 1 of attention over the 8-bit KV cache (include/pda_fp8.h) for up to 32
// query rows per sequence and KV head: decode steps and the verification of a few
// drafted tokens.  The merge kernel is that of the bf16 cache, and so is the order
// kernel of steps with many items.
//
// A work item is (partition of a context, sequence, KV head): row r is head r % G of
// its new token r / G.  Bound by HBM: 2 D + 2 bytes per token and KV head, 256 flop
// each for every row (D = 128).  The 4 wavefronts of a workgroup take contiguous
// runs of the partition's blocks; each streams them through registers, two blocks
// folded while two are in flight, on the layouts of WaveAttention (pda_wave.h), whose
// lanes want exactly what the cache gives: a 16-byte K piece is the lane's A
// fragments of two k-steps, a V piece its 8 columns of two of its four tokens.  Codes
// become bf16 in registers, two per instruction, the row's power of two applied by the
// same instruction, so what is folded is what a bf16 cache of the stored values would
// hold.  256 sequences of 512-4096 tokens, 32 / 8 heads of 128: 195 us, 6.3 TB/s (a bare
// gather of the same tiles takes 180); 5 new tokens each 218 us.  Three and four pairs of
// blocks in flight changed nothing (198): a wavefront has 3 neighbours on its SIMD.
#include "pda_fp8_internal.h"
#include "pda_wave.h"

namespace pda {
namespace {

constexpr int kThreads = kWaves * kWaveSize;

template <int D, int ROWS>
struct DecodeShared {
  float o[kWaves][ROWS][D];
  float m[kWaves][ROWS];
  float l[kWaves][ROWS];
  int bad[kWaves];
};

// The work order (pda_order.hip: largest partition first, placed for the XCDs)
// without its kernel, whose launch is 5 us of a step: each workgroup ranks the
// (sequence, partition) pairs, one per thread, by a counting sort in LDS of which
// it needs one place only.  Pairs of one size class stay in the order of their indexes.
struct PickShared {
  int count[kOrderBuckets];  // pairs of a size class, largest first
  int found[2];              // the class that holds the place, and the place in it
  int waves[kWaves];         // pairs of that class in each wavefront
  int pair;
};

// The pair at place `pos`.  All threads of the workgroup call this.
__device__ __forceinline__ int pick_pair(const StepArgs& a, int pos, PickShared& s) {
  static_assert(kOrderBuckets == kThreads && kPickPairs == kThreads, "a class and a pair per thread");
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1), w = tid / kWaveSize;
  s.count[tid] = 0;
  int cls = -1;
  if (tid < a.num_seqs * a.num_partitions) {
    const int p = tid / a.num_seqs;
    const int L = clamped(a.lens[tid - p * a.num_seqs], a.max_context_len);
    const int tok = min(max(L - p * a.partition_tokens, 0), a.partition_tokens);
    cls = kOrderBuckets - 1 - min((tok + kBlockTokens - 1) / kBlockTokens, kOrderBuckets - 1);
  }
  __syncthreads();
  if (cls >= 0) atomicAdd(&s.count[cls], 1);
  __syncthreads();
  if (w == 0) {
    constexpr int kPer = kOrderBuckets / kWaveSize;
    int v[kPer], sum = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = s.count[kPer * lane + e], sum += v[e];
    int before = sum;  // inclusive scan over the lanes, then exclusive
#pragma unroll
    for (int o = 1; o < kWaveSize; o <<= 1) {
      const int t = __shfl_up(before, o);
      if (lane >= o) before += t;
    }
    before -= sum;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (pos >= before && pos < before + v[e]) s.found[0] = kPer * lane + e, s.found[1] = pos - before;
      before += v[e];
    }
  }
  __syncthreads();
  const uint64_t hits = __builtin_amdgcn_ballot_w64(cls == s.found[0]);
  if (lane == 0) s.waves[w] = __builtin_popcountll(hits);
  __syncthreads();
  int left = s.found[1];  // matches before the one that is wanted
#pragma unroll
  for (int x = 0; x < kWaves; ++x)
    if (x < w) left -= s.waves[x];
  if ((hits >> lane & 1) && left == __builtin_popcountll(hits & ((uint64_t(1) << lane) - 1))) s.pair = tid;
  __syncthreads();
  return s.pair;
}

// One block's codes and scale bytes in a lane's registers.
template <int D>
struct Codes {
  static constexpr int KP = D / 64;         // 16-byte K pieces of a lane
  static constexpr int kTile = 16 * D;      // bytes of a K or V tile
  uint4 k[KP], v[2];  // v: rows 4kg (x, y: 8 columns) and 4kg + 1 (z, w), then 4kg + 2 and 4kg + 3
  unsigned ks, vs;    // the byte of the lane's K token; the bytes of its four V tokens

  // Loads through descriptors of a tile's size: none leaves it, and with !needed
  // (a length of zero) none touches memory.
  __device__ __forceinline__ void load(const DecodeFp8Args& a, const char* kpool, const char* vpool,
                                       const char* spool, size_t block, int phys, bool needed, int lane, bool& bad) {
    if ((unsigned)phys >= (unsigned)a.step.num_blocks) {  // contract violation: never read outside the pool
      bad = true;
      phys = 0;
    }
    const size_t off = (size_t)phys * block;
    const int bytes = needed ? kTile : 0;
    const __amdgpu_buffer_rsrc_t rk = tile_rsrc(kpool + off * kTile, bytes);
    const __amdgpu_buffer_rsrc_t rv = tile_rsrc(vpool + off * kTile, bytes);
    const __amdgpu_buffer_rsrc_t rs = tile_rsrc(spool + off * 32, needed ? 32 : 0);
    const int n = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int c = 0; c < KP; ++c) k[c] = load_stream(rk, 16 * lane + 1024 * c);
#pragma unroll
    for (int j = 0; j < 2; ++j) v[j] = load_stream(rv, ((4 * j + kg) * (D / 8) + n % (D / 8)) * 16);
    ks = __builtin_amdgcn_raw_buffer_load_b8(rs, n, 0, 0);
    vs = __builtin_amdgcn_raw_buffer_load_b32(rs, 16 + 4 * kg, 0, 0);
  }

  // The A fragments of the score products: k-step 2c is the first half of piece c.
  __device__ __forceinline__ void k_frags(uint4 (&kr)[2 * KP]) const {
    const float f = scale_of<0>(ks);
#pragma unroll
    for (int c = 0; c < KP; ++c) {
      kr[2 * c] = to_bf16(k[c].x, k[c].y, f);
      kr[2 * c + 1] = to_bf16(k[c].z, k[c].w, f);
    }
  }

  // Whether row e of the lane's four of V is one of NaN.
  __device__ __forceinline__ bool dead(int e) const { return (vs >> (8 * e) & 255u) == 255u; }

  // Rows of V that hold an infinity become rows of NaN (their codes are in the 16 lanes of the k-group).
  __device__ __forceinline__ void infinite_v(int kg) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint4& c = v[e / 2];
      const unsigned s = vs >> (8 * e) & 255u;
      const uint64_t hits = __builtin_amdgcn_ballot_w64(infinite(e % 2 ? c.z : c.x, s) || infinite(e % 2 ? c.w : c.y, s));
      if (hits >> (16 * kg) & 0xffffu) vs |= 255u << (8 * e);
    }
  }

  // V's codes and scale bytes become zeros from row `rel` of the lane's four on, and
  // in the rows of NaN.
  __device__ __forceinline__ void clear_v(int rel) {
    const bool d0 = dead(0), d1 = dead(1), d2 = dead(2), d3 = dead(3);
    vs &= (d0 ? 0u : 0xffu) | (d1 ? 0u : 0xff00u) | (d2 ? 0u : 0xff0000u) | (d3 ? 0u : 0xff000000u);
    vs = rel <= 0 ? 0u : rel >= 4 ? vs : vs & ((1u << (8 * rel)) - 1);
    if (rel <= 0 || d0) v[0].x = v[0].y = 0u;
    if (rel <= 1 || d1) v[0].z = v[0].w = 0u;
    if (rel <= 2 || d2) v[1].x = v[1].y = 0u;
    if (rel <= 3 || d3) v[1].z = v[1].w = 0u;
  }
};

// The fold of two blocks into the states of NT tiles of 16 rows, on the layouts of
// WaveAttention.  Scores and probabilities are its own; P V runs on MFMA
// f32_16x16x32_bf16 over both blocks at once, and each probability is split into
// three bf16 parts, each the top 16 bits of what is left, which together are all
// of its 24 bits: the third costs MFMAs that the wait for memory hides (with two
// the result was 4.8e-6 of its norm off, ten times what the rest of the arithmetic is).
template <int D>
struct Fold : WaveAttention<D> {
  using WA = WaveAttention<D>;
  __device__ __forceinline__ Fold() : WA(0.f) {}

  // A zero probability would not keep a NaN of V from a row that does not see its
  // token: in the tail, rows of NaN (and of infinities: infinite_v) make the scores of the
  // rows that see them NaN here, and are zeros in the product.
  __device__ __forceinline__ void probabilities(const uint4 (&kr)[2][WA::NC], const Codes<D> (&c)[2], int tok0, int L,
                                                int t_stop, bool tail, bf16x8_t (&part)[3]) {
    float sc[2][4];
    this->template scores<2>(kr, sc);
    if (tail) {
      asm volatile("");  // a branch: as selects the masking would run on every block
      const int rel = min(L - this->lim_off, t_stop) - (tok0 + 4 * this->kg);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (c[b].dead(i)) sc[b][i] = __builtin_nanf("");
          if (kBlockTokens * b + i >= rel) sc[b][i] = WA::kNegInf;
        }
    }
    float top = max3(max3(sc[0][0], sc[0][1], sc[0][2]), sc[0][3], sc[1][0]);
    top = max3(max3(sc[1][1], sc[1][2], sc[1][3]), top, top);
    if (__builtin_amdgcn_ballot_w64(top > this->m_run + WA::kRescaleSlack) != 0) this->rescale(top);
    float pr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pr[i] = exp2_fast(sc[i / 4][i % 4] - this->m_run);
    this->l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      unsigned w[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) w[h] = pack_halves(__float_as_uint(pr[2 * h]), __float_as_uint(pr[2 * h + 1]), true);
      part[k] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] -= __uint_as_float(__float_as_uint(pr[i]) & 0xffff0000u);
    }
  }
};

// Fold blocks c[0], c[1] (tokens tok0 .. tok0 + 31, those from t_stop on not there).
template <int D, int NT>
__device__ __forceinline__ void fold_pair(Fold<D> (&wave)[NT], Codes<D> (&c)[2], int tok0, int L, int l_first, int l_vis,
                                          int t_stop) {
  const bool tail = tok0 + 2 * kBlockTokens > min(l_first, t_stop);  // wavefront-uniform
  if (tail) {
    const unsigned top = (c[0].vs & (c[0].vs << 1)) | (c[1].vs & (c[1].vs << 1));  // bit 7: a byte of 192 or more
    const bool large = __builtin_amdgcn_ballot_w64((top & 0x80808080u) != 0) != 0;
    if (__builtin_expect(large, 0)) c[0].infinite_v(wave[0].kg), c[1].infinite_v(wave[0].kg);
  }
  uint4 kr[2][WaveAttention<D>::NC];
  c[0].k_frags(kr[0]);
  c[1].k_frags(kr[1]);
  bf16x8_t part[NT][3];
#pragma unroll
  for (int x = 0; x < NT; ++x) wave[x].probabilities(kr, c, tok0, L, t_stop, tail, part[x]);
  if (tail) {  // rows that no query row sees, whatever they hold, and those of NaN
    asm volatile("");
#pragma unroll
    for (int b = 0; b < 2; ++b) c[b].clear_v(l_vis - (tok0 + kBlockTokens * b + 4 * wave[0].kg));
  }
  // Output tiles 2 dw and 2 dw + 1 take the two columns of dword dw of the rows (WaveAttention::col_dword): two codes.
  const bool upper = D == 64 && wave[0].n >= 8;
  float f[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    f[b][0] = scale_of<0>(c[b].vs), f[b][1] = scale_of<1>(c[b].vs);
    f[b][2] = scale_of<2>(c[b].vs), f[b][3] = scale_of<3>(c[b].vs);
  }
#pragma unroll
  for (int dw = 0; dw < WaveAttention<D>::VT / 2; ++dw) {
    unsigned w[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint4& v = c[b].v[e / 2];
        const unsigned lo = e % 2 ? v.z : v.x, hi = e % 2 ? v.w : v.y;
        const unsigned codes = D == 64 ? (upper ? hi : lo) : dw < 2 ? lo : hi;
        const bf16x2_t x = dw % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, f[b][e], true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, f[b][e], false);
        w[b][e] = __builtin_bit_cast(unsigned, x);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x8_t a = __builtin_bit_cast(
          bf16x8_t, make_uint4(pack_halves(w[0][0], w[0][1], h), pack_halves(w[0][2], w[0][3], h),
                               pack_halves(w[1][0], w[1][1], h), pack_halves(w[1][2], w[1][3], h)));
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int k = 0; k < 3; ++k)
          wave[x].o[2 * dw + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, part[x][k], wave[x].o[2 * dw + h], 0, 0, 0);
    }
  }
}

// NT: tiles of 16 query rows of a work item (1 or 2), folded from the same
// converted blocks.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(NT == 1 ? 3 : 2)))
decode_fp8_kernel(const DecodeFp8Args args) {
  using WA = WaveAttention<D>;
  using CD = Codes<D>;
  __shared__ __align__(16) DecodeShared<D, NT * kFp8TileRows> sh;
  __shared__ PickShared pick;  // (a place of its own: a wavefront without blocks may be in the epilogue before others read it)
  const StepArgs& a = args.step;
  int g, b, p;  // KV head, sequence, partition
  if (a.order) {
    const int item = a.order[blockIdx.x];
    if ((unsigned)item >= (unsigned)a.num_regular_items) return;
    const int H = a.num_kv_heads;
    g = item % H, b = item / H % a.num_seqs, p = item / (H * a.num_seqs);
  } else if (args.picks) {  // the places of pda_order.hip
    const int H = a.num_kv_heads;
    const int slot = blockIdx.x;
    int pos;
    if (H % 8 == 0) {
      pos = slot / H, g = slot % H;
    } else {
      const int first = slot / (8 * H) * 8, c = min(8, a.num_seqs * a.num_partitions - first);
      const int in = slot - first * H;
      pos = first + in % c, g = in / c;
    }
    const int pair = __builtin_amdgcn_readfirstlane(pick_pair(a, pos, pick));
    p = pair / a.num_seqs, b = pair % a.num_seqs;
  } else {
    g = blockIdx.x, b = blockIdx.y, p = blockIdx.z;
  }
  const int G = a.group, n = a.num_query_tokens, Hq = a.num_q_heads, Tp = a.partition_tokens;
  const int tid = threadIdx.x;
  const int lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int L = clamped(a.lens[b], a.max_context_len);

  const int rows = n * G;  // at most 16 NT
  auto token_of = [&](int r) { return r * a.group_inverse >> 16; };
  auto limit_of = [&](int r) { return L - n + 1 + token_of(r); };  // row r sees tokens below it
  auto out_row = [&](int r) {
    const int i = token_of(r);
    return ((size_t)b * n + i) * Hq + (size_t)g * G + (r - i * G);
  };
  const int l_first = L - n + 1;
  const int l_vis = L;
  if (p == 0 && l_first <= 0) {  // rows that see nothing: zeros
    for (int x = tid; x < rows * (D / 4); x += kThreads)
      if (limit_of(x / (D / 4)) <= 0) store_nt4(a.out + out_row(x / (D / 4)) * D + 4 * (x % (D / 4)), 0.f, 0.f, 0.f, 0.f);
  }
  if (l_vis <= p * Tp) return;
  const int j0 = p * Tp / kBlockTokens;
  const int j1 = (min(l_vis, (p + 1) * Tp) + kBlockTokens - 1) / kBlockTokens;

  Fold<D> wave[NT];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    wave[x].scale_log2 = a.scale_log2;
    const int r = min(x * kFp8TileRows + (lane & 15), rows - 1);  // lanes past the last row repeat it
    wave[x].start(a.q + out_row(r) * D, n - 1 - token_of(r));
  }
  const char* kpool = reinterpret_cast<const char*>(args.k) + (size_t)g * CD::kTile;
  const char* vpool = reinterpret_cast<const char*>(args.v) + (size_t)g * CD::kTile;
  const char* spool = reinterpret_cast<const char*>(args.scale) + (size_t)g * 32;
  const int32_t* table_row = a.table + (size_t)b * a.max_blocks_per_seq;
  const int per_slice = (j1 - j0 + kWaves - 1) / kWaves;
  const int wj0 = min(j1, j0 + w * per_slice);
  const int wj1 = min(j1, wj0 + per_slice);
  bool bad = false;
  CD c0[2], c1[2];  // two pairs of blocks: one is folded, the next in flight
  for (int jc = wj0; jc < wj1; jc += kWaveSize) {
    const int cn = min(kWaveSize, wj1 - jc);
    const int ids = lane < cn ? table_row[jc + lane] : 0;
    auto load = [&](CD (&c)[2], int i) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
        c[x].load(args, kpool, vpool, spool, a.num_kv_heads, __builtin_amdgcn_readlane(ids, min(i + x, cn - 1)), i + x < cn,
                  lane, bad);
    };
    auto fold = [&](CD (&c)[2], int i) {
      fold_pair<D, NT>(wave, c, (jc + i) * kBlockTokens, L, l_first, l_vis, wj1 * kBlockTokens);
    };
    load(c0, 0);
    for (int i = 0; i < cn; i += 4) {
      load(c1, i + 2);
      __builtin_amdgcn_sched_barrier(0);
      fold(c0, i);
      if (i + 2 >= cn) break;
      load(c0, i + 4);
      __builtin_amdgcn_sched_barrier(0);
      fold(c1, i + 2);
    }
  }

  // ---- the wavefronts' states, merged in a fixed order ----
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    wave[x].finish();
    const int h = x * kFp8TileRows + (lane & 15);
    const f32x4_t* o = reinterpret_cast<const f32x4_t*>(wave[x].o);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d0 = wave[x].d_of(i, 0);
      *reinterpret_cast<float4*>(&sh.o[w][h][d0]) = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
      if constexpr (D == 128) *reinterpret_cast<float4*>(&sh.o[w][h][d0 + 4]) = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
    }
    if (lane < 16) {
      sh.m[w][h] = wave[x].m_run;
      sh.l[w][h] = wave[x].l_run;
    }
  }
  if (lane == 0) sh.bad[w] = bad ? 1 : 0;
  __syncthreads();
  int any_bad = 0;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) any_bad |= sh.bad[x];
  for (int x = tid; x < rows * (D / 4); x += kThreads) {
    const int h = x / (D / 4), d0 = 4 * (x % (D / 4));
    const int limit = limit_of(h);
    const int parts = limit > 0 ? (limit + Tp - 1) / Tp : 0;
    if (p >= parts) continue;  // the row sees nothing here
    float M = WA::kFloor, lsum = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < kWaves; ++y) M = fmaxf(M, sh.m[y][h]);
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      const float s = exp2_fast(sh.m[y][h] - M);
      const f32x4_t o = *reinterpret_cast<const f32x4_t*>(&sh.o[y][h][d0]);
      lsum = fmaf(s, sh.l[y][h], lsum);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(s, o[e], acc[e]);
    }
    if (any_bad) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_nanf("");
    }
    const size_t row = out_row(h);
    if (parts == 1) {
      const bool pos = lsum > 0.f;
      store_nt4(a.out + row * D + d0, pos ? acc[0] / lsum : acc[0], pos ? acc[1] / lsum : acc[1],
                pos ? acc[2] / lsum : acc[2], pos ? acc[3] / lsum : acc[3]);
    } else {  // a partial state for the merge
      const size_t slot = row * a.slots_per_row + p;
      *reinterpret_cast<f32x4_t*>(a.part_o + slot * D + d0) = acc;
      if (d0 == 0) {
        a.part_m[slot] = M;
        a.part_l[slot] = lsum;
      }
    }
  }
}

template <int D>
hipError_t launch_d(const DecodeFp8Args& a, hipStream_t stream) {
  const StepArgs& s = a.step;
  if (s.num_query_tokens * s.group > 2 * kFp8TileRows) return launch_wide_fp8(a, D, stream);
  const dim3 grid = s.order || a.picks ? dim3((unsigned)s.num_regular_items)
                            : dim3(s.num_kv_heads, s.num_seqs, s.num_partitions);
  if (s.num_query_tokens * s.group <= kFp8TileRows)
    hipLaunchKernelGGL((decode_fp8_kernel<D, 1>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((decode_fp8_kernel<D, 2>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_fp8(const DecodeFp8Args& a, int head_dim, hipStream_t stream) {
  if (head_dim == 64) return launch_d<64>(a, stream);
  if (head_dim == 128) return launch_d<128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace pda
