// Pass 1 of attention over the 8-bit KV cache for more than 32 query rows per
// sequence and KV head (chunked and fresh prefill, long drafts).
//
// A work item is (partition of a context, sequence, KV head, group of 32 W query
// rows); row r of a sequence and KV head is head r % G of its new token r / G, and each
// of the workgroup's W wavefronts takes 32 of them.  Bound by the matrix cores (54% busy
// in large chunks) and vector issue (52%): 4 D flop per row and token, in bf16, with the
// probabilities in two halves (6 D issued).  As in pda_wide.hip both products run transposed on MFMA
// f32_32x32x16_bf16 (S^T = K Q^T, O^T = V^T P^T: the lane's 16 scores belong to
// one row and are its P^T fragments), and the scores of the next 32 tokens are
// formed while these are folded, one stretch without a branch.  What differs is
// the way in:
//  * Codes come through registers, 16 bytes per lane, and are converted once
//    per workgroup, not per wavefront, on their way to LDS (16 conversions per
//    thread and step at W = 4), with the row's power of two in the same
//    instruction.  LDS holds what a bf16 cache's tiles would be: K in its
//    fragments' order, V in rows whose 16-byte pieces are permuted, so that the 4
//    rows of a transposed read fall on disjoint banks.
//  * Three buffers: one step is folded, the next one's scores are formed, the
//    one after is being written; its successor's codes are in flight.
//  * Rows are dense (no chunks of whole tokens): 7 heads per KV head fill the
//    tiles as well as 8.
#include <type_traits>

#include "pda_fp8_internal.h"
#include "pda_wave.h"

namespace pda {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kTileRows = 32;      // query rows of a wavefront
constexpr int kStageBlocks = 2;    // blocks of a step: 32 tokens

// Two-wavefront workgroups form their scores in the step itself, with two buffers
// instead of three, so that four of them fit a compute unit instead of three.
constexpr bool scores_ahead(int W) { return W == 4; }
constexpr int buffers(int W) { return scores_ahead(W) ? 3 : 2; }
constexpr int window(int W) { return W == 4 ? 1024 : 256; }  // block ids held in LDS at a time

template <int D, int W>
struct WideLds {
  static constexpr int kTilePieces = 2 * D;  // 16-byte pieces of a bf16 K or V tile
  static constexpr int kBlockPieces = 2 * kTilePieces;
  union {
    uint4 buf[buffers(W)][kStageBlocks][kBlockPieces];
    f32x4_t o[W][kTileRows][D / 8];  // the epilogue, half of the columns at a time
  };
  int ids[window(W)];
  unsigned char dead[buffers(W)][kStageBlocks * kBlockTokens];  // per token of a buffer: its values hold a NaN or an infinity
};

template <int D, int W>
__global__ void __launch_bounds__(W * kWaveSize) __attribute__((amdgpu_waves_per_eu(2)))
wide_fp8_kernel(const DecodeFp8Args args) {
  using S = WideLds<D, W>;
  constexpr int kThreads = W * kWaveSize;
  constexpr int kBuffers = buffers(W), kWindow = window(W);
  constexpr bool kAhead = scores_ahead(W);
  constexpr int KS = D / 16;  // score MFMA k-steps
  constexpr int VT = D / 32;  // output tiles of 32 columns
  constexpr int RP = D / 8;   // 16-byte pieces of a bf16 V row
  constexpr int kTile = 16 * D;                             // bytes of an 8-bit tile
  constexpr int NP = 2 * kStageBlocks * D / kThreads;       // 16-byte code pieces of a thread and step
  static_assert(NP >= 1 && D % kWaveSize == 0, "a wavefront's pieces are of one tile");
  __shared__ __align__(16) S st;
  const StepArgs& a = args.step;

  const int item = a.order ? a.order[blockIdx.x] : (int)blockIdx.x;
  if ((unsigned)item >= (unsigned)a.num_regular_items) return;
  const int groups = a.num_chunk_groups;
  const int HC = a.num_kv_heads * groups;
  const int gc = item % HC;
  const int b = item / HC % a.num_seqs;
  const int p = item / (HC * a.num_seqs);
  const int g = gc / groups, rg = gc % groups;
  const int G = a.group, n = a.num_query_tokens, Hq = a.num_q_heads, Tp = a.partition_tokens;
  const int tid = threadIdx.x;
  const int lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5;   // which half of the k-groups the lane holds
  const int col = lane & 31;  // the lane's row of the tile
  const int L = clamped(a.lens[b], a.max_context_len);

  const int R = n * G;
  const int wg0 = rg * (W * kTileRows);
  const int wg_rows = min(W * kTileRows, R - wg0);
  // row wg0 + x: its token is i0 + (m0 + x) / G (m0 + x < 16 + 128: the inverse is exact)
  const int i0 = wg0 / G, m0 = wg0 - i0 * G;
  auto token_of = [&](int x) { return i0 + ((m0 + x) * a.group_inverse >> 16); };
  auto limit_of = [&](int x) { return L - n + 1 + token_of(x); };  // the row sees tokens below it
  auto out_row = [&](int x) {
    const int i = (m0 + x) * a.group_inverse >> 16;
    return ((size_t)b * n + i0 + i) * Hq + (size_t)g * G + (m0 + x - i * G);
  };
  if (p == 0 && limit_of(0) <= 0) {  // rows that see nothing: zeros
    for (int x = tid; x < wg_rows * (D / 4); x += kThreads)
      if (limit_of(x / (D / 4)) <= 0) store_nt4(a.out + out_row(x / (D / 4)) * D + 4 * (x % (D / 4)), 0.f, 0.f, 0.f, 0.f);
  }
  const int t_pe = min((p + 1) * Tp, L);  // tokens at or past it belong to the next partition, or to none
  if (limit_of(wg_rows - 1) <= p * Tp) return;

  // ---- this wavefront's tile ----
  const int x0 = w * kTileRows;
  const bool active = x0 < wg_rows;
  const int my_x = min(x0 + col, wg_rows - 1);  // lanes past the last row repeat it
  const int limit = min(limit_of(my_x), t_pe);
  const int l_some = min(limit_of(0), t_pe);  // from here on some row of the workgroup does not see a token
  const int l_vis = min(max(limit_of(min(x0 + kTileRows, wg_rows) - 1), 0), t_pe);

  float scale = a.scale_log2;
  const unsigned flip = scale < 0.f ? 0x80008000u : 0u;
  const unsigned keep = scale == 0.f ? 0u : 0xffffffffu;  // a zero scale: zero scores, whatever is masked
  scale = keep ? fabsf(scale) : 1.f;
  bf16x8_t q[KS];
  {
    const uint16_t* qp = a.q + out_row(my_x) * D + 8 * hh;
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      uint4 u = *reinterpret_cast<const uint4*>(qp + 16 * c);
      u.x = (u.x ^ flip) & keep, u.y = (u.y ^ flip) & keep, u.z = (u.z ^ flip) & keep, u.w = (u.w ^ flip) & keep;
      q[c] = __builtin_bit_cast(bf16x8_t, u);
    }
  }
  f32x16_t o[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  // The reference of a row's probabilities, exp2(s * scale - m_run): a whole number
  // at most 8 below the largest scaled score so far (nothing overflows, and nothing
  // that counts underflows; past 2^24 a score's own rounding comes to that, up to 2^30 no more
  // than 2^32 of a probability).  The difference is one fused operation on an exact
  // reference, the same for all tokens, so large scores cancel.
  float m_run = -1e30f, l_run = 0.f;

  const int32_t* table_row = a.table + (size_t)b * a.max_blocks_per_seq;
  const int J0 = p * Tp / kBlockTokens;
  const int J1 = (min(limit_of(wg_rows - 1), t_pe) + kBlockTokens - 1) / kBlockTokens;
  bool bad = false;  // a block id outside the pool

  // ---- staging ----
  // Piece k of a thread is piece x = k kThreads + tid of the step's, in [K or V][block][piece] order.
  constexpr bool kOneSide = NP >= 2;  // a thread's piece k is K for k < NP / 2, V for the others, in every wavefront
  uint4 raw[NP];
  unsigned raw_scale[NP];
  int g_off[NP], s_off[NP], dst[NP][2];  // byte offsets in the tile and the scale bytes, LDS pieces
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int x = k * kThreads + tid;
    const int side = kOneSide ? k / (NP / 2 + (NP < 2)) : x / (kStageBlocks * D);
    const int blk = x / D % kStageBlocks;
    const int pc = x % D;
    g_off[k] = 16 * pc;
    if (side == 0) {
      const int slot = pc % 16, kg = pc / 16 % 4, c = pc / 64;
      s_off[k] = slot;
#pragma unroll
      for (int h = 0; h < 2; ++h) dst[k][h] = blk * S::kBlockPieces + (8 * c + 4 * h + kg) * 16 + slot;
    } else {
      const int piece = pc % RP, kg = pc / RP % 4, j = pc / (4 * RP);
      s_off[k] = 16 + 4 * kg + 2 * j;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 4 * kg + 2 * j + e;
        dst[k][e] = blk * S::kBlockPieces + S::kTilePieces + r * RP + (piece ^ (D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1)));
      }
    }
  }
  auto side_of = [&](int k) {
    return kOneSide ? k / (NP / 2 + (NP < 2)) : __builtin_amdgcn_readfirstlane((k * kThreads + w * kWaveSize) / (kStageBlocks * D));
  };
  int ids = 0;  // lane x: the id of block 64 (block / 64) + x of the window
  auto issue = [&](int step) {
    const int j = step * kStageBlocks;
    if (j % kWaveSize == 0) ids = st.ids[j + lane];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int blk = __builtin_amdgcn_readfirstlane((k * kThreads + w * kWaveSize) / D % kStageBlocks);
      const size_t tile = (size_t)(unsigned)__builtin_amdgcn_readlane(ids, j % kWaveSize + blk) * a.num_kv_heads + g;
      const uint8_t* pool = side_of(k) == 0 ? args.k : args.v;
      const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(tile_rsrc(pool + tile * kTile, kTile), g_off[k], 0, 0);
      raw[k] = make_uint4(t[0], t[1], t[2], t[3]);
      const __amdgpu_buffer_rsrc_t rs = tile_rsrc(args.scale + tile * 32, 32);
      if (side_of(k) == 0)
        raw_scale[k] = __builtin_amdgcn_raw_buffer_load_b8(rs, s_off[k], 0, 0);
      else
        raw_scale[k] = __builtin_amdgcn_raw_buffer_load_b16(rs, s_off[k], 0, 0);
    }
  };
  auto commit = [&](int buffer, int tok0) {
    uint4* buf = st.buf[buffer][0];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const bool is_k = side_of(k) == 0;
      const float f0 = scale_of<0>(raw_scale[k]);
      const float f1 = is_k ? f0 : scale_of<1>(raw_scale[k]);
      uint4 lo = to_bf16(raw[k].x, raw[k].y, f0);
      uint4 hi = to_bf16(raw[k].z, raw[k].w, f1);
      // A zero probability would not keep a NaN or an infinity from a row that does not see
      // its token: values past the context, whatever the slots hold, and rows that hold one
      // are zeros there, and the latter make the scores of the rows that see them NaN (mask).
      if (!is_k && tok0 + kStageBlocks * kBlockTokens > l_some) {
        asm volatile("");  // a branch
        const int blk = (k * kThreads + tid) / D % kStageBlocks;
        const int at = blk * kBlockTokens + s_off[k] - 16, t = tok0 + at;
        const unsigned s0 = raw_scale[k] & 255u, s1 = raw_scale[k] >> 8 & 255u;
        bool dead0 = s0 == 255u, dead1 = s1 == 255u;
        if (__builtin_amdgcn_ballot_w64(max(s0, s1) >= kLargeScale) != 0) {  // rows that hold an infinity: in RP lanes
          const uint64_t h0 = __builtin_amdgcn_ballot_w64(infinite(raw[k].x, s0) || infinite(raw[k].y, s0));
          const uint64_t h1 = __builtin_amdgcn_ballot_w64(infinite(raw[k].z, s1) || infinite(raw[k].w, s1));
          const int first = lane / RP * RP;
          dead0 |= (h0 >> first & ((1u << RP) - 1)) != 0, dead1 |= (h1 >> first & ((1u << RP) - 1)) != 0;
        }
        if (t >= L || dead0) lo = make_uint4(0u, 0u, 0u, 0u);
        if (t + 1 >= L || dead1) hi = make_uint4(0u, 0u, 0u, 0u);
        st.dead[buffer][at] = dead0, st.dead[buffer][at + 1] = dead1;  // (the same from every thread of the row)
      }
      buf[dst[k][0]] = lo;
      buf[dst[k][1]] = hi;
    }
  };

  typedef short v4s_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
  const int k_piece = (col >> 4) * S::kBlockPieces + hh * 16 + (lane & 15);
  // transposed V reads: source lane s of each 16 points at row 4 hh + s / 4, columns 16 u + 4 (s % 4)
  const int s16 = lane & 15;
  const int tr_row = (4 * hh + s16 / 4) * D + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3);
  int tr_off[VT];  // (with the row's permutation of pieces)
#pragma unroll
  for (int t = 0; t < VT; ++t) tr_off[t] = tr_row + 32 * (t ^ (D == 128 ? s16 / 4 : s16 / 8));

  f32x16_t s;  // scores of the step to fold: reg i is token tok0 + 8 (i / 4) + 4 hh + i % 4
  float top;   // the largest of them
  auto scores = [&](const uint4* blocks) {
    f32x16_t x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
    for (int c = 0; c < KS; ++c)
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, blocks[k_piece + 32 * c]), q[c], x, 0, 0, 0);
    return x;
  };
  auto largest = [&] {
    float x = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int i = 3; i + 1 < 15; i += 2) x = max3(x, s[i], s[i + 1]);
    top = max3(x, s[15], s[15]);
    asm volatile("" : "+v"(top));  // the MFMA results are first read in their own basic block
  };
  auto mask = [&](int buffer, int tok0) {
    if (tok0 + 32 > l_some) {  // some row of the workgroup does not see some of these tokens
      asm volatile("");  // a branch: as selects the masking would run on every step
      const int rel = limit - (tok0 + 4 * hh);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (st.dead[buffer][8 * (i / 4) + 4 * hh + i % 4]) s[i] = __builtin_nanf("");
        if (8 * (i / 4) + i % 4 >= rel) s[i] = -__builtin_huge_valf();
      }
      largest();
    }
  };
  // Fold the step whose scores are in s (two blocks of a buffer), and form the
  // scores of the next one.
  auto fold = [&](int tok0, int buffer, int next) {
    const uint4 *blocks = st.buf[buffer][0], *next_blocks = st.buf[next][0];
    if constexpr (!kAhead) {
      s = scores(blocks);
      largest();
      mask(buffer, tok0);
    }
    auto v_frag = [&](int m, int t) {
      const uint16_t* v0 = reinterpret_cast<const uint16_t*>(blocks + S::kTilePieces + m * S::kBlockPieces) + tr_off[t];
      const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)v0));
      const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(v0 + 8 * D)));
      return make_uint4(x.x, x.y, y.x, y.y);
    };
    uint4 vf[2][VT];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < VT; ++t) vf[m][t] = v_frag(m, t);
    if (__builtin_amdgcn_ballot_w64(fmaf(top, scale, -m_run) > 8.f) != 0) {
      const float m_new = fmaxf(m_run, __builtin_ceilf(mul_rounded(fmaxf(top, __shfl_xor(top, 32)), scale)));
      const float al = exp2_fast(m_run - m_new);
      m_run = m_new;
      l_run *= al;
#pragma unroll
      for (int t = 0; t < VT; ++t) o[t] *= al;
    }
    f32x16_t ns;
    if constexpr (kAhead) ns = scores(next_blocks);
    // Each probability as two bf16 halves, both rounded to nearest: hi = bf16(p), lo
    // = bf16(p - hi), at most 2^-17 of p off: 2.5e-6 of the result's norm.  A third part
    // (3e-7) takes 24% longer in chunks (32 x 512 new tokens 1565 -> 1935 us) and 15% at
    // up to 64 rows (256 x 16 327 -> 375).
    bf16x8_t bh[2], bl[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float pr[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] = exp2_fast(fmaf(s[8 * m + i], scale, -m_run));
      l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
      unsigned hw[4], lw[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const bf16x2_t h2 = {(__bf16)pr[2 * h], (__bf16)pr[2 * h + 1]};
        hw[h] = __builtin_bit_cast(unsigned, h2);
        asm("" : "+v"(hw[h]));  // (one conversion for both uses)
        const bf16x2_t l2 = {(__bf16)(pr[2 * h] - __uint_as_float(hw[h] << 16)),
                             (__bf16)(pr[2 * h + 1] - __uint_as_float(hw[h] & 0xffff0000u))};
        lw[h] = __builtin_bit_cast(unsigned, l2);
      }
      bh[m] = __builtin_bit_cast(bf16x8_t, make_uint4(hw[0], hw[1], hw[2], hw[3]));
      bl[m] = __builtin_bit_cast(bf16x8_t, make_uint4(lw[0], lw[1], lw[2], lw[3]));
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        const bf16x8_t av = __builtin_bit_cast(bf16x8_t, vf[m][t]);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, bh[m], o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, bl[m], o[t], 0, 0, 0);
      }
    if constexpr (kAhead) {
      s = ns;
      largest();
      mask(next, tok0 + 32);
    }
  };

  for (int jw = J0; jw < J1; jw += kWindow) {
    const int jwe = min(J1, jw + kWindow);
    const int nsteps = (jwe - jw + kStageBlocks - 1) / kStageBlocks;
    const int n_ids = (nsteps * kStageBlocks + kWaveSize - 1) / kWaveSize * kWaveSize;  // (they are read 64 at a time)
    for (int x = tid; x < n_ids; x += kThreads) {
      const int id = table_row[min(jw + x, jwe - 1)];  // past the end: the last block again (masked)
      const bool ok = (unsigned)id < (unsigned)a.num_blocks;  // never read outside the pool
      bad |= !ok;
      st.ids[x] = ok ? id : 0;
    }
    __syncthreads();
    const int tok_w = jw * kBlockTokens;
    constexpr int kStaged = kBuffers - 1;  // steps written before they are folded
#pragma unroll
    for (int x = 0; x < kStaged; ++x)
      if (x < nsteps) {
        issue(x);
        commit(x, tok_w + 32 * x);
      }
    if (kStaged < nsteps) issue(kStaged);
    __syncthreads();
    if (kAhead && active) {
      s = scores(st.buf[0][0]);
      largest();
      mask(0, tok_w);
    }
    // Step `step` is in buffer B = step % kBuffers (a constant, and so are all LDS
    // addresses: the loop is unrolled by the buffers).  False at the last step.
    auto one = [&](auto B, int step) {
      const int tok0 = tok_w + 32 * step;
      // behind the barrier the last step's buffer is free, and what this step reads is written
      if (step > 0) __syncthreads();
      if (step + kStaged < nsteps) commit((B + kStaged) % kBuffers, tok0 + 32 * kStaged);
      if (step + kBuffers < nsteps) issue(step + kBuffers);
      if (active && tok0 < l_vis) fold(tok0, B, (B + 1) % kBuffers);  // wavefront-uniform
      return step + 1 < nsteps;
    };
    for (int step = 0;; step += kBuffers) {
      if (!one(std::integral_constant<int, 0>{}, step)) break;
      if (!one(std::integral_constant<int, 1>{}, step + 1)) break;
      if constexpr (kBuffers == 3)
        if (!one(std::integral_constant<int, 2>{}, step + 2)) break;
    }
    __syncthreads();
  }
  const bool any_bad = __syncthreads_or(bad ? 1 : 0) != 0;  // (and the staging area is free)

  l_run += __shfl_xor(l_run, 32);
  auto parts_of = [&](int x) {
    const int lv = limit_of(x);
    return lv > 0 ? (lv + Tp - 1) / Tp : 0;
  };
  const int my_parts = parts_of(my_x);
  const bool single = my_parts == 1;
  const float mul = any_bad ? __builtin_nanf("") : single && l_run > 0.f ? 1.f / l_run : 1.f;
  constexpr int UH = D / 8;               // 16-byte units of half a row
  const int swz = col & (UH - 1);         // permuted: conflict-free
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int t = 0; t < VT / 2; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x16_t& v = o[half * (VT / 2) + t];
        st.o[w][col][(8 * t + 2 * k + hh) ^ swz] = f32x4_t{v[4 * k] * mul, v[4 * k + 1] * mul, v[4 * k + 2] * mul, v[4 * k + 3] * mul};
      }
    __syncthreads();
    if (!active) continue;
    for (int x = lane; x < kTileRows * UH; x += kWaveSize) {
      const int r32 = x / UH, u = x % UH;
      const int xr = x0 + r32;
      if (xr >= wg_rows) continue;
      const int parts = parts_of(xr);
      if (p >= parts) continue;  // the row sees nothing in this partition
      const size_t row = out_row(xr);
      const int d0 = half * (D / 2) + 4 * u;
      const f32x4_t v = st.o[w][r32][u ^ (r32 & (UH - 1))];
      if (parts == 1)
        store_nt4(a.out + row * D + d0, v[0], v[1], v[2], v[3]);
      else
        *reinterpret_cast<f32x4_t*>(a.part_o + (row * a.slots_per_row + p) * D + d0) = v;
    }
  }
  if (active && hh == 0 && x0 + col < wg_rows && p < my_parts && !single) {
    const size_t slot = out_row(my_x) * a.slots_per_row + p;
    a.part_m[slot] = m_run;
    a.part_l[slot] = l_run;
  }
}

template <int D>
hipError_t launch_d(const DecodeFp8Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.step.num_regular_items);
  if (a.step.num_query_tokens * a.step.group <= 2 * kTileRows)
    hipLaunchKernelGGL((wide_fp8_kernel<D, 2>), grid, dim3(2 * kWaveSize), 0, stream, a);
  else
    hipLaunchKernelGGL((wide_fp8_kernel<D, 4>), grid, dim3(4 * kWaveSize), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_wide_fp8(const DecodeFp8Args& a, int head_dim, hipStream_t stream) {
  if (head_dim == 64) return launch_d<64>(a, stream);
  if (head_dim == 128) return launch_d<128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace pda
