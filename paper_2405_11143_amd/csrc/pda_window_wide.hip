// Attention with a sliding window and sinks (include/pda_window.h) for more than 32 query rows of
// a (sequence, KV head): chunked and fresh prefill, long drafts.
//
// The fold is that of pda_wide.hip (32-row tiles on MFMA f32_32x32x16_bf16, K and V tiles
// from memory straight to LDS, a 32-token step folded while the next one's scores are
// formed), over a list of steps: the sinks', then the window's.  A work item is
// (partition of the list, sequence, KV head, group of up to 8 chunks), one workgroup
// of 4 wavefronts of two chunks each; a wavefront leaves out the steps that none of
// its rows sees.  The items of one (sequence, KV head) run on one XCD next to each
// other: neighbouring groups see almost the same tokens, which then come from its L2.
//
// Bound by the matrix pipes (49% busy, at 1.9 GHz) and vector issue (50%) beside each other: with P in three
// bf16 parts a step is 4 products where the mathematics has 2.  512 new tokens of 32 sequences (32 / 8
// heads of 128) over a window of 1024: 551 to 568 us on different cards, 480 to 500 TFLOP/s by what the rows
// see, 1000 to 1030 by what is issued, 82 to 85% of what a large library product reaches; over whole contexts of
// 4096, where few steps are masked and a workgroup takes 128, 570 and 1140, 94%.  A barrier for every second step only: 1% less time.  With P in two parts, rounded to nearest, 485 us and
// results 2.4e-6 of their norm off instead of 4.5e-7 (plain fp32 operations: 7e-7); three parts rounded to
// nearest 570.  Before, with two parts: steps of 32 aligned tokens 10% more, rows stored through LDS 2%.
//
// A wavefront has up to 32 rows, so with 33 to 64 per KV head two of the four have none: they load, and the
// products run on half of the SIMDs.  256 contexts of 512 to 4096, a window of 1024, the same heads, against a
// gather of the tokens that are seen: 9 new ones (36 rows) 245 / 165 us, 16 (64) 259 / 173, 31 (124) 331 / 189,
// 64 (two workgroups) 596 / 224; 5 (20, pda_window.hip) 189 / 161.
#include "pda_wide.h"
#include "pda_window_internal.h"

namespace pda {
namespace {

constexpr int kXcds = kWindowXcds;
constexpr int kStep = kStageBlocks * kBlockTokens;  // tokens
static_assert(kStep == 2 * kWindowUnit && kWgChunks * 16 == kWindowWideRows, "the plan's units");

template <int D>
__global__ void __launch_bounds__(kWaves * kWaveSize) __attribute__((amdgpu_waves_per_eu(2)))
window_wide_kernel(const WindowArgs a) {
  using S = WideLds<D>;
  constexpr int KS = D / 16;  // score MFMA k-steps
  constexpr int VT = D / 32;  // output tiles of 32 columns
  constexpr int kTileBytes = kBlockTokens * D * 2;
  __shared__ __align__(16) S st;

  const StepArgs& sa = a.step;
  const int Hq = sa.num_q_heads, Hkv = sa.num_kv_heads, G = sa.group, n = sa.num_query_tokens;
  const int per_pair = a.num_groups * sa.num_partitions;
  const int slot = blockIdx.x / kXcds;
  const int pair = slot / per_pair * kXcds + blockIdx.x % kXcds;  // b * Hkv + g
  if (pair >= sa.num_seqs * Hkv) return;
  const int gr = slot % per_pair % a.num_groups, p = slot % per_pair / a.num_groups;
  const int g = pair % Hkv, b = pair / Hkv;
  const int tid = threadIdx.x;
  const int lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5;   // which half of the k-groups the lane holds
  const int col = lane & 31;  // the lane's row of the tile

  int L = sa.lens[b];
  L = L < 0 ? 0 : (L > sa.max_context_len ? sa.max_context_len : L);
  const int i0 = gr * a.group_tokens, i1 = min(n, i0 + a.group_tokens);
  const WindowSpan span = window_span(L, n, i0, i1, a.window, a.sinks);
  const int per_part = sa.partition_tokens / kBlockTokens;  // (even: whole steps)
  const int parts = (span.count() + per_part - 1) / per_part;
  auto out_row = [&](int i, int h) { return ((size_t)b * n + i) * Hq + (size_t)g * G + h; };
  if (p >= parts) {
    if (parts == 0 && p == 0)  // nothing to see
      for (int x = tid; x < (i1 - i0) * G * (D / 4); x += kWaves * kWaveSize) {
        const int r = x / (D / 4);
        store_nt4(sa.out + out_row(i0 + r / G, r % G) * D + 4 * (x % (D / 4)), 0.f, 0.f, 0.f, 0.f);
      }
    return;
  }

  // ---- this wavefront's tile: the new tokens [t0, t1), in chunks of query_chunk ----
  const int qc = sa.query_chunk;
  const int ta = i0 + 2 * w * qc;
  const bool active = ta < i1;
  const int t0 = active ? ta : i0, t1 = min(i1, t0 + 2 * qc);
  const int chunk0 = col < 16 || t0 + qc >= t1 ? t0 : t0 + qc;  // the lane's chunk
  const int my_rows = min(qc, t1 - chunk0) * G;
  const int my_r = (col & 15) % my_rows;  // lane rows past the chunk's last one repeat real rows
  const int my_i = chunk0 + my_r / G;
  const int up = L - n + 1 + my_i, low = window_start(up, a.window);
  // of all rows of the tile
  const int up_min = L - n + 1 + t0, up_max = L - n + t1;
  const int low_min = window_start(up_min, a.window), low_max = window_start(up_max, a.window);
  const int sinks = a.sinks;
  // A step is two entries of the list, v and v + 1.  By where they stand: whole, every row of the tile sees
  // every token of both (some that are so are not found: masking them changes nothing); wanted, some row sees
  // some token.
  const int at_sinks = span.sinks > 0 ? span.sinks : span.count();  // entries from block 0 on
  auto entry = [&](int block) { return max(block, span.first) - span.first + span.sinks; };  // of the window's blocks
  const int sinks_whole = min(min(sinks, max(up_min, 0)) / kBlockTokens, at_sinks);
  const int whole_from = entry((low_max + kBlockTokens - 1) / kBlockTokens), whole_to = entry(max(up_min, 0) / kBlockTokens);
  const int sinks_wanted = min((min(sinks, max(up_max, 0)) + kBlockTokens - 1) / kBlockTokens, at_sinks);
  const int wanted_from = entry(low_min / kBlockTokens), wanted_to = entry((max(up_max, 0) + kBlockTokens - 1) / kBlockTokens);
  auto whole = [&](int v) { return v + 1 < sinks_whole || (v >= whole_from && v + 1 < whole_to); };
  auto wanted = [&](int v) { return active && (v < sinks_wanted || (v + 1 >= wanted_from && v < wanted_to)); };
  // The first tokens of its blocks (past the list's end: past every row).
  struct Step {
    int a, b;
  };
  auto step_of = [&](int v) { return Step{span.token(v), v + 1 < span.count() ? span.token(v + 1) : span.end * kBlockTokens}; };
  // The first x of 32 bits (all, or none).
  auto first_bits = [](int x) { return x >= 32 ? 0xffffffffu : (1u << max(x, 0)) - 1u; };
  // Bit c: whether a row with these limits sees token c + 4 hh of the step.
  auto seen_bits = [&](Step k, int up_, int low_) {
    auto from = [&](int base) { return first_bits(up_ - base) & (first_bits(sinks - base) | ~first_bits(low_ - base)); };
    return (from(k.a + 4 * hh) & 0x0000ffffu) | (from(k.b - kBlockTokens + 4 * hh) & 0xffff0000u);
  };

  float scale = sa.scale_log2;
  const unsigned flip = scale < 0.f ? 0x80008000u : 0u;
  const unsigned keep = scale == 0.f ? 0u : 0xffffffffu;  // a zero scale: zero scores, whatever is masked
  scale = keep ? fabsf(scale) : 1.f;
  bf16x8_t q[KS];
  {
    const uint16_t* qp = sa.q + out_row(my_i, my_r % G) * D + 8 * hh;
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
  // The running maximum before scaling, and scaled and rounded (as in pda_wide.hip).  The rounding, up to
  // kExactMax by 2^-18, comes between the steps that take their probabilities against the one and the other:
  // more than P's 24 bits resolve, and what fp32 operations do to each score of that size once (results with scores
  // of up to 90: 7.0e-7 of their norm off, plain fp32 operations 8.0e-7).
  float m_raw = fmaxf(-1e30f / scale, -__FLT_MAX__), m_run = mul_rounded(m_raw, scale), l_run = 0.f;

  const char* kpool = reinterpret_cast<const char*>(sa.k) + (size_t)g * kTileBytes;
  const char* vpool = reinterpret_cast<const char*>(sa.v) + (size_t)g * kTileBytes;
  const int32_t* table_row = sa.table + (size_t)b * sa.max_blocks_per_seq;
  const size_t block_bytes = (size_t)Hkv * kTileBytes;
  bool bad = false;  // a block id outside the pool, anywhere the item looks

  // Staging, as in pda_wide.hip: 1 KiB of a tile per load instruction, K as it lies in
  // memory, the 16-byte pieces of a V row permuted for the transposed reads.
  constexpr int KPT = kTileBytes / 1024;
  constexpr int kStepLoads = kStageBlocks * 2 * KPT / kWaves;  // per wavefront
  constexpr int RP = D / 8;                                    // pieces of a V row
  const int k_load = (w % KPT) * 1024 + lane * 16;
  const int v_row = lane / RP;
  const int v_load = (w % KPT) * 1024 + v_row * (2 * D) + 16 * ((lane % RP) ^ (D == 128 ? 4 * (v_row & 3) : 4 * ((v_row >> 1) & 1)));
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)&st.buf[0][0][0]) +
                        (w % KPT) * 1024;
  int ids = 0;  // lane x: the id of block 64 (block / 64) + x of the ids held in LDS
  auto issue = [&](int step) {
    const int j = min(step * kStageBlocks, kWindow - kStageBlocks);  // steps past them load what nothing folds
    if (j % kWaveSize == 0) ids = st.ids[j + lane];
    const unsigned dst = lds0 + (step % kBuffers) * (kStageBlocks * S::kBlockPieces * 16);
#pragma unroll
    for (int s = 0; s < kStageBlocks; ++s) {
      if (KPT * 2 == kWaves && (w >> 1) != s) continue;  // D = 64
      const size_t off = (size_t)(unsigned)__builtin_amdgcn_readlane(ids, j % kWaveSize + s) * block_bytes;
      const unsigned at = dst + s * (S::kBlockPieces * 16);
      load_to_lds(kpool + off, k_load, at, vpool + off, v_load, at + kTileBytes);
    }
  };

  typedef short v4s_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
  const int k_piece = (col >> 4) * S::kBlockPieces + hh * 16 + (lane & 15);
  const int s16 = lane & 15;
  const int tr_row = (4 * hh + s16 / 4) * D + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3);
  int tr_off[VT];  // (with the row's permutation of pieces)
#pragma unroll
  for (int t = 0; t < VT; ++t) tr_off[t] = tr_row + 32 * (t ^ (D == 128 ? s16 / 4 : s16 / 8));

  f32x16_t s;  // scores of the step to fold: reg i is token tok0 + 8 (i / 4) + 4 hh + i % 4
  float top;   // the largest of them
  auto k_frags = [&](const uint4* blocks, uint4(&kf)[KS]) {
#pragma unroll
    for (int c = 0; c < KS; ++c) kf[c] = blocks[k_piece + 32 * c];
  };
  auto scores = [&](const uint4(&kf)[KS]) {
    f32x16_t x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
    for (int c = 0; c < KS; ++c)
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[c]), q[c], x, 0, 0, 0);
    return x;
  };
  auto largest = [&] {
    float x = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int i = 3; i + 1 < 15; i += 2) x = max3(x, s[i], s[i + 1]);
    top = max3(x, s[15], s[15]);
    asm volatile("" : "+v"(top));  // the MFMA results are first read in their own basic block
  };
  auto mask = [&](int v) {
    if (!whole(v)) {  // wavefront-uniform: some row does not see some of these tokens
      asm volatile("");  // a branch: as selects the masking would run on every step
      const unsigned seen = seen_bits(step_of(v), up, low);  // then two instructions a score
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)seen, 8 * (i / 4) + i % 4, 1);
        s[i] = __uint_as_float((__float_as_uint(s[i]) & m) | (0xff800000u & ~m));
      }
      largest();
    }
  };
  // 0xffff for every half of x that is an infinity or NaN, as bf16
  auto odd_halves = [](unsigned x) {
    return ((x & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
  };
  // Fold the step whose scores are in s (two blocks of a buffer), and form the scores of
  // the next one.
  auto fold = [&](int v, const uint4* blocks, const uint4* next_blocks) {
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
    uint4 kf[KS];  // read here, not where they are used: the products would wait for each in turn
    k_frags(next_blocks, kf);
    __builtin_amdgcn_sched_barrier(0);
    // Where every element is finite, a token's probability of 0 leaves it out of a row that does not see it.
    bool odd = false;
    if (!whole(v)) {  // wavefront-uniform
      asm volatile("");
      typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
      u16x2_t top16 = {0, 0};
      auto word = [&](unsigned x) { top16 = __builtin_elementwise_max(top16, __builtin_bit_cast(u16x2_t, x & 0x7fff7fffu)); };
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < VT; ++t) word(vf[m][t].x), word(vf[m][t].y), word(vf[m][t].z), word(vf[m][t].w);
      odd = top16[0] >= 0x7f80 || top16[1] >= 0x7f80;
    }
    int any = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_ballot_w64(odd) != 0 ? 1 : 0);
    if (any) {
      const Step at = step_of(v);
      // Infinities and NaN of tokens that only some rows see are left out of the product, and make the
      // rows that do see them NaN there, a token at a time (v - v is 0 for the others).
#pragma unroll 1
      for (int x = 0; x < kStep; ++x) {
        const int t = x < kBlockTokens ? at.a + x : at.b + x - kBlockTokens;
        if (!(t < up_max && (t < sinks || t >= low_min)) || (t < up_min && (t < sinks || t >= low_max))) continue;
        const bool mine = t < up && (t < sinks || t >= low);
        const int perm = D == 128 ? 4 * (x & 3) : 4 * ((x >> 1) & 1);
        const uint2* row = reinterpret_cast<const uint2*>(blocks + (x / 16) * S::kBlockPieces + S::kTilePieces + (x % 16) * RP);
#pragma unroll
        for (int u = 0; u < VT; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint2 v = row[2 * ((4 * u + k) ^ perm) + hh];  // columns 32 u + 8 k + 4 hh .. + 3
            const float vv[4] = {__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                                 __uint_as_float(v.y & 0xffff0000u)};
#pragma unroll
            for (int e = 0; e < 4; ++e) o[u][4 * k + e] = mine ? o[u][4 * k + e] + (vv[e] - vv[e]) : o[u][4 * k + e];
            __builtin_amdgcn_sched_barrier(0);
          }
      }
    }
    asm volatile("" ::: "memory");  // (two branches of their own: as one they spilled 76 bytes a lane)
    any = __builtin_amdgcn_readfirstlane(any);
    if (any) {
      const Step at = step_of(v);  // (V rows that no row of the tile sees are zeroed)
      const unsigned some = seen_bits(at, up_max, low_min), every = seen_bits(at, up_min, low_max);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          // word h of fragment m: tokens 16 m + {0, 2, 8, 10} + 4 hh, and the ones after
          const int c = 16 * m + 8 * (h / 2) + 2 * (h % 2);
          auto halves = [&](unsigned b) {
            return ((unsigned)__builtin_amdgcn_sbfe((int)b, c, 1) & 0x0000ffffu) |
                   ((unsigned)__builtin_amdgcn_sbfe((int)b, c + 1, 1) & 0xffff0000u);
          };
          const unsigned seen = halves(some), by_all = halves(every);
#pragma unroll
          for (int t = 0; t < VT; ++t) {
            unsigned& v = h == 0 ? vf[m][t].x : h == 1 ? vf[m][t].y : h == 2 ? vf[m][t].z : vf[m][t].w;
            v &= seen & (by_all | ~odd_halves(v));
          }
        }
    }
    float ref = m_run;
    if (__builtin_amdgcn_ballot_w64(fmaf(top, scale, -m_run) > 8.f || fabsf(m_run) > kExactMax) != 0) {
      const float mn = fmaxf(m_raw, fmaxf(top, __shfl_xor(top, 32)));
      const float al = exp2_fast((m_raw - mn) * scale);
      m_raw = mn;
      m_run = mul_rounded(mn, scale);
      ref = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] -= m_raw;
      l_run *= al;
#pragma unroll
      for (int t = 0; t < VT; ++t) o[t] *= al;
    }
    const f32x16_t ns = scores(kf);
    // The probabilities in three bf16 parts, all 24 bits: cut off, so that what is left is exact.
    bf16x8_t part[2][3];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float pr[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] = exp2_fast(fmaf(s[8 * m + i], scale, -ref));
      l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
      for (int x = 0; x < 3; ++x) {
        unsigned w[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          w[h] = pack_halves(__float_as_uint(pr[2 * h]), __float_as_uint(pr[2 * h + 1]), true);
          if (x == 2) continue;
          pr[2 * h] -= __uint_as_float(__float_as_uint(pr[2 * h]) & 0xffff0000u);
          pr[2 * h + 1] -= __uint_as_float(__float_as_uint(pr[2 * h + 1]) & 0xffff0000u);
        }
        part[m][x] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int x = 0; x < 3; ++x)
          o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf[m][t]), part[m][x], o[t], 0, 0, 0);
    s = ns;
    largest();
    mask(v + kStageBlocks);
  };

  const int v_end = min(span.count(), (p + 1) * per_part);
  for (int vw = p * per_part; vw < v_end; vw += kWindow) {
    const int nsteps = (min(v_end - vw, kWindow) + kStageBlocks - 1) / kStageBlocks;
    // (as many as the steps and the loads issued past them read, by 64)
    const int n_ids = min(kWindow, (nsteps * kStageBlocks + kBuffers * kStageBlocks + kWaveSize) / kWaveSize * kWaveSize);
    for (int x = tid; x < n_ids; x += kWaves * kWaveSize) {
      const int id = table_row[span.token(min(vw + x, v_end - 1)) / kBlockTokens];  // past the end: the last block again (masked, or not folded)
      const bool ok = (unsigned)id < (unsigned)sa.num_blocks;  // never read outside the pool
      bad |= !ok;
      st.ids[x] = ok ? id : 0;
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kBuffers - 1; ++x) issue(x);
    bool ready = false;  // the scores of the step at hand are formed
    for (int step = 0; step < nsteps; ++step) {
      // the next step's loads of this wavefront, and behind the barrier those
      // of the others; the last step's buffer is free then
      wait_loads<(kBuffers - 3) * kStepLoads>();
      __syncthreads();
      issue(step + kBuffers - 1);
      const int v = vw + kStageBlocks * step;
      if (!wanted(v)) {  // wavefront-uniform
        ready = false;
        continue;
      }
      if (!ready) {
        uint4 kf[KS];
        k_frags(st.buf[step % kBuffers][0], kf);
        s = scores(kf);
        largest();
        mask(v);
      }
      fold(v, st.buf[step % kBuffers][0], st.buf[(step + 1) % kBuffers][0]);
      ready = true;
    }
    wait_loads<0>();
    __syncthreads();
  }
  const bool any_bad = __syncthreads_or(bad ? 1 : 0) != 0;  // (and the staging area is free)

  l_run += __shfl_xor(l_run, 32);
  const float mul = any_bad ? __builtin_nanf("") : parts == 1 && l_run > 0.f ? 1.f / l_run : 1.f;
  if (!active) return;
  // Straight from the registers, 32 bytes of a row by two lanes at a time: L2 puts the
  // lines together (through LDS in whole lines 1-7% longer, with the non-temporal hint 5-50%).
  const bool real = (col & 15) < my_rows && (col < 16 || t0 + qc < t1);
  const size_t my_row = out_row(my_i, my_r % G);
  if (real) {
    float* dst = (parts == 1 ? sa.out + my_row * D : sa.part_o + (my_row * sa.slots_per_row + p) * D) + 4 * hh;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f32x4_t*>(dst + 32 * t + 8 * k) =
            f32x4_t{o[t][4 * k] * mul, o[t][4 * k + 1] * mul, o[t][4 * k + 2] * mul, o[t][4 * k + 3] * mul};
  }
  if (parts > 1 && real && hh == 0) {
    sa.part_m[my_row * sa.slots_per_row + p] = m_run;
    sa.part_l[my_row * sa.slots_per_row + p] = l_run;
  }
}

}  // namespace

hipError_t launch_window_wide(const WindowArgs& a, int head_dim, hipStream_t stream) {
  const unsigned pairs = (unsigned)a.step.num_seqs * (unsigned)a.step.num_kv_heads;
  const dim3 grid((pairs + kXcds - 1) / kXcds * kXcds * (unsigned)a.num_groups * (unsigned)a.step.num_partitions);
  const dim3 threads(kWaves * kWaveSize);
  if (head_dim == 64)
    hipLaunchKernelGGL(window_wide_kernel<64>, grid, threads, 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL(window_wide_kernel<128>, grid, threads, 0, stream, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pda
