// Rows of the 8-bit KV cache back as bf16 (include/pda_fp8.h): bound by memory,
// 2 D + 2 bytes read and 4 D written per row and KV head.  A workgroup takes one
// block of a sequence, and a thread the same 8 elements of the same slot in every
// head (8 bytes read, 16 written), neighbouring threads neighbouring elements of
// the output, which goes out with the non-temporal hint.  64 sequences of 512-4096
// tokens, 8 KV heads of 128 (0.91 GB): 178 us, 5.1 TB/s (a large copy 4.9); threads that
// divided their way through (token, head, piece) and stored plainly took 225.
#include "pda_fp8_internal.h"

namespace pda {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups (a launch has less than 2^32 threads); they loop over the rest

template <int D>
__global__ void __launch_bounds__(kThreads) read_fp8_kernel(const ReadFp8Args a, int blocks) {
  constexpr int P = D / 8;                               // pieces per row
  constexpr int HEADS = kThreads / (P * kBlockTokens);   // heads at a time
  const int H = a.num_kv_heads;
  const int c = threadIdx.x % P, o = threadIdx.x / P % kBlockTokens, sub = threadIdx.x / (P * kBlockTokens);
  const int k_at = ((c / 8 * 4 + c % 4) * 16 + o) * 16 + c / 4 % 2 * 8;
  const int v_at = (((o / 2 % 2) * 4 + o / 4) * P + c) * 16 + o % 2 * 8;
  for (int64_t bj = blockIdx.x; bj < (int64_t)a.num_seqs * blocks; bj += gridDim.x) {
    const int b = (int)(bj / blocks);
    const int j = (int)(bj % blocks);
    const int L = clamped(a.lens[b], a.max_context_len);
    const int first = a.first ? a.first[b] : 0;
    const int64_t row0 = a.row_start[b];
    // tokens [t_lo, t_hi) of this block go to rows row0 + t - first
    const int64_t end = min((int64_t)L, first + (int64_t)a.row_start[b + 1] - row0);
    const int t_lo = max(j * kBlockTokens, first);
    const int t_hi = (int)min((int64_t)(j + 1) * kBlockTokens, end);
    const int t = j * kBlockTokens + o;
    const int64_t row = row0 + ((int64_t)t - first);
    if (t < t_lo || t >= t_hi || row < 0 || row >= a.num_rows) continue;
    const int page = a.table[(size_t)b * a.max_blocks_per_seq + j];
    const bool ok = (unsigned)page < (unsigned)a.num_blocks;
    u32x4_t* k_out = reinterpret_cast<u32x4_t*>(a.k_out) + (size_t)row * H * P + c;
    u32x4_t* v_out = reinterpret_cast<u32x4_t*>(a.v_out) + (size_t)row * H * P + c;
    const size_t tile0 = (size_t)(ok ? page : 0) * H;
#pragma unroll 1  // (by 4: 9% longer)
    for (int g = sub; g < H; g += HEADS) {
      uint4 k = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u), v = k;  // NaN
      if (ok) {
        const size_t tile = tile0 + g;
        const uint2 kc = *reinterpret_cast<const uint2*>(a.k + tile * (16 * D) + k_at);
        const uint2 vc = *reinterpret_cast<const uint2*>(a.v + tile * (16 * D) + v_at);
        const unsigned ks = a.scale[tile * 32 + o], vs = a.scale[tile * 32 + 16 + o];
        // (the conversion takes a factor of 0 for 2^-127: a byte of 0 stands for zeros whatever the codes)
        k = ks ? to_bf16(kc.x, kc.y, scale_of<0>(ks)) : make_uint4(0, 0, 0, 0);
        v = vs ? to_bf16(vc.x, vc.y, scale_of<0>(vs)) : make_uint4(0, 0, 0, 0);
      }
      __builtin_nontemporal_store(u32x4_t{k.x, k.y, k.z, k.w}, k_out + (size_t)g * P);
      __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, v_out + (size_t)g * P);
    }
  }
}

}  // namespace

hipError_t launch_read_fp8(const ReadFp8Args& a, int head_dim, hipStream_t stream) {
  const int blocks = (a.max_context_len + kBlockTokens - 1) / kBlockTokens;
  if (blocks == 0) return hipSuccess;
  const dim3 grid((unsigned)min((int64_t)a.num_seqs * blocks, kMaxGrid));
  if (head_dim == 64)
    hipLaunchKernelGGL((read_fp8_kernel<64>), grid, dim3(kThreads), 0, stream, a, blocks);
  else if (head_dim == 128)
    hipLaunchKernelGGL((read_fp8_kernel<128>), grid, dim3(kThreads), 0, stream, a, blocks);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pda
