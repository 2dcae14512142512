// What the kernels of 32-row tiles share (pda_wide.hip, pda_window_wide.hip): the shape of
// a workgroup, its LDS, and the loads that go straight there.
#pragma once

#include "pda_wave.h"

namespace pda {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kTileRows = 32;          // query rows of a wavefront: two 16-row chunks
constexpr int kWgChunks = 2 * kWaves;  // chunks of a workgroup
constexpr int kStageBlocks = 2;        // blocks of a staged step: 32 tokens
constexpr int kBuffers = 4;            // one step folded, the next one's scores formed, two in flight
constexpr int kWindow = 1024;          // block ids held in LDS at a time
constexpr float kExactMax = 128.f;     // running maxima that may be rounded: by up to 2^-18, as a score of their size is

template <int D>
struct WideLds {
  static constexpr int kTilePieces = 2 * D;  // 16-byte pieces of a K or V tile
  static constexpr int kBlockPieces = 2 * kTilePieces;
  union {
    uint4 buf[kBuffers][kStageBlocks][kBlockPieces];
    f32x4_t o[kWaves][kTileRows][D / 4];
  };
  int ids[kWindow];
};

// 16 bytes per lane from k + k_off and v + v_off straight into LDS, at k_lds and
// v_lds plus 16 lane.  The compiler does not count these loads: the caller waits
// with wait_loads.  (It counts the builtin's, and waits for all of them before
// every LDS read: no load would stay in flight.)  M0, which names the LDS
// address, belongs to the compiler: it gets back what it held.
__device__ __forceinline__ void load_to_lds(const char* k, int k_off, unsigned k_lds, const char* v, int v_off,
                                            unsigned v_lds) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\t"
               "s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
               "s_mov_b32 m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(m0)
               : "v"(k_off), "v"(v_off), "s"(k), "s"(v), "s"(k_lds), "s"(v_lds)
               : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

}  // namespace pda
