// Blocks of 32 keys in LDS, shared by the waves of a workgroup (prefill and
// tree attention), and the direct global-to-LDS copies that fill them.
#pragma once

#include "rp_device.h"

namespace rp {

constexpr int kKeyBlk = 32;

// A staged block holds 32 K and 32 V rows in bf16. One direct copy of one wave
// fills a 1 KiB chunk of kRows rows. Row r lies in chunk r % kChunks, slot
// r / kChunks, and chunks are 32 bytes more than 1 KiB apart, so that the eight
// rows of a 16-byte K read and the four rows of a transposing V read lie in
// different banks (no conflict cycles by the counters), at offsets that are
// immediates of the reads.
template <int D>
struct KeyStage {
  static constexpr int kRows = 512 / D;                 // rows per chunk
  static constexpr int kChunks = kKeyBlk / kRows;       // chunks of a K (or V) block
  static constexpr int kPitch = 512 + 16;               // bf16 elements between chunks
  static constexpr int kElems = kChunks * kPitch;       // a K (or V) block
  static constexpr int kStage = 2 * kElems;
  static constexpr int kPerWave = 2 * kChunks / 4;      // copies per wave and block, of four waves
  static_assert(kChunks % 4 == 0, "chunks per wave");
  __device__ static constexpr int row(int r) { return (r % kChunks) * kPitch + (r / kChunks) * D; }
};

// One direct global-to-LDS copy by a whole wave: 16 bytes per lane from
// base + off (or from the lane's own address) to lds + 16 * lane. Written in
// assembly because the compiler waits for every load in flight before any LDS
// read that follows its own form of it; wait_copies waits for as many as are
// needed.
__device__ inline void copy_to_lds(uint32_t lds, const uint16_t* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "m0", "memory");
}
__device__ inline void copy_to_lds(uint32_t lds, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds), "v"(from)
               : "m0", "memory");
}
// Waits until at most N of the wave's copies are in flight (and its LDS reads
// are done), then for the workgroup's other waves.
template <int N>
__device__ inline void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

}  // namespace rp
