// Prefix sums over the lanes of a wave.
#pragma once
#include "common.h"

namespace taps {

// Inclusive prefix sums over the lanes of a wave (DPP row shifts, then row broadcasts).  64 bits
// in pieces of 22, 22 and 20 bits, whose sums fit 32: a lane crossing costs one instruction each,
// where a shuffle through LDS would cost its latency six times over.
__device__ inline uint32_t wave_scan_u32(uint32_t x) {
  int v = (int)x;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return (uint32_t)v;
}
__device__ inline uint64_t wave_scan_u64(uint64_t v) {
  const uint32_t a = wave_scan_u32((uint32_t)v & 0x3FFFFFu);
  const uint32_t b = wave_scan_u32((uint32_t)(v >> 22) & 0x3FFFFFu);
  const uint32_t c = wave_scan_u32((uint32_t)(v >> 44));
  return (uint64_t)a + ((uint64_t)b << 22) + ((uint64_t)c << 44);
}
__device__ inline uint64_t lane_u64(uint64_t v, int lane) {   // lane uniform
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
  return ((uint64_t)hi << 32) | lo;
}

}  // namespace taps
