// Sums over the lanes of a wavefront (paged cache).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

// Inclusive sums over the lanes of a wavefront, in the vector unit (rows of 16 lanes, then their last ones carried on).
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
#define RF2_ADD(ctrl, rows) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, true)
  RF2_ADD(0x111, 0xf);            // row_shr:1, 2, 4, 8
  RF2_ADD(0x112, 0xf);
  RF2_ADD(0x114, 0xf);
  RF2_ADD(0x118, 0xf);
  RF2_ADD(0x142, 0xa);            // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
  RF2_ADD(0x143, 0xc);
#undef RF2_ADD
  return x;
}

// The same of floats, all of them: the sum, and the least.
__device__ __forceinline__ float wave_total(float x) {
#define RF2_ADD(ctrl, rows) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, true))
  RF2_ADD(0x111, 0xf);
  RF2_ADD(0x112, 0xf);
  RF2_ADD(0x114, 0xf);
  RF2_ADD(0x118, 0xf);
  RF2_ADD(0x142, 0xa);
  RF2_ADD(0x143, 0xc);
#undef RF2_ADD
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_least(float x) {
  // (a lane without a neighbour in a step takes itself)
#define RF2_MIN(ctrl, rows) \
  x = fminf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), ctrl, rows, 0xf, false)))
  RF2_MIN(0x111, 0xf);
  RF2_MIN(0x112, 0xf);
  RF2_MIN(0x114, 0xf);
  RF2_MIN(0x118, 0xf);
  RF2_MIN(0x142, 0xa);
  RF2_MIN(0x143, 0xc);
#undef RF2_MIN
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

}  // namespace
