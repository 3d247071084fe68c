// wave_ops.h -- running sums over the 64 lanes of a wave, by data-parallel
// moves between lanes (a running sum of doubles through LDS permutes takes about
// 900 cycles, this way about 150).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace msa {

// x of the lane that the DPP control names, 0 where there is none (row_mask: the
// rows of 16 lanes that take part)
template <int kCtrl, int kRowMask>
__device__ __forceinline__ int dpp_or_zero(int x) {
  return __builtin_amdgcn_update_dpp(0, x, kCtrl, kRowMask, 0xf, false);
}
template <int kCtrl, int kRowMask>
__device__ __forceinline__ double dpp_or_zero(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)dpp_or_zero<kCtrl, kRowMask>((int)(uint32_t)u);
  const uint32_t hi = (uint32_t)dpp_or_zero<kCtrl, kRowMask>((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// inclusive running sum: within rows of 16 lanes, then row by row, then half by half
template <class T>
__device__ __forceinline__ T wave_scan(T x) {
  x += dpp_or_zero<0x111, 0xf>(x);  // row_shr:1
  x += dpp_or_zero<0x112, 0xf>(x);  // row_shr:2
  x += dpp_or_zero<0x114, 0xf>(x);  // row_shr:4
  x += dpp_or_zero<0x118, 0xf>(x);  // row_shr:8
  x += dpp_or_zero<0x142, 0xa>(x);  // row_bcast:15 into rows 1 and 3
  x += dpp_or_zero<0x143, 0xc>(x);  // row_bcast:31 into rows 2 and 3
  return x;
}

__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// sum over the wave, the same in every lane
template <class T>
__device__ __forceinline__ T wave_sum(T x) {
  return lane_value(wave_scan(x), 63);
}

// x of the lane below, `first` in lane 0
__device__ __forceinline__ int lane_below(int x, int first) {
  return __builtin_amdgcn_update_dpp(first, x, 0x138, 0xf, 0xf, false);  // wave_shr:1
}
__device__ __forceinline__ double lane_below(double x, double first) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x), f = __builtin_bit_cast(uint64_t, first);
  const uint32_t lo = (uint32_t)lane_below((int)(uint32_t)u, (int)(uint32_t)f);
  const uint32_t hi = (uint32_t)lane_below((int)(uint32_t)(u >> 32), (int)(uint32_t)(f >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

}  // namespace msa
