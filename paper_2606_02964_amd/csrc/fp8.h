// fp8.h -- the 8-bit cache's format, shared by the kernels that write and read it:
// e4m3 numbers times 2^(byte - 127), a byte for each (token, KV head).
#pragma once

#include <cstdint>
#include <string>

#include "msa.h"

#ifdef __HIPCC__
#define MSA_HD __host__ __device__ __forceinline__
#else
#define MSA_HD inline
#endif

namespace msa {

constexpr uint32_t kFp8ScaleMin = 17;  // 2^-110: with e4m3's smallest, 2^-9, still a normal bf16 number

// The byte of the smallest power 2^e, e >= -110, with x <= 448 * 2^e, from the bits of
// x >= 0: 448 is 1.75 * 2^8, so e is x's own exponent less 8, and one more past 1.75.
MSA_HD uint32_t fp8_scale_byte(uint32_t x) {
  const int32_t b = (int32_t)(x >> 23) - 8 + ((x & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < (int32_t)kFp8ScaleMin ? kFp8ScaleMin : (uint32_t)b;
}

// what is wrong with a shape's cache strides for 8-bit caches, or ""
inline std::string fp8_strides(const msa_shape& s) {
  auto ok = [](int64_t x) { return x > 0 && x % 16 == 0; };
  if (ok(s.k_stride_block) && ok(s.k_stride_head) && ok(s.k_stride_tok) && ok(s.v_stride_block) &&
      ok(s.v_stride_head) && ok(s.v_stride_dim))
    return std::string();
  return "strides of 8-bit caches must be positive multiples of 16 elements";
}

}  // namespace msa
