// The 8-bit checkpoint's arithmetic, shared by the kernels that write and read it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dcp {

constexpr int kCheckpointBlock = 32;  // channels that share a power of two
__host__ __device__ inline int checkpoint_blocks(int c) { return (c + kCheckpointBlock - 1) / kCheckpointBlock; }

// The stored exponent e + 127 of a block from the largest magnitude's fp32 bits: 255 for
// one that is not finite, else in 1..248. m = 1.f 2^(E-127) < 127.5 2^e holds for
// e = E - 133 where 1.f < 127.5 / 64, and for one more otherwise; 127.5 itself rounds to
// 128 (even). e is at most 121: 64 2^122, the next code over 127 2^121, is no fp32 number.
__device__ __forceinline__ uint32_t checkpoint_exponent(uint32_t top) {
  const uint32_t e = top >> 23;
  if (e == 255) return 255;
  const uint32_t over = (top & 0x7FFFFFu) >= 0x7F0000u;  // 127.5 / 64 = 1 + 127 / 128
  return (uint32_t)min(max((int)(e + over) - 6, 1), 248);
}
// 2^-e and 2^e. Of a block that is not finite: NaN for its values, any finite factor for its codes.
__device__ __forceinline__ float checkpoint_inverse(uint32_t exponent) {
  return __uint_as_float((exponent == 255 ? 127u : 254u - exponent) << 23);
}
__device__ __forceinline__ float checkpoint_scale(uint32_t exponent) {
  return __uint_as_float(exponent == 255 ? 0x7FC00000u : exponent << 23);
}
// x 2^-e to the nearest integer of at most 127 (of a NaN -127, of no meaning)
__device__ __forceinline__ int checkpoint_code(float x, float inverse) {
  return (int)fminf(fmaxf(rintf(x * inverse), -127.0f), 127.0f);
}

}  // namespace dcp
