// Activation checkpoints in 8 bits (gfx950): rows of bf16 or fp32 channels as int8 codes,
// every 32 consecutive channels of a row under one power of two.
//
//   e = the least integer >= -126 with rint(max |x| 2^-e) <= 127, at most 121,
//   code = rint(x 2^-e) (ties to even; at most 127), value = code 2^e, stored exponent e + 127.
//
// A power of two keeps every step exact: the quotient, the comparison with 127 and the
// value read back, which has at most 7 significant bits and so is a bf16 number too. A
// block with a NaN or an infinity has exponent 255 and reads back as NaN. The error is at
// most 2^(e-1), between 1/255 and 1/127.5 of the block's largest magnitude.
//
// Both directions are bound by memory.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"
#include "checkpoint.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

__device__ __forceinline__ void from_f32(float v, float* p) { *p = v; }
__device__ __forceinline__ void from_f32(float v, uint16_t* p) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// One thread per block of 32 channels, one channel at a time: any width and alignment.
template <typename T>
__global__ void __launch_bounds__(256) pack_any_kernel(CheckpointArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int blocks = checkpoint_blocks(a.c);
  if (t >= a.n_rows * blocks) return;
  const int64_t row = t / blocks;
  const int c0 = (int)(t - row * blocks) * kCheckpointBlock, n = min(kCheckpointBlock, a.c - c0);
  const T* x = static_cast<const T*>(a.x) + row * a.c + c0;
  uint32_t top = 0;
  for (int i = 0; i < n; ++i) top = max(top, __float_as_uint(to_f32(x[i])) & 0x7FFFFFFFu);
  const uint32_t e = checkpoint_exponent(top);
  const float scale = checkpoint_inverse(e);
  for (int i = 0; i < n; ++i) a.codes[row * a.c + c0 + i] = (int8_t)checkpoint_code(to_f32(x[i]), scale);
  a.exponents[t] = (uint8_t)e;
}

template <typename T>
__global__ void __launch_bounds__(256) unpack_any_kernel(CheckpointArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int blocks = checkpoint_blocks(a.c);
  if (t >= a.n_rows * blocks) return;
  const int64_t row = t / blocks;
  const int c0 = (int)(t - row * blocks) * kCheckpointBlock, n = min(kCheckpointBlock, a.c - c0);
  const float scale = checkpoint_scale(a.exponents[t]);
  T* x = static_cast<T*>(a.y) + row * a.c + c0;
  for (int i = 0; i < n; ++i) from_f32((float)a.codes[row * a.c + c0 + i] * scale, x + i);
}

}  // namespace

hipError_t launch_checkpoint_pack(const CheckpointArgs& a, bool bf16, hipStream_t st) {
  const int64_t n = a.n_rows * checkpoint_blocks(a.c);
  const dim3 grid((unsigned)((n + 255) / 256));
  if (bf16)
    hipLaunchKernelGGL(pack_any_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(pack_any_kernel<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const CheckpointArgs& a, bool bf16, hipStream_t st) {
  const int64_t n = a.n_rows * checkpoint_blocks(a.c);
  const dim3 grid((unsigned)((n + 255) / 256));
  if (bf16)
    hipLaunchKernelGGL(unpack_any_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(unpack_any_kernel<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
