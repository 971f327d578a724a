// Activation checkpoints in 8 bits (gfx950): rows of bf16 or fp32 channels as int8 codes,
// every 32 consecutive channels of a row under one power of two.
//
//   e = the least integer >= -126 with rint(max |x| 2^-e) <= 127, at most 121,
//   code = rint(x 2^-e) (ties to even; at most 127), value = code 2^e, stored exponent e + 127.
//
// A power of two keeps every step exact: the quotient, the comparison with 127 and the
// value read back, which has at most 7 significant bits and so is a bf16 number too. A
// block with a NaN or an infinity has exponent 255 and reads back as NaN. The error is at
// most 2^(e-1), between 1/255 and 1/127.5 of the block's largest magnitude where e is not
// bounded: from 63.75 2^-126 to 127.5 2^121. Below it is at most 2^-127, above at most 2^121.
//
// Both directions are bound by memory (a million rows of 128 channels in bf16: 62 and 59 us, 6.6 and 6.9 TB/s with what the
// last-level cache holds). Where c is a whole number of blocks the rows are one long list of blocks: a thread
// takes 16 bytes of x, a quarter of a block in bf16 and an eighth in fp32, and the block's largest magnitude is found
// across those lanes. Other widths and alignments take a lane per channel.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"
#include "checkpoint.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void from_f32(float v, float* p) { *p = v; }
__device__ __forceinline__ void from_f32(float v, uint16_t* p) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}

constexpr int kPieces = 4;  // 16-byte pieces of x a thread has in flight

template <typename T>
__global__ void __launch_bounds__(256) pack_kernel(CheckpointArgs a, int64_t n_pieces) {
  constexpr int kVec = 16 / sizeof(T);
  const u32x4* x = static_cast<const u32x4*>(a.x);
  const int64_t first = (a.first_block + blockIdx.x) * (256 * kPieces) + threadIdx.x;
  u32x4 raw[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) raw[k] = __builtin_nontemporal_load(x + min(first + 256 * k, n_pieces - 1));
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t i = first + 256 * k;
    float v[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      v[e] = __uint_as_float(kVec == 4 ? raw[k][e & 3] : e & 1 ? raw[k][e >> 1] & 0xFFFF0000u : raw[k][e >> 1] << 16);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    top = max_dpp<0x4E>(max_dpp<0xB1>(top));      // of four lanes
    if (kVec == 4) top = max_dpp<0x141>(top);     // of eight
    const uint32_t exponent = checkpoint_exponent(top);
    const float inverse = checkpoint_inverse(exponent);
    uint32_t q[kVec / 4];
#pragma unroll
    for (int w = 0; w < kVec / 4; ++w) {
      q[w] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) q[w] |= ((uint32_t)checkpoint_code(v[4 * w + e], inverse) & 255u) << (8 * e);
    }
    if (i >= n_pieces) continue;
    if (kVec == 8)
      reinterpret_cast<u32x2*>(a.codes)[i] = u32x2{q[0], q[kVec / 4 - 1]};
    else
      reinterpret_cast<uint32_t*>(a.codes)[i] = q[0];
    constexpr int kLanes = kCheckpointBlock / kVec;
    if ((threadIdx.x & (kLanes - 1)) == 0) a.exponents[i / kLanes] = (uint8_t)exponent;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) unpack_kernel(CheckpointArgs a, int64_t n_pieces) {
  constexpr int kVec = 16 / sizeof(T), kLanes = kCheckpointBlock / kVec;
  const int64_t first = (a.first_block + blockIdx.x) * (256 * kPieces) + threadIdx.x;
  u32x2 q[kPieces];
  uint32_t exponent[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t i = min(first + 256 * k, n_pieces - 1);
    if (kVec == 8)
      q[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(a.codes) + i);
    else
      q[k][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(a.codes) + i);
    exponent[k] = a.exponents[i / kLanes];
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t i = first + 256 * k;
    const float scale = checkpoint_scale(exponent[k]);
    float v[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = (float)(int8_t)(q[k][e >> 2] >> (8 * (e & 3))) * scale;
    u32x4 o;
    if (kVec == 8) {
      bf16x8 b;
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e % kVec];
      o = __builtin_bit_cast(u32x4, b);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(v[e]);
    }
    if (i < n_pieces) __builtin_nontemporal_store(o, static_cast<u32x4*>(a.y) + i);
  }
}

// A lane per channel, 32 lanes a block: any width and alignment.
template <typename T>
__global__ void __launch_bounds__(256) pack_any_kernel(CheckpointArgs a) {
  const int64_t t = (a.first_block + blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int blocks = checkpoint_blocks(a.c);
  if (t >= a.n_rows * blocks) return;  // 32 lanes together
  const int64_t row = t / blocks;
  const int c = (int)(t - row * blocks) * kCheckpointBlock + (threadIdx.x & 31);
  const float v = c < a.c ? to_f32(static_cast<const T*>(a.x)[row * a.c + c]) : 0.0f;
  uint32_t top = __float_as_uint(v) & 0x7FFFFFFFu;
  for (int m = 16; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 32));
  const uint32_t exponent = checkpoint_exponent(top);
  if (c < a.c) a.codes[row * a.c + c] = (int8_t)checkpoint_code(v, checkpoint_inverse(exponent));
  if ((threadIdx.x & 31) == 0) a.exponents[t] = (uint8_t)exponent;
}

template <typename T>
__global__ void __launch_bounds__(256) unpack_any_kernel(CheckpointArgs a) {
  const int64_t t = (a.first_block + blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int blocks = checkpoint_blocks(a.c);
  if (t >= a.n_rows * blocks) return;
  const int64_t row = t / blocks;
  const int c = (int)(t - row * blocks) * kCheckpointBlock + (threadIdx.x & 31);
  if (c < a.c) from_f32((float)a.codes[row * a.c + c] * checkpoint_scale(a.exponents[t]), static_cast<T*>(a.y) + row * a.c + c);
}

template <typename T>
hipError_t launch(CheckpointArgs a, hipStream_t st) {
  constexpr int kVec = 16 / sizeof(T);
  const auto at = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  const bool whole = a.c % kCheckpointBlock == 0 && at(a.x, 16) && at(a.y, 16) && at(a.codes, kVec);
  const int64_t n_pieces = a.n_rows * a.c / kVec, blocks = a.n_rows * checkpoint_blocks(a.c);
  const int64_t total = whole ? (n_pieces + 256 * kPieces - 1) / (256 * kPieces) : (blocks + 7) / 8;
  hipError_t e = hipSuccess;
  for (; a.first_block < total && e == hipSuccess; a.first_block += kLaunchBlocks) {
    const dim3 grid((unsigned)(total - a.first_block < kLaunchBlocks ? total - a.first_block : kLaunchBlocks));
    if (a.x && whole)
      hipLaunchKernelGGL(pack_kernel<T>, grid, dim3(256), 0, st, a, n_pieces);
    else if (a.x)
      hipLaunchKernelGGL(pack_any_kernel<T>, grid, dim3(256), 0, st, a);
    else if (whole)
      hipLaunchKernelGGL(unpack_kernel<T>, grid, dim3(256), 0, st, a, n_pieces);
    else
      hipLaunchKernelGGL(unpack_any_kernel<T>, grid, dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_checkpoint(const CheckpointArgs& a, bool bf16, hipStream_t st) {
  return bf16 ? launch<uint16_t>(a, st) : launch<float>(a, st);
}

}  // namespace dcp
