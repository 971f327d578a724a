// Relative position encoding of the pair track and its tables' gradient (gfx950).
// (Appendix, relative-position sub-chunking: one-hots of the residue and token offsets
// clipped to +-32, the chain hop clipped to +-2 and the same entity, then a linear layer;
// the product of a one-hot with a table is a row of the table, so no one-hot is formed.)
//
//   bucket_f(i, j) = clamp(position_f[i] - position_f[j], -r_f, r_f) + r_f   in one group of field f,
//                    2 r_f + 1                                             in different ones,
//   z_out[i, j] = z_in[i, j] + sum over f of table[first_f + bucket_f(i, j)],
//   dtable[first_f + b] = sum over the pairs of bucket b of dz[i, j].
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

// The bucket of tokens with positions p, q in groups g, h. The difference of two int32 fits 64 bits.
__device__ __forceinline__ uint32_t bucket_of(int32_t p, int32_t q, int32_t g, int32_t h, int32_t r) {
  const int64_t d = (int64_t)p - q;
  const int32_t clipped = d > r ? r : d < -r ? -r : (int32_t)d;
  return (uint32_t)(g == h ? clipped + r : 2 * r + 1);
}

// Buckets of a pair, a byte per field (at most 2 * 127 + 1)
__device__ __forceinline__ uint32_t buckets_of(const RelativeArgs& a, int64_t i, int64_t j) {
  uint32_t t = 0;
#pragma unroll
  for (int f = 0; f < kRelativeFields; ++f)
    if (f < a.n_fields) {
      const int32_t* group = a.group[f];
      t |= bucket_of(a.position[f][i], a.position[f][j], group ? group[i] : 0, group ? group[j] : 0, a.radius[f]) << (8 * f);
    }
  return t;
}

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_f32(float v, float* p) { *p = v; }
__device__ __forceinline__ void store_f32(float v, uint16_t* p) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// One wave per 64 pairs of a row, a lane per channel and 64 channels at a time: any width and alignment.
template <typename T>
__global__ void __launch_bounds__(256) relative_any_kernel(RelativeArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t blocks = (a.n_tok + 63) / 64;
  if (unit >= a.n_rows * blocks) return;
  const int64_t row = unit / blocks, j0 = (unit - row * blocks) * 64;
  const int n = (int)min((int64_t)64, a.n_tok - j0);
  const uint32_t mine = buckets_of(a, a.row0 + row, min(j0 + lane, a.n_tok - 1));
  for (int k = 0; k < n; ++k) {
    const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)mine, k);
    const int64_t at = (row * a.n_tok + j0 + k) * a.c;
    for (int c = lane; c < a.c; c += 64) {
      float sum = 0.0f;
      for (int f = 0; f < a.n_fields; ++f)
        sum += a.table[(int64_t)(a.first[f] + (int)(t >> (8 * f) & 255)) * a.c + c];
      const float z = a.z_in ? load_f32(static_cast<const T*>(a.z_in) + at + c) : 0.0f;
      store_f32(z + sum, static_cast<T*>(a.z_out) + at + c);
    }
  }
}

// One thread per channel and share of the pairs: a bucket's sum in the workspace, in order.
template <typename T>
__global__ void __launch_bounds__(64) relative_back_any_kernel(RelativeArgs a) {
  const int c = blockIdx.y * 64 + threadIdx.x;
  if (c >= a.c) return;
  float* const part = a.parts + (int64_t)blockIdx.x * a.n_buckets * a.c + c;
  for (int b = 0; b < a.n_buckets; ++b) part[(int64_t)b * a.c] = 0.0f;
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x)
    for (int64_t j = 0; j < a.n_tok; ++j) {
      const uint32_t t = buckets_of(a, a.row0 + row, j);
      const float v = load_f32(static_cast<const T*>(a.dz) + (row * a.n_tok + j) * a.c + c);
      for (int f = 0; f < a.n_fields; ++f) part[(int64_t)(a.first[f] + (int)(t >> (8 * f) & 255)) * a.c] += v;
    }
}

__global__ void __launch_bounds__(256) relative_sum_kernel(RelativeArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.n_buckets * a.c;
  if (t >= n) return;
  float sum = 0.0f;
  for (int p = 0; p < a.n_parts; ++p) sum += a.parts[p * n + t];
  a.dtable[t] = sum;
}

}  // namespace

hipError_t launch_relative(const RelativeArgs& a, bool bf16, hipStream_t st) {
  const int64_t units = a.n_rows * ((a.n_tok + 63) / 64);
  const dim3 grid((unsigned)((units + 3) / 4));
  if (bf16)
    hipLaunchKernelGGL(relative_any_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(relative_any_kernel<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

int relative_back_parts(int64_t n_tok, int64_t n_rows, int32_t c, int32_t n_buckets) {
  (void)n_tok, (void)c, (void)n_buckets;
  return (int)(n_rows < 256 ? n_rows : 256);
}

hipError_t launch_relative_back(const RelativeArgs& a, bool bf16, hipStream_t st) {
  if (a.n_parts > 0) {
    const dim3 grid((unsigned)a.n_parts, (unsigned)((a.c + 63) / 64));
    if (bf16)
      hipLaunchKernelGGL(relative_back_any_kernel<uint16_t>, grid, dim3(64), 0, st, a);
    else
      hipLaunchKernelGGL(relative_back_any_kernel<float>, grid, dim3(64), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t n = (int64_t)a.n_buckets * a.c;
  hipLaunchKernelGGL(relative_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
