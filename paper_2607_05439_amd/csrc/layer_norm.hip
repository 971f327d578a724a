// LayerNorm over the channels of a row, and its backward pass with the gradients
// of the affine weights (gfx950).
//
//   mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd,
//   y = gamma xh + beta;
//   g = gamma dy, dx = rstd (g - mean g - xh mean(g xh)),
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy.
//
// Both are bound by memory: the forward reads x and writes y, the backward reads x
// and dy and writes dx, each once. The statistics are formed again in the
// backward, from the row it holds in registers anyway, so nothing but x is kept.
//
// A row lies in the registers of 2^k consecutive lanes (as few as hold it in three
// 16-byte pieces each, so that a wave takes many narrow rows at once; a row wider
// than a wave takes the workgroup's 256), lane l of them holding pieces l,
// l + lanes, ...; the mean, then the centred squares, are summed in fp32 across
// those lanes. A lane's channels are the same in every row, so its
// share of dgamma and dbeta stays in registers over all rows of its workgroup;
// the workgroups' sums are added up by a second kernel in a fixed order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

constexpr int kLnWaves = 4;

// Sum over 2^k consecutive lanes (lanes = 2^k, wave-uniform); every one of them
// gets the same bits. Up to 16 lanes by row permutations inside the vector unit.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum_lanes(float x, int lanes) {
  if (lanes >= 2) x = add_dpp<0xB1>(x);    // lane ^ 1
  if (lanes >= 4) x = add_dpp<0x4E>(x);    // lane ^ 2
  if (lanes >= 8) x = add_dpp<0x141>(x);   // half-row mirror: the other four, equal among themselves
  if (lanes >= 16) x = add_dpp<0x140>(x);  // row mirror: the other eight
  if (lanes >= 32) {
    float a = x, b = x;
    swap16(a, b);
    x = a + b;
  }
  if (lanes >= 64) {
    float a = x, b = x;
    swap32(a, b);
    x = a + b;
  }
  return x;
}

// VEC consecutive elements (16 bytes, or one) as fp32.
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = (float)*p;
  } else {
    const u32x4 r = *reinterpret_cast<const u32x4*>(p);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r[i] << 16);
        v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    }
  }
}
template <int VEC>
__device__ __forceinline__ void store_vec(void* base, int64_t at, bool bf16, const float (&v)[VEC]) {
  if (bf16) {
    __bf16* p = static_cast<__bf16*>(base) + at;
    if constexpr (VEC == 1) {
      *p = (__bf16)v[0];
    } else {
      typedef __bf16 vec __attribute__((ext_vector_type(VEC)));
      vec r;
#pragma unroll
      for (int i = 0; i < VEC; ++i) r[i] = (__bf16)v[i];
      *reinterpret_cast<vec*>(p) = r;
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if constexpr (VEC == 1) {
      *p = v[0];
    } else {
#pragma unroll
      for (int i = 0; i < VEC; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    }
  }
}
template <int VEC>
__device__ __forceinline__ void load_any(const void* base, int64_t at, bool bf16, float (&v)[VEC]) {
  if (bf16) {
    if constexpr (VEC == 4) {  // half a 16-byte piece
      const u32x2 r = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(base) + at);
      v[0] = __uint_as_float(r[0] << 16), v[1] = __uint_as_float(r[0] & 0xFFFF0000u);
      v[2] = __uint_as_float(r[1] << 16), v[3] = __uint_as_float(r[1] & 0xFFFF0000u);
    } else {
      load_vec<__bf16, VEC>(static_cast<const __bf16*>(base) + at, v);
    }
  } else if constexpr (VEC == 8) {
    float a[4], b[4];
    load_vec<float, 4>(static_cast<const float*>(base) + at, a);
    load_vec<float, 4>(static_cast<const float*>(base) + at + 4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    load_vec<float, VEC>(static_cast<const float*>(base) + at, v);
  }
}

// The same over a workgroup's waves where they share a row (lanes = 256); `turn`
// picks one of two buffers, so that one barrier is enough.
__device__ __forceinline__ float sum_row(float x, int lanes, float (&red)[2][kLnWaves], int turn) {
  if (lanes <= 64) return sum_lanes(x, lanes);
  x = sum_lanes(x, 64);
  if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = x;
  __syncthreads();
  return (red[turn][0] + red[turn][1]) + (red[turn][2] + red[turn][3]);
}

// Centres the row in x and returns rstd. Channels past the row's end are 0 before
// and after.
template <int VEC, int NV>
__device__ __forceinline__ float centre(float (&x)[NV][VEC], const bool (&in)[NV], float inv_c, float eps, int lanes,
                                        float (&red)[2][kLnWaves]) {
  float s = 0.f, v = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) s += x[j][i];
  const float mu = sum_row(s, lanes, red, 0) * inv_c;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      x[j][i] = in[j] ? x[j][i] - mu : 0.f;
      v = fmaf(x[j][i], x[j][i], v);
    }
  return 1.0f / sqrtf(fmaf(sum_row(v, lanes, red, 1), inv_c, eps));
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(64 * kLnWaves) layer_norm_kernel(LayerNormArgs a) {
  __shared__ float red[2][kLnWaves];
  const int lanes = a.lanes, at = threadIdx.x & (lanes - 1), rows_at_once = 64 * kLnWaves / lanes;
  const int64_t step = (int64_t)gridDim.x * rows_at_once, first = (int64_t)blockIdx.x * rows_at_once;
  int64_t row = first + threadIdx.x / lanes;
  int ch[NV];
  bool in[NV];
  float gamma[NV][VEC], beta[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    ch[j] = (j * lanes + at) * VEC;
    in[j] = ch[j] < a.c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      gamma[j][i] = a.gamma && in[j] ? a.gamma[ch[j] + i] : 1.f;
      beta[j][i] = a.beta && in[j] ? a.beta[ch[j] + i] : 0.f;
    }
  }
  const float inv_c = 1.0f / (float)a.c;
  // every lane runs the same rounds: the sums need all lanes of a row, and rows past
  // the last read the last one and write nothing
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step, row += step) {
    const int64_t off = min(row, a.n_rows - 1) * a.c;
    float x[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (in[j]) {
        load_vec<T, VEC>(static_cast<const T*>(a.x) + off + ch[j], x[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[j][i] = 0.f;
      }
    }
    const float rstd = centre<VEC, NV>(x, in, inv_c, a.eps, lanes, red);
    if (row < a.n_rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = fmaf(x[j][i] * rstd, gamma[j][i], beta[j][i]);
        if (in[j]) store_vec<VEC>(a.y, off + ch[j], a.y_bf16, y);
      }
    }
  }
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(64 * kLnWaves) layer_norm_back_kernel(LayerNormBackArgs a) {
  __shared__ float red[2][kLnWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lanes = a.lanes;
  const int at = threadIdx.x & (lanes - 1), rows_at_once = 64 * kLnWaves / lanes;
  const int64_t step = (int64_t)gridDim.x * rows_at_once, first = (int64_t)blockIdx.x * rows_at_once;
  int64_t row = first + threadIdx.x / lanes;
  int ch[NV];
  bool in[NV];
  float gamma[NV][VEC], dgamma[NV][VEC], dbeta[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    ch[j] = (j * lanes + at) * VEC;
    in[j] = ch[j] < a.c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      gamma[j][i] = a.gamma && in[j] ? a.gamma[ch[j] + i] : 1.f;
      dgamma[j][i] = dbeta[j][i] = 0.f;
    }
  }
  const float inv_c = 1.0f / (float)a.c;
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step, row += step) {
    const int64_t off = min(row, a.n_rows - 1) * a.c;
    const bool real = row < a.n_rows;
    float x[NV][VEC], dy[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (in[j]) {
        load_vec<T, VEC>(static_cast<const T*>(a.x) + off + ch[j], x[j]);
        load_any<VEC>(a.dy, off + ch[j], a.dy_bf16, dy[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[j][i] = dy[j][i] = 0.f;
      }
    }
    const float rstd = centre<VEC, NV>(x, in, inv_c, a.eps, lanes, red);
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        // g as rounded here is what the mean is taken of: no fusing of its product into
        // the difference below, which is 0 for a single channel
#pragma clang fp contract(off)
        const float xh = x[j][i] * rstd, g = dy[j][i] * gamma[j][i];
        if (real) {
          dgamma[j][i] = fmaf(dy[j][i], xh, dgamma[j][i]);
          dbeta[j][i] += dy[j][i];
        }
        x[j][i] = xh;
        dy[j][i] = g;
        sg += g;
        sgx = fmaf(g, xh, sgx);
      }
    const float mg = sum_row(sg, lanes, red, 0) * inv_c, mgx = sum_row(sgx, lanes, red, 1) * inv_c;
    if (a.dx && real) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float dx[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) dx[i] = rstd * fmaf(-x[j][i], mgx, dy[j][i] - mg);
        if (in[j]) store_vec<VEC>(a.dx, off + ch[j], sizeof(T) == 2, dx);
      }
    }
  }
  if (!a.parts) return;  // the whole grid
  // the rows of a wave, then its waves, last to first
  extern __shared__ float s_part[];  // [2][c]
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      for (int o = lanes; o < 64; o <<= 1) {
        dgamma[j][i] += __shfl_xor(dgamma[j][i], o);
        dbeta[j][i] += __shfl_xor(dbeta[j][i], o);
      }
  const bool alone = lanes == 64 * kLnWaves;  // a channel lies in one lane of one wave
  for (int w = alone ? 0 : kLnWaves - 1; w >= 0; --w) {
    if (alone || (wave == w && lane < lanes)) {
      float* out = w > 0 ? s_part : a.parts + (int64_t)blockIdx.x * 2 * a.c;
      const bool begin = alone || w == kLnWaves - 1;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (in[j]) {
            const int x = ch[j] + i;
            out[x] = begin ? dgamma[j][i] : dgamma[j][i] + s_part[x];
            out[a.c + x] = begin ? dbeta[j][i] : dbeta[j][i] + s_part[a.c + x];
          }
    }
    __syncthreads();
  }
}

// Column sums of parts[n_parts][2 c]: a workgroup takes 16 columns, its 16 groups of
// 16 lanes every 16th part each.
__global__ void __launch_bounds__(256) layer_norm_sum_kernel(const float* parts, int n_parts, int c, float* dgamma,
                                                            float* dbeta) {
  __shared__ float s[16][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), grp = threadIdx.x >> 4;
  float x = 0.f;
  if (col < 2 * c)
    for (int p = grp; p < n_parts; p += 16) x += parts[(int64_t)p * 2 * c + col];
  s[grp][threadIdx.x & 15] = x;
  __syncthreads();
  if (grp > 0 || col >= 2 * c) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) x += s[i][threadIdx.x];
  float* out = col < c ? dgamma : dbeta;
  if (out) out[col < c ? col : col - c] = x;
}

// Lanes of a row and pieces per lane.
struct LnSplit {
  int lanes, pieces;
};
LnSplit ln_split(int c, int vec) {
  const int chunks = (c + vec - 1) / vec;
  int lanes = 1;
  while (lanes < 64 && lanes * 3 < chunks) lanes *= 2;
  if (lanes * 3 < chunks) lanes = 64 * kLnWaves;
  return {lanes, (chunks + lanes - 1) / lanes};
}

template <typename T, int VEC, int NV>
hipError_t ln_go(const LayerNormArgs& a, int64_t groups, hipStream_t st) {
  hipLaunchKernelGGL((layer_norm_kernel<T, VEC, NV>), dim3((unsigned)groups), dim3(64 * kLnWaves), 0, st, a);
  return hipGetLastError();
}
template <typename T, int VEC, int NV>
hipError_t ln_go(const LayerNormBackArgs& a, int64_t groups, hipStream_t st) {
  const size_t lds = a.parts ? (size_t)2 * a.c * sizeof(float) : 0;
  hipLaunchKernelGGL((layer_norm_back_kernel<T, VEC, NV>), dim3((unsigned)groups), dim3(64 * kLnWaves), lds, st, a);
  return hipGetLastError();
}
template <typename T, int VEC, typename Args>
hipError_t ln_pieces(const Args& a, int pieces, int64_t groups, hipStream_t st) {
  if (pieces <= 1) return ln_go<T, VEC, 1>(a, groups, st);
  if (pieces <= 2) return ln_go<T, VEC, 2>(a, groups, st);
  if (pieces <= 3) return ln_go<T, VEC, 3>(a, groups, st);
  // c <= kLnMaxC: 512 pieces of 8, 1024 of 4 or 4096 of 1 over 256 lanes
  if constexpr (VEC == 1)
    return ln_go<T, VEC, 16>(a, groups, st);
  else
    return ln_go<T, VEC, 4>(a, groups, st);
}
template <typename Args>
hipError_t ln_dispatch(Args a, bool bf16, bool vec, int64_t groups, hipStream_t st) {
  const LnSplit s = ln_split(a.c, vec ? (bf16 ? 8 : 4) : 1);
  a.lanes = s.lanes;
  if (bf16) return vec ? ln_pieces<__bf16, 8>(a, s.pieces, groups, st) : ln_pieces<__bf16, 1>(a, s.pieces, groups, st);
  return vec ? ln_pieces<float, 4>(a, s.pieces, groups, st) : ln_pieces<float, 1>(a, s.pieces, groups, st);
}

// 16-byte pieces need rows of whole pieces and tensors that start on one; a tensor
// of the other type is then read or written in 8 or 32 bytes.
bool ln_vec(int c, bool x_bf16, const void* x, const void* o, const void* o2) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(o2);
  return c % (x_bf16 ? 8 : 4) == 0 && p % 16 == 0;
}

// Rows per round of a workgroup (as if its rows took 16-byte pieces of 2 bytes: the
// count of workgroups must not depend on alignment, which the workspace query does
// not know).
int64_t ln_rounds(int64_t n_rows, int c) {
  const int per_group = 64 * kLnWaves / ln_split(c, 8).lanes;
  return (n_rows + per_group - 1) / per_group;
}

}  // namespace

int layer_norm_back_groups(int64_t n_rows, int32_t c) {
  const int64_t rounds = ln_rounds(n_rows, c);
  return (int)(rounds < 1024 ? rounds : 1024);
}

hipError_t launch_layer_norm(const LayerNormArgs& a, bool x_bf16, hipStream_t st) {
  const int64_t rounds = ln_rounds(a.n_rows, a.c);
  return ln_dispatch(a, x_bf16, ln_vec(a.c, x_bf16, a.x, a.y, nullptr), rounds < 4096 ? rounds : 4096, st);
}

hipError_t launch_layer_norm_back(const LayerNormBackArgs& a, bool x_bf16, hipStream_t st) {
  const int groups = layer_norm_back_groups(a.n_rows, a.c);  // 0 without rows, whose sums are 0
  if (groups > 0) {
    const hipError_t e = ln_dispatch(a, x_bf16, ln_vec(a.c, x_bf16, a.x, a.dy, a.dx), groups, st);
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma && !a.dbeta) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_sum_kernel, dim3((unsigned)((2 * a.c + 15) / 16)), dim3(256), 0, st, a.parts, groups, a.c,
                     a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace dcp
