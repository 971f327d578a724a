// LayerNorm over the channels of a row, and its backward pass with the gradients
// of the affine weights (gfx950).
//
//   mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd,
//   y = gamma xh + beta;
//   g = gamma dy, dx = rstd (g - mean g - xh mean(g xh)),
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy.
//
// Both are bound by memory: the forward reads x and writes y, the backward reads x
// and dy and writes dx, each once. A million rows of 128 bf16 channels: 100 us forward
// (5.4 TB/s read and written; a copy of 8 GiB runs at 4.5), 149 us backward (5.4). 24000
// rows of 384: 20 us backward, of which the sums over workgroups 4. The statistics are
// formed again in the backward, from the row it holds in registers anyway, so nothing
// but x is kept.
//
// A row lies in the registers of 2^k consecutive lanes (as few as hold it in 16-byte
// pieces, so that a wave takes many narrow rows at once; a wide row takes the
// workgroup's 256), lane l of them holding pieces l, l + lanes, ...; the mean, then the
// centred squares, are summed in fp32 across those lanes. A lane's channels are the same
// in every row, so its share of dgamma and dbeta stays in registers over all rows of its
// workgroup; the workgroups' sums are added up by a second kernel in a fixed order.
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

// VEC consecutive elements, as loaded and as fp32: the loads of a row are all issued
// before the first conversion waits for one.
template <typename T, int VEC>
struct Piece {
  static constexpr int kWords = VEC * (int)sizeof(T) / 4;  // 2, 4 or 8; one element: 0
  uint32_t w[kWords > 0 ? kWords : 1];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kWords == 0 || VEC == 1) {
      w[0] = sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (kWords == 2) {
      const u32x2 r = *reinterpret_cast<const u32x2*>(p);
      w[0] = r[0], w[1] = r[1];
    } else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const u32x4 r = reinterpret_cast<const u32x4*>(p)[i / 4];
        w[i] = r[0], w[i + 1] = r[1], w[i + 2] = r[2], w[i + 3] = r[3];
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    *p = (T)v[0];
  } else if constexpr (sizeof(T) == 2) {
    typedef __bf16 vec __attribute__((ext_vector_type(VEC)));
    vec r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r[i] = (__bf16)v[i];
    *reinterpret_cast<vec*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  }
}
// The affine weights of a lane's channels.
template <int VEC>
__device__ __forceinline__ void load_weights(const float* w, bool in, int ch, float absent, float (&v)[VEC]) {
  if (w && in) {
    // 4-byte loads: the weights need no more alignment than that
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = w[ch + i];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = absent;
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

template <typename T, typename TY, int VEC, int NV>
__global__ void __launch_bounds__(64 * kLnWaves) layer_norm_kernel(LayerNormArgs a) {
  __shared__ float red[2][kLnWaves];
  const int lanes = a.lanes, at = threadIdx.x & (lanes - 1), rows_at_once = 64 * kLnWaves / lanes;
  const int64_t step = (int64_t)gridDim.x * rows_at_once, first = (int64_t)blockIdx.x * rows_at_once;
  int64_t row = first + threadIdx.x / lanes;
  int ch[NV];
  bool in[NV];
  float gamma[NV][VEC], beta[NV][VEC];
  Piece<T, VEC> raw[NV];
  // every lane runs the same rounds: the sums need all lanes of a row; rows past the
  // last read the last one and pieces past the row's end its first, and neither
  // is written
  auto load = [&]() {
    const T* p = static_cast<const T*>(a.x) + min(row, a.n_rows - 1) * a.c;
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j].load(p + (in[j] ? ch[j] : 0));
  };
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    ch[j] = (j * lanes + at) * VEC;
    in[j] = ch[j] < a.c;
  }
  load();
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    load_weights<VEC>(a.gamma, in[j], ch[j], 1.f, gamma[j]);
    load_weights<VEC>(a.beta, in[j], ch[j], 0.f, beta[j]);
  }
  const float inv_c = 1.0f / (float)a.c;
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step) {
    float x[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j][i] = in[j] ? raw[j].get(i) : 0.f;
    const int64_t here = row;
    row += step;
    if (r0 + step < a.n_rows) load();  // the next row, in flight during this one's sums
    const float rstd = centre<VEC, NV>(x, in, inv_c, a.eps, lanes, red);
    if (here < a.n_rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = fmaf(x[j][i] * rstd, gamma[j][i], beta[j][i]);
        if (in[j]) store_vec<TY, VEC>(static_cast<TY*>(a.y) + here * a.c + ch[j], y);
      }
    }
  }
}

template <int N>
__device__ __forceinline__ float add_rotated(float x) {  // + the lane N further in its row of 16
  return add_dpp<0x120 + N>(x);
}

template <typename T, typename TY, int VEC, int NV>
__global__ void __launch_bounds__(64 * kLnWaves) layer_norm_back_kernel(LayerNormBackArgs a) {
  __shared__ float red[2][kLnWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lanes = a.lanes;
  const int at = threadIdx.x & (lanes - 1), rows_at_once = 64 * kLnWaves / lanes;
  const int64_t step = (int64_t)gridDim.x * rows_at_once, first = (int64_t)blockIdx.x * rows_at_once;
  int64_t row = first + threadIdx.x / lanes;
  int ch[NV];
  bool in[NV];
  float gamma[NV][VEC], dgamma[NV][VEC], dbeta[NV][VEC];
  Piece<T, VEC> rx[NV];
  Piece<TY, VEC> ry[NV];
  auto load = [&]() {
    const int64_t off = min(row, a.n_rows - 1) * a.c;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      rx[j].load(static_cast<const T*>(a.x) + off + (in[j] ? ch[j] : 0));
      ry[j].load(static_cast<const TY*>(a.dy) + off + (in[j] ? ch[j] : 0));
    }
  };
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    ch[j] = (j * lanes + at) * VEC;
    in[j] = ch[j] < a.c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) dgamma[j][i] = dbeta[j][i] = 0.f;
  }
  load();
#pragma unroll
  for (int j = 0; j < NV; ++j) load_weights<VEC>(a.gamma, in[j], ch[j], 1.f, gamma[j]);
  const float inv_c = 1.0f / (float)a.c;
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step) {
    const bool real = row < a.n_rows;
    float x[NV][VEC], dy[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        x[j][i] = in[j] ? rx[j].get(i) : 0.f;
        dy[j][i] = in[j] ? ry[j].get(i) : 0.f;
      }
    const int64_t here = row;
    row += step;
    if (r0 + step < a.n_rows) load();  // the next row, in flight during this one's sums
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
        if (in[j]) store_vec<T, VEC>(static_cast<T*>(a.dx) + here * a.c + ch[j], dx);
      }
    }
  }
  if (!a.parts) return;  // the whole grid
  // the rows of a wave, by rotations of 16 lanes and exchanges between them, then
  // its waves
  float* out = a.parts + (int64_t)blockIdx.x * 2 * a.c;
  const bool alone = lanes == 64 * kLnWaves;  // a channel lies in one lane of one wave
  extern __shared__ float s_part[];           // [kLnWaves][2][c]
  auto over_rows = [&](float v) {
    if (lanes <= 8) v = add_rotated<8>(v);
    if (lanes <= 4) v = add_rotated<4>(v);
    if (lanes <= 2) v = add_rotated<2>(v);
    if (lanes <= 1) v = add_rotated<1>(v);
    if (lanes <= 16) {
      float p = v, q = v;
      swap16(p, q);
      v = p + q;
    }
    if (lanes <= 32) {
      float p = v, q = v;
      swap32(p, q);
      v = p + q;
    }
    return v;
  };
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float g = over_rows(dgamma[j][i]), b = over_rows(dbeta[j][i]);
      if (in[j] && (alone || lane < lanes)) {
        float* to = alone ? out : s_part + wave * 2 * a.c;
        to[ch[j] + i] = g;
        to[a.c + ch[j] + i] = b;
      }
    }
  if (alone) return;  // the whole workgroup
  __syncthreads();
  for (int x = threadIdx.x; x < 2 * a.c; x += 64 * kLnWaves)
    out[x] = (s_part[x] + s_part[2 * a.c + x]) + (s_part[4 * a.c + x] + s_part[6 * a.c + x]);
}

// Column sums of parts[n_parts][2 c]: a workgroup takes 16 columns, its 64 groups of 16
// lanes every 64th part each, four loads in flight.
constexpr int kSumGroups = 64;
__global__ void __launch_bounds__(16 * kSumGroups) layer_norm_sum_kernel(const float* parts, int n_parts, int c,
                                                                        float* dgamma, float* dbeta) {
  __shared__ float s[kSumGroups][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), grp = threadIdx.x >> 4;
  float x = 0.f;
  if (col < 2 * c)
#pragma unroll 4
    for (int p = grp; p < n_parts; p += kSumGroups) x += parts[(int64_t)p * 2 * c + col];
  s[grp][threadIdx.x & 15] = x;
  __syncthreads();
  if (grp > 0 || col >= 2 * c) return;
#pragma unroll
  for (int i = 1; i < kSumGroups; ++i) x += s[i][threadIdx.x];
  float* out = col < c ? dgamma : dbeta;
  if (out) out[col < c ? col : col - c] = x;
}

// Lanes of a row and pieces per lane: one piece each up to 64 lanes, then up to three,
// then the workgroup's 256 lanes. (The backward holds six registers per channel: rows
// of 128 bf16 channels over 16 lanes rather than 8 took 148 instead of 172 us for a
// million rows, rows of 384 over 64 rather than 16 lanes 20 instead of 27 for 24000;
// the forward is the same either way.)
struct LnSplit {
  int lanes, pieces;
};
LnSplit ln_split(int c, int vec) {
  const int chunks = (c + vec - 1) / vec;
  int lanes = 1;
  while (lanes < 64 && lanes < chunks) lanes *= 2;
  if (lanes * 3 < chunks) lanes = 64 * kLnWaves;
  return {lanes, (chunks + lanes - 1) / lanes};
}

template <typename T, typename TY, int VEC, int NV>
hipError_t ln_go(const LayerNormArgs& a, int64_t groups, hipStream_t st) {
  hipLaunchKernelGGL((layer_norm_kernel<T, TY, VEC, NV>), dim3((unsigned)groups), dim3(64 * kLnWaves), 0, st, a);
  return hipGetLastError();
}
template <typename T, typename TY, int VEC, int NV>
hipError_t ln_go(const LayerNormBackArgs& a, int64_t groups, hipStream_t st) {
  // (up to 48 KB: rows wider than that share no channel between lanes)
  const size_t lds = a.parts && a.lanes <= 64 ? (size_t)kLnWaves * 2 * a.c * sizeof(float) : 0;
  hipLaunchKernelGGL((layer_norm_back_kernel<T, TY, VEC, NV>), dim3((unsigned)groups), dim3(64 * kLnWaves), lds, st, a);
  return hipGetLastError();
}
template <typename T, typename TY, int VEC, typename Args>
hipError_t ln_pieces(const Args& a, int pieces, int64_t groups, hipStream_t st) {
  if (pieces <= 1) return ln_go<T, TY, VEC, 1>(a, groups, st);
  if (pieces <= 2) return ln_go<T, TY, VEC, 2>(a, groups, st);
  if (pieces <= 3) return ln_go<T, TY, VEC, 3>(a, groups, st);
  // c <= kLnMaxC: 512 pieces of 8, 1024 of 4 or 4096 of 1 over 256 lanes
  if constexpr (VEC == 1)
    return ln_go<T, TY, VEC, 16>(a, groups, st);
  else if constexpr (VEC == 4)
    return ln_go<T, TY, VEC, 4>(a, groups, st);
  return hipErrorInvalidValue;  // not reached: two pieces of 8 at most
}
template <typename T, typename TY, typename Args>
hipError_t ln_dispatch(Args a, bool vec, int64_t groups, hipStream_t st) {
  constexpr int kVec = 16 / (int)sizeof(T);
  const LnSplit s = ln_split(a.c, vec ? kVec : 1);
  a.lanes = s.lanes;
  return vec ? ln_pieces<T, TY, kVec>(a, s.pieces, groups, st) : ln_pieces<T, TY, 1>(a, s.pieces, groups, st);
}
template <typename Args>
hipError_t ln_types(const Args& a, bool x_bf16, bool y_bf16, bool vec, int64_t groups, hipStream_t st) {
  if (x_bf16) return y_bf16 ? ln_dispatch<__bf16, __bf16>(a, vec, groups, st) : ln_dispatch<__bf16, float>(a, vec, groups, st);
  return y_bf16 ? ln_dispatch<float, __bf16>(a, vec, groups, st) : ln_dispatch<float, float>(a, vec, groups, st);
}

// 16-byte pieces need rows of whole pieces and tensors that start on one; a tensor
// of the other type is then read or written in 8 or 32 bytes.
bool ln_vec(int c, bool x_bf16, const void* x, const void* o, const void* o2) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(o2);
  return c % (x_bf16 ? 8 : 4) == 0 && p % 16 == 0;
}

// Rounds of workgroups over the rows, counted as if a row lay in pieces of eight elements:
// the count of workgroups must not depend on the type or the alignment, which the workspace
// query does not know. fp32 rows lie in pieces of four, so rows of up to 256 channels take
// twice the rounds that are counted, and rows read element by element more.
int64_t ln_rounds(int64_t n_rows, int c) {
  const int per_group = 64 * kLnWaves / ln_split(c, 8).lanes;
  return (n_rows + per_group - 1) / per_group;
}

}  // namespace

// Workgroups of the backward: four a CU, two up to 1280 counted rounds, since a workgroup's start
// and its sums take as long as some rounds. us a call in 512 and in 1024 workgroups, with the
// rounds counted, below the cut: bf16 4800 rows of 384 (1200) 10.4 and 12.3, 16384 of 128 (1024)
// 9.7 and 11.1; fp32 4800 of 384 (1200) 11.5 and 13.6, 16384 of 128 (1024) 11.6 and 12.1, 60000 of
// 32 (938) 10.8 and 11.0. Beyond it: bf16 8000 of 384 (2000) 12.7 and 14.1, 40000 of 128 (2500)
// 14.1 and 14.2, 24000 of 384 (6000) 22.3 and 20.8, a million of 128 167 and 149 (in 2048 166);
// fp32 8000 of 384 13.9 and 15.5, 20500 of 128 (1282) 12.5 and 12.7, 40000 of 128 (2500) 17.4 and
// 16.8, 100000 of 32 (1563) 13.3 and 12.8. So the cut is right for narrow fp32 rows, which take
// twice the rounds counted, and up to twice too low for the others, which lose up to 17% there.
int layer_norm_back_groups(int64_t n_rows, int32_t c) {
  const int64_t rounds = ln_rounds(n_rows, c), most = rounds <= 1280 ? 512 : 1024;
  return (int)(rounds < most ? rounds : most);
}

hipError_t launch_layer_norm(const LayerNormArgs& a, bool x_bf16, bool y_bf16, hipStream_t st) {
  const int64_t rounds = ln_rounds(a.n_rows, a.c);
  return ln_types(a, x_bf16, y_bf16, ln_vec(a.c, x_bf16, a.x, a.y, nullptr), rounds < 4096 ? rounds : 4096, st);
}

hipError_t launch_layer_norm_back(const LayerNormBackArgs& a, bool x_bf16, bool dy_bf16, hipStream_t st) {
  const int groups = layer_norm_back_groups(a.n_rows, a.c);  // 0 without rows, whose sums are 0
  if (groups > 0) {
    const hipError_t e = ln_types(a, x_bf16, dy_bf16, ln_vec(a.c, x_bf16, a.x, a.dy, a.dx), groups, st);
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma && !a.dbeta) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_sum_kernel, dim3((unsigned)((2 * a.c + 15) / 16)), dim3(16 * kSumGroups), 0, st, a.parts,
                     groups, a.c, a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace dcp
