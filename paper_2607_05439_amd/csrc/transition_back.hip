// Backward pass of the pair transition in bf16 (c_z = 128, hidden = 512) on the matrix cores of gfx950.
// The formulas are those of transition_back_f32.hip, whose last kernels (the sums of the parts, the
// weights' gradients) serve this path too.
//
// Two kernels, each of which forms A, B and dH again: 3 KB a pair of dA, dB and H written and read
// would take three times as long as the products that form them.
//   trans_back_pairs_fast_kernel  dz; the products are transposed (units by pairs)
//   trans_back_sums_fast_kernel   T1 = sum dA zh^T, T2 = sum dB zh^T, T3 = sum H dout^T, S1, S2
//
// Operands are fp16 (11 bits), with powers of two that keep them in its range, so that a result's error is little more
// than its own rounding to bf16. gamma is folded into the weights (W1 diag(gamma), W2 diag(gamma)), and W1 beta, W2 beta
// into the first value of the accumulators, so zh, of at most sqrt(128), is all that is formed of z.
//   A unit's rows of W1 diag(gamma), W2 diag(gamma) and W3^T have powers of two 2^e1, 2^e2, 2^e3 that bring their
//   largest magnitudes (and 1/16 of the biases) below 1: then |A'|, |B'| <= 144, |dH'| <= 128 for |dout'| <= 1, and
//   dA', dB', H' stay under 2^15 whatever the weights are.
//   dout has a power of two per pair, 2^e. In the sums over the pairs that is brought to 2^d, of the largest of all pairs, by
//   2^(d - e) in the sigmoids, of which dA', dB' and H' each have one factor; and where a unit's gates are shut (or its pairs small)
//   they have a power of two of the unit's on top, so that its largest stays in fp16's range (trans_back_sums_fast_kernel).
//   A unit's row in the transposed weights carries 2^-(e1 + e2 + e3), relative to the largest of all units.
// All are taken out of the sums at the end, exactly.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "cdna4.h"
#include "checkpoint.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kCz = kTransCz;       // 128
constexpr int kHid = kTransHidden;  // 512
constexpr int kChunks = kHid / 32;  // of 32 units, two tiles of 16
constexpr int kRowBytes = 24 * 1024, kTrBytes = 16 * 1024;  // a chunk's operands: rows, transposes
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16x8 as_f16x8(u32x4 u) { return __builtin_bit_cast(f16x8, u); }
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float bf16_of(u32x4 v, int i) { return i & 1 ? hi_bf16(v[i >> 1]) : lo_bf16(v[i >> 1]); }

// Channel at accumulator row r of output tile ct (of 16 channels), so that lane group g of tiles 2 ks and
// 2 ks + 1 holds channels 32 ks + 8 g .. + 7, those that it loads of a row.
__host__ __device__ inline int out_channel(int ct, int r) { return 32 * (ct >> 1) + 8 * (r >> 2) + 4 * (ct & 1) + (r & 3); }

// e for which top 2^e is in [1/2, 1); for 0 one past all of these, so that what is 0 never sets the power of two of others
__device__ __forceinline__ int exponent_below_one(float top) {
  int e = -400;
  if (top > 0.0f) (void)frexpf(top, &e);
  return -e;
}

// ----------------------------------------------------------------------------- weights
// In the workspace: rows of every chunk, [tile][ks][W1 | W2 | W3^T][lane] 16 B (row = unit, k-slots = channels
// 32 ks + 8 (lane / 16) .. + 7); transposes of every chunk, [ct][W1 | W2][lane] 16 B (row = channel
// out_channel(ct, lane % 16), k-slot j of lane group g = unit 4g + j of the first tile for j < 4, of the second for j >= 4);
// then per unit, [kUnit*][512]; then the shares' largest |dout| and two exponents.
enum { kUnitLog = 0, kUnitA = 1, kUnitBiasA = 2, kUnitBiasB = 3, kUnitE1 = 4, kUnitE2 = 5, kUnitE3 = 6, kUnitArrays = 7 };
constexpr int kTops = 1024;
constexpr size_t kRowsAt = 0, kTrAt = kRowsAt + (size_t)kChunks * kRowBytes, kUnitsAt = kTrAt + (size_t)kChunks * kTrBytes;
constexpr size_t kTopsAt = kUnitsAt + kUnitArrays * kHid * 4, kExpAt = kTopsAt + kTops * 4, kPrepBytes = kExpAt + 16;

template <typename T>
__device__ __forceinline__ T* prep_at(const TransBackArgs& a, size_t at) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(a.prep) + at);
}
__device__ __forceinline__ int& max_unit_exponent(const TransBackArgs& a) { return prep_at<int>(a, kExpAt)[0]; }
__device__ __forceinline__ int& dout_exponent(const TransBackArgs& a) { return prep_at<int>(a, kExpAt)[1]; }

// Workgroups 0..31: rows of a tile of 16 units, thread (n, q) channels 8 q .. + 7 of unit n. The others: the largest
// finite |dout| of a share each: 57 us for 1024 tokens, 4.7 TB/s.
__global__ void __launch_bounds__(256) trans_back_rows_prep_kernel(TransBackArgs a) {
  __shared__ float s_top[3][16][17], s_bias[2][16][17];
  const int tid = threadIdx.x;
  if (blockIdx.x >= kHid / 16) {
    const int64_t n = a.n_pairs * (kCz / 8), stride = (int64_t)(gridDim.x - kHid / 16) * 256;
    const u32x4* d = static_cast<const u32x4*>(a.dout);
    uint32_t top = 0;  // of |dout|'s bits: finite ones are below 0x7F800000
    for (int64_t i = (int64_t)(blockIdx.x - kHid / 16) * 256 + tid; i < n; i += 8 * stride) {
      u32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = d[min(i + k * stride, n - 1)];
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t lo = (v[k][w] << 16) & 0x7FFFFFFFu, hi = v[k][w] & 0x7FFF0000u;
          top = max(top, lo < 0x7F800000u ? lo : 0u);
          top = max(top, hi < 0x7F800000u ? hi : 0u);
        }
    }
    for (int m = 32; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    __shared__ uint32_t s_max[4];
    if ((tid & 63) == 0) s_max[tid >> 6] = top;
    __syncthreads();
    if (tid == 0) prep_at<uint32_t>(a, kTopsAt)[blockIdx.x - kHid / 16] = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    return;
  }
  const int n = tid & 15, q = tid >> 4, tile = blockIdx.x, unit = 16 * tile + n;
  float w[3][8], top[3] = {0.f, 0.f, 0.f}, bias[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = 8 * q + i;
    const float ga = a.gamma ? a.gamma[c] : 1.0f, be = a.beta ? a.beta[c] : 0.0f;
    w[0][i] = a.w1[unit * kCz + c];
    w[1][i] = a.w2[unit * kCz + c];
    w[2][i] = a.w3[c * kHid + unit];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      bias[m] = fmaf(w[m][i], be, bias[m]);
      w[m][i] *= ga;
    }
#pragma unroll
    for (int m = 0; m < 3; ++m) top[m] = fmaxf(top[m], finite_abs(w[m][i]));
  }
#pragma unroll
  for (int m = 0; m < 3; ++m) s_top[m][n][q] = top[m];
#pragma unroll
  for (int m = 0; m < 2; ++m) s_bias[m][n][q] = bias[m];
  __syncthreads();
  int e[3];
#pragma unroll
  for (int m = 0; m < 3; ++m) {
    for (int k = 0; k < 16; ++k) top[m] = fmaxf(top[m], s_top[m][n][k]);
    if (m < 2) {
      bias[m] = 0.0f;
      for (int k = 0; k < 16; ++k) bias[m] += s_bias[m][n][k];
      top[m] = fmaxf(top[m], finite_abs(bias[m]) * 0.0625f);
    }
    e[m] = exponent_below_one(top[m]);
  }
  u32x4* const rows = prep_at<u32x4>(a, kRowsAt + (size_t)(tile >> 1) * kRowBytes + (size_t)((tile & 1) * 4 + (q >> 2)) * 3 * 1024) + n + 16 * (q & 3);
#pragma unroll
  for (int m = 0; m < 3; ++m) {
    f16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (_Float16)ldexpf(w[m][i], e[m]);
    rows[m * 64] = __builtin_bit_cast(u32x4, v);
  }
  if (q > 0) return;
  float* const units = prep_at<float>(a, kUnitsAt) + unit;
  units[kUnitLog * kHid] = ldexpf(-kLog2e, -e[0]);
  units[kUnitA * kHid] = fminf(ldexpf(1.0f, -e[0]), 32768.0f);  // in fp16's range: past it the slope is that of 0 or 1
  units[kUnitBiasA * kHid] = ldexpf(bias[0], e[0]);
  units[kUnitBiasB * kHid] = ldexpf(bias[1], e[1]);
#pragma unroll
  for (int m = 0; m < 3; ++m) reinterpret_cast<int*>(units)[(kUnitE1 + m) * kHid] = e[m];
}

// The transposes of a chunk's rows from their fragments: a workgroup a chunk; the first also the exponent of dout. 5 us, a few
// loads' latency.
__global__ void __launch_bounds__(256) trans_back_transpose_kernel(TransBackArgs a, int n_tops) {
  __shared__ int s_max[256];
  __shared__ uint32_t s_top[256];
  const int tid = threadIdx.x;
  const int* const e = prep_at<int>(a, kUnitsAt) + kUnitE1 * kHid;
  auto unit_exponent = [&](int u) { return -(e[u] + e[kHid + u] + e[2 * kHid + u]); };
  s_max[tid] = max(unit_exponent(tid), unit_exponent(tid + 256));
  uint32_t top = 0;
  if (blockIdx.x == 0)
    for (int k = tid; k < n_tops; k += 256) top = max(top, prep_at<uint32_t>(a, kTopsAt)[k]);
  s_top[tid] = top;
  __syncthreads();
  for (int m = 128; m > 0; m >>= 1) {
    if (tid < m) {
      s_max[tid] = max(s_max[tid], s_max[tid + m]);
      s_top[tid] = max(s_top[tid], s_top[tid + m]);
    }
    __syncthreads();
  }
  const int most = s_max[0];
  if (blockIdx.x == 0 && tid == 0) {
    max_unit_exponent(a) = most;
    dout_exponent(a) = max(min(exponent_below_one(__uint_as_float(s_top[0])), 126), -126);
  }
  const _Float16* const rows = prep_at<_Float16>(a, kRowsAt + (size_t)blockIdx.x * kRowBytes);
  u32x4* const to = prep_at<u32x4>(a, kTrAt + (size_t)blockIdx.x * kTrBytes);
  for (int k = tid; k < 8 * 2 * 64; k += 256) {
    const int ct = k >> 7, m = (k >> 6) & 1, l = k & 63, c = out_channel(ct, l & 15);
    f16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = 4 * (l >> 4) + (j & 3), tile = j >> 2, lane = n + 16 * ((c >> 3) & 3);
      const float w = (float)rows[((((tile * 4 + (c >> 5)) * 3 + m) * 64) + lane) * 8 + (c & 7)];
      v[j] = (_Float16)ldexpf(w, unit_exponent(32 * blockIdx.x + 16 * tile + n) - most);
    }
    to[k] = __builtin_bit_cast(u32x4, v);
  }
}

// Two elements' A', B', dH' (a, b, d; k: the inverse of A's power of two). With s = sigmoid(A): H' = A' s B', dB' = dH' A' s,
// dA' = dH' B' (s + k A' s (1 - s)). The sigmoid is fp32, what follows packed fp16: the seven roundings of at most 2^-11 in dA'
// together are a third of its rounding to bf16, and the vector work, which does not overlap with the products, falls by a quarter.
// k (1 - s) is formed in fp16 where dz is (an open gate's A > 7 multiplies s's rounding by A there: 1.2e-3 of dA in the root mean
// square, bf16's rounding 1.6e-3); the sums over the pairs take 1 - s from fp32, and s with a factor of its own.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
struct Gated {
  f16x2 h, da, db;
};
__device__ __forceinline__ f16x2 pair_of(float x, float y) { return f16x2{(_Float16)x, (_Float16)y}; }
__device__ __forceinline__ Gated gated(f16x2 a, f16x2 b, f16x2 d, f16x2 s, f16x2 k_rest) {
  const f16x2 silu = a * s, slope = __builtin_elementwise_fma(silu, k_rest, s);
  return {silu * b, d * b * slope, d * silu};
}
__device__ __forceinline__ Gated gated_pairs(float a0, float a1, float b0, float b1, float d0, float d1, f16x2 k, float log0, float log1) {
  const f16x2 s = pair_of(__builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a0 * log0)),
                          __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a1 * log1)));
  return gated(pair_of(a0, a1), pair_of(b0, b1), pair_of(d0, d1), s, __builtin_elementwise_fma(-k, s, k));
}
// For the sums: the sigmoids divided by c, a power of two 2^l for each element.
__device__ __forceinline__ Gated gated_sums(float a0, float a1, float b0, float b1, float d0, float d1, f16x2 k, float log, float c0, float c1,
                                            float l0, float l1, float& s0, float& s1) {
  s0 = __builtin_amdgcn_rcpf(c0 + __builtin_amdgcn_exp2f(fmaf(a0, log, l0)));
  s1 = __builtin_amdgcn_rcpf(c1 + __builtin_amdgcn_exp2f(fmaf(a1, log, l1)));
  return gated(pair_of(a0, a1), pair_of(b0, b1), pair_of(d0, d1), pair_of(s0, s1), k * pair_of(fmaf(-c0, s0, 1.0f), fmaf(-c1, s1, 1.0f)));
}

// ----------------------------------------------------------------------------- rows
// Eight codes (two words) with one power of two, as bf16: exact.
__device__ __forceinline__ u32x4 decode8(u32x2 q, float scale) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)((float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * scale);
  return __builtin_bit_cast(u32x4, v);
}
// A lane (pair n of a tile of 16, group g) holds channels 32 ks + 8g .. + 7 of a row, ks = 0..3.
template <bool CODES>
__device__ __forceinline__ void load_z(const TransBackArgs& a, int64_t pair, int g, u32x4 (&z)[4]) {
  if (CODES) {
    const int8_t* q = static_cast<const int8_t*>(a.z) + pair * kCz + 8 * g;
    const uint32_t e = *reinterpret_cast<const uint32_t*>(a.exponents + pair * 4);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      z[ks] = decode8(*reinterpret_cast<const u32x2*>(q + 32 * ks), checkpoint_scale((e >> (8 * ks)) & 255));
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(a.z) + pair * kCz + 8 * g;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) z[ks] = *reinterpret_cast<const u32x4*>(q + 32 * ks);
  }
}
__device__ __forceinline__ void load_dout(const TransBackArgs& a, int64_t pair, int g, u32x4 (&d)[4]) {
  const uint16_t* q = static_cast<const uint16_t*>(a.dout) + pair * kCz + 8 * g;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) d[ks] = *reinterpret_cast<const u32x4*>(q + 32 * ks);
}
__device__ __forceinline__ void normalise(const u32x4 (&z)[4], float eps, f16x8 (&zf)[4], float& mu, float& rstd) {
  float x[4][8], s = 0.0f, v = 0.0f;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[ks][i] = bf16_of(z[ks], i);
      s += x[ks][i];
    }
  mu = sum4(s) * (1.0f / kCz);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[ks][i] -= mu;
      v = fmaf(x[ks][i], x[ks][i], v);
    }
  rstd = __builtin_amdgcn_rsqf(sum4(v) * (1.0f / kCz) + eps);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // rounded to fp32 first in every kernel: the compiler would fold some of these into one rounding
      float zh = x[ks][i] * rstd;
      asm("" : "+v"(zh));
      zf[ks][i] = (_Float16)zh;
    }
}
// A row of dout in fp16 with a power of two of its own; e: that.
__device__ __forceinline__ void scale_row(const u32x4 (&d)[4], f16x8 (&v)[4], int& e) {
  u16x2 most = {0, 0};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, d[ks][k] & 0x7FFF7FFFu));
  float top = __uint_as_float((uint32_t)(most[0] > most[1] ? most[0] : most[1]) << 16);
  top = max4(top);
  if (!(top < INFINITY)) {  // of the finite ones
    top = 0.0f;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(bf16_of(d[ks], i)));
    top = max4(top);
  }
  e = max(min(exponent_below_one(top), 126), -126);
  const float scale = ldexpf(1.0f, e);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[ks][i] = (_Float16)(bf16_of(d[ks], i) * scale);
}

// What the sums read of a tile of 16 pairs, 8 KB: [zh | dout][ks][lane] 16 B in fp16, with the pairs of odd groups 8
// places on, which spreads the LDS reads of columns over all banks. dout has the power of two of its row, 2^e; the row's factor
// takes that to the one of all pairs: the inverse of that is kept, and its
// logarithm; at most 2^126, which leaves nothing (pairs past the last).
__device__ __forceinline__ int column_lane(int n, int g) { return 16 * g + (n ^ (8 * (g & 1))); }
__device__ __forceinline__ void store_rows(const TransBackArgs& a, int64_t tile, int n, int g, const f16x8 (&zf)[4], const f16x8 (&d)[4], int e) {
  u32x4* const to = reinterpret_cast<u32x4*>(a.zh) + tile * 512 + column_lane(n, g);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    to[ks * 64] = __builtin_bit_cast(u32x4, zf[ks]);
    to[ks * 64 + 256] = __builtin_bit_cast(u32x4, d[ks]);
  }
  if (g == 0) {
    const int l = tile * 16 + n < a.n_pairs ? min(e - dout_exponent(a), 126) : 126;
    a.factors[tile * 16 + n] = ldexpf(1.0f, l);
    a.factor_logs[tile * 16 + n] = (float)l;
  }
}

// These alone, where dz is not wanted or takes dout's place (the sums then come before it). One tile a wave; bound by memory.
template <bool CODES>
__global__ void __launch_bounds__(256) trans_back_rows_kernel(TransBackArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), pair = min(tile * 16 + n, a.n_pairs - 1);
  u32x4 z[4], d[4];
  load_z<CODES>(a, pair, g, z);
  load_dout(a, pair, g, d);
  f16x8 zf[4], dv[4];
  float mu, rstd;
  int e;
  normalise(z, a.eps, zf, mu, rstd);
  scale_row(d, dv, e);
  store_rows(a, tile, n, g, zf, dv, e);
}

// ----------------------------------------------------------------------------- dz
// A workgroup takes groups of 64 TILES pairs, persistently: four waves form A', B' and dH' (units by pairs) of TILES tiles
// of 16 pairs each and, from them, dA' and dB', which are the B operands of the products with the transposed weights;
// those the four other waves form, a chunk of 32 units later, and at a group's end dz. So every weight fragment is read from
// LDS once for TILES tiles of pairs; with each wave doing all of it for two tiles the LDS reads alone took as long as the
// products. 1024 tokens: 900 us, of which the matrix cores are busy 41% and vector work 47%: the two of a SIMD hardly
// overlap, and the gate's 18 vector instructions for two elements, four of them exponentials and reciprocals, are what bounds it
// (2.1 TB/s; each row of z and dout is read twice, as the registers hold none through the chunks).
// The weights stream through LDS by direct-to-LDS loads, the rows one chunk ahead. SPLIT 2, for few pairs: two waves form a tile
// of pairs, 16 units of a chunk each, and two of the others multiply; more loads in flight or chunks ahead gain nothing there.
template <bool CODES, int TILES, int SPLIT>
__global__ void __launch_bounds__(512, 2) trans_back_pairs_fast_kernel(TransBackArgs a) {
  constexpr int kGroup = 64 * TILES / SPLIT;
  __shared__ __attribute__((aligned(16))) char s_rows[2][kRowBytes];
  __shared__ __attribute__((aligned(16))) char s_tr[2][kTrBytes];
  __shared__ __attribute__((aligned(16))) u32x4 s_op[2][4 / SPLIT][2][TILES][64];  // [chunk parity][pairs' share][dA' | dB'][tile][lane]
  __shared__ __attribute__((aligned(16))) float s_u[4][kHid];              // kUnitLog, kUnitA, kUnitBiasA, kUnitBiasB
  __shared__ float s_stat[2][3][kGroup];                                   // [group parity]: mean, rstd, dout's exponent
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), share = wave & 3;
  const int64_t n_groups = (a.n_pairs + kGroup - 1) / kGroup;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  for (int k = tid; k < 4 * kHid; k += 512) (&s_u[0][0])[k] = prep_at<float>(a, kUnitsAt)[k];
  if (wave < 4) {
    const int pairs_share = share / SPLIT, only = share % SPLIT;  // SPLIT 2: the tile of 16 units that this wave takes
    int parity = 0;
    for (int64_t grp = blockIdx.x; grp < n_groups; grp += gridDim.x, parity ^= 1) {
      barrier_lds();
      f16x8 nv[TILES][4], dv[TILES][4];
      constexpr int kPart = TILES < 2 ? TILES : 2;  // tiles whose rows are in flight: more do not fit the registers
#pragma unroll
      for (int p0 = 0; p0 < TILES; p0 += kPart) {
        u32x4 z[kPart][4], d[kPart][4];
#pragma unroll
        for (int q = 0; q < kPart; ++q) {
          const int64_t pair = min(grp * kGroup + (pairs_share * TILES + p0 + q) * 16 + n, a.n_pairs - 1);
          load_z<CODES>(a, pair, g, z[q]);
          load_dout(a, pair, g, d[q]);
        }
#pragma unroll
        for (int q = 0; q < kPart; ++q) {
          const int p = p0 + q, at = (pairs_share * TILES + p) * 16 + n;
          float mu, rstd;
          int e;
          normalise(z[q], a.eps, nv[p], mu, rstd);
          scale_row(d[q], dv[p], e);
          if (a.store_zh && only == 0) store_rows(a, grp * (kGroup / 16) + pairs_share * TILES + p, n, g, nv[p], dv[p], e);
          if (g == 0 && only == 0) {
            s_stat[parity][0][at] = mu;
            s_stat[parity][1][at] = rstd;
            s_stat[parity][2][at] = __int_as_float(e);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll 1
      for (int c = 0; c < kChunks; ++c) {
        barrier_lds();
        const char* const chunk = s_rows[c & 1] + only * (kRowBytes / 2) + lane * 16;
        constexpr int kFrags = 24 / SPLIT, kAhead = 4;
        auto frag = [&](int f) { return *reinterpret_cast<const u32x4*>(chunk + f * 1024); };
        u32x4 wq[kAhead];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) wq[f] = frag(f);
        f32x4 h[3][TILES];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          const int tt = SPLIT == 2 ? only : f / 12, ks = f / 3 % 4, m = f % 3, u = 32 * c + 16 * tt + 4 * g;
          const f16x8 w = as_f16x8(wq[f % kAhead]);
          if (f + kAhead < kFrags) wq[f % kAhead] = frag(f + kAhead);
          f32x4 start = zero;
          if (ks == 0 && m < 2) start = *reinterpret_cast<const f32x4*>(&s_u[m == 0 ? kUnitBiasA : kUnitBiasB][u]);
#pragma unroll
          for (int p = 0; p < TILES; ++p) h[m][p] = mfma(w, m < 2 ? nv[p][ks] : dv[p][ks], ks ? h[m][p] : start);
          if (f % 12 == 11) {
            const f32x4 kl = *reinterpret_cast<const f32x4*>(&s_u[kUnitLog][u]), ka = *reinterpret_cast<const f32x4*>(&s_u[kUnitA][u]);
#pragma unroll
            for (int p = 0; p < TILES; ++p) {
              u32x2 da, db;
#pragma unroll
              for (int i = 0; i < 4; i += 2) {
                const Gated r = gated_pairs(h[0][p][i], h[0][p][i + 1], h[1][p][i], h[1][p][i + 1], h[2][p][i], h[2][p][i + 1],
                                            pair_of(ka[i], ka[i + 1]), kl[i], kl[i + 1]);
                da[i >> 1] = __builtin_bit_cast(uint32_t, r.da);
                db[i >> 1] = __builtin_bit_cast(uint32_t, r.db);
              }
              reinterpret_cast<u32x2*>(&s_op[c & 1][pairs_share][0][p][lane])[tt] = da;
              reinterpret_cast<u32x2*>(&s_op[c & 1][pairs_share][1][p][lane])[tt] = db;
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    barrier_lds();
    return;
  }
  // ---- the products with the transposes, dz, and the weights' copies
  const __amdgpu_buffer_rsrc_t rows_res =
      __builtin_amdgcn_make_buffer_rsrc(prep_at<char>(a, kRowsAt), 0, kChunks * kRowBytes, kRawBufferFlags);
  const __amdgpu_buffer_rsrc_t tr_res =
      __builtin_amdgcn_make_buffer_rsrc(prep_at<char>(a, kTrAt), 0, kChunks * kTrBytes, kRawBufferFlags);
  auto copy_rows = [&](int c) {
#pragma unroll
    for (int i = 0; i < kRowBytes / 4096; ++i) {
      const int piece = share * (kRowBytes / 4096) + i;
      dma_b128(rows_res, c * kRowBytes + piece * 1024 + lane * 16, lds_addr(&s_rows[c & 1][piece * 1024]));
    }
  };
  auto copy_tr = [&](int c) {
#pragma unroll
    for (int i = 0; i < kTrBytes / 4096; ++i) {
      const int piece = share * (kTrBytes / 4096) + i;
      dma_b128(tr_res, c * kTrBytes + piece * 1024 + lane * 16, lds_addr(&s_tr[c & 1][piece * 1024]));
    }
  };
  const bool multiplies = share < 4 / SPLIT;
  f32x4 acc[8][TILES];
  auto products = [&](int c) {
    const char* const chunk = s_tr[c & 1] + lane * 16;
    constexpr int kFrags = 16, kAhead = 4;
    auto frag = [&](int f) { return *reinterpret_cast<const u32x4*>(chunk + f * 1024); };
    f16x8 op[2][TILES];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int p = 0; p < TILES; ++p) op[m][p] = as_f16x8(s_op[c & 1][share][m][p][lane]);
    u32x4 wq[kAhead];
#pragma unroll
    for (int f = 0; f < kAhead; ++f) wq[f] = frag(f);
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      const f16x8 w = as_f16x8(wq[f % kAhead]);
      if (f + kAhead < kFrags) wq[f % kAhead] = frag(f + kAhead);
#pragma unroll
      for (int p = 0; p < TILES; ++p) acc[f / 2][p] = mfma(w, op[f & 1][p], acc[f / 2][p]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const int most = max_unit_exponent(a);
  // acc (ct = 2 ks + s, register i) is gamma dN at channel 32 ks + 8g + 4s + i of pair 16p + n
  auto finish = [&](int64_t grp, int parity) {
    u32x4 z[4], d[4];
    auto load = [&](int p) {
      const int64_t pair = min(grp * kGroup + (share * TILES + p) * 16 + n, a.n_pairs - 1);
      load_z<CODES>(a, pair, g, z);
      load_dout(a, pair, g, d);
    };
    load(0);
    products(kChunks - 1);
#pragma unroll
    for (int p = 0; p < TILES; ++p) {
      const int at = (share * TILES + p) * 16 + n;
      const float mu = s_stat[parity][0][at], rstd = s_stat[parity][1][at];
      const int e = most - __float_as_int(s_stat[parity][2][at]);
      const float shift = -mu * rstd, half = ldexpf(1.0f, e >> 1), rest = ldexpf(rstd, e - (e >> 1));  // 2^e alone may pass fp32's range
      float zh[4][8], m0 = 0.0f, m1 = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          zh[ks][i] = fmaf(bf16_of(z[ks], i), rstd, shift);
          const float gr = acc[2 * ks + (i >> 2)][p][i & 3];
          m0 += gr;
          m1 = fmaf(gr, zh[ks][i], m1);
        }
      m0 = sum4(m0) * (1.0f / kCz);
      m1 = sum4(m1) * (1.0f / kCz);
      uint32_t o[4][4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = (__bf16)fmaf(half * fmaf(-zh[ks][i], m1, acc[2 * ks + (i >> 2)][p][i & 3] - m0), rest, bf16_of(d[ks], i));
        const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[ks][k] = w[k];
      }
      if (p + 1 < TILES) load(p + 1);
      // regrouped across lanes so that a store writes 8 pairs x one whole 128-byte line
      const bool upper = (lane & 4) != 0;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int src = 8 * half + (lane >> 3) + 16 * (lane & 3);
#pragma unroll
        for (int line = 0; line < 2; ++line) {
          u32x4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)o[2 * line][k]);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)o[2 * line + 1][k]);
            v[k] = upper ? hi : lo;
          }
          const int64_t pair = grp * kGroup + (share * TILES + p) * 16 + 8 * half + (lane >> 3);
          if (pair < a.n_pairs)
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.dz) + pair * kCz) + 8 * line + (lane & 7));
        }
      }
    }
  };
  copy_rows(0);
  wait_vm<0>();
  int parity = 0;
  int64_t before = -1;
  for (int64_t grp = blockIdx.x; grp < n_groups; grp += gridDim.x, parity ^= 1) {
    barrier_lds();
    if (before >= 0 && multiplies) finish(before, parity ^ 1);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
      for (int p = 0; p < TILES; ++p) acc[ct][p] = zero;
#pragma unroll 1
    for (int c = 0; c < kChunks; ++c) {
      barrier_lds();
      // rows of the next chunk (the next group's first after the last), in the room of the one before; this chunk's
      // transposes in that of the last but one
      copy_rows(c + 1 == kChunks ? 0 : c + 1);
      copy_tr(c);
      if (c > 0 && multiplies) products(c - 1);
      wait_vm<0>();
    }
    before = grp;
  }
  barrier_lds();
  if (multiplies) finish(before, parity ^ 1);
}

// ----------------------------------------------------------------------------- sums over the pairs
// A workgroup takes 128 units, 32 each of four shares, and a part of the steps of 32 pairs. Of a share, one wave
// keeps the rows of the weights in registers and forms A', B' and dH' (pairs by units: lane (unit n, group g) holds pairs
// 4g .. of both tiles) and dA', dB', H', which are then A operands, k-slot 8g + j = pair 4g + j of the first tile for j < 4,
// of the second for j >= 4; another keeps the sums (192 registers) and adds the products a step later. Their B operands
// are columns of zh and dout, which the LDS's transposing reads bring: 16 lanes read four rows of 16 channels, and
// get four rows of one channel each. The two waves share a SIMD: vector work beside products. (One wave for both, alone
// on its SIMD, took 1110 us for 1024 tokens.) 1024 tokens: 850 us, the matrix cores 57% and vector work 47% busy at 1.7 GHz; the
// waves with the gate, 21 vector instructions for two elements, are what bounds it. Shut gates: below.
constexpr int kStep = 32;
constexpr int kSlice = 128;
constexpr int kStepBytes = 16 * 1024;  // two tiles of 16 pairs: zh, dout
constexpr int kOpBytes = 4 * 6 * 1024;  // dA', dB', H'
constexpr int kAheadSteps = 4;
constexpr int kStepSlots = kAheadSteps + 2;  // and those whose products and whose sums are formed
constexpr int kStepDma = kStepBytes / 1024 / 4;
// A unit's amplification 2^k. |A'|, |B'| <= 144 and |dH'| <= 128 leave 3.5 for 2^k f s (1 + |A|) in fp16, f a pair's factor, and |A| is at
// most 156 where 2^k f s is not 0 (2^(|A| log2(e) - k) is below 2^128): it may be kTop where k > 0, and 1 where k = 0, as s (1 + |A| (1 - s)) is
// 1.1 at most. The largest of a step is brought to 2^-8 at least, one to two bits below kTop, so that k seldom changes again.
constexpr float kTop = 1.0f / 64;
constexpr int kTopBits = 7;
constexpr int kMostBits = 96;  // below this a gate, or a pair, loses its bits in the end

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__global__ void __launch_bounds__(512, 2) trans_back_sums_fast_kernel(TransBackArgs a) {
  __shared__ __attribute__((aligned(16))) char s_x[kStepSlots * kStepBytes];
  __shared__ __attribute__((aligned(16))) char s_op[2 * kOpBytes];
  __shared__ __attribute__((aligned(16))) float s_turn[2][4][32];  // [step parity][share]: factors of the units' sums before this step
  __shared__ __attribute__((aligned(16))) float s_end[4][32];      // and after the last
  __shared__ int s_turns[2][4];                                    // whether there are any
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), share = wave & 3;
  const int chunk = blockIdx.y * (kSlice / 32) + share;  // this wave's 32 units
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int64_t steps = (a.n_pairs + kStep - 1) / kStep;
  const int count = (int)((steps - blockIdx.x + gridDim.x - 1) / gridDim.x);  // of this workgroup
  constexpr int64_t kSize = (int64_t)kHid * kCz;
  float* const part = a.parts + blockIdx.x * (3 * kSize + 2 * kHid);
  char* const my_op = s_op + share * 6 * 1024 + lane * 16;
  if (wave < 4) {
    f16x8 w[3][2][4];
    f16x2 k[2];
    float kl[2], ba[2], bb[2];
#pragma unroll
    for (int ut = 0; ut < 2; ++ut) {
      const u32x4* rows = prep_at<u32x4>(a, kRowsAt + (size_t)chunk * kRowBytes) + ut * 4 * 192 + lane;
      const float* units = prep_at<float>(a, kUnitsAt) + 32 * chunk + 16 * ut + n;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int m = 0; m < 3; ++m) w[m][ut][ks] = as_f16x8(rows[ks * 192 + m * 64]);
      kl[ut] = units[kUnitLog * kHid];
      k[ut] = f16x2{(_Float16)units[kUnitA * kHid], (_Float16)units[kUnitA * kHid]};
      ba[ut] = units[kUnitBiasA * kHid];
      bb[ut] = units[kUnitBiasB * kHid];
    }
    auto sum_at = [&](int m, int ut, int i) { return 3 * kSize + m * kHid + 32 * chunk + 16 * ut + 4 * g + i; };
    f32x4 s[2][2] = {{zero, zero}, {zero, zero}};  // S1, S2: every column of dA^T ones
    int bits[2] = {0, 0};                          // k of unit n
    bool plain = false;                            // no unit of this wave has one: the rest of the steps need no care
    // inverse factors of pairs 4g .. of both tiles, and their logarithms
    const int64_t factors_at = blockIdx.x * (int64_t)kStep + 4 * g;
    const f32x4 *factors = reinterpret_cast<const f32x4*>(a.factors + factors_at), *logs = reinterpret_cast<const f32x4*>(a.factor_logs + factors_at);
    f32x4 f[2] = {zero, zero}, lf[2] = {zero, zero};
    auto load_factors = [&]() {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f[p] = factors[4 * p];
        lf[p] = logs[4 * p];
      }
      factors += (int64_t)gridDim.x * (kStep / 4);
      logs += (int64_t)gridDim.x * (kStep / 4);
    };
    if (count > 0) load_factors();
    f16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (_Float16)1.0f;
    const int row_at = column_lane(n, g) * 16;
    const char* cur = s_x;
    for (int it = 0; it < count; ++it) {
      barrier_lds();
      u32x4 op[3][2];
      float top[2];
      // the first tile of pairs, then the second, and between its products what follows from the first
      auto form = [&](auto amplified) {
        constexpr bool kAmplified = decltype(amplified)::value;
        const float shut[2] = {ldexpf(1.0f, -bits[0]), ldexpf(1.0f, -bits[1])}, by[2] = {(float)-bits[0], (float)-bits[1]};
        top[0] = top[1] = 0.0f;
        auto row = [&](int q, int m) { return as_f16x8(*reinterpret_cast<const u32x4*>(cur + (q >> 2) * 8192 + m * 4096 + (q & 3) * 1024 + row_at)); };
        f32x4 h[3][2][2];
        auto gate = [&](int ut, int p, int i) {  // pairs i, i + 1 of this lane's four
          float c[2] = {f[p][i], f[p][i + 1]}, l[2] = {lf[p][i], lf[p][i + 1]}, t[2];
          if (kAmplified)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              c[j] *= shut[ut];
              l[j] += by[ut];
            }
          const Gated r = gated_sums(h[0][ut][p][i], h[0][ut][p][i + 1], h[1][ut][p][i], h[1][ut][p][i + 1], h[2][ut][p][i], h[2][ut][p][i + 1],
                                     k[ut], kl[ut], c[0], c[1], l[0], l[1], t[0], t[1]);
          if (kAmplified) top[ut] = fmaxf(fmaxf(top[ut], t[0]), t[1]);
          op[0][ut][2 * p + i / 2] = __builtin_bit_cast(uint32_t, r.da);
          op[1][ut][2 * p + i / 2] = __builtin_bit_cast(uint32_t, r.db);
          op[2][ut][2 * p + i / 2] = __builtin_bit_cast(uint32_t, r.h);
#pragma unroll
          for (int m = 0; m < 3; ++m) asm volatile("" : "+v"(op[m][ut][2 * p + i / 2]));  // here, beside the products, not behind them
        };
        constexpr int kQueue = 3;
        f16x8 zq[kQueue], dq[kQueue];
#pragma unroll
        for (int q = 0; q < kQueue - 1; ++q) {
          zq[q] = row(q, 0);
          dq[q] = row(q, 1);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int p = q >> 2, ks = q & 3;
          if (q + kQueue - 1 < 8) {
            zq[(q + kQueue - 1) % kQueue] = row(q + kQueue - 1, 0);
            dq[(q + kQueue - 1) % kQueue] = row(q + kQueue - 1, 1);
          }
#pragma unroll
          for (int ut = 0; ut < 2; ++ut) {
            h[0][ut][p] = mfma(zq[q % kQueue], w[0][ut][ks], ks ? h[0][ut][p] : f32x4{ba[ut], ba[ut], ba[ut], ba[ut]});
            h[1][ut][p] = mfma(zq[q % kQueue], w[1][ut][ks], ks ? h[1][ut][p] : f32x4{bb[ut], bb[ut], bb[ut], bb[ut]});
            h[2][ut][p] = mfma(dq[q % kQueue], w[2][ut][ks], ks ? h[2][ut][p] : zero);
          }
          if (q >= 4) gate(q & 1, 0, (q - 4) & 2);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          gate(0, 1, i);
          gate(1, 1, i);
        }
      };
      float turn[2] = {1.0f, 1.0f};
      bool turned = false;
      if (plain) form(std::false_type());
      while (!plain) {  // once, and again where a unit's k changes: at the first step to what its gates need, then down alone
        form(std::true_type());
        const bool first = it == 0 && !turned;
        bool again = false;
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) {
          const float most = max4(top[ut]);
          if (!first && !(bits[ut] > 0 && most > kTop)) continue;
          int e = -2 * kMostBits;
          if (most > 0.0f) (void)frexpf(most, &e);
          const int to = min(max(bits[ut] - e - kTopBits, 0), kMostBits);
          turn[ut] *= ldexpf(1.0f, to - bits[ut]);
          again |= to != bits[ut];
          bits[ut] = to;
        }
        if (__builtin_amdgcn_ballot_w64(again) == 0) break;
        turned = true;
      }
      plain = __builtin_amdgcn_ballot_w64((bits[0] | bits[1]) != 0) == 0;
      if (it + 1 < count) load_factors();  // the next step's
      if (turned) {
        if (g == 0) {
          s_turn[it & 1][share][n] = turn[0];
          s_turn[it & 1][share][16 + n] = turn[1];
        }
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) {
          const f32x4 by = *reinterpret_cast<const f32x4*>(&s_turn[it & 1][share][16 * ut + 4 * g]);
          s[0][ut] *= by;
          s[1][ut] *= by;
        }
      }
      s_turns[it & 1][share] = turned;
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) *reinterpret_cast<u32x4*>(my_op + (it & 1) * kOpBytes + (m * 2 + ut) * 1024) = op[m][ut];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) s[m][ut] = mfma(as_f16x8(op[m][ut]), ones, s[m][ut]);
      cur = cur + kStepBytes == s_x + kStepSlots * kStepBytes ? s_x : cur + kStepBytes;
    }
    if (g == 0) {
      s_end[share][n] = ldexpf(1.0f, -bits[0]);
      s_end[share][16 + n] = ldexpf(1.0f, -bits[1]);
    }
    barrier_lds();
    if (n == 0)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
        const f32x4 end = *reinterpret_cast<const f32x4*>(&s_end[share][16 * ut + 4 * g]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            part[sum_at(m, ut, i)] = fmaf(s[m][ut][i], end[i], a.add_parts ? part[sum_at(m, ut, i)] : 0.0f);
      }
    return;
  }
  // ---- the sums of the step before, and the copies of the steps to come: pieces 4 share .. of a step's 16
  int slot = 0;
  auto copy = [&](int it) {
    const int64_t step = blockIdx.x + (int64_t)it * gridDim.x;
    const uint32_t to = lds_addr(s_x) + (uint32_t)(slot * kStepBytes);
    slot = slot + 1 == kStepSlots ? 0 : slot + 1;
    const __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc(a.zh + step * kStepBytes, 0, kStepBytes, kRawBufferFlags);
#pragma unroll
    for (int i = 0; i < kStepDma; ++i) {
      const int piece = share * kStepDma + i;
      dma_b128(res, piece * 1024 + lane * 16, to + (uint32_t)(piece * 1024));
    }
  };
#pragma unroll
  for (int it = 0; it < kAheadSteps; ++it)
    if (it < count) copy(it);
  auto part_at = [&](int m, int ut, int ct, int i) { return m * kSize + (32 * chunk + 16 * ut + 4 * g + i) * kCz + 16 * ct + n; };
  f32x4 t[3][2][8];
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) t[m][ut][ct] = zero;
  // a column read's piece: pair 4g + n / 4, channels 4 (n % 4) .. of 16; the chunk of 8 is that of group 2 (ct % 2) + n / 2 % 2
  const int piece_odd = (n >> 1) & 1;
  const int col_at = piece_odd * 256 + ((4 * g + (n >> 2)) ^ (8 * piece_odd)) * 16 + 8 * (n & 1);
  const char* prev = s_x;
  for (int it = 0; it <= count; ++it) {
    // this wave's copies of step `it` have landed: at most those of the ones after it are in flight
    if (it + kAheadSteps - 1 < count)
      wait_vm<(kAheadSteps - 1) * kStepDma>();
    else
      wait_vm<0>();
    barrier_lds();  // and every other wave's; the step before the last has been read
    if (it + kAheadSteps < count) copy(it + kAheadSteps);
    if (it == 0) continue;
    if (__builtin_amdgcn_readfirstlane(s_turns[(it - 1) & 1][share]))
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
        const f32x4 by = *reinterpret_cast<const f32x4*>(&s_turn[(it - 1) & 1][share][16 * ut + 4 * g]);
#pragma unroll
        for (int m = 0; m < 3; ++m)
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) t[m][ut][ct] *= by;
      }
    f16x8 op[3][2];
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut)
        op[m][ut] = as_f16x8(*reinterpret_cast<const u32x4*>(my_op + ((it - 1) & 1) * kOpBytes + (m * 2 + ut) * 1024));
    auto columns = [&](int q) {  // q = 2 ct: zh, 2 ct + 1: dout
      u32x4 v;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(prev + half * 8192 + (q & 1) * 4096 + (q >> 2) * 1024 + ((q >> 1) & 1) * 512 + col_at));
        const u32x2 w = __builtin_bit_cast(u32x2, x);
        v[2 * half] = w[0];
        v[2 * half + 1] = w[1];
      }
      return as_f16x8(v);
    };
    constexpr int kQueue = 3;
    f16x8 cq[kQueue];
#pragma unroll
    for (int q = 0; q < kQueue - 1; ++q) cq[q] = columns(q);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      if (q + kQueue - 1 < 16) cq[(q + kQueue - 1) % kQueue] = columns(q + kQueue - 1);
      const int ct = q >> 1;
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
        if (q & 1) {
          t[2][ut][ct] = mfma(op[2][ut], cq[q % kQueue], t[2][ut][ct]);
        } else {
          t[0][ut][ct] = mfma(op[0][ut], cq[q % kQueue], t[0][ut][ct]);
          t[1][ut][ct] = mfma(op[1][ut], cq[q % kQueue], t[1][ut][ct]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    prev = prev + kStepBytes == s_x + kStepSlots * kStepBytes ? s_x : prev + kStepBytes;
  }
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float sum = t[m][ut][ct][i] * s_end[share][16 * ut + 4 * g + i];
          float* const to = part + part_at(m, ut, ct, i);
          *to = a.add_parts ? *to + sum : sum;  // the pairs before these
        }
}

// As many pairs a workgroup as leave none of the 256 CUs idle. A chunk of weights takes 0.9 us for a tile that two waves share
// (8192 pairs: 19 us, 2025: 17), 1.1 for one tile a wave (22, 21), 1.7 for four.
template <bool CODES>
void launch_pairs(const TransBackArgs& a, hipStream_t st) {
  const int64_t one = (a.n_pairs + 63) / 64;
  if (one <= 128)
    hipLaunchKernelGGL((trans_back_pairs_fast_kernel<CODES, 1, 2>), dim3((unsigned)((a.n_pairs + 31) / 32)), dim3(512), 0, st, a);
  else if (one <= 256)
    hipLaunchKernelGGL((trans_back_pairs_fast_kernel<CODES, 1, 1>), dim3((unsigned)one), dim3(512), 0, st, a);
  else if (one <= 512)
    hipLaunchKernelGGL((trans_back_pairs_fast_kernel<CODES, 2, 1>), dim3((unsigned)((one + 1) / 2)), dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL((trans_back_pairs_fast_kernel<CODES, 4, 1>), dim3((unsigned)((one + 3) / 4 < 256 ? (one + 3) / 4 : 256)), dim3(512), 0, st, a);
}

}  // namespace

size_t trans_back_fast_prep_bytes() { return kPrepBytes; }
void trans_back_fast_units(const float* prep, const int** unit_exponents, const int** dout_exponent) {
  const char* at = reinterpret_cast<const char*>(prep);
  *unit_exponents = reinterpret_cast<const int*>(at + kUnitsAt) + kUnitE1 * kHid;
  *dout_exponent = reinterpret_cast<const int*>(at + kExpAt) + 1;
}

// Shares of the steps: 64, a workgroup for every CU with the four slices of the units, where there are many steps. A step
// takes 1.5 us and a share's sums, written and read again, 0.2: few steps are best in about the root of 7 times as
// many shares (64 steps in 21: 2025 pairs 5 us less than in 64).
int trans_back_fast_splits(int64_t n_pairs) {
  const int64_t steps = (n_pairs + kStep - 1) / kStep;
  if (steps > 585) return 64;
  int64_t s = 1;
  while (s * s < 7 * steps) ++s;
  return (int)(s < steps ? s : steps);
}

// Pairs at a time: 520 B each in the workspace, zh, dout and then the factors.
constexpr int64_t kChunkPairs = (int64_t)1 << 20;
static int64_t rows_held(int64_t n_pairs) { return ((n_pairs < kChunkPairs ? n_pairs : kChunkPairs) + 255) / 256 * 256; }
size_t trans_back_fast_zh_bytes(int64_t n_pairs) { return (size_t)rows_held(n_pairs) * (512 + 2 * sizeof(float)); }

hipError_t launch_trans_back_fast(const TransBackArgs& whole, hipStream_t st) {
  hipError_t e;
  const int64_t shares = (whole.n_pairs * (kCz / 8) + 2047) / 2048;  // eight 16-byte pieces a thread
  const int n_tops = (int)(shares < kTops ? shares : kTops);
  hipLaunchKernelGGL(trans_back_rows_prep_kernel, dim3(kHid / 16 + n_tops), dim3(256), 0, st, whole);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(trans_back_transpose_kernel, dim3(kChunks), dim3(256), 0, st, whole, n_tops);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const bool sums = whole.dw1 || whole.dw2 || whole.dw3 || whole.dgamma || whole.dbeta;
  const bool sums_first = whole.dz == whole.dout || !whole.dz;
  for (int64_t p0 = 0; p0 < whole.n_pairs; p0 += kChunkPairs) {
    TransBackArgs a = whole;
    a.n_pairs = whole.n_pairs - p0 < kChunkPairs ? whole.n_pairs - p0 : kChunkPairs;
    a.z = static_cast<const char*>(whole.z) + p0 * kCz * (whole.exponents ? 1 : 2);
    a.dout = static_cast<const char*>(whole.dout) + p0 * kCz * 2;
    if (whole.exponents) a.exponents += p0 * 4;
    if (whole.dz) a.dz = static_cast<char*>(whole.dz) + p0 * kCz * 2;
    a.store_zh = sums && !sums_first;
    a.factors = reinterpret_cast<float*>(a.zh + rows_held(whole.n_pairs) * 512);
    a.factor_logs = a.factors + rows_held(whole.n_pairs);
    a.add_parts = p0 > 0;
    const dim3 rows_grid((unsigned)((a.n_pairs + 255) / 256 * 4)), sums_grid((unsigned)a.splits, kHid / kSlice);
    if (sums && sums_first) {
      if (a.exponents)
        hipLaunchKernelGGL(trans_back_rows_kernel<true>, rows_grid, dim3(256), 0, st, a);
      else
        hipLaunchKernelGGL(trans_back_rows_kernel<false>, rows_grid, dim3(256), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(trans_back_sums_fast_kernel, sums_grid, dim3(512), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.dz) {
      a.exponents ? launch_pairs<true>(a, st) : launch_pairs<false>(a, st);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (sums && !sums_first) {
      hipLaunchKernelGGL(trans_back_sums_fast_kernel, sums_grid, dim3(512), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace dcp
