// The pair bias of the fused bf16 path on the matrix cores: the bias weights as
// operands, and LayerNorm statistics and projection of one key for 16 rows. Shared
// by the attention, the materialised bias (fast.hip) and the attention's backward
// pass (backward_fast.hip). Operand layouts as in cdna4.h.
#pragma once

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {

// Bias weights as A operands: row = head (lane % 16), k-step s holds channels
// 32s + 8g .. 32s + 8g + 7. W' = scale * W_b * diag(gamma), centred per head
// (subtracting its mean over channels makes sum_c W''_hc z_c = sum_c W'_hc
// (z_c - mean z)), then split into bf16 hi + lo so the pair carries about 16
// significant bits.
// w_b and gamma are 16-byte aligned (checked on the host): each lane reads its
// 8 consecutive channels per k-step as two 16-byte loads, and the absence of
// gamma is one wave-uniform branch, not one per element.
struct BiasRaw {
  float w[4][8], gamma[4][8];
};
__device__ __forceinline__ void bias_weights_load(const float* __restrict__ w_b, const float* __restrict__ gamma,
                                                  int lane, BiasRaw& r) {
  const int h = lane & 15, g = lane >> 4;
  const float4* wr = reinterpret_cast<const float4*>(w_b + h * kFastCz + 8 * g);  // channel 32 s + 8 g + i: float4 8 s + i / 4
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const float4 a = wr[8 * s], b = wr[8 * s + 1];
    r.w[s][0] = a.x, r.w[s][1] = a.y, r.w[s][2] = a.z, r.w[s][3] = a.w;
    r.w[s][4] = b.x, r.w[s][5] = b.y, r.w[s][6] = b.z, r.w[s][7] = b.w;
  }
  if (gamma) {
    const float4* gr = reinterpret_cast<const float4*>(gamma + 8 * g);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float4 a = gr[8 * s], b = gr[8 * s + 1];
      r.gamma[s][0] = a.x, r.gamma[s][1] = a.y, r.gamma[s][2] = a.z, r.gamma[s][3] = a.w;
      r.gamma[s][4] = b.x, r.gamma[s][5] = b.y, r.gamma[s][6] = b.z, r.gamma[s][7] = b.w;
    }
  }
}
__device__ __forceinline__ void bias_weights_finish(BiasRaw& r, bool has_gamma, float scale, bf16x8 (&hi)[4],
                                                    bf16x8 (&lo)[4]) {
  auto& w = r.w;
  if (has_gamma) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[s][i] *= r.gamma[s][i];
  }
  float rs = 0.f;
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[s][i] *= scale;
      rs += w[s][i];
    }
  const float mean = sum4(rs) * (1.0f / kFastCz);
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = w[s][i] - mean;
      const __bf16 x = (__bf16)c;
      hi[s][i] = x;
      lo[s][i] = (__bf16)(c - (float)x);
    }
}
__device__ __forceinline__ void bias_weights(const float* __restrict__ w_b, const float* __restrict__ gamma,
                                             float scale, int lane, bf16x8 (&hi)[4], bf16x8 (&lo)[4]) {
  BiasRaw r;
  bias_weights_load(w_b, gamma, lane, r);
  bias_weights_finish(r, gamma != nullptr, scale, hi, lo);
}

// One key for the wave's 16 rows: z B operands (k-step s = channels 32s+8g..+7
// of row n) -> mean and rstd of the pair and the unnormalised projection acc[i] =
// sum_c W''[4g+i, c] z_c (accumulator rows = heads 4g..4g+3, column = row n).
// The LayerNorm statistics come from the matrix cores as well: ones . z gives
// the row sum in every accumulator register, and the diagonal of the Gram tile
// z . z^T (row n at lane group n/4, register n%4) gives the sum of squares;
// bf16 products are exact in fp32.
__device__ __forceinline__ void pair_bias(const u32x4 (&zb)[4], const bf16x8 (&whi)[4], const bf16x8 (&wlo)[4],
                                          const f32x4& wsum, float eps, int n, f32x4& acc, float& rstd, float& mu) {
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  f32x4 s1 = {0.f, 0.f, 0.f, 0.f}, gram = {0.f, 0.f, 0.f, 0.f};
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const bf16x8 zv = as_bf16x8(zb[s]);
    acc = mfma32(whi[s], zv, acc);
    s1 = mfma32(ones, zv, s1);
    acc = mfma32(wlo[s], zv, acc);
    gram = mfma32(zv, zv, gram);
  }
  // diagonal of the Gram tile: pick register n%4, then fetch it from lane group n/4
  const float t0 = (n & 1) ? gram[1] : gram[0];
  const float t1 = (n & 1) ? gram[3] : gram[2];
  float d = (n & 2) ? t1 : t0;        // (row 4g + n%4, column n)
  const int tg = n >> 2;               // the lane group holding row n
  float lo = d, hi = d;
  swap32(lo, hi);                      // lo: group g&1, hi: group (g&1)|2
  d = (tg & 2) ? hi : lo;              // group (g&1) | (tg&2)
  lo = d;
  hi = d;
  swap16(lo, hi);                      // lo: even group of the pair, hi: odd group
  const float s2 = (tg & 1) ? hi : lo; // group tg: the diagonal entry
  mu = s1[0] * (1.0f / kFastCz);
  // s2/c_z - mu^2 with the square formed exactly inside the fma: one rounding
  // of the exact difference, so a large channel mean (|mu| >> sigma) does not
  // cancel away the variance's significant bits
  const float var = fmaxf(fmaf(-mu, mu, s2 * (1.0f / kFastCz)), 0.0f);
  rstd = __builtin_amdgcn_rsqf(var + eps);
  // the bf16 hi + lo weights sum to wsum (not exactly 0) per head; remove
  // wsum * mu so the projection is that of z - mu even when mu is large
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = fmaf(-mu, wsum[i], acc[i]);
}

// Per-head sums of the bias weight operands, sum_c (hi + lo)[h, c], in the
// accumulator layout of pair_bias (heads 4g..4g+3 in every column): W'' . 1
// on the matrix cores.
__device__ __forceinline__ f32x4 bias_weight_sums(const bf16x8 (&whi)[4], const bf16x8 (&wlo)[4]) {
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    r = mfma32(whi[s], ones, r);
    r = mfma32(wlo[s], ones, r);
  }
  return r;
}

}  // namespace dcp
