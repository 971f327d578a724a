// Backward pass of the pair transition in bf16 (c_z = 128, hidden = 512) on the matrix cores of gfx950.
// The formulas are those of transition_back_f32.hip, whose last kernels (the sums of the parts, the
// weights' gradients) serve this path too.
//
// Two kernels, each of which forms A, B and dH again: 3 KB a pair of dA, dB and H written and read
// would take three times as long as the products that form them.
//   trans_back_pairs_fast_kernel  dz; the products are transposed (units by pairs)
//   trans_back_sums_fast_kernel   T1 = sum dA zh^T, T2 = sum dB zh^T, T3 = sum H dout^T, S1, S2
//
// Operands. gamma is folded into the weights (W1 diag(gamma), W2 diag(gamma)) and W1 beta, W2 beta into
// the first value of the accumulators, so zh, of at most sqrt(128), is all that is formed of z. zh and
// the rows of W1 and W2 enter as fp16, 11 bits, each row times a power of two of its own; A and B are
// then as exact as the results' roundings to bf16 need. dout is bf16 as given; W3, dA, dB, H, the
// transposed weights and zh (where it meets dA and dB) are rounded to bf16, whose range leaves gradients of any size alone.
// A row's powers of two stay in A and B and are taken out by the transposed weights and, from T and S,
// at the end: exact.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"
#include "checkpoint.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kCz = kTransCz;       // 128
constexpr int kHid = kTransHidden;  // 512
constexpr int kHp = kHid / 32;      // pairs of hidden tiles
constexpr int kPairBytes = 40 * 1024;  // operands of 32 units
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ f32x4 mfma_f16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16x8 as_f16x8(u32x4 u) { return __builtin_bit_cast(f16x8, u); }
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Channel at accumulator row r of output tile ct (of 16 channels), so that lane group g of tiles 2 ks and
// 2 ks + 1 holds channels 32 ks + 8 g .. + 7, those that it loads of a row.
__host__ __device__ inline int out_channel(int ct, int r) { return 32 * (ct >> 1) + 8 * (r >> 2) + 4 * (ct & 1) + (r & 3); }

// 2^-k for a row whose largest magnitude is in [2^(k-1), 2^k): from there to [1/2, 1)
__device__ __forceinline__ float row_scale(float top) {
  if (top == 0.0f) return 1.0f;
  int e;
  (void)frexpf(top, &e);
  return ldexpf(1.0f, max(min(-e, 126), -126));
}

// ----------------------------------------------------------------------------- weights
// Operands of 32 units (40 KB): for each of their two tiles and each k-step ks the rows of W1 diag(gamma) and
// W2 diag(gamma) (fp16) and of W3^T (bf16), [tile][ks][matrix][lane] 16 B (row = unit, k-slots = channels
// 32 ks + 8 (lane / 16) .. + 7); then [ct][W1 | W2][lane] 16 B of their transposes (bf16; row = channel
// out_channel(ct, lane % 16), k-slot j of lane group g = unit 4g + j of the first tile for j < 4, of the second for
// j >= 4). After all operands, per unit, [kUnit*][512] fp32.
enum { kUnitLog = 0, kUnitA = 1, kUnitBiasA = 2, kUnitBiasB = 3, kUnitB = 4, kUnitArrays = 5 };
constexpr size_t kPrepBytes = (size_t)kHp * kPairBytes + kUnitArrays * kHid * sizeof(float);

// One workgroup per tile of 16 units; thread (n, q) holds channels 8 q .. + 7 of unit n.
__global__ void __launch_bounds__(256) trans_back_prep_fast_kernel(TransBackArgs a) {
  __shared__ float s_top[2][16][17], s_bias[2][16][17];
  __shared__ float s_w[2][16][kCz + 4];
  const int tid = threadIdx.x, n = tid & 15, q = tid >> 4, tile = blockIdx.x, unit = 16 * tile + n;
  char* const base = reinterpret_cast<char*>(a.prep) + (size_t)(tile >> 1) * kPairBytes;
  float* const units = reinterpret_cast<float*>(reinterpret_cast<char*>(a.prep) + (size_t)kHp * kPairBytes);
  float w[2][8], top[2] = {0.f, 0.f}, bias[2] = {0.f, 0.f};
  bf16x8 w3;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = 8 * q + i;
    const float ga = a.gamma ? a.gamma[c] : 1.0f, be = a.beta ? a.beta[c] : 0.0f;
    w[0][i] = a.w1[unit * kCz + c];
    w[1][i] = a.w2[unit * kCz + c];
    w3[i] = (__bf16)a.w3[c * kHid + unit];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      bias[m] = fmaf(w[m][i], be, bias[m]);
      w[m][i] *= ga;
      top[m] = fmaxf(top[m], finite_abs(w[m][i]));
    }
  }
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    s_top[m][n][q] = top[m];
    s_bias[m][n][q] = bias[m];
  }
  __syncthreads();
  float scale[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    for (int k = 0; k < 16; ++k) top[m] = fmaxf(top[m], s_top[m][n][k]);
    scale[m] = row_scale(top[m]);
  }
  const int ks = q >> 2, lane = n + 16 * (q & 3);
  u32x4* const rows = reinterpret_cast<u32x4*>(base + (size_t)((tile & 1) * 4 + ks) * 3 * 1024) + lane;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    f16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (_Float16)(w[m][i] * scale[m]);
      s_w[m][n][8 * q + i] = w[m][i] / scale[1 - m];
    }
    rows[m * 64] = __builtin_bit_cast(u32x4, v);
  }
  rows[2 * 64] = __builtin_bit_cast(u32x4, w3);
  if (q == 0) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      bias[m] = 0.0f;
      for (int k = 0; k < 16; ++k) bias[m] += s_bias[m][n][k];
    }
    units[kUnitLog * kHid + unit] = -kLog2e / scale[0];
    units[kUnitA * kHid + unit] = 1.0f / scale[0];
    units[kUnitB * kHid + unit] = 1.0f / scale[1];
    units[kUnitBiasA * kHid + unit] = bias[0] * scale[0];
    units[kUnitBiasB * kHid + unit] = bias[1] * scale[1];
  }
  __syncthreads();
  // transposes: dA carries W2's power of two and dB W1's, which s_w has been divided by
  for (int k = tid; k < 2 * 8 * 64; k += 256) {
    const int m = k >> 9, ct = (k >> 6) & 7, l = k & 63, c = out_channel(ct, l & 15), u = 4 * (l >> 4);
    bf16x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (__bf16)s_w[m][u + j][c];
    *reinterpret_cast<u32x2*>(base + 24 * 1024 + (ct * 2 + m) * 1024 + l * 16 + (tile & 1) * 8) = __builtin_bit_cast(u32x2, v);
  }
}

// h0 = A and h1 = B with their powers of two (k: A's inverse, log: -log2(e) times it). With s = sigmoid(A) and
// A' = h0: H' = A' s B', dB' = dH A' s, dA' = dH B' (s + k A' s (1 - s)).
struct Gated {
  float h, da, db;
};
__device__ __forceinline__ Gated gated(float h0, float h1, float dh, float k, float log) {
  const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(h0 * log));
  const float silu = h0 * s;
  return {silu * h1, dh * h1 * fmaf(silu, fmaf(-k, s, k), s), dh * silu};
}

// Eight codes (two words) with one power of two, as bf16: exact.
__device__ __forceinline__ u32x4 decode8(u32x2 q, float scale) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)((float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * scale);
  return __builtin_bit_cast(u32x4, v);
}

// ----------------------------------------------------------------------------- rows
// A lane (pair n of a tile of 16, group g) holds channels 32 ks + 8g .. + 7 of a row, ks = 0..3.
template <bool CODES>
__device__ __forceinline__ void load_row(const TransBackArgs& a, int64_t pair, int g, u32x4 (&z)[4]) {
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
// zh in fp16 and bf16, and the statistics.
__device__ __forceinline__ void normalise(const u32x4 (&z)[4], float eps, f16x8 (&zf)[4], bf16x8 (&zb)[4], float& mu, float& rstd) {
  float x[4][8], s = 0.0f, v = 0.0f;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[ks][i] = i & 1 ? hi_bf16(z[ks][i >> 1]) : lo_bf16(z[ks][i >> 1]);
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
      const float zh = x[ks][i] * rstd;
      zf[ks][i] = (_Float16)zh;
      zb[ks][i] = (__bf16)zh;
    }
}
// zh of a tile of 16 pairs for the sums, 8 KB: [ks][lane] 16 B in fp16, as A operands; then the same in bf16, with
// the pairs of odd groups 8 places on, which spreads the LDS reads of columns over all banks.
__device__ __forceinline__ int column_lane(int n, int g) { return 16 * g + (n ^ (8 * (g & 1))); }
__device__ __forceinline__ void store_zh(const TransBackArgs& a, int64_t tile, int n, int g, const f16x8 (&zf)[4], const bf16x8 (&zb)[4]) {
  u32x4* const to = reinterpret_cast<u32x4*>(a.zh) + tile * 512;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    to[ks * 64 + 16 * g + n] = __builtin_bit_cast(u32x4, zf[ks]);
    to[256 + ks * 64 + column_lane(n, g)] = __builtin_bit_cast(u32x4, zb[ks]);
  }
}

// zh alone, where dz is not wanted or takes dout's place (the sums, which need zh, then come before it). One tile a wave.
template <bool CODES>
__global__ void __launch_bounds__(256) trans_back_rows_kernel(TransBackArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  u32x4 z[4];
  load_row<CODES>(a, min(tile * 16 + n, a.n_pairs - 1), g, z);
  f16x8 zf[4];
  bf16x8 zb[4];
  float mu, rstd;
  normalise(z, a.eps, zf, zb, mu, rstd);
  store_zh(a, tile, n, g, zf, zb);
}

// ----------------------------------------------------------------------------- dz
// A workgroup of 8 waves takes groups of 256 pairs, 32 a wave (two tiles of 16), persistently. zh (fp16) and dout
// (bf16) are B operands in registers: lane (pair n, group g) holds channels 32 ks + 8g .. + 7. For every 32 units: A', B'
// and dH (units by pairs), dA' and dB' in registers, which are the B operands of the products with the
// transposed weights; their sum is gamma dN, at the channels that the lane holds of z and dout. The weights stream
// through two 40 KB LDS buffers by direct-to-LDS loads one chunk ahead; z waits in LDS for the end.
constexpr int kWaves = 8;
constexpr int kGroupPairs = 32 * kWaves;
constexpr int kDmaPerWave = kPairBytes / 1024 / kWaves;

template <bool CODES>
__global__ void __launch_bounds__(64 * kWaves) trans_back_pairs_fast_kernel(TransBackArgs a) {
  __shared__ __attribute__((aligned(16))) char s_w[2][kPairBytes];
  __shared__ __attribute__((aligned(16))) u32x4 s_z[kWaves][8][64];
  __shared__ __attribute__((aligned(16))) float s_u[4][kHid];  // kUnitLog, kUnitA, kUnitBiasA, kUnitBiasB
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t n_groups = (a.n_pairs + kGroupPairs - 1) / kGroupPairs;
  const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(a.prep, 0, kHp * kPairBytes, kRawBufferFlags);
  auto chunk_dma = [&](int c, int b) {
    const uint32_t base = lds_addr(&s_w[b][0]) + (uint32_t)(wave * kDmaPerWave * 1024);
#pragma unroll
    for (int i = 0; i < kDmaPerWave; ++i)
      dma_b128(wres, c * kPairBytes + (wave * kDmaPerWave + i) * 1024 + lane * 16, base + (uint32_t)(i * 1024));
  };
  {
    const float* units = reinterpret_cast<const float*>(reinterpret_cast<const char*>(a.prep) + (size_t)kHp * kPairBytes);
    for (int k = tid; k < 4 * kHid; k += 64 * kWaves) (&s_u[0][0])[k] = units[k];
  }
  int64_t grp = blockIdx.x;
  int seq = 0;
  chunk_dma(0, 0);
  for (; grp < n_groups; grp += gridDim.x) {
    const bool last_group = grp + gridDim.x >= n_groups;
    const int64_t pair0 = grp * kGroupPairs + wave * 32;
    u32x4 dv[2][4];
    f16x8 nv[2][4];
    float mu[2], rstd[2];
    {
      u32x4 zz[2][4];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int64_t pr = min(pair0 + 16 * p + n, a.n_pairs - 1);  // pairs past the end are not stored
        load_row<CODES>(a, pr, g, zz[p]);
        const uint16_t* d = static_cast<const uint16_t*>(a.dout) + pr * kCz + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) dv[p][ks] = *reinterpret_cast<const u32x4*>(d + 32 * ks);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x8 zb[4];
        normalise(zz[p], a.eps, nv[p], zb, mu[p], rstd[p]);
        if (a.store_zh) store_zh(a, pair0 / 16 + p, n, g, nv[p], zb);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) s_z[wave][4 * p + ks][lane] = zz[p][ks];
      }
    }
    f32x4 acc[8][2];
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) acc[ct][0] = acc[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 h[3][2][2];  // A', B', dH [tile][pair tile]
    bf16x8 da[2], db[2];
    for (int c = 0; c < kHp; ++c) {
      const int b = seq & 1;
      barrier_lds();  // every wave is done with buffer b ^ 1
      const bool more = c + 1 < kHp || !last_group;
      if (more) {
        chunk_dma((c + 1) % kHp, b ^ 1);
        wait_vm<kDmaPerWave>();  // this wave's loads of chunk c have landed
      } else {
        wait_vm<0>();
      }
      barrier_lds();  // and every other wave's
      const char* chunk = s_w[b];
      constexpr int kFrags = 40, kAhead = 4;
      auto frag = [&](int f) { return *reinterpret_cast<const u32x4*>(chunk + f * 1024 + lane * 16); };
      u32x4 wq[kAhead];
#pragma unroll
      for (int f = 0; f < kAhead; ++f) wq[f] = frag(f);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int u = 32 * c + 16 * tt + 4 * g;
        const f32x4 ba = *reinterpret_cast<const f32x4*>(&s_u[kUnitBiasA][u]), bb = *reinterpret_cast<const f32x4*>(&s_u[kUnitBiasB][u]);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          h[0][tt][p] = ba;
          h[1][tt][p] = bb;
          h[2][tt][p] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        const u32x4 w = wq[f % kAhead];
        if (f + kAhead < kFrags) wq[f % kAhead] = frag(f + kAhead);
        if (f < 24) {
          const int tt = f / 12, ks = f / 3 % 4, m = f % 3;
#pragma unroll
          for (int p = 0; p < 2; ++p)
            h[m][tt][p] = m < 2 ? mfma_f16(as_f16x8(w), nv[p][ks], h[m][tt][p])
                                : mfma32(as_bf16x8(w), as_bf16x8(dv[p][ks]), h[m][tt][p]);
        } else {
          if (f == 24) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
              const int u = 32 * c + 16 * tt + 4 * g;
              const f32x4 kl = *reinterpret_cast<const f32x4*>(&s_u[kUnitLog][u]), ka = *reinterpret_cast<const f32x4*>(&s_u[kUnitA][u]);
#pragma unroll
              for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const Gated r = gated(h[0][tt][p][i], h[1][tt][p][i], h[2][tt][p][i], ka[i], kl[i]);
                  da[p][4 * tt + i] = (__bf16)r.da;
                  db[p][4 * tt + i] = (__bf16)r.db;
                }
            }
          }
          const int ct = (f - 24) / 2, m = f % 2;
#pragma unroll
          for (int p = 0; p < 2; ++p) acc[ct][p] = mfma32(as_bf16x8(w), m ? db[p] : da[p], acc[ct][p]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      ++seq;
    }
    // acc (ct = 2 ks + s, register i) is gamma dN at channel 32 ks + 8g + 4s + i of pair 16p + n
    uint32_t o[2][4][4];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      float zh[4][8], m0 = 0.0f, m1 = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const u32x4 w = s_z[wave][4 * p + ks][lane];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          zh[ks][i] = ((i & 1 ? hi_bf16(w[i >> 1]) : lo_bf16(w[i >> 1])) - mu[p]) * rstd[p];
          const float gr = acc[2 * ks + (i >> 2)][p][i & 3];
          m0 += gr;
          m1 = fmaf(gr, zh[ks][i], m1);
        }
      }
      m0 = sum4(m0) * (1.0f / kCz);
      m1 = sum4(m1) * (1.0f / kCz);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = i & 1 ? hi_bf16(dv[p][ks][i >> 1]) : lo_bf16(dv[p][ks][i >> 1]);
          v[i] = (__bf16)fmaf(rstd[p], acc[2 * ks + (i >> 2)][p][i & 3] - m0 - zh[ks][i] * m1, d);
        }
        const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
        for (int d = 0; d < 4; ++d) o[p][ks][d] = w[d];
      }
    }
    // regrouped across lanes so that a store writes 8 pairs x one whole 128-byte line
    const bool upper = (lane & 4) != 0;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int src = 8 * half + (lane >> 3) + 16 * (lane & 3);
#pragma unroll
        for (int line = 0; line < 2; ++line) {
          u32x4 v;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)o[p][2 * line][d]);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)o[p][2 * line + 1][d]);
            v[d] = upper ? hi : lo;
          }
          const int64_t pr = pair0 + 16 * p + 8 * half + (lane >> 3);
          if (pr < a.n_pairs)
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.dz) + pr * kCz) + 8 * line + (lane & 7));
        }
      }
  }
  wait_vm<0>();
}

// ----------------------------------------------------------------------------- sums over the pairs
// A workgroup of 4 waves, one per SIMD, takes 128 units (32 a wave) and a share of the steps of 32 pairs. A wave keeps
// its units' operands (96 registers) and its sums (192, of 512) throughout; zh and dout of a step, in LDS, serve
// all four. A', B' and dH come out as pairs (rows) by units: lane (unit n, group g) holds pairs 4g .. of both
// tiles, and so dA', dB' and H' are the A operands of the products over the pairs, k-slot 8g + j = pair 4g + j of
// the first tile for j < 4, of the second for j >= 4. Their B operands are columns of zh and dout, which the LDS's
// transposing reads bring: 16 lanes read four rows of 16 channels, and get four rows of one channel each.
constexpr int kStep = 32;
constexpr int kSlice = 128;
constexpr int kStepBytes = 24 * 1024;  // zh in fp16, zh in bf16, dout: 8 KB each, two tiles of 4 KB
constexpr int kAheadSteps = 2;
constexpr int kStepSlots = kAheadSteps + 2;  // and those whose products and whose sums are formed
constexpr int kStepDma = kStepBytes / 1024 / 4;
constexpr int kOpBytes = 4 * 6 * 1024;  // dA', dB', H' of a step

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__global__ void __launch_bounds__(512, 2) trans_back_sums_fast_kernel(TransBackArgs a) {
  __shared__ __attribute__((aligned(16))) char s_x[kStepSlots * kStepBytes];
  __shared__ __attribute__((aligned(16))) char s_op[2 * kOpBytes];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), share = wave & 3;
  const int hp = blockIdx.y * (kSlice / 32) + share;  // this wave's 32 units
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int64_t steps = (a.n_pairs + kStep - 1) / kStep;
  const int count = (int)((steps - blockIdx.x + gridDim.x - 1) / gridDim.x);  // of this workgroup, at least one
  constexpr int64_t kSize = (int64_t)kHid * kCz;
  float* const part = a.parts + blockIdx.x * (3 * kSize + 2 * kHid);
  char* const my_op = s_op + share * 6 * 1024 + lane * 16;
  if (wave < 4) {
    // ---- A', B', dH and what follows from them
    f16x8 w1[2][4], w2[2][4];
    bf16x8 w3[2][4];
    float k[2], kl[2], ba[2], bb[2];
    {
      const u32x4* base = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.prep) + (size_t)hp * kPairBytes) + lane;
      const float* units = reinterpret_cast<const float*>(reinterpret_cast<const char*>(a.prep) + (size_t)kHp * kPairBytes) + 32 * hp + n;
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          w1[ut][ks] = as_f16x8(base[(ut * 4 + ks) * 192]);
          w2[ut][ks] = as_f16x8(base[(ut * 4 + ks) * 192 + 64]);
          w3[ut][ks] = as_bf16x8(base[(ut * 4 + ks) * 192 + 128]);
        }
        kl[ut] = units[kUnitLog * kHid + 16 * ut];
        k[ut] = units[kUnitA * kHid + 16 * ut];
        ba[ut] = units[kUnitBiasA * kHid + 16 * ut];
        bb[ut] = units[kUnitBiasB * kHid + 16 * ut];
      }
    }
    auto sum_at = [&](int m, int ut, int i) { return 3 * kSize + m * kHid + 32 * hp + 16 * ut + 4 * g + i; };
    f32x4 s[2][2];  // S1, S2: every column of dA^T ones
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[m][ut][i] = a.add_parts ? part[sum_at(m, ut, i)] : 0.0f;
    bf16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
    const int row_at = lane * 16, drow_at = 16384 + column_lane(n, g) * 16;
    const char* cur = s_x;
    for (int it = 0; it < count; ++it) {
      barrier_lds();
      // the first tile of pairs, then the second, and between its products what follows from the first
      auto row = [&](int q) { return *reinterpret_cast<const u32x4*>(cur + (q >> 2) * 4096 + (q & 3) * 1024 + row_at); };
      auto drow = [&](int q) { return *reinterpret_cast<const u32x4*>(cur + (q >> 2) * 4096 + (q & 3) * 1024 + drow_at); };
      f32x4 h[3][2][2];
      bf16x8 op[3][2];
      auto gate = [&](int ut, int p, int i) {
        const Gated r = gated(h[0][ut][p][i], h[1][ut][p][i], h[2][ut][p][i], k[ut], kl[ut]);
        op[0][ut][4 * p + i] = (__bf16)r.da;
        op[1][ut][4 * p + i] = (__bf16)r.db;
        op[2][ut][4 * p + i] = (__bf16)r.h;
      };
      constexpr int kQueue = 3;
      u32x4 zq[kQueue], dq[kQueue];
#pragma unroll
      for (int q = 0; q < kQueue - 1; ++q) {
        zq[q] = row(q);
        dq[q] = drow(q);
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int p = q >> 2, ks = q & 3;
        if (q + kQueue - 1 < 8) {
          zq[(q + kQueue - 1) % kQueue] = row(q + kQueue - 1);
          dq[(q + kQueue - 1) % kQueue] = drow(q + kQueue - 1);
        }
        const f16x8 za = as_f16x8(zq[q % kQueue]);
        const bf16x8 d = as_bf16x8(dq[q % kQueue]);
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) {
          h[0][ut][p] = mfma_f16(za, w1[ut][ks], ks ? h[0][ut][p] : f32x4{ba[ut], ba[ut], ba[ut], ba[ut]});
          h[1][ut][p] = mfma_f16(za, w2[ut][ks], ks ? h[1][ut][p] : f32x4{bb[ut], bb[ut], bb[ut], bb[ut]});
          h[2][ut][p] = mfma32(d, w3[ut][ks], ks ? h[2][ut][p] : zero);
        }
        if (q >= 4) {
          gate(0, 0, q - 4);
          gate(1, 0, q - 4);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        gate(0, 1, i);
        gate(1, 1, i);
      }
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int ut = 0; ut < 2; ++ut)
          *reinterpret_cast<u32x4*>(my_op + (it & 1) * kOpBytes + (m * 2 + ut) * 1024) = __builtin_bit_cast(u32x4, op[m][ut]);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) s[m][ut] = mfma32(op[m][ut], ones, s[m][ut]);
      cur = cur + kStepBytes == s_x + kStepSlots * kStepBytes ? s_x : cur + kStepBytes;
    }
    barrier_lds();
    if (n == 0)
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int ut = 0; ut < 2; ++ut)
#pragma unroll
          for (int i = 0; i < 4; ++i) part[sum_at(m, ut, i)] = s[m][ut][i];
    return;
  }
  // ---- the sums of the step before, and the copies of the steps to come
  // This wave's share of a step's copies: pieces 6 share .. of 24 (piece = 4 KB tile, then ks)
  auto copy = [&](int it) {
    const int64_t step = blockIdx.x + (int64_t)it * gridDim.x;
    const uint32_t to = lds_addr(s_x) + (uint32_t)((it & (kStepSlots - 1)) * kStepBytes);
    const __amdgpu_buffer_rsrc_t zres = __builtin_amdgcn_make_buffer_rsrc(a.zh + step * (2 * 8192), 0, 2 * 8192, kRawBufferFlags);
    // pairs past the end read as zeros
    const int left = (int)min((int64_t)kStep, a.n_pairs - step * kStep);
    const __amdgpu_buffer_rsrc_t dres = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(a.dout) + step * (kStep * kCz * 2)), 0, left * kCz * 2, kRawBufferFlags);
#pragma unroll
    for (int i = 0; i < kStepDma; ++i) {
      const int piece = share * kStepDma + i, kind = piece >> 3, tile = (piece >> 2) & 1, ks = piece & 3;
      if (kind < 2)
        dma_b128(zres, tile * 8192 + kind * 4096 + ks * 1024 + lane * 16, to + (uint32_t)(piece * 1024));
      else
        dma_b128(dres, (16 * tile + (n ^ (8 * (g & 1)))) * (kCz * 2) + 64 * ks + 16 * g, to + (uint32_t)(piece * 1024));
    }
  };
  static_assert((kStepSlots & (kStepSlots - 1)) == 0, "slots by a mask");
#pragma unroll
  for (int it = 0; it < kAheadSteps; ++it)
    if (it < count) copy(it);
  auto part_at = [&](int m, int ut, int ct, int i) { return m * kSize + (32 * hp + 16 * ut + 4 * g + i) * kCz + 16 * ct + n; };
  f32x4 t[3][2][8];
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) t[m][ut][ct] = zero;
  if (a.add_parts)  // the pairs before these
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut)
#pragma unroll
        for (int ct = 0; ct < 8; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) t[m][ut][ct][i] = part[part_at(m, ut, ct, i)];
  // a column read's piece: pair 4g + n / 4, channels 4 (n % 4) .. of 16; the chunk of 8 is that of group 2 (ct % 2) + n / 2 % 2
  const int piece_odd = (n >> 1) & 1;
  const int col_at = piece_odd * 256 + ((4 * g + (n >> 2)) ^ (8 * piece_odd)) * 16 + 8 * (n & 1);
  const char* prev = s_x;
  for (int it = 0; it <= count; ++it) {
    // this wave's copies of step `it` have landed: at most those of the one after it are in flight
    if (it + 1 < count)
      wait_vm<kStepDma>();
    else
      wait_vm<0>();
    barrier_lds();  // and every other wave's; the step before the last has been read
    if (it + kAheadSteps < count) copy(it + kAheadSteps);
    if (it == 0) continue;
    bf16x8 op[3][2];
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut)
        op[m][ut] = as_bf16x8(*reinterpret_cast<const u32x4*>(my_op + ((it - 1) & 1) * kOpBytes + (m * 2 + ut) * 1024));
    auto columns = [&](int q) {  // q = 2 ct: zh, 2 ct + 1: dout
      u32x4 v;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(prev + 8192 + (q & 1) * 8192 + half * 4096 + (q >> 2) * 1024 + ((q >> 1) & 1) * 512 + col_at));
        const u32x2 w = __builtin_bit_cast(u32x2, x);
        v[2 * half] = w[0];
        v[2 * half + 1] = w[1];
      }
      return as_bf16x8(v);
    };
    constexpr int kQueue = 3;
    bf16x8 cq[kQueue];
#pragma unroll
    for (int q = 0; q < kQueue - 1; ++q) cq[q] = columns(q);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      if (q + kQueue - 1 < 16) cq[(q + kQueue - 1) % kQueue] = columns(q + kQueue - 1);
      const int ct = q >> 1;
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
        if (q & 1) {
          t[2][ut][ct] = mfma32(op[2][ut], cq[q % kQueue], t[2][ut][ct]);
        } else {
          t[0][ut][ct] = mfma32(op[0][ut], cq[q % kQueue], t[0][ut][ct]);
          t[1][ut][ct] = mfma32(op[1][ut], cq[q % kQueue], t[1][ut][ct]);
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
        for (int i = 0; i < 4; ++i) part[part_at(m, ut, ct, i)] = t[m][ut][ct][i];
}

}  // namespace

size_t trans_back_fast_prep_bytes() { return kPrepBytes; }
void trans_back_fast_units(const float* prep, const float** unit_a, const float** unit_b) {
  const float* units = reinterpret_cast<const float*>(reinterpret_cast<const char*>(prep) + (size_t)kHp * kPairBytes);
  *unit_a = units + kUnitA * kHid;
  *unit_b = units + kUnitB * kHid;
}

int trans_back_fast_splits(int64_t n_pairs) {
  const int64_t steps = (n_pairs + kStep - 1) / kStep;
  return (int)(steps < 64 ? steps : 64);
}

// Pairs at a time: 512 B of zh each in the workspace.
constexpr int64_t kChunkPairs = (int64_t)1 << 20;
size_t trans_back_fast_zh_bytes(int64_t n_pairs) {
  const int64_t groups = ((n_pairs < kChunkPairs ? n_pairs : kChunkPairs) + kGroupPairs - 1) / kGroupPairs;
  return (size_t)groups * kGroupPairs * 512;
}

hipError_t launch_trans_back_fast(const TransBackArgs& whole, hipStream_t st) {
  hipError_t e;
  hipLaunchKernelGGL(trans_back_prep_fast_kernel, dim3(kHid / 16), dim3(256), 0, st, whole);
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
    a.add_parts = p0 > 0;
    const int64_t n_groups = (a.n_pairs + kGroupPairs - 1) / kGroupPairs;
    const dim3 pairs_grid((unsigned)(n_groups < 256 ? n_groups : 256)), rows_grid((unsigned)(n_groups * 4));
    const dim3 sums_grid((unsigned)a.splits, kHid / kSlice);
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
      if (a.exponents)
        hipLaunchKernelGGL(trans_back_pairs_fast_kernel<true>, pairs_grid, dim3(64 * kWaves), 0, st, a);
      else
        hipLaunchKernelGGL(trans_back_pairs_fast_kernel<false>, pairs_grid, dim3(64 * kWaves), 0, st, a);
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
