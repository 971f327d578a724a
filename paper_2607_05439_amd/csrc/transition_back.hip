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
    u32x4 dv[2][4], zz[2][4];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int64_t pr = min(pair0 + 16 * p + n, a.n_pairs - 1);  // pairs past the end are not stored
      if (CODES) {
        const int8_t* q = static_cast<const int8_t*>(a.z) + pr * kCz + 8 * g;
        const uint32_t e = *reinterpret_cast<const uint32_t*>(a.exponents + pr * 4);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          zz[p][ks] = decode8(*reinterpret_cast<const u32x2*>(q + 32 * ks), checkpoint_scale((e >> (8 * ks)) & 255));
      } else {
        const uint16_t* q = static_cast<const uint16_t*>(a.z) + pr * kCz + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) zz[p][ks] = *reinterpret_cast<const u32x4*>(q + 32 * ks);
      }
      const uint16_t* d = static_cast<const uint16_t*>(a.dout) + pr * kCz + 8 * g;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) dv[p][ks] = *reinterpret_cast<const u32x4*>(d + 32 * ks);
    }
    f16x8 nv[2][4];
    float mu[2], rstd[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      float x[4][8], s = 0.0f, v = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        s_z[wave][4 * p + ks][lane] = zz[p][ks];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[ks][i] = i & 1 ? hi_bf16(zz[p][ks][i >> 1]) : lo_bf16(zz[p][ks][i >> 1]);
          s += x[ks][i];
        }
      }
      mu[p] = sum4(s) * (1.0f / kCz);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[ks][i] -= mu[p];
          v = fmaf(x[ks][i], x[ks][i], v);
        }
      rstd[p] = __builtin_amdgcn_rsqf(sum4(v) * (1.0f / kCz) + a.eps);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) nv[p][ks][i] = (_Float16)(x[ks][i] * rstd[p]);
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

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16-byte chunk `c` of row r of a [32][16] tile. A row is the LDS's banks once over: rows read together (16 at one
// chunk, or four at two chunks) have other chunks in other rows.
__device__ __forceinline__ int chunk_of_row(int r, int c) { return r * 16 + (c ^ (2 * (r & 7) + ((r >> 3) & 1))); }

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
// Sum over 8 consecutive lanes, the same bits in each.
__device__ __forceinline__ float sum8(float x) { return add_dpp<0x141>(add_dpp<0x4E>(add_dpp<0xB1>(x))); }

template <bool CODES>
__global__ void __launch_bounds__(256, 1) trans_back_sums_fast_kernel(TransBackArgs a) {
  __shared__ __attribute__((aligned(16))) u32x4 s_x[2][3][kStep * 16];  // zh in fp16, zh in bf16, dout
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hp = blockIdx.y * (kSlice / 32) + wave;  // this wave's 32 units
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
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
  f32x4 t[3][2][8], s[2][2];
#pragma unroll
  for (int ut = 0; ut < 2; ++ut) {
    s[0][ut] = s[1][ut] = zero;
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) t[m][ut][ct] = zero;
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;

  // staging: thread (pair sp of the step, sixteen channels from 16 sq)
  const int sp = tid >> 3, sq = tid & 7;
  const int64_t steps = (a.n_pairs + kStep - 1) / kStep;
  u32x4 zr[2], dr[2];
  float scale = 1.0f;
  bool there = false;
  auto fetch = [&](int64_t step) {
    const int64_t pair = step * kStep + sp, pr = min(pair, a.n_pairs - 1);
    there = pair < a.n_pairs;
    if (CODES) {
      zr[0] = *reinterpret_cast<const u32x4*>(static_cast<const int8_t*>(a.z) + pr * kCz + 16 * sq);
      scale = checkpoint_scale(a.exponents[pr * 4 + (sq >> 1)]);
    } else {
      const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.z) + pr * kCz) + 2 * sq;
      zr[0] = q[0];
      zr[1] = q[1];
    }
    const u32x4* d = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.dout) + pr * kCz) + 2 * sq;
    dr[0] = d[0];
    dr[1] = d[1];
  };
  auto stage = [&](int b) {
    float x[16], sum = 0.0f, var = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (CODES)
        x[i] = (float)(int8_t)(zr[0][i >> 2] >> (8 * (i & 3))) * scale;
      else
        x[i] = i & 1 ? hi_bf16(zr[i >> 3][(i >> 1) & 3]) : lo_bf16(zr[i >> 3][(i >> 1) & 3]);
      sum += x[i];
    }
    const float mu = sum8(sum) * (1.0f / kCz);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] -= mu;
      var = fmaf(x[i], x[i], var);
    }
    const float rstd = __builtin_amdgcn_rsqf(sum8(var) * (1.0f / kCz) + a.eps);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f16x8 zf;
      bf16x8 zb;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float zh = there ? x[8 * half + i] * rstd : 0.0f;
        zf[i] = (_Float16)zh;
        zb[i] = (__bf16)zh;
      }
      const int at = chunk_of_row(sp, 2 * sq + half);
      s_x[b][0][at] = __builtin_bit_cast(u32x4, zf);
      s_x[b][1][at] = __builtin_bit_cast(u32x4, zb);
      s_x[b][2][at] = there ? dr[half] : u32x4{0u, 0u, 0u, 0u};
    }
  };
  // columns of 16 channels, over the 32 pairs of tile m in buffer b
  const int tr = n >> 2, tq = n & 3;
  auto columns = [&](int b, int m, int ct) {
    u32x4 v;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = chunk_of_row(16 * half + 4 * g + tr, 2 * ct + (tq >> 1));
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(reinterpret_cast<char*>(&s_x[b][m][at]) + 8 * (tq & 1)));
      const u32x2 w = __builtin_bit_cast(u32x2, x);
      v[2 * half] = w[0];
      v[2 * half + 1] = w[1];
    }
    return as_bf16x8(v);
  };

  int64_t step = blockIdx.x;
  if (step < steps) {
    fetch(step);
    stage(0);
    if (step + gridDim.x < steps) fetch(step + gridDim.x);
  }
  __syncthreads();
  for (int b = 0; step < steps; step += gridDim.x, b ^= 1) {
    f32x4 h[3][2][2];  // A', B', dH [unit tile][pair tile]
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        h[0][ut][p] = f32x4{ba[ut], ba[ut], ba[ut], ba[ut]};
        h[1][ut][p] = f32x4{bb[ut], bb[ut], bb[ut], bb[ut]};
        h[2][ut][p] = zero;
      }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int at = chunk_of_row(16 * p + n, 4 * ks + g);
        const f16x8 zf = as_f16x8(s_x[b][0][at]);
        const bf16x8 dv = as_bf16x8(s_x[b][2][at]);
#pragma unroll
        for (int ut = 0; ut < 2; ++ut) {
          h[0][ut][p] = mfma_f16(zf, w1[ut][ks], h[0][ut][p]);
          h[1][ut][p] = mfma_f16(zf, w2[ut][ks], h[1][ut][p]);
          h[2][ut][p] = mfma32(dv, w3[ut][ks], h[2][ut][p]);
        }
      }
    bf16x8 hv[2], da[2], db[2];
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const Gated r = gated(h[0][ut][j >> 2][j & 3], h[1][ut][j >> 2][j & 3], h[2][ut][j >> 2][j & 3], k[ut], kl[ut]);
        hv[ut][j] = (__bf16)r.h;
        da[ut][j] = (__bf16)r.da;
        db[ut][j] = (__bf16)r.db;
      }
#pragma unroll
    for (int ut = 0; ut < 2; ++ut) {
      s[0][ut] = mfma32(da[ut], ones, s[0][ut]);
      s[1][ut] = mfma32(db[ut], ones, s[1][ut]);
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const bf16x8 zc = columns(b, 1, ct), dc = columns(b, 2, ct);
#pragma unroll
      for (int ut = 0; ut < 2; ++ut) {
        t[0][ut][ct] = mfma32(da[ut], zc, t[0][ut][ct]);
        t[1][ut][ct] = mfma32(db[ut], zc, t[1][ut][ct]);
        t[2][ut][ct] = mfma32(hv[ut], dc, t[2][ut][ct]);
      }
    }
    if (step + gridDim.x < steps) {
      stage(b ^ 1);
      if (step + 2 * gridDim.x < steps) fetch(step + 2 * gridDim.x);
    }
    __syncthreads();
  }
  constexpr int64_t kSize = (int64_t)kHid * kCz;
  float* part = a.parts + blockIdx.x * (3 * kSize + 2 * kHid);
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int ut = 0; ut < 2; ++ut)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[m * kSize + (32 * hp + 16 * ut + 4 * g + i) * kCz + 16 * ct + n] = t[m][ut][ct][i];
  if (n == 0)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int ut = 0; ut < 2; ++ut)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[3 * kSize + m * kHid + 32 * hp + 16 * ut + 4 * g + i] = s[m][ut][i];
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

hipError_t launch_trans_back_fast(const TransBackArgs& a, hipStream_t st) {
  hipError_t e;
  hipLaunchKernelGGL(trans_back_prep_fast_kernel, dim3(kHid / 16), dim3(256), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  // The sums read dout, which dz may take the place of: they come first.
  if (a.dw1 || a.dw2 || a.dw3 || a.dgamma || a.dbeta) {
    const dim3 grid((unsigned)a.splits, kHid / kSlice);
    if (a.exponents)
      hipLaunchKernelGGL(trans_back_sums_fast_kernel<true>, grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(trans_back_sums_fast_kernel<false>, grid, dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!a.dz) return hipSuccess;
  const int64_t n_groups = (a.n_pairs + kGroupPairs - 1) / kGroupPairs;
  const dim3 grid((unsigned)(n_groups < 256 ? n_groups : 256));
  if (a.exponents)
    hipLaunchKernelGGL(trans_back_pairs_fast_kernel<true>, grid, dim3(64 * kWaves), 0, st, a);
  else
    hipLaunchKernelGGL(trans_back_pairs_fast_kernel<false>, grid, dim3(64 * kWaves), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
