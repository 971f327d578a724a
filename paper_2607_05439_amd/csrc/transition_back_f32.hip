// Backward pass of the pair transition in fp32, and the sums that every path of it ends in (gfx950).
//
// Per pair, with zh = (z - mean z) rstd, N = gamma zh + beta, A = W1 N, B = W2 N, s = sigmoid(A):
//   H = A s B,  dH = W3^T dout,  dB = dH A s,  dA = dH B (s + A s (1 - s)),
//   dN = W1^T dA + W2^T dB,  g = gamma dN,
//   dz = dout + rstd (g - mean g - zh mean(g zh)).
// Over the pairs, T1 = sum dA zh^T, T2 = sum dB zh^T, S1 = sum dA, S2 = sum dB:
//   dW1 = T1 diag(gamma) + S1 beta^T, dW2 likewise, dW3 = sum dout H^T,
//   dgamma = sum over units of W1 T1 + W2 T2, dbeta = sum over units of W1 S1 + W2 S2,
// so that the affine weights' gradients need no sums over the pairs of their own.
//
// Nothing of the hidden width leaves a kernel: one kernel forms dz and another the sums,
// and each forms A, B and dH again. Products and sums are fp32 on the fp32 matrix cores.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"
#include "checkpoint.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

struct Gated {
  float h, da, db;
};
// The hardware's exp2 and reciprocal are off by 2^-23 of the result, and log2(e) a by 2^-24 of itself, so the sigmoid by
// 2^-22 + 2^-24 |a| at most.
__device__ __forceinline__ Gated gated(float a, float b, float dh) {
  const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * a)), silu = a * s;
  return {silu * b, dh * b * (s + silu * (1.0f - s)), dh * silu};
}

// ----------------------------------------------------------------------------- weights
// The weights and their transposes, filled up with zeros to whole tiles of 16 (hp units, cp
// channels): [hp][cp] W1, W2, W3^T, then [cp][hp] W1^T, W2^T, then gamma and beta [cp].
__global__ void __launch_bounds__(256) trans_back_prep_kernel(TransBackArgs a) {
  const int cp = (a.c + 15) & ~15, hp = (a.hidden + 15) & ~15, n = cp * hp;
  for (int t = blockIdx.x * 256 + threadIdx.x; t < n + cp; t += gridDim.x * 256) {
    if (t >= n) {
      const int c = t - n;
      a.prep[5 * (int64_t)n + c] = c < a.c ? (a.gamma ? a.gamma[c] : 1.0f) : 0.0f;
      a.prep[5 * (int64_t)n + cp + c] = c < a.c && a.beta ? a.beta[c] : 0.0f;
      continue;
    }
    const int u = t / cp, c = t - u * cp;
    const bool in = u < a.hidden && c < a.c;
    const float w1 = in ? a.w1[(int64_t)u * a.c + c] : 0.0f, w2 = in ? a.w2[(int64_t)u * a.c + c] : 0.0f;
    a.prep[t] = w1;
    a.prep[(int64_t)n + t] = w2;
    a.prep[2 * (int64_t)n + t] = in ? a.w3[(int64_t)c * a.hidden + u] : 0.0f;
    a.prep[3 * (int64_t)n + (int64_t)c * hp + u] = w1;
    a.prep[4 * (int64_t)n + (int64_t)c * hp + u] = w2;
  }
}

// ----------------------------------------------------------------------------- rows as they are stored
// Four channels from c0 of a pair, zeros past c and past the last pair.
__device__ __forceinline__ f32x4 load4(const TransBackArgs& a, const void* x, bool codes, bool vec, int64_t pair, int c0) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (pair >= a.n_pairs || c0 >= a.c) return v;
  const int64_t at = pair * a.c + c0;
  const int n = min(4, a.c - c0);
  if (codes) {
    const int8_t* q = static_cast<const int8_t*>(x) + at;
    const float scale = checkpoint_scale(a.exponents[pair * checkpoint_blocks(a.c) + c0 / kCheckpointBlock]);
    if (vec) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(q);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * scale;
    } else {
      for (int i = 0; i < n; ++i) v[i] = (float)q[i] * scale;
    }
  } else if (vec) {
    v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + at);
  } else {
    for (int i = 0; i < n; ++i) v[i] = static_cast<const float*>(x)[at + i];
  }
  return v;
}

// ----------------------------------------------------------------------------- sums over the pairs
// A workgroup takes 64 units (16 a wave) and a share of the tiles of 16 pairs. A wave keeps its
// units' rows of W1, W2 and W3^T and its sums in registers. A, B and dH come out as pairs 4g + i
// (rows) of unit n (column), which is the A operand of the products over the pairs: step i has
// pair 4g + i in k-slot g. Their B operand is zh or dout of that pair at channel 16j + n, from LDS. Bound by the matrix cores where
// there are many pairs (65536 of 32 channels and 128 units 53 us), by the loads' latency of a tile below (16384: 21 us).
template <int CT>
__global__ void __launch_bounds__(256, CT > 8 ? 1 : 2) trans_back_sums_kernel(TransBackArgs a) {
  constexpr int kC = 16 * CT, kRow = kC + 4;
  __shared__ f32x4 s_n[CT][64], s_d[CT][64];  // N and dout as operands: lane (pair n, g), channels 16j + 4g ..
  __shared__ float s_zh[16][kRow], s_do[16][kRow];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cp = (a.c + 15) & ~15, hp = (a.hidden + 15) & ~15;
  const int u0 = blockIdx.x * 64 + wave * 16;
  const bool active = u0 < hp;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  constexpr int kHeld = CT > 8 ? 1 : CT;  // wide rows: the weights from L2 for every tile
  f32x4 w[3][kHeld], t[3][CT];
  const float* const wrow = a.prep + (int64_t)(active ? u0 + n : 0) * cp + 4 * g;
  float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      t[m][j] = zero;
      if (CT > 8) continue;
      w[m][j] = zero;
      if (active && 16 * j < cp) w[m][j] = *reinterpret_cast<const f32x4*>(wrow + m * (int64_t)hp * cp + 16 * j);
    }
  // Staging: 16 threads a pair, thread q of them channels 4 (q + 16 k)
  constexpr int kQ = (CT * 4 + 15) / 16;
  const int sp = tid >> 4, sq = tid & 15;
  const float* gb = a.prep + 5 * (int64_t)hp * cp;
  const int64_t tiles = (a.n_pairs + 15) / 16;
  f32x4 z[kQ], d[kQ];
  auto fetch = [&](int64_t tile) {
#pragma unroll
    for (int k = 0; k < kQ; ++k) {
      z[k] = load4(a, a.z, a.exponents != nullptr, a.z_vec, tile * 16 + sp, 4 * (sq + 16 * k));
      d[k] = load4(a, a.dout, false, a.d_vec, tile * 16 + sp, 4 * (sq + 16 * k));
    }
  };
  int64_t tile = blockIdx.y;
  if (tile < tiles) fetch(tile);
  for (; tile < tiles; tile += gridDim.y) {
    float sum = 0.0f, var = 0.0f;
#pragma unroll
    for (int k = 0; k < kQ; ++k) sum += (z[k][0] + z[k][1]) + (z[k][2] + z[k][3]);
    for (int m = 8; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    const float mu = sum / (float)a.c;
    const bool there = tile * 16 + sp < a.n_pairs;
#pragma unroll
    for (int k = 0; k < kQ; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[k][i] = there && 4 * (sq + 16 * k) + i < a.c ? z[k][i] - mu : 0.0f;
        var = fmaf(z[k][i], z[k][i], var);
      }
    for (int m = 8; m > 0; m >>= 1) var += __shfl_xor(var, m);
    const float rstd = there ? 1.0f / sqrtf(var / (float)a.c + a.eps) : 0.0f;
    __syncthreads();  // the tile before has been read
#pragma unroll
    for (int k = 0; k < kQ; ++k) {
      const int q = sq + 16 * k, c0 = 4 * q;
      if (q >= 4 * CT) continue;
      f32x4 nv = zero;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[k][i] *= rstd;
        if (there && c0 + i < a.c) nv[i] = fmaf(z[k][i], gb[c0 + i], gb[cp + c0 + i]);
      }
      s_n[q >> 2][sp + 16 * (q & 3)] = nv;
      s_d[q >> 2][sp + 16 * (q & 3)] = d[k];
      *reinterpret_cast<f32x4*>(&s_zh[sp][c0]) = z[k];
      *reinterpret_cast<f32x4*>(&s_do[sp][c0]) = d[k];
    }
    __syncthreads();
    if (tile + gridDim.y < tiles) fetch(tile + gridDim.y);
    f32x4 x = zero, y = zero, dh = zero;
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      if (16 * j >= cp) continue;
      const f32x4 nv = s_n[j][lane], dv = s_d[j][lane];
      if (CT > 8)
#pragma unroll
        for (int m = 0; m < 3; ++m) w[m][0] = *reinterpret_cast<const f32x4*>(wrow + m * (int64_t)hp * cp + 16 * j);
      constexpr int kLast = kHeld - 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x = mfma4(nv[i], w[0][min(j, kLast)][i], x);
        y = mfma4(nv[i], w[1][min(j, kLast)][i], y);
        dh = mfma4(dv[i], w[2][min(j, kLast)][i], dh);
      }
    }
    f32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Gated r = gated(x[i], y[i], dh[i]);
      h[i] = r.h;
      x[i] = r.da;
      y[i] = r.db;
      s1 += r.da;
      s2 += r.db;
    }
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float zh = s_zh[4 * g + i][16 * j + n], dv = s_do[4 * g + i][16 * j + n];
        t[0][j] = mfma4(x[i], zh, t[0][j]);
        t[1][j] = mfma4(y[i], zh, t[1][j]);
        t[2][j] = mfma4(h[i], dv, t[2][j]);
      }
  }
  if (!active) return;
  const int64_t size = (int64_t)hp * cp;
  float* part = a.parts + blockIdx.y * (3 * size + 2 * hp);
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int j = 0; j < CT; ++j)
      if (16 * j < cp)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[m * size + (int64_t)(u0 + 4 * g + i) * cp + 16 * j + n] = t[m][j][i];
  s1 = sum4(s1);
  s2 = sum4(s2);
  if (g == 0) {
    part[3 * size + u0 + n] = s1;
    part[3 * size + hp + u0 + n] = s2;
  }
}

// The same for 65 to 128 channels: there the weights and sums of a wave leave no room for a second wave on its SIMD (36864
// pairs of 128 channels and 512 units: 410 us). The weights of the 64 units lie in LDS instead, for eight waves,
// of which four take one tile of 16 pairs and four another, with sums of their own: a workgroup's two parts. 298 us, the matrix
// cores 72% busy; they wait for the rows' statistics, which all waves form between two barriers.
constexpr int kWideTiles = 8;  // of 16 channels
__global__ void __launch_bounds__(512, 2) trans_back_sums_wide_kernel(TransBackArgs a) {
  constexpr int CT = kWideTiles, kRow = 16 * CT + 4;
  __shared__ f32x4 s_w[4][3][CT][64];
  __shared__ __attribute__((aligned(16))) float s_x[3][2][16][kRow];  // N, zh, dout of both tiles
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), ut = wave & 3, half = wave >> 2;
  const int cp = (a.c + 15) & ~15, hp = (a.hidden + 15) & ~15;
  const int64_t size = (int64_t)hp * cp;
  const int u0 = blockIdx.x * 64 + ut * 16;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  for (int k = tid; k < 4 * 3 * CT * 64; k += 512) {
    const int l = k & 63, j = (k >> 6) % CT, m = (k / (64 * CT)) % 3, t = k / (64 * CT * 3), u = blockIdx.x * 64 + 16 * t + (l & 15);
    (&s_w[0][0][0][0])[k] = u < hp && 16 * j < cp ? *reinterpret_cast<const f32x4*>(a.prep + m * size + (int64_t)u * cp + 16 * j + 4 * (l >> 4)) : zero;
  }
  f32x4 t[3][CT];
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int j = 0; j < CT; ++j) t[m][j] = zero;
  float s1 = 0.0f, s2 = 0.0f;
  // staging: 16 threads a pair, thread q of them channels 4 q and 4 (q + 16)
  const int sh = tid >> 8, sp = (tid >> 4) & 15, sq = tid & 15;
  const float* gb = a.prep + 5 * size;
  f32x4 ga[2], be[2], z[2], d[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c0 = 4 * (sq + 16 * k);
    ga[k] = c0 < cp ? *reinterpret_cast<const f32x4*>(gb + c0) : zero;
    be[k] = c0 < cp ? *reinterpret_cast<const f32x4*>(gb + cp + c0) : zero;
  }
  const int64_t tiles = (a.n_pairs + 31) / 32;
  auto fetch = [&](int64_t tile) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      z[k] = load4(a, a.z, a.exponents != nullptr, a.z_vec, tile * 32 + 16 * sh + sp, 4 * (sq + 16 * k));
      d[k] = load4(a, a.dout, false, a.d_vec, tile * 32 + 16 * sh + sp, 4 * (sq + 16 * k));
    }
  };
  int64_t tile = blockIdx.y;
  if (tile < tiles) fetch(tile);
  for (; tile < tiles; tile += gridDim.y) {
    float sum = 0.0f, var = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k) sum += (z[k][0] + z[k][1]) + (z[k][2] + z[k][3]);
    for (int m = 8; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    const float mu = sum / (float)a.c;
    const bool there = tile * 32 + 16 * sh + sp < a.n_pairs;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[k][i] = there && 4 * (sq + 16 * k) + i < a.c ? z[k][i] - mu : 0.0f;
        var = fmaf(z[k][i], z[k][i], var);
      }
    for (int m = 8; m > 0; m >>= 1) var += __shfl_xor(var, m);
    const float rstd = there ? 1.0f / sqrtf(var / (float)a.c + a.eps) : 0.0f;
    barrier_lds();  // the tiles before have been read
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int c0 = 4 * (sq + 16 * k);
      f32x4 nv;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[k][i] *= rstd;
        nv[i] = there && c0 + i < a.c ? fmaf(z[k][i], ga[k][i], be[k][i]) : 0.0f;
      }
      *reinterpret_cast<f32x4*>(&s_x[0][sh][sp][c0]) = nv;
      *reinterpret_cast<f32x4*>(&s_x[1][sh][sp][c0]) = z[k];
      *reinterpret_cast<f32x4*>(&s_x[2][sh][sp][c0]) = d[k];
    }
    barrier_lds();
    if (tile + gridDim.y < tiles) fetch(tile + gridDim.y);
    f32x4 x = zero, y = zero, h = zero;
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const f32x4 nv = *reinterpret_cast<const f32x4*>(&s_x[0][half][n][16 * j + 4 * g]);
      const f32x4 dv = *reinterpret_cast<const f32x4*>(&s_x[2][half][n][16 * j + 4 * g]);
      const f32x4 w1 = s_w[ut][0][j][lane], w2 = s_w[ut][1][j][lane], w3 = s_w[ut][2][j][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x = mfma4(nv[i], w1[i], x);
        y = mfma4(nv[i], w2[i], y);
        h = mfma4(dv[i], w3[i], h);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Gated r = gated(x[i], y[i], h[i]);
      h[i] = r.h;
      x[i] = r.da;
      y[i] = r.db;
      s1 += r.da;
      s2 += r.db;
    }
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float zh = s_x[1][half][4 * g + i][16 * j + n], dv = s_x[2][half][4 * g + i][16 * j + n];
        t[0][j] = mfma4(x[i], zh, t[0][j]);
        t[1][j] = mfma4(y[i], zh, t[1][j]);
        t[2][j] = mfma4(h[i], dv, t[2][j]);
      }
  }
  if (u0 >= hp) return;
  float* part = a.parts + (2 * (int64_t)blockIdx.y + half) * (3 * size + 2 * hp);
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int j = 0; j < CT; ++j)
      if (16 * j < cp)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[m * size + (int64_t)(u0 + 4 * g + i) * cp + 16 * j + n] = t[m][j][i];
  s1 = sum4(s1);
  s2 = sum4(s2);
  if (g == 0) {
    part[3 * size + u0 + n] = s1;
    part[3 * size + hp + u0 + n] = s2;
  }
}

// ----------------------------------------------------------------------------- dz
// A workgroup takes P tiles of 16 pairs; its waves take every fourth tile of 16 units. The
// products are transposed (units by pairs), so that A, B and dH lie as the B operands of the
// products with W1^T and W2^T, and dN as z does: channels 16j + 4g .. of pair n. The waves' dN
// meet in LDS. 36864 pairs of 128 channels and 512 units: 277 us, the matrix cores 72% busy; 1152 workgroups are two rounds
// and a quarter.
template <int CT, int P>
__global__ void __launch_bounds__(256, CT > 8 ? 1 : 2) trans_back_pairs_kernel(TransBackArgs a) {
  __shared__ union {
    struct {
      f32x4 n[P][CT][64], d[P][CT][64];
    } in;
    f32x4 red[4][P][CT][64];
  } s;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cp = (a.c + 15) & ~15, hp = (a.hidden + 15) & ~15;
  const int64_t size = (int64_t)hp * cp, tile0 = (a.first_block + blockIdx.x) * P;
  const float* gb = a.prep + 5 * size;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto chunk = [](const float* p) { return *reinterpret_cast<const f32x4*>(p); };
  // zh of a tile's pairs, and rstd
  f32x4 zh[CT];
  auto normalised = [&](int64_t pair) {
    float sum = 0.0f, var = 0.0f;
#pragma unroll
    for (int j = 0; j < CT; ++j) zh[j] = load4(a, a.z, a.exponents != nullptr, a.z_vec, pair, 16 * j + 4 * g);
#pragma unroll
    for (int j = 0; j < CT; ++j) sum += (zh[j][0] + zh[j][1]) + (zh[j][2] + zh[j][3]);
    const float mu = sum4(sum) / (float)a.c;
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        zh[j][i] = 16 * j + 4 * g + i < a.c ? zh[j][i] - mu : 0.0f;
        var = fmaf(zh[j][i], zh[j][i], var);
      }
    const float rstd = 1.0f / sqrtf(sum4(var) / (float)a.c + a.eps);
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) zh[j][i] *= rstd;
    return rstd;
  };
  if (wave < P) {
    const int64_t pair = (tile0 + wave) * 16 + n;
    normalised(pair);
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      f32x4 nv = zero;
      const int c0 = 16 * j + 4 * g;
      if (c0 < cp) {
        const f32x4 ga = chunk(gb + c0), be = chunk(gb + cp + c0);
#pragma unroll
        for (int i = 0; i < 4; ++i) nv[i] = c0 + i < a.c ? fmaf(zh[j][i], ga[i], be[i]) : 0.0f;
      }
      s.in.n[wave][j][lane] = nv;
      s.in.d[wave][j][lane] = load4(a, a.dout, false, a.d_vec, pair, c0);
    }
  }
  __syncthreads();
  // a product waits for the one before it on the same sum: with one tile of pairs two sums, of even and of odd steps (4096 pairs of
  // 128 channels: 53 -> 48 us)
  constexpr int kWays = P == 1 && CT <= 8 ? 2 : 1;
  f32x4 dn[P * kWays][CT];
#pragma unroll
  for (int p = 0; p < P * kWays; ++p)
#pragma unroll
    for (int j = 0; j < CT; ++j) dn[p][j] = zero;
  if constexpr (CT > 8) {  // one wave a SIMD: loads as far ahead as 512 registers let the compiler place them (a queue: half as fast)
    for (int ht = wave; ht < hp / 16; ht += 4) {
      const float* w = a.prep + (int64_t)(16 * ht + n) * cp + 4 * g;
      f32x4 x[P], y[P], dh[P];
#pragma unroll
      for (int p = 0; p < P; ++p) x[p] = y[p] = dh[p] = zero;
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        if (16 * j >= cp) continue;
        const f32x4 w1 = chunk(w + 16 * j), w2 = chunk(w + size + 16 * j), w3 = chunk(w + 2 * size + 16 * j);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const f32x4 nv = s.in.n[p][j][lane], dv = s.in.d[p][j][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[p] = mfma4(w1[i], nv[i], x[p]);
            y[p] = mfma4(w2[i], nv[i], y[p]);
            dh[p] = mfma4(w3[i], dv[i], dh[p]);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Gated r = gated(x[p][i], y[p][i], dh[p][i]);
          x[p][i] = r.da;
          y[p][i] = r.db;
        }
      const float* wt = a.prep + 3 * size + (int64_t)n * hp + 16 * ht + 4 * g;
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        if (16 * j >= cp) continue;
        const f32x4 w1 = chunk(wt + (int64_t)16 * j * hp), w2 = chunk(wt + size + (int64_t)16 * j * hp);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dn[p][j] = mfma4(w1[i], x[p][i], dn[p][j]);
            dn[p][j] = mfma4(w2[i], y[p][i], dn[p][j]);
          }
      }
    }
  } else {
    // Weights of a tile of units in the order of their use: rows of W1, W2 and W3^T at 16 channels each, then of the
    // transposes. They come from L2, five ahead across the tiles (36864 pairs: 316 us without, 20 ahead spill).
    constexpr int kFrags = 5 * CT, kAhead = 5;
    const int last = hp / 16 - 1;
    auto frag = [&](int ht, int f) {
      const int j = f < 3 * CT ? f / 3 : (f - 3 * CT) / 2, m = f < 3 * CT ? f % 3 : 3 + (f - 3 * CT) % 2, in = 16 * j < cp ? j : 0;
      ht = min(ht, last);
      return chunk(a.prep + m * size + (m < 3 ? (int64_t)(16 * ht + n) * cp + 16 * in : (int64_t)(16 * in + n) * hp + 16 * ht) + 4 * g);
    };
    f32x4 wq[kAhead];
#pragma unroll
    for (int f = 0; f < kAhead; ++f) wq[f] = frag(wave, f);
#pragma unroll 1
    for (int ht = wave; ht <= last; ht += 4) {
      f32x4 h[3][P * kWays];
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int p = 0; p < P * kWays; ++p) h[m][p] = zero;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        const f32x4 w = wq[f % kAhead];
        wq[f % kAhead] = f + kAhead < kFrags ? frag(ht, f + kAhead) : frag(ht + 4, f + kAhead - kFrags);
        if (f < 3 * CT) {
          const int j = f / 3, m = f % 3;
          f32x4 v[P];
          if (16 * j < cp)
#pragma unroll
            for (int p = 0; p < P; ++p) v[p] = m < 2 ? s.in.n[p][j][lane] : s.in.d[p][j][lane];
          if (16 * j < cp)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int p = 0; p < P; ++p) h[m][p + i % kWays] = mfma4(w[i], v[p][i], h[m][p + i % kWays]);
        } else {
          const int j = (f - 3 * CT) / 2, m = (f - 3 * CT) % 2;
          if (16 * j < cp)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int p = 0; p < P; ++p) dn[p + i % kWays][j] = mfma4(w[i], h[m][p][i], dn[p + i % kWays][j]);
        }
        if (f == 3 * CT - 1)
#pragma unroll
          for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (kWays == 2)
#pragma unroll
                for (int m = 0; m < 3; ++m) h[m][p][i] += h[m][p + kWays - 1][i];
              const Gated r = gated(h[0][p][i], h[1][p][i], h[2][p][i]);
              h[0][p][i] = r.da;
              h[1][p][i] = r.db;
            }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  __syncthreads();  // N and dout have been read
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < CT; ++j) s.red[wave][p][j][lane] = kWays == 2 ? dn[p][j] + dn[p + kWays - 1][j] : dn[p][j];
  __syncthreads();
  if (wave >= P) return;
  const int64_t pair = (tile0 + wave) * 16 + n;
  const float rstd = normalised(pair);
  f32x4 gr[CT];
  float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    const int c0 = 16 * j + 4 * g;
    const f32x4 sum = ((s.red[0][wave][j][lane] + s.red[1][wave][j][lane]) + s.red[2][wave][j][lane]) + s.red[3][wave][j][lane];
    gr[j] = c0 < cp ? sum * chunk(gb + c0) : zero;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m0 += gr[j][i];
      m1 = fmaf(gr[j][i], zh[j][i], m1);
    }
  }
  m0 = sum4(m0) / (float)a.c;
  m1 = sum4(m1) / (float)a.c;
  if (pair >= a.n_pairs) return;
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    const int c0 = 16 * j + 4 * g;
    if (c0 >= a.c) continue;
    const f32x4 dv = load4(a, a.dout, false, a.d_vec, pair, c0);
    const int64_t at = pair * a.c + c0;
    f32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = dv[i] + rstd * (gr[j][i] - m0 - zh[j][i] * m1);
    if (a.d_vec) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.dz) + at) = o;
    } else {
      for (int i = 0; i < min(4, a.c - c0); ++i) static_cast<float*>(a.dz)[at + i] = o[i];
    }
  }
}

// ----------------------------------------------------------------------------- weights' gradients from the parts
__device__ __forceinline__ void put(void* p, int64_t at, float v, bool bf16) {
  if (bf16)
    static_cast<uint16_t*>(p)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
  else
    static_cast<float*>(p)[at] = v;
}

// One unit a workgroup: the splits' sums, dW1, dW2 and dW3, and the unit's shares of dgamma and dbeta. Threads of
// four channels take every `ways`-th split, and their sums are added in order: 64 splits of 512 x 128 in 8 us, where
// one thread per channel over all splits took 24.
__global__ void __launch_bounds__(256) trans_back_finish_kernel(TransBackArgs a) {
  __shared__ f32x4 s_t[3][256];
  __shared__ float s_s[2][64];
  const int cp = (a.c + 15) & ~15, hp = (a.hidden + 15) & ~15, u = blockIdx.x;
  const int quads = cp / 4, ways = 256 / quads, way = threadIdx.x / quads, q = threadIdx.x - way * quads;
  const int64_t size = (int64_t)hp * cp, stride = 3 * size + 2 * hp;
  if (way < ways) {
    f32x4 t[3] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 8
    for (int sp = way; sp < a.splits; sp += ways) {
      const float* p = a.parts + sp * stride + (int64_t)u * cp + 4 * q;
#pragma unroll
      for (int m = 0; m < 3; ++m) t[m] += *reinterpret_cast<const f32x4*>(p + m * size);
      s1 += a.parts[sp * stride + 3 * size + u];
      s2 += a.parts[sp * stride + 3 * size + hp + u];
    }
#pragma unroll
    for (int m = 0; m < 3; ++m) s_t[m][threadIdx.x] = t[m];
    if (q == 0) {
      s_s[0][way] = s1;
      s_s[1][way] = s2;
    }
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= a.c) return;
  float t[3] = {0.f, 0.f, 0.f}, s[2] = {0.f, 0.f};
  for (int w = 0; w < ways; ++w) {
#pragma unroll
    for (int m = 0; m < 3; ++m) t[m] += reinterpret_cast<const float*>(&s_t[m][w * quads])[c];
#pragma unroll
    for (int m = 0; m < 2; ++m) s[m] += s_s[m][w];
  }
  if (a.unit_exponents) {
    const int e1 = a.unit_exponents[u], e2 = a.unit_exponents[a.hidden + u], e3 = a.unit_exponents[2 * a.hidden + u], d = *a.dout_exponent;
    t[0] = ldexpf(t[0], -(e2 + e3 + d));
    s[0] = ldexpf(s[0], -(e2 + e3 + d));
    t[1] = ldexpf(t[1], -(e1 + e3 + d));
    s[1] = ldexpf(s[1], -(e1 + e3 + d));
    t[2] = ldexpf(t[2], -(e1 + e2 + d));
  }
  const float ga = a.gamma ? a.gamma[c] : 1.0f, be = a.beta ? a.beta[c] : 0.0f;
  const int64_t at = (int64_t)u * a.c + c;
  if (a.dw1) put(a.dw1, at, fmaf(t[0], ga, s[0] * be), a.grads_bf16);
  if (a.dw2) put(a.dw2, at, fmaf(t[1], ga, s[1] * be), a.grads_bf16);
  if (a.dw3) put(a.dw3, (int64_t)c * a.hidden + u, t[2], a.grads_bf16);
  const float w1 = a.w1[at], w2 = a.w2[at];
  a.affine_parts[(int64_t)u * 2 * a.c + c] = fmaf(w1, t[0], w2 * t[1]);
  a.affine_parts[((int64_t)u * 2 + 1) * a.c + c] = fmaf(w1, s[0], w2 * s[1]);
}

// dgamma and dbeta: 16 of the 2 c sums a workgroup, 16 threads each.
__global__ void __launch_bounds__(256) trans_back_affine_kernel(TransBackArgs a) {
  __shared__ float s_sum[16][17];
  const int lane = threadIdx.x & 15, way = threadIdx.x >> 4, k = blockIdx.x * 16 + lane;
  float sum = 0.0f;
  if (k < 2 * a.c)
#pragma unroll 8
    for (int u = way; u < a.hidden; u += 16) sum += a.affine_parts[(int64_t)u * 2 * a.c + k];
  s_sum[way][lane] = sum;
  __syncthreads();
  if (way > 0 || k >= 2 * a.c) return;
  sum = 0.0f;
  for (int w = 0; w < 16; ++w) sum += s_sum[w][lane];
  void* out = k < a.c ? a.dgamma : a.dbeta;
  if (out) put(out, k < a.c ? k : k - a.c, sum, a.grads_bf16);
}

template <int CT, int P>
hipError_t launch_pairs(TransBackArgs a, hipStream_t st) {
  const int64_t total = (a.n_pairs + 16 * P - 1) / (16 * P);
  hipError_t e = hipSuccess;
  for (; a.first_block < total && e == hipSuccess; a.first_block += kLaunchBlocks) {
    const dim3 grid((unsigned)(total - a.first_block < kLaunchBlocks ? total - a.first_block : kLaunchBlocks));
    hipLaunchKernelGGL((trans_back_pairs_kernel<CT, P>), grid, dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}
template <int CT>
hipError_t launch_sums(const TransBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((trans_back_sums_kernel<CT>), dim3((unsigned)((a.hidden + 63) / 64), (unsigned)a.splits), dim3(256), 0,
                     st, a);
  return hipGetLastError();
}

// One round of workgroups, of which a CU holds two where rows are of at most 64 channels and one where they are wider; those
// of the wide kernel give two parts.
bool wide(int32_t c) { return c > 64 && c <= 16 * kWideTiles; }

}  // namespace

int trans_back_gen_splits(int64_t n_pairs, int32_t c, int32_t hidden) {
  const int pairs = wide(c) ? 32 : 16;
  const int64_t tiles = (n_pairs + pairs - 1) / pairs, groups = (hidden + 63) / 64, room = c > 64 ? 256 : 512;
  const int64_t most = room > groups ? room / groups : 1;
  return (int)(tiles < most ? tiles : most) * (wide(c) ? 2 : 1);
}

hipError_t launch_trans_back_gen(const TransBackArgs& a, hipStream_t st) {
  hipError_t e;
  hipLaunchKernelGGL(trans_back_prep_kernel, dim3(128), dim3(256), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.dw1 || a.dw2 || a.dw3 || a.dgamma || a.dbeta) {
    if (wide(a.c))
      hipLaunchKernelGGL(trans_back_sums_wide_kernel, dim3((unsigned)((a.hidden + 63) / 64), (unsigned)(a.splits / 2)), dim3(512), 0, st, a);
    e = wide(a.c) ? hipGetLastError() : a.c > 128 ? launch_sums<16>(a, st) : a.c > 32 ? launch_sums<4>(a, st) : launch_sums<2>(a, st);
    if (e != hipSuccess) return e;
  }
  if (!a.dz) return hipSuccess;
  // Two tiles of pairs share the weights' loads, unless that leaves CUs idle (256 channels: 4096 pairs 250 us with one, 326 with
  // two; 20000 pairs 1208 and 971).
  if (a.n_pairs <= 4096)
    return a.c > 128 ? launch_pairs<16, 1>(a, st) : a.c > 64 ? launch_pairs<8, 1>(a, st) : a.c > 32 ? launch_pairs<4, 1>(a, st) : launch_pairs<2, 1>(a, st);
  return a.c > 128 ? launch_pairs<16, 2>(a, st) : a.c > 64 ? launch_pairs<8, 2>(a, st) : a.c > 32 ? launch_pairs<4, 2>(a, st) : launch_pairs<2, 2>(a, st);
}

hipError_t launch_trans_back_finish(const TransBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(trans_back_finish_kernel, dim3((unsigned)a.hidden), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.dgamma && !a.dbeta)) return e;
  hipLaunchKernelGGL(trans_back_affine_kernel, dim3((unsigned)((2 * a.c + 15) / 16)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
