// Backward pass of the attention on the matrix cores: c_z = 128, H = 16, d = 24, bf16
// activations (gfx950). The formulas are in backward.hip.
//
// Kernels, in order:
//   prep_kernel   the weights as operands; the largest |dout| of each row
//   (token_gemm.hip: q, k, v, g, and the largest |q|, |k|, |v|)
//   pack_kernel   q, do of the rows and k, v of the keys as fp16 operands; dg
//   stats_kernel  16 query rows and a range of keys per workgroup: maximum and sum of the
//                 weights, and sum P dP, of the logits that pairs_kernel forms
//   pairs_kernel  the same rows and keys again: bias, P, dS, dz, dq, T
//   keys_kernel   64 keys of a head per workgroup: dk, dv from the stored P
// then sums of parts (backward.hip), ds and dW (token_gemm.hip) and the gradients in their
// own types (backward.hip).
//
// Operands are fp16, not bf16: 11 significant bits where bf16 has 8, at the same rate, so
// that the roundings inside stay an eighth of the result's own rounding to bf16. Their
// range is served by powers of two: every tensor is scaled so that its largest
// magnitude lies in [2^11, 2^12) (P, at most 1, by 2^14; dS then by what keeps it below
// 2^16), fp16 holds 11 bits down to 2^-25 of that, and the fp32 results are scaled
// back exactly. Every row of dout has a power of its own for what stays in the row (dS,
// dz, dq), and joins the others at the tensor's where rows are summed. Only z enters as
// the bf16 it is, against bias weights split into bf16 hi + lo (pair_bias.h).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"
#include "dcp_internal.h"
#include "pair_bias.h"

namespace dcp {
namespace {

constexpr int kCz = kFastCz, kH = kFastH, kD = kFastD, kDp = kFastDp, kHD = kFastH * kFastD;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInvSqrtD = 0.20412414523193150818f;  // 1 / sqrt(24)
constexpr int kPShift = 14;       // P is stored times 2^14
constexpr int kTop = 11;          // operands have their largest magnitude in [2^11, 2^12)
constexpr int kDsShift = 14;      // dS = P (dP' - D') 2^-14: |dP' - D'| <= 2 * 24 * 2^24

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma32h(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16h(f16x4 a, f16x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16x8 as_f16x8(u32x4 u) { return __builtin_bit_cast(f16x8, u); }
__device__ __forceinline__ f16x4 to_f16(f32x4 v) {
  f16x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (_Float16)v[i];
  return r;
}

// The power of two that takes a largest magnitude into [2^kTop, 2^(kTop + 1)): 1 where
// there is none (all zero). It is taken over the finite values: one that is not stays so at
// any power, and the others keep theirs.
__device__ __forceinline__ int scale_exp(float top) {
  if (!(top > 0.0f)) return 0;
  int e;
  (void)frexpf(top, &e);  // top = f 2^e, f in [0.5, 1)
  return max(-100, min(100, kTop + 1 - e));
}

// ----------------------------------------------------------------------------- weights, dout
// Block 0: the bias weights. Blocks 1 .. kBackTops: the largest |dout| of each row and of a
// share of the rows.
// The others: the projections' weights split into bf16 hi + lo, four a thread.
__global__ void __launch_bounds__(256) prep_kernel(FastBackArgs a) {
  const int tid = threadIdx.x, lane = tid & 63;
  __shared__ float s_top[4];
  if (blockIdx.x > kBackTops) {
    const int64_t n = (int64_t)kHD * a.c_s, x = ((int64_t)(blockIdx.x - 1 - kBackTops) * 256 + tid) * 4;
    if (x >= 4 * n) return;
    const int mat = (x >= n) + (x >= 2 * n) + (x >= 3 * n);
    const float* w = mat == 0 ? a.w[0] : mat == 1 ? a.w[1] : mat == 2 ? a.w[2] : a.w[3];
    u32x2 hi, lo;
    split4(*reinterpret_cast<const f32x4*>(w + x - mat * n), hi, lo);
    *reinterpret_cast<u32x2*>(a.w_split + x) = hi;
    *reinterpret_cast<u32x2*>(a.w_split + 4 * n + x) = lo;
    return;
  }
  if (blockIdx.x > 0) {
    // 16 lanes a row, 24 channels a lane
    const int sub = tid & 15;
    float top = 0.0f;
    for (int64_t r = (int64_t)(blockIdx.x - 1) * 16 + (tid >> 4); r < a.nq_pad; r += 16 * kBackTops) {
      float row_top = 0.0f;
      if (r < a.n_q) {
        if (a.dout_bf16) {
          const u32x4* from = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.dout) + r * kHD) + sub;
#pragma unroll
          for (int x = 0; x < kHD / 128; ++x) {
            const u32x4 v = from[16 * x];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              row_top = fmaxf(row_top, fmaxf(finite_abs(__uint_as_float(v[i] << 16)), finite_abs(__uint_as_float(v[i] & 0xFFFF0000u))));
          }
        } else {
          const f32x4* from = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.dout) + r * kHD) + sub;
#pragma unroll
          for (int x = 0; x < kHD / 64; ++x) {
            const f32x4 v = from[16 * x];
            row_top = fmaxf(row_top, fmaxf(fmaxf(finite_abs(v[0]), finite_abs(v[1])), fmaxf(finite_abs(v[2]), finite_abs(v[3]))));
          }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) row_top = fmaxf(row_top, __shfl_xor(row_top, o));
      }
      if (sub == 0) a.row_exp[r] = scale_exp(row_top);
      top = fmaxf(top, row_top);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) s_top[tid >> 6] = top;
    __syncthreads();
    if (tid == 0) a.tops[3 * kBackTops + blockIdx.x - 1] = __float_as_uint(fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3])));
    return;
  }
  if (tid < 3 * kBackTops) a.tops[tid] = 0u;  // |q|, |k|, |v|: the projection's maxima go here
  if (tid >= 64) return;
  const int n = lane & 15, g = lane >> 4;
  bf16x8 hi[4], lo[4];
  bias_weights(a.w_b, a.gamma, kLog2e, lane, hi, lo);
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    a.w_ops[64 * s + lane] = __builtin_bit_cast(u32x4, hi[s]);
    a.w_ops[64 * (4 + s) + lane] = __builtin_bit_cast(u32x4, lo[s]);
  }
  // W'' = W' - mean, natural units, as the A operand of dz: tile m = 2 x + half, row r =
  // channel 32 x + 8 (r / 4) + 4 half + r % 4, k-slots = heads 4g..4g+3
  float w[4][8], top = 0.0f;
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    const int c = 32 * (m >> 1) + 8 * (n >> 2) + 4 * (m & 1) + (n & 3);
    const float gamma = a.gamma ? a.gamma[c] : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i][m] = a.w_b[(4 * g + i) * kCz + c] * gamma;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float sum = 0.0f;
#pragma unroll
    for (int m = 0; m < 8; ++m) sum += w[i][m];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      w[i][m] -= sum * (1.0f / kCz);
      top = fmaxf(top, finite_abs(w[i][m]));
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const int ew = scale_exp(top);
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    f16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (_Float16)ldexpf(w[i][m], ew);
    reinterpret_cast<u32x2*>(a.w_ops + 512)[64 * m + lane] = __builtin_bit_cast(u32x2, v);
  }
  if (lane == 0) a.exps[4] = ew;
}

// ----------------------------------------------------------------------------- operands
// A wave takes 16 tokens and four heads, a lane one of each: first the tiles of the
// stripe's rows, then those of the keys. [H][tokens][32] operands hold a head's channels
// and 8 zeros; transposed ones, [H][tile][64 lanes][2][4], hold in lane (n, g) and slot
// (u, i) channel 16 u + n of token 4g + i. Both leave through LDS in kilobytes, the
// transposed one by the transposing LDS read, which hands lane i of 16 column i of
// four rows.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
struct PackTile {
  u32x4 w[kTileQ][4];  // [token][32 halfs]
};
__device__ __forceinline__ void pack_row(const float (&x)[kD], int e2, PackTile& to, int tok) {
  f16x8 v[4];
#pragma unroll
  for (int e = 0; e < kDp; ++e) v[e >> 3][e & 7] = (_Float16)(e < kD ? ldexpf(x[e < kD ? e : 0], e2) : 0.0f);
#pragma unroll
  for (int j = 0; j < 4; ++j) to.w[tok][j] = __builtin_bit_cast(u32x4, v[j]);
}
__device__ __forceinline__ void pack_out(const PackTile& t, int h, int64_t tile, int64_t padded, int lane, uint16_t* rows) {
  const int64_t at = ((int64_t)h * (padded >> 4) + tile) * 64 + lane;  // 1 KB per head and tile in both layouts
  reinterpret_cast<u32x4*>(rows)[at] = (&t.w[0][0])[lane];
}
__device__ __forceinline__ void pack_transposed(const PackTile& t, int h, int64_t tile, int64_t padded, int lane,
                                                uint16_t* transposed) {
  const int64_t at = ((int64_t)h * (padded >> 4) + tile) * 64 + lane;
  const int n = lane & 15, g = lane >> 4;
  const uint32_t from = lds_addr(&t) + 64 * (4 * g + (n >> 2)) + 8 * (n & 3);
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)from));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(from + 32)));
  reinterpret_cast<u32x4*>(transposed)[at] = u32x4{a[0], a[1], b[0], b[1]};
}

__global__ void __launch_bounds__(64) pack_kernel(FastBackArgs a) {
  __shared__ PackTile s_x[4], s_y[4], s_t[4];  // q or k; do or v; do at the tensor's power
  const int lane = threadIdx.x, h = 4 * blockIdx.y + (lane >> 4);
  const bool is_row = blockIdx.x < a.nq_pad / 16;
  const int64_t tile = (int64_t)blockIdx.x - (is_row ? 0 : a.nq_pad / 16), tok = tile * 16 + (lane & 15);
  // every load before the first use of one
  float tops[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) tops[x] = __uint_as_float(a.tops[kBackTops * x + lane]);
  f32x4 in[4][kD / 4];  // rows: q, g, acc, dout; keys: k, v
  float l = 0.0f;
  const int er = is_row ? a.row_exp[tok] : 0;  // the power of two of the row's do
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int64_t at = tok * kHD + h * kD;
  const bool there = is_row ? tok < a.n_q : tok < a.n_tok && (!a.mask || a.mask[tok] != 0);
  if (is_row) {
    if (there) l = a.l[(int64_t)h * a.n_q + tok];
#pragma unroll
    for (int e = 0; e < kD / 4; ++e) {
      in[0][e] = there ? *reinterpret_cast<const f32x4*>(a.q + at + 4 * e) : zero;
      in[1][e] = there ? *reinterpret_cast<const f32x4*>(a.g + at + 4 * e) : zero;
      in[2][e] = there ? *reinterpret_cast<const f32x4*>(a.acc + at + 4 * e) : zero;
    }
    if (a.dout_bf16) {
#pragma unroll
      for (int e = 0; e < kD / 8; ++e) {
        const u32x4 r = there ? *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.dout) + at + 8 * e) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          in[3][2 * e + (i >> 2)][i & 3] = __uint_as_float(i & 1 ? r[i >> 1] & 0xFFFF0000u : r[i >> 1] << 16);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kD / 4; ++e)
        in[3][e] = there ? *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.dout) + at + 4 * e) : zero;
    }
  } else {
#pragma unroll
    for (int e = 0; e < kD / 4; ++e) {
      in[0][e] = there ? *reinterpret_cast<const f32x4*>(a.k + at + 4 * e) : zero;
      in[1][e] = there ? *reinterpret_cast<const f32x4*>(a.v + at + 4 * e) : zero;
    }
  }
  int e2[4];  // powers of two of q (with its factor), k, v, and of dout for do (|do| <= |dout|)
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    float top = tops[x];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    e2[x] = scale_exp(x == 0 ? top * (kLog2e * kInvSqrtD) : top);
    if (blockIdx.x == 0 && blockIdx.y == 0 && lane == 0) a.exps[x] = e2[x];
  }
  float x[kD], y[kD];
  if (is_row) {
    const float inv_l = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < kD; e += 4) {
      f32x4 dg;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float gt = in[1][e / 4][i], up = in[3][e / 4][i];
        const float o = l == 0.0f ? 0.0f : in[2][e / 4][i] * inv_l;
        x[e + i] = in[0][e / 4][i] * (kLog2e * kInvSqrtD);
        y[e + i] = gt * up;
        dg[i] = up * o * gt * (1.0f - gt);
      }
      if (there) {
        u32x2 hi, lo;
        split4(dg, hi, lo);
        *reinterpret_cast<u32x2*>(a.dg + at + e) = hi;
        *reinterpret_cast<u32x2*>(a.dg + a.n_q * kHD + at + e) = lo;
      }
    }
    if (h == 0) a.row_scale[tok] = ldexpf(1.0f, e2[3] - er);
    pack_row(y, e2[3], s_t[lane >> 4], lane & 15);
  } else {
#pragma unroll
    for (int e = 0; e < kD; ++e) x[e] = in[0][e / 4][e % 4], y[e] = in[1][e / 4][e % 4];
    const uint32_t bits = (uint32_t)(__ballot(there) & 0xFFFFull);
    if (blockIdx.y == 0 && lane == 0) a.tile_valid[tile] = bits;
  }
  pack_row(x, e2[is_row ? 0 : 1], s_x[lane >> 4], lane & 15);
  pack_row(y, is_row ? er : e2[2], s_y[lane >> 4], lane & 15);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int hh = 4 * blockIdx.y + j;
    if (is_row) {
      pack_out(s_x[j], hh, tile, a.nq_pad, lane, a.qf);
      pack_transposed(s_x[j], hh, tile, a.nq_pad, lane, a.qt);
      pack_out(s_y[j], hh, tile, a.nq_pad, lane, a.of);
      pack_transposed(s_t[j], hh, tile, a.nq_pad, lane, a.ot);
    } else {
      pack_out(s_x[j], hh, tile, a.n_pad, lane, a.kf);
      pack_transposed(s_x[j], hh, tile, a.n_pad, lane, a.kt);
      pack_out(s_y[j], hh, tile, a.n_pad, lane, a.vf);
    }
  }
}

// One key's z for 16 rows as an operand; a key that does not attend reads nothing, and is 0.
__device__ __forceinline__ void load_key(__amdgpu_buffer_rsrc_t zres, int zoff, int64_t t, int k, uint32_t bits, u32x4 (&z)[4]) {
  const int at = (bits >> k) & 1u ? zoff + (int)(t * 16 + k) * (kCz * 2) : kOutOfRange;
#pragma unroll
  for (int x = 0; x < 4; ++x) z[x] = __builtin_amdgcn_raw_buffer_load_b128(zres, at + 64 * x, 0, 0);
}

// ----------------------------------------------------------------------------- row statistics
// M, L = sum 2^(S - M) and sum 2^(S - M) dP of every row and head over a part's keys, S in base 2.
// The forward's saved m, l and acc will not do for them: it forms S from bf16 q and k and sums
// bf16 v, so that P = exp(S - m) / l with the S of fp16 operands has rows that do not sum to 1,
// and D = do . acc / l is not sum P dP, by 2^-9 of the logits' size: gradients were off by 1.4e-2 at
// logits of 22 and 2.9e-2 at 44, with these sums by 2.0e-3 and 2.5e-3. That takes z once more:
// 2400 rows of 4800 tokens 535 us in a call of 2162, 1024 tokens 59 in 273, 333 tokens 12.5 in
// 81. Of the state there remain o for dg (pack_kernel) and the rows whose l is 0.
// Bound by memory: 2.98 GB at 5.6 TB/s for those 2400 rows, 60% of the waves' time waiting
// for it.
// A workgroup's four waves split a tile's keys for the bias, which goes through LDS in two
// buffers, and the heads for the rest, as in pairs_kernel; a lane keeps a running maximum of its
// own (row n, keys 4g..4g+3), and the four lanes of a row meet at the end.
typedef const __attribute__((address_space(4))) uint32_t* const_u32_ptr;
constexpr float kLowest = -3e38f;  // below every logit, and finite: kLowest - kLowest is 0

__global__ void __launch_bounds__(256, 2) stats_kernel(FastBackArgs a) {
  __shared__ f32x4 s_bias[2][kH][kTileQ][4];  // [buffer][head][row][4 keys, chunk ^ row / 4]
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t q0 = (int64_t)blockIdx.x * kTileQ;
  int64_t t_count, t_begin;
  chunk_of_32((uint32_t)(a.n_pad / 16), a.stat_parts, blockIdx.y, &t_count, &t_begin);
  const int64_t t_end = t_begin + t_count;
  constexpr int kHw = kH / 4;
  // (a scalar load: a vector load's wait would be for all of z that came before it)
  const const_u32_ptr valid_bits = (const_u32_ptr)(uintptr_t)a.tile_valid;
  uint32_t bits = t_begin < t_end ? valid_bits[t_begin] : 0u;
  const float s_scale = ldexpf(1.0f, -a.exps[0] - a.exps[1]);
  const int64_t rows_here = min((int64_t)kTileQ, a.n_q - q0);
  const int row_bytes = (int)(a.n_tok * (kCz * 2));
  const __amdgpu_buffer_rsrc_t zres = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t*>(a.z) + q0 * a.n_tok * kCz, 0, (int)(rows_here * row_bytes), kRawBufferFlags);
  const int zoff = n * row_bytes + 16 * g, n_tiles = (int)(a.n_pad / 16);
  u32x4 z[4][4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) load_key(zres, zoff, t_begin, 4 * wave + kk, bits, z[kk]);
  const __amdgpu_buffer_rsrc_t kres = __builtin_amdgcn_make_buffer_rsrc(a.kf, 0, (int)(kH * a.n_pad * kDp * 2), kRawBufferFlags);
  const __amdgpu_buffer_rsrc_t vres = __builtin_amdgcn_make_buffer_rsrc(a.vf, 0, (int)(kH * a.n_pad * kDp * 2), kRawBufferFlags);
  bf16x8 whi[4], wlo[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    whi[x] = as_bf16x8(a.w_ops[64 * x + lane]);
    wlo[x] = as_bf16x8(a.w_ops[64 * (4 + x) + lane]);
  }
  f16x8 q[kHw], o[kHw];
  float top[kHw], sum[kHw], dot[kHw];
#pragma unroll
  for (int j = 0; j < kHw; ++j) {
    const int64_t at = ((int64_t)(kHw * wave + j) * a.nq_pad + q0 + n) * 4 + g;
    q[j] = as_f16x8(reinterpret_cast<const u32x4*>(a.qf)[at]);
    o[j] = as_f16x8(reinterpret_cast<const u32x4*>(a.of)[at]);
    top[j] = kLowest;
    sum[j] = dot[j] = 0.0f;
  }
  const f32x4 wsum = bias_weight_sums(whi, wlo), zero = {0.f, 0.f, 0.f, 0.f};
  const bool row_there = n < rows_here;
  int buf = 0;
  for (int64_t t = t_begin; t < t_end; ++t, buf ^= 1) {
    const uint32_t bits_next = t + 1 < t_end ? valid_bits[t + 1] : 0u;
    f16x8 k[kHw], v[kHw];  // in flight during the bias, and ahead of the next z, which their waits leave in flight
#pragma unroll
    for (int j = 0; j < kHw; ++j) {
      const int so = ((kHw * wave + j) * n_tiles + (int)t) * 1024;
      k[j] = as_f16x8(__builtin_amdgcn_raw_buffer_load_b128(kres, 64 * n + 16 * g, so, 0));
      v[j] = as_f16x8(__builtin_amdgcn_raw_buffer_load_b128(vres, 64 * n + 16 * g, so, 0));
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x4 b[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      f32x4 acc;
      float rstd, mu;
      pair_bias(z[kk], whi, wlo, wsum, a.eps, n, acc, rstd, mu);
      load_key(zres, zoff, t + 1, 4 * wave + kk, bits_next, z[kk]);
      const bool valid = row_there && ((bits >> (4 * wave + kk)) & 1u);
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i][kk] = valid ? acc[i] * rstd : -INFINITY;
    }
    bits = bits_next;
#pragma unroll
    for (int i = 0; i < 4; ++i) s_bias[buf][4 * g + i][n][wave ^ (n >> 2)] = b[i];
    barrier_lds();  // and every wave is through with the other buffer's tile before last
#pragma unroll
    for (int j = 0; j < kHw; ++j) {
      const f32x4 bias = s_bias[buf][kHw * wave + j][n][g ^ (n >> 2)];
      const f32x4 x = mfma32h(k[j], q[j], zero), dp = mfma32h(v[j], o[j], zero);
      f32x4 l;
#pragma unroll
      for (int i = 0; i < 4; ++i) l[i] = fmaf(x[i], s_scale, bias[i]);
      const float m = fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), top[j]);
      const float c = __builtin_amdgcn_exp2f(top[j] - m);
      sum[j] *= c;
      dot[j] *= c;
      top[j] = m;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(l[i] - m);
        sum[j] += e;
        dot[j] = fmaf(e, dp[i], dot[j]);
      }
    }
  }
  const int64_t plane = kH * a.nq_pad;
#pragma unroll
  for (int j = 0; j < kHw; ++j) {
    const int h = kHw * wave + j;
    const float m = max4(top[j]), c = __builtin_amdgcn_exp2f(top[j] - m);
    const float l = sum4(sum[j] * c), d = sum4(dot[j] * c);
    // no weights where the state has none
    const bool keys = row_there && a.l[(int64_t)h * a.n_q + q0 + min(n, (int)rows_here - 1)] != 0.0f;
    float* to = a.stats + 3 * blockIdx.y * plane + (int64_t)h * a.nq_pad + q0 + n;
    if (g == 0) {
      to[0] = keys ? m : kLowest;
      to[plane] = keys ? l : 0.0f;
      to[2 * plane] = keys ? d : 0.0f;
    }
  }
}

// ----------------------------------------------------------------------------- pairs
// A workgroup of four waves takes 16 query rows and a range of 16-key tiles. Per tile:
//   1. the waves split the keys: LayerNorm statistics and bias of all heads
//      (pair_bias), z staying in the registers; the bias goes through LDS
//      [head][row][key];
//   2. the waves split the heads: S = K Q^T + bias, P = exp2(S - M) / L, dP = V dO^T,
//      dS = P (dP - D) with M, L and D = sum P dP of all parts of stats_kernel, dq += K^T dS; P, transposed on the matrix cores (the
//      accumulator's registers as the A operand of a product with the identity:
//      exact), goes to memory as an operand of the keys kernel, and dS to LDS
//      [key][row][head];
//   3. the waves split the keys again: dzh = W''^T dS, dz = rstd (dzh - zh t) with
//      t = sum_h dS_h b_h / c_z (the mean of dzh zh; W'' is centred, so dzh has no mean),
//      and T += dS^T zh over the rows. dz leaves through LDS, four whole rows of 256
//      bytes to a store. A key's registers are refilled with the next tile's z as soon
//      as its dz is formed.
// The rows' q and do stay in LDS: read again from L2 for each tile, calls took 2 us more for
// 1024 tokens and 27 for 2400 rows of 4800.
// 2400 rows of 4800 tokens: 1417 us for 3.14 GB read and 3.37 written (z and dz 2.95 each, P
// 0.37), 4.6 TB/s, where LayerNorm's kernels read and write at 5.4. Of the waves' time a vector
// instruction is active a fifth and waits are a third; registers and LDS allow two workgroups a
// CU, with three barriers a tile. 1024 tokens, where 512 workgroups have eight tiles each: 143
// us, 4.1 TB/s.
struct PairLds {
  union {
    f32x4 bias[kH][kTileQ][4];         // 16 KB: [head][row][4 keys, chunk ^ row / 4]
    u32x4 out[4][kTileQ][16];          // a key's dz per wave, 16-byte chunk ^ row
  };
  u32x4 q[kH][kTileQ][4], o[kH][kTileQ][4];  // 32 KB: the rows' q and do, 16-byte chunk ^ row / 4
  u32x2 ds[kTileK][kTileQ][4];         // 8 KB: [key][row][4 heads]
  float t[4][kTileK][kTileQ];          // 4 KB: each wave's heads' share of sum dS b
  u32x4 w[8][64];                      // 8 KB: bias weights, hi then lo
  u32x2 wt[8][64];                     // 4 KB: W'' for dz
  float stat[kH][kTileQ][3];           // 3 KB: M, 2^kPShift / L and D of the rows
  float row_scale[kTileQ];             // from a row's power of two to the tensor's
  int row_exp[kTileQ];                 // the power of two of a row's dS
};

__global__ void __launch_bounds__(256, 2) pairs_kernel(FastBackArgs a) {
  __shared__ PairLds s;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.y;
  const int64_t r0 = (int64_t)blockIdx.x * kTileQ, q0 = a.row0 + r0;  // within the chunk, within the stripe
  int64_t t_count, t_begin;
  chunk_of_32((uint32_t)(a.n_pad / 16), a.n_parts, part, &t_count, &t_begin);
  const int64_t t_end = t_begin + t_count;
  constexpr int kHw = kH / 4;

  uint32_t bits = t_begin < t_end ? a.tile_valid[t_begin] : 0u;
  const int eq = a.exps[0], ek = a.exps[1], ev = a.exps[2], ed = a.exps[3], ew = a.exps[4];
  const float s_scale = ldexpf(1.0f, -eq - ek);
  const float t_scale = ldexpf(kLn2 / kCz, ew);   // sum dS b (base 2) -> t, in dzh's units
  f16x4 id;
#pragma unroll
  for (int i = 0; i < 4; ++i) id[i] = (_Float16)(4 * g + i == n ? 1.0f : 0.0f);

  const int64_t rows_here = min((int64_t)kTileQ, a.n_q - q0);
  const int row_bytes = (int)(a.n_tok * (kCz * 2));
  const __amdgpu_buffer_rsrc_t zres = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t*>(a.z) + q0 * a.n_tok * kCz, 0, (int)(rows_here * row_bytes), kRawBufferFlags);
  const __amdgpu_buffer_rsrc_t dzres = __builtin_amdgcn_make_buffer_rsrc(
      a.dz ? a.dz + q0 * a.n_tok * kCz : nullptr, 0, a.dz ? (int)(rows_here * row_bytes) : 0, kRawBufferFlags);
  const int zoff = n * row_bytes + 16 * g;
  u32x4 z[4][4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) load_key(zres, zoff, t_begin, 4 * wave + kk, bits, z[kk]);
  for (int x = tid; x < 512; x += 256) {
    (&s.w[0][0])[x] = a.w_ops[x];
    (&s.wt[0][0])[x] = reinterpret_cast<const u32x2*>(a.w_ops + 512)[x];
  }
  const __amdgpu_buffer_rsrc_t kres = __builtin_amdgcn_make_buffer_rsrc(a.kf, 0, (int)(kH * a.n_pad * kDp * 2), kRawBufferFlags);
  const __amdgpu_buffer_rsrc_t vres = __builtin_amdgcn_make_buffer_rsrc(a.vf, 0, (int)(kH * a.n_pad * kDp * 2), kRawBufferFlags);
  const __amdgpu_buffer_rsrc_t ktres = __builtin_amdgcn_make_buffer_rsrc(a.kt, 0, (int)(kH * a.n_pad * kDp * 2), kRawBufferFlags);
  const int n_tiles = (int)(a.n_pad / 16);

  {
    const int64_t at = (int64_t)(tid >> 4) * a.nq_pad + q0 + n;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s.q[tid >> 4][n][x ^ (n >> 2)] = reinterpret_cast<const u32x4*>(a.qf)[at * 4 + x];
      s.o[tid >> 4][n][x ^ (n >> 2)] = reinterpret_cast<const u32x4*>(a.of)[at * 4 + x];
    }
    // M, L and D from the parts, in order
    float top = kLowest, sum = 0.0f, dot = 0.0f;
    const int64_t plane = kH * a.nq_pad;
#pragma unroll 4
    for (int p = 0; p < a.stat_parts; ++p) {
      const float* from = a.stats + 3 * p * plane + at;
      const float m = from[0], l = from[plane], d = from[2 * plane];
      const float both = fmaxf(top, m), c0 = __builtin_amdgcn_exp2f(top - both), c1 = __builtin_amdgcn_exp2f(m - both);
      sum = fmaf(sum, c0, l * c1);
      dot = fmaf(dot, c0, d * c1);
      top = both;
    }
    const bool keys = sum != 0.0f;  // (NaN too)
    const float inv = keys ? 1.0f / sum : 0.0f;
    s.stat[tid >> 4][n][0] = keys ? top : INFINITY;
    s.stat[tid >> 4][n][1] = inv * (float)(1 << kPShift);
    s.stat[tid >> 4][n][2] = dot * inv;
    if (part == 0) a.dot[at] = dot * inv;  // for keys_kernel
    if (tid < kTileQ) {
      s.row_scale[n] = a.row_scale[q0 + n];
      s.row_exp[n] = a.row_exp[q0 + n] + ev - kDsShift;
    }
  }
  f32x4 dq[kHw][2], T[8];
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kHw; ++j) dq[j][0] = dq[j][1] = zero;
#pragma unroll
  for (int m = 0; m < 8; ++m) T[m] = zero;
  const bool row_there = n < rows_here;
  __syncthreads();
  f32x4 wsum;
  {
    bf16x8 whi[4], wlo[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      whi[x] = as_bf16x8(s.w[x][lane]);
      wlo[x] = as_bf16x8(s.w[4 + x][lane]);
    }
    wsum = bias_weight_sums(whi, wlo);
  }

  for (int64_t t = t_begin; t < t_end; ++t) {
    const uint32_t bits_next = t + 1 < t_end ? a.tile_valid[t + 1] : 0u;
    float mu[4], rstd[4];
    {
      f32x4 b[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        // the weights again for each key: held over all four they would not fit the registers
        asm volatile("" ::: "memory");
        bf16x8 whi[4], wlo[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          whi[x] = as_bf16x8(s.w[x][lane]);
          wlo[x] = as_bf16x8(s.w[4 + x][lane]);
        }
        f32x4 acc;
        pair_bias(z[kk], whi, wlo, wsum, a.eps, n, acc, rstd[kk], mu[kk]);
        const bool valid = (bits >> (4 * wave + kk)) & 1u;
        if (!valid || !row_there) rstd[kk] = mu[kk] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i][kk] = valid ? acc[i] * rstd[kk] : -INFINITY;
      }
      barrier_lds();  // every wave is through with the last tile's dz, in the same room
#pragma unroll
      for (int i = 0; i < 4; ++i) s.bias[4 * g + i][n][wave ^ (n >> 2)] = b[i];
    }
    barrier_lds();

    f16x4 dsh[kHw];
    f32x4 tp = zero;
#pragma unroll
    for (int j = 0; j < kHw; ++j) {
      const int h = kHw * wave + j, so = (h * n_tiles + (int)t) * 1024;
      const f16x8 k = as_f16x8(__builtin_amdgcn_raw_buffer_load_b128(kres, 64 * n + 16 * g, so, 0));
      const f16x8 v = as_f16x8(__builtin_amdgcn_raw_buffer_load_b128(vres, 64 * n + 16 * g, so, 0));
      const f16x8 q = as_f16x8(s.q[h][n][g ^ (n >> 2)]), o = as_f16x8(s.o[h][n][g ^ (n >> 2)]);
      const u32x4 kt = __builtin_amdgcn_raw_buffer_load_b128(ktres, 16 * lane, so, 0);
      const f32x4 bias = s.bias[h][n][g ^ (n >> 2)];
      const float top = s.stat[h][n][0], inv_l = s.stat[h][n][1], dot = s.stat[h][n][2];
      const f32x4 x = mfma32h(k, q, zero), dp = mfma32h(v, o, zero);
      f32x4 p, ds;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // P times 2^kPShift, dS times 2^-kDsShift
        p[i] = __builtin_amdgcn_exp2f(fmaf(x[i], s_scale, bias[i]) - top) * inv_l;
        ds[i] = p[i] * (dp[i] - dot) * (1.0f / (1 << (kPShift + kDsShift)));
        tp[i] = fmaf(ds[i], p[i] == 0.0f ? 0.0f : bias[i], tp[i]);
      }
      const f16x4 p16 = to_f16(p), ds16 = to_f16(ds);
      dsh[j] = ds16;
      const u32x2 kt0 = {kt[0], kt[1]}, kt1 = {kt[2], kt[3]};
      dq[j][0] = mfma16h(__builtin_bit_cast(f16x4, kt0), ds16, dq[j][0]);
      dq[j][1] = mfma16h(__builtin_bit_cast(f16x4, kt1), ds16, dq[j][1]);
      const u32x2 pt = __builtin_bit_cast(u32x2, to_f16(mfma16h(p16, id, zero)));
      a.p[(((int64_t)h * (a.chunk_pad >> 4) + (r0 >> 4)) * n_tiles + t) * 64 + lane] = pt;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f16x4 v;
#pragma unroll
      for (int j = 0; j < kHw; ++j) v[j] = dsh[j][i];
      s.ds[4 * g + i][n][wave] = __builtin_bit_cast(u32x2, v);
      s.t[wave][4 * g + i][n] = tp[i];
    }
    barrier_lds();

#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int k = 4 * wave + kk;
      const bool valid = (bits >> k) & 1u;
      const f16x4 d8 = __builtin_bit_cast(f16x4, s.ds[k][n][g]);
      const float tt = ((s.t[0][k][n] + s.t[1][k][n]) + (s.t[2][k][n] + s.t[3][k][n])) * t_scale;
      const f16x4 dst = to_f16(mfma16h(d8, id, zero) * *reinterpret_cast<const f32x4*>(&s.row_scale[4 * g]));
      const float shift = -mu[kk] * rstd[kk], out_scale = ldexpf(rstd[kk], -s.row_exp[n] - ew);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        bf16x8 r;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          f32x4 zh;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = z[kk][x][2 * half + (i >> 1)];
            zh[i] = fmaf(__uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16), rstd[kk], shift);
          }
          const f32x4 acc = mfma16h(__builtin_bit_cast(f16x4, s.wt[2 * x + half][lane]), d8, zero);
          const f16x4 zt = to_f16(mfma16h(to_f16(zh), id, zero));
          T[2 * x + half] = mfma16h(dst, zt, T[2 * x + half]);
#pragma unroll
          for (int i = 0; i < 4; ++i) r[4 * half + i] = (__bf16)(out_scale * fmaf(-zh[i], tt, acc[i]));
        }
        s.out[wave][n][(4 * x + g) ^ n] = __builtin_bit_cast(u32x4, r);
      }
      load_key(zres, zoff, t + 1, k, bits_next, z[kk]);
      if (a.dz) {
        // the wave's own LDS: its writes complete before its reads, in order
        const bool there = t * 16 + k < a.n_tok;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int row = 4 * x + g;
          u32x4 v = s.out[wave][row][n ^ row];
          if (!valid) v = u32x4{0u, 0u, 0u, 0u};
          __builtin_amdgcn_raw_buffer_store_b128(v, dzres, there ? row * row_bytes + (int)(t * 16 + k) * (kCz * 2) + 16 * n : kOutOfRange,
                                                 0, 2);
        }
      }
    }
    bits = bits_next;
  }

  // dq of the part: accumulator rows = channels 4g..4g+3 (+ 16), column = row n
  if (row_there) {
#pragma unroll
    for (int j = 0; j < kHw; ++j) {
      float* to = a.dq_parts + ((int64_t)part * a.n_q + q0 + n) * kHD + (kHw * wave + j) * kD;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (u == 1 && g >= 2) break;  // channels 24 .. 31
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ldexpf(dq[j][u][i] * kInvSqrtD, -s.row_exp[n] - ek);
        *reinterpret_cast<f32x4*>(to + 16 * u + 4 * g) = v;
      }
    }
  }
  // T: the four waves' keys in order. Tile m = 2 x + half, accumulator rows = heads
  // 4g..4g+3, column n = channel 32 x + 8 (n / 4) + 4 half + n % 4
  __syncthreads();
  float* st = reinterpret_cast<float*>(&s.bias[0][0][0]);
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        const int c = 32 * (m >> 1) + 8 * (n >> 2) + 4 * (m & 1) + (n & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* at = st + (4 * g + i) * kCz + c;
          *at = w == 0 ? T[m][i] : *at + T[m][i];
        }
      }
    }
    __syncthreads();
  }
  float* to = a.t_parts + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kH * kCz;
  for (int x = tid; x < kH * kCz; x += 256) {
    const float v = ldexpf(st[x], kDsShift - ev - ed);
    to[x] = a.first ? v : to[x] + v;
  }
}

// ----------------------------------------------------------------------------- keys
// dk and dv of 64 keys of one head over a share of the chunk's row tiles: the four waves
// take every fourth of them, and their sums meet in LDS. dS = P (dP - D) is formed again
// from P and one more product, dP = dO V^T: stored beside P it took as many bytes again,
// written and read (112 us more in a call for 2400 rows of 4800 tokens), and P's 32 bytes a
// pair are what bounds this kernel: 102 us there, 3.6 TB/s.
__global__ void __launch_bounds__(256, 3) keys_kernel(FastBackArgs a) {
  __shared__ f32x4 s_sum[16][64];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y, split = blockIdx.z, n_tiles = (int)(a.n_pad / 16);
  const int t0 = blockIdx.x * 4;
  int64_t count, first;
  chunk_of_32((uint32_t)((a.rows + 15) / 16), a.kv_splits, split, &count, &first);
  f32x4 acc[4][2][2];  // [key tile][dk, dv][channels 0..15, 16..31]
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < 16; ++x) acc[x >> 2][(x >> 1) & 1][x & 1] = zero;
  f16x8 v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    v[k] = as_f16x8(reinterpret_cast<const u32x4*>(a.vf)[((int64_t)h * n_tiles + min(t0 + k, n_tiles - 1)) * 64 + 4 * n + g]);
  // a row tile's operands, loaded one step ahead
  u32x2 x[4];
  u32x4 qt, ot, of;
  f32x4 dt, rs;
  auto load = [&](int64_t r) {
    const int64_t row_tile = (int64_t)h * (a.nq_pad >> 4) + (a.row0 >> 4) + r;
    const u32x2* pp = a.p + (((int64_t)h * (a.chunk_pad >> 4) + r) * n_tiles + t0) * 64 + lane;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = t0 + k < n_tiles ? __builtin_nontemporal_load(pp + 64 * k) : u32x2{0u, 0u};
    qt = reinterpret_cast<const u32x4*>(a.qt)[row_tile * 64 + lane];
    ot = reinterpret_cast<const u32x4*>(a.ot)[row_tile * 64 + lane];
    of = reinterpret_cast<const u32x4*>(a.of)[row_tile * 64 + 4 * n + g];
    dt = *reinterpret_cast<const f32x4*>(a.dot + row_tile * 16 + 4 * g);
    rs = *reinterpret_cast<const f32x4*>(a.row_scale + a.row0 + r * 16 + 4 * g);
  };
  if (wave < count) load(first + wave);
  for (int64_t r = first + wave; r < first + count; r += 4) {
    const f16x4 pk[4] = {__builtin_bit_cast(f16x4, x[0]), __builtin_bit_cast(f16x4, x[1]), __builtin_bit_cast(f16x4, x[2]),
                         __builtin_bit_cast(f16x4, x[3])};
    const u32x4 q = qt, og = ot;
    const f16x8 o = as_f16x8(of);
    const f32x4 dot = dt, scale = rs * (1.0f / (1 << (kDsShift + kPShift)));  // dS at the tensor's power of two
    if (r + 4 < first + count) load(r + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // accumulator rows = query rows 4g..4g+3, column = key n: as P lies
      const f32x4 dp = mfma32h(o, v[k], zero);
      const f16x4 p = pk[k];
      f32x4 d;
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = (float)p[i] * ((dp[i] - dot[i]) * scale[i]);
      const f16x4 ds = to_f16(d);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x2 qu = {q[2 * u], q[2 * u + 1]}, ou = {og[2 * u], og[2 * u + 1]};
        acc[k][0][u] = mfma16h(ds, __builtin_bit_cast(f16x4, qu), acc[k][0][u]);
        acc[k][1][u] = mfma16h(p, __builtin_bit_cast(f16x4, ou), acc[k][1][u]);
      }
    }
  }
  for (int w = 3; w >= 1; --w) {
    if (wave == w) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const f32x4 v = acc[x >> 2][(x >> 1) & 1][x & 1];
        s_sum[x][lane] = w == 3 ? v : s_sum[x][lane] + v;
      }
    }
    __syncthreads();
  }
  if (wave > 0) return;
  const int eq = a.exps[0], ev = a.exps[2], ed = a.exps[3];
  const int64_t v_at = a.n_tok * kHD;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t key = 16 * (int64_t)(t0 + k) + 4 * g + i;
      if (key >= a.n_tok) continue;
      float* to = a.kv_parts + ((int64_t)split * 2 * a.n_tok + key) * kHD + h * kD + n;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (16 * u + n >= kD) continue;
        const float dk = ldexpf((acc[k][0][u][i] + s_sum[4 * k + u][lane][i]) * kLn2, kDsShift - ev - ed - eq);
        const float dv = ldexpf(acc[k][1][u][i] + s_sum[4 * k + 2 + u][lane][i], -kPShift - ed);
        to[16 * u] = a.first ? dk : to[16 * u] + dk;
        to[v_at + 16 * u] = a.first ? dv : to[v_at + 16 * u] + dv;
      }
    }
}

}  // namespace

hipError_t launch_fast_back_prep(const FastBackArgs& a, hipStream_t st) {
  const unsigned split_blocks = (unsigned)((4 * (int64_t)kHD * a.c_s / 4 + 255) / 256);
  hipLaunchKernelGGL(prep_kernel, dim3(1 + kBackTops + split_blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fast_back_pack(const FastBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(pack_kernel, dim3((unsigned)((a.nq_pad + a.n_pad) / 16), kH / 4), dim3(64), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fast_back_stats(const FastBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(stats_kernel, dim3((unsigned)(a.nq_pad / 16), (unsigned)a.stat_parts), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fast_back_pairs(const FastBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(pairs_kernel, dim3((unsigned)((a.rows + 15) / 16), (unsigned)a.n_parts), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fast_back_keys(const FastBackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(keys_kernel, dim3((unsigned)((a.n_pad / 16 + 3) / 4), kH, (unsigned)a.kv_splits), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
