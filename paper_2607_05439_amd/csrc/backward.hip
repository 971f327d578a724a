// Backward pass of the pair-biased gated attention: the steps that every shape
// shares, and the pair kernels of the general fp32 path (gfx950).
//
// With P = exp(l - m) / L recomputed from the saved state (the fused shape sums its own
// M, L and D: backward_fast.hip), o = acc / L, and dout the gradient of the gated output:
//   do = g dout, D = do . o, dP = do . v, dS = P (dP - D),
//   dq_i = sum_j dS k_j / sqrt(d), dk_j = sum_i dS q_i / sqrt(d), dv_j = sum_i P do_i,
//   dg = dout o g (1 - g)                      (before the sigmoid)
// and through the bias, with zh the normalised pair vector and W' = W_b diag(gamma):
//   dzh_c = sum_h dS_h W'_hc, dz = rstd (dzh - mean dzh - zh mean(dzh zh)),
//   T_hc = sum_ij dS_h zh_c, dW_b = T diag(gamma), dgamma_c = sum_h W_b,hc T_hc.
// The rows of dS sum to 0, so LayerNorm's beta and the bias of the projection,
// constants per head, have no gradient and no part in the others'.
// Token side: ds = dq W_q + dg W_g + dk W_k + dv W_v, dW_x = dx^T s.
//
// P and dS meet sums that run across each other: dq over a row's keys, dk and dv
// over a key's rows. The pair kernel writes P and dS (8 bytes a pair and head in
// fp32), and a second kernel sums dq in workgroups that hold rows, dk and dv in
// workgroups that hold keys. Chunks of rows bound the room for P and dS.
//
// 601 tokens, 128 pair channels, 4 heads of 32, fp32: 176 us, of them the pair kernel 130
// (z read and dz written, 0.41 GB with P and dS, at 3.3 TB/s: a vector instruction is active a
// fifth of its waves' time, and two workgroups a CU, as the registers allow, do not cover
// the loads' latency and the tiles' two barriers), the sums over pairs 18, the token products 20.
// 128 tokens of 32 channels: 33 us, seven launches that depend on each other.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

__device__ __forceinline__ float load_one(const void* p, int bf16, int64_t at) {
  return bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void store_one(void* p, int bf16, int64_t at, float v) {
  if (bf16)
    static_cast<__bf16*>(p)[at] = (__bf16)v;
  else
    static_cast<float*>(p)[at] = v;
}
// Four consecutive elements from i0 of a row of len, zeros past its end; `vec`:
// len is a multiple of 4 and the row 16-byte (bf16: 8-byte) aligned.
__device__ __forceinline__ f32x4 load_four(const void* p, int bf16, int vec, int64_t row, int i0, int len) {
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  if (vec) {
    if (i0 < len) {
      if (bf16) {
        const u32x2 t = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + row + i0);
        r = f32x4{__uint_as_float(t[0] << 16), __uint_as_float(t[0] & 0xFFFF0000u), __uint_as_float(t[1] << 16),
                  __uint_as_float(t[1] & 0xFFFF0000u)};
      } else {
        r = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + row + i0);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i0 + i < len) r[i] = load_one(p, bf16, row + i0 + i);
  }
  return r;
}

// v_mfma_f32_16x16x4_f32: A holds row n, B column n (n = lane % 16), both at
// k-slot g = lane / 16; the accumulator holds rows 4g..4g+3 of column n.
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Sum over the four lanes of a quad; each gets the same bits.
__device__ __forceinline__ float quad_sum(float x) {
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0xB1, 0xF, 0xF, true));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x4E, 0xF, 0xF, true));
  return x;
}

// ----------------------------------------------------------------------------- query rows
// Eight lanes per row and head: do, q in padded rows of dp floats per head, the
// statistics {m, 1 / L, D, -}, and dg. A row without keys (L = 0) gets weights of 0. All
// loads before the first store, which the compiler could not tell from them. The
// blocks behind those lay out k and v, with zeros for masked keys, which may hold
// anything, so that a weight of 0 times them is 0: k in padded rows for dq, both as the
// pair kernel's lanes read them, [heads / 4][keys / 16][dp / 4][16 keys][4 heads][4] with
// zeros for the heads and keys that are not there.
__global__ void __launch_bounds__(256) back_rows_kernel(BackRowsArgs a) {
  constexpr int kMost = kGenMaxD / 8;
  if (blockIdx.x >= a.row_blocks) {
    // a piece of four channels a thread
    const int64_t x = (int64_t)(blockIdx.x - a.row_blocks) * 256 + threadIdx.x;
    // (rows of at least 64 bytes in memory: fewer than 2^32)
    const int pieces = a.dp / 4, shift = __builtin_ctz(pieces), piece = (int)x & (pieces - 1), c = 4 * piece;
    const int64_t n_keys = back_keys_padded(a.n_tok);
    const uint32_t hj = (uint32_t)(x >> shift);
    const int h = (int)(hj / (uint32_t)n_keys);
    const int64_t j = hj % (uint32_t)n_keys;
    if (h >= back_heads_padded(a.n_heads)) return;
    const bool here = h < a.n_heads && j < a.n_tok, valid = here && (!a.mask || a.mask[j] != 0);
    const int64_t at = (j * a.n_heads + h) * a.head_dim;
    f32x4 k = {0.f, 0.f, 0.f, 0.f}, v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (valid && c + i < a.head_dim) {
        k[i] = a.k[at + c + i];
        v[i] = a.v[at + c + i];
      }
    const int64_t to = (((h >> 2) * (n_keys >> 4) + (j >> 4)) * pieces + piece) * 64 + 4 * (j & 15) + (h & 3);
    if (here) reinterpret_cast<f32x4*>(a.kr)[((int64_t)h * a.n_tok + j) * pieces + piece] = k;
    reinterpret_cast<f32x4*>(a.kp)[to] = k;
    reinterpret_cast<f32x4*>(a.vp)[to] = v;
    return;
  }
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
  if (t >= a.n_q * a.n_heads) return;  // eight lanes alike
  const int sub = threadIdx.x & 7, d = a.head_dim;
  const int64_t row = (uint32_t)t / (uint32_t)a.n_heads;
  const int h = (int)(t - row * a.n_heads);
  const int64_t at = row * a.n_heads * d + (int64_t)h * d, to = ((int64_t)h * a.n_q + row) * a.dp;
  const float l = a.l[(int64_t)h * a.n_q + row], inv_l = l == 0.0f ? 0.0f : 1.0f / l;
  const float m = l == 0.0f ? 0.0f : a.m[(int64_t)h * a.n_q + row];
  float g[kMost], up[kMost], o[kMost], q[kMost], dot = 0.0f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int e = sub + 8 * i;
    const bool in = e < d;
    g[i] = in ? a.g[at + e] : 0.0f;
    up[i] = in ? load_one(a.dout, a.dout_bf16, at + e) : 0.0f;
    o[i] = in && l != 0.0f ? a.acc[at + e] * inv_l : 0.0f;
    q[i] = in ? a.q[at + e] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < kMost; ++i) dot = fmaf(g[i] * up[i], o[i], dot);
  dot = quad_sum(dot);
  dot += __shfl_xor(dot, 4);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int e = sub + 8 * i;
    if (e >= a.dp) break;
    a.dop[to + e] = g[i] * up[i];
    a.qp[to + e] = q[i];
    if (e < d) a.dg[at + e] = up[i] * o[i] * g[i] * (1.0f - g[i]);
  }
  if (sub == 0) *reinterpret_cast<f32x4*>(a.stat + 4 * ((int64_t)h * a.n_q + row)) = f32x4{m, inv_l, dot, 0.0f};
}

// ----------------------------------------------------------------------------- pairs
// A workgroup takes an equal share of the chunk's tiles, 64 keys of one query row each,
// in row order. Four lanes per key share its channels for the LayerNorm, the bias
// and dz, and its heads for the logits and dS; T is then a sum over the tile's keys
// by output element, written once per workgroup. CT: pieces of 16 channels of z; NH:
// heads per lane. W' loses its mean over the channels first, so that dzh has none, and
// t, the mean of dzh zh, is sum_h dS_h b_h / c_z: no sum over the channels after the products.
// k and v come a kilobyte to a load (k and v in rows per head, 64 lines to a load: 601
// tokens of 128 pair channels 186 us, so 174).
constexpr int kHeadStride = kGenMaxD + 4;

// Four consecutive elements from i0 of a row of len as loaded: whole pieces (len a
// multiple of four, the row aligned) or one by one; past the end, the last ones again.
template <bool BF16>
struct Raw4 {
  uint32_t w[BF16 ? 2 : 4];
  __device__ __forceinline__ void load(const void* p, int64_t row, int i0, int len) {
    const int at = min(i0, len - 4);
    if constexpr (BF16) {
      const u32x2 r = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + row + at);
      w[0] = r[0], w[1] = r[1];
    } else {
      const u32x4 r = *reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + row + at);
      w[0] = r[0], w[1] = r[1], w[2] = r[2], w[3] = r[3];
    }
  }
  __device__ __forceinline__ void load_each(const void* p, int64_t row, int i0, int len) {
    uint32_t e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t x = row + min(i0 + i, len - 1);
      e[i] = BF16 ? (uint32_t)static_cast<const uint16_t*>(p)[x] : static_cast<const uint32_t*>(p)[x];
    }
    if constexpr (BF16) {
      w[0] = e[0] | (e[1] << 16), w[1] = e[2] | (e[3] << 16);
    } else {
      w[0] = e[0], w[1] = e[1], w[2] = e[2], w[3] = e[3];
    }
    __builtin_amdgcn_sched_barrier(0);  // (four addresses at a time)
  }
  __device__ __forceinline__ f32x4 get() const {
    if constexpr (BF16)
      return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                   __uint_as_float(w[1] & 0xFFFF0000u)};
    else
      return f32x4{__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
  }
};

template <int CT, int NH, bool BF16>
__global__ void __launch_bounds__(256, CT <= 8 && CT * NH < 32 ? 2 : 1) back_pairs_kernel(BackPairsArgs a) {
  constexpr int CZ = 16 * CT, HP = 4 * NH;
  constexpr bool kHeld = CT * HP <= 8;  // W' of the lane's channels stays in registers
  __shared__ __attribute__((aligned(16))) float s_w[HP * CZ];
  __shared__ __attribute__((aligned(16))) float s_zh[kBackKeys * (CZ + 4)];
  __shared__ __attribute__((aligned(16))) float s_ds[kBackKeys * (HP + 4)];
  __shared__ f32x4 s_stat[HP];
  __shared__ __attribute__((aligned(16))) float s_q[HP * kHeadStride], s_do[HP * kHeadStride];
  const int tid = threadIdx.x, key = tid >> 2, qd = tid & 3;
  const int H = a.n_heads, d = a.head_dim, hd = H * d, c_z = a.c_z;
  const float inv_c = 1.0f / (float)c_z, scale = 1.0f / sqrtf((float)d);
  const int z_vec = c_z % 4 == 0;
  const bool whole = c_z == CZ;
  const int chunks = a.dp / 8;
  for (int x = tid; x < HP * CZ; x += 256) {
    const int h = x / CZ, c = x % CZ;
    s_w[x] = h < H && c < c_z ? a.w_b[(int64_t)h * c_z + c] * (a.gamma ? a.gamma[c] : 1.0f) : 0.0f;
  }
  for (int x = tid; x < HP * kHeadStride; x += 256) s_q[x] = s_do[x] = 0.0f;
  __syncthreads();
  {
    // W' less its mean over the channels, 16 lanes a head: the bias stays (zh has no mean)
    // and dzh has no mean either
    const int h = tid >> 4;
    float sum = 0.0f;
    if (h < HP)
      for (int c = tid & 15; c < c_z; c += 16) sum += s_w[h * CZ + c];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (h < HP)
      for (int c = tid & 15; c < c_z; c += 16) s_w[h * CZ + c] -= sum * inv_c;
  }
  __syncthreads();
  f32x4 w_held[kHeld ? HP : 1][kHeld ? CT : 1];
  if constexpr (kHeld)
#pragma unroll
    for (int h = 0; h < HP; ++h)
#pragma unroll
      for (int m = 0; m < CT; ++m) w_held[h][m] = *reinterpret_cast<const f32x4*>(&s_w[h * CZ + 16 * m + 4 * qd]);
  auto weights = [&](int h, int m) {
    if constexpr (kHeld)
      return w_held[h][m];
    else
      return *reinterpret_cast<const f32x4*>(&s_w[h * CZ + 16 * m + 4 * qd]);
  };
  const int lane = tid & 63, n = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int kTiles = (CT + 3) / 4;
  f32x4 T[kTiles];
#pragma unroll
  for (int y = 0; y < kTiles; ++y) T[y] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t tiles = (a.n_tok + kBackKeys - 1) / kBackKeys;  // of a row
  int64_t share, begin;
  chunk_of_32((uint32_t)(a.rows * tiles), gridDim.x, blockIdx.x, &share, &begin);
  int64_t r = (uint32_t)begin / (uint32_t)tiles, t_first = begin - r * tiles, left = share;  // row of the stripe's chunk, tile
  // z and the mask of a tile, keys past the last reading that one's
  Raw4<BF16> raw[CT];
  uint8_t attends = 1;
  auto load_z = [&](int64_t rr, int64_t t) {
    const int64_t j = min(t * kBackKeys + key, a.n_tok - 1);
    const int64_t off = ((a.row0 + rr) * a.n_tok + j) * c_z;
    if (a.mask) attends = a.mask[j];
    int c = 4 * qd;
    asm volatile("" : "+v"(c));  // (or the indices of the one-by-one loads would fill the registers)
    if (z_vec) {
#pragma unroll
      for (int m = 0; m < CT; ++m) raw[m].load(a.z, off, 16 * m + c, c_z);
    } else {
#pragma unroll
      for (int m = 0; m < CT; ++m) raw[m].load_each(a.z, off, 16 * m + c, c_z);
    }
  };
  if (left > 0) load_z(r, t_first);
  for (; left > 0; ++r, t_first = 0) {
    const int64_t row = a.row0 + r;  // row of the stripe
    const int64_t t_end = min(tiles, t_first + left);
    left -= t_end - t_first;
    int first = tid;
    asm volatile("" : "+v"(first));  // (as above)
    for (int x = first; x < hd; x += 256) {
      const int h = x / d, e = x - h * d;
      s_q[h * kHeadStride + e] = a.qp[((int64_t)h * a.n_q + row) * a.dp + e] * scale;
      s_do[h * kHeadStride + e] = a.dop[((int64_t)h * a.n_q + row) * a.dp + e];
    }
    if (first < HP) s_stat[first] = *reinterpret_cast<const f32x4*>(a.stat + 4 * ((int64_t)min(first, H - 1) * a.n_q + row));
    __syncthreads();
    for (int64_t t = t_first; t < t_end; ++t) {
      asm volatile("" ::: "memory");  // q, do and W' come from LDS again for each tile, not from registers
      const int64_t j = t * kBackKeys + key;
      const bool there = j < a.n_tok, valid = there && attends != 0;
      // k and v of the lane's heads, eight channels at a time, two such pieces in flight; the
      // first head's during the statistics and the bias
      f32x4 kk[2][2], vv[2][2];
      auto load_kv = [&](int i, int c, int buf) {
        const int64_t at = (((int64_t)i * 4 * tiles + 4 * t + wave) * (a.dp >> 2) + 2 * c) * 64 + lane;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          kk[buf][x] = reinterpret_cast<const f32x4*>(a.k)[at + 64 * x];
          vv[buf][x] = reinterpret_cast<const f32x4*>(a.v)[at + 64 * x];
        }
      };
      load_kv(0, 0, 0);
      load_kv(0, 1, 1);
      f32x4 zh[CT];
      float s = 0.0f, v = 0.0f, t_sum = 0.0f;
      const bool plain = whole && __ballot(valid) == ~0ull;  // nothing of the wave's keys to leave out
      int c4 = 4 * qd;
      asm volatile("" : "+v"(c4));  // (as above)
#pragma unroll
      for (int m = 0; m < CT; ++m) {
        const int c = 16 * m + c4;
        zh[m] = raw[m].get();
        if (!plain)
#pragma unroll
          for (int i = 0; i < 4; ++i) zh[m][i] = valid && (whole || c + i < c_z) ? zh[m][i] : 0.0f;
        s += (zh[m][0] + zh[m][1]) + (zh[m][2] + zh[m][3]);
      }
      const float mu = quad_sum(s) * inv_c;
#pragma unroll
      for (int m = 0; m < CT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          zh[m][i] = zh[m][i] - mu;
          if (!plain) zh[m][i] = whole || 16 * m + c4 + i < c_z ? zh[m][i] : 0.0f;
          v = fmaf(zh[m][i], zh[m][i], v);
        }
      const float rstd = valid ? 1.0f / sqrtf(fmaf(quad_sum(v), inv_c, a.eps)) : 0.0f;
#pragma unroll
      for (int m = 0; m < CT; ++m) {
        zh[m] *= rstd;  // 0 for a key that does not attend, whose mean is 0 too
        *reinterpret_cast<f32x4*>(&s_zh[key * (CZ + 4) + 16 * m + 4 * qd]) = zh[m];
      }
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        // the bias of heads 4i .. 4i + 3, summed over the quad; this lane keeps head 4i + qd
        if (i > 0) asm volatile("" ::: "memory");  // (W' of four heads at a time)
        float b = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int m = 0; m < CT; ++m) {
            const f32x4 w = weights(4 * i + x, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = fmaf(w[e], zh[m][e], p[e]);
          }
          const float sum = quad_sum((p[0] + p[1]) + (p[2] + p[3]));
          b = qd == x ? sum : b;
        }
        const int h = 4 * i + qd;
        f32x4 lg = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
        if (i > 0) {
          load_kv(i, 0, 0);
          load_kv(i, 1, 1);
        }
        auto dots = [&](int c, auto buf) {
          constexpr int kBuf = decltype(buf)::value;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(&s_q[h * kHeadStride + 8 * c + 4 * x]);
            const f32x4 o = *reinterpret_cast<const f32x4*>(&s_do[h * kHeadStride + 8 * c + 4 * x]);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              lg[y] = fmaf(q[y], kk[kBuf][x][y], lg[y]);
              dp[y] = fmaf(o[y], vv[kBuf][x][y], dp[y]);
            }
          }
          if (c + 2 < chunks) load_kv(i, c + 2, kBuf);
        };
#pragma unroll 1
        for (int c = 0; c < chunks; c += 2) {
          dots(c, std::integral_constant<int, 0>());
          dots(c + 1, std::integral_constant<int, 1>());
        }
        float ds = 0.0f, p = 0.0f;
        if (valid && h < H) {
          const f32x4 stat = s_stat[h];
          const float l = (lg[0] + lg[1]) + (lg[2] + lg[3]) + b;
          p = stat[1] == 0.0f ? 0.0f : expf(l - stat[0]) * stat[1];
          ds = p * (((dp[0] + dp[1]) + (dp[2] + dp[3])) - stat[2]);
        }
        t_sum = fmaf(ds, b, t_sum);
        s_ds[key * (HP + 4) + h] = ds;
        if (there && h < H) {
          const int64_t at = ((int64_t)h * a.rows + r) * a.n_tok + j;
          a.p[at] = p;
          a.ds[at] = ds;
        }
      }
      // in flight during dz and T, and behind k and v, which wait for nothing else
      if (t + 1 < t_end)
        load_z(r, t + 1);
      else if (left > 0)
        load_z(r + 1, 0);
      __syncthreads();
      if (a.dz && there) {
        int at = key;
        asm volatile("" : "+v"(at));  // (formed here, not held from the top)
        const int64_t off = (row * a.n_tok + t * kBackKeys + at) * c_z;
        // dz = rstd (dzh - zh t), t = the mean of dzh zh = sum_h dS_h b_h / c_z
        f32x4 acc[CT];
        const float t_mean = quad_sum(t_sum) * inv_c * rstd;
#pragma unroll
        for (int m = 0; m < CT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NH; ++i) {
          if (i > 0) asm volatile("" ::: "memory");  // (W' of four heads at a time)
          const f32x4 ds = *reinterpret_cast<const f32x4*>(&s_ds[key * (HP + 4) + 4 * i]) * rstd;
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int m = 0; m < CT; ++m) {
              const f32x4 w = weights(4 * i + x, m);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[m][e] = fmaf(ds[x], w[e], acc[m][e]);
            }
#pragma unroll
          for (int m = 0; m < CT; ++m) asm volatile("" : "+v"(acc[m]));  // (summed here: W' is not held until the stores)
        }
#pragma unroll
        for (int m = 0; m < CT; ++m) {
          const int c = 16 * m + c4;
          f32x4 g;
#pragma unroll
          for (int e = 0; e < 4; ++e) g[e] = fmaf(-zh[m][e], t_mean, acc[m][e]);  // 0 for a key that does not attend
          if (z_vec) {
            if (c < c_z) {
              if (BF16) {
                bf16x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (__bf16)g[e];
                *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.dz) + off + c) = o;
              } else {
                *reinterpret_cast<f32x4*>(static_cast<float*>(a.dz) + off + c) = g;
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (c + e < c_z) store_one(a.dz, BF16, off + c + e, g[e]);
          }
        }
      }
      // T += dS^T zh: heads by 16 channels, four keys a step; wave w takes tiles w, w + 4, ..
#pragma unroll 4
      for (int x = 0; x < kBackKeys; x += 4) {
        const float ds = n < HP ? s_ds[(x + g) * (HP + 4) + n] : 0.0f;
#pragma unroll
        for (int y = 0; y < kTiles; ++y)
          if (CT >= 4 || wave < CT) T[y] = mfma4(ds, s_zh[(x + g) * (CZ + 4) + 16 * (wave + 4 * y) + n], T[y]);
      }
      __syncthreads();
    }
  }
  // T of this workgroup, added to what earlier chunks left
  float* out = a.t_parts + (int64_t)blockIdx.x * H * c_z;
#pragma unroll
  for (int y = 0; y < kTiles; ++y)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int h = 4 * g + i, c = 16 * (wave + 4 * y) + n;
      if (h < H && c < c_z) out[h * c_z + c] = a.first ? T[y][i] : out[h * c_z + c] + T[y][i];
    }
}

// ----------------------------------------------------------------------------- keys
// The sums over pairs on the fp32 matrix cores, 16 keys or rows of one head a wave.
// Blocks of keys: dk^T, dv^T of 64 keys (a wave each 16) over a share of the chunk's rows,
// 16 rows a step. Blocks of rows: dq of 16 rows over all keys, 16 keys a step, every
// fourth step a wave. A step's loads are all in flight at once; past the last row or
// key they repeat that one, with a P and dS of 0.
template <int DP>
__device__ __forceinline__ void row_sums(const BackKeysArgs& a, int h, int64_t r0, f32x4 (&s_sum)[4][DP / 16][64]) {
  constexpr int U = DP / 16;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t last = a.n_tok - 1;
  const float* ds = a.ds + ((int64_t)h * a.rows + min(r0 + n, a.rows - 1)) * a.n_tok;
  const float* k = a.k + (int64_t)h * a.n_tok * DP + n;
  f32x4 acc[U];
#pragma unroll
  for (int u = 0; u < U; ++u) acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = 16 * wave; j0 <= last; j0 += 64) {
    float x[4], y[4][U];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t j = j0 + 4 * g + i, jj = min(j, last);
      x[i] = ds[jj];
#pragma unroll
      for (int u = 0; u < U; ++u) y[i][u] = k[jj * DP + 16 * u];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = j0 + 4 * g + i <= last ? x[i] : 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) acc[u] = mfma4(v, y[i][u], acc[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) s_sum[wave][u][lane] = acc[u];
  __syncthreads();
  if (wave >= U) return;
  // wave u: channels 16 u + n of rows 4g..4g+3
  const f32x4 v = (s_sum[0][wave][lane] + s_sum[1][wave][lane]) + (s_sum[2][wave][lane] + s_sum[3][wave][lane]);
  const int hd = a.n_heads * a.head_dim, e = 16 * wave + n;
  const float scale = 1.0f / sqrtf((float)a.head_dim);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (r0 + 4 * g + i < a.rows && e < a.head_dim)
      a.dq[(a.row0 + r0 + 4 * g + i) * hd + (int64_t)h * a.head_dim + e] = v[i] * scale;
}

template <int DP>
__global__ void __launch_bounds__(256) back_keys_kernel(BackKeysArgs a) {
  constexpr int U = DP / 16;
  __shared__ f32x4 s_sum[4][U][64];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y;
  if (blockIdx.x >= a.key_blocks) {
    row_sums<DP>(a, h, (int64_t)(blockIdx.x - a.key_blocks) * 16, s_sum);
    return;
  }
  const int64_t j0 = (int64_t)(blockIdx.x / a.n_splits) * 64 + 16 * wave;
  const int split = blockIdx.x % a.n_splits;
  int64_t count, first;
  chunk_of_32((uint32_t)a.rows, a.n_splits, split, &count, &first);
  const int64_t jj = min(j0 + n, a.n_tok - 1), end = first + count;
  const float *q = a.qp + ((int64_t)h * a.n_q + a.row0) * DP + n, *o = a.dop + ((int64_t)h * a.n_q + a.row0) * DP + n;
  f32x4 dk[U], dv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) dk[u] = dv[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t r0 = first; r0 < end; r0 += 16) {
    float p[4], ds[4], x[4][U], y[4][U];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = min(r0 + 4 * i + g, end - 1), at = ((int64_t)h * a.rows + r) * a.n_tok + jj;
      p[i] = a.p[at];
      ds[i] = a.ds[at];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[i][u] = q[r * DP + 16 * u];
        y[i][u] = o[r * DP + 16 * u];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = r0 + 4 * i + g < end;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        dk[u] = mfma4(in ? ds[i] : 0.0f, x[i][u], dk[u]);
        dv[u] = mfma4(in ? p[i] : 0.0f, y[i][u], dv[u]);
      }
    }
  }
  const int hd = a.n_heads * a.head_dim;
  const float scale = 1.0f / sqrtf((float)a.head_dim);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t j = j0 + 4 * g + i;
    if (j >= a.n_tok) continue;
    float* out = a.kv_parts + ((int64_t)split * 2 * a.n_tok + j) * hd + (int64_t)h * a.head_dim + n;
    const int64_t v_at = a.n_tok * hd;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (16 * u + n >= a.head_dim) continue;
      const float x = dk[u][i] * scale, y = dv[u][i];
      out[16 * u] = a.first ? x : out[16 * u] + x;
      out[v_at + 16 * u] = a.first ? y : out[v_at + 16 * u] + y;
    }
  }
}

// ----------------------------------------------------------------------------- sums of parts
// dq, dk and dv: W elements a thread (4 where H d is a multiple of that), parts in
// order. T: 16 columns by 16 groups of parts per workgroup.
template <int W>
__device__ __forceinline__ void sum_parts(const float* parts, int n, int64_t stride, float* out, int64_t x, int split) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    if constexpr (W == 4)
      v += *reinterpret_cast<const f32x4*>(parts + p * stride + x);
    else
      v[0] += parts[p * stride + x];
  }
  if constexpr (W == 4) {
    if (split) {
      u32x2 hi, lo;
      split4(v, hi, lo);
      *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + x) = hi;
      *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + stride + x) = lo;
      return;
    }
    *reinterpret_cast<f32x4*>(out + x) = v;
  } else {
    out[x] = v[0];
  }
}
template <int W>
__global__ void __launch_bounds__(256) back_sum_kernel(BackSumArgs a) {
  __shared__ float s[16][17];
  const int64_t n_dq = a.dq_parts ? a.n_q * a.hd : 0, n_kv = 2 * a.n_tok * a.hd;
  if (blockIdx.x < a.token_blocks) {
    const int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) * W;
    if (x < n_dq)
      sum_parts<W>(a.dq_parts, a.dq_n, n_dq, a.dq, x, a.split);
    else if (x < n_dq + n_kv)
      sum_parts<W>(a.kv_parts, a.kv_n, n_kv, a.dkv, x - n_dq, a.split);
    return;
  }
  const int cols = a.t_cols, col = (int)(blockIdx.x - a.token_blocks) * 16 + (threadIdx.x & 15), grp = threadIdx.x >> 4;
  float v = 0.0f;
  if (col < cols)
#pragma unroll 8
    for (int p = grp; p < a.t_n; p += 16) v += a.t_parts[(int64_t)p * cols + col];
  s[grp][threadIdx.x & 15] = v;
  __syncthreads();
  if (grp > 0 || col >= cols) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) v += s[i][threadIdx.x];
  a.t[col] = v;
}

// ----------------------------------------------------------------------------- token products
// ds = sum over x of dx W_x (64 tokens by 64 channels per workgroup) and dW_x = dx^T s
// (64 outputs by 64 channels), on the fp32 matrix cores: a workgroup's four waves
// take 32 x 32 each, operands 32 deep through LDS, the next 32 in flight.
constexpr int kGemm = 64, kDeep = 32, kGemmStride = kGemm + 16;

__global__ void __launch_bounds__(256) back_gemm_kernel(BackGemmArgs a) {
  __shared__ __attribute__((aligned(16))) float s_a[2][kDeep][kGemmStride], s_b[2][kDeep][kGemmStride];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c_tiles = (a.c_s + kGemm - 1) / kGemm;
  uint32_t b = blockIdx.x;
  const bool is_ds = b < a.ds_blocks;
  if (!is_ds) b -= (uint32_t)a.ds_blocks;
  const int c0 = (int)(b % c_tiles) * kGemm;
  b /= c_tiles;
  const int splits = is_ds ? a.ds_splits : a.w_splits, split = (int)(b % splits);
  b /= splits;
  const int hd_deep = (a.hd + kDeep - 1) / kDeep * kDeep;
  const int64_t m0 = is_ds ? (int64_t)b * kGemm : 0;                            // first token
  const int o_tiles = (a.hd + kGemm - 1) / kGemm;
  const int mat = is_ds ? 0 : (int)(b / o_tiles), o0 = is_ds ? 0 : (int)(b % o_tiles) * kGemm;
  // terms of ds in the order k, v, q, g; the matrices of dW in the order q, k, v, g
  const bool with_rows = m0 < a.q_row0 + a.n_q && m0 + kGemm > a.q_row0;
  const bool stripe = mat == 0 || mat == 3;
  const int64_t w_rows = stripe ? a.n_q : a.n_tok, s_row0 = stripe ? a.q_row0 : 0;
  const float* dx = mat == 0 ? a.dq : mat == 1 ? a.dk : mat == 2 ? a.dv : a.dg;
  const int64_t depth = is_ds ? (int64_t)hd_deep * (with_rows ? 4 : 2) : (w_rows + kDeep - 1) / kDeep * kDeep;
  int64_t steps, first;
  chunk_of_32((uint32_t)(depth / kDeep), splits, split, &steps, &first);
  const int hd_vec = a.hd % 4 == 0, s_vec = a.c_s % 4 == 0;
  const int r16 = tid >> 4, x4 = (tid & 15) * 4;  // 16 deep by 64 wide, four a thread, twice
  f32x4 av[2], bv[2];
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto fetch = [&](int64_t step) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (is_ds) {
        const int k0 = (int)step * kDeep, term = k0 / hd_deep, o = k0 - term * hd_deep + 16 * u;
        const float* x = term == 0 ? a.dk : term == 1 ? a.dv : term == 2 ? a.dq : a.dg;
        const float* w = term == 0 ? a.w_k : term == 1 ? a.w_v : term == 2 ? a.w_q : a.w_g;
        // A: token tid / 4, outputs o + 4 (tid % 4) ..
        const int64_t row = m0 + (tid >> 2) - (term >= 2 ? a.q_row0 : 0), rows = term >= 2 ? a.n_q : a.n_tok;
        av[u] = row >= 0 && row < rows ? load_four(x, 0, hd_vec, row * a.hd, o + 4 * (tid & 3), a.hd) : zero;
        bv[u] = o + r16 < a.hd ? load_four(w, 0, s_vec && a.w_vec, (int64_t)(o + r16) * a.c_s, c0 + x4, a.c_s) : zero;
      } else {
        const int64_t t = step * kDeep + 16 * u + r16;
        const bool in = t < w_rows;
        av[u] = in ? load_four(dx, 0, hd_vec, t * a.hd, o0 + x4, a.hd) : zero;
        // a masked token's s does not enter the gradients of W_k and W_v
        const bool used = in && (stripe || !a.mask || a.mask[t] != 0);
        bv[u] = used ? load_four(a.s, a.s_bf16, s_vec, (s_row0 + t) * a.c_s, c0 + x4, a.c_s) : zero;
      }
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (is_ds) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s_a[buf][16 * u + 4 * (tid & 3) + i][tid >> 2] = av[u][i];
      } else {
        *reinterpret_cast<f32x4*>(&s_a[buf][16 * u + r16][x4]) = av[u];
      }
      *reinterpret_cast<f32x4*>(&s_b[buf][16 * u + r16][x4]) = bv[u];
    }
  };
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int am = 32 * (wave >> 1), bn = 32 * (wave & 1);
  if (steps > 0) {
    fetch(first);
    stage(0);
  }
  for (int64_t i = 0; i < steps; ++i) {
    __syncthreads();
    const int buf = (int)(i & 1);
    if (i + 1 < steps) fetch(first + i + 1);
#pragma unroll
    for (int k = 0; k < kDeep / 4; ++k) {
      float x[2], y[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        x[u] = s_a[buf][4 * k + g][am + 16 * u + n];
        y[u] = s_b[buf][4 * k + g][bn + 16 * u + n];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) acc[u][w] = mfma4(x[u], y[w], acc[u][w]);
    }
    if (i + 1 < steps) stage(buf ^ 1);
  }
  const int64_t m_end = is_ds ? a.n_tok : a.hd;
  float* out = is_ds ? a.ds_parts + (int64_t)split * a.n_tok * a.c_s : a.w_parts + ((int64_t)split * 4 + mat) * a.hd * a.c_s;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t m = (is_ds ? m0 : o0) + am + 16 * u + 4 * g + i;
        const int c = c0 + bn + 16 * w + n;
        if (m < m_end && c < a.c_s) out[m * a.c_s + c] = acc[u][w][i];
      }
}

// The gradients in their own type: sums of the products' splits, then dW_b and dgamma
// from T. W consecutive elements a thread: 4 where every tensor has a multiple of that.
template <int W>
__device__ __forceinline__ void finish_sum(const float* parts, int n, int64_t stride, void* out, int bf16, int64_t at) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    if constexpr (W == 4)
      v += *reinterpret_cast<const f32x4*>(parts + p * stride);
    else
      v[0] += parts[p * stride];
  }
  if constexpr (W == 1) {
    store_one(out, bf16, at, v[0]);
  } else if (bf16) {
    bf16x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(out) + at) = r;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
  }
}
template <int W>
__global__ void __launch_bounds__(256) back_finish_kernel(BackFinishArgs a) {
  const int64_t n_ds = a.ds ? a.n_tok * a.c_s : 0, n_w = (int64_t)a.hd * a.c_s;
  if (blockIdx.x >= a.sum_blocks) {
    const int n_b = a.n_heads * a.c_z, x = (int)(blockIdx.x - a.sum_blocks) * 256 + threadIdx.x;
    if (x < n_b) {
      if (a.dw_b) store_one(a.dw_b, a.bf16, x, a.t ? a.t[x] * (a.gamma ? a.gamma[x % a.c_z] : 1.0f) : 0.0f);
    } else if (x < n_b + a.c_z && a.dgamma) {
      float v = 0.0f;
#pragma unroll 4
      for (int h = 0; h < (a.t ? a.n_heads : 0); ++h) v = fmaf(a.w_b[h * a.c_z + x - n_b], a.t[h * a.c_z + x - n_b], v);
      store_one(a.dgamma, a.bf16, x - n_b, v);
    }
    return;
  }
  int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) * W;
  if (x < n_ds) {
    finish_sum<W>(a.ds_parts + x, a.ds_splits, n_ds, a.ds, a.bf16, x);
    return;
  }
  x -= n_ds;
  if (x >= 4 * n_w) return;
  const int mat = (x >= n_w) + (x >= 2 * n_w) + (x >= 3 * n_w);
  void* const out = mat == 0 ? a.dw[0] : mat == 1 ? a.dw[1] : mat == 2 ? a.dw[2] : a.dw[3];
  if (out) finish_sum<W>(a.w_parts + x, a.w_splits, 4 * n_w, out, a.bf16, x - mat * n_w);
}

template <int CT, bool BF16>
hipError_t pairs_go(const BackPairsArgs& a, unsigned grid, hipStream_t st) {
  if (back_heads_padded(a.n_heads) == 4)
    hipLaunchKernelGGL((back_pairs_kernel<CT, 1, BF16>), dim3(grid), dim3(256), 0, st, a);
  else if (back_heads_padded(a.n_heads) == 8)
    hipLaunchKernelGGL((back_pairs_kernel<CT, 2, BF16>), dim3(grid), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((back_pairs_kernel<CT, 4, BF16>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int CT>
hipError_t pairs_go(const BackPairsArgs& a, unsigned grid, hipStream_t st) {
  return a.z_bf16 ? pairs_go<CT, true>(a, grid, st) : pairs_go<CT, false>(a, grid, st);
}

unsigned blocks_of(int64_t items) { return (unsigned)((items + 255) / 256); }

}  // namespace

hipError_t launch_back_rows(const BackRowsArgs& a, hipStream_t st) {
  BackRowsArgs b = a;
  b.row_blocks = blocks_of(8 * a.n_q * a.n_heads);
  const unsigned key_blocks = blocks_of(back_keys_padded(a.n_tok) * back_heads_padded(a.n_heads) * (a.dp / 4));
  hipLaunchKernelGGL(back_rows_kernel, dim3(b.row_blocks + key_blocks), dim3(256), 0, st, b);
  return hipGetLastError();
}

int back_pairs_groups(int64_t rows, int64_t n_tok) {
  const int64_t tiles = rows * ((n_tok + kBackKeys - 1) / kBackKeys);
  return (int)(tiles < kBackMaxGroups ? tiles : kBackMaxGroups);
}

hipError_t launch_back_pairs(const BackPairsArgs& a, int groups, hipStream_t st) {
  if (a.c_z <= 32) return pairs_go<2>(a, (unsigned)groups, st);
  if (a.c_z <= 64) return pairs_go<4>(a, (unsigned)groups, st);
  if (a.c_z <= 128) return pairs_go<8>(a, (unsigned)groups, st);
  return pairs_go<16>(a, (unsigned)groups, st);
}

hipError_t launch_back_keys(const BackKeysArgs& a, int dp, hipStream_t st) {
  BackKeysArgs b = a;
  b.key_blocks = (uint32_t)((a.n_tok + 63) / 64 * a.n_splits);
  const dim3 grid(b.key_blocks + (unsigned)((a.rows + 15) / 16), (unsigned)a.n_heads);
  if (dp == 16)
    hipLaunchKernelGGL(back_keys_kernel<16>, grid, dim3(256), 0, st, b);
  else if (dp == 32)
    hipLaunchKernelGGL(back_keys_kernel<32>, grid, dim3(256), 0, st, b);
  else
    hipLaunchKernelGGL(back_keys_kernel<64>, grid, dim3(256), 0, st, b);
  return hipGetLastError();
}

hipError_t launch_back_sum(const BackSumArgs& a, hipStream_t st) {
  BackSumArgs b = a;
  const int64_t n = (a.dq_parts ? a.n_q * a.hd : 0) + 2 * a.n_tok * a.hd;
  const bool four = a.hd % 4 == 0;
  b.token_blocks = blocks_of(four ? n / 4 : n);
  const dim3 grid(b.token_blocks + (unsigned)((a.t_cols + 15) / 16));
  if (four)
    hipLaunchKernelGGL(back_sum_kernel<4>, grid, dim3(256), 0, st, b);
  else
    hipLaunchKernelGGL(back_sum_kernel<1>, grid, dim3(256), 0, st, b);
  return hipGetLastError();
}

// Splits of the token products' depths: one workgroup a CU where they are `step` deep,
// about four where they are twice that; dW, whose depth grows with the tokens and whose
// tiles do not, in up to four all the same. Fused, step 128, us of a call: 128 tokens with ds in
// 12 splits 62, in 6 64; 333 in 7 or 12 81; 1024 in 5 272, in 2 278, and with dW in 4 272, in
// 7 274, in one 280. General, step 32 (64): 128 tokens 33 us (34), 601 175 (177).
void back_gemm_splits(int64_t n_tok, int32_t hd, int32_t c_s, int32_t step, int* ds_splits, int* w_splits) {
  const int64_t c_tiles = (c_s + kGemm - 1) / kGemm, o_tiles = (hd + kGemm - 1) / kGemm;
  const int64_t ds_tiles = (n_tok + kGemm - 1) / kGemm * c_tiles, w_tiles = 4 * o_tiles * c_tiles, ds_depth = 4 * (int64_t)hd;
  auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
  auto fit = [least](int64_t a, int64_t b) {
    const int64_t n = least(a > b ? a : b, 16);
    return (int)(n < 1 ? 1 : n);
  };
  *ds_splits = fit(least(ds_depth / step, 256 / ds_tiles), least(ds_depth / (2 * step), 512 / ds_tiles));
  *w_splits = fit(least(n_tok / step, 4), least(n_tok / (2 * step), 1024 / w_tiles));
}

hipError_t launch_back_gemm(const BackGemmArgs& a, hipStream_t st) {
  BackGemmArgs b = a;
  const int64_t c_tiles = (a.c_s + kGemm - 1) / kGemm;
  const int64_t ds_blocks = a.ds_parts ? (a.n_tok + kGemm - 1) / kGemm * c_tiles * a.ds_splits : 0;
  const int64_t w_blocks = a.w_parts ? 4 * ((a.hd + kGemm - 1) / kGemm) * c_tiles * a.w_splits : 0;
  if (ds_blocks + w_blocks == 0) return hipSuccess;
  b.ds_blocks = ds_blocks;
  b.w_vec = ((reinterpret_cast<uintptr_t>(a.w_q) | reinterpret_cast<uintptr_t>(a.w_k) | reinterpret_cast<uintptr_t>(a.w_v) |
              reinterpret_cast<uintptr_t>(a.w_g)) & 15) == 0;
  hipLaunchKernelGGL(back_gemm_kernel, dim3((unsigned)(ds_blocks + w_blocks)), dim3(256), 0, st, b);
  return hipGetLastError();
}

hipError_t launch_back_finish(const BackFinishArgs& a, hipStream_t st) {
  BackFinishArgs b = a;
  const int64_t n = (a.ds ? a.n_tok * a.c_s : 0) + (a.dw[0] || a.dw[1] || a.dw[2] || a.dw[3] ? 4 * (int64_t)a.hd * a.c_s : 0);
  const int64_t tail = a.dw_b || a.dgamma ? (int64_t)a.n_heads * a.c_z + a.c_z : 0;
  const bool four = a.c_s % 4 == 0;
  b.sum_blocks = blocks_of(four ? (n + 3) / 4 : n);
  const unsigned blocks = b.sum_blocks + blocks_of(tail);
  if (blocks == 0) return hipSuccess;
  if (four)
    hipLaunchKernelGGL(back_finish_kernel<4>, dim3(blocks), dim3(256), 0, st, b);
  else
    hipLaunchKernelGGL(back_finish_kernel<1>, dim3(blocks), dim3(256), 0, st, b);
  return hipGetLastError();
}

}  // namespace dcp
