// Products over tokens for the fused shape's backward pass (H d = 384, c_s a multiple of
// 32, s in bf16; gfx950):
//   q, k, v, g = s W^T   (with the sigmoid of g, and the largest |q|, |k|, |v|)
//   ds = dq W_q + dg W_g + dk W_k + dv W_v
//   dW_x = dx^T s
// fp32 operands enter the bf16 matrix cores as hi + lo, 16 significant bits, s as it
// is: two products each for q, k, v, g and dW, three (hi hi, hi lo, lo hi) for ds, at 16
// times the fp32 matrix rate. bf16 has fp32's range, so nothing is scaled. The kernels
// that write an operand split it (prep_kernel and pack_kernel in backward_fast.hip,
// back_sum_kernel in backward.hip): splitting each time it is staged took longer than
// the products.
//
// 4800 tokens and a stripe of 2400, c_s = 384: 32 us for q, k, v, g and 55 for ds and dW (265
// and 385 TFLOP/s of bf16 products), bound by the staging of 64-wide tiles; tiles of 128 gained
// under 1% of the call and lost on small ones. 333 tokens: 10 and 11 us, the latency of
// 12 and 11 dependent steps.
//
// A workgroup of four waves takes 64 x 64 outputs, 32 x 32 a wave; operands 32 deep go
// through LDS in two buffers, the next two steps in flight in registers. An operand whose
// depth runs along its rows lies in LDS by rows of 32 (16-byte pieces XOR-swizzled by
// row); one whose depth runs across them lies as it came, and is read with the
// transposing LDS read, which hands lane i of 16 column i of four rows.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

constexpr int kHD = kFastH * kFastD;
constexpr int kTile = 64, kDeep = 32;
constexpr int kRow = kTile + 16;  // halfs per row of a transposed operand

// One operand's buffer: [64][32] or [32][80], hi or lo.
struct Side {
  u32x4 w[kDeep * kRow / 8];
};
struct GemmLds {
  Side a[2][2], b[2][2];  // [buffer][hi, lo]
};

// Eight consecutive elements: hi and, of a split operand, lo.
struct Eight {
  u32x4 hi, lo;
};
template <bool SPLIT>
__device__ __forceinline__ void load8(Eight& e, bool in, const uint16_t* p, int64_t lo) {
  const u32x4 zero = {0u, 0u, 0u, 0u};
  e.hi = in ? *reinterpret_cast<const u32x4*>(p) : zero;
  if constexpr (SPLIT) e.lo = in ? *reinterpret_cast<const u32x4*>(p + lo) : zero;
}

// Where a thread's eight elements go. Depth along the rows (ALONG): row tid / 4, depth
// 8 (tid % 4); across: depth tid / 8, columns 8 (tid % 8).
template <bool ALONG>
__device__ __forceinline__ int piece_at(int tid) {
  if constexpr (ALONG) return (tid >> 2) * 4 + ((tid & 3) ^ ((tid >> 4) & 3));
  return (tid >> 3) * (kRow / 8) + (tid & 7);
}
template <bool ALONG, bool SPLIT>
__device__ __forceinline__ void stage(Side (&to)[2], const Eight& e, int tid) {
  to[0].w[piece_at<ALONG>(tid)] = e.hi;
  if constexpr (SPLIT) to[1].w[piece_at<ALONG>(tid)] = e.lo;
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
// The operand of 16 rows (or columns) from r0: lane (n, g), depth 8g .. 8g + 7.
template <bool ALONG>
__device__ __forceinline__ bf16x8 operand(const Side& s, int r0, int lane) {
  const int n = lane & 15, g = lane >> 4;
  if constexpr (ALONG) {
    const int row = r0 + n;
    return as_bf16x8(s.w[row * 4 + (g ^ ((row >> 2) & 3))]);
  } else {
    const uint32_t at = lds_addr(&s) + 2 * ((8 * g + (n >> 2)) * kRow + r0 + 4 * (n & 3));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + 2 * 4 * kRow));
    const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
    return as_bf16x8(u32x4{l[0], l[1], h[0], h[1]});
  }
}

// acc += A B over `steps` steps of 32; fetch(step, a, b) loads a thread's pieces, two
// steps ahead of their use.
template <bool A_ALONG, bool A_SPLIT, bool B_ALONG, bool B_SPLIT, typename Fetch>
__device__ __forceinline__ void product(GemmLds& s, int64_t steps, Fetch fetch, f32x4 (&acc)[2][2]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int am = 32 * (wave >> 1), bn = 32 * (wave & 1);
  Eight a[2], b[2];
  auto put = [&](auto buf) {
    stage<A_ALONG, A_SPLIT>(s.a[buf], a[buf], tid);
    stage<B_ALONG, B_SPLIT>(s.b[buf], b[buf], tid);
  };
  auto step = [&](int64_t i, auto buf) {
    constexpr int kBuf = decltype(buf)::value;
    __syncthreads();  // the buffer is staged, and the other one read
    if (i + 2 < steps) fetch(i + 2, a[kBuf], b[kBuf]);
    bf16x8 ah[2], al[2], bh[2], bl[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ah[u] = operand<A_ALONG>(s.a[kBuf][0], am + 16 * u, lane);
      bh[u] = operand<B_ALONG>(s.b[kBuf][0], bn + 16 * u, lane);
      if constexpr (A_SPLIT) al[u] = operand<A_ALONG>(s.a[kBuf][1], am + 16 * u, lane);
      if constexpr (B_SPLIT) bl[u] = operand<B_ALONG>(s.b[kBuf][1], bn + 16 * u, lane);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        acc[u][w] = mfma32(ah[u], bh[w], acc[u][w]);
        if constexpr (B_SPLIT) acc[u][w] = mfma32(ah[u], bl[w], acc[u][w]);
        if constexpr (A_SPLIT) acc[u][w] = mfma32(al[u], bh[w], acc[u][w]);
      }
    if (i + 1 < steps) put(std::integral_constant<int, 1 - kBuf>());
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  if (steps > 0) fetch(0, a[0], b[0]);
  if (steps > 1) fetch(1, a[1], b[1]);
  if (steps > 0) put(even);
  for (int64_t i = 0; i < steps; i += 2) {
    step(i, even);
    if (i + 1 < steps) step(i + 1, odd);
  }
}

__device__ __forceinline__ void clear(f32x4 (&acc)[2][2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// ----------------------------------------------------------------------------- q, k, v, g
// Blocks: 12 tiles of the side's two projections, token tiles of the keys then of the
// stripe's rows.
__global__ void __launch_bounds__(256) token_proj_kernel(TokenArgs p) {
  __shared__ GemmLds s;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int kTiles = kHD / kTile;  // 6 of a projection
  const int64_t key_tiles = (p.n_tok + kTile - 1) / kTile;
  const int64_t tile = blockIdx.x / (2 * kTiles);
  const int col = (int)(blockIdx.x % (2 * kTiles));
  const bool q_side = tile >= key_tiles, second = col >= kTiles;
  const int64_t row0 = (tile - (q_side ? key_tiles : 0)) * kTile, rows = q_side ? p.n_q : p.n_tok;
  const int o0 = (col % kTiles) * kTile;
  const int which = q_side ? (second ? 3 : 0) : (second ? 2 : 1);  // q, k, v, g
  float* dst = which == 0 ? p.q : which == 1 ? p.k : which == 2 ? p.v : p.g;
  const int64_t row = min(row0 + (tid >> 2), rows - 1);  // rows past the last repeat it
  const uint16_t* sp = p.s + ((q_side ? p.q_row0 : 0) + row) * p.c_s + 8 * (tid & 3);
  const uint16_t* wp = p.w + ((int64_t)which * kHD + o0 + (tid >> 2)) * p.c_s + 8 * (tid & 3);
  const int64_t w_lo = (int64_t)4 * kHD * p.c_s;
  f32x4 acc[2][2];
  clear(acc);
  product<true, false, true, true>(
      s, p.c_s / kDeep,
      [&](int64_t i, Eight& a, Eight& b) {
        load8<false>(a, true, sp + i * kDeep, 0);
        load8<true>(b, true, wp + i * kDeep, w_lo);
      },
      acc);
  float top = 0.0f;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = row0 + 32 * (wave >> 1) + 16 * u + 4 * g + i;
      if (t >= rows) continue;
      const bool masked = !q_side && p.mask && p.mask[t] == 0;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float v = acc[u][x][i];
        if (!masked) top = fmaxf(top, finite_abs(v));
        if (q_side && second) v = 1.0f / (1.0f + expf(-v));
        dst[t * kHD + o0 + 32 * (wave & 1) + 16 * x + n] = v;
      }
    }
  if (q_side && second) return;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  // a maximum does not depend on its order; 64 words per tensor, since atomics on one
  // word go one after another
  if (lane == 0)
    atomicMax(p.tops + 64 * (q_side ? 0 : second ? 2 : 1) + ((4 * (int)blockIdx.x + wave) & 63), __float_as_uint(top));
}

// ----------------------------------------------------------------------------- ds, dW
__global__ void __launch_bounds__(256) token_grad_kernel(TokenArgs p) {
  __shared__ GemmLds s;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c_tiles = (p.c_s + kTile - 1) / kTile;
  uint32_t b = blockIdx.x;
  const bool is_ds = b < p.ds_blocks;
  if (!is_ds) b -= (uint32_t)p.ds_blocks;
  const int c0 = (int)(b % c_tiles) * kTile;
  b /= c_tiles;
  const int splits = is_ds ? p.ds_splits : p.w_splits, split = (int)(b % splits);
  b /= splits;
  const int c = c0 + 8 * (tid & 7);
  const bool c_in = c < p.c_s;
  const int64_t kv_lo = 2 * p.n_tok * kHD, q_lo = p.n_q * kHD;
  f32x4 acc[2][2];
  clear(acc);
  int64_t m0, m_end;
  float* out;
  if (is_ds) {
    m0 = (int64_t)b * kTile;
    m_end = p.n_tok;
    out = p.ds_parts + (int64_t)split * p.n_tok * p.c_s;
    // the terms k, v, and q, g where the tile holds rows of the stripe
    const bool with_rows = m0 < p.q_row0 + p.n_q && m0 + kTile > p.q_row0;
    constexpr int kSteps = kHD / kDeep;
    int64_t steps, first;
    chunk_of_32(kSteps * (with_rows ? 4 : 2), splits, split, &steps, &first);
    const int64_t t = m0 + (tid >> 2), tq = t - p.q_row0, w_lo = (int64_t)4 * kHD * p.c_s;
    const bool kv_in = t < p.n_tok, q_in = tq >= 0 && tq < p.n_q;
    const int64_t kv_at = t * kHD + 8 * (tid & 3), q_at = tq * kHD + 8 * (tid & 3), w_at = (int64_t)(tid >> 3) * p.c_s + c;
    product<true, true, false, true>(
        s, steps,
        [&](int64_t i, Eight& a, Eight& bb) {
          const int step = (int)(first + i), term = step / kSteps, o = (step - term * kSteps) * kDeep;
          const uint16_t* x = term == 0 ? p.dkv : term == 1 ? p.dkv + p.n_tok * kHD : term == 2 ? p.dq : p.dg;
          const int mat = term == 0 ? 1 : term == 1 ? 2 : term == 2 ? 0 : 3;
          load8<true>(a, term < 2 ? kv_in : q_in, x + (term < 2 ? kv_at : q_at) + o, term < 2 ? kv_lo : q_lo);
          load8<true>(bb, c_in, p.w + ((int64_t)mat * kHD + o) * p.c_s + w_at, w_lo);
        },
        acc);
  } else {
    const int mat = (int)(b / (kHD / kTile));  // q, k, v, g
    m0 = (b % (kHD / kTile)) * kTile;
    m_end = kHD;
    out = p.w_parts + ((int64_t)split * 4 + mat) * kHD * p.c_s;
    const bool stripe = mat == 0 || mat == 3;
    const int64_t rows = stripe ? p.n_q : p.n_tok, s_row0 = stripe ? p.q_row0 : 0;
    const uint16_t* x = mat == 0 ? p.dq : mat == 1 ? p.dkv : mat == 2 ? p.dkv + p.n_tok * kHD : p.dg;
    int64_t steps, first;
    chunk_of_32((uint32_t)((rows + kDeep - 1) / kDeep), splits, split, &steps, &first);
    const int64_t t0 = first * kDeep + (tid >> 3);
    const uint16_t *xp = x + t0 * kHD + m0 + 8 * (tid & 7), *sp = p.s + (s_row0 + t0) * p.c_s + c;
    product<false, true, false, false>(
        s, steps,
        [&](int64_t i, Eight& a, Eight& bb) {
          const int64_t t = t0 + i * kDeep;
          const bool in = t < rows;
          load8<true>(a, in, xp + i * kDeep * kHD, stripe ? q_lo : kv_lo);
          // a masked token's s does not enter the gradients of W_k and W_v
          load8<false>(bb, in && c_in && (stripe || !p.mask || p.mask[t] != 0), sp + i * kDeep * p.c_s, 0);
        },
        acc);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + 32 * (wave >> 1) + 16 * u + 4 * g + i;
        const int cc = c0 + 32 * (wave & 1) + 16 * x + n;
        if (m < m_end && cc < p.c_s) out[m * p.c_s + cc] = acc[u][x][i];
      }
}

}  // namespace

hipError_t launch_token_proj(const TokenArgs& a, hipStream_t st) {
  const int64_t tiles = (a.n_tok + kTile - 1) / kTile + (a.n_q + kTile - 1) / kTile;
  hipLaunchKernelGGL(token_proj_kernel, dim3((unsigned)(tiles * 2 * (kHD / kTile))), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_token_grad(const TokenArgs& a, hipStream_t st) {
  TokenArgs b = a;
  const int64_t c_tiles = (a.c_s + kTile - 1) / kTile;
  b.ds_blocks = a.ds_parts ? (a.n_tok + kTile - 1) / kTile * c_tiles * a.ds_splits : 0;
  const int64_t w_blocks = a.w_parts ? 4 * (kHD / kTile) * c_tiles * a.w_splits : 0;
  if (b.ds_blocks + w_blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(token_grad_kernel, dim3((unsigned)(b.ds_blocks + w_blocks)), dim3(256), 0, st, b);
  return hipGetLastError();
}

}  // namespace dcp
