// Relative position encoding of the pair track and its tables' gradient (gfx950).
// (Appendix, relative-position sub-chunking: one-hots of the residue and token offsets
// clipped to +-32, the chain hop clipped to +-2 and the same entity, then a linear layer;
// the product of a one-hot with a table is a row of the table, so no one-hot is formed.)
//
//   bucket_f(i, j) = clamp(position_f[i] - position_f[j], -r_f, r_f) + r_f   in one group of field f,
//                    2 r_f + 1                                             in different ones,
//   z_out[i, j] = z_in[i, j] + sum over f of table[first_f + bucket_f(i, j)],
//   dtable[first_f + b] = sum over the pairs of bucket b of dz[i, j].
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cdna4.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

// The bucket of tokens with positions p, q in groups g, h. A difference past 32 bits saturates, far outside +-r.
__device__ __forceinline__ uint32_t bucket_of(int32_t p, int32_t q, int32_t g, int32_t h, int32_t r) {
  const int32_t d = __builtin_elementwise_sub_sat(p, q);
  return (uint32_t)(g == h ? max(min(d, r), -r) + r : 2 * r + 1);
}

// Buckets of a pair, a byte per field (at most 2 * 127 + 1)
__device__ __forceinline__ uint32_t buckets_of(const RelativeArgs& a, int64_t i, int64_t j) {
  uint32_t t = 0;
#pragma unroll
  for (int f = 0; f < kRelativeFields; ++f)
    if (f < a.n_fields) {
      const int32_t* group = a.group[f];
      t |= bucket_of(a.position[f][i], a.position[f][j], group ? group[i] : 0, group ? group[j] : 0, a.radius[f]) << (8 * f);
    }
  return t;
}

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_f32(float v, float* p) { *p = v; }
__device__ __forceinline__ void store_f32(float v, uint16_t* p) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// One wave per 64 pairs of a row, a lane per channel and 64 channels at a time: any width and alignment. Eight pairs' values are in
// flight at once, and where these do not all have the buckets of the pair before them, their rows of the table: 1024 tokens of 101
// channels in bf16 297 us (one pair at a time 601), bound by the number of loads and stores of two bytes a lane.
template <typename T>
__global__ void __launch_bounds__(256) relative_any_kernel(RelativeArgs a) {
  constexpr int kBatch = 8;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (a.first_block + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t blocks = (a.n_tok + 63) / 64;
  if (unit >= a.n_rows * blocks) return;
  const int64_t row = unit / blocks, j0 = (unit - row * blocks) * 64;
  const int n = (int)min((int64_t)64, a.n_tok - j0);
  const uint32_t mine = buckets_of(a, a.row0 + row, min(j0 + lane, a.n_tok - 1));
  for (int c0 = 0; c0 < a.c; c0 += 64) {
    const int c = min(c0 + lane, a.c - 1);
    const int64_t first = (row * a.n_tok + j0) * a.c + c;
    float sum = 0.0f;  // of the pair before
    uint32_t last = 0;
    bool any = false;
    for (int k0 = 0; k0 < n; k0 += kBatch) {
      float z[kBatch], s[kBatch];
      uint32_t t[kBatch];
      bool same = any;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int p = min(k0 + k, n - 1);
        z[k] = a.z_in ? load_f32(static_cast<const T*>(a.z_in) + first + (int64_t)p * a.c) : 0.0f;
        t[k] = (uint32_t)__builtin_amdgcn_readlane((int)mine, p);
        same = same && t[k] == last;
        s[k] = sum;
      }
      if (!same) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) s[k] = 0.0f;
#pragma unroll
        for (int f = 0; f < kRelativeFields; ++f)
          if (f < a.n_fields)
#pragma unroll
            for (int k = 0; k < kBatch; ++k) s[k] += a.table[(int64_t)(a.first[f] + (int)(t[k] >> (8 * f) & 255)) * a.c + c];
      }
      any = true;
      last = t[kBatch - 1];
      sum = s[kBatch - 1];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (k0 + k < n && c0 + lane < a.c) store_f32(z[k] + s[k], static_cast<T*>(a.z_out) + first + (int64_t)(k0 + k) * a.c);
    }
  }
}

// Rows of whole 16-byte pieces: 2^k lanes a pair, a piece each, and so 64 / 2^k pairs at a time; the lanes of a pair
// go through 2^k consecutive ones. The sum of the table's rows is kept while the buckets stay the same, as they do
// where the offsets are clipped or the chains differ; else its rows come from the caches (71 KB of the paper's
// fields at 128 channels). Bound by memory: 1024 tokens of 128 channels in bf16 111 us, 4.9 TB/s.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) relative_kernel(RelativeArgs a) {
  constexpr int kVec = 16 / sizeof(T), kBatch = LANES < 8 ? LANES : 8;
  const int lane = threadIdx.x & 63, piece = lane & (LANES - 1), base = lane & ~(LANES - 1);
  const int64_t unit = (a.first_block + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t blocks = (a.n_tok + 63) / 64;
  if (unit >= a.n_rows * blocks) return;
  const int64_t row = unit / blocks, j0 = (unit - row * blocks) * 64;
  const int left = (int)min((int64_t)64, a.n_tok - j0);
  const uint32_t mine = buckets_of(a, a.row0 + row, min(j0 + lane, a.n_tok - 1));
  const bool holds = piece * kVec < a.c;
  const int pieces = a.c / kVec;
  const int64_t first = (row * a.n_tok + j0 + base) * pieces + piece;
  const float* const table = a.table + piece * kVec;
  float sum[kVec];
  uint32_t last = 0;
  bool any = false;
#pragma unroll 1
  for (int k0 = 0; k0 < LANES; k0 += kBatch) {
    u32x4 z[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      z[k] = u32x4{0u, 0u, 0u, 0u};
      if (a.z_in && holds && base + k0 + k < left)
        z[k] = __builtin_nontemporal_load(static_cast<const u32x4*>(a.z_in) + first + (int64_t)(k0 + k) * pieces);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const uint32_t t = (uint32_t)__shfl((int)mine, base + k0 + k);
      if (!holds || base + k0 + k >= left) continue;
      if (!any || t != last) {
        any = true;
        last = t;
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
#pragma unroll
        for (int f = 0; f < kRelativeFields; ++f)
          if (f < a.n_fields) {
            const float* r = table + (int64_t)(a.first[f] + (int)(t >> (8 * f) & 255)) * a.c;
#pragma unroll
            for (int e = 0; e < kVec; e += 4) {
              const f32x4 v = *reinterpret_cast<const f32x4*>(r + e);
#pragma unroll
              for (int i = 0; i < 4; ++i) sum[e + i] += v[i];
            }
          }
      }
      u32x4 o;
      if (kVec == 8) {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          b[e] = (__bf16)(__uint_as_float(e & 1 ? z[k][e >> 1] & 0xFFFF0000u : z[k][e >> 1] << 16) + sum[e % kVec]);
        o = __builtin_bit_cast(u32x4, b);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(__uint_as_float(z[k][e]) + sum[e]);
      }
      __builtin_nontemporal_store(o, static_cast<u32x4*>(a.z_out) + first + (int64_t)(k0 + k) * pieces);
    }
  }
}

// ----------------------------------------------------------------------------- the table's gradient
// dtable = one-hot^T dz on the matrix cores: v_mfma_f32_16x16x32_bf16 with 16 buckets of one field as rows, 32 pairs
// as k-slots and 16 channels as columns. A one-hot's products are exact, and so are fp32 gradients in three bf16 pieces
// (8 bits each); the sums are fp32, in an order that the sizes and the fields alone fix. Only the tiles of buckets that
// occur among the 32 pairs are multiplied, near the diagonal three or four of twelve. 32 pairs with the same buckets in all
// fields, or with two kinds of them, as most have far from the diagonal, are summed by kind ("class"), up to 16 kinds
// side by side in one tile, and the kinds' sums added to their buckets when there is no room for another and at the end: two
// products where a product per field took eight and twelve comparisons. (2400 x 4800 pairs of 60 chains: 909 us so, 749 with one kind at
// a time, which is the better for one long chain, 500 to 635.)
//   A workgroup takes consecutive tiles of 128 S pairs of a row (fp32: 64 S) and 32 CG channels (S CG = 4): CG
// waves take 32 channels each, and S such sets a share of the pairs, each with sums of its own. dz comes through
// registers, a tile ahead, into LDS as [pair][channel], whose transposing reads bring 16 channels of eight pairs as a B operand;
// k-slot 8g + j is pair 4g + j of the 32 for j < 4, 16 + 4g + j - 4 for j >= 4. Wave f finds the buckets of field f, a
// byte of each pair's word in LDS.
//   A value that is not finite would make NaN of every bucket (0 times infinity): it enters as 0 and is added to its
// own buckets afterwards. 2400 x 4800 pairs of 128 channels in bf16: 600 us, 5.0 TB/s; 453 without the products, 6.5: bound by memory and
// by the chains of comparisons between them.
constexpr int kWindow = 12;  // tiles of buckets at a time: the paper's fields have 5 + 5 + 1 + 1

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Pairs of a tile that a set of waves has to itself: a tile is 32 KB, which are in flight while the one before is worked on.
constexpr int relative_own_pairs(bool bf16) { return bf16 ? 128 : 64; }

template <typename T, int CG, bool VEC>
__global__ void __launch_bounds__(256, 2) relative_back_kernel(RelativeArgs a) {
  constexpr int kVec = 16 / sizeof(T), S = 4 / CG, kOwn = relative_own_pairs(sizeof(T) == 2), kPairs = kOwn * S, kChannels = 32 * CG;
  constexpr int kPlanes = sizeof(T) == 2 ? 1 : 3, kRow = 2 * kChannels + 32, kPlane = kPairs * kRow;
  constexpr int kRowPieces = kChannels / kVec, kMine = kPairs * kRowPieces / 256;
  __shared__ __attribute__((aligned(16))) char s_d[kPlanes * kPlane];
  __shared__ __attribute__((aligned(16))) uint32_t s_b[kPairs];
  __shared__ __attribute__((aligned(16))) int s_bad[4];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), cg = wave % CG, stream = wave / CG;
  const int c0 = blockIdx.y * kChannels, w0 = blockIdx.z * kWindow;
  const int64_t row_tiles = (a.n_tok + kPairs - 1) / kPairs;
  int64_t todo, first;
  chunk_of(a.n_rows * row_tiles, gridDim.x, blockIdx.x, &todo, &first);
  f32x4 acc[kWindow][2];
#pragma unroll
  for (int w = 0; w < kWindow; ++w) acc[w][0] = acc[w][1] = f32x4{0.f, 0.f, 0.f, 0.f};

  // this window's tiles: where the field's byte is, and the tile's place among the field's (16 for none)
  int shift[kWindow];
  uint32_t place[kWindow];
#pragma unroll
  for (int w = 0; w < kWindow; ++w) {
    const bool there = w0 + w < a.n_tiles;
    shift[w] = __builtin_amdgcn_readfirstlane(there ? 8 * a.tile_field[w0 + w] : 0);
    place[w] = (uint32_t)__builtin_amdgcn_readfirstlane(there ? a.tile_of_field[w0 + w] : 16);
  }
  // the tile to be fetched next, and the one that is worked on
  int64_t row = first / row_tiles, j0 = (first - row * row_tiles) * kPairs, this_row = row, this_j0 = j0;
  const int field = min(wave, a.n_fields - 1);
  const int32_t *const position = a.position[field], *const group = a.group[field];
  const T* const dz = static_cast<const T*>(a.dz);
  int offset[kMine];  // bytes in a tile
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int p = (tid + 256 * k) / kRowPieces, c = c0 + (tid + 256 * k) % kRowPieces * kVec;
    offset[k] = c < a.c ? (p * a.c + c) * (int)sizeof(T) : kOutOfRange;
  }
  constexpr int kLanes = kPairs / 64;  // pairs of a tile that a lane finds the bucket of
  u32x4 raw[kMine];
  int32_t pos_i, grp_i, pos_j[kLanes], grp_j[kLanes];
  auto places = [&](int64_t row, int64_t j0) {
    pos_i = position[a.row0 + row];
    grp_i = group ? group[a.row0 + row] : 0;
#pragma unroll
    for (int s = 0; s < kLanes; ++s) {
      const int64_t j = min(j0 + 64 * s + lane, a.n_tok - 1);
      pos_j[s] = position[j];
      grp_j[s] = group ? group[j] : 0;
    }
  };
  auto fetch = [&]() {
    const T* const base = dz + (row * a.n_tok + j0) * a.c;
    const int left = (int)min((int64_t)kPairs, a.n_tok - j0);
    if (VEC) {
      const __amdgpu_buffer_rsrc_t res =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, left * a.c * (int)sizeof(T), kRawBufferFlags);
#pragma unroll
      for (int k = 0; k < kMine; ++k) raw[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(res, offset[k], 0, 2));
    } else {
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        const int p = (tid + 256 * k) / kRowPieces, c = c0 + (tid + 256 * k) % kRowPieces * kVec;
        raw[k] = u32x4{0u, 0u, 0u, 0u};
        if (p >= left) continue;
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (c + e < a.c) {
            const float v = load_f32(base + p * a.c + c + e);
            if (sizeof(T) == 2)
              raw[k][e >> 1] |= (__float_as_uint(v) >> 16) << (16 * (e & 1));
            else
              raw[k][e & 3] = __float_as_uint(v);
          }
      }
    }
    if (VEC) places(row, j0);
    j0 += kPairs;
    if (j0 >= a.n_tok) {
      j0 = 0;
      ++row;
    }
  };
  // Sums of up to 16 classes, of pairs that are alike in all fields: row n of `run` is that of the buckets `cls` of lane n
  f32x4 run[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  uint32_t cls = 0;
  int n_cls = 0;
  // Their sums to those of the buckets of window tile w: a class is k-slot g of step i = 4g + i, so that `run` is the B operands as
  // it lies. of: the classes' buckets, of this lane's k-slots.
  // Halves, which the products take twice: a sum past fp32's range is then finite here, as 0 times infinity would make NaN of other
  // buckets, and infinite in its own. (Exact from 2^-125 on.)
  auto halve_run = [&]() {
#pragma unroll
    for (int ct = 0; ct < 2; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) run[ct][i] = __builtin_amdgcn_fmed3f(0.5f * run[ct][i], -3.402823466e38f, 3.402823466e38f);
  };
  auto end_classes = [&](const uint32_t (&of)[4], int w, f32x4 (&to)[2]) {
    float hot[4];
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool here = 4 * g + i < n_cls && (of[i] >> shift[w] >> 4 & 15) == place[w];
      hot[i] = here && (of[i] >> shift[w] & 15) == (uint32_t)n ? 2.0f : 0.0f;
      any |= here;
    }
    if (__builtin_amdgcn_ballot_w64(any) == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int ct = 0; ct < 2; ++ct)
        to[ct] = __builtin_amdgcn_mfma_f32_16x16x4f32(hot[i], run[ct][i], to[ct], 0, 0, 0);
  };
  for (int k = tid; k < kPairs; k += 256) s_b[k] = 0;  // bytes of fields that are not there: alike in all pairs
  if (todo > 0) fetch();
  for (int64_t k_tile = 0; k_tile < todo; ++k_tile) {
    barrier_lds();  // the tile before has been read
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      char* const to = s_d + (tid + 256 * k) / kRowPieces * kRow + (tid + 256 * k) % kRowPieces * (2 * kVec);
      u32x4 r = raw[k];
      if (sizeof(T) == 2) {
        u16x2 top = {0, 0};
#pragma unroll
        for (int d = 0; d < 4; ++d) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, r[d] & 0x7FFF7FFFu));
        if (max(top[0], top[1]) >= 0x7F80) {
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            if ((r[d] & 0x7F800000u) == 0x7F800000u) r[d] &= 0xFFFFu;
            if ((r[d] & 0x7F80u) == 0x7F80u) r[d] &= 0xFFFF0000u;
          }
          bad = true;
        }
        *reinterpret_cast<u32x4*>(to) = r;
      } else {
        uint32_t piece[3][2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = __uint_as_float(r[e]);
          if ((r[e] & 0x7F800000u) == 0x7F800000u) {
            v = 0.0f;
            bad = true;
          }
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            const uint32_t top = __float_as_uint(v) & 0xFFFF0000u;
            v -= __uint_as_float(top);
            piece[q][e >> 1] = e & 1 ? piece[q][e >> 1] | top : top >> 16;
          }
        }
#pragma unroll
        for (int q = 0; q < kPlanes; ++q) *reinterpret_cast<u32x2*>(to + q * kPlane) = u32x2{piece[q][0], piece[q][1]};
      }
    }
    if (!VEC) places(this_row, this_j0);  // a tile ahead there are no registers for them
    if (wave < a.n_fields)
#pragma unroll
      for (int s = 0; s < kLanes; ++s)
        reinterpret_cast<uint8_t*>(s_b)[4 * (64 * s + lane) + wave] =
            (uint8_t)bucket_of(pos_i, pos_j[s], grp_i, grp_j[s], a.radius[field]);
    const uint64_t any_bad = __builtin_amdgcn_ballot_w64(bad);
    if (lane == 0) s_bad[wave] = any_bad != 0;
    barrier_lds();
    if (k_tile + 1 < todo) fetch();
#pragma unroll 1
    for (int ks = 0; ks < kOwn / 32; ++ks) {
      const int p0 = kOwn * stream + 32 * ks;  // these 32 pairs
      const uint32_t buckets = s_b[p0 + (lane & 31)];
      bf16x8 d[kPlanes][2];
#pragma unroll
      for (int q = 0; q < kPlanes; ++q)
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
          u32x4 v;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4*)(s_d + q * kPlane + (p0 + 16 * half + 4 * g + (n >> 2)) * kRow + 64 * cg + 32 * ct +
                             8 * (n & 3)));
            const u32x2 w = __builtin_bit_cast(u32x2, x);
            v[2 * half] = w[0];
            v[2 * half + 1] = w[1];
          }
          d[q][ct] = as_bf16x8(v);
        }
      const u32x4 b0 = *reinterpret_cast<const u32x4*>(&s_b[p0 + 4 * g]), b1 = *reinterpret_cast<const u32x4*>(&s_b[p0 + 16 + 4 * g]);
      const uint32_t one = (uint32_t)__builtin_amdgcn_readfirstlane((int)buckets);
      const uint32_t two = (uint32_t)__builtin_amdgcn_readlane((int)buckets, 31);
      const bool few = __builtin_amdgcn_ballot_w64(buckets != one && buckets != two) == 0;
      const bool has_one = (__builtin_amdgcn_ballot_w64(cls == one) & ((1u << n_cls) - 1)) != 0, has_two = (__builtin_amdgcn_ballot_w64(cls == two) & ((1u << n_cls) - 1)) != 0;
      const bool full = few && !(has_one && has_two) && n_cls > 14;
      if (!few || full) {
        uint32_t of[4] = {0, 0, 0, 0};
        if (full) halve_run();
        if (full)
#pragma unroll
          for (int i = 0; i < 4; ++i) of[i] = (uint32_t)__shfl((int)cls, 4 * g + i);
#pragma unroll
        for (int w = 0; w < kWindow; ++w) {
          if (full) end_classes(of, w, acc[w]);
          if (few || __builtin_amdgcn_ballot_w64((buckets >> shift[w] >> 4 & 15) == place[w]) == 0) continue;
          const uint32_t want = 16 * place[w] + (uint32_t)n;
          auto is = [&](uint32_t b, uint32_t v) { return (b >> shift[w] & 255) == want ? v : 0u; };
          u32x4 hot;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            hot[i] = is(b0[2 * i], 0x3F80u) | is(b0[2 * i + 1], 0x3F800000u);
            hot[2 + i] = is(b1[2 * i], 0x3F80u) | is(b1[2 * i + 1], 0x3F800000u);
          }
#pragma unroll
          for (int q = 0; q < kPlanes; ++q)
#pragma unroll
            for (int ct = 0; ct < 2; ++ct) acc[w][ct] = mfma32(as_bf16x8(hot), d[q][ct], acc[w][ct]);
        }
        if (!few) continue;
        run[0] = run[1] = f32x4{0.f, 0.f, 0.f, 0.f};
        n_cls = 0;
      }
      if (full || !has_one) {
        cls = n == n_cls ? one : cls;
        ++n_cls;
      }
      if ((full || !has_two) && two != one) {
        cls = n == n_cls ? two : cls;
        ++n_cls;
      }
      const bool used = n < n_cls;
      auto is = [&](uint32_t b, uint32_t v) { return used && b == cls ? v : 0u; };
      const uint32_t v = is(one, 0x3F803F80u);
      u32x4 hot = {v, v, v, v};
      if (one != two)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          hot[i] = is(b0[2 * i], 0x3F80u) | is(b0[2 * i + 1], 0x3F800000u);
          hot[2 + i] = is(b1[2 * i], 0x3F80u) | is(b1[2 * i + 1], 0x3F800000u);
        }
#pragma unroll
      for (int q = 0; q < kPlanes; ++q)
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) run[ct] = mfma32(as_bf16x8(hot), d[q][ct], run[ct]);
    }
    if (s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3]) {
#pragma unroll 1
      for (int p = 0; p < kOwn; ++p) {
        const int64_t j = this_j0 + kOwn * stream + p;
        if (j >= a.n_tok) break;
        const uint32_t b = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_b[kOwn * stream + p]);
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
          const int c = c0 + 32 * cg + 16 * ct + n;
          const float v = c < a.c ? load_f32(dz + (this_row * a.n_tok + j) * a.c + c) : 0.0f;
          const bool add = (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u;
          if (!__builtin_amdgcn_ballot_w64(add)) continue;
#pragma unroll
          for (int w = 0; w < kWindow; ++w) {
            const uint32_t of_tile = (b >> shift[w] & 255) - 16u * place[w];  // of none: not below 16
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (add && of_tile == (uint32_t)(4 * g + i)) acc[w][ct][i] += v;
          }
        }
      }
    }
    this_j0 += kPairs;
    if (this_j0 >= a.n_tok) {
      this_j0 = 0;
      ++this_row;
    }
  }
  const int64_t part = (int64_t)blockIdx.x * S + stream;
  uint32_t of[4];
  halve_run();
#pragma unroll
  for (int i = 0; i < 4; ++i) of[i] = (uint32_t)__shfl((int)cls, 4 * g + i);
#pragma unroll
  for (int w = 0; w < kWindow; ++w) {
    if (w0 + w >= a.n_tiles) continue;
    end_classes(of, w, acc[w]);
#pragma unroll
    for (int ct = 0; ct < 2; ++ct) {
      const int c = c0 + 32 * cg + 16 * ct + n;
      if (c < a.c)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.parts[(part * a.n_tiles * 16 + (w0 + w) * 16 + 4 * g + i) * a.c + c] = acc[w][ct][i];
    }
  }
}

// A bucket and 64 channels a workgroup: four waves each add up every fourth part, in order. 500 parts: 10 us, 49 MB from the
// last-level cache.
__global__ void __launch_bounds__(256) relative_sum_kernel(RelativeArgs a) {
  __shared__ float s_sum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 64 + lane;
  int f = 0, b = blockIdx.x, tile = 0;
  while (b >= 2 * a.radius[f] + 2) {
    b -= 2 * a.radius[f] + 2;
    tile += (2 * a.radius[f] + 17) / 16;
    ++f;
  }
  const int64_t rows = 16 * a.n_tiles, at = (16 * tile + b) * (int64_t)a.c + c;
  float sum = 0.0f;
  if (c < a.c)
#pragma unroll 8
    for (int p = wave; p < a.n_parts; p += 4) sum += a.parts[p * rows * a.c + at];
  s_sum[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < a.c)
    a.dtable[(int64_t)blockIdx.x * a.c + c] = (s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane]);
}

bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T>
hipError_t launch_forward(RelativeArgs a, hipStream_t st) {
  constexpr int kVec = 16 / sizeof(T);
  const int64_t units = a.n_rows * ((a.n_tok + 63) / 64), total = (units + 3) / 4;
  const dim3 block(256);
  const int pieces = a.c / kVec;
  hipError_t e = hipSuccess;
  for (; a.first_block < total && e == hipSuccess; a.first_block += kLaunchBlocks) {
    const dim3 grid((unsigned)(total - a.first_block < kLaunchBlocks ? total - a.first_block : kLaunchBlocks));
    if (a.c % kVec || pieces > 64 || !at16(a.table) || !at16(a.z_in) || !at16(a.z_out))
      hipLaunchKernelGGL(relative_any_kernel<T>, grid, block, 0, st, a);
    else if (pieces > 32)
      hipLaunchKernelGGL((relative_kernel<T, 64>), grid, block, 0, st, a);
    else if (pieces > 16)
      hipLaunchKernelGGL((relative_kernel<T, 32>), grid, block, 0, st, a);
    else if (pieces > 8)
      hipLaunchKernelGGL((relative_kernel<T, 16>), grid, block, 0, st, a);
    else if (pieces > 4)
      hipLaunchKernelGGL((relative_kernel<T, 8>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((relative_kernel<T, 4>), grid, block, 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

int channel_sets(int32_t c) { return c > 64 ? 4 : c > 32 ? 2 : 1; }

template <typename T, bool VEC>
void launch_backward(const RelativeArgs& a, hipStream_t st) {
  const int cg = channel_sets(a.c);
  const dim3 grid((unsigned)a.n_groups, (unsigned)((a.c + 32 * cg - 1) / (32 * cg)), (unsigned)((a.n_tiles + kWindow - 1) / kWindow));
  if (cg == 4)
    hipLaunchKernelGGL((relative_back_kernel<T, 4, VEC>), grid, dim3(256), 0, st, a);
  else if (cg == 2)
    hipLaunchKernelGGL((relative_back_kernel<T, 2, VEC>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((relative_back_kernel<T, 1, VEC>), grid, dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_relative(const RelativeArgs& a, bool bf16, hipStream_t st) {
  return bf16 ? launch_forward<uint16_t>(a, st) : launch_forward<float>(a, st);
}

void relative_back_split(RelativeArgs* a) {
  // the workspace's size does not know the type: tiles of the larger of the two, as in bf16
  const int cg = channel_sets(a->c), s = 4 / cg, pairs = relative_own_pairs(true) * s;
  const int64_t tiles = a->n_rows * ((a->n_tok + pairs - 1) / pairs);
  const int64_t per = (int64_t)((a->c + 32 * cg - 1) / (32 * cg)) * ((a->n_tiles + kWindow - 1) / kWindow);
  int64_t most = 512 / per;  // two workgroups a CU
  if (most < 64) most = 64;
  const int64_t want = (tiles + 1) / 2;
  a->n_groups = (int32_t)(want < most ? want : most);
  a->n_parts = a->n_groups * s;
}

hipError_t launch_relative_back(const RelativeArgs& a, bool bf16, hipStream_t st) {
  if (a.n_groups > 0) {
    const bool vec = at16(a.dz) && a.c % (bf16 ? 8 : 4) == 0;
    if (bf16)
      vec ? launch_backward<uint16_t, true>(a, st) : launch_backward<uint16_t, false>(a, st);
    else
      vec ? launch_backward<float, true>(a, st) : launch_backward<float, false>(a, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(relative_sum_kernel, dim3((unsigned)a.n_buckets, (unsigned)((a.c + 63) / 64)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dcp
