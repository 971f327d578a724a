// Internal launch interface between the C-ABI layer (dcp_api.hip) and the
// kernels. Not installed; the public interface is include/dcp.h.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cdna4.h"

namespace dcp {

// Shape of the fused MFMA path.
constexpr int kFastCz = 128;   // pair channels
constexpr int kFastH = 16;     // heads
constexpr int kFastD = 24;     // head dim
// Logits of the fused path are in base-2 units plus this offset inside the
// kernel (exact power-of-two rescaling); its partial maxima are written
// without it
constexpr float kFastShift = 192.0f;
constexpr int kFastDp = 32;    // head dim padded to the MFMA k width
constexpr int kTileQ = 16;     // query rows per workgroup of the fused attention, and per projection tile
constexpr int kTileK = 16;     // keys per tile
// 16 rows of z must be addressable with 31-bit byte offsets: 16 * N * 256 < 2^31
constexpr int64_t kFastMaxTokens = 500000;

// Limits of the general fp32 path.
constexpr int kGenMaxCz = 256;
constexpr int kGenMaxH = 16;
constexpr int kGenMaxHD = 128;
constexpr int kGenMaxD = 64;
constexpr int kMaxCs = 4096;

// The paper's chunk rule (Appendix "Chunk distribution algorithm"): part p of
// `total` items over `parts` parts has floor(total/parts) items, plus one when
// p < total mod parts, and starts at p*floor(total/parts) + min(p, total mod parts).
__host__ __device__ inline void chunk_of(int64_t total, int64_t parts, int64_t p, int64_t* size, int64_t* start) {
  const int64_t q = total / parts, r = total % parts;
  *size = q + (p < r ? 1 : 0);
  *start = p * q + (p < r ? p : r);
}
// The same where the counts fit 32 bits: 64-bit divisions at the start of short kernels took
// 0.5 us of the 34.5 of a backward pass of 128 tokens.
__device__ inline void chunk_of_32(uint32_t total, uint32_t parts, uint32_t p, int64_t* size, int64_t* start) {
  const uint32_t q = total / parts, r = total % parts;
  *size = q + (p < r ? 1 : 0);
  *start = (int64_t)p * q + (p < r ? p : r);
}

// |x|, and 0 where x is not finite.
__device__ inline float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }

struct FastProjArgs {
  const uint16_t* s;  // [N, c_s] bf16
  const float *w_q, *w_k, *w_v, *w_g;
  const uint8_t* mask;  // [N] or null
  int64_t n_tok, q_row0, n_q, nq_pad, n_pad;
  int64_t key_tile0, key_tiles;  // k, vt and tile_valid are written for these 16-key tiles
  int32_t c_s;
  uint16_t* q;   // [H][nq_pad][32] bf16, scaled by log2(e)/sqrt(d)
  uint16_t* k;   // [H][n_pad][32] bf16
  uint16_t* vt;  // [H][n_pad/16][64][2][4] bf16: V^T tiles (lane, M-tile) with a row of ones at e = 24
  float* g;      // [n_q][H*d] fp32, sigmoid applied
  uint32_t* tile_valid;  // [n_pad/16]: bit i = key 16t+i exists and is not masked
  void* w_split;         // fast_proj_split_bytes(c_s): the weights as bf16 hi + lo matrix-core operands
};

struct FastAttnArgs {
  const uint16_t* z;  // [n_q][N][128] bf16
  const uint8_t* mask;
  const float *w_b, *gamma;
  const uint16_t *q, *k, *vt;
  const uint32_t* tile_valid;
  int64_t n_tok, n_q, nq_pad, n_pad;
  int64_t k_lo, k_len;  // keys [k_lo, k_lo + k_len), split into n_parts parts of whole 16-key tiles
  int32_t n_parts;
  float eps;
  float *m_parts, *l_parts, *acc_parts;  // [P][H][n_q], [P][H][n_q], [P][n_q][H][d]
};

struct FastBiasArgs {
  const uint16_t* z;
  const float *w_b, *b_b, *gamma, *beta;
  int64_t n_rows, n_cols, row_stride;
  int32_t cols_per_wave;
  float eps;
  float* out;  // [n_rows][n_cols][16]
};

struct GenProjArgs {
  const void* s;
  int32_t s_bf16;
  const float *w_q, *w_k, *w_v, *w_g;
  int64_t n_tok, q_row0, n_q;
  int32_t c_s, hd;
  float *q, *k, *v, *g;  // q, g: [n_q][hd]; k, v: [N][hd]; g holds the sigmoid (16-byte aligned, or null: not wanted)
  const uint8_t* mask;   // [N] or null: v of masked keys is written as 0
  int32_t kv_head_dim;   // k, v in the tiled attention's layout, with this head size; 0: row-major [N][hd]
  int32_t s_vec;         // set by the launcher: rows of s take 4-element loads
};

struct GenAttnArgs {
  const void* z;
  int32_t z_bf16;
  const uint8_t* mask;
  const float *w_b, *gamma;
  const float *q, *k, *v;
  int64_t n_tok, n_q;
  int64_t k_lo, k_len;  // keys [k_lo, k_lo + k_len), split into n_parts parts
  int32_t c_z, n_heads, head_dim, n_parts;
  float eps;
  float *m_parts, *l_parts, *acc_parts;
  const float* g;       // with out: the gate [n_q][hd]
  void* out;            // n_parts = 1: the gated, normalised output in place of the partial state; else null
  int32_t out_bf16;
};

struct GenBiasArgs {
  const void* z;
  int32_t z_bf16;
  const float *w_b, *b_b, *gamma, *beta;
  int64_t n_rows, n_cols, row_stride;
  int32_t c_z, n_heads;
  float eps;
  float* out;
};

struct MergeArgs {
  int32_t n_parts, n_heads, head_dim;
  int64_t n_rows;
  const float *m, *l, *acc, *gate;
  float *m_out, *l_out, *acc_out;
  void* out;
  int32_t out_bf16;
  int32_t log2_units;  // 1: m is in base-2 units with integer differences (the fused path)
  int32_t m_natural;   // with log2_units: write m_out in natural-log units
};

// Sparse (kNN) atom attention: the paper's atom-attention shape (4 heads of
// 32, 16 pair channels), up to 256 neighbour slots per query.
constexpr int kSparseH = 4;
constexpr int kSparseD = 32;
constexpr int kSparseCap = 16;
constexpr int kSparseMaxK = 256;
// Neighbour indices are packed with their slot number into 32 bits (24 + 8),
// and an fp32 K or V array of this many atoms stays below 2^31 bytes.
constexpr int64_t kSparseMaxAtoms = 4000000;

struct SparseProjArgs {
  const uint16_t* a;  // [L, c_atom] bf16
  const float *w_q, *w_k, *w_v, *w_g;
  int64_t n_atoms, q_row0, n_q;
  int32_t c_atom;
  float *q, *g;       // [n_q][128] fp32 (g after the sigmoid)
  uint16_t *k, *v;    // [L][128] bf16
};

struct SparseAttnArgs {
  const void* p;          // pair rows of the query stripe (dense [n_q][L][16] or gathered [n_q][k][16])
  const int32_t* nbr;     // [n_q][k]
  const float *w_b, *gamma;
  const float *q, *g;     // [n_q][128] fp32
  const void *k, *v;      // [L][128] in the activation dtype
  int64_t n_atoms, n_q;
  int64_t p_row_elems;    // elements per query row of p
  int32_t k_slots, n_kb, p_gathered, out_bf16;
  float eps;
  void* out;              // [n_q][128]
};

// k nearest neighbours: up to 256 per query; candidate indices fit in int32.
constexpr int kKnnMaxK = 256;

struct KnnArgs {
  const float* x_q;       // [n_q][3]
  const float* x_c;       // [n_c][3]
  const int32_t *group_q, *group_c;
  int64_t n_q, n_c, c_index0, q_self0;
  int32_t k, group_mode;
  int32_t* idx_out;       // [n_q][k]
  float* d2_out;          // [n_q][k] or null
  void *cand, *box;       // workspace: [n_c] float4 candidates, [ceil(n_c / 128)][2] float4 boxes
};

struct TopkMergeArgs {
  int64_t n_rows;
  int32_t k;
  const int32_t *idx_a, *idx_b;
  const float *d2_a, *d2_b;
  int32_t* idx_out;
  float* d2_out;
};

// Pair transition: the matrix-core path serves c_z = 128 with a 4x expansion;
// the fp32 path c_z <= 256 and hidden <= 1024.
constexpr int kTransCz = 128;
constexpr int kTransHidden = 512;
constexpr int kTransGenMaxHidden = 1024;

struct TransArgs {
  int64_t n_pairs;
  const float *w1, *w2, *w3, *gamma, *beta;
  const void* z_in;    // [n_pairs][128] bf16
  void* z_out;         // may equal z_in
  void* w_prep;        // operand tiles (trans_prep_bytes(): tiles, then gamma and beta)
  float* gb_prep;      // [2][128] gamma, beta inside w_prep
  float eps;
};

struct TransGenArgs {
  int64_t n_pairs;
  int32_t c_z, hidden;
  const float *w1, *w2, *w3, *gamma, *beta;
  const float* z_in;
  float* z_out;        // may equal z_in
  float eps;
};

size_t trans_prep_bytes();

// Atom -> token mean: up to 512 channels.
constexpr int kScatterMaxC = 512;
constexpr int kScatterFlags = 256;  // most order-check flags of one pooling call

struct ScatterArgs {
  int64_t n_atoms, n_tokens;
  int32_t c, a_bf16, out_bf16;
  const void* a;          // [n_atoms][c]
  const int32_t* tok_idx; // [n_atoms]
  int64_t* acc;           // [n_tokens][c] fixed-point sums (workspace)
  uint32_t* cnt;          // [n_tokens] (workspace)
  void* out;              // [n_tokens][c]
  int32_t* flags;         // [kScatterFlags] order-check flags (workspace); NULL: general path only
  int32_t n_flags;        // flags written by this call (set by the launcher)
  int64_t* plan;          // [n_tokens][2] first atom and one past the last of each token (workspace)
};

// LayerNorm over rows of up to 4096 channels.
constexpr int kLnMaxC = 4096;

struct LayerNormArgs {
  int64_t n_rows;
  int32_t c;
  const void* x;               // [n_rows][c]
  const float *gamma, *beta;   // [c] or null
  void* y;                     // [n_rows][c], may be x
  float eps;
  int32_t lanes;               // set by the launcher: lanes that share a row
};

struct LayerNormBackArgs {
  int64_t n_rows;
  int32_t c;
  const void *x, *dy;          // [n_rows][c]
  const float* gamma;          // [c] or null
  void* dx;                    // [n_rows][c] in x's type, or null
  float *dgamma, *dbeta;       // [c] or null
  float* parts;                // [layer_norm_back_groups()][2][c] (workspace); null: no weights' gradient wanted
  float eps;
  int32_t lanes;               // as above
};

// Backward pass of the attention (backward.hip). Rows are those of the stripe;
// [H][n_q][dp] holds a head's channels padded with zeros to dp.
constexpr int kBackMaxGroups = 512;  // workgroups (one T each) of the general pair kernel: two fit a CU

constexpr int kBackKeys = 64;        // its keys per tile
__host__ __device__ constexpr int64_t back_keys_padded(int64_t n_tok) { return (n_tok + kBackKeys - 1) / kBackKeys * kBackKeys; }
__host__ __device__ constexpr int back_heads_padded(int n_heads) { return n_heads <= 4 ? 4 : n_heads <= 8 ? 8 : 16; }

struct BackRowsArgs {
  int64_t n_q;
  int32_t n_heads, head_dim, dp, dout_bf16;
  const float *m, *l;      // [H][n_q]
  const float *acc, *g, *q;  // [n_q][hd]
  const void* dout;        // [n_q][hd]
  float *qp, *dop;         // [H][n_q][dp]
  float* stat;             // [H][n_q][4]: m, 1 / L, D, -
  float* dg;               // [n_q][hd]
  int64_t n_tok;
  const uint8_t* mask;     // [N] or null
  const float *k, *v;      // [N][hd]
  float* kr;               // [H][N][dp], zeros for masked keys
  float *kp, *vp;          // in the order of the pair kernel's lanes, back_heads_padded x back_keys_padded x dp
  uint32_t row_blocks;     // set by the launcher
};

struct BackPairsArgs {
  const void* z;           // [n_q][N][c_z]
  int32_t z_bf16;
  const uint8_t* mask;     // [N] or null
  const float *w_b, *gamma;
  const float *k, *v;      // as BackRowsArgs::kp, vp
  const float *qp, *dop, *stat;
  int64_t n_tok, n_q, row0, rows;  // rows [row0, row0 + rows) of the stripe
  int32_t c_z, n_heads, head_dim, dp, first;
  float eps;
  float *p, *ds;           // [H][rows][N]
  void* dz;                // as z, or null
  float* t_parts;          // [groups][H][c_z]
};

struct BackKeysArgs {
  const float *p, *ds, *qp, *dop, *k;  // k [H][N][dp]
  int64_t n_tok, n_q, row0, rows;
  int32_t n_heads, head_dim, n_splits, first;
  float* kv_parts;         // [n_splits][2][N][hd]
  float* dq;               // [n_q][hd]
  uint32_t key_blocks;     // set by the launcher
};

// The fused shape (backward_fast.hip). fp16 operands: *f [H][tokens][32], *t
// [H][tokens / 16][64][2][4].
constexpr int kBackTops = 64;  // one wave's lanes
struct FastBackArgs {
  const uint16_t* z;       // [n_q][N][128] bf16
  const uint8_t* mask;     // [N] or null
  const float *w_b, *gamma;
  const float *q, *g, *k, *v;  // [n_q][384], [N][384] fp32
  const float *l, *acc;
  const void* dout;
  int32_t dout_bf16;
  int64_t n_tok, n_q, nq_pad, n_pad;
  uint32_t* tops;          // [4][kBackTops]: largest |q|, |k|, |v|, |dout| of shares of each (bits of floats)
  int32_t* exps;           // [5]: the powers of two of q, k, v, do and W''
  u32x4* w_ops;            // [768]: bias weights, W''
  uint16_t *qf, *qt, *of, *ot, *kf, *kt, *vf;
  int32_t stat_parts;
  float* stats;            // [stat_parts][3][H][nq_pad]: M, L and sum P dP of a part of the keys
  float* dot;              // [H][nq_pad]: D
  int32_t* row_exp;        // [nq_pad]: the power of two of each row's do
  float* row_scale;        // [nq_pad]: from there to the tensor's
  const float* w[4];       // W_q, W_k, W_v, W_g [384][c_s]
  int32_t c_s;
  uint16_t *w_split, *dg;  // [2][4][384][c_s], [2][n_q][384]: bf16 hi, then lo
  uint32_t* tile_valid;    // [n_pad / 16]
  float eps;
  // per chunk of rows
  int64_t row0, rows, chunk_pad;  // row0 and chunk_pad multiples of 16
  int32_t n_parts, kv_splits, first;
  u32x2* p;                // [H][chunk_pad / 16][n_pad / 16][64]: P of 16 rows by 16 keys
  uint16_t* dz;            // as z, or null
  float* dq_parts;         // [n_parts][n_q][384]
  float* t_parts;          // [n_parts * row tiles][16][128]
  float* kv_parts;         // [kv_splits][2][N][384]
};

struct BackSumArgs {
  int64_t n_tok, n_q;
  int32_t hd, dq_n, kv_n, t_n, t_cols;
  const float *dq_parts, *kv_parts, *t_parts;  // dq_parts null: dq is there already
  float *dq, *dkv, *t;     // [n_q][hd], [2][N][hd], [H][c_z]
  int32_t split;           // dq and dkv in bf16, hi then lo, in the same room (hd a multiple of four)
  uint32_t token_blocks;   // set by the launcher
};

struct BackGemmArgs {
  int64_t n_tok, q_row0, n_q;
  int32_t hd, c_s, s_bf16;
  const void* s;
  const uint8_t* mask;
  const float *w_q, *w_k, *w_v, *w_g;
  const float *dq, *dk, *dv, *dg;
  int32_t ds_splits, w_splits;
  float *ds_parts, *w_parts;  // [splits][N][c_s], [splits][4][hd][c_s]; null: not wanted
  int64_t ds_blocks;          // set by the launcher, with the next
  int32_t w_vec;
};

// Token products of the fused shape (token_gemm.hip). Split operands: bf16 hi, then lo.
struct TokenArgs {
  int64_t n_tok, q_row0, n_q;
  int32_t c_s;
  const uint16_t* s;       // [N][c_s] bf16
  const uint8_t* mask;
  const uint16_t* w;       // [2][4][384][c_s]: W_q, W_k, W_v, W_g
  float *q, *k, *v, *g;    // [n_q][384] (q, g), [N][384]
  uint32_t* tops;          // [3][kBackTops]: largest |q|, |k|, |v| of shares of each (cleared before)
  const uint16_t *dq, *dg, *dkv;  // [2][n_q][384] twice, [2][2][N][384]
  int32_t ds_splits, w_splits;
  float *ds_parts, *w_parts;      // as in BackGemmArgs
  int64_t ds_blocks;              // set by the launcher
};

struct BackFinishArgs {
  int64_t n_tok;
  int32_t n_heads, hd, c_s, c_z, bf16, ds_splits, w_splits;
  const float *ds_parts, *w_parts, *t, *w_b, *gamma;
  void *ds, *dw[4], *dw_b, *dgamma;  // null: not wanted
  uint32_t sum_blocks;               // set by the launcher
};

// Backward pass of the pair transition
struct TransBackArgs {
  int64_t n_pairs;
  int32_t c, hidden;
  float eps;
  const float *w1, *w2, *w3, *gamma, *beta;  // gamma, beta or null
  const void *z, *dout;      // [n_pairs][c]; z as codes where exponents is not null
  const uint8_t* exponents;  // [n_pairs][checkpoint_blocks(c)] or null
  void* dz;                  // or null, as all gradients
  void *dw1, *dw2, *dw3, *dgamma, *dbeta;
  int32_t grads_bf16;
  int32_t z_vec, d_vec;      // fp32: rows of z, of dout and dz in whole aligned groups of four channels
  int64_t first_block;       // fp32, of a launch for dz
  int32_t splits;            // shares of the pairs that are summed on their own
  float* prep;               // weights as operands
  float* parts;              // [splits]: T1, T2, T3 [hp][cp], S1, S2 [hp] (hidden and c filled up to 16)
  // Powers of two in the parts, or null: with e1, e2, e3 [hidden] and the exponent of dout d, T1 and S1 carry
  // 2^(e2 + e3 + d), T2 and S2 2^(e1 + e3 + d), T3 2^(e1 + e2 + d)
  const int *unit_exponents, *dout_exponent;
  float* affine_parts;       // [hidden][2][c]
  float *factors, *factor_logs;  // bf16: the inverse of what takes each pair's dout to the power of two of all, and its logarithm
  char* zh;                  // bf16: zh and dout, 512 B a pair; set by the launcher: whether dz's kernel writes them,
  int32_t store_zh, add_parts;  // whether the sums are added to the parts
};

// Blocks of 256 threads in one launch: a launch holds fewer than 2^32 threads. Kernels with a grid of the data's size take
// their first block as an argument.
constexpr int64_t kLaunchBlocks = (int64_t)1 << 23;

struct CheckpointArgs {
  int64_t n_rows, first_block;
  int32_t c;
  const void* x;  // to be packed, or null
  void* y;        // where to unpack, or null
  int8_t* codes;  // [n_rows][c]
  uint8_t* exponents;
};

constexpr int kRelativeFields = 4;
constexpr int kRelativeMaxRadius = 127;  // a bucket fits a byte
constexpr int kRelativeMaxC = 1024;
struct RelativeArgs {
  int64_t n_tok, row0, n_rows, first_block;  // first_block: of a launch of the encoding
  int32_t c, n_fields, n_buckets;
  const int32_t* position[kRelativeFields];  // [n_tok]
  const int32_t* group[kRelativeFields];     // [n_tok] or null
  int32_t radius[kRelativeFields], first[kRelativeFields];
  const float* table;  // [n_buckets][c]
  const void* z_in;    // or null
  void* z_out;
  const void* dz;
  float* dtable;
  // The gradient's buckets in tiles of 16, each of one field: the field, and the tile's place in it
  uint8_t tile_field[kRelativeFields * 16], tile_of_field[kRelativeFields * 16];
  int32_t n_tiles;
  float* parts;  // [n_parts][16 n_tiles][c]
  int32_t n_groups, n_parts;  // workgroups over the pairs, and sums of their own
};

size_t fast_proj_split_bytes(int32_t c_s);
bool fast_proj_small(int64_t key_tiles, int64_t query_tiles);  // one kernel, w_split unused
hipError_t launch_fast_proj(const FastProjArgs& a, hipStream_t st);
hipError_t launch_fast_attn(const FastAttnArgs& a, hipStream_t st);
hipError_t launch_fast_bias(const FastBiasArgs& a, hipStream_t st);
hipError_t launch_gen_proj(const GenProjArgs& a, hipStream_t st);
bool gen_attn_tiled(int64_t n_tok, int32_t c_z, int32_t n_heads, int32_t head_dim);
hipError_t launch_gen_attn(const GenAttnArgs& a, hipStream_t st);
hipError_t launch_gen_bias(const GenBiasArgs& a, hipStream_t st);
hipError_t launch_merge(const MergeArgs& a, hipStream_t st);
hipError_t launch_sparse_proj(const SparseProjArgs& a, hipStream_t st);
hipError_t launch_sparse_attn(const SparseAttnArgs& a, bool bf16, hipStream_t st);
size_t knn_workspace_bytes(int64_t n_c, size_t* box_offset);
hipError_t launch_knn(const KnnArgs& a, hipStream_t st);
hipError_t launch_topk_merge(const TopkMergeArgs& a, hipStream_t st);
hipError_t launch_transition(const TransArgs& a, hipStream_t st);
hipError_t launch_transition_gen(const TransGenArgs& a, hipStream_t st);
hipError_t launch_scatter_mean(const ScatterArgs& a, hipStream_t st);
hipError_t launch_layer_norm(const LayerNormArgs& a, bool x_bf16, bool y_bf16, hipStream_t st);
int layer_norm_back_groups(int64_t n_rows, int32_t c);  // workgroups, one partial sum each
hipError_t launch_layer_norm_back(const LayerNormBackArgs& a, bool x_bf16, bool dy_bf16, hipStream_t st);
hipError_t launch_back_rows(const BackRowsArgs& a, hipStream_t st);
int back_pairs_groups(int64_t rows, int64_t n_tok);
hipError_t launch_back_pairs(const BackPairsArgs& a, int groups, hipStream_t st);
hipError_t launch_back_keys(const BackKeysArgs& a, int dp, hipStream_t st);
hipError_t launch_fast_back_prep(const FastBackArgs& a, hipStream_t st);
hipError_t launch_fast_back_pack(const FastBackArgs& a, hipStream_t st);
hipError_t launch_fast_back_stats(const FastBackArgs& a, hipStream_t st);
hipError_t launch_fast_back_pairs(const FastBackArgs& a, hipStream_t st);
hipError_t launch_fast_back_keys(const FastBackArgs& a, hipStream_t st);
hipError_t launch_back_sum(const BackSumArgs& a, hipStream_t st);
void back_gemm_splits(int64_t n_tok, int32_t hd, int32_t c_s, int32_t step, int* ds_splits, int* w_splits);
hipError_t launch_back_gemm(const BackGemmArgs& a, hipStream_t st);
hipError_t launch_token_proj(const TokenArgs& a, hipStream_t st);
hipError_t launch_token_grad(const TokenArgs& a, hipStream_t st);
hipError_t launch_back_finish(const BackFinishArgs& a, hipStream_t st);
int trans_back_gen_splits(int64_t n_pairs, int32_t c, int32_t hidden);
hipError_t launch_trans_back_gen(const TransBackArgs& a, hipStream_t st);
size_t trans_back_fast_prep_bytes();
void trans_back_fast_units(const float* prep, const int** unit_exponents, const int** dout_exponent);
int trans_back_fast_splits(int64_t n_pairs);
size_t trans_back_fast_zh_bytes(int64_t n_pairs);
hipError_t launch_trans_back_fast(const TransBackArgs& a, hipStream_t st);
hipError_t launch_trans_back_finish(const TransBackArgs& a, hipStream_t st);
hipError_t launch_checkpoint(const CheckpointArgs& a, bool bf16, hipStream_t st);
hipError_t launch_relative(const RelativeArgs& a, bool bf16, hipStream_t st);
void relative_back_split(RelativeArgs* a);  // sets n_groups and n_parts
hipError_t launch_relative_back(const RelativeArgs& a, bool bf16, hipStream_t st);
int scatter_order_flags(int64_t n_atoms);  // plan workgroups (one flag each) for n_atoms (<= kScatterFlags)

}  // namespace dcp
