// MXFP4 on gfx950: the layouts of the 4-bit matrices and cache, and what the kernels that read and write them share.
//
// A matrix is cut into records of 16 rows x 256 columns (8 k-tiles of 32): 2 KiB of codes and 128 bytes of scales.  Codes: two
// halves of 4 k-tiles, 16 bytes per lane (lane = g * 16 + row), word j of a lane the 8 codes of columns 8 g .. 8 g + 7 of k-tile j, the
// first in the lowest bits - an operand of v_mfma_f32_16x16x32_bf16 in lane order once it is converted, so a wave fetches four operands
// with one 16-byte load a lane.  Scales: 8 bytes per row, one per k-tile.
//
// The cache holds a record of 17 * head_dim bytes per (layer, block of 16 positions, kv head).  K codes: as above, word j of lane
// (g, token) features 32 j + 8 g .. + 7.  V codes: byte i of word j of lane (g, p) holds features 32 j + 2 p and + 1 of token 4 g + i.
// K scales: per token a byte per 32 features.  V scales: [g][32 features][4 tokens].
#pragma once
#include "../../include/llm42_mx4.h"
#include "llm42_dev.h"

namespace mx4 {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 256;                  // columns of a record
constexpr int kRecord = 2176;               // its bytes
constexpr int kScales = 2048;               // where its scales begin

__host__ __device__ inline int units_of(int cols) { return (cols + kUnit - 1) / kUnit; }
inline size_t matrix_bytes(int rows, int cols) { return (size_t)((rows + 15) / 16) * units_of(cols) * kRecord; }
__host__ __device__ constexpr int kv_record(int head_dim) { return 17 * head_dim; }

// The scale byte of a block by the largest of its magnitudes' bit patterns: a float's exponent less 2, none below 0; 255 where there is
// an infinity or a NaN (whose patterns are the largest).
__device__ inline uint32_t scale_byte(uint32_t top) {
  return top >= 0x7F800000u ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}

// 2^E of byte i of a word of scale bytes, as the conversions take it: of a float's bits they use the eight of the exponent alone, so
// what stands beside the byte does not matter (all 256 exponents and 256 pairs of codes compared).
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) { return __uint_as_float(i < 3 ? bytes << (23 - 8 * i) : bytes >> 1); }

// The hardware's conversions.  To 4 bits: nearest level, ties to the even index, saturating - the format's own rule, compared for every
// bf16 and 16 M floats, subnormal ones too, in blocks of up to 2^13 times their size.  From 4 bits: exact; NaN under byte 255.
// (Pair e of a word of 8: the builtins want a constant, which e is once unrolled.)
__device__ __forceinline__ uint32_t pair_bf16(uint32_t codes, float scale, int e) {
  return __builtin_bit_cast(uint32_t, e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)
                                      : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)
                                      : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}
__device__ __forceinline__ f32x2 pair_f32(uint32_t codes, float scale, int e) {
  return e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0)
         : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1)
         : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2)
                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
}
// 8 codes as bf16: an MFMA operand.
__device__ __forceinline__ bf16x8 operand(uint32_t codes, float scale) {
  u32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = pair_bf16(codes, scale, e);
  return __builtin_bit_cast(bf16x8, r);
}
// Codes of two bf16 in the bytes `e` of a word, the rest of which stays.
__device__ __forceinline__ uint32_t put_pair(uint32_t word, uint32_t two, float scale, int e) {
  const bf16x2 v = __builtin_bit_cast(bf16x2, two);
  return e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, v, scale, 0)
         : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, v, scale, 1)
         : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, v, scale, 2)
                  : __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, v, scale, 3);
}
__device__ __forceinline__ uint32_t put_pair(uint32_t word, float a, float b, float scale, int e) {
  return e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, scale, 0)
         : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, scale, 1)
         : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, scale, 2)
                  : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, scale, 3);
}
// The larger magnitudes of two pairs of bf16, half by half, and of a pair, as a float's bits.
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7FFF7FFFu), __builtin_bit_cast(u16x2, b & 0x7FFF7FFFu)));
}
__device__ __forceinline__ uint32_t larger_half(uint32_t a) { return max(a << 16 & 0x7FFF0000u, a & 0x7FFF0000u); }

}  // namespace mx4

// The 4-bit copy of a model's matrices.
struct llm42_mx4_model {
  const llm42_model* model;
  char* arena;
  struct Layer {
    char *wqkv, *wo, *wgu, *wdown;
  }* layers;
  char* lm_head;
};

constexpr int32_t kMostContext4 = 1 << 30;   // (positions and steps of keys past it stay within 32 bits)

// Attention over a 4-bit cache: who sees what, and how the work is split.
struct Attention4 {
  char* base;                  // the layer's records
  int64_t num_blocks;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_len;      // cached length before the window (tiles: -1 takes no part)
  const int32_t* seq_n;        // rows of the window that are there, or null: all
  int32_t* seq_status;         // or null
  int32_t* merge_n;            // [seq][kv head]: rows of a sequence that is in order, for the launch that joins its parts
  const uint16_t* q;           // rows of q_stride, or (tiles) the layout that the QKV projection leaves
  uint16_t* out;               // rows of out_stride, or (tiles) operand of the O-projection
  int64_t q_stride, out_stride;
  bool tiles;
  int num_seqs, n_kv_heads, group, head_dim, window, max_context;
  int num_cus;
  int splits, split_steps;     // parts of a sequence, steps of 64 keys in each
  float* part_acc;             // [seq][kv head][split][row][head_dim]
  float* part_ml;              // [seq][kv head][split][row][2]
  // tiles: the layer's K and V in the bf16 cache and a row's block there, from which the newest position is stored first
  const uint16_t *k_plane, *v_plane;
  const int32_t* row_blk;
};

void launch_mx4_quantize(const void* src, int type, int64_t stride, int rows, int cols, void* dst, hipStream_t st);
// src: a matrix in the tile layout of the bf16 GEMMs, rows a multiple of 16, cols of 32
void launch_mx4_quantize_tiles(const uint16_t* src, int rows, int cols, void* dst, hipStream_t st);
void launch_mx4_dequantize(const void* src, int rows, int cols, void* dst, int type, int64_t stride, hipStream_t st);
// x to the tile layout, columns padded with zeros to a multiple of 32
void launch_mx4_pack_x(const uint16_t* x, int64_t stride, int rows, int k, uint16_t* dst, hipStream_t st);

// HIP takes fewer than 2^32 threads along x: so many workgroups of 256.
constexpr unsigned kMostGroups256 = 0xFFFFFFFFu / 256;

// Up to this many rows of x are read as they lie if they are 4-byte aligned (loose).
int mx4_loose_rows();
// x: row-major (x_stride > 0; loose, or 16-byte aligned and k a multiple of 32) or tile layout (0).  parts:
// mx4_matmul_part_bytes bytes, or null: the sum is not split.
size_t mx4_matmul_part_bytes(int n, int k, int rows, int num_cus);
bool mx4_matmul_fits(int n, int k, int rows, bool loose, int num_cus, bool parts);   // ... what a launch takes
void launch_mx4_matmul(const void* w, int n, int k, const uint16_t* x, int64_t x_stride, bool loose, int rows, void* out, int out_type,
                       int64_t out_stride, int num_cus, float* parts, hipStream_t st);
void launch_mx4_qkv(const llm42_mx4_model* m4, int layer, const llm42_kv_cache* kv, const Workspace& ws, hipStream_t st);
// Most parts that a residual projection's sum is taken in, and the scratch that takes beside the workspace of the pass.
inline int mx4_residual_parts(int m_rows) { return m_rows <= 256 ? 8 : m_rows <= 1024 ? 4 : 1; }
inline size_t mx4_residual_bytes(int m_rows, int m_pad, int d_model) {
  return mx4_residual_parts(m_rows) > 1 ? 4ull * mx4_residual_parts(m_rows) * m_pad * d_model : 0;
}
// true: the residual stream is not complete yet; the halves are in split_part, for the RMSNorm that follows
bool launch_mx4_residual(const void* w, const uint16_t* x, int n, int k, float* parts, const Workspace& ws, hipStream_t st);
void launch_mx4_swiglu(const llm42_mx4_model* m4, int layer, const Workspace& ws, hipStream_t st);
int launch_mx4_logits(const llm42_mx4_model* m4, const llm42_sampling* sampling, const Workspace& ws, hipStream_t st);

void launch_kv4_store(const llm42_model* m, const llm42_kv_cache* kv, const llm42_kv_cache* kv4, const int32_t* first,
                      const int32_t* count, int num_seqs, int max_count, int32_t* seq_status, hipStream_t st);
void launch_kv4_read(const llm42_model* m, const llm42_kv_cache* kv4, const int32_t* first, const int32_t* count, int num_seqs,
                     int max_count, uint16_t* out_k, uint16_t* out_v, int32_t* seq_status, hipStream_t st);
// A decoding step's sequences against the 4-bit cache's own block table; those that fail are switched off as by launch_prepare.
void launch_kv4_step_check(const llm42_model* m, const llm42_kv_cache* kv4, int num_seqs, int32_t* seq_status,
                           const Workspace& ws, hipStream_t st);
void plan_kv4_attention(int num_seqs, int n_kv_heads, int rows, int max_context, int num_cus, int& splits, int& split_steps);
void launch_kv4_attention(const Attention4& a, hipStream_t st);
