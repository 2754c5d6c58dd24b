// MXFP4 on gfx950: the layouts of the 4-bit matrices and cache, and what the kernels that read and write them share.
//
// A matrix is cut into records of 16 rows x 256 columns (8 k-tiles of 32): 2 KiB of codes and 128 bytes of scales.  Codes: two
// halves of 4 k-tiles, 16 bytes per lane (lane = g * 16 + row), word j of a lane the 8 codes of columns 8 g .. 8 g + 7 of k-tile j, the
// first in the lowest bits - an operand of v_mfma_f32_16x16x32_bf16 in lane order once it is converted, so a wave fetches four operands
// with one 16-byte load a lane.  Scales: 8 bytes per row, one per k-tile.
//
// The cache holds a record of 17 * head_dim bytes per (layer, block of 16 positions, kv head).  K codes: as above, word j of lane
// (g, token) features 32 j + 8 g .. + 7.  V codes: lane (g, f) has 2 bytes per block of 16 features, tokens 4 g .. 4 g + 3 of
// feature 16 b + f: the operand of P V.  K scales: per token a byte per 32 features.  V scales: [g][32 features][4 tokens].
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
// The code of x in a block of that byte: nearest level, ties to the even index.
__device__ inline uint32_t code_of(float x, uint32_t byte) {
  const float m = ldexpf(fabsf(x), 127 - (int)byte);           // exact wherever it matters
  const uint32_t c = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.0f);
  return byte == 255u ? 0u : c | (__float_as_uint(x) >> 31) << 3;
}
// What a code stands for in a block of scale 1, and 2^E.
__device__ inline float level(uint32_t code) {
  const uint32_t m = code & 7;
  const uint32_t bits = m >= 2 ? (m + 252) << 22 : m ? 0x3F000000u : 0u;
  return __uint_as_float(bits | (code & 8) << 28);
}
__device__ inline float value_of(uint32_t code, uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(level(code), (int)byte - 127);
}

// 8 codes to an MFMA operand, times `scale` (its exponent bits are what counts).
__device__ __forceinline__ bf16x8 operand(uint32_t codes, float scale) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_;
  u32x4_ r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}
// 2^E of byte i of a word of scale bytes, as the conversion takes it.
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) { return __uint_as_float((bytes >> (8 * i) & 255u) << 23); }

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

// Attention over a 4-bit cache: who sees what, and how the work is split.
struct Attention4 {
  const char* base;            // the layer's records
  int64_t num_blocks;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_len;      // cached length before the window; -1: takes no part
  const int32_t* seq_n;        // rows of the window that are there, or null: all
  const uint16_t* q;           // rows of q_stride, or (tiles) the layout that the QKV projection leaves
  uint16_t* out;               // rows of out_stride, or (tiles) operand of the O-projection
  int64_t q_stride, out_stride;
  bool tiles;
  int num_seqs, n_kv_heads, group, head_dim, window;
  int splits, split_steps;     // parts of a sequence, steps of 64 keys in each
  float* part_acc;             // [seq][kv head][split][row][head_dim]
  float* part_ml;              // [seq][kv head][split][row][2]
};

void launch_mx4_quantize(const void* src, int type, int64_t stride, int rows, int cols, void* dst, hipStream_t st);
// src: a matrix in the tile layout of the bf16 GEMMs, rows a multiple of 16, cols of 32
void launch_mx4_quantize_tiles(const uint16_t* src, int rows, int cols, void* dst, hipStream_t st);
void launch_mx4_dequantize(const void* src, int rows, int cols, void* dst, int type, int64_t stride, hipStream_t st);
// x to the tile layout, columns padded with zeros to a multiple of 32
void launch_mx4_pack_x(const uint16_t* x, int64_t stride, int rows, int k, uint16_t* dst, hipStream_t st);

// x: row-major (x_stride > 0; k a multiple of 32) or tile layout (0).  parts: mx4_matmul_part_bytes bytes, or null: the sum is not split.
size_t mx4_matmul_part_bytes(int n, int k, int rows, int num_cus);
void launch_mx4_matmul(const void* w, int n, int k, const uint16_t* x, int64_t x_stride, int rows, void* out, int out_type,
                       int64_t out_stride, int num_cus, float* parts, hipStream_t st);
void launch_mx4_qkv(const llm42_mx4_model* m4, int layer, const llm42_kv_cache* kv, const Workspace& ws, hipStream_t st);
// true: the residual stream is not complete yet; the halves are in split_part, for the RMSNorm that follows
bool launch_mx4_residual(const void* w, const uint16_t* x, int n, int k, const Workspace& ws, hipStream_t st);
void launch_mx4_swiglu(const llm42_mx4_model* m4, int layer, const Workspace& ws, hipStream_t st);
int launch_mx4_logits(const llm42_mx4_model* m4, const llm42_sampling* sampling, const Workspace& ws, hipStream_t st);

// count null: 1 each, of sequences whose `first` is not negative.  layer < 0: all.
void launch_kv4_store(const llm42_model* m, int layer, const llm42_kv_cache* kv, const llm42_kv_cache* kv4, const int32_t* first,
                      const int32_t* count, int num_seqs, int max_count, int32_t* seq_status, hipStream_t st);
void launch_kv4_read(const llm42_model* m, const llm42_kv_cache* kv4, const int32_t* first, const int32_t* count, int num_seqs,
                     int max_count, uint16_t* out_k, uint16_t* out_v, int32_t* seq_status, hipStream_t st);
// A decoding step's sequences against the 4-bit cache's own block table; those that fail are switched off as by launch_prepare.
void launch_kv4_step_check(const llm42_model* m, const llm42_kv_cache* kv4, int num_seqs, int32_t* seq_status,
                           const Workspace& ws, hipStream_t st);
void launch_kv4_attention_check(const int32_t* seq_lens, const int32_t* n_valid, int window, int max_context, int num_seqs,
                                const llm42_kv_cache* kv4, int32_t* seq_status, int32_t* ws_len, int32_t* ws_n, hipStream_t st);
void plan_kv4_attention(int num_seqs, int n_kv_heads, int rows, int max_context, int num_cus, int& splits, int& split_steps);
void launch_kv4_attention(const Attention4& a, hipStream_t st);
