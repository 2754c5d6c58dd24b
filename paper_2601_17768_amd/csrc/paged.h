// The operators around the paged bf16 cache (include/llm42_paged.h): argument blocks, launchers and what their kernels share.
//
// A call's rows are (sequence, token of its window); a layer's K and V planes are [block][kv head] tiles of 16 x head_dim: token t and feature f of K at
// ((f / 8) * 16 + t) * 8 + f % 8, of V at v_tile_off(f, t).
#pragma once
#include "../../include/llm42_paged.h"
#include "llm42_dev.h"

struct llm42_rope {
  int device, rot_dim, layout, max_position;
  float2* table;               // [position][pair] (cos, sin), each times the attention factor
};

constexpr int32_t kMostContextPaged = 1 << 30;   // (positions past it stay within 32 bits)

namespace paged {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ constexpr int bounds_record(int head_dim) { return 2 * head_dim + 16; }
constexpr int kBoundsBias = 64, kBoundsNone = 255, kLeastExponent = -40, kMostExponent = 40;

// What every call knows of its sequences.
struct Rows {
  const int32_t* block_table;
  int width;                   // of the table
  int64_t num_blocks;
  const int32_t* seq_len;
  const int32_t* seq_n;        // or null: window
  int num_seqs, window, max_context;
};

// Status of a sequence by its lengths alone.
__device__ inline int length_status(const Rows& r, int len, int n) {
  return len < 0 || n < 0 || n > r.window || (int64_t)len + n > r.max_context ? LLM42_SEQ_BAD_LENGTH : LLM42_SEQ_OK;
}

// The smallest e >= -40 with top <= 127 * 2^e, top a finite magnitude that is a bf16: 127 = 1.984375 * 2^6, and a larger significand of 8 bits is 255 / 128 alone.
__device__ inline int bounds_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - 6 + ((u >> 16 & 0x7F) == 0x7F ? 1 : 0);
  return max(e, kLeastExponent);
}
__device__ inline float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // (-126 .. 127)

__device__ inline float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The value of another lane of the same 16: l ^ 1, l ^ 2, the mirrored one of its 4, 8 or 16, l ^ 8.
template <int CTRL>
__device__ inline uint32_t other_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror4 = 0x1B, kMirror8 = 0x141, kMirror16 = 0x140, kXor8 = 0x128;
// f over the 16 lanes of a group.
template <class F>
__device__ inline float over_lanes(float x, F f) {
  x = f(x, __uint_as_float(other_lane<kXor1>(__float_as_uint(x))));
  x = f(x, __uint_as_float(other_lane<kXor2>(__float_as_uint(x))));
  x = f(x, __uint_as_float(other_lane<kMirror8>(__float_as_uint(x))));
  return f(x, __uint_as_float(other_lane<kMirror16>(__float_as_uint(x))));
}
// f over a value and the same lanes' of the other 16 of its 32, and of the other 32: for all of the wave's groups of 16 lanes alike.
template <class F>
__device__ inline float over_rows(float x, F f) {
  const u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(a.x), __uint_as_float(a.y));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(b.x), __uint_as_float(b.y));
}

// Writes the bounds of a block of keys, of which this lane has features 8 c .. 8 c + 7 (c = lane % (HD / 8)) of HD / 32 tokens: one maximum and minimum a feature over
// all tokens, the block's power of two, and both in whole multiples of it.  Exact throughout (bf16 keys, powers of two).
template <int HD>
__device__ inline void write_bounds(const u32x4 (&key)[HD / 32], char* rec, int lane) {
  constexpr int LANES = HD / 8, N = HD / 32;
  float mx[8], mn[8];
  bool bad = false;
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    mx[f] = -INFINITY;
    mn[f] = INFINITY;
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t x = key[t][w];
      bad |= (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
      mx[2 * w] = fmaxf(mx[2 * w], lo_bf16(x));
      mn[2 * w] = fminf(mn[2 * w], lo_bf16(x));
      mx[2 * w + 1] = fmaxf(mx[2 * w + 1], hi_bf16(x));
      mn[2 * w + 1] = fminf(mn[2 * w + 1], hi_bf16(x));
    }
  const auto larger = [](float a, float b) { return fmaxf(a, b); };
  const auto smaller = [](float a, float b) { return fminf(a, b); };
  float top = 0.f;
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    if constexpr (LANES == 8) {
      mx[f] = fmaxf(mx[f], __uint_as_float(other_lane<kXor8>(__float_as_uint(mx[f]))));
      mn[f] = fminf(mn[f], __uint_as_float(other_lane<kXor8>(__float_as_uint(mn[f]))));
    }
    mx[f] = over_rows(mx[f], larger);
    mn[f] = over_rows(mn[f], smaller);
    top = fmaxf(top, fmaxf(mx[f], -mn[f]));
  }
  const auto with = [&](uint32_t x) { top = fmaxf(top, __uint_as_float(x)); };
  with(other_lane<kXor1>(__float_as_uint(top)));
  with(other_lane<kXor2>(__float_as_uint(top)));
  with(other_lane<kMirror8>(__float_as_uint(top)));
  if constexpr (LANES == 16) with(other_lane<kMirror16>(__float_as_uint(top)));
  const int e = __any(bad) ? kMostExponent + 1 : bounds_exponent(top);
  const bool none = e > kMostExponent;
  const float unit = none ? 0.f : power_of_two(-e);
  uint32_t up[2] = {0, 0}, down[2] = {0, 0};
  if (!none) {
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      up[f >> 2] |= ((uint32_t)(int)ceilf(mx[f] * unit) & 255u) << (8 * (f & 3));
      down[f >> 2] |= ((uint32_t)(int)floorf(mn[f] * unit) & 255u) << (8 * (f & 3));
    }
  }
  if (lane < LANES) {
    *(u32x2*)(rec + 8 * lane) = (u32x2){up[0], up[1]};
    *(u32x2*)(rec + HD + 8 * lane) = (u32x2){down[0], down[1]};
    if (lane == 0) *(u32x4*)(rec + 2 * HD) = (u32x4){none ? kBoundsNone : (uint32_t)(e + kBoundsBias), 0, 0, 0};
  }
}

// Blocks that a run of `count` positions can touch, of those that a table names.
inline int slots_of(int count, int width) {
  const int64_t n = ((int64_t)count + 14) / 16 + 1;
  return (int)(n < width ? n : width);
}

struct Append {
  Rows rows;
  const void *q, *k, *v;       // q may be null
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const uint16_t *q_norm, *k_norm;
  float eps;
  const float2* rope;          // or null
  int rot_dim, layout;
  uint16_t *q_out, *k_plane, *v_plane;
  char* bounds;                // the layer's, or null
  int n_q_heads, n_kv_heads, head_dim, type;
  int32_t* seq_status;
};
struct Select {
  Rows rows;
  const char* bounds;          // the layer's
  const uint16_t* q;           // rows of q_stride, or (tiles) the layout that the QKV projection leaves
  int64_t q_stride;
  bool tiles;
  int n_kv_heads, group, head_dim;
  int budget, sink, recent;
  int32_t* selected;
  int32_t* seq_status;
  uint32_t* keys;              // workspace, or null: the scores stay in LDS
  int num_cus;
};
// Partials of a call whose lists are cut into parts.
struct SparseWorkspace {
  float *acc, *ml;
  int32_t* ok;
  size_t bytes;
};
SparseWorkspace carve_sparse(int rows, int n_kv_heads, int group, int head_dim, int parts, char* base);

struct SparseAttention {
  Rows rows;
  const uint16_t *k_plane, *v_plane;
  const uint16_t* q;
  uint16_t* out;               // rows of out_stride, or (tiles) operand of the O-projection
  int64_t q_stride, out_stride;
  bool tiles;
  int n_kv_heads, group, head_dim;
  const int32_t* selected;
  int width;                   // entries of a list
  int parts, per_part;         // workgroups of a list, and entries of each
  int num_cus;
  float scale;
  float *part_acc, *part_ml;   // [row][kv head][part][head][head_dim], [..][2]
  int32_t* part_ok;            // [row][kv head][part]
  int32_t* seq_status;
};

}  // namespace paged

void launch_rope_table(const double* freq, double factor, int pairs, int max_position, float2* table, hipStream_t st);
void launch_kv_append(const paged::Append& a, hipStream_t st);
// count null: max_count everywhere.
void launch_bounds_store(int n_layers, int n_kv_heads, int head_dim, const uint16_t* k_plane, int64_t layer_stride, char* bounds,
                         const int32_t* block_table, int width, int64_t num_blocks, const int32_t* first, const int32_t* count, int num_seqs,
                         int max_count, int32_t* seq_status, hipStream_t st);
void launch_bounds_read(int n_layers, int n_kv_heads, int head_dim, const char* bounds, int64_t num_blocks, const int32_t* ids, int num_ids,
                        uint16_t* out_lo, uint16_t* out_hi, hipStream_t st);
// Whether the scores of a call's blocks go through the workspace, and the bytes they take there.
size_t select_workspace(int num_seqs, int window, int n_kv_heads, int group, int max_context, int budget, int num_cus);
void launch_kv_select(const paged::Select& a, hipStream_t st);
void plan_sparse_attention(int rows, int n_kv_heads, int head_dim, int width, int num_cus, int& parts, int& per_part);
void launch_sparse_attention(const paged::SparseAttention& a, hipStream_t st);
