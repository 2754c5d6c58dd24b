// New tokens' rows into the paged cache: head norms, rotation, Q beside it; and the rotary table.
#include <algorithm>
#include <type_traits>

#include "paged.h"

using namespace paged;

namespace {

// One thread per (position, pair): the angle and its functions in 64 bits.
__global__ __launch_bounds__(256) void rope_table_kernel(const double* __restrict__ freq, double factor, int pairs, int64_t all,
                                                         float2* __restrict__ table) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= all) return;
  double s, c;
  sincos((double)(at / pairs) * freq[at % pairs], &s, &c);
  table[at] = make_float2((float)(c * factor), (float)(s * factor));
}

template <typename T>
__device__ inline void load8(float (&x)[8], const T* p) {
  if constexpr (std::is_same_v<T, float>) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  } else {
    const u32x4 w = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = lo_bf16(w[i]);
      x[2 * i + 1] = hi_bf16(w[i]);
    }
  }
}

__device__ inline u32x4 pack8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(x[2 * i], x[2 * i + 1]);
  return w;
}

// A head of HD features in HD / 8 lanes, features 8 c .. 8 c + 7 in lane c of them: its norm and its rotation, fp32.  `room`: 512 floats of
// LDS that are this wave's own; every lane of the wave takes part.  The partner of a feature may be in any lane and at any place there (rot_dim / 2 is any
// number), so a head goes through LDS once, element e of lane l at e * 64 + l: all lanes of a half look at one e at a time, no bank conflicts.
template <int HD>
__device__ inline void norm_and_rotate(float (&x)[8], const uint16_t* gain, float eps, const float2* rope, int pos, int rot_dim, int layout,
                                       float* room, int lane) {
  constexpr int LANES = HD / 8;
  const int c = lane % LANES, base = lane - c;
  if (gain) {
    float sum = 0.f;
#pragma unroll
    for (int f = 0; f < 8; ++f) sum = fmaf(x[f], x[f], sum);
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
    const float r = 1.0f / sqrtf(sum / HD + eps);
    float g[8];
    load8(g, gain + c * 8);
#pragma unroll
    for (int f = 0; f < 8; ++f) x[f] = x[f] * r * g[f];
  }
  if (!rope) return;
  const int half = rot_dim / 2;
  const float2* cs = rope + (size_t)pos * half;
  if (layout == LLM42_ROPE_INTERLEAVED) {
#pragma unroll
    for (int f = 0; f < 8; f += 2) {
      const int j = c * 4 + f / 2;
      if (j >= half) break;
      const float2 t = cs[j];
      const float a = x[f], b = x[f + 1];
      x[f] = a * t.x - b * t.y;
      x[f + 1] = b * t.x + a * t.y;
    }
    return;
  }
#pragma unroll
  for (int f = 0; f < 8; ++f) room[f * 64 + lane] = x[f];
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    const int at = c * 8 + f;
    if (at >= rot_dim) break;
    const bool first = at < half;
    const int other = first ? at + half : at - half;
    const float2 t = cs[first ? at : other];
    const float y = room[(other & 7) * 64 + base + (other >> 3)];
    x[f] = first ? x[f] * t.x - y * t.y : x[f] * t.x + y * t.y;
  }
  __builtin_amdgcn_wave_barrier();
}

// Status of a sequence, asked by the `lanes` neighbouring lanes that work for one row or block of it (all lanes of the wave ask together).
__device__ inline int sequence_status(const Rows& r, int s, int len, int n, int lane, int lanes) {
  int status = length_status(r, len, n);
  bool bad = false;
  if (status == LLM42_SEQ_OK && n > 0)
    for (int b = len / LLM42_KV_BLOCK + lane % lanes; b <= (len + n - 1) / LLM42_KV_BLOCK; b += lanes) {
      const int id = r.block_table[(size_t)s * r.width + b];
      bad |= id < 0 || id >= r.num_blocks;
    }
  const uint64_t mine = (lanes == 64 ? ~0ull : ((1ull << lanes) - 1)) << (lane - lane % lanes);
  if (__ballot(bad) & mine) status = LLM42_SEQ_BAD_BLOCK;
  return status;
}

// The launch's first workgroups take a (sequence, block, kv head) of K or of V per wave, the others a (row, head) of Q per HD / 8 lanes.
template <int HD, typename T>
__global__ __launch_bounds__(256) void append_kernel(Append a, int slots, unsigned kv_groups) {
  constexpr int LANES = HD / 8, UNITS = 64 / LANES, N = HD / 32, PAD = HD + 4;
  __shared__ float room[4][512];
  __shared__ __align__(16) uint16_t values[4][16 * PAD];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % LANES, unit = lane / LANES;
  const Rows& r = a.rows;
  if (blockIdx.x >= kv_groups) {
    const int64_t all = (int64_t)r.num_seqs * r.window * a.n_q_heads;
    const int64_t at = ((int64_t)(blockIdx.x - kv_groups) * 4 + wave) * UNITS + unit;
    const bool there = at < all;
    const int64_t row = (there ? at : all - 1) / a.n_q_heads;
    const int h = (int)((there ? at : all - 1) % a.n_q_heads), s = (int)(row / r.window), i = (int)(row % r.window);
    float x[8];
    load8(x, (const T*)a.q + row * a.q_stride + h * HD + c * 8);
    const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
    const bool live = sequence_status(r, s, len, n, lane, LANES) == LLM42_SEQ_OK && i < n && there;
    norm_and_rotate<HD>(x, a.q_norm, a.eps, a.rope, live ? len + i : 0, a.rot_dim, a.layout, room[wave], lane);
    if (live) *(u32x4*)(a.q_out + row * a.q_out_stride + h * HD + c * 8) = pack8(x);
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  const bool is_v = item & 1;
  const int h = (int)(item / 2 % a.n_kv_heads), slot = (int)(item / 2 / a.n_kv_heads % slots), s = (int)(item / 2 / a.n_kv_heads / slots);
  if (s >= r.num_seqs) return;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  const int status = sequence_status(r, s, len, n, lane, 64);
  if (a.seq_status && slot == 0 && h == 0 && !is_v && lane == 0) a.seq_status[s] = status;
  if (status != LLM42_SEQ_OK || n == 0) return;
  const int block = len / LLM42_KV_BLOCK + slot, end = len + n;
  if (block * LLM42_KV_BLOCK >= end) return;
  // tokens lo .. hi - 1 of the block are rows of the call; token 0 would be row `row0`
  const int lo = max(len - block * 16, 0), hi = min(end - block * 16, 16);
  const int64_t row0 = (int64_t)s * r.window + (block * 16 - len);
  const size_t at = (size_t)r.block_table[(size_t)s * r.width + block] * a.n_kv_heads + h;
  if (is_v) {
    uint16_t* tile = a.v_plane + at * 16 * HD;
    uint16_t* mine = values[wave];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = j * UNITS + unit;
      if (t < lo || t >= hi) continue;
      float x[8];
      load8(x, (const T*)a.v + (row0 + t) * a.v_stride + h * HD + c * 8);
      const u32x4 w = pack8(x);
      *(u32x2*)(mine + t * PAD + c * 8) = (u32x2){w[0], w[1]};
      *(u32x2*)(mine + t * PAD + c * 8 + 4) = (u32x2){w[2], w[3]};
    }
    __builtin_amdgcn_wave_barrier();
    // four tokens of a feature lie together: lane (g, f) has tokens 4 g .. 4 g + 3 of feature 16 j + f
    const int t = lane >> 4 << 2;
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) {
      const int f = j * 16 + (lane & 15);
      uint16_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = mine[(t + i) * PAD + f];
      uint16_t* o = tile + v_tile_off(f, t);
      if (t >= lo && t + 4 <= hi) {
        *(u32x2*)o = (u32x2){x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t + i >= lo && t + i < hi) o[i] = x[i];
      }
    }
    return;
  }
  uint16_t* tile = a.k_plane + at * 16 * HD;
  u32x4 key[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int t = j * UNITS + unit;
    if ((j + 1) * UNITS <= lo || j * UNITS >= hi) continue;       // (none of these tokens, for the whole wave)
    const bool live = t >= lo && t < hi;
    float x[8];
    load8(x, (const T*)a.k + (row0 + min(max(t, lo), hi - 1)) * a.k_stride + h * HD + c * 8);
    norm_and_rotate<HD>(x, a.k_norm, a.eps, a.rope, live ? block * 16 + t : len, a.rot_dim, a.layout, room[wave], lane);
    key[j] = pack8(x);
    if (live) *(u32x4*)(tile + (c * 16 + t) * 8) = key[j];
  }
  if (!a.bounds || hi < 16) return;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int t = j * UNITS + unit;
    if (t < lo) key[j] = *(const u32x4*)(tile + (c * 16 + t) * 8);
  }
  write_bounds<HD>(key, a.bounds + at * bounds_record(HD), lane);
}

}  // namespace

void launch_rope_table(const double* freq, double factor, int pairs, int max_position, float2* table, hipStream_t st) {
  const int64_t all = (int64_t)pairs * max_position;
  rope_table_kernel<<<(unsigned)((all + 255) / 256), 256, 0, st>>>(freq, factor, pairs, all, table);
}

void launch_kv_append(const Append& a, hipStream_t st) {
  const Rows& r = a.rows;
  const int slots = slots_of(r.window, r.width), units = 4 * (512 / a.head_dim);
  const unsigned kv = (unsigned)(((int64_t)r.num_seqs * slots * a.n_kv_heads * 2 + 3) / 4);
  const unsigned q = a.q ? (unsigned)(((int64_t)r.num_seqs * r.window * a.n_q_heads + units - 1) / units) : 0;
  const auto go = [&](auto kernel) { kernel<<<kv + q, 256, 0, st>>>(a, slots, kv); };
  if (a.head_dim == 128) a.type == LLM42_F32 ? go(append_kernel<128, float>) : go(append_kernel<128, uint16_t>);
  else a.type == LLM42_F32 ? go(append_kernel<64, float>) : go(append_kernel<64, uint16_t>);
}
