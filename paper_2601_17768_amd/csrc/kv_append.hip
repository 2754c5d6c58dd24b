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

// Eight neighbouring features as they lie in memory, and as fp32.
template <typename T>
struct Eight {
  u32x4 w[sizeof(T) / 2];
  __device__ inline void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ((const u32x4*)p)[i];
  }
  __device__ inline void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[0][i]);
        x[4 + i] = __uint_as_float(w[1][i]);
      } else {
        x[2 * i] = lo_bf16(w[0][i]);
        x[2 * i + 1] = hi_bf16(w[0][i]);
      }
    }
  }
};
template <typename T>
__device__ inline void load8(float (&x)[8], const T* p) {
  Eight<T> d;
  d.load(p);
  d.get(x);
}

__device__ inline u32x4 pack8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(x[2 * i], x[2 * i + 1]);
  return w;
}

// How features are paired: not at all, neighbours, halves of the whole head, halves of a part of it.
enum class Pairs { NONE, NEAR, HALVES, PART };

// What a lane with features 8 c .. 8 c + 7 needs to turn them: feature f becomes x[f] * cos[f] + partner * sin[f] (the sign of its place in the pair in sin).
struct Turn {
  float cos[8], sin[8];
};
__device__ inline void load_turn(Turn& d, Pairs pairs, const float2* rope, int pos, int rot_dim, int c) {
  if (pairs == Pairs::NONE) return;
  const int half = rot_dim / 2;
  const float2* cs = rope + (size_t)pos * half;
  if (pairs == Pairs::HALVES) {                                   // (half is 32 or 64: rows of the table are 16-byte aligned)
    const bool first = c * 8 < half;
    const f32x4* p = (const f32x4*)(cs + (first ? c * 8 : c * 8 - half));
#pragma unroll
    for (int f = 0; f < 8; f += 2) {
      const f32x4 t = p[f / 2];
      d.cos[f] = t[0];
      d.sin[f] = first ? -t[1] : t[1];
      d.cos[f + 1] = t[2];
      d.sin[f + 1] = first ? -t[3] : t[3];
    }
    return;
  }
  if (pairs == Pairs::NEAR && half % 4 == 0) {
    const f32x4* p = (const f32x4*)(cs + min(c * 4, half - 4));
#pragma unroll
    for (int f = 0; f < 8; f += 4) {
      const f32x4 t = p[f / 4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        d.cos[f + 2 * i] = d.cos[f + 2 * i + 1] = t[2 * i];
        d.sin[f + 2 * i] = -t[2 * i + 1];
        d.sin[f + 2 * i + 1] = t[2 * i + 1];
      }
    }
    return;
  }
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    const int at = c * 8 + f;
    const bool first = pairs == Pairs::NEAR ? !(f & 1) : at < half;
    const int j = pairs == Pairs::NEAR ? at / 2 : first ? at : at - half;
    const float2 t = cs[min(j, half - 1)];                        // (features behind rot_dim make no use of theirs)
    d.cos[f] = t.x;
    d.sin[f] = first ? -t.y : t.y;
  }
}

template <int LANES>
__device__ inline float head_sum(float v) {
  const auto with = [&](uint32_t x) __attribute__((always_inline)) { v += __uint_as_float(x); };
  with(other_lane<kXor1>(__float_as_uint(v)));
  with(other_lane<kXor2>(__float_as_uint(v)));
  with(other_lane<kMirror8>(__float_as_uint(v)));
  if constexpr (LANES == 16) with(other_lane<kMirror16>(__float_as_uint(v)));
  return v;
}

// The norm of a head of HD features in HD / 8 lanes, fp32.
template <int HD>
__device__ inline void norm(float (&x)[8], const float (&gain)[8], float eps) {
  float sum = 0.f;
#pragma unroll
  for (int f = 0; f < 8; ++f) sum = fmaf(x[f], x[f], sum);
  const float r = 1.0f / sqrtf(head_sum<HD / 8>(sum) / HD + eps);
#pragma unroll
  for (int f = 0; f < 8; ++f) x[f] = x[f] * r * gain[f];
}

// Its rotation, fp32; every lane of the wave takes part.  Halves of the whole head: the partner is at the same place of the lane half a head away.  Of a part: it may be in any
// lane and at any place there (rot_dim / 2 is any number), so a head goes through `room`, 512 floats of LDS that are this wave's own, element e of lane l
// at e * 64 + l: all lanes of a half look at one e at a time, no bank conflicts.
template <int HD>
__device__ inline void rotate(float (&x)[8], const Turn& t, Pairs pairs, int rot_dim, float* room, int lane) {
  constexpr int LANES = HD / 8;
  const int c = lane % LANES, base = lane - c, half = rot_dim / 2;
  float y[8];
  if (pairs == Pairs::NONE) return;
  if (pairs == Pairs::NEAR) {
#pragma unroll
    for (int f = 0; f < 8; ++f) y[f] = x[f ^ 1];
  } else if (pairs == Pairs::HALVES) {
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      const uint32_t u = __float_as_uint(x[f]);
      y[f] = __uint_as_float(LANES == 16 ? other_lane<kXor8>(u) : other_lane<kMirror4>(other_lane<kMirror8>(u)));
    }
  } else {
#pragma unroll
    for (int f = 0; f < 8; ++f) room[f * 64 + lane] = x[f];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      const int at = c * 8 + f, other = at < half ? at + half : at < rot_dim ? at - half : at;
      y[f] = room[(other & 7) * 64 + base + (other >> 3)];
    }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int f = 0; f < 8; ++f)
    if (c * 8 + f < rot_dim) x[f] = fmaf(y[f], t.sin[f], x[f] * t.cos[f]);
}

// Whether a block that a row of a sequence (in order by its lengths, or without rows) lies in has no entry in the table, asked by the `lanes` neighbouring lanes that work
// for it (all lanes of the wave ask together).
__device__ inline bool bad_block(const Rows& r, int s, int len, int n, int lane, int lanes) {
  bool bad = false;
  if (n > 0)
    for (int b = len / LLM42_KV_BLOCK + lane % lanes; b <= (len + n - 1) / LLM42_KV_BLOCK; b += lanes) {
      const int id = r.block_table[(size_t)s * r.width + b];
      bad |= id < 0 || id >= r.num_blocks;
    }
  const uint64_t mine = (lanes == 64 ? ~0ull : ((1ull << lanes) - 1)) << (lane - lane % lanes);
  return (__ballot(bad) & mine) != 0;
}

// The launch's first workgroups take a (sequence, block, kv head) of K or of V per wave, the others a row and some heads of Q per HD / 8 lanes: its position's
// cos and sin are read once for them.  8 x 512 rows of 32 + 2 x 8 heads of 128 with norms, 103 MB, take 29 us (a head at a time 47, four 33, sixteen 37), of which memory is
// 21, as a copy of as many bytes takes: without norms and rotation the launch takes 24.5, without norms 27.6, without rotation 25.6, so a sixth is arithmetic and the loads of cos and sin, which
// wait behind the rows.  K and V alone take 12.4, 9.6 without norms and rotation; from fp32 all takes 36.8, and with the bounds kept up 30.6.  (Three sets of inputs in turn;
// one, part of which the caches hold, 22.6, and a copy 15.6.)  Few rows: launch and two trips, one row 3.8, 128 4.8, with bounds 5.9.
template <int HD, typename T>
__global__ __launch_bounds__(256) void append_kernel(Append a, Pairs pairs, int slots, unsigned kv_groups, int q_heads) {
  constexpr int LANES = HD / 8, UNITS = 64 / LANES, N = HD / 32, PAD = HD + 4;
  __shared__ float room[4][512];
  __shared__ __align__(16) uint16_t values[4][16 * PAD];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % LANES, unit = lane / LANES;
  const Rows& r = a.rows;
  float gain[8];
  Turn turn;
  if (blockIdx.x >= kv_groups) {
    const int per_row = (a.n_q_heads + q_heads - 1) / q_heads;
    const int64_t all = (int64_t)r.num_seqs * r.window * per_row, mine = ((int64_t)(blockIdx.x - kv_groups) * 4 + wave) * UNITS + unit;
    const int64_t row = min(mine, all - 1) / per_row;
    const int h0 = (int)(min(mine, all - 1) % per_row) * q_heads, s = (int)(row / r.window), i = (int)(row % r.window);
    const T* src = (const T*)a.q + row * a.q_stride + c * 8;
    Eight<T> next;
    next.load(src + h0 * HD);
    if (a.q_norm) load8(gain, a.q_norm + c * 8);
    const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
    bool live = mine < all && length_status(r, len, n) == LLM42_SEQ_OK && i < n;
    load_turn(turn, pairs, a.rope, live ? len + i : 0, a.rot_dim, c);
    if (bad_block(r, s, len, live ? n : 0, lane, LANES)) live = false;
    for (int h = h0; h < h0 + q_heads; ++h) {                     // (heads behind the last one repeat it)
      float x[8];
      next.get(x);
      if (h + 1 < h0 + q_heads) next.load(src + min(h + 1, a.n_q_heads - 1) * HD);
      if (a.q_norm) norm<HD>(x, gain, a.eps);
      rotate<HD>(x, turn, pairs, a.rot_dim, room[wave], lane);
      if (live && h < a.n_q_heads) *(u32x4*)(a.q_out + row * a.q_out_stride + h * HD + c * 8) = pack8(x);
    }
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  const bool is_v = item & 1;
  const int h = (int)(item / 2 % a.n_kv_heads), slot = (int)(item / 2 / a.n_kv_heads % slots), s = (int)(item / 2 / a.n_kv_heads / slots);
  if (s >= r.num_seqs) return;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  int status = length_status(r, len, n);
  if (bad_block(r, s, len, status == LLM42_SEQ_OK ? n : 0, lane, 64)) status = LLM42_SEQ_BAD_BLOCK;
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
    Eight<T> in[N];
#pragma unroll
    for (int j = 0; j < N; ++j) in[j].load((const T*)a.v + (row0 + min(max(j * UNITS + unit, lo), hi - 1)) * a.v_stride + h * HD + c * 8);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = j * UNITS + unit;
      if (t < lo || t >= hi) continue;
      float x[8];
      in[j].get(x);
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
  Eight<T> in[N];
#pragma unroll
  for (int j = 0; j < N; ++j) in[j].load((const T*)a.k + (row0 + min(max(j * UNITS + unit, lo), hi - 1)) * a.k_stride + h * HD + c * 8);
  if (a.k_norm) load8(gain, a.k_norm + c * 8);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int t = j * UNITS + unit;
    if ((j + 1) * UNITS <= lo || j * UNITS >= hi) continue;       // (none of these tokens, for the whole wave)
    const bool live = t >= lo && t < hi;
    const int from = min(max(t, lo), hi - 1);
    float x[8];
    in[j].get(x);
    load_turn(turn, pairs, a.rope, block * 16 + from, a.rot_dim, c);
    if (a.k_norm) norm<HD>(x, gain, a.eps);
    rotate<HD>(x, turn, pairs, a.rot_dim, room[wave], lane);
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
  const int64_t rows = (int64_t)r.num_seqs * r.window;
  const Pairs pairs = !a.rope ? Pairs::NONE : a.layout == LLM42_ROPE_INTERLEAVED ? Pairs::NEAR : a.rot_dim == a.head_dim ? Pairs::HALVES : Pairs::PART;
  // (a head at a time while heads are no more than lanes enough to fill the device)
  const int q_heads = rows * a.n_q_heads <= 32768 ? 1 : 8;
  const unsigned kv = (unsigned)((rows / r.window * slots * a.n_kv_heads * 2 + 3) / 4);
  const unsigned q = a.q ? (unsigned)((rows * ((a.n_q_heads + q_heads - 1) / q_heads) + units - 1) / units) : 0;
  const auto go = [&](auto kernel) { kernel<<<kv + q, 256, 0, st>>>(a, pairs, slots, kv, q_heads); };
  if (a.head_dim == 128) a.type == LLM42_F32 ? go(append_kernel<128, float>) : go(append_kernel<128, uint16_t>);
  else a.type == LLM42_F32 ? go(append_kernel<64, float>) : go(append_kernel<64, uint16_t>);
}
