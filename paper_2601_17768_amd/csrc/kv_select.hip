// The blocks that a query reads: scores from the bounds of the cached keys, and the highest of them.
#include <algorithm>
#include <type_traits>

#include "paged.h"

using namespace paged;

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// Unsigned keys in the order of the scores; a block whose bounds are infinite comes before all.
__device__ inline uint32_t key_of(float score) {
  const uint32_t u = __float_as_uint(score);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Query heads as operands of the scores: column l16 of the product is head l16 % group of tile row l16 / group.  Lane (g, l16) has features 64 c + 16 g .. + 15
// of its column, positive values in one operand and negative ones in the other: the first meets the upper bounds, the other the
// lower ones, and their sum is the sum of the larger products.
template <int HD>
struct Query {
  i32x4 pos[HD / 64], neg[HD / 64];
  float unit;                  // 2^e of the column
};
template <int HD>
__device__ inline void quantize(Query<HD>& d, const uint16_t* const (&src)[HD / 64][2]) {
  constexpr int C = HD / 64;
  u32x4 w[C][2];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p) w[c][p] = *(const u32x4*)src[c][p];
  float top = 0.f;
  bool bad = false;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = w[c][p][i];
        bad |= (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
        top = fmaxf(top, fmaxf(fabsf(lo_bf16(x)), fabsf(hi_bf16(x))));
      }
  top = bad ? INFINITY : top;                                     // (only ever compared with what is larger: a column's four lanes agree)
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const int e = top == INFINITY ? kMostExponent + 1 : bounds_exponent(top);
  const bool none = e > kMostExponent;
  const float inverse = none ? 0.f : power_of_two(-e);
  d.unit = none ? 0.f : power_of_two(e);
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t p = 0, n = 0;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint32_t x = w[c][j >> 1][(j & 1) * 2 + (b >> 1)];
        const int q = none ? 0 : (int)rintf((b & 1 ? hi_bf16(x) : lo_bf16(x)) * inverse);
        p |= (uint32_t)max(q, 0) << (8 * b);
        n |= ((uint32_t)min(q, 0) & 255u) << (8 * b);
      }
      d.pos[c][j] = (int)p;
      d.neg[c][j] = (int)n;
    }
}

// Keys of 16 blocks, of which lane l16 of every group of 16 has the record: lane (g, column) gets those of blocks 4 g .. 4 g + 3 for its column's tile row (the largest
// over the columns of the same tile row).
template <int HD>
__device__ inline void score16(uint32_t (&key)[4], const char* rec, const Query<HD>& q, int group, int lane) {
  constexpr int C = HD / 64;
  const int g = lane >> 4, l16 = lane & 15;
  i32x4 up[C], down[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    up[c] = *(const i32x4*)(rec + c * 64 + g * 16);
    down[c] = *(const i32x4*)(rec + HD + c * 64 + g * 16);
  }
  const int e = *(const uint8_t*)(rec + 2 * HD);
  i32x4 acc = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < C; ++c) {
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[c], q.pos[c], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[c], q.neg[c], acc, 0, 0, 0);
  }
  float s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = (float)acc[i] * q.unit;
  const int first = lane - l16 % group;                           // (columns behind the last tile row: whatever they get is not used)
  if ((group & (group - 1)) == 0) {
    for (int d = 1; d < group; d *= 2)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fmaxf(s[i], __shfl_xor(s[i], d));
  } else {
    float m[4] = {s[0], s[1], s[2], s[3]};
    for (int d = 0; d < group; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], __shfl(s[i], first + d));
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = m[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int eb = __shfl(e, g * 4 + i);
    key[i] = eb == kBoundsNone ? 0xFFFFFFFFu : key_of(s[i] * power_of_two(eb - kBoundsBias));
  }
}

struct Scratch {
  int hist[256], bin, need, gt[kWaves * 4], eq[kWaves * 4];
};

// The `k` highest of keys[begin .. end - 1], the lowest index on ties, ascending to out; the whole workgroup of T threads together.  The k-th highest key is
// found a byte at a time, from counts of the keys that agree with it so far; then one pass in order.
template <int T>
__device__ inline void pick(const uint32_t* keys, int begin, int end, int k, int32_t* out, Scratch& sh) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  uint32_t prefix = 0, mask = 0;
  int need = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += T) sh.hist[i] = 0;
    __syncthreads();
    for (int i = begin + tid; i < end; i += T) {
      const uint32_t u = keys[i];
      if ((u & mask) == prefix) atomicAdd(&sh.hist[u >> shift & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {                                              // bins from the highest down, four to a lane
      int c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = sh.hist[255 - (lane * 4 + j)];
      int before = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(before, d);
        if (lane >= d) before += x;
      }
      before -= sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < need && before + c[j] >= need) {
          sh.bin = 255 - (lane * 4 + j);
          sh.need = need - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    prefix |= (uint32_t)sh.bin << shift;
    mask |= 255u << shift;
    need = sh.need;
  }
  int gt_before = 0, eq_before = 0;
  for (int base = begin; base < end; base += T) {
    const int i = base + tid;
    const uint32_t u = i < end ? keys[i] : 0;
    const bool gt = i < end && u > prefix, eq = i < end && u == prefix;
    const uint64_t bg = __ballot(gt), be = __ballot(eq), below = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) {
      sh.gt[wave] = __popcll(bg);
      sh.eq[wave] = __popcll(be);
    }
    __syncthreads();
    int ng = gt_before + __popcll(bg & below), ne = eq_before + __popcll(be & below);
    for (int v = 0; v < T / 64; ++v) {
      if (v < wave) {
        ng += sh.gt[v];
        ne += sh.eq[v];
      }
      gt_before += sh.gt[v];
      eq_before += sh.eq[v];
    }
    if (gt || (eq && ne < need)) out[ng + min(ne, need)] = i;
  }
}

// What a row selects, given the keys of its blocks (keys[b], read where it sees more than the budget).
template <int T>
__device__ inline void select_row(const Select& a, const uint32_t* keys, int own, int32_t* out, Scratch& sh) {
  const int seen = own + 1;
  if (seen <= a.budget) {
    for (int j = threadIdx.x; j < a.budget; j += T) out[j] = j < seen ? j : -1;
    return;
  }
  const int k = a.budget - a.sink - a.recent;
  for (int j = threadIdx.x; j < a.sink + a.recent; j += T) {
    if (j < a.sink) out[j] = j;
    else out[k + j] = own - a.recent + 1 + (j - a.sink);
  }
  if (k > 0) pick<T>(keys, a.sink, seen - a.recent, k, out + a.sink, sh);
}

// Pointers to the query of column l16 of a tile of rows i0 .. i0 + rows - 1, features 64 c + 16 g + 8 p.
template <int HD>
__device__ inline void query_of(const uint16_t* (&src)[HD / 64][2], const Select& a, int s, int kvh, int i0, int rows, int lane) {
  const int g = lane >> 4, l16 = lane & 15, i = min(i0 + l16 / a.group, i0 + rows - 1), h = l16 % a.group;
#pragma unroll
  for (int c = 0; c < HD / 64; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int f = c * 64 + g * 16 + p * 8;
      src[c][p] = a.tiles ? a.q + ((size_t)s * a.n_kv_heads + kvh) * 16 * HD + pk_off(h, f, HD)
                          : a.q + ((int64_t)s * a.rows.window + i) * a.q_stride + (int64_t)(kvh * a.group + h) * HD + f;
    }
}

// Status of a sequence, its whole table looked at by the workgroup.
__device__ inline int whole_status(const Rows& r, int s, int len, int n) {
  const int status = length_status(r, len, n);
  bool bad = false;
  if (status == LLM42_SEQ_OK && n > 0)
    for (int b = threadIdx.x; b <= (len + n - 1) / LLM42_KV_BLOCK; b += blockDim.x) {
      const int id = r.block_table[(size_t)s * r.width + b];
      bad |= id < 0 || id >= r.num_blocks;
    }
  return __syncthreads_or(bad) ? LLM42_SEQ_BAD_BLOCK : status;
}

// Keys of blocks begin .. end - 1 (of the sequence) for a tile of rows, by the waves of a workgroup in turn; keys of tile row r at keys + r * stride.
template <int HD>
__device__ inline void score_blocks(const Select& a, int s, int kvh, int i0, int rows, int begin, int end, uint32_t* keys, int64_t stride) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const uint16_t* src[HD / 64][2];
  query_of<HD>(src, a, s, kvh, i0, rows, lane);
  Query<HD> q;
  quantize<HD>(q, src);
  const int32_t* ids = a.rows.block_table + (size_t)s * a.rows.width;
  for (int t = begin / 16 + wave; t * 16 < end; t += waves) {
    const int b = min(max(t * 16 + l16, begin), end - 1);
    const char* rec = a.bounds + ((size_t)ids[b] * a.n_kv_heads + kvh) * bounds_record(HD);
    uint32_t key[4];
    score16<HD>(key, rec, q, a.group, lane);
    if (l16 % a.group == 0 && l16 / a.group < rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = t * 16 + g * 4 + i;
        if (at >= begin && at < end) keys[(l16 / a.group) * stride + at] = key[i];
      }
    }
  }
}

// Scores in LDS: a workgroup per (sequence, tile of 16 / group rows), blockIdx.y: kv head.
template <int HD>
__global__ __launch_bounds__(kThreads) void select_kernel(Select a, int tile_rows, int tiles, int stride) {
  extern __shared__ uint32_t sh_keys[];
  __shared__ Scratch sh;
  const Rows& r = a.rows;
  const int s = blockIdx.x / tiles, i0 = blockIdx.x % tiles * tile_rows, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  const int status = whole_status(r, s, len, n);
  if (a.seq_status && i0 == 0 && kvh == 0 && threadIdx.x == 0) a.seq_status[s] = status;
  if (status != LLM42_SEQ_OK || i0 >= n) return;
  const int rows = min(tile_rows, n - i0), last = (len + i0 + rows - 1) / LLM42_KV_BLOCK;
  if (last + 1 > a.budget && a.budget > a.sink + a.recent) {
    score_blocks<HD>(a, s, kvh, i0, rows, a.sink, last + 1 - a.recent, sh_keys, stride);
    __syncthreads();
  }
  for (int i = 0; i < rows; ++i) {
    select_row<kThreads>(a, sh_keys + i * stride, (len + i0 + i) / LLM42_KV_BLOCK,
                         a.selected + (((size_t)s * r.window + i0 + i) * a.n_kv_heads + kvh) * a.budget, sh);
    __syncthreads();
  }
}

// Scores through the workspace, first launch: a workgroup per (sequence, tile of rows) and chunk of blocks (blockIdx.z).
template <int HD>
__global__ __launch_bounds__(kThreads) void score_kernel(Select a, int tile_rows, int tiles, int64_t stride, int chunk) {
  const Rows& r = a.rows;
  const int s = blockIdx.x / tiles, i0 = blockIdx.x % tiles * tile_rows, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  if (length_status(r, len, n) != LLM42_SEQ_OK || i0 >= n) return;
  const int rows = min(tile_rows, n - i0), last = (len + i0 + rows - 1) / LLM42_KV_BLOCK;
  if (last + 1 <= a.budget || a.budget == a.sink + a.recent) return;
  const int begin = max(a.sink, (int)blockIdx.z * chunk), end = min(last + 1 - a.recent, ((int)blockIdx.z + 1) * chunk);
  if (begin >= end) return;
  bool bad = false;
  for (int b = begin + threadIdx.x; b < end; b += kThreads) {
    const int id = r.block_table[(size_t)s * r.width + b];
    bad |= id < 0 || id >= r.num_blocks;
  }
  if (__syncthreads_or(bad)) return;                              // (the second launch sees it too)
  score_blocks<HD>(a, s, kvh, i0, rows, begin, end, a.keys + (((size_t)s * r.window + i0) * a.n_kv_heads + kvh) * stride,
                   a.n_kv_heads * stride);
}

// ... and second: a workgroup per row, blockIdx.y: kv head.
constexpr int kPickThreads = 1024;
__global__ __launch_bounds__(kPickThreads) void pick_kernel(Select a, int64_t stride) {
  __shared__ Scratch sh;
  const Rows& r = a.rows;
  const int s = blockIdx.x / r.window, i = blockIdx.x % r.window, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  const int status = whole_status(r, s, len, n);
  if (a.seq_status && i == 0 && kvh == 0 && threadIdx.x == 0) a.seq_status[s] = status;
  if (status != LLM42_SEQ_OK || i >= n) return;
  const size_t at = ((size_t)s * r.window + i) * a.n_kv_heads + kvh;
  select_row<kPickThreads>(a, a.keys + at * stride, (len + i) / LLM42_KV_BLOCK, a.selected + at * a.budget, sh);
}

// Keys of a tile row, one for each block that max_context positions can have.
int64_t keys_of(int max_context) { return (max_context + 15) / 16; }
int tile_rows_of(int group, int window) { return std::min(16 / group, window); }
constexpr int64_t kMostLdsKeys = 12288;      // 48 KiB

}  // namespace

size_t select_workspace(int num_seqs, int window, int n_kv_heads, int group, int max_context, int budget, int num_cus) {
  const int64_t keys = keys_of(max_context);
  if (keys <= budget || tile_rows_of(group, window) * keys <= kMostLdsKeys) return 0;
  return 4ull * num_seqs * window * n_kv_heads * keys;
}

void launch_kv_select(const Select& a, hipStream_t st) {
  const Rows& r = a.rows;
  const int tile_rows = tile_rows_of(a.group, r.window), tiles = (r.window + tile_rows - 1) / tile_rows;
  const int64_t keys = keys_of(r.max_context);
  const auto go = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    if (!a.keys) {
      const size_t lds = keys <= a.budget ? 0 : 4 * tile_rows * keys;
      select_kernel<HD><<<dim3(r.num_seqs * tiles, a.n_kv_heads), kThreads, lds, st>>>(a, tile_rows, tiles, (int)keys);
      return;
    }
    const int chunk = (int)std::max<int64_t>(256, (keys + 4095) / 4096);
    score_kernel<HD><<<dim3(r.num_seqs * tiles, a.n_kv_heads, (unsigned)((keys + chunk - 1) / chunk)), kThreads, 0, st>>>(a, tile_rows, tiles, keys, chunk);
    pick_kernel<<<dim3(r.num_seqs * r.window, a.n_kv_heads), kPickThreads, 0, st>>>(a, keys);
  };
  if (a.head_dim == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 64>{});
}
