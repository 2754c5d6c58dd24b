// Attention of each row over the blocks that its list names.
#include <algorithm>
#include <type_traits>

#include "paged.h"

using namespace paged;

namespace {

// Maximum / sum over the four lanes that hold a head's keys (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float v) {
  const u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a.x), __uint_as_float(a.y));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Two blocks of 16 keys as they come from memory.
template <int HD>
struct Pair {
  u32x4 k[2][HD / 32];
  u32x2 v[2][HD / 16];
};

// A workgroup takes a part of the list of a (row, kv head; blockIdx.y); its NW waves take the part's blocks two at a time in turn, each with a maximum and sum of
// its own, and are joined through LDS.  The heads of the kv head are the columns of the products:
//   scores: D[key][head] = K Q, a tile of K being an operand as it lies in memory;
//   weights: p = exp2((s - ref) scale log2 e) in fp32; ref moves when a pair's maximum exceeds it by more than 8.  They enter the product with V as
//   the sum of two bf16, so that what is lost is 2^-16 of a weight: the launch waits for memory, not for the matrix cores;
//   output: D[feature][head] = V P, a tile of V being four tokens of a feature for each lane, as D's rows of the scores are.
// Bound by memory: 128 sequences x 64 blocks of 8 kv heads of 128, group 4, 539 MB, take 97 - 105 us, 5.1 - 5.5 TB/s; a lone workgroup by what a CU fetches, 1 x 64 9.6 us.
// (K of a wave's next two blocks asked for behind the scores, V behind the output: 105 and 12.8; all of two blocks asked for before the first wait: 106 and 12.4.)
template <int NW, int HD, bool TILES>
__global__ __launch_bounds__(64 * NW) void sparse_attention_kernel(SparseAttention a, float scale_log2) {
  constexpr int KT = HD / 32, FB = HD / 16;
  extern __shared__ int2 sh_list[];                               // [entry of the part, made even]: physical block (-1: none), keys that are seen of it
  __shared__ float sh_ml[NW][2][16];
  __shared__ f32x4 sh_acc[NW][64 * FB];
  __shared__ int sh_used[NW];                                     // entries up to the last one that is a block, among those that a wave looks at
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const Rows& r = a.rows;
  const int part = blockIdx.x % a.parts, row = blockIdx.x / a.parts, kvh = blockIdx.y, s = row / r.window, i = row % r.window;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  if (length_status(r, len, n) != LLM42_SEQ_OK || i >= n) return;
  const int pos = len + i, own = pos / LLM42_KV_BLOCK;
  const int begin = part * a.per_part, count = min(a.width - begin, a.per_part);
  const size_t at = (size_t)row * a.n_kv_heads + kvh, slot = at * a.parts + part;
  bool bad = false;
  int used = 0;
  for (int e0 = wave * 64; e0 < ((count + 1) & ~1); e0 += 64 * NW) {
    const int e = e0 + lane, b = e < count ? a.selected[at * a.width + begin + e] : -1;
    int2 x = make_int2(-1, 0);
    if (b >= 0 && b <= own) {
      x = make_int2(r.block_table[(size_t)s * r.width + b], min(pos - b * LLM42_KV_BLOCK + 1, 16));
      bad |= x.x < 0 || x.x >= r.num_blocks;
    }
    if (e < ((count + 1) & ~1)) sh_list[e] = x;
    const uint64_t there = __ballot(x.y > 0);
    if (there) used = e0 + 64 - __clzll((long long)there);
  }
  if (lane == 0) sh_used[wave] = used;
  bad = __syncthreads_or(bad);
  if (a.parts > 1 && threadIdx.x == 0) a.part_ok[slot] = !bad;
  if (bad) {
    if (a.seq_status && threadIdx.x == 0) atomicOr(a.seq_status + s, LLM42_SEQ_BAD_BLOCK);
    return;
  }

  bf16x8 q[KT];
  {
    const int h = min(l16, a.group - 1);                          // (columns behind the last head repeat it)
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      if constexpr (TILES)
        q[j] = *(const bf16x8*)(a.q + ((size_t)s * a.n_kv_heads + kvh) * 16 * HD + pk_off(h, j * 32 + g * 8, HD));
      else
        q[j] = *(const bf16x8*)(a.q + (int64_t)row * a.q_stride + (int64_t)(kvh * a.group + h) * HD + j * 32 + g * 8);
    }
  }
  f32x4 acc[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) acc[f] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  used = 0;
#pragma unroll
  for (int v = 0; v < NW; ++v) used = max(used, sh_used[v]);
  const int pairs = __builtin_amdgcn_readfirstlane((used + 1) / 2);
  const int64_t to_block = (int64_t)a.n_kv_heads * 16 * HD;
  const uint16_t *kp = a.k_plane + (int64_t)kvh * 16 * HD, *vp = a.v_plane + (int64_t)kvh * 16 * HD;
  for (int p = wave; p < pairs; p += NW) {
    const int2 x[2] = {sh_list[2 * p], sh_list[2 * p + 1]};
    if (x[0].x < 0 && x[1].x < 0) continue;
    Pair<HD> d;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t off = (x[t].x < 0 ? x[1 - t].x : x[t].x) * to_block;      // (an entry that is none reads its neighbour's block, and sees nothing of it)
#pragma unroll
      for (int j = 0; j < KT; ++j) d.k[t][j] = *(const u32x4*)(kp + off + (j * 64 + lane) * 8);
#pragma unroll
      for (int f = 0; f < FB; ++f) d.v[t][f] = *(const u32x2*)(vp + off + (f * 64 + lane) * 4);
    }
    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KT; ++j) sc[t] = mfma16(__builtin_bit_cast(bf16x8, d.k[t][j]), q[j], sc[t]);
    }
    // keys that the row does not see: no weight, and V as zeros (it may hold anything)
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (x[t].y < 16) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (g * 4 + k >= x[t].y) sc[t][k] = -INFINITY;
        const uint32_t keep0 = (g * 4 < x[t].y ? 0xFFFFu : 0u) | (g * 4 + 1 < x[t].y ? 0xFFFF0000u : 0u);
        const uint32_t keep1 = (g * 4 + 2 < x[t].y ? 0xFFFFu : 0u) | (g * 4 + 3 < x[t].y ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int f = 0; f < FB; ++f) d.v[t][f] &= (u32x2){keep0, keep1};
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) mx = fmaxf(mx, sc[t][k]);
    }
    mx = row_max(mx) * scale_log2;
    const bool moves = mx > m + 8.f;
    if (__any(moves)) {
      const float next = moves ? mx : m, alpha = __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.f : next));
      m = next;
      l *= alpha;
#pragma unroll
      for (int f = 0; f < FB; ++f) acc[f] *= alpha;
    }
    const float ref = m == -INFINITY ? 0.f : m;                   // (nothing seen yet: every weight is 0)
    float w[8], sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      w[k] = __builtin_amdgcn_exp2f(fmaf(sc[k >> 2][k & 3], scale_log2, -ref));
      sum += w[k];
    }
    l += sum;
    // (cut off, not rounded: the second part is never below zero, nor zero where the weight is not - an infinite V stays what it is)
    u32x4 hi, lo;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float a = w[2 * k], b = w[2 * k + 1];
      hi[k] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
      lo[k] = pack2_bf16(fmaxf(a - lo_bf16(hi[k]), fminf(a, 0x1p-126f)), fmaxf(b - hi_bf16(hi[k]), fminf(b, 0x1p-126f)));
    }
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const bf16x8 v = __builtin_bit_cast(bf16x8, (u32x4){d.v[0][f].x, d.v[0][f].y, d.v[1][f].x, d.v[1][f].y});
      acc[f] = mfma16(v, __builtin_bit_cast(bf16x8, hi), acc[f]);
      acc[f] = mfma16(v, __builtin_bit_cast(bf16x8, lo), acc[f]);
    }
  }
  // join the waves
  l = row_sum(l);
  if (g == 0) {
    sh_ml[wave][0][l16] = m;
    sh_ml[wave][1][l16] = l;
  }
#pragma unroll
  for (int f = 0; f < FB; ++f) sh_acc[wave][f * 64 + lane] = acc[f];
  __syncthreads();
  float top = -INFINITY, wv[NW], sum = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) top = fmaxf(top, sh_ml[v][0][l16]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    wv[v] = __builtin_amdgcn_exp2f(sh_ml[v][0][l16] - ref);
    sum += wv[v] * sh_ml[v][1][l16];
  }
  if (l16 >= a.group) return;
  if (a.parts > 1 && wave == 0 && g == 0) {
    float* o = a.part_ml + (slot * a.group + l16) * 2;
    o[0] = top;
    o[1] = used ? sum : -1.f;                                 // (a part without keys: see the join)
  }
  for (int f = wave; f < FB; f += NW) {                           // features 16 f + 4 g .. + 3
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NW; ++v) x += sh_acc[v][f * 64 + lane] * wv[v];
    if (a.parts > 1) {
      *(f32x4*)(a.part_acc + (slot * a.group + l16) * HD + f * 16 + g * 4) = x;
      continue;
    }
    const u32x2 packed = used ? (u32x2){pack2_bf16(x[0] / sum, x[1] / sum), pack2_bf16(x[2] / sum, x[3] / sum)} : (u32x2){0, 0};
    const int col = (kvh * a.group + l16) * HD + f * 16 + g * 4;
    if constexpr (TILES) *(u32x2*)(a.out + pk_off(s, col, a.n_kv_heads * a.group * HD)) = packed;
    else *(u32x2*)(a.out + (int64_t)row * a.out_stride + col) = packed;
  }
}

// One wave per (row, kv head, head): the parts of its list, at most 64, a part's maximum and sum in a lane each.
template <int HD, bool TILES>
__global__ __launch_bounds__(256) void sparse_join_kernel(SparseAttention a) {
  const Rows& r = a.rows;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, h = (int)(at % a.group), row = (int)(at / a.group), kvh = blockIdx.y;
  if (row >= r.num_seqs * r.window) return;
  const int s = row / r.window, i = row % r.window, len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  if (length_status(r, len, n) != LLM42_SEQ_OK || i >= n) return;
  const size_t slot0 = ((size_t)row * a.n_kv_heads + kvh) * a.parts;
  const bool mine = lane < a.parts;
  const size_t slot = slot0 + (mine ? lane : 0);
  const int ok = a.part_ok[slot];
  const float part_top = a.part_ml[(slot * a.group + h) * 2], part_sum = a.part_ml[(slot * a.group + h) * 2 + 1];
  if (__any(!ok)) return;                                         // (the parts of such a list wrote nothing else)
  const bool used = mine && part_sum != -1.f;
  const float top = over_rows(over_lanes(used ? part_top : -INFINITY, [](float x, float y) { return fmaxf(x, y); }), [](float x, float y) { return fmaxf(x, y); });
  const bool any = __any(used);
  const float w = used ? __builtin_amdgcn_exp2f(part_top - (top == -INFINITY ? 0.f : top)) : 0.f;
  constexpr int E = HD / 64;
  float o[E] = {}, sum = 0.f;
  for (int p = 0; p < a.parts; ++p) {
    if (!(__ballot(used) >> p & 1)) continue;
    const float wp = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p));
    sum += wp * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(part_sum), p));
    const float* acc = a.part_acc + ((slot0 + p) * a.group + h) * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += wp * acc[e];
  }
  const int col = (kvh * a.group + h) * HD + lane * E;
  uint16_t* out = TILES ? a.out + pk_off(s, col, a.n_kv_heads * a.group * HD) : a.out + (int64_t)row * a.out_stride + col;
  if constexpr (E == 2) *(uint32_t*)out = any ? pack2_bf16(o[0] / sum, o[1] / sum) : 0;
  else *out = any ? (uint16_t)pack2_bf16(o[0] / sum, 0.f) : 0;
}

// Status of every sequence by its lengths; the attention adds what it finds in the table.
__global__ __launch_bounds__(256) void sparse_status_kernel(SparseAttention a) {
  const Rows& r = a.rows;
  const int s = blockIdx.x * 256 + threadIdx.x;
  if (s < r.num_seqs) a.seq_status[s] = length_status(r, r.seq_len[s], r.seq_n ? r.seq_n[s] : r.window);
}

constexpr int kMostPart = 1024;   // entries of a part: 8 KiB of LDS

template <int HD, bool TILES>
void launch(const SparseAttention& a, hipStream_t st) {
  const int rows = a.rows.num_seqs * a.rows.window;
  const float scale_log2 = 1.4426950408889634f * (a.scale > 0.f ? a.scale : 1.0f / sqrtf((float)HD));
  if (a.seq_status) sparse_status_kernel<<<(a.rows.num_seqs + 255) / 256, 256, 0, st>>>(a);
  const dim3 grid(rows * a.parts, a.n_kv_heads);
  const size_t lds = sizeof(int2) * ((a.per_part + 1) & ~1);
  // (eight waves where a CU has no second workgroup: us by eight / four, sequences x 64 blocks, 1 9.6 / 10.4, 8 11.0 / 14.0, 16 14.1 / 15.3, 24 19.3 / 19.3)
  if ((int64_t)grid.x * grid.y <= a.num_cus) sparse_attention_kernel<8, HD, TILES><<<grid, 512, lds, st>>>(a, scale_log2);
  else sparse_attention_kernel<4, HD, TILES><<<grid, 256, lds, st>>>(a, scale_log2);
  if (a.parts > 1) sparse_join_kernel<HD, TILES><<<dim3((unsigned)(((int64_t)rows * a.group + 3) / 4), a.n_kv_heads), 256, 0, st>>>(a);
}

}  // namespace

void plan_sparse_attention(int rows, int n_kv_heads, int head_dim, int width, int num_cus, int& parts, int& per_part) {
  // A list is cut where that spreads it over an idle device: a CU takes about 1.4 us for every 16 of its blocks, the join 3 (us whole / in parts of 32 / 64 blocks,
  // sequences x blocks, 8 kv heads of 128, group 4: 1 x 64 9.6 / 9.9, 1 x 128 15.1 / 10.9, 1 x 256 25.8 / 12.4 / 14.1, 1 x 1024 in parts of 256 / 32 / 64
  // 31 / 25 / 21, 4 x 256 27 / 18.9 / 17.9, 16 x 256 55 / 48.7 / 47.8; but 16 x 64 14.2 / 17.6, 32 x 256 99 / 108 / 105, 128 x 128 194 / 204 / 200).
  const int64_t lists = (int64_t)rows * n_kv_heads, want = 4 * lists < num_cus ? num_cus / 2 : num_cus;
  int parts_ = lists < num_cus && width >= 96 ? (int)((want + lists - 1) / lists) : 1;
  parts_ = std::max(parts_, (width + kMostPart - 1) / kMostPart);
  per_part = std::max(std::min(width, 32), (width + parts_ - 1) / parts_ + 1 & ~1);
  per_part = std::max(per_part, (width + 63) / 64);              // (the join has a lane for every part)
  parts = (width + per_part - 1) / per_part;
}

void launch_sparse_attention(const SparseAttention& a, hipStream_t st) {
  if (a.head_dim == 128) a.tiles ? launch<128, true>(a, st) : launch<128, false>(a, st);
  else a.tiles ? launch<64, true>(a, st) : launch<64, false>(a, st);
}
