// Causal attention of the last positions of every sequence over the 4-bit cache.
#include <type_traits>

#include "kv4_store.h"

using namespace mx4;

namespace {

// A decoding step whose 4-bit cache has a block table of its own: one wave per sequence.
__global__ __launch_bounds__(64) void kv4_step_check_kernel(const int32_t* __restrict__ table, int width, int64_t num_blocks,
                                                            int32_t* __restrict__ seq_status, int32_t* __restrict__ ws_len,
                                                            int32_t* __restrict__ row_pos, uint16_t* __restrict__ attn, int d_attn) {
  const int s = blockIdx.x, lane = threadIdx.x, len = ws_len[s];
  if (len < 0) return;
  bool bad = false;
  for (int b = lane; b <= len / LLM42_KV_BLOCK; b += 64) {
    const int id = table[(size_t)s * width + b];
    bad |= id < 0 || id >= num_blocks;
  }
  if (!__any(bad)) return;
  for (int c = lane * 8; c < d_attn; c += 512) *(uint4*)(attn + pk_off(s, c, d_attn)) = make_uint4(0, 0, 0, 0);
  if (lane == 0) {
    ws_len[s] = row_pos[s] = -1;
    if (seq_status) seq_status[s] = LLM42_SEQ_BAD_BLOCK;
  }
}

constexpr int kWaves = 4;   // of a workgroup, or twice as many
constexpr int kStep = 64;   // keys

// The keys of one step as they come from memory: four blocks of 16 positions.
template <int HD>
struct Step {
  static constexpr int KT = HD / 32;
  uint32_t k[4][KT], ks[4], v[4][KT], vs[4][KT];
};

template <int HD, bool NT>
__device__ __forceinline__ void load_words(uint32_t (&d)[HD / 32], const char* p) {
  if constexpr (HD == 128) {
    const u32x4 w = NT ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = w[i];
  } else {
    const u32x2 w = NT ? __builtin_nontemporal_load((const u32x2*)p) : *(const u32x2*)p;
    d[0] = w.x;
    d[1] = w.y;
  }
}

// Maximum / sum over the four lanes that hold a query row's keys (lanes l, l ^ 16, l ^ 32, l ^ 48).
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

// A workgroup takes RB blocks of 16 query rows of a (sequence, kv head) over one of the parts of its context; its NW waves take the
// part's steps of 64 keys in turn, each with a maximum and sum of its own, and are joined through LDS.
//   scores: D[key][row] = K Q, K converted with its scales (exact in bf16);
//   weights: p = exp2((s - ref) / sqrt(head_dim) log2 e) in fp32; ref moves to a step's maximum when that exceeds it by more than 8, so
//   that most steps rescale nothing and p stays below 2^8; rounded to bf16 (2^-8 of a weight: what the matrix instruction takes, and what the
//   bf16 attention does), their sum is taken before that.  Outputs are off by up to 0.0023 of their size so, 0.0017 by their own rounding;
//   a second operand with what the first lacks is exact to 2^-17, for twice the P V products (us without / with: 1 x 512 7.0 / 7.4,
//   24 x 4000 25.5 / 28, 128 x 4000 103 / 111, 4 windows of 64 x 4000 34 / 40).  D's layout is that of the P V operand: no exchange between lanes;
//   output: D[feature][row] = V P.  An operand holds 8 keys of one feature, and a scale belongs to 32 features of one key: two neighbouring
//   features of a key are converted together, with its scale, and the halves of 8 keys gathered into the operands of the one and
//   the other feature.  Where a row does not see all keys of the step, the scales go into its weights instead (the same products): V that a row must not
//   see may stand for NaN, and 0 NaN is NaN.
// One block of rows is bound by memory: 128 sequences of 1024 - 8192 keys (8 kv heads of 128, group 4) 129 us, 4.9 TB/s; 1 of 512 keys is
// launch and waiting, 7 us.
template <int NW, int HD, int RB, bool TILES, bool NT>
__global__ __launch_bounds__(64 * NW, NW == 4 && RB == 1 ? 3 : 2) void kv4_attention_kernel(Attention4 a, float scale_log2) {
  constexpr int KT = HD / 32, FB = HD / 16;
  __shared__ float sh_ml[NW][RB][2][16];
  __shared__ f32x4 sh_acc[NW][64 * FB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int rows_all = a.group * a.window, row_groups = (rows_all + 16 * RB - 1) / (16 * RB);
  int id = blockIdx.x;
  const int split = id % a.splits;
  id /= a.splits;
  const int rg = id % row_groups;
  id /= row_groups;
  const int kvh = id % a.n_kv_heads, s = id / a.n_kv_heads;
  int len = a.seq_len[s], n = a.window;
  if constexpr (TILES) {
    if (len < 0) return;
  } else {
    // a call by itself: every workgroup of a sequence checks it (a launch of its own took 2 - 5 us)
    if (a.seq_n) n = a.seq_n[s];
    int status = len < 0 || n < 0 || n > a.window || (int64_t)len + n > a.max_context ? LLM42_SEQ_BAD_LENGTH : LLM42_SEQ_OK;
    bool bad = false;
    if (status == LLM42_SEQ_OK && n > 0)
      for (int b = threadIdx.x; b <= (len + n - 1) / LLM42_KV_BLOCK; b += 64 * NW) {
        const int block = a.block_table[(size_t)s * a.max_blocks + b];
        bad |= block < 0 || block >= a.num_blocks;
      }
    if (__syncthreads_or(bad)) status = LLM42_SEQ_BAD_BLOCK;
    if (a.seq_status && kvh == 0 && rg == 0 && split == 0 && threadIdx.x == 0) a.seq_status[s] = status;
    if (a.merge_n && rg == 0 && split == 0 && threadIdx.x == 0) a.merge_n[(size_t)s * a.n_kv_heads + kvh] = status == LLM42_SEQ_OK ? n : 0;
    if (status != LLM42_SEQ_OK) return;
  }
  const int r0 = rg * 16 * RB, rows = n * a.group;               // rows past the last one repeat it
  if (r0 >= rows) return;
  const int keys = len + (min(r0 + 16 * RB, rows) - 1) / a.group + 1;
  const int steps = (keys + kStep - 1) / kStep, begin = split * a.split_steps, end = min(steps, begin + a.split_steps);
  if (begin >= end) return;

  bf16x8 q[RB][KT];
  int limit[RB];                                                  // the row of this lane sees keys below it
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int r = min(r0 + b * 16 + l16, rows - 1), i = r / a.group, h = r - i * a.group;
    limit[b] = len + i + 1;
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      if constexpr (TILES)
        q[b][j] = *(const bf16x8*)(a.q + ((size_t)s * a.n_kv_heads + kvh) * 16 * HD + pk_off(r, j * 32 + g * 8, HD));
      else
        q[b][j] = *(const bf16x8*)(a.q + ((size_t)s * a.window + i) * a.q_stride + (size_t)(kvh * a.group + h) * HD + j * 32 + g * 8);
    }
  }
  f32x4 acc[RB][FB];                                              // [2 j]: features 32 j + 8 g + 0, 2, 4, 6; [2 j + 1]: 1, 3, 5, 7
  float m[RB], l[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    m[b] = -INFINITY;
    l[b] = 0.f;
#pragma unroll
    for (int f = 0; f < FB; ++f) acc[b][f] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  const int32_t* ids = a.block_table + (size_t)s * a.max_blocks;
  const int last_block = (keys - 1) / LLM42_KV_BLOCK;
  const int64_t to_block = (int64_t)a.n_kv_heads * kv_record(HD);
  const char* base = a.base + (int64_t)kvh * kv_record(HD);
  // block ids of a step are asked for a step ahead of the loads that need them
  auto blocks_of = [&](int (&id)[4], int step) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) id[t] = ids[min(step * 4 + t, last_block)];
  };
  auto load_k = [&](Step<HD>& d, const int (&id)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char* rec = base + id[t] * to_block;
      load_words<HD, NT>(d.k[t], rec + lane * KT * 4);
      d.ks[t] = KT == 4 ? *(const uint32_t*)(rec + 16 * HD + l16 * 4) : *(const uint16_t*)(rec + 16 * HD + l16 * 2);
    }
  };
  auto load_v = [&](Step<HD>& d, const int (&id)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char* rec = base + id[t] * to_block;
      load_words<HD, NT>(d.v[t], rec + 8 * HD + lane * KT * 4);
      load_words<HD, NT>(d.vs[t], rec + 16 * HD + HD / 2 + g * KT * 4);
    }
  };
  float p[RB][4][4];
  auto weights = [&](const Step<HD>& d, int step, auto is_edge) __attribute__((always_inline)) {
    constexpr bool edge = decltype(is_edge)::value;
    f32x4 sc[4][RB];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[t][b] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bf16x8 k = operand(d.k[t][j], scale_of(d.ks[t], j));
#pragma unroll
        for (int b = 0; b < RB; ++b) sc[t][b] = mfma16(k, q[b][j], sc[t][b]);
        __builtin_amdgcn_sched_barrier(0);                        // (left alone, the compiler converts far ahead and runs out of registers)
      }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[b][t][i] = edge && step * kStep + t * 16 + g * 4 + i >= limit[b] ? -INFINITY : sc[t][b][i];
          mx = fmaxf(mx, p[b][t][i]);
        }
      mx = row_max(mx) * scale_log2;
      const bool moves = mx > m[b] + 8.f;
      if (__any(moves)) {
        const float next = moves ? mx : m[b], alpha = __builtin_amdgcn_exp2f(m[b] - (next == -INFINITY ? 0.f : next));
        m[b] = next;
        l[b] *= alpha;
#pragma unroll
        for (int f = 0; f < FB; ++f) acc[b][f] *= alpha;
      }
      const float ref = m[b] == -INFINITY ? 0.f : m[b];           // (nothing seen yet: every weight is 0)
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[b][t][i] = __builtin_amdgcn_exp2f(fmaf(p[b][t][i], scale_log2, -ref));
          sum += p[b][t][i];
        }
      l[b] += sum;
    }
  };
  auto pack = [&](const float (&w)[8]) __attribute__((always_inline)) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pack2_bf16(w[2 * i], w[2 * i + 1]);
    return __builtin_bit_cast(bf16x8, u);
  };
  // pairs [i]: features 2 p and 2 p + 1 of 8 keys -> the operands of the one and of the other
  auto gather = [&](const uint32_t (&r)[8], bool odd) __attribute__((always_inline)) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(r[2 * i + 1], r[2 * i], odd ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, u);
  };
  auto values = [&](const Step<HD>& d, int step, auto is_edge) __attribute__((always_inline)) {
    constexpr bool edge = decltype(is_edge)::value;
#pragma unroll
    for (int t = 0; t < 4; t += 2) {
      bf16x8 pw[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = p[b][t + (i >> 2)][i & 3];
        pw[b] = pack(w);
      }
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        uint32_t r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          r[i] = pair_bf16(d.v[t + (i >> 2)][j], edge ? 1.0f : scale_of(d.vs[t + (i >> 2)][j], i & 3), i & 3);
        if (edge) {
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float e = __uint_as_float((d.vs[t + (i >> 2)][j] >> (8 * (i & 3)) & 255u) << 23);
              w[i] = step * kStep + (t + (i >> 2)) * 16 + g * 4 + (i & 3) >= limit[b] ? 0.f : p[b][t + (i >> 2)][i & 3] * e;
            }
            pw[b] = pack(w);
          }
        }
        const bf16x8 even = gather(r, false), odd = gather(r, true);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          acc[b][2 * j] = mfma16(even, pw[b], acc[b][2 * j]);
          acc[b][2 * j + 1] = mfma16(odd, pw[b], acc[b][2 * j + 1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // The newest position of a decoding step is in the bf16 cache: the wave whose last step holds it stores it before it reads anything
  // (nobody else reads that block; a launch of its own took 5 - 7 us).
  if constexpr (TILES) {
    if (end == steps && (end - 1 - begin) % NW == wave) {
      const size_t tile = ((size_t)a.row_blk[s] * a.n_kv_heads + kvh) * 16 * HD;
      const int t = len % LLM42_KV_BLOCK;
      store_positions<HD>(a.k_plane + tile, a.v_plane + tile, a.base + kvh * (int64_t)kv_record(HD) + ids[len / LLM42_KV_BLOCK] * to_block, t, t + 1, lane);
      __threadfence_block();
    }
  }
  // Steps that every row sees whole, then the last ones.
  const int inner = min(end, (len + 1) / kStep);
  int step = begin + wave;
  if (step < end) {
    // K of the next step is asked for behind the scores, V behind the output
    Step<HD> d;
    int now[4], next[4];
    blocks_of(now, step);
    load_k(d, now);
    load_v(d, now);
    blocks_of(now, min(step + NW, end - 1));
    const auto one = [&](auto is_edge) __attribute__((always_inline)) {
      blocks_of(next, min(step + 2 * NW, end - 1));
      weights(d, step, is_edge);
      load_k(d, now);
      __builtin_amdgcn_sched_barrier(0);
      values(d, step, is_edge);
      load_v(d, now);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 4; ++t) now[t] = next[t];
      step += NW;
    };
    while (step < inner) one(std::false_type{});
    while (step < end) one(std::true_type{});
  }
  // join the waves
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float sum = row_sum(l[b]);
    if (g == 0) {
      sh_ml[wave][b][0][l16] = m[b];
      sh_ml[wave][b][1][l16] = sum;
    }
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FB; ++f) sh_acc[wave][f * 64 + lane] = acc[b][f];
    __syncthreads();
    float top = -INFINITY, w[NW], sum = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v) top = fmaxf(top, sh_ml[v][b][0][l16]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      w[v] = __builtin_amdgcn_exp2f(sh_ml[v][b][0][l16] - ref);
      sum += w[v] * sh_ml[v][b][1][l16];
    }
    const int r = r0 + b * 16 + l16;
    if (r >= rows) continue;
    const int i = r / a.group, h = r - i * a.group;
    const size_t slot = (((size_t)s * a.n_kv_heads + kvh) * a.splits + split) * rows_all + r;
    if (a.splits > 1 && wave == 0 && g == 0) {
      a.part_ml[2 * slot] = top;
      a.part_ml[2 * slot + 1] = sum;
    }
    for (int j = wave; j < KT; j += NW) {                     // features 32 j + 8 g .. + 7
      f32x4 even = {0.f, 0.f, 0.f, 0.f}, odd = even;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        even += sh_acc[v][2 * j * 64 + lane] * w[v];
        odd += sh_acc[v][(2 * j + 1) * 64 + lane] * w[v];
      }
      if (a.splits > 1) {
        float* o = a.part_acc + slot * HD + j * 32 + g * 8;
        *(f32x4*)o = (f32x4){even[0], odd[0], even[1], odd[1]};
        *(f32x4*)(o + 4) = (f32x4){even[2], odd[2], even[3], odd[3]};
        continue;
      }
      u32x4 packed;
#pragma unroll
      for (int e = 0; e < 4; ++e) packed[e] = pack2_bf16(even[e] / sum, odd[e] / sum);
      const int col = (kvh * a.group + h) * HD + j * 32 + g * 8;
      if constexpr (TILES) *(u32x4*)(a.out + pk_off(s, col, a.n_kv_heads * a.group * HD)) = packed;
      else *(u32x4*)(a.out + ((size_t)s * a.window + i) * a.out_stride + col) = packed;
    }
  }
}

// One wave per (sequence, kv head, query row): the parts of its context, first to last.
template <int HD, bool TILES>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Attention4 a) {
  const int rows_all = a.group * a.window;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= (int64_t)a.num_seqs * a.n_kv_heads * rows_all) return;
  const int lane = threadIdx.x & 63, r = (int)(at % rows_all), kvh = (int)(at / rows_all % a.n_kv_heads), s = (int)(at / rows_all / a.n_kv_heads);
  const int len = a.seq_len[s];
  const int i = r / a.group, h = r - i * a.group;
  const int n = TILES ? (len < 0 ? 0 : 1) : a.merge_n[(size_t)s * a.n_kv_heads + kvh];
  if (i >= n) return;
  // the parts that the row's workgroup went through (its block of rows sees as much as its last row does)
  const int rb = rows_all > 16 ? 32 : 16, last = min((r / rb + 1) * rb, n * a.group) - 1;
  const int keys = len + last / a.group + 1, steps = (keys + kStep - 1) / kStep, parts = (steps + a.split_steps - 1) / a.split_steps;
  const size_t slot0 = (((size_t)s * a.n_kv_heads + kvh) * a.splits) * rows_all + r;
  float top = -INFINITY;
  for (int p = 0; p < parts; ++p) top = fmaxf(top, a.part_ml[2 * (slot0 + (size_t)p * rows_all)]);
  const float ref = top == -INFINITY ? 0.f : top;
  constexpr int E = HD / 64;
  float o[E] = {}, sum = 0.f;
  for (int p = 0; p < parts; ++p) {
    const size_t slot = slot0 + (size_t)p * rows_all;
    const float w = __builtin_amdgcn_exp2f(a.part_ml[2 * slot] - ref);
    sum += w * a.part_ml[2 * slot + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += w * a.part_acc[slot * HD + lane * E + e];
  }
  const int col = (kvh * a.group + h) * HD + lane * E;
  uint16_t* out = TILES ? a.out + pk_off(s, col, a.n_kv_heads * a.group * HD) : a.out + ((size_t)s * a.window + i) * a.out_stride + col;
  if constexpr (E == 2) *(uint32_t*)out = pack2_bf16(o[0] / sum, o[1] / sum);
  else *out = (uint16_t)pack2_bf16(o[0] / sum, 0.f);
}

template <int HD, bool TILES>
void launch(const Attention4& a, hipStream_t st) {
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  const int rows = a.group * a.window, rb = rows > 16 ? 2 : 1, groups = (rows + 16 * rb - 1) / (16 * rb);
  const unsigned grid = (unsigned)((int64_t)a.num_seqs * a.n_kv_heads * groups * a.splits);
  // K and V past the caches where there is no more than one block of rows to read them and they may be more than the memory-side cache holds
  // (128 sequences of 1024 - 8192 keys 149 -> 134 us, of 8192 220 -> 193; what the caches do hold is slower so, 1 x 8192 16 -> 17.6)
  const bool nt = rb == 1 && (int64_t)a.num_seqs * a.max_context * a.n_kv_heads * kv_record(HD) / LLM42_KV_BLOCK > (256 << 20);
  // No more workgroups than CUs: eight waves in each, where they have more than two rounds of four waves between them (a wave alone on its SIMD
  // waits for its own conversions: us by four / eight waves 24 x 2000 18.8 / 16.7, 32 x 4000 30.7 / 27.5, 16 x 2000 17.7 / 15.4, 1 x 1000
  // 9.9 / 9.6; but 1 x 511 7.1 / 7.3, 48 x 2000 25.8 / 30.1)
  const bool eight = grid <= (unsigned)a.num_cus && a.split_steps > 2 * kWaves;
  const auto go = [&](auto waves, auto blocks, auto past) {
    constexpr int NW = decltype(waves)::value, RB = decltype(blocks)::value;
    kv4_attention_kernel<NW, HD, RB, TILES, decltype(past)::value><<<grid, 64 * NW, 0, st>>>(a, scale_log2);
  };
  const auto by_waves = [&](auto blocks, auto past) {
    if (eight) go(std::integral_constant<int, 2 * kWaves>{}, blocks, past);
    else go(std::integral_constant<int, kWaves>{}, blocks, past);
  };
  using One = std::integral_constant<int, 1>;
  if (nt) by_waves(One{}, std::true_type{});
  else if (rb == 1) by_waves(One{}, std::false_type{});
  else if constexpr (!TILES) by_waves(std::integral_constant<int, 2>{}, std::false_type{});
  if (a.splits > 1) {
    const int64_t all = (int64_t)a.num_seqs * a.n_kv_heads * rows;
    kv4_merge_kernel<HD, TILES><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a);
  }
}

}  // namespace

void launch_kv4_step_check(const llm42_model* m, const llm42_kv_cache* kv4, int num_seqs, int32_t* seq_status, const Workspace& ws,
                           hipStream_t st) {
  kv4_step_check_kernel<<<num_seqs, 64, 0, st>>>(kv4->block_table, kv4->max_blocks_per_seq, kv4->num_blocks, seq_status, ws.seq_len,
                                                 ws.row_pos, ws.attn, m->d_attn);
}

// Parts of a context: two workgroups for every CU, parts of 8 steps (2 a wave) or more - if that is worth the launch that joins them: a wave's step
// takes about 1 us, the launch 4 - 5, and a device half full of workgroups hides some of the former (us in parts / whole, sequences x
// keys, 8 kv heads: 1 x 2000 12.8 / 15.9, 1 x 8192 16.9 / 41, 16 x 8192 34 / 50; but 8 x 1000
// 12.8 / 12.0, 64 x 2048 34.7 / 29.6).  Not where whole contexts put a workgroup of eight waves on more than half of the CUs (24 x 4000
// 30.0 / 26.3, 24 x 8000 47.9 / 43.5, 4 of window 64 x 4000 41.4 / 36.3).
void plan_kv4_attention(int num_seqs, int n_kv_heads, int rows, int max_context, int num_cus, int& splits, int& split_steps) {
  const int rb = rows > 16 ? 2 : 1;
  const int64_t wgs = (int64_t)num_seqs * n_kv_heads * ((rows + 16 * rb - 1) / (16 * rb));
  const int steps = (max_context + kStep - 1) / kStep;
  const int64_t want = (2LL * num_cus + wgs - 1) / wgs;
  int part = (int)((steps + want - 1) / want);
  part = (part < 8 ? 8 : part + kWaves - 1) / kWaves * kWaves;
  const bool whole = 2 * wgs > num_cus && wgs <= num_cus;
  const bool split = !whole && (steps + kWaves - 1) / kWaves - part / kWaves >= (2 * wgs < num_cus ? 6 : 8);
  split_steps = split ? part : steps;
  splits = (steps + split_steps - 1) / split_steps;
}

void launch_kv4_attention(const Attention4& a, hipStream_t st) {
  if (a.head_dim == 128) a.tiles ? launch<128, true>(a, st) : launch<128, false>(a, st);
  else a.tiles ? launch<64, true>(a, st) : launch<64, false>(a, st);
}
