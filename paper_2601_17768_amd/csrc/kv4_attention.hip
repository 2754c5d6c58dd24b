// Causal attention of the last positions of every sequence over the 4-bit cache.
#include "mx4.h"

using namespace mx4;

namespace {

// One workgroup per sequence, for a call that has no prepare pass of its own.
__global__ __launch_bounds__(64) void kv4_attention_check_kernel(const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ n_valid,
                                                                 int window, int max_context, const int32_t* __restrict__ table, int width,
                                                                 int64_t num_blocks, int32_t* __restrict__ seq_status,
                                                                 int32_t* __restrict__ ws_len, int32_t* __restrict__ ws_n) {
  const int s = blockIdx.x, lane = threadIdx.x;
  const int64_t len = seq_lens[s], n = n_valid ? n_valid[s] : window;
  int status = len < 0 || n < 0 || n > window || len + n > max_context ? LLM42_SEQ_BAD_LENGTH : LLM42_SEQ_OK;
  if (status == LLM42_SEQ_OK) {
    const int blocks = n ? (int)((len + n + LLM42_KV_BLOCK - 1) / LLM42_KV_BLOCK) : 0;   // (<= width: checked on the host)
    bool bad = false;
    for (int b = lane; b < blocks; b += 64) {
      const int id = table[(size_t)s * width + b];
      bad |= id < 0 || id >= num_blocks;
    }
    if (__any(bad)) status = LLM42_SEQ_BAD_BLOCK;
  }
  if (lane == 0) {
    if (seq_status) seq_status[s] = status;
    ws_len[s] = status == LLM42_SEQ_OK && n > 0 ? (int)len : -1;
    ws_n[s] = (int)n;
  }
}

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

constexpr int kWaves = 4;
constexpr int kStep = 64;   // keys

// The keys of one step as they come from memory: four blocks of 16 positions.
template <int HD>
struct Step {
  static constexpr int KT = HD / 32;
  uint32_t k[4][KT], v[4][KT], ks[4], vs[4][KT];
};

template <int HD>
__device__ __forceinline__ void load_words(uint32_t (&d)[HD / 32], const char* p) {
  if constexpr (HD == 128) {
    const u32x4 w = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = w[i];
  } else {
    const u32x2 w = *(const u32x2*)p;
    d[0] = w.x;
    d[1] = w.y;
  }
}

// Maximum / sum over the four lanes that hold a query row's keys (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A workgroup takes RB blocks of 16 query rows of a (sequence, kv head) over one of the parts of its context; its four waves take the
// part's steps of 64 keys in turn, each with a running maximum and sum of its own, and are joined through LDS.
//   scores: D[key][row] = K Q, K converted with its scales (exact in bf16);
//   weights: p = exp2((s - max) / sqrt(head_dim) log2 e) in fp32; D's layout is that of the P V operand, no exchange between lanes;
//   output: D[feature][row] = V P, V's codes converted with scale 1, V's scales - one per key and 32 features, and an operand holds 8 keys of
//   one feature - multiplied into p, before it is rounded to bf16.
template <int HD, int RB, bool TILES>
__global__ __launch_bounds__(64 * kWaves) void kv4_attention_kernel(Attention4 a, float scale_log2) {
  constexpr int KT = HD / 32, FB = HD / 16;
  __shared__ float sh_ml[kWaves][RB][2][16];
  __shared__ f32x4 sh_acc[kWaves][64 * FB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int rows_all = a.group * a.window, row_groups = (rows_all + 16 * RB - 1) / (16 * RB);
  int id = blockIdx.x;
  const int split = id % a.splits;
  id /= a.splits;
  const int rg = id % row_groups;
  id /= row_groups;
  const int kvh = id % a.n_kv_heads, s = id / a.n_kv_heads;
  const int len = a.seq_len[s];
  if (len < 0) return;
  const int n = a.seq_n ? a.seq_n[s] : a.window;
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
  f32x4 acc[RB][FB];
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
  auto load = [&](Step<HD>& d, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int blk = ids[min(step * 4 + t, last_block)];
      const char* rec = a.base + ((size_t)blk * a.n_kv_heads + kvh) * kv_record(HD);
      load_words<HD>(d.k[t], rec + lane * KT * 4);
      load_words<HD>(d.v[t], rec + 8 * HD + lane * KT * 4);
      d.ks[t] = KT == 4 ? *(const uint32_t*)(rec + 16 * HD + l16 * 4) : *(const uint16_t*)(rec + 16 * HD + l16 * 2);
      load_words<HD>(d.vs[t], rec + 16 * HD + HD / 2 + g * KT * 4);
    }
  };
  auto compute = [&](const Step<HD>& d, int step) __attribute__((always_inline)) {
    const bool edge = (step + 1) * kStep > len + 1;               // keys that some row does not see
    float p[RB][4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 sc[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[b] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        const bf16x8 k = operand(d.k[t][j], scale_of(d.ks[t], j));
#pragma unroll
        for (int b = 0; b < RB; ++b) sc[b] = mfma16(k, q[b][j], sc[b]);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[b][t][i] = sc[b][i];
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      if (edge) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (step * kStep + t * 16 + g * 4 + i >= limit[b]) p[b][t][i] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, p[b][t][i]);
      const float m_new = fmaxf(m[b], row_max(mx) * scale_log2);
      const float ref = m_new == -INFINITY ? 0.f : m_new;         // (nothing seen yet: every weight is 0)
      const float alpha = exp2f(m[b] - ref);
      m[b] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[b][t][i] = exp2f(fmaf(p[b][t][i], scale_log2, -ref));
          sum += p[b][t][i];
        }
      l[b] = l[b] * alpha + sum;
#pragma unroll
      for (int f = 0; f < FB; ++f) acc[b][f] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < 4; t += 2) {
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        bf16x8 pw[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          float w[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = p[b][t][i] * scale_of(d.vs[t][j], i);
            w[4 + i] = p[b][t + 1][i] * scale_of(d.vs[t + 1][j], i);
          }
          if (edge) {                                             // (whatever scale stands behind the last key)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (step * kStep + t * 16 + g * 4 + i >= limit[b]) w[i] = 0.f;
              if (step * kStep + t * 16 + 16 + g * 4 + i >= limit[b]) w[4 + i] = 0.f;
            }
          }
          u32x4 u;
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = pack2_bf16(w[2 * i], w[2 * i + 1]);
          pw[b] = __builtin_bit_cast(bf16x8, u);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int f = 2 * j + half;
          u32x4 u;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t w = d.v[t + x][j];
            u[2 * x] = __builtin_bit_cast(uint32_t, half ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2)
                                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
            u[2 * x + 1] = __builtin_bit_cast(uint32_t, half ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3)
                                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
          }
          const bf16x8 v = __builtin_bit_cast(bf16x8, u);
#pragma unroll
          for (int b = 0; b < RB; ++b) acc[b][f] = mfma16(v, pw[b], acc[b][f]);
        }
      }
    }
  };
  Step<HD> cur, next;
  if (begin + wave < end) load(cur, begin + wave);
  for (int step = begin + wave; step < end; step += kWaves) {
    load(next, min(step + kWaves, end - 1));
    compute(cur, step);
    cur = next;
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
    float top = -INFINITY, w[kWaves], sum = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) top = fmaxf(top, sh_ml[v][b][0][l16]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      w[v] = exp2f(sh_ml[v][b][0][l16] - ref);
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
    for (int f = wave; f < FB; f += kWaves) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < kWaves; ++v) o += sh_acc[v][f * 64 + lane] * w[v];
      if (a.splits > 1) {
        *(f32x4*)(a.part_acc + slot * HD + f * 16 + g * 4) = o;
        continue;
      }
      o /= sum;
      const u32x2 packed = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
      const int col = (kvh * a.group + h) * HD + f * 16 + g * 4;
      if constexpr (TILES) *(u32x2*)(a.out + pk_off(s, col, a.n_kv_heads * a.group * HD)) = packed;
      else *(u32x2*)(a.out + ((size_t)s * a.window + i) * a.out_stride + col) = packed;
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
  if (len < 0 || (a.seq_n && i >= a.seq_n[s])) return;
  const int n = a.seq_n ? a.seq_n[s] : a.window;
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
    const float w = exp2f(a.part_ml[2 * slot] - ref);
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
  if (rb == 1) kv4_attention_kernel<HD, 1, TILES><<<grid, 64 * kWaves, 0, st>>>(a, scale_log2);
  else if constexpr (!TILES) kv4_attention_kernel<HD, 2, TILES><<<grid, 64 * kWaves, 0, st>>>(a, scale_log2);
  if (a.splits > 1) {
    const int64_t all = (int64_t)a.num_seqs * a.n_kv_heads * rows;
    kv4_merge_kernel<HD, TILES><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a);
  }
}

}  // namespace

void launch_kv4_attention_check(const int32_t* seq_lens, const int32_t* n_valid, int window, int max_context, int num_seqs,
                                const llm42_kv_cache* kv4, int32_t* seq_status, int32_t* ws_len, int32_t* ws_n, hipStream_t st) {
  kv4_attention_check_kernel<<<num_seqs, 64, 0, st>>>(seq_lens, n_valid, window, max_context, kv4->block_table, kv4->max_blocks_per_seq,
                                                      kv4->num_blocks, seq_status, ws_len, ws_n);
}

void launch_kv4_step_check(const llm42_model* m, const llm42_kv_cache* kv4, int num_seqs, int32_t* seq_status, const Workspace& ws,
                           hipStream_t st) {
  kv4_step_check_kernel<<<num_seqs, 64, 0, st>>>(kv4->block_table, kv4->max_blocks_per_seq, kv4->num_blocks, seq_status, ws.seq_len,
                                                 ws.row_pos, ws.attn, m->d_attn);
}

// Parts of a context: as many as it takes to put four workgroups on every CU, none of fewer than four steps.
void plan_kv4_attention(int num_seqs, int n_kv_heads, int rows, int max_context, int num_cus, int& splits, int& split_steps) {
  const int rb = rows > 16 ? 2 : 1;
  const int64_t wgs = (int64_t)num_seqs * n_kv_heads * ((rows + 16 * rb - 1) / (16 * rb));
  const int steps = (max_context + kStep - 1) / kStep;
  int64_t want = (4LL * num_cus + wgs - 1) / wgs;
  if (want > (steps + kWaves - 1) / kWaves) want = (steps + kWaves - 1) / kWaves;
  if (want < 1) want = 1;
  split_steps = (int)((steps + want - 1) / want);
  split_steps = (split_steps + kWaves - 1) / kWaves * kWaves;
  splits = (steps + split_steps - 1) / split_steps;
}

void launch_kv4_attention(const Attention4& a, hipStream_t st) {
  if (a.head_dim == 128) a.tiles ? launch<128, true>(a, st) : launch<128, false>(a, st);
  else a.tiles ? launch<64, true>(a, st) : launch<64, false>(a, st);
}
