// Products with 4-bit matrices, D[feature][token] = sum_k W[feature][k] X[token][k], W in MXFP4, X bf16, with the epilogues of the
// bf16 GEMMs.  The codes are converted to bf16 operands with their scales in registers - exactly, a 4-bit value times a
// power of two being a bf16 - and multiplied by v_mfma_f32_16x16x32_bf16, sums in fp32.
#include "gemm_parts.h"
#include "mx4.h"

using namespace gemm;
using mx4::u32x4;

namespace {

// Plain rows, for a product by itself.
template <bool F32>
struct PlainEpi {
  void* out;
  int64_t stride;
  int rows, n;
  bool wide;                // four values of a row can be stored at once
  struct Row {};
  struct Pre {};
  __device__ Row row_info(int) const { return Row{}; }
  __device__ Pre pre(int, int, int, const Row&) const { return Pre{}; }
  __device__ void operator()(int nb, int lane, int row, const f32x4 acc, const Pre&) const {
    const int f = nb * 16 + (lane >> 4) * 4;
    if (row >= rows || f >= n) return;
    const int64_t at = (int64_t)row * stride + f;
    if constexpr (F32) {
      float* p = (float*)out + at;
      if (wide && f + 4 <= n) *(f32x4*)p = acc;
      else
        for (int i = 0; i < 4 && f + i < n; ++i) p[i] = acc[i];
    } else {
      uint16_t* p = (uint16_t*)out + at;
      const u32x2 w = {pack2_bf16(acc[0], acc[1]), pack2_bf16(acc[2], acc[3])};
      if (wide && f + 4 <= n) *(u32x2*)p = w;
      else
        for (int i = 0; i < 4 && f + i < n; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
};

// Where the activations lie: the tile layout, or plain rows of `stride` elements.
struct X {
  const uint16_t* p;
  int64_t stride;           // 0: tiles
  int k_tiles, last_row;
  // what lane `lane` of token block `block` takes of k-tile 0, and from a k-tile to the next; rows that only pad repeat the last one
  __device__ const uint16_t* at(int block, int lane) const {
    const int row = min(block * 16 + (lane & 15), last_row);
    return stride ? p + (int64_t)row * stride + (lane >> 4) * 8
                  : p + ((size_t)(row >> 4) * k_tiles * 64 + (lane >> 4) * 16 + (row & 15)) * 8;
  }
  __device__ int step() const { return stride ? 32 : 512; }
};

// Few rows.  A workgroup owns FB feature blocks and TB token blocks; its eight waves take the records of 256 columns in turn, each with
// accumulators of its own for all of them, and are added through LDS.
constexpr int kStreamWaves = 8;
template <int FB, int TB, class Epi>
__global__ __launch_bounds__(64 * kStreamWaves) void mx4_stream_kernel(const char* __restrict__ w, X x, int n_blocks, int units, Epi epi) {
  constexpr int NW = kStreamWaves, ALL = FB * TB;
  __shared__ f32x4 part[NW][NW * 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n0 = blockIdx.x * FB, m0 = blockIdx.y * TB;
  const char* wp[FB];
#pragma unroll
  for (int i = 0; i < FB; ++i) wp[i] = w + (size_t)min(n0 + i, n_blocks - 1) * units * mx4::kRecord;
  const uint16_t* xp[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) xp[b] = x.at(m0 + b, lane);
  const int xs = x.step();
  f32x4 acc[FB][TB];
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[i][b] = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int u = wave; u < units; u += NW) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int k0 = u * 8 + half * 4;
      if (k0 >= x.k_tiles) break;
      u32x4 codes[FB];
      uint32_t scales[FB];
      bf16x8 xv[TB][4];
#pragma unroll
      for (int i = 0; i < FB; ++i) {
        const char* rec = wp[i] + (size_t)u * mx4::kRecord;
        codes[i] = *(const u32x4*)(rec + half * 1024 + lane * 16);
        scales[i] = *(const uint32_t*)(rec + mx4::kScales + (lane & 15) * 8 + half * 4);
      }
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[b][j] = *(const bf16x8*)(xp[b] + (size_t)min(k0 + j, x.k_tiles - 1) * xs);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k0 + j >= x.k_tiles) break;                // (columns that only pad: X has none there)
#pragma unroll
        for (int i = 0; i < FB; ++i) {
          const bf16x8 a = mx4::operand(codes[i][j], mx4::scale_of(scales[i], j));
#pragma unroll
          for (int b = 0; b < TB; ++b) acc[i][b] = mfma16(a, xv[b][j], acc[i][b]);
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < ALL; c += NW) {
    if (c) __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i)
      if (c + i < ALL) part[wave][i * 64 + lane] = acc[(c + i) / TB][(c + i) % TB];
    __syncthreads();
    const int at = c + wave, nb = n0 + at / TB;
    if (at < ALL && nb < n_blocks) {
      f32x4 sum = part[0][wave * 64 + lane];
#pragma unroll
      for (int v = 1; v < NW; ++v) sum += part[v][wave * 64 + lane];
      const int row = (m0 + at % TB) * 16 + (lane & 15);
      epi(nb, lane, row, sum, epi.pre(nb, lane, row, epi.row_info(row)));
    }
  }
}

template <class Epi>
void launch(const void* w, int n_blocks, const X& x, int rows, int num_cus, const Epi& epi, hipStream_t st) {
  const int units = (x.k_tiles + 7) / 8, blocks = (rows + 15) / 16;
  const char* wp = (const char*)w;
  const auto go = [&](auto fb, auto tb) {
    constexpr int FB = decltype(fb)::value, TB = decltype(tb)::value;
    mx4_stream_kernel<FB, TB, Epi><<<dim3((n_blocks + FB - 1) / FB, (blocks + TB - 1) / TB), 64 * kStreamWaves, 0, st>>>(wp, x, n_blocks, units, epi);
  };
  using std::integral_constant;
  const auto by_rows = [&](auto fb) {
    if (blocks == 1) go(fb, integral_constant<int, 1>{});
    else if (blocks == 2) go(fb, integral_constant<int, 2>{});
    else go(fb, integral_constant<int, 4>{});
  };
  if (n_blocks <= num_cus) by_rows(integral_constant<int, 1>{});
  else if (n_blocks <= 4 * num_cus) by_rows(integral_constant<int, 2>{});
  else by_rows(integral_constant<int, 4>{});
}

X tiles_of(const uint16_t* x, int k, const Workspace& ws) { return {x, 0, k / 32, ws.m_rows - 1}; }

}  // namespace

void launch_mx4_matmul(const void* w, int n, int k, const uint16_t* x, int64_t x_stride, int rows, void* out, int out_type,
                       int64_t out_stride, int num_cus, hipStream_t st) {
  const X xs{x, x_stride, (k + 31) / 32, rows - 1};
  const int n_blocks = (n + 15) / 16;
  if (out_type == LLM42_F32)
    launch(w, n_blocks, xs, rows, num_cus, PlainEpi<true>{out, out_stride, rows, n, (uintptr_t)out % 16 == 0 && out_stride % 4 == 0}, st);
  else
    launch(w, n_blocks, xs, rows, num_cus, PlainEpi<false>{out, out_stride, rows, n, (uintptr_t)out % 8 == 0 && out_stride % 4 == 0}, st);
}

void launch_mx4_qkv(const llm42_mx4_model* m4, int layer, const llm42_kv_cache* kv, const Workspace& ws, hipStream_t st) {
  const QkvEpi e = qkv_epilogue(m4->model, layer, kv, 1, ws);
  launch(m4->layers[layer].wqkv, m4->model->n_qkv / 16, tiles_of(ws.normed, m4->model->cfg.d_model, ws), ws.m_rows, ws.num_cus, e, st);
}

void launch_mx4_residual(const void* w, const uint16_t* x, int n, int k, const Workspace& ws, hipStream_t st) {
  launch(w, n / 16, tiles_of(x, k, ws), ws.m_rows, ws.num_cus, ResidualEpi{ws.resid, ws.rl, n}, st);
}

void launch_mx4_swiglu(const llm42_mx4_model* m4, int layer, const Workspace& ws, hipStream_t st) {
  const llm42_model* m = m4->model;
  launch(m4->layers[layer].wgu, m->gu_blocks, tiles_of(ws.normed, m->cfg.d_model, ws), ws.m_rows, ws.num_cus, SwigluEpi{ws.hidden, m->ffn_k}, st);
}

int launch_mx4_logits(const llm42_mx4_model* m4, const llm42_sampling* sampling, const Workspace& ws, hipStream_t st) {
  const llm42_model* m = m4->model;
  const int n_blocks = m->cfg.vocab / 16;
  const X x = tiles_of(ws.normed, m->cfg.d_model, ws);
  if (sampling && sampling->temperature > 0.f) {
    LogitsEpi<true> e = logits_epilogue<true>(m, 1, nullptr, sampling, ws);
    e.parts = n_blocks;
    launch(m4->lm_head, n_blocks, x, ws.m_rows, ws.num_cus, e, st);
  } else {
    LogitsEpi<false> e = logits_epilogue<false>(m, 1, nullptr, sampling, ws);
    e.parts = n_blocks;
    launch(m4->lm_head, n_blocks, x, ws.m_rows, ws.num_cus, e, st);
  }
  return n_blocks;
}
