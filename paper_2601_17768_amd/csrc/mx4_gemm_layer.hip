// Products by the 4-bit matrices of a layer: QKV, residual projections, gate/up.
#include "mx4_gemm.h"

using namespace mx4;

void launch_mx4_qkv(const llm42_mx4_model* m4, int layer, const llm42_kv_cache* kv, const Workspace& ws, hipStream_t st) {
  const QkvEpi e = qkv_epilogue(m4->model, layer, kv, 1, ws);
  const int n_blocks = m4->model->n_qkv / 16, k = m4->model->cfg.d_model;
  launch(plan(n_blocks, k / 32, ws.m_rows, ws.num_cus, 1), m4->layers[layer].wqkv, n_blocks, tiles_of(ws.normed, k, ws), ws.m_rows, e, st);
}

// x + the parts of a split product, first to last, over the rows of the pass.
__global__ __launch_bounds__(256) static void mx4_add_parts_kernel(float* __restrict__ x, const float* __restrict__ parts, int count, size_t plane,
                                                                   size_t quads) {
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= quads) return;
  f32x4 sum = *(const f32x4*)(parts + at * 4);
  for (int p = 1; p < count; ++p) sum += *(const f32x4*)(parts + p * plane + at * 4);
  *(f32x4*)(x + at * 4) = *(const f32x4*)(x + at * 4) + sum;
}

bool launch_mx4_residual(const void* w, const uint16_t* x, int n, int k, float* parts, const Workspace& ws, hipStream_t st) {
  const bool joined = norm_adds_halves(ws.m_pad, n);
  const Plan p = plan(n / 16, k / 32, ws.m_rows, ws.num_cus, mx4_residual_parts(ws.m_rows), joined);
  const size_t plane = (size_t)ws.m_pad * n;
  if (p.parts == 1) {
    launch(p, w, n / 16, tiles_of(x, k, ws), ws.m_rows, ResidualEpi{ws.resid, ws.rl, n}, st);
    return false;
  }
  const bool halves = joined && p.parts == 2;
  launch(p, w, n / 16, tiles_of(x, k, ws), ws.m_rows, StorePartialEpi{halves ? ws.split_part : parts, ws.rl, n, plane}, st);
  if (!halves) {
    const size_t quads = (size_t)((ws.m_rows + 15) / 16) * 16 * n / 4;      // (whole blocks of rows in either layout of the stream)
    mx4_add_parts_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(ws.resid, parts, p.parts, plane, quads);
  }
  return halves;
}

void launch_mx4_swiglu(const llm42_mx4_model* m4, int layer, const Workspace& ws, hipStream_t st) {
  const llm42_model* m = m4->model;
  launch(plan(m->gu_blocks, m->cfg.d_model / 32, ws.m_rows, ws.num_cus, 1), m4->layers[layer].wgu, m->gu_blocks,
         tiles_of(ws.normed, m->cfg.d_model, ws), ws.m_rows, SwigluEpi{ws.hidden, m->ffn_k}, st);
}
