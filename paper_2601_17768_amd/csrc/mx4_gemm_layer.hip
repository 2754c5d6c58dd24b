// Products by the 4-bit matrices of a layer: QKV, residual projections, gate/up.
#include "mx4_gemm.h"

using namespace mx4;

void launch_mx4_qkv(const llm42_mx4_model* m4, int layer, const llm42_kv_cache* kv, const Workspace& ws, hipStream_t st) {
  const QkvEpi e = qkv_epilogue(m4->model, layer, kv, 1, ws);
  const int n_blocks = m4->model->n_qkv / 16, k = m4->model->cfg.d_model;
  launch(plan(n_blocks, k / 32, ws.m_rows, ws.num_cus, 1), m4->layers[layer].wqkv, n_blocks, tiles_of(ws.normed, k, ws), ws.m_rows, e, st);
}

bool launch_mx4_residual(const void* w, const uint16_t* x, int n, int k, const Workspace& ws, hipStream_t st) {
  const Plan p = plan(n / 16, k / 32, ws.m_rows, ws.num_cus, norm_adds_halves(ws.m_pad, n) ? 2 : 1, true);
  if (p.parts == 2) launch(p, w, n / 16, tiles_of(x, k, ws), ws.m_rows, StorePartialEpi{ws.split_part, ws.rl, n, (size_t)ws.m_pad * n}, st);
  else launch(p, w, n / 16, tiles_of(x, k, ws), ws.m_rows, ResidualEpi{ws.resid, ws.rl, n}, st);
  return p.parts == 2;
}

void launch_mx4_swiglu(const llm42_mx4_model* m4, int layer, const Workspace& ws, hipStream_t st) {
  const llm42_model* m = m4->model;
  launch(plan(m->gu_blocks, m->cfg.d_model / 32, ws.m_rows, ws.num_cus, 1), m4->layers[layer].wgu, m->gu_blocks,
         tiles_of(ws.normed, m->cfg.d_model, ws), ws.m_rows, SwigluEpi{ws.hidden, m->ffn_k}, st);
}
