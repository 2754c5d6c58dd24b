// Product by the 4-bit LM head.
#include "mx4_gemm.h"

using namespace mx4;

int launch_mx4_logits(const llm42_mx4_model* m4, const llm42_sampling* sampling, const Workspace& ws, hipStream_t st) {
  const llm42_model* m = m4->model;
  const int n_blocks = m->cfg.vocab / 16;
  const X x = tiles_of(ws.normed, m->cfg.d_model, ws);
  const Plan p = plan(n_blocks, x.k_tiles, ws.m_rows, ws.num_cus, 1);
  if (sampling && sampling->temperature > 0.f)
    return launch(p, m4->lm_head, n_blocks, x, ws.m_rows, logits_epilogue<true>(m, 1, nullptr, sampling, ws), st);
  return launch(p, m4->lm_head, n_blocks, x, ws.m_rows, logits_epilogue<false>(m, 1, nullptr, sampling, ws), st);
}
