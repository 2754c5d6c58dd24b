// C ABI of the operators around the paged bf16 cache (declared in include/llm42_paged.h): host-side validation.
#include <cmath>
#include <new>

#include "paged.h"

using namespace paged;

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

llm42_status launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LLM42_OK : fail(LLM42_EHIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

llm42_status check_heads(const char* who, const llm42_heads* h) {
  if (!h) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (h->n_layers < 1 || h->n_layers > 65535 || h->n_q_heads < 1 || h->n_q_heads > 1024 || h->n_kv_heads < 1)
    return fail(LLM42_EINVAL, "%s: heads: 1..65535 layers, 1..1024 query heads and 1 or more kv heads", who);
  if (h->head_dim != 64 && h->head_dim != 128) return fail(LLM42_ESHAPE, "%s: head_dim must be 64 or 128", who);
  if (h->n_q_heads % h->n_kv_heads || h->n_q_heads / h->n_kv_heads > 16)
    return fail(LLM42_ESHAPE, "%s: n_q_heads must be 1..16 times n_kv_heads", who);
  return LLM42_OK;
}

llm42_status check_layer(const char* who, const llm42_heads* h, int32_t layer, bool all) {
  if (layer < (all ? -1 : 0) || layer >= h->n_layers) return fail(LLM42_EINVAL, "%s: layer must be %d..%d", who, all ? -1 : 0, h->n_layers - 1);
  return LLM42_OK;
}

llm42_status check_cache(const char* who, const llm42_kv_cache* kv, bool base) {
  if (!kv || !kv->block_table || kv->num_blocks < 1 || kv->num_blocks > 0x7FFFFFFF || kv->max_blocks_per_seq < 1 ||
      (base && (!kv->kv_base || (uintptr_t)kv->kv_base % 16)))
    return fail(LLM42_EINVAL, "%s: bad kv_cache view", who);
  return LLM42_OK;
}

llm42_status check_shape(const char* who, int32_t num_seqs, int32_t window, int32_t max_context) {
  if (window < 1 || window > LLM42_MAX_WINDOW) return fail(LLM42_EINVAL, "%s: window must be 1..%d", who, LLM42_MAX_WINDOW);
  if (num_seqs < 1 || (int64_t)num_seqs * window > LLM42_MAX_ROWS)
    return fail(LLM42_EINVAL, "%s: num_seqs * window must be 1..%d", who, LLM42_MAX_ROWS);
  if (max_context < 1 || max_context > kMostContextPaged) return fail(LLM42_EINVAL, "%s: max_context must be 1..%d", who, kMostContextPaged);
  return LLM42_OK;
}

llm42_status check_rows(const char* who, const llm42_kv_cache* kv, const int32_t* seq_lens, int32_t num_seqs, int32_t window, int32_t max_context) {
  if (!seq_lens) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (llm42_status st = check_shape(who, num_seqs, window, max_context)) return st;
  if ((int64_t)max_context > (int64_t)kv->max_blocks_per_seq * LLM42_KV_BLOCK)
    return fail(LLM42_ECAPACITY, "%s: max_context %d exceeds block-table capacity %lld", who, max_context,
                (long long)kv->max_blocks_per_seq * LLM42_KV_BLOCK);
  return LLM42_OK;
}

// Plain rows of `heads` heads, elements of `size` bytes.
llm42_status check_plain(const char* who, const char* name, const void* p, int64_t stride, int heads, int head_dim, int size) {
  if (!p) return fail(LLM42_EINVAL, "%s: null argument", who);
  if ((uintptr_t)p % 16 || stride % (16 / size) || stride < (int64_t)heads * head_dim)
    return fail(LLM42_EINVAL, "%s: %s needs 16-byte aligned rows of at least %d", who, name, heads * head_dim);
  return LLM42_OK;
}

Rows rows_of(const llm42_kv_cache* kv, const int32_t* seq_lens, int32_t window, const int32_t* n_valid, int32_t num_seqs, int32_t max_context) {
  return {kv->block_table, kv->max_blocks_per_seq, kv->num_blocks, seq_lens, n_valid, num_seqs, window, max_context};
}

// A K or V plane of a cache, and the bounds of a layer.
int64_t plane_of(const llm42_heads* h, int64_t num_blocks) { return num_blocks * h->n_kv_heads * 16 * h->head_dim; }
const uint16_t* k_plane_of(const llm42_heads* h, const llm42_kv_cache* kv, int32_t layer) {
  return (const uint16_t*)kv->kv_base + 2 * layer * plane_of(h, kv->num_blocks);
}
int64_t bounds_of(const llm42_heads* h, int64_t num_blocks) { return num_blocks * h->n_kv_heads * bounds_record(h->head_dim); }

// Frequencies of the pairs, scaled.
void frequencies(const llm42_rope_config& c, double* f) {
  const int half = c.rot_dim / 2;
  const double two_pi = 6.283185307179586476925286766559, n = c.original_max_position;
  double lo = 0, hi = 0;
  if (c.scaling == LLM42_ROPE_YARN) {
    const auto at = [&](double turns) { return c.rot_dim * std::log(n / (turns * two_pi)) / (2 * std::log(c.theta)); };
    lo = std::fmax(0.0, std::floor(at(c.beta_fast)));
    hi = std::fmin(c.rot_dim - 1.0, std::ceil(at(c.beta_slow)));
    if (hi == lo) hi += 0.001;
  }
  for (int j = 0; j < half; ++j) {
    const double x = std::pow(c.theta, -2.0 * j / c.rot_dim);
    const auto clamp = [](double v) { return v < 0 ? 0.0 : v > 1 ? 1.0 : v; };
    if (c.scaling == LLM42_ROPE_LINEAR) f[j] = x / c.factor;
    else if (c.scaling == LLM42_ROPE_LLAMA3) {
      const double keep = clamp((n * x / two_pi - c.low_freq_factor) / (c.high_freq_factor - c.low_freq_factor));
      f[j] = x * (keep + (1 - keep) / c.factor);
    } else if (c.scaling == LLM42_ROPE_YARN) {
      const double ramp = clamp((j - lo) / (hi - lo));
      f[j] = x * (1 - ramp) + x / c.factor * ramp;
    } else f[j] = x;
  }
}

llm42_status check_workspace(const char* who, const void* workspace, size_t bytes, size_t need) {
  if (need && (!workspace || (uintptr_t)workspace % 256)) return fail(LLM42_EWORKSPACE, "%s: the call needs a workspace, 256-byte aligned", who);
  if (bytes < need) return fail(LLM42_EWORKSPACE, "%s: workspace %zu < %zu bytes", who, bytes, need);
  return LLM42_OK;
}

llm42_status check_budget(const char* who, int32_t budget) {
  if (budget < 1 || budget > LLM42_MAX_SELECTED) return fail(LLM42_EINVAL, "%s: a list has 1..%d blocks", who, LLM42_MAX_SELECTED);
  return LLM42_OK;
}

}  // namespace

paged::SparseWorkspace paged::carve_sparse(int rows, int n_kv_heads, int group, int head_dim, int parts, char* base) {
  SparseWorkspace w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off = align_up(off + bytes, 256);
    return p;
  };
  const size_t lists = parts > 1 ? (size_t)rows * n_kv_heads * parts : 0, slots = lists * group;
  w.ok = (int32_t*)take(4 * lists);
  w.acc = (float*)take(4 * slots * head_dim);
  w.ml = (float*)take(8 * slots);
  w.bytes = off;
  return w;
}

extern "C" {

llm42_status llm42_heads_kv_bytes(const llm42_heads* h, int64_t num_blocks, size_t* out_bytes) {
  const char* who = "heads_kv_bytes";
  if (llm42_status st = check_heads(who, h)) return st;
  if (!out_bytes || num_blocks < 0 || num_blocks > 0x7FFFFFFF) return fail(LLM42_EINVAL, "%s: bad argument", who);
  *out_bytes = (size_t)h->n_layers * 2 * plane_of(h, num_blocks) * 2;
  return LLM42_OK;
}

llm42_status llm42_model_heads(const llm42_model* m, llm42_heads* out) {
  if (!m || !out) return fail(LLM42_EINVAL, "model_heads: null argument");
  *out = {m->cfg.n_layers, m->cfg.n_q_heads, m->cfg.n_kv_heads, m->cfg.head_dim};
  return LLM42_OK;
}

llm42_status llm42_rope_create(const llm42_rope_config* cfg, llm42_rope** out) {
  const char* who = "rope_create";
  if (!cfg || !out) return fail(LLM42_EINVAL, "%s: null argument", who);
  *out = nullptr;
  const llm42_rope_config& c = *cfg;
  if (c.rot_dim < 2 || c.rot_dim > 128 || c.rot_dim % 2) return fail(LLM42_EINVAL, "%s: rot_dim must be even, 2..128", who);
  if (c.layout != LLM42_ROPE_HALF && c.layout != LLM42_ROPE_INTERLEAVED) return fail(LLM42_EINVAL, "%s: unknown layout %d", who, c.layout);
  if (c.scaling < LLM42_ROPE_NONE || c.scaling > LLM42_ROPE_YARN) return fail(LLM42_EINVAL, "%s: unknown scaling %d", who, c.scaling);
  if (c.max_position < 1 || c.max_position > (1 << 24)) return fail(LLM42_EINVAL, "%s: max_position must be 1..%d", who, 1 << 24);
  if (!(c.theta > 1) || !std::isfinite(c.theta)) return fail(LLM42_EINVAL, "%s: theta must be above 1", who);
  if (!(c.attention_factor >= 0) || !std::isfinite(c.attention_factor)) return fail(LLM42_EINVAL, "%s: bad attention_factor", who);
  if (c.scaling != LLM42_ROPE_NONE && (!(c.factor >= 1) || !std::isfinite(c.factor))) return fail(LLM42_EINVAL, "%s: factor must be 1 or more", who);
  if (c.scaling >= LLM42_ROPE_LLAMA3 && c.original_max_position < 1) return fail(LLM42_EINVAL, "%s: original_max_position must be positive", who);
  if (c.scaling == LLM42_ROPE_LLAMA3 && (!(c.low_freq_factor > 0) || !(c.high_freq_factor > c.low_freq_factor) || !std::isfinite(c.high_freq_factor)))
    return fail(LLM42_EINVAL, "%s: 0 < low_freq_factor < high_freq_factor", who);
  if (c.scaling == LLM42_ROPE_YARN && (!(c.beta_slow > 0) || !(c.beta_fast >= c.beta_slow) || !std::isfinite(c.beta_fast)))
    return fail(LLM42_EINVAL, "%s: 0 < beta_slow <= beta_fast", who);
  const double factor = c.attention_factor > 0 ? c.attention_factor : c.scaling == LLM42_ROPE_YARN ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
  const int half = c.rot_dim / 2;
  double freq[64];
  frequencies(c, freq);
  llm42_rope* r = new (std::nothrow) llm42_rope();
  if (!r) return fail(LLM42_EHIP, "%s: out of host memory", who);
  r->rot_dim = c.rot_dim;
  r->layout = c.layout;
  r->max_position = c.max_position;
  r->table = nullptr;
  const size_t bytes = sizeof(float2) * (size_t)half * c.max_position;
  double* dev = nullptr;
  hipError_t e = hipGetDevice(&r->device);
  if (e == hipSuccess) e = hipMalloc((void**)&r->table, bytes);
  if (e == hipSuccess) e = hipMalloc((void**)&dev, sizeof freq);
  if (e == hipSuccess) e = hipMemcpy(dev, freq, sizeof(double) * half, hipMemcpyHostToDevice);
  if (e == hipSuccess) {
    launch_rope_table(dev, factor, half, c.max_position, r->table, nullptr);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
  if (dev) (void)hipFree(dev);
  if (e != hipSuccess) {
    llm42_rope_destroy(r);
    return fail(LLM42_EHIP, "%s: %s", who, hipGetErrorString(e));
  }
  *out = r;
  return LLM42_OK;
}

void llm42_rope_destroy(llm42_rope* r) {
  if (!r) return;
  if (r->table) (void)hipFree(r->table);
  delete r;
}

llm42_status llm42_kv_append(const llm42_heads* heads, int32_t layer, const llm42_kv_cache* kv, void* kv_bounds, const void* q, int64_t q_stride,
                             const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t type, const void* q_norm,
                             const void* k_norm, float norm_eps, const llm42_rope* rope, const int32_t* seq_lens, int32_t window,
                             const int32_t* n_valid, int32_t num_seqs, int32_t max_context, void* q_out, int64_t q_out_stride,
                             int32_t* seq_status, void* hip_stream) {
  const char* who = "kv_append";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (llm42_status st = check_layer(who, heads, layer, false)) return st;
  if (llm42_status st = check_cache(who, kv, true)) return st;
  if (llm42_status st = check_rows(who, kv, seq_lens, num_seqs, window, max_context)) return st;
  if (type != LLM42_BF16 && type != LLM42_F32) return fail(LLM42_EINVAL, "%s: unknown element type %d", who, type);
  const int size = type == LLM42_F32 ? 4 : 2, hd = heads->head_dim;
  if (llm42_status st = check_plain(who, "k", k, k_stride, heads->n_kv_heads, hd, size)) return st;
  if (llm42_status st = check_plain(who, "v", v, v_stride, heads->n_kv_heads, hd, size)) return st;
  if (!q != !q_out) return fail(LLM42_EINVAL, "%s: q and q_out go together", who);
  if (q) {
    if (llm42_status st = check_plain(who, "q", q, q_stride, heads->n_q_heads, hd, size)) return st;
    if (llm42_status st = check_plain(who, "q_out", q_out, q_out_stride, heads->n_q_heads, hd, 2)) return st;
  }
  if ((uintptr_t)q_norm % 16 || (uintptr_t)k_norm % 16 || (uintptr_t)kv_bounds % 16)
    return fail(LLM42_EINVAL, "%s: gains and bounds must be 16-byte aligned", who);
  if (!(norm_eps >= 0.f)) return fail(LLM42_EINVAL, "%s: norm_eps must not be negative", who);
  if (rope) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != rope->device)
      return fail(LLM42_EINVAL, "%s: the rotary table lives on device %d, current device is %d", who, rope->device, dev);
    if (rope->rot_dim > hd) return fail(LLM42_EINVAL, "%s: rot_dim %d exceeds head_dim %d", who, rope->rot_dim, hd);
    if (max_context > rope->max_position)
      return fail(LLM42_ECAPACITY, "%s: max_context %d exceeds the rotary table's %d positions", who, max_context, rope->max_position);
  }
  if ((int64_t)num_seqs * (window / 16 + 2) * heads->n_kv_heads > (1 << 24))
    return fail(LLM42_EINVAL, "%s: num_seqs * (window / 16 + 2) * n_kv_heads too large", who);
  Append a;
  a.rows = rows_of(kv, seq_lens, window, n_valid, num_seqs, max_context);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.q_norm = (const uint16_t*)q_norm;
  a.k_norm = (const uint16_t*)k_norm;
  a.eps = norm_eps;
  a.rope = rope ? rope->table : nullptr;
  a.rot_dim = rope ? rope->rot_dim : 0;
  a.layout = rope ? rope->layout : LLM42_ROPE_HALF;
  a.q_out = (uint16_t*)q_out;
  a.k_plane = const_cast<uint16_t*>(k_plane_of(heads, kv, layer));
  a.v_plane = a.k_plane + plane_of(heads, kv->num_blocks);
  a.bounds = kv_bounds ? (char*)kv_bounds + layer * bounds_of(heads, kv->num_blocks) : nullptr;
  a.n_q_heads = heads->n_q_heads;
  a.n_kv_heads = heads->n_kv_heads;
  a.head_dim = hd;
  a.type = type;
  a.seq_status = seq_status;
  launch_kv_append(a, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv_bounds_bytes(const llm42_heads* heads, int64_t num_blocks, size_t* out_bytes) {
  const char* who = "kv_bounds_bytes";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (!out_bytes || num_blocks < 0 || num_blocks > 0x7FFFFFFF) return fail(LLM42_EINVAL, "%s: bad argument", who);
  *out_bytes = (size_t)heads->n_layers * bounds_of(heads, num_blocks);
  return LLM42_OK;
}

llm42_status llm42_kv_bounds_store(const llm42_heads* heads, int32_t layer, const llm42_kv_cache* kv, void* kv_bounds, const int32_t* first,
                                   const int32_t* count, int32_t num_seqs, int32_t max_count, int32_t* seq_status, void* hip_stream) {
  const char* who = "kv_bounds_store";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (llm42_status st = check_layer(who, heads, layer, true)) return st;
  if (llm42_status st = check_cache(who, kv, true)) return st;
  if (!kv_bounds || !first || !count) return fail(LLM42_EINVAL, "%s: null argument", who);
  if ((uintptr_t)kv_bounds % 16) return fail(LLM42_EINVAL, "%s: bounds must be 16-byte aligned", who);
  if (num_seqs < 1 || max_count < 1) return fail(LLM42_EINVAL, "%s: num_seqs and max_count must be positive", who);
  // (below 2^26 waves: four of them are a workgroup of 256 threads, of which a launch takes fewer than 2^32)
  if ((int64_t)num_seqs * (((int64_t)max_count + 14) / 16 + 1) > ((1 << 26) - 1) / heads->n_kv_heads)
    return fail(LLM42_EINVAL, "%s: num_seqs * max_count too large", who);
  const int from = layer < 0 ? 0 : layer;
  launch_bounds_store(layer < 0 ? heads->n_layers : 1, heads->n_kv_heads, heads->head_dim, k_plane_of(heads, kv, from),
                      2 * plane_of(heads, kv->num_blocks), (char*)kv_bounds + from * bounds_of(heads, kv->num_blocks), kv->block_table,
                      kv->max_blocks_per_seq, kv->num_blocks, first, count, num_seqs, max_count, seq_status, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv_bounds_read(const llm42_heads* heads, const void* kv_bounds, int64_t num_blocks, const int32_t* block_ids, int32_t num_ids,
                                  void* out_lo, void* out_hi, void* hip_stream) {
  const char* who = "kv_bounds_read";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (num_ids < 0 || num_blocks < 1 || num_blocks > 0x7FFFFFFF || (int64_t)num_ids * heads->n_kv_heads > (1 << 27))
    return fail(LLM42_EINVAL, "%s: num_blocks / num_ids out of range", who);
  if (num_ids == 0) return LLM42_OK;
  if (!kv_bounds || !block_ids || !out_lo || !out_hi) return fail(LLM42_EINVAL, "%s: null argument", who);
  if ((uintptr_t)kv_bounds % 16 || (uintptr_t)out_lo % 16 || (uintptr_t)out_hi % 16)
    return fail(LLM42_EINVAL, "%s: bounds, out_lo and out_hi must be 16-byte aligned", who);
  launch_bounds_read(heads->n_layers, heads->n_kv_heads, heads->head_dim, (const char*)kv_bounds, num_blocks, block_ids, num_ids,
                     (uint16_t*)out_lo, (uint16_t*)out_hi, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv_select_workspace_bytes(const llm42_heads* heads, int32_t num_seqs, int32_t window, int32_t max_context, int32_t budget,
                                             size_t* out_bytes) {
  const char* who = "kv_select_workspace_bytes";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (!out_bytes) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (llm42_status st = check_shape(who, num_seqs, window, max_context)) return st;
  if (llm42_status st = check_budget(who, budget)) return st;
  *out_bytes = select_workspace(num_seqs, window, heads->n_kv_heads, heads->n_q_heads / heads->n_kv_heads, max_context, budget, current_cus());
  return LLM42_OK;
}

llm42_status llm42_kv_select(const llm42_heads* heads, int32_t layer, const llm42_kv_cache* kv, const void* kv_bounds, const void* q,
                             int64_t q_stride, const int32_t* seq_lens, int32_t window, const int32_t* n_valid, int32_t num_seqs,
                             int32_t max_context, int32_t budget, int32_t sink, int32_t recent, int32_t* selected, int32_t* seq_status,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "kv_select";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (llm42_status st = check_layer(who, heads, layer, false)) return st;
  if (llm42_status st = check_cache(who, kv, false)) return st;
  if (llm42_status st = check_rows(who, kv, seq_lens, num_seqs, window, max_context)) return st;
  if (llm42_status st = check_plain(who, "q", q, q_stride, heads->n_q_heads, heads->head_dim, 2)) return st;
  if (llm42_status st = check_budget(who, budget)) return st;
  if (sink < 0 || recent < 1 || (int64_t)sink + recent > budget)
    return fail(LLM42_EINVAL, "%s: sink and recent must be at least 0 and 1, and no more than the budget together", who);
  if (!kv_bounds || !selected) return fail(LLM42_EINVAL, "%s: null argument", who);
  if ((uintptr_t)kv_bounds % 16) return fail(LLM42_EINVAL, "%s: bounds must be 16-byte aligned", who);
  Select a;
  a.rows = rows_of(kv, seq_lens, window, n_valid, num_seqs, max_context);
  a.bounds = (const char*)kv_bounds + layer * bounds_of(heads, kv->num_blocks);
  a.q = (const uint16_t*)q;
  a.q_stride = q_stride;
  a.tiles = false;
  a.n_kv_heads = heads->n_kv_heads;
  a.group = heads->n_q_heads / heads->n_kv_heads;
  a.head_dim = heads->head_dim;
  a.budget = budget;
  a.sink = sink;
  a.recent = recent;
  a.selected = selected;
  a.seq_status = seq_status;
  a.num_cus = current_cus();
  const size_t need = select_workspace(num_seqs, window, a.n_kv_heads, a.group, max_context, budget, a.num_cus);
  if (llm42_status st = check_workspace(who, workspace, workspace_bytes, need)) return st;
  a.keys = need ? (uint32_t*)workspace : nullptr;
  launch_kv_select(a, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv_sparse_attention_workspace_bytes(const llm42_heads* heads, int32_t num_seqs, int32_t window, int32_t width,
                                                       size_t* out_bytes) {
  const char* who = "kv_sparse_attention_workspace_bytes";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (!out_bytes) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (llm42_status st = check_shape(who, num_seqs, window, 1)) return st;
  if (llm42_status st = check_budget(who, width)) return st;
  int parts, per_part;
  plan_sparse_attention(num_seqs * window, heads->n_kv_heads, heads->head_dim, width, current_cus(), parts, per_part);
  *out_bytes = carve_sparse(num_seqs * window, heads->n_kv_heads, heads->n_q_heads / heads->n_kv_heads, heads->head_dim, parts, nullptr).bytes;
  return LLM42_OK;
}

llm42_status llm42_kv_sparse_attention(const llm42_heads* heads, int32_t layer, const llm42_kv_cache* kv, const void* q, int64_t q_stride,
                                       const int32_t* seq_lens, int32_t window, const int32_t* n_valid, int32_t num_seqs, int32_t max_context,
                                       const int32_t* selected, int32_t width, float scale, void* out, int64_t out_stride, int32_t* seq_status,
                                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "kv_sparse_attention";
  if (llm42_status st = check_heads(who, heads)) return st;
  if (llm42_status st = check_layer(who, heads, layer, false)) return st;
  if (llm42_status st = check_cache(who, kv, true)) return st;
  if (llm42_status st = check_rows(who, kv, seq_lens, num_seqs, window, max_context)) return st;
  if (llm42_status st = check_plain(who, "q", q, q_stride, heads->n_q_heads, heads->head_dim, 2)) return st;
  if (llm42_status st = check_plain(who, "out", out, out_stride, heads->n_q_heads, heads->head_dim, 2)) return st;
  if (llm42_status st = check_budget(who, width)) return st;
  if (!selected) return fail(LLM42_EINVAL, "%s: null argument", who);
  // (it is multiplied by log2 e, which must stay finite: a score of 0 counts whatever the scale)
  if (!(scale >= 0.f) || scale > 0x1p126f) return fail(LLM42_EINVAL, "%s: scale must be 0..2^126", who);
  SparseAttention a;
  a.rows = rows_of(kv, seq_lens, window, n_valid, num_seqs, max_context);
  a.k_plane = k_plane_of(heads, kv, layer);
  a.v_plane = a.k_plane + plane_of(heads, kv->num_blocks);
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.tiles = false;
  a.n_kv_heads = heads->n_kv_heads;
  a.group = heads->n_q_heads / heads->n_kv_heads;
  a.head_dim = heads->head_dim;
  a.selected = selected;
  a.width = width;
  a.scale = scale;
  a.seq_status = seq_status;
  a.num_cus = current_cus();
  plan_sparse_attention(num_seqs * window, a.n_kv_heads, a.head_dim, width, a.num_cus, a.parts, a.per_part);
  const SparseWorkspace ws = carve_sparse(num_seqs * window, a.n_kv_heads, a.group, a.head_dim, a.parts, (char*)workspace);
  if (llm42_status st = check_workspace(who, workspace, workspace_bytes, a.parts > 1 ? ws.bytes : 0)) return st;
  a.part_acc = ws.acc;
  a.part_ml = ws.ml;
  a.part_ok = ws.ok;
  launch_sparse_attention(a, (hipStream_t)hip_stream);
  return launched(who);
}

}  // extern "C"
