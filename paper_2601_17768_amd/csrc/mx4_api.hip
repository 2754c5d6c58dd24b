// C ABI of the 4-bit operators (declared in include/llm42_mx4.h): host-side validation.  The calls that belong to a model's passes are
// in api.hip.
#include <atomic>

#include "mx4.h"

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Largest matrix: index arithmetic in 32 bits stays in range below it.
constexpr int32_t kMostRows = 1 << 30, kMostCols = 1 << 26;

bool known_type(int32_t t) { return t == LLM42_BF16 || t == LLM42_F32; }
size_t size_of(int32_t t) { return t == LLM42_F32 ? 4 : 2; }

llm42_status launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LLM42_OK : fail(LLM42_EHIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

// What quantize and dequantize ask of a matrix and of the plain array beside it.
llm42_status check_matrix(const char* who, const void* packed, size_t bytes, int32_t rows, int32_t cols, const void* plain, int32_t type,
                          int64_t stride) {
  if (!packed || !plain) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (rows < 1 || cols < 1 || rows > kMostRows || cols > kMostCols)
    return fail(LLM42_EINVAL, "%s: a matrix has 1..%d rows and 1..%d columns", who, kMostRows, kMostCols);
  if (!known_type(type)) return fail(LLM42_EINVAL, "%s: unknown element type %d", who, type);
  if (stride < cols) return fail(LLM42_EINVAL, "%s: stride %lld is less than cols", who, (long long)stride);
  if ((uintptr_t)plain % size_of(type)) return fail(LLM42_EINVAL, "%s: plain array not aligned to its type", who);
  if ((uintptr_t)packed % 16) return fail(LLM42_EINVAL, "%s: 4-bit matrix not 16-byte aligned", who);
  const size_t need = mx4::matrix_bytes(rows, cols);
  if (need / mx4::kRecord > 4 * kMostGroups256) return fail(LLM42_EINVAL, "%s: a matrix of more than %u records of 16 x 256", who, 4 * kMostGroups256);
  if (bytes < need) return fail(LLM42_EWORKSPACE, "%s: 4-bit matrix of %zu < %zu bytes", who, bytes, need);
  return LLM42_OK;
}

size_t packed_x_bytes(int rows, int k) { return align_up(2 * align_up(rows, 16) * align_up(k, 32), 256); }

llm42_status check_cache(const char* who, const char* name, const llm42_kv_cache* kv) {
  if (!kv || !kv->kv_base || !kv->block_table || kv->num_blocks < 1 || kv->max_blocks_per_seq < 1 || (uintptr_t)kv->kv_base % 16)
    return fail(LLM42_EINVAL, "%s: bad %s view", who, name);
  return LLM42_OK;
}

llm42_status check_ranges(const char* who, const llm42_model* m, const int32_t* first, const int32_t* count, int32_t num_seqs,
                          int32_t max_count) {
  if (!m || !first || !count) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (num_seqs < 1 || max_count < 1) return fail(LLM42_EINVAL, "%s: num_seqs and max_count must be positive", who);
  if (m->cfg.n_layers > 65535 || (int64_t)num_seqs * (((int64_t)max_count + 14) / 16 + 1) > 0x7FFFFFFF / ((m->cfg.n_kv_heads + 3) / 4))
    return fail(LLM42_EINVAL, "%s: num_seqs * max_count too large", who);
  return LLM42_OK;
}

// Workspace of llm42_kv4_attention: partials, and the rows that those of a sequence hold.
struct Attention4Workspace {
  int32_t* n;
  float *acc, *ml;
  size_t bytes;
};
Attention4Workspace carve(const llm42_model* m, int num_seqs, int window, int splits, char* base) {
  Attention4Workspace w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off = align_up(off + bytes, 256);
    return p;
  };
  w.n = (int32_t*)take(4ull * num_seqs * m->cfg.n_kv_heads);
  const size_t slots = splits > 1 ? (size_t)num_seqs * m->cfg.n_kv_heads * splits * m->group * window : 0;
  w.acc = (float*)take(4 * slots * m->cfg.head_dim);
  w.ml = (float*)take(8 * slots);
  w.bytes = off;
  return w;
}

llm42_status check_attention(const char* who, const llm42_model* m, int32_t num_seqs, int32_t window, int32_t max_context) {
  if (!m) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (window < 1 || window > LLM42_MAX_WINDOW) return fail(LLM42_EINVAL, "%s: window must be 1..%d", who, LLM42_MAX_WINDOW);
  if (num_seqs < 1 || (int64_t)num_seqs * window > LLM42_MAX_ROWS)
    return fail(LLM42_EINVAL, "%s: num_seqs * window must be 1..%d", who, LLM42_MAX_ROWS);
  if (max_context < 1 || max_context > kMostContext4) return fail(LLM42_EINVAL, "%s: max_context must be 1..%d", who, kMostContext4);
  return LLM42_OK;
}

}  // namespace

// Compute units of the current device (asked for once per device).
int current_cus() {
  constexpr int kMax = 64;
  static std::atomic<int> known[kMax];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
  if (dev < kMax && (cus = known[dev].load(std::memory_order_relaxed)) > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) cus = 256;
  if (dev < kMax) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

extern "C" {

llm42_status llm42_mx4_bytes(int32_t rows, int32_t cols, size_t* out_bytes) {
  if (!out_bytes) return fail(LLM42_EINVAL, "mx4_bytes: null argument");
  if (rows < 1 || cols < 1 || rows > kMostRows || cols > kMostCols)
    return fail(LLM42_EINVAL, "mx4_bytes: a matrix has 1..%d rows and 1..%d columns", kMostRows, kMostCols);
  *out_bytes = mx4::matrix_bytes(rows, cols);
  return LLM42_OK;
}

llm42_status llm42_mx4_quantize(const void* src, int32_t src_type, int64_t src_stride, int32_t rows, int32_t cols, void* dst,
                                size_t dst_bytes, void* hip_stream) {
  if (llm42_status st = check_matrix("mx4_quantize", dst, dst_bytes, rows, cols, src, src_type, src_stride)) return st;
  launch_mx4_quantize(src, src_type, src_stride, rows, cols, dst, (hipStream_t)hip_stream);
  return launched("mx4_quantize");
}

llm42_status llm42_mx4_dequantize(const void* src, size_t src_bytes, int32_t rows, int32_t cols, void* dst, int32_t dst_type,
                                  int64_t dst_stride, void* hip_stream) {
  if (llm42_status st = check_matrix("mx4_dequantize", src, src_bytes, rows, cols, dst, dst_type, dst_stride)) return st;
  launch_mx4_dequantize(src, rows, cols, dst, dst_type, dst_stride, (hipStream_t)hip_stream);
  return launched("mx4_dequantize");
}

llm42_status llm42_mx4_matmul_workspace_bytes(int32_t rows, int32_t n, int32_t k, size_t* out_bytes) {
  if (!out_bytes) return fail(LLM42_EINVAL, "mx4_matmul_workspace_bytes: null argument");
  if (rows < 1 || rows > LLM42_MAX_ROWS || n < 1 || k < 1 || n > kMostRows || k > kMostCols)
    return fail(LLM42_EINVAL, "mx4_matmul_workspace_bytes: sizes out of range");
  *out_bytes = packed_x_bytes(rows, k) + mx4_matmul_part_bytes(n, k, rows, current_cus());
  return LLM42_OK;
}

llm42_status llm42_mx4_matmul(const void* w, size_t w_bytes, int32_t n, int32_t k, const void* x, int64_t x_stride, int32_t rows, void* out,
                              int32_t out_type, int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "mx4_matmul";
  if (!x) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (llm42_status st = check_matrix(who, w, w_bytes, n, k, out, out_type, k)) return st;
  if (out_stride < n) return fail(LLM42_EINVAL, "%s: out_stride %lld is less than n", who, (long long)out_stride);
  if (rows < 1 || rows > LLM42_MAX_ROWS) return fail(LLM42_EINVAL, "%s: rows must be 1..%d", who, LLM42_MAX_ROWS);
  if (x_stride < k) return fail(LLM42_EINVAL, "%s: x_stride %lld is less than k", who, (long long)x_stride);
  if ((uintptr_t)x % 2) return fail(LLM42_EINVAL, "%s: x not aligned to its type", who);
  hipStream_t st = (hipStream_t)hip_stream;
  const size_t packed = packed_x_bytes(rows, k), need = packed + mx4_matmul_part_bytes(n, k, rows, current_cus());
  const bool plain = k % 32 == 0 && (uintptr_t)x % 16 == 0 && (rows == 1 || (x_stride % 8 == 0 && x_stride <= (1 << 26)));
  const bool loose = !plain && rows <= mx4_loose_rows() && (uintptr_t)x % 4 == 0 && (rows == 1 || x_stride % 2 == 0), pack = !plain && !loose;
  const bool room = workspace && (uintptr_t)workspace % 256 == 0 && workspace_bytes >= need;
  if (pack && !room) {
    if (!workspace || (uintptr_t)workspace % 256) return fail(LLM42_EWORKSPACE, "%s: this x needs a workspace, 256-byte aligned", who);
    return fail(LLM42_EWORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  }
  if (pack && align_up(rows, 16) * align_up(k, 32) / 8 > (size_t)kMostGroups256 * 256)
    return fail(LLM42_EINVAL, "%s: rows * k too large for rows that are not aligned", who);
  // (up to 2^28 values any tile's workgroups, at most eight parts of 384 threads for 64 x 32 of them, are within a launch)
  if ((int64_t)rows * n > (1 << 28) && !mx4_matmul_fits(n, k, rows, loose, current_cus(), room && need > packed))
    return fail(LLM42_EINVAL, "%s: rows * features too large for one launch", who);
  if (pack) launch_mx4_pack_x((const uint16_t*)x, x_stride, rows, k, (uint16_t*)workspace, st);
  launch_mx4_matmul(w, n, k, (const uint16_t*)(pack ? workspace : x), pack ? 0 : x_stride, loose, rows, out, out_type, out_stride,
                    current_cus(), room && need > packed ? (float*)((char*)workspace + packed) : nullptr, st);
  return launched(who);
}

llm42_status llm42_kv4_bytes(const llm42_model* m, int64_t num_blocks, size_t* out_bytes) {
  if (!m || !out_bytes || num_blocks < 0) return fail(LLM42_EINVAL, "kv4_bytes: bad argument");
  *out_bytes = (size_t)m->cfg.n_layers * (size_t)num_blocks * m->cfg.n_kv_heads * mx4::kv_record(m->cfg.head_dim);
  return LLM42_OK;
}

llm42_status llm42_kv4_store(const llm42_model* m, const llm42_kv_cache* kv, const llm42_kv_cache* kv4, const int32_t* first,
                             const int32_t* count, int32_t num_seqs, int32_t max_count, int32_t* seq_status, void* hip_stream) {
  const char* who = "kv4_store";
  if (llm42_status st = check_ranges(who, m, first, count, num_seqs, max_count)) return st;
  if (llm42_status st = check_cache(who, "kv_cache", kv)) return st;
  if (llm42_status st = check_cache(who, "kv4_cache", kv4)) return st;
  launch_kv4_store(m, kv, kv4, first, count, num_seqs, max_count, seq_status, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv4_read(const llm42_model* m, const llm42_kv_cache* kv4, const int32_t* first, const int32_t* count, int32_t num_seqs,
                            int32_t max_count, void* out_k, void* out_v, int32_t* seq_status, void* hip_stream) {
  const char* who = "kv4_read";
  if (llm42_status st = check_ranges(who, m, first, count, num_seqs, max_count)) return st;
  if (llm42_status st = check_cache(who, "kv4_cache", kv4)) return st;
  if (!out_k || !out_v || (uintptr_t)out_k % 16 || (uintptr_t)out_v % 16)
    return fail(LLM42_EINVAL, "%s: out_k and out_v must be 16-byte aligned", who);
  launch_kv4_read(m, kv4, first, count, num_seqs, max_count, (uint16_t*)out_k, (uint16_t*)out_v, seq_status, (hipStream_t)hip_stream);
  return launched(who);
}

llm42_status llm42_kv4_attention_workspace_bytes(const llm42_model* m, int32_t num_seqs, int32_t window, int32_t max_context,
                                                 size_t* out_bytes) {
  const char* who = "kv4_attention_workspace_bytes";
  if (!out_bytes) return fail(LLM42_EINVAL, "%s: null argument", who);
  if (llm42_status st = check_attention(who, m, num_seqs, window, max_context)) return st;
  int splits, steps;
  plan_kv4_attention(num_seqs, m->cfg.n_kv_heads, m->group * window, max_context, m->num_cus, splits, steps);
  *out_bytes = carve(m, num_seqs, window, splits, nullptr).bytes;
  return LLM42_OK;
}

llm42_status llm42_kv4_attention(const llm42_model* m, int32_t layer, const llm42_kv_cache* kv4, const void* q, int64_t q_stride,
                                 const int32_t* seq_lens, int32_t window, const int32_t* n_valid, int32_t num_seqs, int32_t max_context,
                                 void* out, int64_t out_stride, int32_t* seq_status, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  const char* who = "kv4_attention";
  if (llm42_status st = check_attention(who, m, num_seqs, window, max_context)) return st;
  if (llm42_status st = check_cache(who, "kv4_cache", kv4)) return st;
  if (!q || !seq_lens || !out || !workspace) return fail(LLM42_EINVAL, "%s: null argument", who);
  const llm42_config& c = m->cfg;
  if (layer < 0 || layer >= c.n_layers) return fail(LLM42_EINVAL, "%s: layer must be 0..%d", who, c.n_layers - 1);
  if ((uintptr_t)q % 16 || (uintptr_t)out % 16 || q_stride % 8 || out_stride % 8 || q_stride < m->d_attn || out_stride < m->d_attn)
    return fail(LLM42_EINVAL, "%s: q and out need 16-byte aligned rows of at least %d", who, m->d_attn);
  if ((int64_t)max_context > (int64_t)kv4->max_blocks_per_seq * LLM42_KV_BLOCK)
    return fail(LLM42_ECAPACITY, "%s: max_context %d exceeds block-table capacity %lld", who, max_context,
                (long long)kv4->max_blocks_per_seq * LLM42_KV_BLOCK);
  if ((uintptr_t)workspace % 256) return fail(LLM42_EWORKSPACE, "%s: workspace not 256-byte aligned", who);
  Attention4 a;
  plan_kv4_attention(num_seqs, c.n_kv_heads, m->group * window, max_context, m->num_cus, a.splits, a.split_steps);
  const Attention4Workspace ws = carve(m, num_seqs, window, a.splits, (char*)workspace);
  if (ws.bytes > workspace_bytes) return fail(LLM42_EWORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, ws.bytes);
  a.base = (char*)kv4->kv_base + (size_t)layer * kv4->num_blocks * c.n_kv_heads * mx4::kv_record(c.head_dim);
  a.num_blocks = kv4->num_blocks;
  a.block_table = kv4->block_table;
  a.max_blocks = kv4->max_blocks_per_seq;
  a.seq_len = seq_lens;
  a.seq_n = n_valid;
  a.seq_status = seq_status;
  a.merge_n = a.splits > 1 ? ws.n : nullptr;
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.tiles = false;
  a.num_seqs = num_seqs;
  a.n_kv_heads = c.n_kv_heads;
  a.group = m->group;
  a.head_dim = c.head_dim;
  a.window = window;
  a.max_context = max_context;
  a.num_cus = m->num_cus;
  a.part_acc = ws.acc;
  a.part_ml = ws.ml;
  a.k_plane = a.v_plane = nullptr;
  a.row_blk = nullptr;
  launch_kv4_attention(a, (hipStream_t)hip_stream);
  return launched(who);
}

}  // extern "C"
