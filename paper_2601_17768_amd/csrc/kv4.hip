// The 4-bit cache: K and V from the bf16 cache into it, and what it stands for.
#include <algorithm>

#include "kv4_store.h"

using namespace mx4;

namespace {

// Positions first .. first + count - 1 of a sequence, and whether they and the block-table entries they need are in order (a wave
// asks together; every wave that works for the sequence comes to the same answer).
struct Table {
  const int32_t* ids;       // [seq][width]
  int width;
  int64_t num_blocks;
};
__device__ inline int range_status(int64_t first, int64_t count, int max_count, const Table& a, const Table& b, int s, int lane) {
  const int64_t room = (int64_t)min(a.width, b.width) * LLM42_KV_BLOCK;
  if (first < 0 || count < 0 || count > max_count || first + count > room) return LLM42_SEQ_BAD_LENGTH;
  const int end = count ? (int)((first + count + LLM42_KV_BLOCK - 1) / LLM42_KV_BLOCK) : 0;
  bool bad = false;
  for (int i = (int)(first / LLM42_KV_BLOCK) + lane; i < end; i += 64) {
    const int x = a.ids[(size_t)s * a.width + i], y = b.ids[(size_t)s * b.width + i];
    bad |= x < 0 || x >= a.num_blocks || y < 0 || y >= b.num_blocks;
  }
  return __any(bad) ? LLM42_SEQ_BAD_BLOCK : LLM42_SEQ_OK;
}

// One wave per (block of 16 positions, kv head), four heads of a block to a workgroup, the launch's first workgroup being `group0`;
// blockIdx.y: layer.  A record is its wave's alone, so a partly covered one needs no atomics.  Long runs are bound by memory (4 x 1500 - 2048 tokens of 32 layers of 8 heads of 128, stored
// and read back: 2.4 GB in 445 us, 5.4 TB/s), a single token by three loads that wait for each other (24 sequences 7 us).
template <int HD>
__global__ __launch_bounds__(256) void kv4_store_kernel(const uint16_t* __restrict__ kv, Table src, char* __restrict__ kv4, Table dst,
                                                        int n_kv_heads, const int32_t* __restrict__ first_,
                                                        const int32_t* __restrict__ count_, int max_count, int slots,
                                                        int32_t* __restrict__ seq_status, unsigned group0) {
  const int hg = (n_kv_heads + 3) / 4, group = (int)(group0 + blockIdx.x), at_slot = group / hg;
  const int s = at_slot / slots, slot = at_slot % slots, layer = blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = group % hg * 4 + wave;
  const int64_t first = first_[s], count = count_[s];
  const int block = (int)(first / LLM42_KV_BLOCK) + slot;
  // (asked for together with what the check reads)
  const int sb_ = src.ids[(size_t)s * src.width + min(max(block, 0), src.width - 1)], db_ = dst.ids[(size_t)s * dst.width + min(max(block, 0), dst.width - 1)];
  const int status = range_status(first, count, max_count, src, dst, s, lane);
  if (seq_status && blockIdx.y == 0 && slot == 0 && h == 0 && lane == 0) seq_status[s] = status;
  if (status != LLM42_SEQ_OK || (int64_t)block * LLM42_KV_BLOCK >= first + count || h >= n_kv_heads) return;
  const int lo = (int)max(first - (int64_t)block * 16, (int64_t)0), hi = (int)min(first + count - (int64_t)block * 16, (int64_t)16);
  const size_t sb = sb_, db = db_;
  const size_t plane = (size_t)src.num_blocks * n_kv_heads * 16 * HD;
  const uint16_t* kt = kv + (size_t)layer * 2 * plane + (sb * n_kv_heads + h) * 16 * HD;
  char* rec = kv4 + (((size_t)layer * dst.num_blocks + db) * n_kv_heads + h) * kv_record(HD);
  store_positions<HD>(kt, kt + plane, rec, lo, hi, lane);
}

// The other way.  A wave's values lie in LDS between the cache's order and rows, so that every store is of 256 (head_dim 64: 128) bytes of a
// position's row (in pieces of 64 as they come from the records 455 us for 4 x 1500 - 2048 tokens of 32 layers of 8 heads of 128).
template <int HD>
__global__ __launch_bounds__(256) void kv4_read_kernel(const char* __restrict__ kv4, Table src, int n_kv_heads,
                                                       const int32_t* __restrict__ first_, const int32_t* __restrict__ count_,
                                                       int num_seqs, int max_count, int slots, uint16_t* __restrict__ out_k,
                                                       uint16_t* __restrict__ out_v, int32_t* __restrict__ seq_status,
                                                       unsigned group0) {
  constexpr int KT = HD / 32, ROW = HD / 8, PER = 64 / ROW;       // 16-byte pieces of a row, rows that a wave stores at once
  __shared__ u32x4 rows[4][16 * (ROW + 1)];                       // (a piece between the rows: 16 rows start in different banks)
  const int hg = (n_kv_heads + 3) / 4, group = (int)(group0 + blockIdx.x), at_slot = group / hg;
  const int s = at_slot / slots, slot = at_slot % slots, layer = blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15, h = group % hg * 4 + wave;
  const int64_t first = first_[s], count = count_[s];
  const int status = range_status(first, count, max_count, src, src, s, lane);
  if (seq_status && blockIdx.y == 0 && slot == 0 && h == 0 && lane == 0) seq_status[s] = status;
  const int block = (int)(first / LLM42_KV_BLOCK) + slot;
  if (status != LLM42_SEQ_OK || (int64_t)block * LLM42_KV_BLOCK >= first + count || h >= n_kv_heads) return;
  const int lo = (int)max(first - (int64_t)block * 16, (int64_t)0), hi = (int)min(first + count - (int64_t)block * 16, (int64_t)16);
  const size_t sb = src.ids[(size_t)s * src.width + block];
  // element of position 0 of the block in the plain arrays (it may lie before the sequence's first row: only lo .. hi - 1 are written)
  const int64_t row0 = ((int64_t)layer * num_seqs + s) * max_count + ((int64_t)block * 16 - first);
  const char* rec = kv4 + (((size_t)layer * src.num_blocks + sb) * n_kv_heads + h) * kv_record(HD);
  uint32_t kc[KT], vc[KT], vs[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) kc[j] = ((const uint32_t*)(rec + lane * KT * 4))[j];
#pragma unroll
  for (int j = 0; j < KT; ++j) vc[j] = ((const uint32_t*)(rec + 8 * HD + lane * KT * 4))[j];
  const uint32_t ks = KT == 4 ? *(const uint32_t*)(rec + 16 * HD + l16 * 4) : *(const uint16_t*)(rec + 16 * HD + l16 * 2);
#pragma unroll
  for (int j = 0; j < KT; ++j) vs[j] = ((const uint32_t*)(rec + 16 * HD + HD / 2 + g * KT * 4))[j];
  // (the rows are this wave's own: its LDS accesses are in order)
  auto store = [&](uint16_t* out) __attribute__((always_inline)) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 16 / PER; ++i) {
      const int t = i * PER + lane / ROW, piece = lane % ROW;
      const u32x4 w = rows[wave][t * (ROW + 1) + piece];
      if (t >= lo && t < hi) __builtin_nontemporal_store(w, (u32x4*)(out + ((row0 + t) * n_kv_heads + h) * HD + piece * 8));
    }
    __builtin_amdgcn_wave_barrier();
  };
#pragma unroll
  for (int j = 0; j < KT; ++j) rows[wave][l16 * (ROW + 1) + j * 4 + g] = __builtin_bit_cast(u32x4, operand(kc[j], scale_of(ks, j)));
  store(out_k);
#pragma unroll
  for (int j = 0; j < KT; ++j)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      ((uint32_t*)&rows[wave][(4 * g + t) * (ROW + 1)])[j * 16 + l16] = pair_bf16(vc[j], scale_of(vs[j], t), t);
  store(out_v);
}

// Blocks that a run of max_count positions can touch, of those that a table names.
int slots_of(int max_count, int width) { return (int)std::min<int64_t>(((int64_t)max_count + 14) / 16 + 1, width); }

// As many launches as the workgroups need.
template <class Go>
void in_launches(const llm42_model* m, int num_seqs, int slots, const Go& go) {
  const unsigned groups = (unsigned)(num_seqs * slots * ((m->cfg.n_kv_heads + 3) / 4));
  for (unsigned at = 0; at < groups; at += kMostGroups256) go(dim3(std::min(groups - at, kMostGroups256), m->cfg.n_layers), at);
}

Table table_of(const llm42_kv_cache* c) { return {c->block_table, c->max_blocks_per_seq, c->num_blocks}; }

}  // namespace

void launch_kv4_store(const llm42_model* m, const llm42_kv_cache* kv, const llm42_kv_cache* kv4, const int32_t* first,
                      const int32_t* count, int num_seqs, int max_count, int32_t* seq_status, hipStream_t st) {
  const int slots = slots_of(max_count, std::min(kv->max_blocks_per_seq, kv4->max_blocks_per_seq));
  const auto go = [&](auto kernel) {
    in_launches(m, num_seqs, slots, [&](dim3 grid, unsigned at) {
      kernel<<<grid, 256, 0, st>>>((const uint16_t*)kv->kv_base, table_of(kv), (char*)kv4->kv_base, table_of(kv4), m->cfg.n_kv_heads,
                                   first, count, max_count, slots, seq_status, at);
    });
  };
  if (m->cfg.head_dim == 128) go(kv4_store_kernel<128>);
  else go(kv4_store_kernel<64>);
}

void launch_kv4_read(const llm42_model* m, const llm42_kv_cache* kv4, const int32_t* first, const int32_t* count, int num_seqs,
                     int max_count, uint16_t* out_k, uint16_t* out_v, int32_t* seq_status, hipStream_t st) {
  const int slots = slots_of(max_count, kv4->max_blocks_per_seq);
  const auto go = [&](auto kernel) {
    in_launches(m, num_seqs, slots, [&](dim3 grid, unsigned at) {
      kernel<<<grid, 256, 0, st>>>((const char*)kv4->kv_base, table_of(kv4), m->cfg.n_kv_heads, first, count, num_seqs, max_count, slots,
                                   out_k, out_v, seq_status, at);
    });
  };
  if (m->cfg.head_dim == 128) go(kv4_read_kernel<128>);
  else go(kv4_read_kernel<64>);
}
