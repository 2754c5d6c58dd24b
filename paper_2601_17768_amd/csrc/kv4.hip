// The 4-bit cache: K and V from the bf16 cache into it, and what it stands for.
#include "mx4.h"

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

// The largest over the 16 lanes of a group.
__device__ inline uint32_t max_of_16(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

// One wave per (block of 16 positions, kv head), four heads of a block to a workgroup at a time; blockIdx.y: layer.
template <int HD>
__global__ __launch_bounds__(256) void kv4_store_kernel(const uint16_t* __restrict__ kv, Table src, char* __restrict__ kv4, Table dst,
                                                        int n_kv_heads, int layer0, const int32_t* __restrict__ first_,
                                                        const int32_t* __restrict__ count_, int max_count, int slots,
                                                        int32_t* __restrict__ seq_status) {
  constexpr int KT = HD / 32, FB = HD / 16;
  const int s = blockIdx.x / slots, slot = blockIdx.x % slots, layer = layer0 + blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int64_t first = first_[s], count = count_ ? count_[s] : first >= 0;   // (no counts: of sequences that take part one each)
  const int status = range_status(first, count, max_count, src, dst, s, lane);
  if (seq_status && blockIdx.y == 0 && slot == 0 && threadIdx.x == 0) seq_status[s] = status;
  const int block = (int)(first / LLM42_KV_BLOCK) + slot;
  if (status != LLM42_SEQ_OK || (int64_t)block * LLM42_KV_BLOCK >= first + count) return;
  const int lo = (int)max(first - (int64_t)block * 16, (int64_t)0), hi = (int)min(first + count - (int64_t)block * 16, (int64_t)16);
  const size_t sb = src.ids[(size_t)s * src.width + block], db = dst.ids[(size_t)s * dst.width + block];
  const size_t plane = (size_t)src.num_blocks * n_kv_heads * 16 * HD;
  for (int h = wave; h < n_kv_heads; h += 4) {
    const uint16_t* kt = kv + (size_t)layer * 2 * plane + (sb * n_kv_heads + h) * 16 * HD;
    const uint16_t* vt = kt + plane;
    char* rec = kv4 + (((size_t)layer * dst.num_blocks + db) * n_kv_heads + h) * kv_record(HD);
    u32x4 kw[KT];
    u32x2 vw[FB];
#pragma unroll
    for (int j = 0; j < KT; ++j) kw[j] = *(const u32x4*)(kt + j * 512 + lane * 8);
#pragma unroll
    for (int b = 0; b < FB; ++b) vw[b] = *(const u32x2*)(vt + b * 256 + lane * 4);
    // K: lane (g, token) has features 32 j + 8 g .. + 7
    uint32_t kc[KT], ks = 0;
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(kw[j][i] << 16 & 0x7FFF0000u, kw[j][i] & 0x7FFF0000u));
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const uint32_t byte = scale_byte(top);
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        word |= code_of(__uint_as_float(kw[j][i] << 16), byte) << (8 * i) |
                code_of(__uint_as_float(kw[j][i] & 0xFFFF0000u), byte) << (8 * i + 4);
      kc[j] = word;
      ks |= byte << (8 * j);
    }
    if (l16 >= lo && l16 < hi) {
      uint32_t* p = (uint32_t*)(rec + lane * KT * 4);
#pragma unroll
      for (int j = 0; j < KT; ++j) p[j] = kc[j];
      if (g == 0) {
        if constexpr (HD == 128) *(uint32_t*)(rec + 16 * HD + l16 * 4) = ks;
        else *(uint16_t*)(rec + 16 * HD + l16 * 2) = (uint16_t)ks;
      }
    }
    // V: lane (g, f) has tokens 4 g .. 4 g + 3 of feature 16 b + f
    uint32_t vs[KT], vc[FB / 2];
#pragma unroll
    for (int q = 0; q < KT; ++q) {
      vs[q] = 0;
      vc[q] = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t sh = t & 1 ? 0 : 16;
        const uint32_t x = vw[2 * q][t >> 1] << sh & 0xFFFF0000u, y = vw[2 * q + 1][t >> 1] << sh & 0xFFFF0000u;
        const uint32_t byte = scale_byte(max_of_16(max(x & 0x7FFFFFFFu, y & 0x7FFFFFFFu)));
        vs[q] |= byte << (8 * t);
        vc[q] |= code_of(__uint_as_float(x), byte) << (4 * t) | code_of(__uint_as_float(y), byte) << (16 + 4 * t);
      }
    }
    // tokens of this lane that are in range: a nibble of each half word, a byte of each scale word
    uint32_t nib = 0, byt = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (4 * g + t >= lo && 4 * g + t < hi) nib |= 0x000F000Fu << (4 * t), byt |= 0xFFu << (8 * t);
    if (nib) {
      uint32_t* p = (uint32_t*)(rec + 8 * HD + lane * KT * 4);
      uint32_t* q = (uint32_t*)(rec + 16 * HD + HD / 2 + (g * KT) * 4);
      const bool part = nib != 0xFFFFFFFFu;          // (codes of other positions share the word: this wave alone writes it)
#pragma unroll
      for (int j = 0; j < KT; ++j) p[j] = part ? (p[j] & ~nib) | (vc[j] & nib) : vc[j];
      if (l16 == 0) {
#pragma unroll
        for (int j = 0; j < KT; ++j) q[j] = part ? (q[j] & ~byt) | (vs[j] & byt) : vs[j];
      }
    }
  }
}

template <int HD>
__global__ __launch_bounds__(256) void kv4_read_kernel(const char* __restrict__ kv4, Table src, int n_kv_heads,
                                                       const int32_t* __restrict__ first_, const int32_t* __restrict__ count_,
                                                       int num_seqs, int max_count, int slots, uint16_t* __restrict__ out_k,
                                                       uint16_t* __restrict__ out_v, int32_t* __restrict__ seq_status) {
  constexpr int KT = HD / 32, FB = HD / 16;
  const int s = blockIdx.x / slots, slot = blockIdx.x % slots, layer = blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int64_t first = first_[s], count = count_[s];
  const int status = range_status(first, count, max_count, src, src, s, lane);
  if (seq_status && blockIdx.y == 0 && slot == 0 && threadIdx.x == 0) seq_status[s] = status;
  const int block = (int)(first / LLM42_KV_BLOCK) + slot;
  if (status != LLM42_SEQ_OK || (int64_t)block * LLM42_KV_BLOCK >= first + count) return;
  const int lo = (int)max(first - (int64_t)block * 16, (int64_t)0), hi = (int)min(first + count - (int64_t)block * 16, (int64_t)16);
  const size_t sb = src.ids[(size_t)s * src.width + block];
  // element of position 0 of the block in the plain arrays (it may lie before the sequence's first row: only lo .. hi - 1 are written)
  const int64_t row0 = ((int64_t)layer * num_seqs + s) * max_count + ((int64_t)block * 16 - first);
  for (int h = wave; h < n_kv_heads; h += 4) {
    const char* rec = kv4 + (((size_t)layer * src.num_blocks + sb) * n_kv_heads + h) * kv_record(HD);
    const int64_t at = row0 * n_kv_heads + h;
    if (l16 >= lo && l16 < hi) {
      const uint32_t* p = (const uint32_t*)(rec + lane * KT * 4);
      const uint8_t* sc = (const uint8_t*)rec + 16 * HD + l16 * KT;
      uint16_t* o = out_k + (at + (int64_t)l16 * n_kv_heads) * HD + g * 8;
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        const uint32_t word = p[j], byte = sc[j];
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __float_as_uint(value_of(word >> (8 * i) & 15u, byte)) >> 16 | (__float_as_uint(value_of(word >> (8 * i + 4) & 15u, byte)) & 0xFFFF0000u);
        *(u32x4*)(o + j * 32) = w;
      }
    }
    const uint32_t* p = (const uint32_t*)(rec + 8 * HD + lane * KT * 4);
    const uint8_t* sc = (const uint8_t*)rec + 16 * HD + HD / 2 + g * KT * 4;
    uint16_t* o = out_v + at * HD + l16;
#pragma unroll
    for (int b = 0; b < FB; ++b) {
      const uint32_t word = p[b >> 1] >> (16 * (b & 1));
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (4 * g + t >= lo && 4 * g + t < hi)
          o[(int64_t)(4 * g + t) * n_kv_heads * HD + b * 16] = (uint16_t)(__float_as_uint(value_of(word >> (4 * t) & 15u, sc[(b >> 1) * 4 + t])) >> 16);
    }
  }
}

Table table_of(const llm42_kv_cache* c) { return {c->block_table, c->max_blocks_per_seq, c->num_blocks}; }

}  // namespace

void launch_kv4_store(const llm42_model* m, int layer, const llm42_kv_cache* kv, const llm42_kv_cache* kv4, const int32_t* first,
                      const int32_t* count, int num_seqs, int max_count, int32_t* seq_status, hipStream_t st) {
  const int slots = (max_count + 14) / 16 + 1;                 // blocks that a run of max_count positions can touch
  const dim3 grid((unsigned)(num_seqs * slots), layer < 0 ? m->cfg.n_layers : 1);
  const auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, st>>>((const uint16_t*)kv->kv_base, table_of(kv), (char*)kv4->kv_base, table_of(kv4), m->cfg.n_kv_heads,
                                 layer < 0 ? 0 : layer, first, count, max_count, slots, seq_status);
  };
  if (m->cfg.head_dim == 128) go(kv4_store_kernel<128>);
  else go(kv4_store_kernel<64>);
}

void launch_kv4_read(const llm42_model* m, const llm42_kv_cache* kv4, const int32_t* first, const int32_t* count, int num_seqs,
                     int max_count, uint16_t* out_k, uint16_t* out_v, int32_t* seq_status, hipStream_t st) {
  const int slots = (max_count + 14) / 16 + 1;
  const dim3 grid((unsigned)(num_seqs * slots), m->cfg.n_layers);
  const auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, st>>>((const char*)kv4->kv_base, table_of(kv4), m->cfg.n_kv_heads, first, count, num_seqs, max_count, slots,
                                 out_k, out_v, seq_status);
  };
  if (m->cfg.head_dim == 128) go(kv4_read_kernel<128>);
  else go(kv4_read_kernel<64>);
}
