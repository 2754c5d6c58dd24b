// Bounds of the cached keys: from the bf16 cache, and what they stand for.
#include <algorithm>
#include <type_traits>

#include "paged.h"

using namespace paged;

namespace {

// One wave per (block of 16 positions, kv head) and L layers (blockIdx.y), the next layer's keys asked for before this one's are looked at; four waves to a
// workgroup.  Bound by memory where blocks are many: the keys of 4 x 1500 - 2048 tokens of 32 layers of 8 heads of 128, 461 MB, and their bounds take 102 us,
// 4.8 TB/s (a copy of as many bytes runs at 5.3; a layer to a wave 130: three loads that wait for each other stand before every 4 KiB).  Where there are
// few waves those trips are the time, and cost less than four layers in turn: 24 x 1 - 32 tokens, 30 MB, 14.6 / 16.6.
// MANY: a wave takes some blocks in turn (see the launch).
template <int HD, int L, bool MANY>
__global__ __launch_bounds__(256) void bounds_store_kernel(const uint16_t* __restrict__ k_plane, int64_t layer_stride, char* __restrict__ bounds,
                                                           const int32_t* __restrict__ table, int width, int64_t num_blocks, int n_kv_heads,
                                                           const int32_t* __restrict__ first_, const int32_t* __restrict__ count_, int num_seqs,
                                                           int max_count, int groups, int at_once, int n_layers, int32_t* __restrict__ seq_status) {
  constexpr int LANES = HD / 8, N = HD / 32;
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int h = (int)(item % n_kv_heads), group = (int)(item / n_kv_heads % groups), s = (int)(item / n_kv_heads / groups), layer = blockIdx.y * L;
  if (s >= num_seqs) return;
  const int64_t first = first_[s], count = count_ ? count_[s] : max_count;
  int status = LLM42_SEQ_OK;
  const int begin = (int)(first / LLM42_KV_BLOCK), end = (int)min((first + count) / LLM42_KV_BLOCK, (int64_t)width);   // whole blocks end here
  if (first < 0 || count < 0 || count > max_count || first + count > (int64_t)width * LLM42_KV_BLOCK) {
    status = LLM42_SEQ_BAD_LENGTH;
  } else if (count > 0) {
    bool bad = false;
    constexpr int U = MANY ? 8 : 1;
    for (int b = begin + lane; b < end; b += 64 * U) {
      int id[U];
#pragma unroll
      for (int u = 0; u < U; ++u) id[u] = table[(size_t)s * width + (MANY ? min(b + 64 * u, end - 1) : b)];
#pragma unroll
      for (int u = 0; u < U; ++u) bad |= id[u] < 0 || id[u] >= num_blocks;
    }
    if (__any(bad)) status = LLM42_SEQ_BAD_BLOCK;
  }
  if (seq_status && layer == 0 && group == 0 && h == 0 && lane == 0) seq_status[s] = status;
  if (status != LLM42_SEQ_OK || count == 0) return;
  const int from = begin + group * (MANY ? at_once : 1);          // (far below 2^31)
  if (from >= end) return;
  const int blocks = MANY ? min(at_once, end - from) : 1;
  const int c = lane % LANES, t0 = lane / LANES, layers = min(L, n_layers - layer);
  const size_t rec_stride = (size_t)num_blocks * n_kv_heads * bounds_record(HD);
  for (int i = 0; i < blocks; ++i) {
    const size_t at = (size_t)table[(size_t)s * width + from + i] * n_kv_heads + h;
    const uint16_t* tile = k_plane + layer * layer_stride + at * 16 * HD + (c * 16 + t0) * 8;
    char* rec = bounds + ((size_t)layer * num_blocks * n_kv_heads + at) * bounds_record(HD);
    u32x4 key[2][N];
    const auto load = [&](u32x4 (&d)[N], int l) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < N; ++j) d[j] = *(const u32x4*)(tile + l * layer_stride + j * (64 / LANES) * 8);
    };
    load(key[0], 0);
#pragma unroll
    for (int l = 0; l < L; ++l) {
      if (l >= layers) break;
      if (L > 1) load(key[(l + 1) & 1], min(l + 1, layers - 1));
      write_bounds<HD>(key[l & 1], rec + l * rec_stride, lane);
    }
  }
}

// A thread per 8 features of a (block, kv head); blockIdx.y: layer.
template <int HD>
__global__ __launch_bounds__(256) void bounds_read_kernel(const char* __restrict__ bounds, int64_t num_blocks, int n_kv_heads,
                                                          const int32_t* __restrict__ ids, int num_ids, uint16_t* __restrict__ out_lo,
                                                          uint16_t* __restrict__ out_hi) {
  constexpr int LANES = HD / 8;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x, head = item / LANES;
  const int c = (int)(item % LANES), h = (int)(head % n_kv_heads);
  const int64_t j = head / n_kv_heads;
  if (j >= num_ids) return;
  const int id = ids[j];
  const bool there = id >= 0 && id < num_blocks;
  const char* rec = bounds + (((size_t)blockIdx.y * num_blocks + (there ? id : 0)) * n_kv_heads + h) * bounds_record(HD);
  const int e = *(const uint8_t*)(rec + 2 * HD);
  const bool none = e == kBoundsNone;
  const float unit = none ? 0.f : power_of_two(e - kBoundsBias);
  const size_t at = (((size_t)blockIdx.y * num_ids + j) * n_kv_heads + h) * HD + c * 8;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const u32x2 w = *(const u32x2*)(rec + part * HD + c * 8);
    const float inf = part ? -INFINITY : INFINITY;
    float x[8];
#pragma unroll
    for (int f = 0; f < 8; ++f) x[f] = !there ? 0.f : none ? inf : (float)(int8_t)(w[f >> 2] >> (8 * (f & 3))) * unit;
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack2_bf16(x[2 * i], x[2 * i + 1]);
    *(u32x4*)((part ? out_lo : out_hi) + at) = o;
  }
}

}  // namespace

void launch_bounds_store(int n_layers, int n_kv_heads, int head_dim, const uint16_t* k_plane, int64_t layer_stride, char* bounds,
                         const int32_t* block_table, int width, int64_t num_blocks, const int32_t* first, const int32_t* count, int num_seqs,
                         int max_count, int32_t* seq_status, hipStream_t st) {
  // Every wave looks at the entries of all the blocks that its sequence's call touches.  Where those are many it takes some blocks in turn, about 1024 waves to a sequence and
  // kv head, so that the time does not grow with the square of the context (one layer, us with a block to a wave / so: 131072 positions of 8 kv heads of 128
  // 279 / 90, 2^22 of one of 64 16166 / 560, 2^24 528945 / 2181; with eight entries asked for at a time and the loop, shorter ones lose 4 %).
  const int slots = slots_of(max_count, width), at_once = std::max(1, slots / 1024), groups = (slots + at_once - 1) / at_once;
  const int64_t items = (int64_t)num_seqs * groups * n_kv_heads;
  const auto go = [&](auto kernel, int layers) {
    kernel<<<dim3((unsigned)((items + 3) / 4), (n_layers + layers - 1) / layers), 256, 0, st>>>(
        k_plane, layer_stride, bounds, block_table, width, num_blocks, n_kv_heads, first, count, num_seqs, max_count, groups, at_once, n_layers, seq_status);
  };
  const bool few = items * n_layers <= 32768;
  const auto by_blocks = [&](auto hd, auto layers) {
    constexpr int HD = decltype(hd)::value, L = decltype(layers)::value;
    at_once > 1 ? go(bounds_store_kernel<HD, L, true>, L) : go(bounds_store_kernel<HD, L, false>, L);
  };
  const auto by_layers = [&](auto hd) { few ? by_blocks(hd, std::integral_constant<int, 1>{}) : by_blocks(hd, std::integral_constant<int, 4>{}); };
  if (head_dim == 128) by_layers(std::integral_constant<int, 128>{});
  else by_layers(std::integral_constant<int, 64>{});
}

void launch_bounds_read(int n_layers, int n_kv_heads, int head_dim, const char* bounds, int64_t num_blocks, const int32_t* ids, int num_ids,
                        uint16_t* out_lo, uint16_t* out_hi, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)num_ids * n_kv_heads * (head_dim / 8) + 255) / 256), n_layers);
  const auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(bounds, num_blocks, n_kv_heads, ids, num_ids, out_lo, out_hi); };
  if (head_dim == 128) go(bounds_read_kernel<128>);
  else go(bounds_read_kernel<64>);
}
