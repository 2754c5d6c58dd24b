// The blocks that a query reads: scores from the bounds of the cached keys, and the highest of them.
#include <algorithm>
#include <type_traits>

#include "paged.h"

using namespace paged;

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kChunk = 256;    // blocks that a workgroup scores where scores go through the workspace; more where that is too many workgroups

// Unsigned keys in the order of the scores; a block whose bounds are infinite comes before all.
__device__ inline uint32_t key_of(float score) {
  const uint32_t u = __float_as_uint(score);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Query heads as operands of the scores: column l16 of the product is head l16 % cols of tile row l16 / cols, `cols` the group rounded up to a power of two (what is
// behind the group repeats its last head).  Lane (g, l16) has features 64 c + 16 g .. + 15 of its column, positive values in one operand and negative ones in
// the other: the first meets the upper bounds, the other the lower ones, and their sum is the sum of the larger products.
template <int HD>
struct Query {
  i32x4 pos[HD / 64], neg[HD / 64];
  float unit;                  // 2^e of the column
};
template <int HD>
__device__ inline void quantize(Query<HD>& d, const uint16_t* const (&src)[HD / 64][2]) {
  constexpr int C = HD / 64;
  u32x4 w[C][2];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p) w[c][p] = *(const u32x4*)src[c][p];
  float top = 0.f;
  bool bad = false;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = w[c][p][i];
        bad |= (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
        top = fmaxf(top, fmaxf(fabsf(lo_bf16(x)), fabsf(hi_bf16(x))));
      }
  top = bad ? INFINITY : top;                                     // (only ever compared with what is larger: a column's four lanes agree)
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const int e = top == INFINITY ? kMostExponent + 1 : bounds_exponent(top);
  const bool none = e > kMostExponent;
  const float inverse = none ? 0.f : power_of_two(-e);
  d.unit = none ? 0.f : power_of_two(e);
  // x / 2^e rounded to a whole number, ties to even, in the low byte of x / 2^e + 1.5 * 2^23
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t r[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint32_t x = w[c][j >> 1][(j & 1) * 2 + (b >> 1)];
        r[b] = __float_as_uint(fmaf(b & 1 ? hi_bf16(x) : lo_bf16(x), inverse, 12582912.0f));
      }
      const uint32_t q = none ? 0 : __builtin_amdgcn_perm(__builtin_amdgcn_perm(r[3], r[2], 0x0C0C0400u), __builtin_amdgcn_perm(r[1], r[0], 0x0C0C0400u), 0x05040100u);
      const uint32_t sign = q >> 7 & 0x01010101u, minus = (sign << 8) - sign;     // 255 in the bytes below zero
      d.pos[c][j] = (int)(q & ~minus);
      d.neg[c][j] = (int)(q & minus);
    }
}

// The bounds of 16 blocks.  As operands of the products, lane (g, l16) needs 16 bytes here and there of record l16; asked for like that, every lane of a load looks up a cache line of
// its own.  So a wave reads whole records, 16 neighbouring lanes (head_dim 64: 8) each, and turns them through LDS: piece p of record r lies at place p ^ r of the record,
// so that neither way has lanes in one bank (128 sequences of 1024 - 8192 positions 27.6 -> 23.3 us, 3.2 TB/s; single workgroups gain nothing).
template <int HD>
struct Record {
  static constexpr int P = HD / 8, J = P / 4;                     // pieces of a record, loads of 64 lanes for 16 of them
  u32x4 w[J];
  int e;
  // rec_of(r): record r of the 16
  template <class Rec>
  __device__ inline void load(Rec rec_of, int lane) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int r = j * (64 / P) + lane / P;
      w[j] = *(const u32x4*)(rec_of(r) + ((lane % P) ^ (r % P)) * 16);
    }
    e = *(const uint8_t*)(rec_of(lane & 15) + 2 * HD);
  }
};

// Keys of U times 16 blocks, of which lane l16 of every group of 16 has the records: lane (g, column) gets those of blocks 4 g .. 4 g + 3 for its column's tile row (the
// largest over the columns of the same tile row).
template <int HD, int COLS, int U>
__device__ inline void score16(u32x4 (&key)[U], const Record<HD> (&d)[U], const Query<HD>& q, u32x4* stage, int lane) {
  constexpr int C = HD / 64, P = Record<HD>::P;
  const int g = lane >> 4, l16 = lane & 15;
  i32x4 acc[U], up[U][C], down[U][C];
  // (a wave's LDS accesses are in order: the next 16 records may follow as soon as these have been asked for)
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int j = 0; j < Record<HD>::J; ++j) stage[j * 64 + lane] = d[u].w[j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      up[u][c] = __builtin_bit_cast(i32x4, stage[l16 * P + ((c * 4 + g) ^ (l16 % P))]);
      down[u][c] = __builtin_bit_cast(i32x4, stage[l16 * P + ((P / 2 + c * 4 + g) ^ (l16 % P))]);
    }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int u = 0; u < U; ++u) acc[u] = (i32x4){0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll
    for (int u = 0; u < U; ++u) acc[u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[u][c], q.pos[c], acc[u], 0, 0, 0);
#pragma unroll
    for (int u = 0; u < U; ++u) acc[u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[u][c], q.neg[c], acc[u], 0, 0, 0);
  }
  int e[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) e[u][i] = __shfl(d[u].e, g * 4 + i);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float s = (float)acc[u][i] * q.unit;
      const auto with = [&](uint32_t x) __attribute__((always_inline)) { s = fmaxf(s, __uint_as_float(x)); };
      if constexpr (COLS > 1) with(other_lane<kXor1>(__float_as_uint(s)));
      if constexpr (COLS > 2) with(other_lane<kXor2>(__float_as_uint(s)));
      if constexpr (COLS > 4) with(other_lane<kMirror8>(__float_as_uint(s)));
      if constexpr (COLS > 8) with(other_lane<kMirror16>(__float_as_uint(s)));
      key[u][i] = e[u][i] == kBoundsNone ? 0xFFFFFFFFu : key_of(s * power_of_two(e[u][i] - kBoundsBias));
    }
}

struct Scratch {
  int hist[256], bin, need;
  uint32_t all, any, counts[256];
};

// The bits in which the keys of a row differ (the scores of a row share their sign and most of their exponent, and are whole numbers times a power of
// two: a third of the bits or more are the same), asked by a wave.
__device__ inline void reduce_bits(uint32_t& all, uint32_t& any) {
  all &= other_lane<kXor1>(all), any |= other_lane<kXor1>(any);
  all &= other_lane<kXor2>(all), any |= other_lane<kXor2>(any);
  all &= other_lane<kMirror8>(all), any |= other_lane<kMirror8>(any);
  all &= other_lane<kMirror16>(all), any |= other_lane<kMirror16>(any);
  const u32x2 a16 = __builtin_amdgcn_permlane16_swap(all, all, false, false), o16 = __builtin_amdgcn_permlane16_swap(any, any, false, false);
  all = a16.x & a16.y, any = o16.x | o16.y;
  const u32x2 a32 = __builtin_amdgcn_permlane32_swap(all, all, false, false), o32 = __builtin_amdgcn_permlane32_swap(any, any, false, false);
  all = a32.x & a32.y, any = o32.x | o32.y;
}

// Sum of a value over this lane and those before it.
__device__ inline uint32_t sum_up_to(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);     // one lane down in its group of 16, two, four, eight
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);     // the last lane of the group before, to groups 1 and 3
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);     // lane 31 to groups 2 and 3
  return x;
}

// The `k` highest of keys[begin .. end - 1], the lowest index on ties, ascending to out; the whole workgroup of T threads together.  The k-th highest key is
// found eight bits at a time, among those that differ, from counts of the keys that agree with it so far; then one pass in order.  R keys to a thread are held in
// registers; R 0: any number of them, read again in every pass.
template <int T, int R>
struct Held {
  uint32_t u[R ? R : 1];
  __device__ inline void load(const uint32_t* keys, int begin, int end) {
    if constexpr (R > 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = begin + r * T + (int)threadIdx.x;
        u[r] = i < end ? keys[i] : 0;                             // (no key is 0: that is the pattern of a NaN)
      }
    }
  }
};
template <int T, int R>
__device__ inline void pick(const Held<T, R>& held, const uint32_t* keys, int begin, int end, int k, int32_t* out, Scratch& sh) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const auto& u = held.u;
  uint32_t all = 0xFFFFFFFFu, any = 0;
  const auto each = [&](const auto& f) __attribute__((always_inline)) {
    if constexpr (R > 0) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (begin + r * T + tid < end) f(u[r]);
    } else {
      for (int i = begin + tid; i < end; i += T) f(keys[i]);
    }
  };
  each([&](uint32_t x) { all &= x, any |= x; });
  reduce_bits(all, any);
  if (tid == 0) {
    sh.all = 0xFFFFFFFFu;
    sh.any = 0;
  }
  __syncthreads();
  if (lane == 0) {
    atomicAnd(&sh.all, all);
    atomicOr(&sh.any, any);
  }
  __syncthreads();
  const uint32_t differ = sh.all ^ sh.any;
  uint32_t prefix = sh.all & ~differ, mask = ~differ;
  int need = k;
  for (int top = differ ? 31 - __clz((int)differ) : -1; top >= 0;) {
    const int shift = max(top - 7, 0), bins = (2 << (top - shift)) - 1;
    for (int i = tid; i < 256; i += T) sh.hist[i] = 0;
    __syncthreads();
    each([&](uint32_t x) {
      if ((x & mask) == (prefix & mask)) atomicAdd(&sh.hist[x >> shift & bins], 1);
    });
    __syncthreads();
    if (wave == 0) {                                              // bins from the highest down, four to a lane
      int c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = sh.hist[255 - (lane * 4 + j)];
      int before = (int)sum_up_to((uint32_t)sum) - sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < need && before + c[j] >= need) {
          sh.bin = 255 - (lane * 4 + j);
          sh.need = need - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    prefix = (prefix & ~((uint32_t)bins << shift)) | (uint32_t)sh.bin << shift;
    mask |= (uint32_t)bins << shift;
    need = sh.need;
    const uint32_t below = differ & ((1u << shift) - 1);
    top = below ? 31 - __clz((int)below) : -1;
  }
  // in order: counts of every wave's 64 keys (those above in the low half, those that are the k-th itself in the high one: R * T is below 2^16), what comes before each, places
  constexpr int S = R ? R : 1, W = T / 64, E = S * W;
  static_assert(E <= 256 && S * T < 65536);
  const uint64_t below = (1ull << lane) - 1;
  uint32_t base = 0;
  for (int from = begin; from < end; from += S * T) {
    uint64_t bg[S], be[S];
#pragma unroll
    for (int r = 0; r < S; ++r) {
      const int i = from + r * T + tid;
      uint32_t x;
      if constexpr (R > 0) x = u[r];
      else x = i < end ? keys[i] : 0;
      bg[r] = __ballot(i < end && x > prefix);
      be[r] = __ballot(i < end && x == prefix);
      if (lane == 0) sh.counts[r * W + wave] = (uint32_t)__popcll(be[r]) << 16 | (uint32_t)__popcll(bg[r]);
    }
    __syncthreads();
    if (wave == 0) {
      constexpr int C = (E + 63) / 64;
      uint32_t c[C], sum = 0;
#pragma unroll
      for (int j = 0; j < C; ++j) sum += c[j] = lane * C + j < E ? sh.counts[lane * C + j] : 0;
      uint32_t before = sum_up_to(sum);
      if (lane == 63) sh.any = before;
      before -= sum;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        if (lane * C + j < E) sh.counts[lane * C + j] = before;
        before += c[j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < S; ++r) {
      const uint32_t before = sh.counts[r * W + wave];
      const int ng = (int)(base & 0xFFFFu) + (int)(before & 0xFFFFu) + __popcll(bg[r] & below);
      const int ne = (int)(base >> 16) + (int)(before >> 16) + __popcll(be[r] & below);
      const bool gt = bg[r] >> lane & 1, eq = be[r] >> lane & 1;
      if (gt || (eq && ne < need)) out[ng + min(ne, need)] = from + r * T + tid;
    }
    // (what is above is fewer than k, at most 4096; of the k-th itself no more than that have to be told apart)
    const uint32_t total = sh.any, e = min((base >> 16) + (total >> 16), 32767u);
    base = e << 16 | ((base + total) & 0xFFFFu);
    __syncthreads();
  }
}

// The same by one wave with its keys in registers, R to a lane: the k-th highest key a bit at a time.  (A key is never 0: that is the pattern of a NaN.)
template <int R>
__device__ inline void pick_by_wave(const uint32_t* keys, int begin, int end, int k, int32_t* out, int lane) {
  uint32_t u[R], all = 0xFFFFFFFFu, any = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = begin + r * 64 + lane;
    u[r] = i < end ? keys[i] : 0;
    all &= i < end ? u[r] : 0xFFFFFFFFu;
    any |= u[r];
  }
  reduce_bits(all, any);
  uint32_t differ = __builtin_amdgcn_readfirstlane(all ^ any), least = __builtin_amdgcn_readfirstlane(all) & ~differ;
  auto at_least = [&](uint32_t x) __attribute__((always_inline)) {
    int n = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) n += __popcll(__ballot(u[r] >= x));
    return n;
  };
  int need = 0;                                                   // of the keys that are `least` itself
  bool exact = false;
  while (differ) {
    const uint32_t bit = 0x80000000u >> __clz((int)differ);
    differ ^= bit;
    const int n = at_least(least | bit);
    if (n >= k) least |= bit;
    if (n == k) {
      exact = true;
      break;
    }
  }
  if (exact) --least;
  else {                                                          // (counted by what is above it: the key of infinite bounds has no successor)
    need = k;
#pragma unroll
    for (int r = 0; r < R; ++r) need -= __popcll(__ballot(u[r] > least));
  }
  int ng = 0, ne = 0;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool gt = u[r] > least, eq = u[r] == least;
    const uint64_t bg = __ballot(gt), be = __ballot(eq);
    const int rank = ne + __popcll(be & below);
    if (gt || (eq && rank < need)) out[ng + __popcll(bg & below) + min(rank, need)] = begin + r * 64 + lane;
    ng += __popcll(bg);
    ne += __popcll(be);
  }
}

// What a row selects without a look at scores, by T threads; returns how many it selects by them.
template <int T>
__device__ inline int select_plain(const Select& a, int own, int32_t* out, int tid) {
  const int seen = own + 1;
  if (seen <= a.budget) {
    for (int j = tid; j < a.budget; j += T) out[j] = j < seen ? j : -1;
    return 0;
  }
  const int k = a.budget - a.sink - a.recent;
  for (int j = tid; j < a.sink + a.recent; j += T) {
    if (j < a.sink) out[j] = j;
    else out[k + j] = own - a.recent + 1 + (j - a.sink);
  }
  return k;
}

// Pointers to the query of column l16 of a tile of rows i0 .. i0 + rows - 1, features 64 c + 16 g + 8 p.
template <int HD, int COLS>
__device__ inline void query_of(const uint16_t* (&src)[HD / 64][2], const Select& a, int s, int kvh, int i0, int rows, int lane) {
  const int g = lane >> 4, l16 = lane & 15, i = min(i0 + l16 / COLS, i0 + rows - 1), h = min(l16 % COLS, a.group - 1);
#pragma unroll
  for (int c = 0; c < HD / 64; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int f = c * 64 + g * 16 + p * 8;
      src[c][p] = a.tiles ? a.q + ((size_t)s * a.n_kv_heads + kvh) * 16 * HD + pk_off(h, f, HD)
                          : a.q + ((int64_t)s * a.rows.window + i) * a.q_stride + (int64_t)(kvh * a.group + h) * HD + f;
    }
}

// Status of a sequence, its whole table looked at by the workgroup.
__device__ inline int whole_status(const Rows& r, int s, int len, int n) {
  const int status = length_status(r, len, n);
  bool bad = false;
  if (status == LLM42_SEQ_OK && n > 0) {
    constexpr int U = 8;
    const int32_t* ids = r.block_table + (size_t)s * r.width;
    const int last = (len + n - 1) / LLM42_KV_BLOCK;
    for (int b = threadIdx.x; b <= last; b += U * blockDim.x) {
      int id[U];
#pragma unroll
      for (int u = 0; u < U; ++u) id[u] = ids[min(b + u * (int)blockDim.x, last)];
#pragma unroll
      for (int u = 0; u < U; ++u) bad |= id[u] < 0 || id[u] >= r.num_blocks;
    }
  }
  return __syncthreads_or(bad) ? LLM42_SEQ_BAD_BLOCK : status;
}

// Keys of blocks begin .. end - 1 (of the sequence) for a tile of rows, by the waves of a workgroup in turn, four times 16 blocks at once; keys of tile row r at
// keys + r * stride, a multiple of 16 (those around begin and end - 1 may be anything).  id_of(b): the physical block.
template <int HD, int COLS, class Ids>
__device__ inline void score_blocks(const Select& a, const Query<HD>& q, int kvh, int rows, int begin, int end, uint32_t* keys, int64_t stride,
                                    u32x4 (&stage)[kWaves][16 * Record<HD>::P], Ids id_of) {
  constexpr int U = 4;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int end_tile = (end + 15) / 16;
  for (int t0 = begin / 16 + wave * U; t0 < end_tile; t0 += kWaves * U) {
    Record<HD> d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const auto rec_of = [&](int r) __attribute__((always_inline)) {
        const int b = min(max((t0 + u) * 16 + r, begin), end - 1);
        return a.bounds + ((size_t)id_of(b) * a.n_kv_heads + kvh) * bounds_record(HD);
      };
      d[u].load(rec_of, lane);
    }
    __builtin_amdgcn_sched_barrier(0);                            // (all of them asked for before the first is waited for)
    u32x4 key[U];
    score16<HD, COLS, U>(key, d, q, stage[wave], lane);
    if (l16 % COLS == 0 && l16 / COLS < rows) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (t0 + u < end_tile) *(u32x4*)(keys + (l16 / COLS) * stride + (t0 + u) * 16 + g * 4) = key[u];
    }
  }
}

template <int HD, int COLS>
__device__ inline Query<HD> query(const Select& a, int s, int kvh, int i0, int rows) {
  const uint16_t* src[HD / 64][2];
  query_of<HD, COLS>(src, a, s, kvh, i0, rows, threadIdx.x & 63);
  Query<HD> q;
  quantize<HD>(q, src);
  return q;
}

// Scores in LDS: a workgroup per (sequence, tile of 16 / group rows), blockIdx.y: kv head.  The ids of the blocks wait in the first row's place in LDS until
// their scores take it (a wave reads and writes the same 64 of them).  128 rows of 1024 - 8191 positions and 8 kv heads of 128, 75 MB, take 23 us: the records at 5 TB/s, then
// the pick of a row by one wave, 4, which all workgroups reach together; few rows take five trips that wait for each other and the pick, 7 - 9.
template <int HD, int COLS>
__global__ __launch_bounds__(kThreads) void select_kernel(Select a, int tile_rows, int tiles, int stride) {
  extern __shared__ __align__(16) uint32_t sh_keys[];
  __shared__ u32x4 stage[kWaves][16 * Record<HD>::P];
  __shared__ Scratch sh;
  const Rows& r = a.rows;
  const int s = blockIdx.x / tiles, i0 = blockIdx.x % tiles * tile_rows, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  int status = length_status(r, len, n);
  const int rows = min(tile_rows, n - i0), last = (len + i0 + rows - 1) / LLM42_KV_BLOCK, scored = last + 1 - a.recent;
  const bool scores = status == LLM42_SEQ_OK && rows > 0 && last + 1 > a.budget && a.budget > a.sink + a.recent;
  bool bad = false;
  if (status == LLM42_SEQ_OK && n > 0)
    for (int b = threadIdx.x; b <= (len + n - 1) / LLM42_KV_BLOCK; b += kThreads) {
      const int id = r.block_table[(size_t)s * r.width + b];
      bad |= id < 0 || id >= r.num_blocks;
      if (scores && b < scored) sh_keys[b] = (uint32_t)id;
    }
  Query<HD> q;
  if (scores) q = query<HD, COLS>(a, s, kvh, i0, rows);
  if (__syncthreads_or(bad)) status = LLM42_SEQ_BAD_BLOCK;
  if (a.seq_status && i0 == 0 && kvh == 0 && threadIdx.x == 0) a.seq_status[s] = status;
  if (status != LLM42_SEQ_OK || rows <= 0) return;
  if (scores) {
    score_blocks<HD, COLS>(a, q, kvh, rows, a.sink, scored, sh_keys, stride, stage, [&](int b) { return sh_keys[b]; });
    __syncthreads();
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const auto out_of = [&](int i) { return a.selected + (((size_t)s * r.window + i0 + i) * a.n_kv_heads + kvh) * a.budget; };
  const int most = scored - a.sink;
  if (!scores || most <= 1024) {                                  // a row to a wave
    for (int i = wave; i < rows; i += kWaves) {
      const int own = (len + i0 + i) / LLM42_KV_BLOCK, end = own + 1 - a.recent;
      int32_t* out = out_of(i);
      const int k = select_plain<64>(a, own, out, lane);
      const uint32_t* keys = sh_keys + i * stride;
      if (k == 0) continue;
      if (most <= 256) pick_by_wave<4>(keys, a.sink, end, k, out + a.sink, lane);
      else if (most <= 512) pick_by_wave<8>(keys, a.sink, end, k, out + a.sink, lane);
      else pick_by_wave<16>(keys, a.sink, end, k, out + a.sink, lane);
    }
    return;
  }
  for (int i = 0; i < rows; ++i) {
    const int own = (len + i0 + i) / LLM42_KV_BLOCK;
    const int k = select_plain<kThreads>(a, own, out_of(i), threadIdx.x);
    if (k) pick<kThreads, 0>(Held<kThreads, 0>(), sh_keys + i * stride, a.sink, own + 1 - a.recent, k, out_of(i) + a.sink, sh);
    __syncthreads();
  }
}

// Scores through the workspace, first launch: a workgroup per (sequence, tile of rows) and chunk of blocks (blockIdx.z).
template <int HD, int COLS>
__global__ __launch_bounds__(kThreads) void score_kernel(Select a, int tile_rows, int tiles, int64_t stride, int chunk) {
  const Rows& r = a.rows;
  const int s = blockIdx.x / tiles, i0 = blockIdx.x % tiles * tile_rows, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  if (length_status(r, len, n) != LLM42_SEQ_OK || i0 >= n) return;
  const int rows = min(tile_rows, n - i0), last = (len + i0 + rows - 1) / LLM42_KV_BLOCK;
  if (last + 1 <= a.budget || a.budget == a.sink + a.recent) return;
  const int begin = max(a.sink, (int)blockIdx.z * chunk), end = min(last + 1 - a.recent, ((int)blockIdx.z + 1) * chunk);
  if (begin >= end) return;
  // (the ids wait in LDS where they are no more than that)
  __shared__ int32_t sh_ids[kChunk];
  __shared__ u32x4 stage[kWaves][16 * Record<HD>::P];
  const int32_t* ids = r.block_table + (size_t)s * r.width;
  bool bad = false;
  for (int b = begin + threadIdx.x; b < end; b += kThreads) {
    const int id = ids[b];
    bad |= id < 0 || id >= r.num_blocks;
    if (chunk == kChunk) sh_ids[b - (int)blockIdx.z * kChunk] = id;
  }
  const Query<HD> q = query<HD, COLS>(a, s, kvh, i0, rows);
  if (__syncthreads_or(bad)) return;                              // (the second launch sees it too)
  uint32_t* keys = a.keys + (((size_t)s * r.window + i0) * a.n_kv_heads + kvh) * stride;
  if (chunk == kChunk)
    score_blocks<HD, COLS>(a, q, kvh, rows, begin, end, keys, a.n_kv_heads * stride, stage, [&](int b) { return sh_ids[b - (int)blockIdx.z * kChunk]; });
  else
    score_blocks<HD, COLS>(a, q, kvh, rows, begin, end, keys, a.n_kv_heads * stride, stage, [&](int b) { return ids[b]; });
}

// ... and second: a workgroup per row, blockIdx.y: kv head.  R: keys that a thread holds, 0 any number.  They are asked for together with the table that says whether the sequence is in
// order (what the workspace holds where it is not is of no use and does no harm).
constexpr int kPickThreads = 1024;
template <int R>
__global__ __launch_bounds__(kPickThreads) void pick_kernel(Select a, int64_t stride) {
  __shared__ Scratch sh;
  const Rows& r = a.rows;
  const int s = blockIdx.x / r.window, i = blockIdx.x % r.window, kvh = blockIdx.y;
  const int len = r.seq_len[s], n = r.seq_n ? r.seq_n[s] : r.window;
  const size_t at = ((size_t)s * r.window + i) * a.n_kv_heads + kvh;
  const uint32_t* keys = a.keys + at * stride;
  const int own = (len + i) / LLM42_KV_BLOCK, end = own + 1 - a.recent;
  Held<kPickThreads, R> held;
  if (length_status(r, len, n) == LLM42_SEQ_OK && i < n) held.load(keys, a.sink, end);   // (a row that is not there may lie behind max_context)
  const int status = whole_status(r, s, len, n);
  if (a.seq_status && i == 0 && kvh == 0 && threadIdx.x == 0) a.seq_status[s] = status;
  if (status != LLM42_SEQ_OK || i >= n) return;
  int32_t* out = a.selected + at * a.budget;
  const int k = select_plain<kPickThreads>(a, own, out, threadIdx.x);
  if (k) pick<kPickThreads, R>(held, keys, a.sink, end, k, out + a.sink, sh);
}

// Keys of a tile row, one for each block that max_context positions can have, a multiple of 16.
int64_t keys_of(int max_context) { return ((int64_t)max_context + 255) / 256 * 16; }
int cols_of(int group) { return group > 8 ? 16 : group > 4 ? 8 : group > 2 ? 4 : group; }
int tile_rows_of(int group, int window) { return std::min(16 / cols_of(group), window); }
constexpr int64_t kMostLdsKeys = 12288;      // 48 KiB, beside 8 or 16 for the records that are turned and 2 of counts: two workgroups to a CU
// Scores that wait in the workspace at once, unless one sequence alone has more: a call of more goes through it some sequences at a time.
constexpr size_t kMostScores = 256u << 20;
size_t scores_of(int window, int n_kv_heads, int max_context) { return 4ull * window * n_kv_heads * keys_of(max_context); }   // (of a sequence)

}  // namespace

size_t select_workspace(int num_seqs, int window, int n_kv_heads, int group, int max_context, int budget, int num_cus) {
  const int64_t keys = keys_of(max_context);
  const int tile_rows = tile_rows_of(group, window);
  const int64_t wgs = (int64_t)num_seqs * ((window + tile_rows - 1) / tile_rows) * n_kv_heads;
  if (keys <= budget) return 0;
  // A workgroup gets about 20 bytes a ns from memory, so few of them with long contexts leave the
  // device idle: their scores go through the workspace, 256 blocks to a workgroup, and a second launch picks (us so / in LDS, sequences x positions, 8 kv heads
  // of 128, group 4: 1 x 4096 12.0 / 8.8, 1 x 8192 12.3 / 12.5, 1 x 16384 13.0 / 19.6, 8 x 16384 13.6 / 20.6, 16 x 32768 25.7 / 34.7, 1 x 131072
  // 27 / 109, 1 window of 64 x 30000 22.7 / 59; 32 x 32768 36.7 / 38.8; but 64 x 32768 75 / 62, 128 x 8192 42 / 32, 4 windows of 32 x 8000 25 / 16.5).  Those of a tile of rows that LDS does not
  // hold go there too.
  if (tile_rows * keys <= kMostLdsKeys && (2 * wgs > num_cus || keys <= 512)) return 0;
  const size_t one = scores_of(window, n_kv_heads, max_context);
  return std::min(num_seqs * one, std::max(one, kMostScores));
}

// The call's sequences from .. from + n - 1 as a call of their own.
static Select sequences_from(Select a, int from, int n) {
  Rows& r = a.rows;
  r.num_seqs = n;
  r.block_table += (size_t)from * r.width;
  r.seq_len += from;
  if (r.seq_n) r.seq_n += from;
  a.q += a.tiles ? (int64_t)from * a.n_kv_heads * 16 * a.head_dim : (int64_t)from * r.window * a.q_stride;
  a.selected += (size_t)from * r.window * a.n_kv_heads * a.budget;
  if (a.seq_status) a.seq_status += from;
  return a;
}

void launch_kv_select(const Select& a, hipStream_t st) {
  const Rows& r = a.rows;
  const int tile_rows = tile_rows_of(a.group, r.window), tiles = (r.window + tile_rows - 1) / tile_rows;
  const int64_t keys = keys_of(r.max_context);
  const auto go = [&](auto hd, auto cols) {
    constexpr int HD = decltype(hd)::value, COLS = decltype(cols)::value;
    if (!a.keys) {
      const size_t lds = keys <= a.budget ? 0 : 4 * tile_rows * keys;
      select_kernel<HD, COLS><<<dim3(r.num_seqs * tiles, a.n_kv_heads), kThreads, lds, st>>>(a, tile_rows, tiles, (int)keys);
      return;
    }
    const int chunk = (int)std::max<int64_t>(kChunk, (keys + 65535) / 65536 * 16);
    const int at_once = (int)std::min<size_t>(r.num_seqs, std::max<size_t>(1, kMostScores / scores_of(r.window, a.n_kv_heads, r.max_context)));
    for (int from = 0; from < r.num_seqs; from += at_once) {
      const Select b = sequences_from(a, from, std::min(at_once, r.num_seqs - from));
      const int rows = b.rows.num_seqs * r.window;
      score_kernel<HD, COLS><<<dim3(b.rows.num_seqs * tiles, a.n_kv_heads, (unsigned)((keys + chunk - 1) / chunk)), kThreads, 0, st>>>(b, tile_rows, tiles, keys, chunk);
      const auto pick = [&](auto held) { pick_kernel<decltype(held)::value><<<dim3(rows, a.n_kv_heads), kPickThreads, 0, st>>>(b, keys); };
      if (keys <= 2 * kPickThreads) pick(std::integral_constant<int, 2>{});
      else if (keys <= 8 * kPickThreads) pick(std::integral_constant<int, 8>{});
      else pick(std::integral_constant<int, 0>{});
    }
  };
  const auto by_cols = [&](auto hd) {
    switch (cols_of(a.group)) {
      case 1: return go(hd, std::integral_constant<int, 1>{});
      case 2: return go(hd, std::integral_constant<int, 2>{});
      case 4: return go(hd, std::integral_constant<int, 4>{});
      case 8: return go(hd, std::integral_constant<int, 8>{});
      default: return go(hd, std::integral_constant<int, 16>{});
    }
  };
  if (a.head_dim == 128) by_cols(std::integral_constant<int, 128>{});
  else by_cols(std::integral_constant<int, 64>{});
}
