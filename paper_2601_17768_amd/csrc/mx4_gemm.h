// Products with 4-bit matrices, D[feature][token] = sum_k W[feature][k] X[token][k], W in MXFP4, X bf16, with the epilogues of the
// bf16 GEMMs.  The codes are converted to bf16 operands with their scales in registers - exactly, a 4-bit value times a
// power of two being a bf16 - and multiplied by v_mfma_f32_16x16x32_bf16, sums in fp32.  A template of the epilogue; each
// mx4_gemm_*.hip holds the kernels of one or two.
#pragma once
#include <utility>

#include "gemm_parts.h"
#include "mx4.h"

namespace mx4 {

using namespace gemm;

// Where the activations lie: the tile layout, or plain rows of `stride` elements.
struct X {
  const uint16_t* p;
  int64_t stride;           // 0: tiles
  int k_tiles, last_row;
  int tail = 0;             // mx4_stream_kernel of loose rows: columns behind the k-tiles (which are the whole ones then)
  // what lane `lane` of token block `block` takes of k-tile 0, and from a k-tile to the next; rows that only pad repeat the last one
  __device__ const uint16_t* at(int block, int lane) const {
    const int row = min(block * 16 + (lane & 15), last_row);
    return stride ? p + (int64_t)row * stride + (lane >> 4) * 8
                  : p + ((size_t)(row >> 4) * k_tiles * 64 + (lane >> 4) * 16 + (row & 15)) * 8;
  }
  __device__ int step() const { return stride ? 32 : 512; }
  // where token block `block` begins: the wave-uniform part of an address; a block past the last one repeats it
  __device__ const uint16_t* block_base(int block) const {
    const int b = min(block, last_row >> 4);
    return p + (stride ? (int64_t)b * 16 * stride : (int64_t)b * k_tiles * 512);
  }
};

// Up to 16 or 32 rows (TB token blocks).  A workgroup owns FB feature blocks; its eight waves take the groups of 4 k-tiles in turn, each
// with accumulators of its own for all of them, and are added through LDS.  Codes and activations of two groups are on their way at
// a time; no barrier, for no two waves want the same bytes.  A wave has four groups of a 4096-column matrix, so nothing is loaded past the
// last one (1 row of 6144 x 4096 so 6.2 -> 4.6 us, from memory 7.7 -> 5.8; 28672 x 4096 from memory 15.1 -> 13.9, 4.5 TB/s).  LOOSE: plain
// rows of any number of columns that are only 4-byte aligned are read as they lie (behind a launch that brings them in order first 13
// rows of 1000 x 700 took 7.8 us instead of 4.6, 16 of 4096 x 4100 11.6 instead of 8.9); the last wave takes the columns behind
// the last whole k-tile.  (Rows that begin in the middle of a word are brought in order: 16 rows of 4096 x 4097 took 28 us by loads of
// 16 bytes, 13.4 by aligned words and shifts, 11.7 so.)
constexpr int kStreamWaves = 8, kStreamRows = 16, kStreamWide = 4;   // (feature blocks that fit beside 32 rows)
template <int FB, int TB, bool LOOSE, class Epi>
__global__ __launch_bounds__(64 * kStreamWaves) void mx4_stream_kernel(const char* __restrict__ w, X x, int n_blocks, int units, Epi epi) {
  constexpr int NW = kStreamWaves;
  static_assert(TB == 1 || !LOOSE, "loose rows are those of one token block");
  __shared__ f32x4 part[NW][FB * TB * 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n0 = blockIdx.x * FB;
  const char* wp[FB];
#pragma unroll
  for (int i = 0; i < FB; ++i) wp[i] = w + (size_t)min(n0 + i, n_blocks - 1) * units * kRecord;
  const uint16_t* xp[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) xp[b] = x.at(b, lane);
  const int xs = x.step(), mine = ((x.k_tiles + 3) / 4 - wave + NW - 1) / NW;
  f32x4 acc[FB][TB];
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[i][b] = (f32x4){0.f, 0.f, 0.f, 0.f};
  u32x4 codes[2][FB];
  uint32_t scales[2][FB];
  bf16x8 xv[2][4][TB];
  auto load = [&](auto set, int i) __attribute__((always_inline)) {
    constexpr int U = decltype(set)::value;
    const int g = i * NW + wave;
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const char* rec = wp[f] + (size_t)(g >> 1) * kRecord;
      codes[U][f] = __builtin_nontemporal_load((const u32x4*)(rec + (g & 1) * 1024 + lane * 16));
      scales[U][f] = *(const uint32_t*)(rec + kScales + (g & 1) * 4 + (lane & 15) * 8);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        typedef bf16x8 words __attribute__((aligned(4)));
        const uint16_t* from = xp[b] + (size_t)min(g * 4 + j, x.k_tiles - 1) * xs;
        xv[U][j][b] = LOOSE ? (bf16x8)*(const words*)from : *(const bf16x8*)from;
      }
  };
  auto compute = [&](auto set, int i) __attribute__((always_inline)) {
    constexpr int U = decltype(set)::value;
    const int k0 = (i * NW + wave) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (k0 + j >= x.k_tiles) break;                // (columns that only pad: X has none there)
#pragma unroll
      for (int f = 0; f < FB; ++f) {
        const bf16x8 a = operand(codes[U][f][j], scale_of(scales[U][f], j));
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[f][b] = mfma16(a, xv[U][j][b], acc[f][b]);
      }
    }
  };
  using Set0 = std::integral_constant<int, 0>;
  using Set1 = std::integral_constant<int, 1>;
  if (mine >= 2) {
    load(Set0{}, 0);
    load(Set1{}, 1);
    int i = 0;
    const auto step = [&](auto set, int at, bool more) __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      compute(set, at);
      __builtin_amdgcn_sched_barrier(0);
      if (more) load(set, at + 2);
    };
    for (; i + 4 <= mine; i += 2) {                  // (a branch around the loads would have them waited for too early)
      step(Set0{}, i, true);
      step(Set1{}, i + 1, true);
    }
    step(Set0{}, i, i + 2 < mine);
    step(Set1{}, i + 1, false);
    if (i + 2 < mine) compute(Set0{}, i + 2);
  } else if (mine == 1) {
    load(Set0{}, 0);
    compute(Set0{}, 0);
  }
  if (LOOSE && x.tail && wave == NW - 1) {
    const uint16_t* from = xp[0] + (size_t)x.k_tiles * 32;
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((lane >> 4) * 8 + i < x.tail) v[i >> 1] |= (uint32_t)from[i] << (16 * (i & 1));
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const char* rec = wp[f] + (size_t)(x.k_tiles >> 3) * kRecord;
      const uint32_t word = *(const uint32_t*)(rec + (x.k_tiles >> 2 & 1) * 1024 + lane * 16 + (x.k_tiles & 3) * 4);
      const uint32_t byte = *(const uint8_t*)(rec + kScales + (lane & 15) * 8 + (x.k_tiles & 7));
      acc[f][0] = mfma16(operand(word, scale_of(byte, 0)), __builtin_bit_cast(bf16x8, v), acc[f][0]);
    }
  }
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int b = 0; b < TB; ++b) part[wave][(i * TB + b) * 64 + lane] = acc[i][b];
  __syncthreads();
  const int nb = n0 + wave / TB, row = wave % TB * 16 + (lane & 15);
  static_assert(FB * TB <= NW, "a wave adds up one block");
  if (wave < FB * TB && nb < n_blocks) {
    f32x4 sum = part[0][wave * 64 + lane];
#pragma unroll
    for (int v = 1; v < NW; ++v) sum += part[v][wave * 64 + lane];
    epi(nb, lane, row, sum, epi.pre(nb, lane, row, epi.row_info(row)));
  }
}

// At most `rounds` rounds of PW fetches each are still on their way.
template <int MOST, int PW>
__device__ __forceinline__ void wait_rounds(int rounds) {
  static_assert(MOST >= 1 && MOST <= 4 && MOST * PW <= 63, "vmcnt counts up to 63");
  if (MOST >= 4 && rounds >= 4) lds_fetch_wait<(MOST >= 4 ? 4 : 0) * PW>();
  else if (MOST >= 3 && rounds >= 3) lds_fetch_wait<(MOST >= 3 ? 3 : 0) * PW>();
  else if (MOST >= 2 && rounds >= 2) lds_fetch_wait<(MOST >= 2 ? 2 : 0) * PW>();
  else if (rounds >= 1) lds_fetch_wait<PW>();
  else lds_fetch_wait<0>();
}

// Many rows.  A workgroup owns NW * FB feature blocks x TB token blocks.  Each of NW waves owns FB of the feature blocks and all the
// token blocks; it loads its codes straight into registers, NSET groups of 4 k-tiles (one in use, the others on their way), and converts
// an operand for every TB products.  F further waves move the activations into a ring of R rounds of CH k-tiles in LDS, one
// barrier per round: behind barrier r rounds r and r + 1 have landed, so that a wave's operand reads run on across the barrier, and
// the slot of round r - 1 is refilled.
// Plain rows are fetched in runs of CH * 64 bytes of a row and lie in LDS as they come, a row's 16-byte pieces exchanged by the row's
// number so that the 16 rows of an operand read are in 16 different bank groups (pieces of 64 bytes, 16 rows apart by a
// power of two, meet in few of the L2's channels; 128 rows of 28672 x 4096 so 44 us, in runs 35).
// Many rows are bound by the matrix cores: 4096 rows of 28672 x 4096 679 us, 1.42 PFLOP/s (the library's product of the two in bf16 723), the
// conversions hidden behind 16 products each.  Up to 128 rows wait for loads (copies without activations / weights / products / either kind of
// load, from memory: 128 rows of 28672 x 4096 29.0 / 28.4 / 28.7 / 23 of 31 us, 24 of it 18.6 / 14.9 / 21 / 8.7 of 22, 128 of 4096 x 4096
// 12.1 / 9.6 / 14.5 / 5.2 of 14.7), sums in parts for launches and planes as well (24 of 4096 x 14336 14.6 / 14.1 / 15.8 / 12.7 of 16.4).
template <int NW, int FB, int TB, int CH, int R, int F, int NSET, class Epi>
__global__ __launch_bounds__(64 * (NW + F), (NW + F + 3) / 4) void mx4_tile_kernel(const char* __restrict__ w, X x, int n_blocks, int units,
                                                                                   int tiles_n, int tiles_m, int parts, int part_groups, Epi epi) {
  constexpr int TBN = NW * FB, PW = CH * TB / F, PB = TB / F, SUB = 4 / CH, PD = 7;
  static_assert(TB % F == 0 && (CH == 2 || CH == 4) && CH * TB % (PD + 1) == 0, "the fetching waves take whole token blocks");
  __shared__ bf16x8 ring[R][CH * TB * 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15;
  const int all = tiles_n * tiles_m, per_xcd = (all * parts + 7) / 8;
  const int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3), part = tile / all, at = tile - part * all;
  if ((int)(blockIdx.x >> 3) >= per_xcd || part >= parts) return;
  if constexpr (std::is_same<Epi, StorePartialEpi>::value) epi.partial += part * epi.plane;
  // an XCD takes a contiguous run of the tiles, panel by panel of about 1024 tokens, token tiles fastest within a panel
  constexpr int PANEL = 64 / TB;
  const int panel = at / (tiles_n * PANEL), in = at - panel * tiles_n * PANEL, width = min(PANEL, tiles_m - panel * PANEL);
  const int n0 = in / width * TBN, m0 = (panel * PANEL + in % width) * TB;
  const int k_begin = part * part_groups * 4, k_tiles = min(x.k_tiles - k_begin, part_groups * 4), rounds = (k_tiles + CH - 1) / CH;
  // Up to 32 rows the workgroups of an XCD begin at different columns, so that they do not all ask one L2 channel for the same activations
  // (24 rows of 4096 x 14336 15.9 -> 14.9 us, of 28672 x 4096 18.6 -> 17.8; 64 of 6144 x 4096 12.0 -> 12.6, 512 of 4096 x 14336 54 -> 60:
  // with several tiles of rows they share what each has just fetched)
  const int turn = TB > 2 || tiles_m > 1 || k_tiles % 4 ? 0 : (int)((uint32_t)(blockIdx.x >> 3) * (uint32_t)(k_tiles / 4) / (uint32_t)per_xcd);
  if (wave >= NW) {
    const int fw = wave - NW;
    const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&ring[0][0] + fw * PW * 1024;
    const uint16_t* src[PB];
    uint32_t off[PW], piece[CH];                     // a lane's row (or place in a tile), and where in the round's run of it
#pragma unroll
    for (int i = 0; i < PB; ++i) src[i] = x.block_base(m0 + fw * PB + i) + (size_t)k_begin * x.step();
    if (x.stride) {
      constexpr int PIECES = CH * 4, ROWS = 64 / PIECES;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int r = j * ROWS + lane / PIECES;
        piece[j] = (uint32_t)((lane % PIECES) ^ (CH == 4 ? r : r >> 1)) * 16u;
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        const int block = m0 + fw * PB + i / CH, r = min(i % CH * ROWS + lane / PIECES, x.last_row - min(block, x.last_row >> 4) * 16);
        off[i] = (uint32_t)r * (uint32_t)x.stride * 2u;
      }
    } else {
#pragma unroll
      for (int j = 0; j < CH; ++j) piece[j] = j * 1024u;
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        const int block = m0 + fw * PB + i / CH;
        off[i] = (uint32_t)((lane >> 4) * 16 + min(l16, x.last_row - min(block, x.last_row >> 4) * 16)) * 16u;
      }
    }
    const uint32_t run = CH * x.step() * 2, most = x.stride ? k_tiles * 64u - 16u : (k_tiles - 1) * 1024u;
    auto fetch = [&](int r) {                        // (past the last k-tile: within it)
      const int from = r + turn * SUB < rounds ? r + turn * SUB : r + turn * SUB - rounds;
#pragma unroll
      for (int i = 0; i < PW; ++i)
        lds_fetch_1k(src[i / CH], min((uint32_t)from * run + piece[i % CH], most) + off[i], dst + (uint32_t)((r % R) * CH * TB + i) * 1024u);
    };
    for (int r = 0; r < min(R - 1, rounds); ++r) fetch(r);
    wait_rounds<R - 3, PW>(min(R - 3, rounds - 2));
    __syncthreads();                                 // (before the first operand reads)
    for (int r = 0; r < rounds; ++r) {
      wait_rounds<R - 3, PW>(min(R - 3, rounds - 2 - r));
      __syncthreads();                               // rounds r and r + 1 are in LDS; everyone is done with round r - 1
      if (r + R - 1 < rounds) fetch(r + R - 1);      // into the slot of round r - 1
    }
    return;
  }
  const char* wp[FB];
#pragma unroll
  for (int i = 0; i < FB; ++i) wp[i] = w + (size_t)min(n0 + wave * FB + i, n_blocks - 1) * units * kRecord;
  const int first_group = part * part_groups;
  uint32_t at_k[CH];                                 // a lane's bytes of k-tile j of a token block's part of a round
#pragma unroll
  for (int j = 0; j < CH; ++j)
    at_k[j] = x.stride ? (uint32_t)l16 * CH * 64u + (uint32_t)((j * 4 + (lane >> 4)) ^ (CH == 4 ? l16 : l16 >> 1)) * 16u : j * 1024u + lane * 16u;
  f32x4 acc[FB][TB];
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  u32x4 codes[NSET][FB];
  uint32_t scales[NSET][FB];
  const int groups = (k_tiles + 3) / 4;
  auto load = [&](auto set, int g) __attribute__((always_inline)) {   // (groups past the range re-read the last one)
    constexpr int U = decltype(set)::value;
    const int to = min(g, groups - 1) + turn, c = (to < groups ? to : to - groups) + first_group;
#pragma unroll
    for (int i = 0; i < FB; ++i) {
      const char* rec = wp[i] + (size_t)(c >> 1) * kRecord;
      codes[U][i] = *(const u32x4*)(rec + (c & 1) * 1024 + lane * 16);
      scales[U][i] = *(const uint32_t*)(rec + kScales + (c & 1) * 4 + (lane & 15) * 8);
    }
  };
  bf16x8 q[PD + 1];                                  // activation operands, requested PD products ahead, across rounds
  auto operand_x = [&](const char* round, int idx) { return *(const bf16x8*)(round + at_k[idx / TB] + idx % TB * CH * 1024); };
  // Group g of 4 k-tiles on register set U; FULL: all four are in range.
  auto group = [&](auto set, auto is_full, int g) __attribute__((always_inline)) {
    constexpr int U = decltype(set)::value, N = CH * TB;
    constexpr bool FULL = decltype(is_full)::value;
    bf16x8 a[2][FB];
#pragma unroll
    for (int i = 0; i < FB; ++i) a[0][i] = operand(codes[U][i][0], scale_of(scales[U][i], 0));
    u32x4 conv[FB];                                  // the next k-tile's operands on the way, 4 FB conversions dealt to TB products
#pragma unroll
    for (int c = 0; c < SUB; ++c) {
      const int r = g * SUB + c;
      if (!FULL && r >= rounds) break;
      const char *here = (const char*)ring[r % R], *next = (const char*)ring[(r + 1) % R];
      __syncthreads();
      if (c == 0) load(std::integral_constant<int, (U + NSET - 1) % NSET>{}, g + NSET - 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int idx = 0; idx < N; ++idx) {
        const int j = c * CH + idx / TB;
        q[(idx + PD) % (PD + 1)] = idx + PD < N ? operand_x(here, idx + PD) : operand_x(next, idx + PD - N);
        if (j < 3) {
#pragma unroll
          for (int e = idx % TB * 4 * FB / TB; e < (idx % TB + 1) * 4 * FB / TB; ++e) {
            const int i = e >> 2;
            conv[i][e & 3] = pair_bf16(codes[U][i][(j + 1) & 3], scale_of(scales[U][i], (j + 1) & 3), e & 3);
            if ((e & 3) == 3) a[(j + 1) & 1][i] = __builtin_bit_cast(bf16x8, conv[i]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (FULL || g * 4 + j < k_tiles) {
#pragma unroll
          for (int i = 0; i < FB; ++i) acc[i][idx % TB] = mfma16(a[j & 1][i], q[idx % (PD + 1)], acc[i][idx % TB]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto each_set = [&](const auto& f) __attribute__((always_inline)) {
    f(std::integral_constant<int, 0>{});
    f(std::integral_constant<int, 1>{});
    if constexpr (NSET > 2) f(std::integral_constant<int, NSET == 2 ? 0 : 2>{});
    if constexpr (NSET > 3) f(std::integral_constant<int, NSET == 2 ? 0 : 3>{});
  };
  static_assert(NSET >= 2 && NSET <= 4, "the groups are written out for 2 .. 4 register sets");
  each_set([&](auto u) __attribute__((always_inline)) {
    if constexpr (decltype(u)::value < NSET - 1) load(u, decltype(u)::value);
  });
  __syncthreads();                                   // rounds 0 and 1 are in LDS
#pragma unroll
  for (int t = 0; t < PD; ++t) q[t] = operand_x((const char*)ring[0], t);
  int g = 0;
  for (; (g + NSET) * 4 <= k_tiles; g += NSET)       // without an exit in between
    each_set([&](auto u) __attribute__((always_inline)) { group(u, std::true_type{}, g + decltype(u)::value); });
  each_set([&](auto u) __attribute__((always_inline)) {
    if (g + decltype(u)::value < groups) group(u, std::false_type{}, g + decltype(u)::value);
  });
  // epilogue; token blocks behind the last row have none
  const int blocks = (x.last_row >> 4) + 1;
  constexpr int EG = TB % 4 == 0 && FB <= 2 ? 4 : 2;
  constexpr bool kLogits = is_logits<Epi>::value;
  float2* best = (float2*)ring;                      // LM head: [NW][16 TB] best of a wave's features
  if constexpr (kLogits) __syncthreads();            // everyone is done with the ring (the fetching waves have left)
#pragma unroll
  for (int j0 = 0; j0 < TB; j0 += EG) {
    if (m0 + j0 >= blocks) break;
    typename Epi::Row info[EG];
    typename Epi::Pre pre[EG][FB];
#pragma unroll
    for (int j = 0; j < EG; ++j) {
      const int row = min(m0 + j0 + j, blocks - 1) * 16 + (lane & 15);
      info[j] = epi.row_info(row);
#pragma unroll
      for (int i = 0; i < FB; ++i) pre[j][i] = epi.pre(min(n0 + wave * FB + i, n_blocks - 1), lane, row, info[j]);
    }
#pragma unroll
    for (int j = 0; j < EG; ++j) {
      if constexpr (kLogits) {
        typename Epi::Best b;
#pragma unroll
        for (int i = 0; i < FB; ++i) {
          const int nb = n0 + wave * FB + i;
          if (nb < n_blocks) epi.rank(nb, lane, acc[i][j0 + j], info[j], b);
        }
        b = Epi::over_lanes(b);
        if (lane < 16) best[wave * 16 * TB + (j0 + j) * 16 + lane] = make_float2(b.v, __int_as_float(b.i));
      } else {
#pragma unroll
        for (int i = 0; i < FB; ++i) {
          const int nb = n0 + wave * FB + i;
          if (nb < n_blocks && m0 + j0 + j < blocks) epi(nb, lane, (m0 + j0 + j) * 16 + (lane & 15), acc[i][j0 + j], pre[j][i]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (kLogits) {
    __syncthreads();
    for (int t = threadIdx.x; t < 16 * TB; t += 64 * NW) {
      if (m0 + (t >> 4) >= blocks) break;
      typename Epi::Best b;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float2 p = best[v * 16 * TB + t];
        b.take(p.x, __float_as_int(p.y));
      }
      epi.amax[(size_t)(m0 * 16 + t) * tiles_n + n0 / TBN] = make_float2(b.v, __int_as_float(b.i));
    }
  }
}

// Tiles of mx4_tile_kernel, and what a round of one workgroup per CU takes by them: ns, ns per k-tile, and by how many percent more
// of that with every CU at work (fitted to times of 1 - 4096 rows, 16 - 131072 features and 256 - 14336 columns; they rank the tiles, and are
// no measurement of any one call).
struct Tile4 {
  int nw, fb, tb, ch, r, f, nset;
  int round_ns, k_ns, full;
  constexpr int bn() const { return nw * fb; }
};
constexpr Tile4 kTiles4[] = {
    {7, 2, 16, 2, 4, 1, 2, 3254, 499, 16}, {8, 2, 8, 4, 4, 4, 2, 2573, 267, 30}, {7, 1, 8, 4, 4, 4, 4, 2374, 131, 46},
    {4, 2, 8, 4, 4, 4, 4, 2644, 143, 40},  {8, 2, 4, 4, 6, 4, 3, 2475, 171, 38}, {4, 2, 4, 4, 6, 4, 4, 2035, 110, 50},
    {4, 1, 4, 4, 6, 4, 4, 1665, 68, 86},   {8, 1, 2, 4, 7, 2, 4, 1509, 85, 59},  {4, 1, 2, 4, 7, 2, 4, 1040, 64, 53}};
constexpr int kTileCount4 = sizeof kTiles4 / sizeof kTiles4[0];

template <int T, class Epi>
bool launch_tile4(int tile, const char* w, const X& x, int n_blocks, int rows, int parts, int part_groups, const Epi& epi, hipStream_t st) {
  if (tile != T) return false;
  constexpr Tile4 q = kTiles4[T];
  const int tiles_n = (n_blocks + q.bn() - 1) / q.bn(), tiles_m = (rows + 16 * q.tb - 1) / (16 * q.tb);
  const int per_xcd = (tiles_n * tiles_m * parts + 7) / 8;
  mx4_tile_kernel<q.nw, q.fb, q.tb, q.ch, q.r, q.f, q.nset, Epi><<<8 * per_xcd, 64 * (q.nw + q.f), 0, st>>>(
      w, x, n_blocks, (x.k_tiles + 7) / 8, tiles_n, tiles_m, parts, part_groups, epi);
  return true;
}
template <int... T, class Epi>
void launch_tiles4(std::integer_sequence<int, T...>, int tile, const char* w, const X& x, int n_blocks, int rows, int parts, int part_groups,
                   const Epi& epi, hipStream_t st) {
  (void)(launch_tile4<T>(tile, w, x, n_blocks, rows, parts, part_groups, epi, st) || ...);
}

// How a product runs.
struct Plan {
  int tile;                // of mx4_tile_kernel; -1: mx4_stream_kernel ...
  int fb;                  // ... by this many feature blocks
  int parts, part_groups;  // of the sum over k, and how many groups of 4 k-tiles each has
};
// mx4_stream_kernel for up to 16 rows (us, it / the best tile: 1 row of 4096 x 4096 4.8 / 9.2, 16 6.7 / 9.8; 1 of 28672 x 4096 13.1 / 19.6 from the memory-side cache, 16
// 14.6 / 19.9; 16 of 50304 x 512 7.4 / 7.9), except where more than 8 rows are summed over many columns for few features: it has but eight
// waves for a sum, each of which takes 0.6 us and 28 ns a row for a group, a tile several workgroups (16 rows of 512 x 14336 16.1 / 10.7,
// of 512 x 4096 6.1 / 7.7).  Up to 32 rows where four feature blocks a workgroup put one on every CU, by a like rule (24 rows of 1024 x 1024
// 3.8 / 5.3, 6144 x 4096 9.8 / 13.6 in one piece, 16384 x 4096 12.4 / 15.3; 32 of 4096 x 4096 10.3 / 8.9: every wave reads its columns of all
// rows, which bounds it).  A workgroup per CU where eight feature blocks are enough for that, else seven or eight, whichever leave fewer
// idle in the last round (16 rows, us by 1 / 2 / 3 / 4 / 7 / 8 of them: 8192 x 4096 11.5 / 7.6 / 8.2 / 9.0 / 11.9 / 12.9,
// 16384 x 4096 21 / 12.5 / 14.6 / 9.7 / 12.7 / 13.7, 28672 x 4096 36 / 22 / 21 / 18 / 14.6 / 15.6, 128256 x 4096 153 / 77 / 72 / 67 / 62 / 57).
// Else the tile and the number of parts that cost least; a part has a plane of fp32 sums of its own, written and
// read again by a launch that adds them (2.6 us and 2.8 TB/s; nothing but that where `joined`: the launch that follows adds two of them
// anyway), and is taken for a tenth less (32 rows of 4096 x 14336 33.6 -> 17.1, 1024 x 4096 12.1 -> 8.7; 128 rows of 4096 x 14336
// 38.4 -> 25.1).
inline Plan stream_plan(int n_blocks, int k_tiles, int num_cus) {
  const int g8 = (n_blocks + 7) / 8, g7 = (n_blocks + 6) / 7;
  const bool seven = (g7 + num_cus - 1) / num_cus * 7 < (g8 + num_cus - 1) / num_cus * 8;
  return {-1, g8 <= num_cus ? (n_blocks + num_cus - 1) / num_cus : seven ? 7 : 8, 1, (k_tiles + 3) / 4};
}
inline Plan plan(int n_blocks, int k_tiles, int rows, int num_cus, int most_parts, bool joined = false) {
  const int groups = (k_tiles + 3) / 4, blocks = (rows + 15) / 16;
  Plan best = stream_plan(n_blocks, k_tiles, num_cus);
  if (rows <= 8 || (rows <= kStreamRows && n_blocks > num_cus)) return best;
  double least = rows <= kStreamRows                                      ? 2300 + groups / 8. * (600 + 28 * rows)
                 : rows <= 2 * kStreamRows && n_blocks <= kStreamWide * num_cus ? 2600 + groups / 8. * (150 + 250 * best.fb + 50 * rows)
                                                                              : 1e30;
  for (int t = 0; t < kTileCount4; ++t)
    for (int want = 1; want <= most_parts; want *= 2) {
      const int pg = (groups + want - 1) / want, parts = (groups + pg - 1) / pg;
      if (want > 1 && parts < want) break;           // (no more groups than that)
      const Tile4& q = kTiles4[t];
      const double tiles = (double)((n_blocks + q.bn() - 1) / q.bn()) * ((blocks + q.tb - 1) / q.tb) * parts;
      const double rounds = (double)(((long long)tiles + num_cus - 1) / num_cus), full = tiles / (rounds * num_cus);
      double ns = 2100 + rounds * (q.round_ns + q.k_ns * (1 + 0.01 * q.full * full) * pg * 4);
      if (parts > 1) ns = (ns + (joined && parts == 2 ? 0 : 2600) + parts * (double)rows * n_blocks * 64 / 2840) * 1.1;
      if (ns < least) {
        best = {t, 0, parts, pg};
        least = ns;
      }
    }
  return best;
}

template <bool LOOSE, class Epi>
void launch_stream(const Plan& p, const char* w, int n_blocks, const X& x, const Epi& epi, hipStream_t st) {
  const int units = (x.k_tiles + (x.tail > 0) + 7) / 8;
  const auto go = [&](auto fb) {
    constexpr int FB = decltype(fb)::value;
    const unsigned grid = (n_blocks + FB - 1) / FB, threads = 64 * kStreamWaves;
    if (p.fb != FB) return;
    if constexpr (!LOOSE && FB <= kStreamWide) {
      if (x.last_row >= kStreamRows) return mx4_stream_kernel<FB, 2, false, Epi><<<grid, threads, 0, st>>>(w, x, n_blocks, units, epi);
    }
    mx4_stream_kernel<FB, 1, LOOSE, Epi><<<grid, threads, 0, st>>>(w, x, n_blocks, units, epi);
  };
  [&]<int... FB>(std::integer_sequence<int, FB...>) { (go(std::integral_constant<int, FB + 1>{}), ...); }(std::make_integer_sequence<int, 8>{});
}

// Returns the number of arg-max partials per row (LM head).
template <class Epi>
int launch(const Plan& p, const void* w, int n_blocks, const X& x, int rows, Epi epi, hipStream_t st) {
  const char* wp = (const char*)w;
  if (p.tile >= 0) {
    const int partials = (n_blocks + kTiles4[p.tile].bn() - 1) / kTiles4[p.tile].bn();
    if constexpr (is_logits<Epi>::value) epi.parts = partials;
    launch_tiles4(std::make_integer_sequence<int, kTileCount4>{}, p.tile, wp, x, n_blocks, rows, p.parts, p.part_groups, epi, st);
    return partials;
  }
  if constexpr (is_logits<Epi>::value) epi.parts = n_blocks;
  if constexpr (!std::is_same<Epi, StorePartialEpi>::value) launch_stream<false>(p, wp, n_blocks, x, epi, st);   // (never in parts)
  return n_blocks;
}

// Threads of a plan's product along x.
inline int64_t threads_of(const Plan& p, int n_blocks, int rows) {
  if (p.tile < 0) return ((int64_t)n_blocks + p.fb - 1) / p.fb * 64 * kStreamWaves;
  const Tile4& q = kTiles4[p.tile];
  const int64_t tiles = ((int64_t)n_blocks + q.bn() - 1) / q.bn() * ((rows + 16 * q.tb - 1) / (16 * q.tb)) * p.parts;
  return (tiles + 7) / 8 * 8 * 64 * (q.nw + q.f);
}

inline X tiles_of(const uint16_t* x, int k, const Workspace& ws) { return {x, 0, k / 32, ws.m_rows - 1}; }

}  // namespace mx4
