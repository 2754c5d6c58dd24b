// Positions of a block into its record of the 4-bit cache.
#pragma once
#include "mx4.h"

namespace mx4 {

// The larger of two magnitudes, half by half, over the 16 lanes of a group.
__device__ inline uint32_t max_of_16(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) v = larger(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

// Positions lo .. hi - 1 of a block of 16: kt, vt its K and V tiles of the bf16 cache, rec its record.  One wave; it alone writes the record.
template <int HD>
__device__ __forceinline__ void store_positions(const uint16_t* __restrict__ kt, const uint16_t* __restrict__ vt, char* rec, int lo, int hi,
                                                int lane) {
  constexpr int KT = HD / 32;
  const int g = lane >> 4, l16 = lane & 15;
  u32x4 kw[KT], vw[KT];                            // V: features 32 j + 2 p and + 1, four tokens of each
#pragma unroll
  for (int j = 0; j < KT; ++j) kw[j] = vw[j] = (u32x4){0, 0, 0, 0};
  if (l16 >= lo && l16 < hi) {                     // (a single token is 3 KiB of lines so, 8 as a whole tile)
#pragma unroll
    for (int j = 0; j < KT; ++j) kw[j] = *(const u32x4*)(kt + j * 512 + lane * 8);
  }
  if (4 * g + 3 >= lo && 4 * g < hi) {
#pragma unroll
    for (int j = 0; j < KT; ++j) vw[j] = *(const u32x4*)(vt + v_tile_off(32 * j + 2 * l16, 4 * g));
  }
  // tokens of this lane that are in range: a byte of each word of V's codes and scales.  Other positions may share the word (this wave alone
  // writes it): what it holds is asked for with the values.
  uint32_t take = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (4 * g + t >= lo && 4 * g + t < hi) take |= 0xFFu << (8 * t);
  uint32_t* p = (uint32_t*)(rec + 8 * HD + lane * KT * 4);
  uint32_t* q = (uint32_t*)(rec + 16 * HD + HD / 2 + g * KT * 4);
  uint32_t old_c[KT], old_s[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) old_c[j] = old_s[j] = 0;
  if (take && take != 0xFFFFFFFFu) {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      old_c[j] = p[j];
      old_s[j] = q[j];
    }
  }
  // K: lane (g, token) has features 32 j + 8 g .. + 7
  uint32_t kc[KT], ks = 0;
#pragma unroll
  for (int j = 0; j < KT; ++j) {
    uint32_t top = larger_half(larger(larger(kw[j][0], kw[j][1]), larger(kw[j][2], kw[j][3])));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const uint32_t byte = scale_byte(top);
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) word = put_pair(word, kw[j][e], scale_of(byte, 0), e);
    kc[j] = byte == 255u ? 0u : word;
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
  // V: byte i of word j is token 4 g + i
  uint32_t vs[KT], vc[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) {
    const uint32_t pair[2] = {max_of_16(larger(vw[j][0], vw[j][2])), max_of_16(larger(vw[j][1], vw[j][3]))};   // tokens 0, 1 and 2, 3
    vs[j] = vc[j] = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t byte = scale_byte(t & 1 ? pair[t >> 1] & 0xFFFF0000u : pair[t >> 1] << 16);
      const uint32_t two = t & 1 ? vw[j][t >> 1] >> 16 | (vw[j][2 + (t >> 1)] & 0xFFFF0000u) : (vw[j][t >> 1] & 0xFFFFu) | vw[j][2 + (t >> 1)] << 16;
      vs[j] |= byte << (8 * t);
      vc[j] = put_pair(vc[j], two, scale_of(byte, 0), t);
      if (byte == 255u) vc[j] &= ~(255u << (8 * t));
    }
  }
  if (take) {
#pragma unroll
    for (int j = 0; j < KT; ++j) p[j] = (old_c[j] & ~take) | (vc[j] & take);
    if (l16 == 0) {
#pragma unroll
      for (int j = 0; j < KT; ++j) q[j] = (old_s[j] & ~take) | (vs[j] & take);
    }
  }
}

}  // namespace mx4
