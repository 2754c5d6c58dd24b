// Matrices to MXFP4 and back, and activations to the tile layout.
#include "mx4.h"

using namespace mx4;

namespace {

// Where the values of a record come from: 8 consecutive columns of a row, zeros outside the matrix, as words of two bf16 (or 8 floats), and
// the bits of the largest magnitude.  wide: rows are 16-byte aligned and the record lies within the columns; rows past the last
// one are then read from it.
struct PlainBf16 {
  const uint16_t* src;
  int64_t stride;
  int rows, cols;
  bool aligned;
  struct V {
    u32x4 w;
    __device__ uint32_t top() const { return larger_half(larger(larger(w[0], w[1]), larger(w[2], w[3]))); }
    __device__ uint32_t codes(float scale) const {
      uint32_t word = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) word = put_pair(word, w[e], scale, e);
      return word;
    }
  };
  __device__ V wide(int r, int c) const { return {*(const u32x4*)(src + (int64_t)min(r, rows - 1) * stride + c)}; }
  __device__ V any(int r, int c) const {
    V v{{0, 0, 0, 0}};
    const uint16_t* p = src + (int64_t)r * stride + c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r < rows && c + i < cols) v.w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
  }
};
struct PlainF32 {
  const float* src;
  int64_t stride;
  int rows, cols;
  bool aligned;
  struct V {
    f32x4 a, b;
    __device__ uint32_t top() const {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) t = max(t, max(__float_as_uint(a[i]) & 0x7FFFFFFFu, __float_as_uint(b[i]) & 0x7FFFFFFFu));
      return t;
    }
    __device__ uint32_t codes(float scale) const {
      uint32_t word = put_pair(0, a[0], a[1], scale, 0);
      word = put_pair(word, a[2], a[3], scale, 1);
      word = put_pair(word, b[0], b[1], scale, 2);
      return put_pair(word, b[2], b[3], scale, 3);
    }
  };
  __device__ V wide(int r, int c) const {
    const float* p = src + (int64_t)min(r, rows - 1) * stride + c;
    return {*(const f32x4*)p, *(const f32x4*)(p + 4)};
  }
  __device__ V any(int r, int c) const {
    V v{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    const float* p = src + (int64_t)r * stride + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (r < rows && c + i < cols) v.a[i] = p[i];
      if (r < rows && c + 4 + i < cols) v.b[i] = p[4 + i];
    }
    return v;
  }
};
struct Tiles {             // the tile layout of the bf16 GEMMs (whole blocks of rows and columns)
  const uint16_t* src;
  int rows, cols;
  static constexpr bool aligned = true;
  typedef PlainBf16::V V;
  __device__ V wide(int r, int c) const { return {*(const u32x4*)(src + pk_off(r, c, cols))}; }
  __device__ V any(int r, int c) const { return c < cols ? wide(r, c) : V{{0, 0, 0, 0}}; }
};

// A wave makes a record.  A block of 32 columns lies in the four lanes of a row, 8 columns each: its maximum takes two exchanges, and every
// lane stores what it converted.  Bound by memory: 28672 x 4096 bf16 there and back 124 us, 4.8 TB/s, what a large copy reaches.
template <class Src>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(Src src, char* __restrict__ dst, int units, size_t records) {
  const size_t rec = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rec >= records) return;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int r = (int)(rec / units) * 16 + (lane & 15), c0 = (int)(rec % units) * kUnit;
  char* out = dst + rec * kRecord;
  typename Src::V v[8];
  if (src.aligned && c0 + kUnit <= src.cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = src.wide(r, c0 + j * 32 + g * 8);
    if (r >= src.rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = {};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = src.any(r, c0 + j * 32 + g * 8);
  }
  u32x4 codes[2];
  uint32_t scales[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t top = v[j].top();
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const uint32_t byte = scale_byte(top), word = v[j].codes(scale_of(byte, 0));
    codes[j >> 2][j & 3] = byte == 255u ? 0u : word;
    scales[j >> 2] |= byte << (8 * (j & 3));
  }
  *(u32x4*)(out + lane * 16) = codes[0];
  *(u32x4*)(out + 1024 + lane * 16) = codes[1];
  if (g == 0) *(u32x2*)(out + kScales + lane * 8) = (u32x2){scales[0], scales[1]};
}

template <bool F32>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const char* __restrict__ src, void* __restrict__ dst, int64_t stride, int rows,
                                                             int cols, bool wide, int units, size_t records) {
  const size_t rec = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rec >= records) return;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int r = (int)(rec / units) * 16 + (lane & 15), c0 = (int)(rec % units) * kUnit;
  if (r >= rows) return;
  const char* in = src + rec * kRecord;
  const u32x4 codes[2] = {*(const u32x4*)(in + lane * 16), *(const u32x4*)(in + 1024 + lane * 16)};
  const u32x2 scales = *(const u32x2*)(in + kScales + (lane & 15) * 8);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = c0 + j * 32 + g * 8;
    const uint32_t word = codes[j >> 2][j & 3];
    const float scale = scale_of(scales[j >> 2], j & 3);
    if constexpr (F32) {
      float* p = (float*)dst + (int64_t)r * stride + c;
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x2 two = pair_f32(word, scale, e);
        v[2 * e] = two.x;
        v[2 * e + 1] = two.y;
      }
      if (wide && c + 8 <= cols) {
        *(f32x4*)p = (f32x4){v[0], v[1], v[2], v[3]};
        *(f32x4*)(p + 4) = (f32x4){v[4], v[5], v[6], v[7]};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) p[i] = v[i];
      }
    } else {
      uint16_t* p = (uint16_t*)dst + (int64_t)r * stride + c;
      const u32x4 w = __builtin_bit_cast(u32x4, operand(word, scale));
      if (wide && c + 8 <= cols) *(u32x4*)p = w;
      else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}

__global__ __launch_bounds__(256) void mx4_pack_x_kernel(const uint16_t* __restrict__ x, int64_t stride, int rows, int k,
                                                         uint4* __restrict__ dst, int k_tiles, size_t groups) {
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= groups) return;
  const int lane = (int)(at & 63), kt = (int)((at >> 6) % k_tiles);
  const int r = (int)((at >> 6) / k_tiles) * 16 + (lane & 15), c = kt * 32 + (lane >> 4) * 8;
  uint32_t w[4] = {0, 0, 0, 0};
  const uint16_t* p = x + (int64_t)r * stride + c;
  if (r < rows)
    for (int i = 0; i < 8; ++i)
      if (c + i < k) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
  dst[at] = make_uint4(w[0], w[1], w[2], w[3]);
}

template <class Src>
void quantize(const Src& src, int rows, int cols, void* dst, hipStream_t st) {
  const size_t records = matrix_bytes(rows, cols) / kRecord;
  mx4_quantize_kernel<<<(unsigned)((records + 3) / 4), 256, 0, st>>>(src, (char*)dst, units_of(cols), records);
}

}  // namespace

void launch_mx4_quantize(const void* src, int type, int64_t stride, int rows, int cols, void* dst, hipStream_t st) {
  const bool wide = (uintptr_t)src % 16 == 0 && stride % (type == LLM42_F32 ? 4 : 8) == 0;
  if (type == LLM42_F32) quantize(PlainF32{(const float*)src, stride, rows, cols, wide}, rows, cols, dst, st);
  else quantize(PlainBf16{(const uint16_t*)src, stride, rows, cols, wide}, rows, cols, dst, st);
}

void launch_mx4_quantize_tiles(const uint16_t* src, int rows, int cols, void* dst, hipStream_t st) {
  quantize(Tiles{src, rows, cols}, rows, cols, dst, st);
}

void launch_mx4_dequantize(const void* src, int rows, int cols, void* dst, int type, int64_t stride, hipStream_t st) {
  const size_t records = matrix_bytes(rows, cols) / kRecord;
  const bool wide = (uintptr_t)dst % 16 == 0 && stride % (type == LLM42_F32 ? 4 : 8) == 0;
  const unsigned grid = (unsigned)((records + 3) / 4);
  if (type == LLM42_F32) mx4_dequantize_kernel<true><<<grid, 256, 0, st>>>((const char*)src, dst, stride, rows, cols, wide, units_of(cols), records);
  else mx4_dequantize_kernel<false><<<grid, 256, 0, st>>>((const char*)src, dst, stride, rows, cols, wide, units_of(cols), records);
}

void launch_mx4_pack_x(const uint16_t* x, int64_t stride, int rows, int k, uint16_t* dst, hipStream_t st) {
  const int k_tiles = (k + 31) / 32;
  const size_t groups = (size_t)((rows + 15) / 16) * k_tiles * 64;
  mx4_pack_x_kernel<<<(unsigned)((groups + 255) / 256), 256, 0, st>>>(x, stride, rows, k, (uint4*)dst, k_tiles, groups);
}
