// Matrices to MXFP4 and back, and activations to the tile layout.
#include "mx4.h"

using namespace mx4;

namespace {

constexpr int kLane = 8;   // columns of a k-tile that a lane has

// Where the values of a record come from: 8 consecutive columns of a row as fp32, zeros outside the matrix.
struct PlainBf16 {
  const uint16_t* src;
  int64_t stride;
  int rows, cols;
  bool wide;               // rows are 16-byte aligned
  __device__ void load(int r, int c, float (&v)[8]) const {
    const uint16_t* p = src + (int64_t)r * stride + c;
    if (wide && r < rows && c + 8 <= cols) {
      const u32x4 w = *(const u32x4*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = r < rows && c + i < cols ? bf16_bits_to_f32(p[i]) : 0.f;
    }
  }
};
struct PlainF32 {
  const float* src;
  int64_t stride;
  int rows, cols;
  bool wide;
  __device__ void load(int r, int c, float (&v)[8]) const {
    const float* p = src + (int64_t)r * stride + c;
    if (wide && r < rows && c + 8 <= cols) {
      const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = r < rows && c + i < cols ? p[i] : 0.f;
    }
  }
};
struct Tiles {             // the tile layout of the bf16 GEMMs
  const uint16_t* src;
  int cols;
  __device__ void load(int r, int c, float (&v)[8]) const {
    if (c >= cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
      return;
    }
    const u32x4 w = *(const u32x4*)(src + pk_off(r, c, cols));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};

// A wave makes a record.  A block of 32 columns lies in the four lanes of a row, 8 columns each.
template <class Src>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(Src src, char* __restrict__ dst, int units, size_t records) {
  const size_t rec = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rec >= records) return;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int r = (int)(rec / units) * 16 + (lane & 15), c0 = (int)(rec % units) * kUnit;
  char* out = dst + rec * kRecord;
  u32x4 codes[2];
  uint32_t scales[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v[8];
    src.load(r, c0 + j * 32 + g * kLane, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const uint32_t byte = scale_byte(top);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= code_of(v[i], byte) << (4 * i);
    codes[j >> 2][j & 3] = word;
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
    const int c = c0 + j * 32 + g * kLane;
    const uint32_t byte = scales[j >> 2] >> (8 * (j & 3)) & 255u, word = codes[j >> 2][j & 3];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value_of(word >> (4 * i) & 15u, byte);
    if constexpr (F32) {
      float* p = (float*)dst + (int64_t)r * stride + c;
      if (wide && c + 8 <= cols) {
        *(f32x4*)p = (f32x4){v[0], v[1], v[2], v[3]};
        *(f32x4*)(p + 4) = (f32x4){v[4], v[5], v[6], v[7]};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) p[i] = v[i];
      }
    } else {
      uint16_t* p = (uint16_t*)dst + (int64_t)r * stride + c;   // (the values are bf16s: the upper halves)
      if (wide && c + 8 <= cols) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[2 * i]) >> 16 | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
        *(u32x4*)p = w;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) p[i] = (uint16_t)(__float_as_uint(v[i]) >> 16);
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
  quantize(Tiles{src, cols}, rows, cols, dst, st);
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
