// Product by a 4-bit matrix: plain rows.
#include "mx4_gemm.h"

namespace {

template <bool F32>
struct PlainEpi {
  void* out;
  int64_t stride;
  int rows, n;
  bool wide;                // four values of a row can be stored at once
  struct Row {};
  struct Pre {};
  __device__ Row row_info(int) const { return Row{}; }
  __device__ Pre pre(int, int, int, const Row&) const { return Pre{}; }
  __device__ void operator()(int nb, int lane, int row, const f32x4 acc, const Pre&) const {
    const int f = nb * 16 + (lane >> 4) * 4;
    if (row >= rows || f >= n) return;
    const int64_t at = (int64_t)row * stride + f;
    if constexpr (F32) {
      float* p = (float*)out + at;
      if (wide && f + 4 <= n) *(f32x4*)p = acc;
      else
        for (int i = 0; i < 4 && f + i < n; ++i) p[i] = acc[i];
    } else {
      uint16_t* p = (uint16_t*)out + at;
      const mx4::u32x2 w = {pack2_bf16(acc[0], acc[1]), pack2_bf16(acc[2], acc[3])};
      if (wide && f + 4 <= n) *(mx4::u32x2*)p = w;
      else
        for (int i = 0; i < 4 && f + i < n; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
};

// The parts of a split product, first to last.
template <bool F32>
__global__ __launch_bounds__(256) void mx4_join_kernel(const float* __restrict__ parts, int count, size_t plane, int n_pad, int64_t quads, PlainEpi<F32> epi) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= quads) return;
  f32x4 sum = *(const f32x4*)(parts + at * 4);
  for (int p = 1; p < count; ++p) sum += *(const f32x4*)(parts + p * plane + at * 4);
  const int row = (int)(at / (n_pad / 4)), f = (int)(at % (n_pad / 4)) * 4;
  epi(f >> 4, f >> 2 << 4 & 63, row, sum, {});      // (block, and the lane that holds these four features)
}

template <bool F32>
void matmul(const void* w, int n, const mx4::X& x, int rows, const PlainEpi<F32>& epi, const mx4::Plan& p, bool loose, float* parts, hipStream_t st) {
  const int n_blocks = (n + 15) / 16;
  if (loose) {
    mx4::launch_stream<true>(p, (const char*)w, n_blocks, x, epi, st);
    return;
  }
  if (p.parts == 1) {
    mx4::launch(p, w, n_blocks, x, rows, epi, st);
    return;
  }
  const int n_pad = n_blocks * 16;
  const size_t plane = (size_t)((rows + 15) / 16 * 16) * n_pad;
  mx4::launch(p, w, n_blocks, x, rows, gemm::StorePartialEpi{parts, ResidLayout{n_pad, 4}, n_pad, plane}, st);
  const int64_t quads = (int64_t)rows * n_pad / 4;
  mx4_join_kernel<F32><<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(parts, p.parts, plane, n_pad, quads, epi);
}

constexpr int kMostParts = 8;

mx4::Plan matmul_plan(int n, int k, int rows, bool loose, int num_cus, bool parts) {
  const int n_blocks = (n + 15) / 16;
  return loose ? mx4::stream_plan(n_blocks, k / 32, num_cus) : mx4::plan(n_blocks, (k + 31) / 32, rows, num_cus, parts ? kMostParts : 1);
}

}  // namespace

bool mx4_matmul_fits(int n, int k, int rows, bool loose, int num_cus, bool parts) {
  const mx4::Plan p = matmul_plan(n, k, rows, loose, num_cus, parts);
  return mx4::threads_of(p, (n + 15) / 16, rows) <= 0xFFFFFFFFll &&
         (p.parts == 1 || (int64_t)rows * ((n + 15) / 16 * 4) <= (int64_t)kMostGroups256 * 256);
}

size_t mx4_matmul_part_bytes(int n, int k, int rows, int num_cus) {
  const mx4::Plan p = mx4::plan((n + 15) / 16, (k + 31) / 32, rows, num_cus, kMostParts);
  return p.parts > 1 ? 4ull * p.parts * ((rows + 15) / 16 * 16) * ((n + 15) / 16 * 16) : 0;
}

int mx4_loose_rows() { return mx4::kStreamRows; }

void launch_mx4_matmul(const void* w, int n, int k, const uint16_t* x, int64_t x_stride, bool loose, int rows, void* out, int out_type,
                       int64_t out_stride, int num_cus, float* parts, hipStream_t st) {
  const mx4::X xs = loose ? mx4::X{x, x_stride, k / 32, rows - 1, k % 32} : mx4::X{x, x_stride, (k + 31) / 32, rows - 1};
  const mx4::Plan p = matmul_plan(n, k, rows, loose, num_cus, parts != nullptr);
  if (out_type == LLM42_F32)
    matmul(w, n, xs, rows, PlainEpi<true>{out, out_stride, rows, n, (uintptr_t)out % 16 == 0 && out_stride % 4 == 0}, p, loose, parts, st);
  else
    matmul(w, n, xs, rows, PlainEpi<false>{out, out_stride, rows, n, (uintptr_t)out % 8 == 0 && out_stride % 4 == 0}, p, loose, parts, st);
}
