// Product of 4-bit microscaled operands with bias, activation and residual.
#include "mx.cuh"

namespace approxifer {
namespace {

constexpr int kTile = 64, kDepth = 32, kThreads = 256;

__device__ __forceinline__ float mx_element(const uint8_t* codes, int64_t rstride, const uint8_t* scales, int64_t cols, int64_t row, int64_t k) {
  const float table[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  const uint32_t pair = codes[row * rstride + k / 2], code = k & 1 ? pair >> 4 : pair & 15;
  const uint32_t byte = scales[((row / kMxRows) * cols + k / kMxCols) * kMxBlock + (row % 32) * 16 + (row / 32 % 4) * 4 + k / kMxGroup % 4];
  return (code & 8 ? -table[code & 7] : table[code & 7]) * mx_value(byte);
}

// One CTA = a 64 x 64 tile of Y, a thread 4 x 4 of it; both operands go through shared memory 32 columns at a time as fp32.
template <typename Out>
__global__ void __launch_bounds__(kThreads) mx_linear_element_kernel(const __grid_constant__ approxifer_mx_linear_args a, int64_t tiles_n) {
  __shared__ float xs[kDepth][kTile + 4], ws[kDepth][kTile + 4];
  const int64_t m0 = (blockIdx.x / tiles_n) * kTile, n0 = (blockIdx.x % tiles_n) * kTile, cols = (a.K + kMxCols - 1) / kMxCols;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < a.K; k0 += kDepth) {
    for (int e = threadIdx.x; e < kTile * kDepth; e += kThreads) {
      const int row = e / kDepth, col = e % kDepth;
      xs[col][row] = m0 + row < a.M ? mx_element(static_cast<const uint8_t*>(a.X), a.x_rstride, a.x_scales, cols, m0 + row, k0 + col) : 0.f;
      ws[col][row] = n0 + row < a.N ? mx_element(a.Wt, a.w_rstride, a.w_scales, cols, n0 + row, k0 + col) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      float x[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = xs[k][ty * 4 + i], w[i] = ws[k][tx * 4 + i];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], w[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= a.M || n >= a.N) continue;
      float y = acc[i][j];
      if (a.bias) y += widen(reinterpret_cast<const bf16*>(a.bias)[n]);
      y = activate<Out>(a.activation, y);
      if (a.R) y += widen(static_cast<const Out*>(a.R)[m * a.r_rstride + n]);
      static_cast<Out*>(a.Y)[m * a.y_rstride + n] = narrow<Out>(y);
    }
}

}  // namespace

int64_t mx_linear_workspace(const approxifer_mx_linear_args& a) {
  return a.x_scales || a.M == 0 ? 0 : a.M * (a.K / 2) + mx_blocks(a.M, a.K) * kMxBlock;
}

cudaError_t launch_mx_linear(const approxifer_mx_linear_args& given, cudaStream_t stream) {
  approxifer_mx_linear_args a = given;
  if (a.x_scales == nullptr) {
    approxifer_mx_array_args q{a.M, a.K, APPROXIFER_TYPE_BF16, 0, const_cast<void*>(a.X), a.x_rstride, static_cast<uint8_t*>(a.workspace), a.K / 2, nullptr};
    q.scales = q.codes + a.M * (a.K / 2);
    const cudaError_t e = launch_mx_quantize(q, stream);
    if (e != cudaSuccess) return e;
    a.X = q.codes, a.x_rstride = q.c_rstride, a.x_scales = q.scales;
  }
  const int64_t tiles_n = (a.N + kTile - 1) / kTile, tiles = tiles_n * ((a.M + kTile - 1) / kTile);
  if (tiles > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  if (a.out_type == APPROXIFER_TYPE_F32)
    mx_linear_element_kernel<float><<<(unsigned)tiles, kThreads, 0, stream>>>(a, tiles_n);
  else
    mx_linear_element_kernel<bf16><<<(unsigned)tiles, kThreads, 0, stream>>>(a, tiles_n);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
