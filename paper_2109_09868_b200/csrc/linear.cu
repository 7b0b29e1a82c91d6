// Matrix product with bias, activation and residual: choice of kernel, and the element-wise kernel for operands that
// the tensor-core kernels cannot take (bases or row strides that are not whole 16 bytes).
#include "hosted.cuh"

namespace approxifer {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

// One CTA = a 64 x 64 tile of Y, a thread 4 x 4 of it; both operands go through shared memory 16 columns at a time as
// fp32.  Bound by the fp32 pipe (a path for odd layouts, not for speed).
template <typename Out>
__global__ void __launch_bounds__(kThreads) linear_element_kernel(const __grid_constant__ approxifer_linear_args a, int64_t tiles_n) {
  __shared__ float xs[kDepth][kTile + 4], ws[kDepth][kTile + 4];
  const int64_t m0 = (blockIdx.x / tiles_n) * kTile, n0 = (blockIdx.x % tiles_n) * kTile;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const bf16* X = reinterpret_cast<const bf16*>(a.X);
  const bf16* Wt = reinterpret_cast<const bf16*>(a.Wt);
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < a.K; k0 += kDepth) {
    for (int e = threadIdx.x; e < kTile * kDepth; e += kThreads) {
      const int row = e / kDepth, col = e % kDepth;
      const bool in_k = k0 + col < a.K;
      xs[col][row] = (in_k && m0 + row < a.M) ? widen(X[(m0 + row) * a.x_rstride + k0 + col]) : 0.f;
      ws[col][row] = (in_k && n0 + row < a.N) ? widen(Wt[(n0 + row) * a.w_rstride + k0 + col]) : 0.f;
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

cudaError_t launch_linear(const approxifer_linear_args& a, cudaStream_t stream) {
  if (linear_tile_eligible(a)) {
    const DeviceInfo* dev;
    const cudaError_t e = current_device_info(&dev);
    if (e != cudaSuccess) return e;
    if (linear_few_wanted(a, dev->sms)) return launch_linear_few(a, stream);
    // 256 x 256 tiles on pairs of CTAs once the 128 x 128 tiles of the other kernel would need a second turn.  Measured, tile
    // against pair kernel, us, 256 x 256 tiles: 32 (2,048 x 1,024 x 4,096) 22.4 / 26.9, 40 (1,024 x 2,560 x 4,096) 43.3 / 28.3,
    // 48 (1,536 x 2,048 x 4,096) 44.2 / 28.6, 256 (4,096^2 x 512) 55 / 25.  (Pairs with 256 x 128 tiles, to leave fewer of them
    // idle in the last turn, reach 70 % of the rate and win nowhere.)
    if (a.M > 128 && a.N > 128 && ((a.M + 127) / 128) * ((a.N + 127) / 128) > dev->sms) return launch_linear_pair(a, stream);
    return launch_linear_tile(a, stream);
  }
  const int64_t tiles_n = (a.N + kTile - 1) / kTile, tiles = tiles_n * ((a.M + kTile - 1) / kTile);
  if (tiles > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  if (a.out_type == APPROXIFER_TYPE_F32)
    linear_element_kernel<float><<<(unsigned)tiles, kThreads, 0, stream>>>(a, tiles_n);
  else
    linear_element_kernel<bf16><<<(unsigned)tiles, kThreads, 0, stream>>>(a, tiles_n);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
