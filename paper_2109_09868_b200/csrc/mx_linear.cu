// Product of 4-bit microscaled operands with bias, activation and residual: choice of kernel.  Both operands go to the tensor cores
// as they are held (two to a byte, scales beside them), which form the products of the values that the codes and scales stand for;
// their sums are fp32.  X in bfloat16 is brought into that form within the product where it has few rows, else by a launch of its
// own into the workspace (8,192 x 4,096 18 us).
#include "mx.cuh"

namespace approxifer {
namespace {

// The product as linear_tile.cu takes it: rows of K / 4 16-bit elements, the same bytes; X as codes unless `raw`.
approxifer_linear_args as_words(const approxifer_mx_linear_args& a, bool raw) {
  approxifer_linear_args b{};
  b.M = a.M, b.N = a.N, b.K = a.K / 4;
  b.X = static_cast<const uint16_t*>(a.X), b.x_rstride = raw ? a.x_rstride : a.x_rstride / 2;
  b.Wt = reinterpret_cast<const uint16_t*>(a.Wt), b.w_rstride = a.w_rstride / 2;
  b.bias = a.bias, b.R = a.R, b.r_rstride = a.r_rstride, b.Y = a.Y, b.y_rstride = a.y_rstride, b.activation = a.activation, b.out_type = a.out_type;
  return b;
}

bool takes_raw(const approxifer_mx_linear_args& a) {
  const DeviceInfo* dev;
  return a.x_scales == nullptr && a.M <= kMxRawRows && current_device_info(&dev) == cudaSuccess && linear_tile_takes_raw(as_words(a, true), dev->sms);
}

}  // namespace

int64_t mx_linear_workspace(const approxifer_mx_linear_args& a) {
  return a.x_scales || a.M == 0 || takes_raw(a) ? 0 : a.M * (a.K / 2) + mx_blocks(a.M, a.K) * kMxBlock;
}

cudaError_t launch_mx_linear(const approxifer_mx_linear_args& given, cudaStream_t stream) {
  approxifer_mx_linear_args a = given;
  const bool raw = takes_raw(a);
  if (a.x_scales == nullptr && !raw) {
    approxifer_mx_array_args q{a.M, a.K, APPROXIFER_TYPE_BF16, 0, const_cast<void*>(a.X), a.x_rstride, static_cast<uint8_t*>(a.workspace), a.K / 2, nullptr};
    q.scales = q.codes + a.M * (a.K / 2);
    const cudaError_t e = launch_mx_quantize(q, stream);
    if (e != cudaSuccess) return e;
    a.X = q.codes, a.x_rstride = q.c_rstride, a.x_scales = q.scales;
  }
  const DeviceInfo* dev;
  const cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  // As for bfloat16: pairs of CTAs once the tiles of one CTA would need a second turn.
  if (a.M > 128 && a.N > 128 && ((a.M + 127) / 128) * ((a.N + 127) / 128) > dev->sms) return launch_mx_pair(a, stream);
  const MxScales scales{a.x_scales, a.w_scales, a.K};
  return launch_linear_tile(as_words(a, raw), &scales, stream);
}

}  // namespace approxifer
