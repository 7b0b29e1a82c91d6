// Shared declarations of the hosted-model operators (linear, per-head norm with rotary positions, attention over a
// paged cache, also behind a common prefix, norms around a block, 4-bit arrays and their products).  The C structs of include/approxifer.h are what the launchers take: they hold device pointers and
// strides, already checked by hosted_api.cu.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "../../include/approxifer.h"
#include "common.cuh"

namespace approxifer {

using bf16 = __nv_bfloat16;

// s with 2^s = v, or -1.
inline int exact_log2(int32_t v) {
  for (int s = 0; s < 31; ++s)
    if ((1 << s) == v) return s;
  return -1;
}

constexpr int kMxRawRows = 32;
// The scales of a product's 4-bit microscaled operands.  Such a product goes through linear_tile.cu as one of rows of K / 4
// 16-bit elements (the same bytes), with these.
struct MxScales {
  const uint8_t *x, *w;  // x NULL: X is bfloat16 and brought into the 4-bit form within the kernel, which takes few rows of it
  int64_t K;  // in 4-bit elements
};
cudaError_t launch_linear(const approxifer_linear_args& a, cudaStream_t stream);
bool linear_tile_eligible(const approxifer_linear_args& a);  // see linear_tile.cu
cudaError_t launch_linear_tile(const approxifer_linear_args& a, const MxScales* mx, cudaStream_t stream);
bool linear_tile_takes_raw(const approxifer_linear_args& a, int sms);
cudaError_t read_linear_tile_wait_timeouts(unsigned int* out);
cudaError_t reset_linear_tile_wait_timeouts();
bool linear_few_wanted(const approxifer_linear_args& a, int sms);  // see linear_few.cu
cudaError_t launch_linear_few(const approxifer_linear_args& a, cudaStream_t stream);
cudaError_t launch_linear_pair(const approxifer_linear_args& a, cudaStream_t stream);  // see linear_pair.cu
cudaError_t read_linear_pair_wait_timeouts(unsigned int* out);
cudaError_t reset_linear_pair_wait_timeouts();
cudaError_t launch_norm_rope(const approxifer_norm_rope_args& a, cudaStream_t stream);
bool attention_token_eligible(const approxifer_attention_args& a);  // see attention_token.cu
int64_t attention_token_workspace(const approxifer_attention_args& a);
cudaError_t launch_attention_token(const approxifer_attention_args& a, cudaStream_t stream);
bool attention_tile_eligible(const approxifer_attention_args& a);  // see attention_tile.cu
cudaError_t launch_attention_tile(const approxifer_attention_args& a, cudaStream_t stream);
cudaError_t read_attention_tile_wait_timeouts(unsigned int* out);
cudaError_t reset_attention_tile_wait_timeouts();
cudaError_t launch_attention(const approxifer_attention_args& a, cudaStream_t stream);
cudaError_t launch_block_norm(const approxifer_block_norm_args& a, cudaStream_t stream);
cudaError_t read_block_norm_wait_timeouts(unsigned int* out);
cudaError_t reset_block_norm_wait_timeouts();
cudaError_t launch_mx_quantize(const approxifer_mx_array_args& a, cudaStream_t stream);
cudaError_t launch_mx_dequantize(const approxifer_mx_array_args& a, cudaStream_t stream);
int64_t mx_linear_workspace(const approxifer_mx_linear_args& a);
cudaError_t launch_mx_linear(const approxifer_mx_linear_args& a, cudaStream_t stream);
cudaError_t launch_mx_pair(const approxifer_mx_linear_args& a, cudaStream_t stream);  // X as codes
cudaError_t read_mx_pair_wait_timeouts(unsigned int* out);
cudaError_t reset_mx_pair_wait_timeouts();
int64_t prefix_attention_workspace(const approxifer_prefix_attention_args& a);
cudaError_t launch_prefix_attention(const approxifer_prefix_attention_args& a, cudaStream_t stream);

#ifdef __CUDACC__
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 narrow<bf16>(float v) { return __float2bfloat16_rn(v); }

// e^x to the accuracy that an output of type Out shows.  __expf errs by some 1.2 |x| units in the last place: 5e-6 relative at
// |x| = 40, which bfloat16 (4e-3) hides and fp32 does not.
template <typename Out>
__device__ __forceinline__ float exponential(float x) {
  if constexpr (sizeof(Out) == 4) return expf(x);
  return __expf(x);
}

// The activations of approxifer_linear, in fp32, for an output of type Out.
template <int ACT, typename Out>
__device__ __forceinline__ float activate(float x) {
  if constexpr (ACT == APPROXIFER_ACT_RELU) return x > 0.f ? x : (x == x ? 0.f : x);  // (a NaN stays one)
  if constexpr (ACT == APPROXIFER_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678f));
  if constexpr (ACT == APPROXIFER_ACT_GELU_TANH) return x / (1.f + exponential<Out>(-1.5957691f * (x + 0.044715f * x * x * x)));  // 0.5 (1 + tanh u) = 1 / (1 + e^-2u)
  if constexpr (ACT == APPROXIFER_ACT_SILU) return x / (1.f + exponential<Out>(-x));
  return x;
}
template <typename Out>
__device__ __forceinline__ float activate(int act, float x) {
  switch (act) {
    case APPROXIFER_ACT_RELU: return activate<APPROXIFER_ACT_RELU, Out>(x);
    case APPROXIFER_ACT_GELU: return activate<APPROXIFER_ACT_GELU, Out>(x);
    case APPROXIFER_ACT_GELU_TANH: return activate<APPROXIFER_ACT_GELU_TANH, Out>(x);
    case APPROXIFER_ACT_SILU: return activate<APPROXIFER_ACT_SILU, Out>(x);
    default: return x;
  }
}

// Two fp32 values in one register pair, and the packed operations on them (each half rounds to nearest).
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// The sequence a packed token belongs to: the last b with q_start[b] <= t (q_start ascending, q_start[0] = 0).
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int batch, int64_t t) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (__ldg(q_start + mid) <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
#endif

}  // namespace approxifer
