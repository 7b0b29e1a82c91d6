// Partial results of attention over a common prefix: what the kernel over the prefix leaves and those over the sequences' own keys
// join.
#pragma once
#include "hosted.cuh"

namespace approxifer {

// The prefix is cut into `parts`; of each, for every row (token, query head), the weighted sum of the values (fp32, the head size
// rounded up to 64 or 128) and the maximum (of the scores in powers of two) and sum of the weights.
struct PrefixParts {
  float* o;    // [parts][rows][64 or 128]
  float2* ml;  // [parts][rows]
  int64_t rows;
  int64_t last_token;          // from this token on (the last query block of the kernel over the prefix)
  int32_t parts, last_parts;   // so many parts instead
};

#ifdef __CUDACC__
// A row's partial results: their weights in the joined row, divided by its sum.
struct PriorRow {
  int parts;
  float top, inv;

  __device__ __forceinline__ void load(const PrefixParts& p, int64_t row, int64_t token) {
    parts = token >= p.last_token ? p.last_parts : p.parts;
    top = -CUDART_INF_F, inv = 0.f;
    for (int i = 0; i < parts; ++i) {
      const float2 v = __ldcg(p.ml + i * p.rows + row);
      if (v.x > top) inv *= pow2_of(top - v.x), top = v.x;
      inv += v.y * pow2_of(v.x - (top == -CUDART_INF_F ? 0.f : top));
    }
  }
  // Joins the row's own maximum and sum; what its own sums are to be multiplied with.
  __device__ __forceinline__ float weigh(float m, float l) {
    const float most = fmaxf(top, m), base = most == -CUDART_INF_F ? 0.f : most;
    const float sum = inv * pow2_of(top - base) + l * pow2_of(m - base);
    top = base;
    inv = sum == 0.f ? 0.f : 1.f / sum;
    return pow2_of(m - base) * inv;
  }
  // Adds columns col .. col + N - 1 of the partial results.
  template <int N>
  __device__ __forceinline__ void add(const PrefixParts& p, int64_t row, int width, int col, float (&y)[N]) const {
    constexpr int kWide = N >= 4 ? 4 : N;
    for (int i = 0; i < parts; ++i) {
      const float w = pow2_of(__ldcg(p.ml + i * p.rows + row).x - top) * inv;
      const float* from = p.o + (i * p.rows + row) * width + col;
#pragma unroll
      for (int c = 0; c < N; c += kWide) {
        if constexpr (kWide == 4) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(from + c));
          y[c] = fmaf(w, v.x, y[c]), y[c + 1] = fmaf(w, v.y, y[c + 1]), y[c + 2] = fmaf(w, v.z, y[c + 2]), y[c + 3] = fmaf(w, v.w, y[c + 3]);
        } else if constexpr (kWide == 1) {
          y[c] = fmaf(w, __ldcg(from + c), y[c]);
        } else {
          const float2 v = __ldcg(reinterpret_cast<const float2*>(from + c));
          y[c] = fmaf(w, v.x, y[c]), y[c + 1] = fmaf(w, v.y, y[c + 1]);
        }
      }
    }
  }
  static __device__ __forceinline__ float pow2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
  }
};
#endif

PrefixParts prefix_parts(const approxifer_prefix_attention_args& a, const DeviceInfo& dev);  // (pointers left out); see attention_tile.cu
cudaError_t launch_attention_over_prefix(const approxifer_prefix_attention_args& a, const PrefixParts& parts, cudaStream_t stream);
cudaError_t launch_attention_tile_behind(const approxifer_attention_args& a, const PrefixParts& parts, cudaStream_t stream);
cudaError_t launch_attention_token_behind(const approxifer_attention_args& a, const PrefixParts& parts, cudaStream_t stream);

}  // namespace approxifer
