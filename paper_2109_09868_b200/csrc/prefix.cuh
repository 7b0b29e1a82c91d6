// Partial results of attention over a common prefix: what the kernel over the prefix leaves and those over the sequences' own keys
// join.
#pragma once
#include "hosted.cuh"

namespace approxifer {

// The prefix is cut into `parts`; of each, for every row (token, query head), the weighted sum of the values (fp32, the head size
// rounded up to 64 or 128) and the maximum (of the scores in powers of two) and sum of the weights.
struct PrefixParts {
  float* o;    // [most, or one more][rows][64 or 128]
  float2* ml;  // [most, or one more][rows]
  int64_t rows;
  int64_t last_token;          // from this token on (the query blocks from `cut` on of the kernel over the prefix)
  int32_t parts, last_parts;   // so many parts instead
  int32_t most;                // the larger of the two
  int32_t apart;               // the own keys' result is a partial result too, the one after `most`: a kernel of its own joins them
  int32_t cut;
  int32_t split;               // CTAs that share a part, as a cluster
  double time;                 // what the kernel over the prefix is thought to take, in steps
  // (single tokens that walk the prefix themselves) its table, its last position
  const int32_t* table;
  int32_t last;
};

constexpr int kOnTheWay = 2;  // as many partial results the kernels over several tokens' own keys join; more are joined apart

#ifdef __CUDACC__
__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row's partial results: their weights in the joined row, divided by its sum.  Loads go out several parts at a time.
struct PriorRow {
  int parts;
  float top, inv;
  float first[2];  // the maxima of the first two

  __device__ __forceinline__ void load(const PrefixParts& p, int64_t row, int64_t token) {
    constexpr int kAt = 8;
    parts = token >= p.last_token ? p.last_parts : p.parts;
    top = -CUDART_INF_F, inv = 0.f;
    for (int i = 0; i < parts; i += kAt) {
      float2 v[kAt];
#pragma unroll
      for (int e = 0; e < kAt; ++e) v[e] = i + e < parts ? __ldcg(p.ml + (i + e) * p.rows + row) : make_float2(-CUDART_INF_F, 0.f);
      if (i == 0) first[0] = v[0].x, first[1] = v[1].x;
      float most = top;
#pragma unroll
      for (int e = 0; e < kAt; ++e) most = fmaxf(most, v[e].x);
      const float base = most == -CUDART_INF_F ? 0.f : most;
      inv *= power_of_two(top - base);
#pragma unroll
      for (int e = 0; e < kAt; ++e) inv = fmaf(v[e].y, power_of_two(v[e].x - base), inv);
      top = most;
    }
  }
  // Joins the row's own maximum and sum; what its own sums are to be multiplied with.
  __device__ __forceinline__ float weigh(float m, float l) {
    const float most = fmaxf(top, m), base = most == -CUDART_INF_F ? 0.f : most;
    const float sum = inv * power_of_two(top - base) + l * power_of_two(m - base);
    top = base;
    inv = sum == 0.f ? 0.f : 1.f / sum;
    return power_of_two(m - base) * inv;
  }
  // The weight of a part whose maximum is m.
  __device__ __forceinline__ float weight(float m) const { return power_of_two(m - top) * inv; }
  // Adds columns col .. col + N - 1 of the partial results.
  template <int N>
  __device__ __forceinline__ void add(const PrefixParts& p, int64_t row, int width, int col, float (&y)[N]) const {
    constexpr int kWide = N >= 4 ? 4 : 2, kAt = 8;
    static_assert(N % kWide == 0, "whole pairs or fours");
    for (int i = 0; i < parts; i += kAt) {
      float m[kAt], v[kAt][N];
#pragma unroll
      for (int e = 0; e < kAt; ++e) {
        const bool there = i + e < parts;
        const int64_t at = there ? (i + e) * p.rows + row : row;
        m[e] = there ? __ldcg(p.ml + at).x : -CUDART_INF_F;
        const float* from = p.o + at * width + col;
#pragma unroll
        for (int c = 0; c < N; c += kWide) {
          if constexpr (kWide == 4) {
            const float4 u = there ? __ldcg(reinterpret_cast<const float4*>(from + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[e][c] = u.x, v[e][c + 1] = u.y, v[e][c + 2] = u.z, v[e][c + 3] = u.w;
          } else {
            const float2 u = there ? __ldcg(reinterpret_cast<const float2*>(from + c)) : make_float2(0.f, 0.f);
            v[e][c] = u.x, v[e][c + 1] = u.y;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < kAt; ++e) {
        if (i + e >= parts) break;
        const float w = weight(m[e]);
#pragma unroll
        for (int c = 0; c < N; ++c) y[c] = fmaf(w, v[e][c], y[c]);
      }
    }
  }
};
#endif

PrefixParts prefix_parts(const approxifer_prefix_attention_args& a, const DeviceInfo& dev);  // (pointers left out); see attention_tile.cu
cudaError_t launch_attention_over_prefix(const approxifer_prefix_attention_args& a, const PrefixParts& parts, cudaStream_t stream);
bool attention_tile_through_wanted(const approxifer_prefix_attention_args& a, const PrefixParts& parts, int sms);
cudaError_t launch_attention_tile_through(const approxifer_prefix_attention_args& a, cudaStream_t stream);
cudaError_t launch_attention_tile_behind(const approxifer_attention_args& a, const PrefixParts& parts, cudaStream_t stream);
int64_t attention_token_behind_workspace(const approxifer_attention_args& a);
bool attention_token_balanced(const approxifer_attention_args& a);  // ... joins by a kernel of its own in any case
bool attention_token_through_wanted(const approxifer_attention_args& a, int64_t prefix_len);
cudaError_t launch_attention_token_through(const approxifer_attention_args& a, const int32_t* prefix_table, int32_t last, cudaStream_t stream);
cudaError_t launch_attention_token_behind(const approxifer_attention_args& a, const PrefixParts& parts, cudaStream_t stream);

}  // namespace approxifer
