// Attention over a paged cache with a sliding window and sinks: choice of kernel, and the element-wise kernel for
// layouts that the others cannot take.
#include "hosted.cuh"

namespace approxifer {
namespace {

constexpr int kElementThreads = 128;

// One warp = one (token, query head); a lane holds every 32nd element of q and of the output.  The keys are walked one
// by one with the running maximum and sum of the softmax.  The path for odd head sizes, page sizes and strides: for layouts,
// not for speed (a warp spends some 40 instructions on a key).
__global__ void __launch_bounds__(kElementThreads) attention_element_kernel(const __grid_constant__ approxifer_attention_args a) {
  const int lane = threadIdx.x % 32;
  const int64_t unit = (int64_t)blockIdx.x * (kElementThreads / 32) + threadIdx.x / 32;
  if (unit >= a.T * a.Hq) return;
  const int64_t t = unit / a.Hq;
  const int h = (int)(unit % a.Hq), hk = h / (a.Hq / a.Hkv);
  const int b = sequence_of(a.q_start, a.batch, t);
  const int64_t p = (int64_t)__ldg(a.kv_len + b) - (__ldg(a.q_start + b + 1) - t);  // kv_len - q_len + (t - start)
  const bf16* q = reinterpret_cast<const bf16*>(a.q) + t * a.q_tstride + h * a.q_hstride;
  float qv[8], acc[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) qv[i] = lane + 32 * i < a.D ? widen(q[lane + 32 * i]) * a.scale : 0.f;
  float best = -CUDART_INF_F, total = 0.f;
  const int64_t last = min(p, a.table_pages * a.page_size - 1);
  const int64_t first = a.window ? max((int64_t)0, p - a.window + 1) : 0;
  const int64_t sinks = min((int64_t)a.sinks, first);
  for (int64_t j = sinks > 0 ? 0 : first; j <= last; j = j + 1 == sinks ? first : j + 1) {  // the sinks before the window, then the window
    const int32_t page = __ldg(a.block_table + b * a.table_stride + j / a.page_size);
    if (page < 0 || page >= a.num_pages) continue;
    const bf16* k = reinterpret_cast<const bf16*>(a.k_cache) + page * a.kc_pstride + hk * a.kc_hstride + (j % a.page_size) * a.kc_rstride;
    const bf16* v = reinterpret_cast<const bf16*>(a.v_cache) + page * a.vc_pstride + hk * a.vc_hstride + (j % a.page_size) * a.vc_rstride;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < a.D) s = fmaf(qv[i], widen(k[lane + 32 * i]), s);
    s = warp_sum(s);
    const float top = s == s ? fmaxf(best, s) : s;  // (a NaN score makes the row NaN)
    const float keep = best == -CUDART_INF_F ? 0.f : expf(best - top);
    const float w = s == -CUDART_INF_F ? 0.f : expf(s - top);
    total = total * keep + w;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < a.D) acc[i] = acc[i] * keep + w * widen(v[lane + 32 * i]);
    best = top;
  }
  bf16* out = reinterpret_cast<bf16*>(a.out) + t * a.o_tstride + h * a.o_hstride;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < a.D) out[lane + 32 * i] = narrow<bf16>(total == 0.f ? 0.f : acc[i] / total);
}

}  // namespace

cudaError_t launch_attention(const approxifer_attention_args& a, cudaStream_t stream) {
  if (attention_token_eligible(a)) return launch_attention_token(a, stream);
  if (attention_tile_eligible(a)) return launch_attention_tile(a, stream);
  const int64_t units = a.T * a.Hq, per = kElementThreads / 32;
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  attention_element_kernel<<<(unsigned)blocks, kElementThreads, 0, stream>>>(a);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
