// Per-head norm of queries and keys with the position rotation, keys and values written to the paged cache.
#include "hosted.cuh"

namespace approxifer {
namespace {

constexpr int kElementThreads = 128;

// One warp = one (token, head) of q, k or v; a lane holds every 32nd element.  The path for head sizes, strides and
// rotations that do not split into whole 16-byte columns.
template <typename T>
__global__ void __launch_bounds__(kElementThreads) norm_rope_element_kernel(const __grid_constant__ approxifer_norm_rope_args a) {
  __shared__ float rows[kElementThreads / 32][256];
  float* row = rows[threadIdx.x / 32];
  const int lane = threadIdx.x % 32;
  const int heads = a.Hq + 2 * a.Hkv;
  const int64_t unit = (int64_t)blockIdx.x * (kElementThreads / 32) + threadIdx.x / 32;
  if (unit >= a.T * heads) return;
  const int64_t t = unit / heads;
  int h = (int)(unit % heads);
  const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
  const bool first = h == 0;
  const int64_t pos = a.rot ? __ldg(a.positions + t) : 0;
  const bool placed = a.rot == 0 || (pos >= 0 && pos < a.positions_max);
  const int64_t slot = a.slots ? __ldg(a.slots + t) : -1;
  const bool fits = slot < a.num_pages * a.page_size;
  if (first && lane == 0 && a.status) a.status[t] = (placed ? 0u : APPROXIFER_ST_POSITION) | (fits ? 0u : APPROXIFER_ST_SLOT);

  const T* in;
  T* out;
  const T* weight = nullptr;
  if (is_q) {
    in = static_cast<const T*>(a.q) + t * a.q_tstride + h * a.q_hstride;
    out = static_cast<T*>(a.q_out) + t * a.qo_tstride + h * a.qo_hstride;
    weight = static_cast<const T*>(a.q_weight);
  } else {
    if (!placed || !fits || slot < 0) return;
    const int64_t page = slot / a.page_size, at = slot % a.page_size;
    h -= is_k ? a.Hq : a.Hq + a.Hkv;
    if (is_k) {
      if (!a.k) return;
      in = static_cast<const T*>(a.k) + t * a.k_tstride + h * a.k_hstride;
      out = static_cast<T*>(a.k_cache) + page * a.kc_pstride + h * a.kc_hstride + at * a.kc_rstride;
      weight = static_cast<const T*>(a.k_weight);
    } else {
      if (!a.v) return;
      in = static_cast<const T*>(a.v) + t * a.v_tstride + h * a.v_hstride;
      out = static_cast<T*>(a.v_cache) + page * a.vc_pstride + h * a.vc_hstride + at * a.vc_rstride;
      for (int d = lane; d < a.D; d += 32) out[d] = in[d];
      return;
    }
  }
  float sq = 0.f;
  for (int d = lane; d < a.D; d += 32) {
    const float x = placed ? widen(in[d]) : 0.f;
    row[d] = x;
    sq = fmaf(x, x, sq);
  }
  sq = warp_sum(sq);
  const float r = weight ? rsqrtf(sq / (float)a.D + a.eps) : 1.f;
  for (int d = lane; d < a.D; d += 32) row[d] = weight ? row[d] * r * widen(weight[d]) : row[d];
  __syncwarp();
  const int half = a.rot / 2;
  for (int d = lane; d < a.D; d += 32) {
    float y = row[d];
    if (d < a.rot && placed) {
      const int i = a.interleaved ? d / 2 : d % half;
      const bool second = a.interleaved ? (d & 1) : d >= half;
      const float c = a.cos_sin[pos * a.rot + i], s = a.cos_sin[pos * a.rot + half + i];
      const float other = row[a.interleaved ? (d ^ 1) : (second ? d - half : d + half)];
      y = second ? fmaf(y, c, other * s) : fmaf(y, c, -other * s);
    }
    out[d] = narrow<T>(y);
  }
}

}  // namespace

cudaError_t launch_norm_rope(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  const int64_t units = a.T * (a.Hq + 2 * a.Hkv), per = kElementThreads / 32;
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  if (a.type == APPROXIFER_TYPE_F32)
    norm_rope_element_kernel<float><<<(unsigned)blocks, kElementThreads, 0, stream>>>(a);
  else
    norm_rope_element_kernel<bf16><<<(unsigned)blocks, kElementThreads, 0, stream>>>(a);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
