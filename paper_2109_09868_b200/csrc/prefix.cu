// Attention of a batch behind a common prefix: choice of kernels, and the element-wise kernel for layouts that the others cannot
// take.
#include "prefix.cuh"

namespace approxifer {
namespace {

constexpr int kElementThreads = 128;

// One warp = one (token, query head); a lane holds every 32nd element of q and of the output.  The keys, the prefix's and then the
// sequence's own, are walked one by one with the running maximum and sum of the softmax.  The path for odd head sizes, page sizes
// and strides: for layouts, not for speed.
__global__ void __launch_bounds__(kElementThreads) prefix_element_kernel(const __grid_constant__ approxifer_prefix_attention_args g) {
  const approxifer_attention_args& a = g.own;
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
  auto walk = [&](const int32_t* table, int64_t keys) {
    for (int64_t j = 0; j < keys; ++j) {
      const int32_t page = __ldg(table + j / a.page_size);
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
  };
  if (p >= 0) {
    walk(g.prefix_table, min(g.prefix_len, g.prefix_pages * a.page_size));
    walk(a.block_table + b * a.table_stride, min(p + 1, a.table_pages * a.page_size));
  }
  bf16* out = reinterpret_cast<bf16*>(a.out) + t * a.o_tstride + h * a.o_hstride;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < a.D) out[lane + 32 * i] = narrow<bf16>(total == 0.f ? 0.f : acc[i] / total);
}

}  // namespace

namespace {
// Whether the call runs on the tensor cores: what the kernel over the prefix takes, the ones over the own keys take too.
bool on_tensor_cores(const approxifer_prefix_attention_args& p) {
  approxifer_attention_args a = p.own;
  if (!attention_tile_eligible(a)) return false;
  a.table_pages = p.prefix_pages;
  return attention_tile_eligible(a);
}
int64_t parts_bytes(const PrefixParts& p, const approxifer_attention_args& a) { return p.most * p.rows * ((a.D <= 64 ? 64 : 128) + 2) * (int64_t)sizeof(float); }
bool has_prefix(const approxifer_prefix_attention_args& p) { return p.prefix_len > 0 && p.prefix_pages > 0; }
}  // namespace

int64_t prefix_attention_workspace(const approxifer_prefix_attention_args& p) {
  const DeviceInfo* dev;
  if (!on_tensor_cores(p) || current_device_info(&dev) != cudaSuccess) return 0;
  const bool behind = has_prefix(p), token = attention_token_eligible(p.own);
  int64_t bytes = !token ? 0 : behind ? attention_token_behind_workspace(p.own) : attention_token_workspace(p.own);
  if (behind) bytes += (parts_bytes(prefix_parts(p, *dev), p.own) + 15) / 16 * 16;
  return bytes;
}

cudaError_t launch_prefix_attention(const approxifer_prefix_attention_args& p, cudaStream_t stream) {
  if (on_tensor_cores(p)) {
    if (!has_prefix(p)) return launch_attention(p.own, stream);
    const DeviceInfo* dev;
    cudaError_t e = current_device_info(&dev);
    if (e != cudaSuccess) return e;
    PrefixParts parts = prefix_parts(p, *dev);
    approxifer_attention_args own = p.own;
    parts.o = static_cast<float*>(own.workspace);
    parts.ml = reinterpret_cast<float2*>(parts.o + parts.most * parts.rows * (own.D <= 64 ? 64 : 128));
    const int64_t used = (parts_bytes(parts, own) + 15) / 16 * 16;
    own.workspace = static_cast<char*>(own.workspace) + used, own.workspace_bytes -= used;
    if ((e = launch_attention_over_prefix(p, parts, stream)) != cudaSuccess) return e;
    return attention_token_eligible(own) ? launch_attention_token_behind(own, parts, stream) : launch_attention_tile_behind(own, parts, stream);
  }
  const int64_t units = p.own.T * p.own.Hq, per = kElementThreads / 32;
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  prefix_element_kernel<<<(unsigned)blocks, kElementThreads, 0, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
