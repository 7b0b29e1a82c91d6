// Attention of a batch behind a common prefix: choice of kernels, the kernel that joins many partial results, and the element-wise
// kernel for layouts that the others cannot take.
//
// The softmax over prefix and own keys is taken apart: of each part its maximum m, the sum l of its weights 2^(s - m) and the weighted
// sum o of its values; joined, out = sum 2^(m_i - m) o_i / sum 2^(m_i - m) l_i.  The kernel over the prefix (attention_tile.cu) has the
// tokens of all sequences side by side as the rows of its tiles, so that the prefix's keys and values are read once for them, and cuts
// the prefix so that its CTAs fill the GPU; the kernels over the own keys (attention_token.cu for single tokens, attention_tile.cu) start
// while its last CTAs run and need what it left only at their end.  A short prefix, or one of few sequences, each sequence walks itself;
// so do single tokens in layouts that the kernel over the prefix does not take.
//
// Measured: 96 single tokens behind 32,768, 32 heads on 8 of 128, up to 700 own keys, 112 to 119 us (under a profiler the prefix 69, own
// keys 41, joining 13); eight prompts of 100 to 300 tokens behind 4,096 139 to 145 us; five single tokens
// behind 1,003, heads of 64, 7.1 to 8.6 us.
#include "async.cuh"
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
  const int end = __ldg(a.q_start + b + 1);
  if (t >= end) return;  // (behind the last sequence: left as it is)
  const int64_t p = (int64_t)__ldg(a.kv_len + b) - (end - t);  // kv_len - q_len + (t - start)
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

// Joins the partial results of the prefix and of the own keys, a CTA to a row (token, query head): teams of DP / 4 lanes take them
// in turn, kAhead loads in flight, and meet in shared memory, in order.
template <int DP>
__global__ void __launch_bounds__(128) prefix_join_kernel(const __grid_constant__ approxifer_attention_args a, const __grid_constant__ PrefixParts prior) {
  constexpr int kLanes = DP / 4, kTeams = 128 / kLanes, kAhead = 6;
  __shared__ __align__(16) float sy[kTeams][DP];
  __shared__ float sm[kTeams], sl[kTeams];
  let_next_start();
  const int64_t row = blockIdx.x, t = row / a.Hq;
  const int h = (int)(row % a.Hq), team = threadIdx.x / kLanes, at4 = (threadIdx.x % kLanes) * 4;
  // (the call's inputs are there: the kernel before this one has started, and so has the one before that waited for them)
  const int b = sequence_of(a.q_start, a.batch, t), end = __ldg(a.q_start + b + 1);
  const int64_t p = (int64_t)__ldg(a.kv_len + b) - (end - t);
  wait_for_inputs();
  if (t >= end) return;  // (behind the last sequence: left as it is)
  bf16* out = reinterpret_cast<bf16*>(a.out) + t * a.o_tstride + h * a.o_hstride;
  if (p < 0) {
    for (int d = threadIdx.x; d < a.D; d += 128) out[d] = narrow<bf16>(0.f);
    return;
  }
  const int parts = t >= prior.last_token ? prior.last_parts : prior.parts;
  float m = -CUDART_INF_F, l = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = team; i0 <= parts; i0 += kAhead * kTeams) {
    float2 ml[kAhead];
    float4 v[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int i = i0 + e * kTeams;
      ml[e] = make_float2(-CUDART_INF_F, 0.f), v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i <= parts) {
        const int64_t from = (i < parts ? i : prior.most) * prior.rows + row;
        ml[e] = __ldcg(prior.ml + from);
        v[e] = __ldcg(reinterpret_cast<const float4*>(prior.o + from * DP + at4));
      }
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) top = fmaxf(top, ml[e].x);
    const float base = top == -CUDART_INF_F ? 0.f : top, keep = power_of_two(m - base);
    l *= keep, y.x *= keep, y.y *= keep, y.z *= keep, y.w *= keep;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const float k = power_of_two(ml[e].x - base);
      l = fmaf(k, ml[e].y, l);
      y.x = fmaf(k, v[e].x, y.x), y.y = fmaf(k, v[e].y, y.y), y.z = fmaf(k, v[e].z, y.z), y.w = fmaf(k, v[e].w, y.w);
    }
    m = top;
  }
  if (at4 == 0) sm[team] = m, sl[team] = l;
  *reinterpret_cast<float4*>(&sy[team][at4]) = y;
  __syncthreads();
  float best = sm[0];
#pragma unroll
  for (int i = 1; i < kTeams; ++i) best = fmaxf(best, sm[i]);
  if (best == -CUDART_INF_F) best = 0.f;
  for (int d = threadIdx.x; d < a.D; d += 128) {
    float sum = 0.f, z = 0.f;
#pragma unroll
    for (int i = 0; i < kTeams; ++i) {
      const float k = power_of_two(sm[i] - best);
      sum = fmaf(k, sl[i], sum), z = fmaf(k, sy[i][d], z);
    }
    out[d] = narrow<bf16>(sum == 0.f ? 0.f : z / sum);
  }
}

// Whether the kernel over the prefix takes the call: the ones over the own keys then take it too.  (Of single tokens attention_token.cu
// takes more: pages of any size, queries and outputs at 4 bytes, any number of query heads to a key head.  Those walk the prefix each for
// itself: 16 behind 4,096 in pages of 24, 32 heads on 8 of 128, 65 us, where the element-wise kernel takes 3.9 ms.)
bool tiles_take(const approxifer_prefix_attention_args& p) {
  approxifer_attention_args a = p.own;
  if (!attention_tile_eligible(a)) return false;
  a.table_pages = p.prefix_pages;
  return attention_tile_eligible(a);
}
// Positions of the prefix that its table has pages for.
int64_t positions_of(const approxifer_prefix_attention_args& p) { return p.prefix_len < p.prefix_pages * p.own.page_size ? p.prefix_len : p.prefix_pages * p.own.page_size; }
bool has_prefix(const approxifer_prefix_attention_args& p) { return positions_of(p) > 0; }
// Whether the sequences, or their query blocks, walk the prefix each for itself.
bool through(const approxifer_prefix_attention_args& p, const DeviceInfo& dev) {
  if (attention_token_eligible(p.own)) return !tiles_take(p) || attention_token_through_wanted(p.own, positions_of(p));
  return positions_of(p) + p.own.table_pages * p.own.page_size < (1LL << 30) && attention_tile_through_wanted(p, prefix_parts(p, dev), dev.sms);
}

// The parts of the prefix and the bytes that they, with one more for the own keys where that is kept apart, take.  Few partial results
// are joined on the way by the kernels over the own keys; of many each row's would be read one batch after another by the few CTAs
// that such calls have.  Measured, joined on the way against apart, us: 2 sequences of 59 tokens behind 4,096, 8 heads on 1 of 80,
// 15 parts 58 / 24; 42 tokens behind 13,961, 8 heads on 1 of 80, 36 parts 35 / 23.
PrefixParts parts_of(const approxifer_prefix_attention_args& p, const DeviceInfo& dev, int64_t* bytes) {
  PrefixParts parts = prefix_parts(p, dev);
  const bool token = attention_token_eligible(p.own);
  parts.apart = token ? parts.most > 8 && !attention_token_balanced(p.own) : parts.most > kOnTheWay;
  *bytes = ((parts.most + parts.apart) * parts.rows * ((p.own.D <= 64 ? 64 : 128) + 2) * (int64_t)sizeof(float) + 15) / 16 * 16;
  return parts;
}

}  // namespace

int64_t prefix_attention_workspace(const approxifer_prefix_attention_args& p) {
  const DeviceInfo* dev;
  const bool token = attention_token_eligible(p.own);
  if (!(token || tiles_take(p)) || current_device_info(&dev) != cudaSuccess) return 0;
  if (!has_prefix(p)) return token ? attention_token_workspace(p.own) : 0;
  if (through(p, *dev)) return 0;
  int64_t bytes;
  parts_of(p, *dev, &bytes);
  return bytes + (token ? attention_token_behind_workspace(p.own) : 0);
}

cudaError_t launch_prefix_attention(const approxifer_prefix_attention_args& p, cudaStream_t stream) {
  if (attention_token_eligible(p.own) || tiles_take(p)) {
    if (!has_prefix(p)) return launch_attention(p.own, stream);
    const DeviceInfo* dev;
    cudaError_t e = current_device_info(&dev);
    if (e != cudaSuccess) return e;
    if (through(p, *dev))
      return attention_token_eligible(p.own) ? launch_attention_token_through(p.own, p.prefix_table, (int32_t)(positions_of(p) - 1), stream)
                                             : launch_attention_tile_through(p, stream);
    int64_t used;
    PrefixParts parts = parts_of(p, *dev, &used);
    approxifer_attention_args own = p.own;
    const int dp = own.D <= 64 ? 64 : 128;
    parts.o = static_cast<float*>(own.workspace);
    parts.ml = reinterpret_cast<float2*>(parts.o + (parts.most + parts.apart) * parts.rows * dp);
    own.workspace = static_cast<char*>(own.workspace) + used, own.workspace_bytes -= used;
    if ((e = launch_attention_over_prefix(p, parts, stream)) != cudaSuccess) return e;
    e = attention_token_eligible(own) ? launch_attention_token_behind(own, parts, stream) : launch_attention_tile_behind(own, parts, stream);
    if (e != cudaSuccess || !parts.apart) return e;
    return launch_kernel(dp == 64 ? prefix_join_kernel<64> : prefix_join_kernel<128>, own.T * own.Hq, 128, 0, 1, stream, own, parts);
  }
  const int64_t units = p.own.T * p.own.Hq, per = kElementThreads / 32;
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  prefix_element_kernel<<<(unsigned)blocks, kElementThreads, 0, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace approxifer
