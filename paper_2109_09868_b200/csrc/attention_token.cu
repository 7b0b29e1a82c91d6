// Attention of one token per sequence over a paged cache: every visible key and value is read once, so the call is bound
// by HBM, and the work is cut along the cache.
//
// A cluster of S CTAs takes one (sequence, key head, 16 of the query heads that share it); its visible positions -- the
// sinks, then the window -- are dealt to the cluster's warps in chunks of 16 keys.  Every WARP is a pipeline of its own:
// it copies chunks into its private ring (16-byte asynchronous copies, pages looked up one chunk ahead, positions that are
// not there filled with zeros) and reduces the oldest with mma.m16n8k16 (the query heads are the 16 rows; a tcgen05 tile
// of 128 rows would be seven eighths padding, and the tensor pipes idle either way), keeping the running maximum and sum of
// the softmax and the output in fp32 registers.  The warps' results meet in shared memory, the CTAs' in the shared memory
// of their cluster, each time in a fixed order.
#include "async.cuh"

namespace approxifer {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kKeys = 16;   // keys per chunk
constexpr int kRows = 16;   // query heads per CTA
constexpr int kStages = 3;
constexpr unsigned kFull = 0xffffffffu;

constexpr int chunk_bytes(int dp) { return kKeys * dp * 2; }                            // keys, or values, of a chunk
constexpr int smem_bytes(int dp) { return kWarps * kStages * 2 * chunk_bytes(dp) + 1024; }
// After the loop the rings hold the results: float o[warp][16][DP], then m[warp][16], l[warp][16].
static_assert(kWarps * kRows * 128 * 4 + kWarps * kRows * 8 <= kWarps * kStages * 2 * chunk_bytes(128), "results exceed the rings");
static_assert(kWarps * kRows * 64 * 4 + kWarps * kRows * 8 <= kWarps * kStages * 2 * chunk_bytes(64), "results exceed the rings");

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DP>
__global__ void __launch_bounds__(kThreads) attention_token_kernel(const __grid_constant__ approxifer_attention_args a, int row_tiles) {
  extern __shared__ __align__(1024) unsigned char smem[];
  constexpr int kCols = DP / 8;  // 16-byte columns of a row
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int S = (int)cluster_size(), rank = (int)cluster_rank();
  int unit = blockIdx.x / S;
  const int rt = unit % row_tiles;
  unit /= row_tiles;
  const int hk = unit % a.Hkv, b = unit / a.Hkv;
  const int group = a.Hq / a.Hkv, row0 = rt * kRows, rows = min(kRows, group - row0);
  const int t = __ldg(a.q_start + b), queries = __ldg(a.q_start + b + 1) - t;
  const bool live = queries == 1 && t >= 0 && t < a.T;  // (max_q = 1; a sequence without a new token has no row)

  // visible positions: 0 .. sinks-1, then first .. last
  const int64_t held = a.table_pages * a.page_size;
  const int64_t p = live ? (int64_t)__ldg(a.kv_len + b) - 1 : -1;
  const int64_t last = p < held ? p : held - 1;
  const int64_t first = a.window && p >= a.window ? p - a.window + 1 : 0;
  const int64_t sinks = a.sinks < first ? a.sinks : first;
  const int64_t span = last >= first ? last - first + 1 : 0;
  const int64_t seen = sinks + span;  // (sinks may lie beyond `last` only where the table is too short: masked below)
  const int chunks = (int)((seen + kKeys - 1) / kKeys);
  const int32_t* table = a.block_table + (int64_t)b * a.table_stride;

  unsigned char* ring = smem + warp * (kStages * 2 * chunk_bytes(DP));
  const uint32_t ring_addr = smem_addr(ring);
  if (a.D < DP)  // columns beyond D are never copied: zero for good
    for (int i = lane; i < kStages * 2 * chunk_bytes(DP) / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
  __syncwarp();

  // queries: fragments of the 16 x DP matrix, scaled scores are formed after the product
  uint32_t qf[DP / 16][4];
  {
    const bf16* q = reinterpret_cast<const bf16*>(a.q) + (int64_t)t * a.q_tstride + (int64_t)(hk * group + row0) * a.q_hstride;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = lane / 4 + (i & 1) * 8, c = ks * 16 + (lane % 4) * 2 + (i >> 1) * 8;
        qf[ks][i] = (live && r < rows && c < a.D) ? *reinterpret_cast<const uint32_t*>(q + (int64_t)r * a.q_hstride + c) : 0u;
      }
  }

  // lanes 0..15: where the rows of a chunk are (both caches), and which are there at all
  const int stride = S * kWarps, c0 = rank * kWarps + warp;
  auto look_up = [&](int c, int64_t* j) -> int32_t {  // page of this lane's position of chunk c, -1 if there is none
    const int64_t u = (int64_t)c * kKeys + (lane % kKeys);
    *j = u < sinks ? u : first + (u - sinks);
    if (c >= chunks || u >= seen || *j > last) return -1;
    const int32_t page = __ldg(table + *j / a.page_size);
    return page >= 0 && page < a.num_pages ? page : -1;
  };
  auto fetch = [&](int slot, int32_t page, int64_t j) -> uint32_t {  // starts the copies of a chunk; which keys are there
    const uint32_t there = __ballot_sync(kFull, page >= 0) & 0xffffu;
    const int64_t at = page >= 0 ? j % a.page_size : 0, pg = page >= 0 ? page : 0;
    const int64_t ko = pg * a.kc_pstride + at * a.kc_rstride + (int64_t)hk * a.kc_hstride;
    const int64_t vo = pg * a.vc_pstride + at * a.vc_rstride + (int64_t)hk * a.vc_hstride;
    const uint32_t kdst = ring_addr + slot * 2 * chunk_bytes(DP), vdst = kdst + chunk_bytes(DP);
#pragma unroll
    for (int i = 0; i < kKeys * kCols / 32; ++i) {
      const int row = (lane + 32 * i) / kCols, col = (lane + 32 * i) % kCols;
      const int64_t k = __shfl_sync(kFull, ko, row), v = __shfl_sync(kFull, vo, row);
      const uint32_t to = row * DP * 2 + ((col ^ (row & 7)) << 4);
      if (col * 8 < a.D) {
        const bool ok = (there >> row) & 1;
        copy16(kdst + to, reinterpret_cast<const bf16*>(a.k_cache) + k + col * 8, ok);
        copy16(vdst + to, reinterpret_cast<const bf16*>(a.v_cache) + v + col * 8, ok);
      }
    }
    return there;
  };

  float o[DP / 8][4] = {};
  float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
  const float scale = a.scale * 1.4426950408889634f;  // the softmax runs on powers of two
  uint32_t there[kStages];
  int64_t j;
  int32_t page;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    page = look_up(c0 + s * stride, &j);
    there[s] = fetch(s, page, j);
    copy_commit();
  }
  page = look_up(c0 + (kStages - 1) * stride, &j);
  int slot = 0;
  for (int c = c0; c < chunks; c += stride) {
    // `there` and the ring turn together; kStages is small, so the rotation is three moves
    const uint32_t newest = fetch((slot + kStages - 1) % kStages, page, j);
    copy_commit();
    page = look_up(c + kStages * stride, &j);
    copy_wait<kStages - 1>();
    __syncwarp();
    const uint32_t mask = there[0];
#pragma unroll
    for (int s = 0; s + 1 < kStages - 1; ++s) there[s] = there[s + 1];
    there[kStages - 2] = newest;
    const uint32_t ks_addr = ring_addr + slot * 2 * chunk_bytes(DP), vs_addr = ks_addr + chunk_bytes(DP);

    float s[2][4] = {};
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
      uint32_t kb[4];
      const int key = (lane / 16) * 8 + lane % 8, col = ks * 2 + (lane / 8) % 2;
      ldmatrix4(ks_addr + key * DP * 2 + ((col ^ (key & 7)) << 4), kb);
      mma16816(s[0], qf[ks], kb[0], kb[1]);
      mma16816(s[1], qf[ks], kb[2], kb[3]);
    }
    float top[2] = {m[0], m[1]};
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = n * 8 + (lane % 4) * 2 + (i & 1);
        s[n][i] = (mask >> key) & 1 ? s[n][i] * scale : -CUDART_INF_F;
        top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
      }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor_sync(kFull, top[r], 1));
      top[r] = fmaxf(top[r], __shfl_xor_sync(kFull, top[r], 2));
    }
    const float base[2] = {top[0] == -CUDART_INF_F ? 0.f : top[0], top[1] == -CUDART_INF_F ? 0.f : top[1]};
    if (__any_sync(kFull, top[0] != m[0] || top[1] != m[1])) {
      const float keep[2] = {exp2f(m[0] - base[0]), exp2f(m[1] - base[1])};
      l[0] *= keep[0], l[1] *= keep[1];
#pragma unroll
      for (int d = 0; d < DP / 8; ++d) o[d][0] *= keep[0], o[d][1] *= keep[0], o[d][2] *= keep[1], o[d][3] *= keep[1];
      m[0] = top[0], m[1] = top[1];
    }
    uint32_t pf[4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float e0 = exp2f(s[n][0] - base[0]), e1 = exp2f(s[n][1] - base[0]), e2 = exp2f(s[n][2] - base[1]), e3 = exp2f(s[n][3] - base[1]);
      l[0] += e0 + e1, l[1] += e2 + e3;
      pf[2 * n] = pack_bf16x2(e0, e1), pf[2 * n + 1] = pack_bf16x2(e2, e3);
    }
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt) {
      uint32_t vb[4];
      const int key = lane % 16, col = dt * 2 + lane / 16;
      ldmatrix4_t(vs_addr + key * DP * 2 + ((col ^ (key & 7)) << 4), vb);
      mma16816(o[2 * dt], pf, vb[0], vb[1]);
      mma16816(o[2 * dt + 1], pf, vb[2], vb[3]);
    }
    __syncwarp();  // the slot may be filled again
    slot = (slot + 1) % kStages;
  }
  copy_wait<0>();
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(kFull, l[r], 1);
    l[r] += __shfl_xor_sync(kFull, l[r], 2);
  }
  // warps -> CTA.  o[16][DP], m[16], l[16] of warp 0's place receive the CTA's result.
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);
  float* sm = so + kWarps * kRows * DP;
  float* sl = sm + kWarps * kRows;
#pragma unroll
  for (int d = 0; d < DP / 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int r = lane / 4 + (i / 2) * 8;
      *reinterpret_cast<float2*>(so + (warp * kRows + r) * DP + d * 8 + (lane % 4) * 2) = make_float2(o[d][i], o[d][i + 1]);
    }
  if (lane % 4 == 0) {
    sm[warp * kRows + lane / 4] = m[0], sm[warp * kRows + lane / 4 + 8] = m[1];
    sl[warp * kRows + lane / 4] = l[0], sl[warp * kRows + lane / 4 + 8] = l[1];
  }
  __syncthreads();
  bf16* out = reinterpret_cast<bf16*>(a.out) + (int64_t)t * a.o_tstride + (int64_t)(hk * group + row0) * a.o_hstride;
  if (S > 1) cluster_sync();
  // every CTA joins its share of the rows' elements over all warps of the cluster, in order
  const int cells = rows * (a.D / 2), x0 = cells * rank / S, x1 = cells * (rank + 1) / S;
  const int parts = S * kWarps;
  const uint32_t so_addr = smem_addr(so), sm_addr = smem_addr(sm), sl_addr = smem_addr(sl);
  for (int x = x0 + threadIdx.x; x < x1 && live; x += kThreads) {
    const int r = x / (a.D / 2), d = (x % (a.D / 2)) * 2;
    auto far = [&](uint32_t addr, int part) { return S == 1 ? addr : peer_smem(addr, part / kWarps); };
    auto get = [&](uint32_t addr) {
      float v;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
      return v;
    };
    float best = -CUDART_INF_F;
    for (int w = 0; w < parts; ++w) {
      const float v = get(far(sm_addr + ((w % kWarps) * kRows + r) * 4, w));
      best = fmaxf(best, v);
    }
    if (best == -CUDART_INF_F) best = 0.f;
    float total = 0.f, y0 = 0.f, y1 = 0.f;
    for (int w = 0; w < parts; ++w) {
      const int at = (w % kWarps) * kRows + r;
      const float k = exp2f(get(far(sm_addr + at * 4, w)) - best);
      total = fmaf(k, get(far(sl_addr + at * 4, w)), total);
      y0 = fmaf(k, get(far(so_addr + (at * DP + d) * 4, w)), y0);
      y1 = fmaf(k, get(far(so_addr + (at * DP + d + 1) * 4, w)), y1);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    *reinterpret_cast<uint32_t*>(out + (int64_t)r * a.o_hstride + d) = pack_bf16x2(total == 0.f ? 0.f : y0 * inv, total == 0.f ? 0.f : y1 * inv);
  }
  if (S > 1) cluster_sync();  // (a CTA's shared memory stays until all have read it)
}

template <int DP>
cudaError_t launch_one(const approxifer_attention_args& a, int row_tiles, int64_t units, int split, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  auto kernel = attention_token_kernel<DP>;
  struct Tag {};
  if ((e = ensure_dynamic_smem<Tag>(kernel, dev->ordinal, smem_bytes(DP))) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_bytes(DP);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kernel, a, row_tiles);
  count_launch();
  return e;
}

}  // namespace

bool attention_token_eligible(const approxifer_attention_args& a) {
  return a.max_q == 1 && a.D % 8 == 0 && a.D <= 128 && aligned16(a.k_cache) && aligned16(a.v_cache) && (reinterpret_cast<uintptr_t>(a.q) & 3) == 0 &&
         (reinterpret_cast<uintptr_t>(a.out) & 3) == 0 && a.q_tstride % 2 == 0 && a.q_hstride % 2 == 0 && a.o_tstride % 2 == 0 && a.o_hstride % 2 == 0 &&
         (a.kc_pstride | a.kc_hstride | a.kc_rstride | a.vc_pstride | a.vc_hstride | a.vc_rstride) % 8 == 0;
}

cudaError_t launch_attention_token(const approxifer_attention_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  const cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  const int group = a.Hq / a.Hkv, row_tiles = (group + kRows - 1) / kRows;
  const int64_t units = (int64_t)a.batch * a.Hkv * row_tiles;
  // The lengths are on the device; what a sequence can see at most says how far it is worth cutting: until there are
  // about four CTAs for every place on the GPU, none with less than two chunks for each warp.
  int64_t most = a.table_pages * a.page_size;
  if (a.window && (int64_t)a.window + a.sinks < most) most = (int64_t)a.window + a.sinks;
  int split = 1;
  while (split < 8 && units * split < 4LL * 2 * dev->sms && most >= (int64_t)split * 2 * kWarps * kKeys * 2) split *= 2;
  if (units * split > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  return a.D <= 64 ? launch_one<64>(a, row_tiles, units, split, stream) : launch_one<128>(a, row_tiles, units, split, stream);
}

}  // namespace approxifer
