// Attention of one token per sequence over a paged cache: every visible key and value is read once, so the call is bound
// by HBM, and the work is cut along the cache.
//
// One unit of work = (sequence, key head, 16 of the query heads that share it); its visible positions -- the sinks, then
// the window -- are cut into chunks of 8 KB of keys and values (16 keys up to D = 128, 32 up to D = 64).  Every WARP is a
// pipeline of its own: it copies chunks into its private ring (16-byte asynchronous copies, pages looked up one chunk ahead,
// positions that are not there filled with zeros) and reduces the oldest with mma.m16n8k16 (the query heads are the 16
// rows; a tcgen05 tile of 128 rows would be seven eighths padding, and the tensor pipes idle either way), keeping the
// running maximum and sum of the softmax and the output in fp32 registers.  Two ways to deal the chunks:
//
//   cluster form   a cluster of up to 8 CTAs takes one unit; its warps' results meet in the cluster's shared memory.  One
//                  launch, no workspace: the form for small calls.
//   balanced form  all chunks of the call in one row, cut into equal runs, one to each warp that the GPU holds: lengths may
//                  differ as they like.  A run that covers a whole unit writes its output; the others leave partial sums
//                  in the workspace, which a second small launch joins, in order.
//
// Measured: one token, 1,028 visible of 1,500 cached, 32 heads on 8 of 128: 7.0 us (latency: three loads that wait for one
// another, the joining); 48 tokens, window 4,096: 134 us, 6.0 TB/s, from a graph, 142 to 145 us, 5.6 TB/s, call by call; 4
// contexts of up to 131,072, 2 key heads of 64: 43 us, 4.6 TB/s (the joining of 148 partial results a unit is 5 us of it).
#include "async.cuh"

namespace approxifer {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kCtasPerSm = 2;
constexpr int kRows = 16;   // query heads per unit
constexpr int kStages = 3;
constexpr int kJoinWarps = 8, kJoinAhead = 6;
constexpr int kMaxSplit = 8;  // CTAs of a cluster
constexpr unsigned kFull = 0xffffffffu;

constexpr int keys_of(int dp) { return dp <= 64 ? 32 : 16; }                 // keys per chunk
constexpr int half_bytes(int dp) { return keys_of(dp) * dp * 2; }            // keys, or values, of a chunk
constexpr int ring_bytes(int dp) { return kStages * 2 * half_bytes(dp); }    // of a warp
constexpr int smem_bytes(int dp) { return kWarps * ring_bytes(dp); }
// After the loop of the cluster form the rings hold the results of the warps and of the CTA.
constexpr int result_bytes(int dp) { return (kWarps + 1) * kRows * (dp * 4 + 8); }
static_assert(result_bytes(128) <= smem_bytes(128) && result_bytes(64) <= smem_bytes(64), "results exceed the rings");

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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

__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// What one sequence's token sees -- positions 0 .. sinks-1 and first .. last -- as chunks of `keys` positions that start at
// multiples of `keys`: those that hold sinks, then those that hold the window.
struct Seen {
  const int32_t* table;
  int32_t first, last, sinks;
  int32_t token;  // its index, or -1 where the sequence has no new token (max_q = 1)
  int32_t sink_chunks, skip, chunks;
  __device__ __forceinline__ int32_t position(int c, int keys) const { return (c < sink_chunks ? c : c + skip) * keys; }
  // which of the keys of the chunk at `pos` are seen, a bit per key
  __device__ __forceinline__ uint32_t sees(int32_t pos, int keys) const {
    return bits_below(keys) & bits_below(last + 1 - pos) & (~bits_below(first - pos) | bits_below(sinks - pos));
  }
};
__device__ __forceinline__ Seen seen_by(const approxifer_attention_args& a, int b, int keys) {
  Seen s;
  const int t = __ldg(a.q_start + b), end = __ldg(a.q_start + b + 1);
  const bool live = end - t == 1 && t >= 0 && t < a.T;
  s.token = live ? t : -1;
  const int64_t held = a.table_pages * a.page_size;
  const int p = live ? __ldg(a.kv_len + b) - 1 : -1;
  s.last = p < held ? p : (int)held - 1;
  s.first = a.window && p >= a.window ? p - a.window + 1 : 0;
  s.sinks = a.sinks < s.first ? a.sinks : s.first;
  s.sinks = s.sinks < s.last + 1 ? s.sinks : s.last + 1;
  s.sink_chunks = s.sinks > 0 ? (s.sinks + keys - 1) / keys : 0;
  const int from = s.first / keys > s.sink_chunks ? s.first / keys : s.sink_chunks;
  s.skip = from - s.sink_chunks;
  const int in_window = s.last >= 0 ? s.last / keys - from + 1 : 0;
  s.chunks = s.last >= 0 ? s.sink_chunks + (in_window > 0 ? in_window : 0) : 0;
  s.table = a.block_table + (int64_t)b * a.table_stride;
  return s;
}

// Where the keys of a chunk lie.  WHOLE (pages of whole chunks): the chunk's page and first row, the same in all lanes, and which
// keys are there (none: page 0, never read).  Else: those of this lane's key (lane % keys), page -1 where it is not there.
struct Spot {
  int32_t page, row;
  uint32_t sees;
};
template <bool WHOLE>
__device__ __forceinline__ Spot nowhere() {
  return Spot{WHOLE ? 0 : -1, 0, 0};
}

// One warp's share of a unit.
template <int DP, bool WHOLE>
struct Warp {
  static constexpr int kKeys = keys_of(DP);
  static constexpr int kCols = DP / 8;  // 16-byte columns of a row
  static constexpr uint32_t kAll = kKeys == 32 ? 0xffffffffu : (1u << kKeys) - 1u;
  uint32_t q[DP / 16][4];               // fragments of the 16 x DP queries
  float o[DP / 8][4];
  float m[2], l[2];
  uint32_t ring;
  int lane;

  __device__ __forceinline__ void setup(unsigned char* at, int D) {
    lane = threadIdx.x % 32;
    ring = smem_addr(at);
    if (D < DP)  // columns beyond D are never copied: zero for good
      for (int i = lane; i < ring_bytes(DP) / 16; i += 32) reinterpret_cast<uint4*>(at)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
  }

  __device__ __forceinline__ void start(const approxifer_attention_args& a, int token, int head0, int rows) {
    const bf16* from = reinterpret_cast<const bf16*>(a.q) + (int64_t)token * a.q_tstride + (int64_t)head0 * a.q_hstride;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = lane / 4 + (i & 1) * 8, c = ks * 16 + (lane % 4) * 2 + (i >> 1) * 8;
        q[ks][i] = (token >= 0 && r < rows && c < a.D) ? *reinterpret_cast<const uint32_t*>(from + (int64_t)r * a.q_hstride + c) : 0u;
      }
#pragma unroll
    for (int d = 0; d < DP / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
    m[0] = m[1] = -CUDART_INF_F;
    l[0] = l[1] = 0.f;
  }

  __device__ __forceinline__ Spot look_up(const approxifer_attention_args& a, int page_shift, const Seen& s, int c) const {
    Spot at = nowhere<WHOLE>();
    if (c >= s.chunks) return at;
    const int32_t pos = s.position(c, kKeys);
    at.sees = s.sees(pos, kKeys);
    if constexpr (WHOLE) {
      at.page = __ldg(s.table + (pos >> page_shift));
      at.row = pos & ((1 << page_shift) - 1);
      if (at.page < 0 || at.page >= a.num_pages) at.page = 0, at.sees = 0;
    } else {
      const uint32_t j = (uint32_t)pos + lane % kKeys, entry = j / (uint32_t)a.page_size;
      at.row = (int32_t)(j - entry * (uint32_t)a.page_size);
      if ((at.sees >> (lane % kKeys)) & 1) at.page = __ldg(s.table + entry);
      if (at.page >= a.num_pages) at.page = -1;
    }
    return at;
  }

  // Starts the copies of a chunk; which of its keys are there.
  __device__ __forceinline__ uint32_t fetch(const approxifer_attention_args& a, int slot, const Spot& at, int hk) const {
    constexpr int kStep = 32 / kCols;  // rows from one copy of a lane to its next
    const int r0 = lane / kCols, col = lane % kCols;
    const uint32_t kdst = ring + slot * 2 * half_bytes(DP) + r0 * DP * 2, x = (col ^ r0) << 4;
    const bool in = col * 8 < a.D;
    if constexpr (WHOLE) {
      const bf16* k = reinterpret_cast<const bf16*>(a.k_cache) + at.page * a.kc_pstride + hk * a.kc_hstride + (at.row + r0) * a.kc_rstride + col * 8;
      const bf16* v = reinterpret_cast<const bf16*>(a.v_cache) + at.page * a.vc_pstride + hk * a.vc_hstride + (at.row + r0) * a.vc_rstride + col * 8;
      const int64_t kst = kStep * a.kc_rstride, vst = kStep * a.vc_rstride;
      if (at.sees == kAll) {
#pragma unroll
        for (int i = 0; i < kKeys / kStep; ++i, k += kst, v += vst) {
          const uint32_t to = kdst + i * kStep * DP * 2 + (x ^ (((i * kStep) & 7) << 4));
          if (in) copy16(to, k), copy16(to + half_bytes(DP), v);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kKeys / kStep; ++i, k += kst, v += vst) {
          const uint32_t to = kdst + i * kStep * DP * 2 + (x ^ (((i * kStep) & 7) << 4));
          const bool ok = (at.sees >> (r0 + i * kStep)) & 1;
          if (in) copy16(to, k, ok), copy16(to + half_bytes(DP), v, ok);
        }
      }
      return at.sees;
    } else {
      const uint32_t there = __ballot_sync(kFull, at.page >= 0);
      const int64_t pg = at.page >= 0 ? at.page : 0, row = at.page >= 0 ? at.row : 0;
      const int64_t ko = pg * a.kc_pstride + row * a.kc_rstride + (int64_t)hk * a.kc_hstride;
      const int64_t vo = pg * a.vc_pstride + row * a.vc_rstride + (int64_t)hk * a.vc_hstride;
#pragma unroll
      for (int i = 0; i < kKeys / kStep; ++i) {
        const int r = r0 + i * kStep;
        const int64_t k = __shfl_sync(kFull, ko, r), v = __shfl_sync(kFull, vo, r);
        const uint32_t to = kdst + i * kStep * DP * 2 + (x ^ (((i * kStep) & 7) << 4));
        const bool ok = (there >> r) & 1;
        if (in) {
          copy16(to, reinterpret_cast<const bf16*>(a.k_cache) + k + col * 8, ok);
          copy16(to + half_bytes(DP), reinterpret_cast<const bf16*>(a.v_cache) + v + col * 8, ok);
        }
      }
      return there & kAll;
    }
  }

  // scale: of the scores, times log2 e (the softmax runs on powers of two).
  __device__ __forceinline__ void reduce(int slot, uint32_t there, float scale) {
    const uint32_t kat = ring + slot * 2 * half_bytes(DP) + ((lane / 16) * 8 + lane % 8) * DP * 2, kx = ((lane / 8) % 2 ^ (lane & 7)) << 4;
    const uint32_t vat = ring + slot * 2 * half_bytes(DP) + half_bytes(DP) + (lane % 16) * DP * 2, vx = (lane / 16 ^ (lane & 7)) << 4;
    float s[kKeys / 8][4];
#pragma unroll
    for (int n = 0; n < kKeys / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int n = 0; n < kKeys / 16; ++n) {
        uint32_t kb[4];
        ldmatrix4(kat + n * 16 * DP * 2 + (kx ^ (ks << 5)), kb);
        mma16816(s[2 * n], q[ks], kb[0], kb[1]);
        mma16816(s[2 * n + 1], q[ks], kb[2], kb[3]);
      }
#pragma unroll
    for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] *= scale;
    if (there != kAll) {
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = (there >> (n * 8 + (lane % 4) * 2 + (i & 1))) & 1 ? s[n][i] : -CUDART_INF_F;
    }
    float top[2] = {m[0], m[1]};
#pragma unroll
    for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor_sync(kFull, top[r], 1));
      top[r] = fmaxf(top[r], __shfl_xor_sync(kFull, top[r], 2));
    }
    const float base[2] = {top[0] == -CUDART_INF_F ? 0.f : top[0], top[1] == -CUDART_INF_F ? 0.f : top[1]};
    if (__any_sync(kFull, top[0] != m[0] || top[1] != m[1])) {
      const float keep[2] = {pow2(m[0] - base[0]), pow2(m[1] - base[1])};
      l[0] *= keep[0], l[1] *= keep[1];
#pragma unroll
      for (int d = 0; d < DP / 8; ++d) o[d][0] *= keep[0], o[d][1] *= keep[0], o[d][2] *= keep[1], o[d][3] *= keep[1];
      m[0] = top[0], m[1] = top[1];
    }
#pragma unroll
    for (int kk = 0; kk < kKeys / 16; ++kk) {
      uint32_t p[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float(&x)[4] = s[2 * kk + n];
        const float e0 = pow2(x[0] - base[0]), e1 = pow2(x[1] - base[0]), e2 = pow2(x[2] - base[1]), e3 = pow2(x[3] - base[1]);
        l[0] += e0 + e1, l[1] += e2 + e3;
        p[2 * n] = pack_bf16x2(e0, e1), p[2 * n + 1] = pack_bf16x2(e2, e3);
      }
#pragma unroll
      for (int dt = 0; dt < DP / 16; ++dt) {
        uint32_t vb[4];
        ldmatrix4_t(vat + kk * 16 * DP * 2 + (vx ^ (dt << 5)), vb);
        mma16816(o[2 * dt], p, vb[0], vb[1]);
        mma16816(o[2 * dt + 1], p, vb[2], vb[3]);
      }
    }
    __syncwarp();  // the slot may be filled again
  }

  __device__ __forceinline__ void finish() {  // the sums of the rows, from the four lanes that share them
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(kFull, l[r], 1);
      l[r] += __shfl_xor_sync(kFull, l[r], 2);
    }
  }
};

// N partial results (maximum and sum, two elements) as one.
struct Joined {
  float m, l;
  float2 v;
};
template <int N>
__device__ __forceinline__ Joined join(const float2 (&ml)[N], const float2 (&v)[N]) {
  Joined j{ml[0].x, 0.f, make_float2(0.f, 0.f)};
#pragma unroll
  for (int p = 1; p < N; ++p) j.m = fmaxf(j.m, ml[p].x);
  const float base = j.m == -CUDART_INF_F ? 0.f : j.m;
#pragma unroll
  for (int p = 0; p < N; ++p) {
    const float k = pow2(ml[p].x - base);
    j.l = fmaf(k, ml[p].y, j.l);
    j.v.x = fmaf(k, v[p].x, j.v.x), j.v.y = fmaf(k, v[p].y, j.v.y);
  }
  return j;
}

template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) attention_token_cluster_kernel(const __grid_constant__ approxifer_attention_args a, int row_tiles,
                                                                                        int page_shift) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int S = (int)cluster_size(), rank = (int)cluster_rank();
  let_next_start();
  wait_for_inputs();
  int unit = blockIdx.x / S;
  const int rt = unit % row_tiles;
  unit /= row_tiles;
  const int hk = unit % a.Hkv, b = unit / a.Hkv;
  const int group = a.Hq / a.Hkv, head0 = hk * group + rt * kRows, rows = min(kRows, group - rt * kRows);
  const Seen seen = seen_by(a, b, keys_of(DP));
  const int stride = S * kWarps, c0 = rank * kWarps + warp;

  Warp<DP, WHOLE> w;
  w.setup(smem + warp * ring_bytes(DP), a.D);
  uint32_t there[kStages];
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    there[s] = w.fetch(a, s, w.look_up(a, page_shift, seen, c0 + s * stride), hk);
    copy_commit();
  }
  Spot ahead = w.look_up(a, page_shift, seen, c0 + (kStages - 1) * stride);
  w.start(a, seen.token, head0, rows);
  const float scale = a.scale * 1.4426950408889634f;
  int slot = 0;
  for (int c = c0; c < seen.chunks; c += stride) {
    there[kStages - 1] = w.fetch(a, (slot + kStages - 1) % kStages, ahead, hk);
    copy_commit();
    ahead = w.look_up(a, page_shift, seen, c + kStages * stride);
    copy_wait<kStages - 1>();
    __syncwarp();
    w.reduce(slot, there[0], scale);
#pragma unroll
    for (int s = 0; s + 1 < kStages; ++s) there[s] = there[s + 1];
    slot = (slot + 1) % kStages;
  }
  copy_wait<0>();
  w.finish();
  // The warps' results meet in the CTA, the CTAs' in the cluster: every CTA takes its share of the rows' elements (pairs of
  // them), all the loads of one side by side.
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);                      // [warp][16][DP]
  float2* sml = reinterpret_cast<float2*>(so + kWarps * kRows * DP);  // [warp][16] m, l
  float2* cta_o = sml + kWarps * kRows;                            // [16][DP / 2] of this CTA
  float2* cta_ml = cta_o + kRows * DP / 2;                         // [16]
#pragma unroll
  for (int d = 0; d < DP / 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      *reinterpret_cast<float2*>(so + (warp * kRows + lane / 4 + i * 4) * DP + d * 8 + (lane % 4) * 2) = make_float2(w.o[d][i], w.o[d][i + 1]);
  if (lane % 4 == 0) {
    sml[warp * kRows + lane / 4] = make_float2(w.m[0], w.l[0]);
    sml[warp * kRows + lane / 4 + 8] = make_float2(w.m[1], w.l[1]);
  }
  __syncthreads();
  const int pairs = a.D / 2, cells = seen.token < 0 ? 0 : rows * pairs;
  for (int x = threadIdx.x; x < cells; x += kThreads) {
    const int r = x / pairs, d = x % pairs;
    float2 ml[kWarps], v[kWarps];
#pragma unroll
    for (int p = 0; p < kWarps; ++p) ml[p] = sml[p * kRows + r], v[p] = *reinterpret_cast<const float2*>(so + (p * kRows + r) * DP + 2 * d);
    const Joined j = join<kWarps>(ml, v);
    cta_o[r * (DP / 2) + d] = j.v;
    if (d == 0) cta_ml[r] = make_float2(j.m, j.l);
  }
  if (S > 1) cluster_sync();
  else __syncthreads();
  bf16* out = reinterpret_cast<bf16*>(a.out) + (int64_t)seen.token * a.o_tstride + (int64_t)head0 * a.o_hstride;
  const int x0 = cells * rank / S, x1 = cells * (rank + 1) / S;
  for (int x = x0 + threadIdx.x; x < x1; x += kThreads) {
    const int r = x / pairs, d = x % pairs;
    float2 ml[kMaxSplit], v[kMaxSplit];
#pragma unroll
    for (int p = 0; p < kMaxSplit; ++p) {
      ml[p] = make_float2(-CUDART_INF_F, 0.f), v[p] = make_float2(0.f, 0.f);
      if (p < S) ml[p] = peer_load2(peer_smem(smem_addr(cta_ml + r), p)), v[p] = peer_load2(peer_smem(smem_addr(cta_o + r * (DP / 2) + d), p));
    }
    const Joined j = join<kMaxSplit>(ml, v);
    const float inv = j.l == 0.f ? 0.f : 1.f / j.l;
    *reinterpret_cast<uint32_t*>(out + (int64_t)r * a.o_hstride + 2 * d) = j.l == 0.f ? 0u : pack_bf16x2(j.v.x * inv, j.v.y * inv);
  }
  if (S > 1) cluster_sync();  // (a CTA's shared memory stays until all have read it)
}

// ---- balanced form ----

// Workspace: two partial results for each warp (of a run's first unit, if the run starts inside it, and of its last, if it
// ends inside it): float o[2 * warps][16][DP], then m, l [2 * warps][16].
int64_t partial_floats(int dp) { return 2 * kRows * (dp + 2); }

// All chunks of the call stand in a row: sequence after sequence, and of a sequence unit after unit.  The warp that finds a
// place in the row: the sequence and the number of chunks before it.
struct Place {
  int b;
  int64_t before;
};
// Adds up the chunks of all sequences (returned) and finds the one that holds chunk `x`, or, with x < 0, sequence `b_of`.
__device__ __forceinline__ int64_t count_chunks(const approxifer_attention_args& a, int units, int keys, int64_t x, int b_of, Place* place) {
  const int lane = threadIdx.x % 32;
  int64_t total = 0;
  place->b = -1;
  place->before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    const int b = b0 + lane;
    const int64_t n = b < a.batch ? (int64_t)seen_by(a, b, keys).chunks * units : 0;
    int64_t upto = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(kFull, upto, d);
      if (lane >= d) upto += v;
    }
    const bool here = x >= 0 ? (total + upto - n <= x && x < total + upto) : b == b_of;
    const unsigned who = __ballot_sync(kFull, here);
    if (who) {
      place->b = b0 + __ffs(who) - 1;
      place->before = total + __shfl_sync(kFull, upto - n, __ffs(who) - 1);
    }
    total += __shfl_sync(kFull, upto, 31);
  }
  return total;
}

// Where a warp stands in the row of chunks.
struct Cursor {
  Seen seen;
  int b, unit, c;  // unit of the sequence: key head and row tile
  __device__ __forceinline__ void next(const approxifer_attention_args& a, int units, int keys) {
    if (++c < seen.chunks) return;
    c = 0;
    if (++unit < units) return;
    unit = 0;
    do {
      ++b;
      if (b >= a.batch) break;
      seen = seen_by(a, b, keys);
    } while (seen.chunks == 0);
  }
};

template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 3) attention_token_balanced_kernel(const __grid_constant__ approxifer_attention_args a, int row_tiles,
                                                                                         int page_shift, float* partial) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const int warp = blockIdx.x * kWarps + threadIdx.x / 32, warps = gridDim.x * kWarps, lane = threadIdx.x % 32;
  const int units = a.Hkv * row_tiles, group = a.Hq / a.Hkv;
  wait_for_inputs();
  let_next_start();  // (only now: the kernel that joins counts the chunks, from the call's inputs, before it waits for this one)
  Place at;
  const int64_t total = count_chunks(a, units, keys_of(DP), 0, 0, &at);
  const int runs = total < warps ? (int)total : warps;  // (no empty runs)
  if (warp >= runs) return;
  const int64_t x0 = total * warp / runs, x1 = total * (warp + 1) / runs;
  count_chunks(a, units, keys_of(DP), x0, 0, &at);
  Cursor get, use;
  get.b = at.b;
  get.seen = seen_by(a, at.b, keys_of(DP));
  get.unit = (int)((x0 - at.before) / get.seen.chunks);
  get.c = (int)((x0 - at.before) % get.seen.chunks);
  use = get;
  int64_t to_get = x1 - x0;

  Warp<DP, WHOLE> w;
  w.setup(smem + (threadIdx.x / 32) * ring_bytes(DP), a.D);
  uint32_t there[kStages];
  Spot ahead;
  int hk = 0;
  auto look_ahead = [&]() {
    if (to_get-- > 0) {
      ahead = w.look_up(a, page_shift, get.seen, get.c);
      hk = get.unit / row_tiles;
      if (to_get > 0) get.next(a, units, keys_of(DP));
    } else {
      ahead = nowhere<WHOLE>();
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    look_ahead();
    there[s] = w.fetch(a, s, ahead, hk);
    copy_commit();
  }
  look_ahead();
  const float scale = a.scale * 1.4426950408889634f;
  int slot = 0;
  bool from_start = use.c == 0;
  int head0 = (use.unit / row_tiles) * group + (use.unit % row_tiles) * kRows;
  int rows = min(kRows, group - (use.unit % row_tiles) * kRows);
  w.start(a, use.seen.token, head0, rows);
  for (int64_t x = x0; x < x1; ++x) {
    there[kStages - 1] = w.fetch(a, (slot + kStages - 1) % kStages, ahead, hk);
    copy_commit();
    look_ahead();
    copy_wait<kStages - 1>();
    __syncwarp();
    w.reduce(slot, there[0], scale);
#pragma unroll
    for (int s = 0; s + 1 < kStages; ++s) there[s] = there[s + 1];
    slot = (slot + 1) % kStages;
    const bool whole = use.c + 1 == use.seen.chunks;
    if (whole || x + 1 == x1) {  // the end of the unit or of the run
      w.finish();
      if (whole && from_start) {
        const float inv[2] = {w.l[0] == 0.f ? 0.f : 1.f / w.l[0], w.l[1] == 0.f ? 0.f : 1.f / w.l[1]};
        bf16* out = reinterpret_cast<bf16*>(a.out) + (int64_t)use.seen.token * a.o_tstride + (int64_t)head0 * a.o_hstride;
#pragma unroll
        for (int d = 0; d < DP / 8; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = lane / 4 + h * 8, col = d * 8 + (lane % 4) * 2;
            if (r < rows && col < a.D)
              *reinterpret_cast<uint32_t*>(out + (int64_t)r * a.o_hstride + col) =
                  w.l[h] == 0.f ? 0u : pack_bf16x2(w.o[d][2 * h] * inv[h], w.o[d][2 * h + 1] * inv[h]);
          }
      } else {
        const int64_t part = 2 * (int64_t)warp + (from_start ? 1 : 0);
        float* po = partial + part * kRows * DP;
        float* pm = partial + 2 * (int64_t)warps * kRows * DP + part * kRows * 2;
#pragma unroll
        for (int d = 0; d < DP / 8; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = lane / 4 + h * 8;
            if (r < rows) *reinterpret_cast<float2*>(po + r * DP + d * 8 + (lane % 4) * 2) = make_float2(w.o[d][2 * h], w.o[d][2 * h + 1]);
          }
        if (lane % 4 == 0)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (lane / 4 + h * 8 < rows) *reinterpret_cast<float2*>(pm + (lane / 4 + h * 8) * 2) = make_float2(w.m[h], w.l[h]);
      }
      if (x + 1 < x1) {
        use.next(a, units, keys_of(DP));
        from_start = true;
        head0 = (use.unit / row_tiles) * group + (use.unit % row_tiles) * kRows;
        rows = min(kRows, group - (use.unit % row_tiles) * kRows);
        w.start(a, use.seen.token, head0, rows);
      }
    } else {
      ++use.c;
    }
  }
  copy_wait<0>();
}

// Joins the partial results of every unit that more than one run shares, and zeroes the rows that see nothing.  One CTA =
// one row; its warps (for short rows their halves) take the partial results in turn, kJoinAhead loads in flight, and meet in
// shared memory.
template <int DP, int JW>
__global__ void __launch_bounds__(JW * 32) attention_token_join_kernel(const __grid_constant__ approxifer_attention_args a, int row_tiles, int warps,
                                                                              const float* partial) {
  constexpr int kLanes = DP / 4, kTeams = JW * 32 / kLanes;  // lanes to a partial row, partial rows at a time
  __shared__ __align__(16) float sy[kTeams][DP];
  __shared__ float sm[kTeams], sl[kTeams];
  let_next_start();
  const int team = threadIdx.x / kLanes, at4 = (threadIdx.x % kLanes) * 4;
  const int units = a.Hkv * row_tiles, group = a.Hq / a.Hkv;
  const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, in_group = h % group;
  Place at;
  const int64_t total = count_chunks(a, units, keys_of(DP), -1, b, &at);
  const Seen seen = seen_by(a, b, keys_of(DP));
  wait_for_inputs();
  if (seen.token < 0) return;
  bf16* out = reinterpret_cast<bf16*>(a.out) + (int64_t)seen.token * a.o_tstride + (int64_t)h * a.o_hstride;
  if (seen.chunks == 0) {
    for (int d = threadIdx.x; d < a.D; d += JW * 32) out[d] = narrow<bf16>(0.f);
    return;
  }
  const int64_t x0 = at.before + (int64_t)((h / group) * row_tiles + in_group / kRows) * seen.chunks, x1 = x0 + seen.chunks;
  const int64_t runs = total < warps ? total : warps;
  const int w0 = (int)(((x0 + 1) * runs - 1) / total), w1 = (int)((x1 * runs - 1) / total);  // the runs that hold its first and its last chunk
  if (w0 == w1) return;
  const float* pm = partial + 2 * (int64_t)warps * kRows * DP;
  const int r = in_group % kRows;
  auto part = [&](int w) { return (2 * (int64_t)w + (w == w0 ? 1 : 0)) * kRows + r; };  // the first of them ends inside the unit
  float m = -CUDART_INF_F, l = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = w0 + team; w <= w1; w += kJoinAhead * kTeams) {
    float2 ml[kJoinAhead];
    float4 v[kJoinAhead];
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      const int wi = w + i * kTeams;
      ml[i] = make_float2(-CUDART_INF_F, 0.f);
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (wi <= w1) {
        const int64_t p = part(wi);
        ml[i] = __ldcg(reinterpret_cast<const float2*>(pm + p * 2));
        v[i] = __ldcg(reinterpret_cast<const float4*>(partial + p * DP + at4));
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) top = fmaxf(top, ml[i].x);
    const float base = top == -CUDART_INF_F ? 0.f : top, keep = pow2(m - base);
    l *= keep, y.x *= keep, y.y *= keep, y.z *= keep, y.w *= keep;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      const float k = pow2(ml[i].x - base);
      l = fmaf(k, ml[i].y, l);
      y.x = fmaf(k, v[i].x, y.x), y.y = fmaf(k, v[i].y, y.y), y.z = fmaf(k, v[i].z, y.z), y.w = fmaf(k, v[i].w, y.w);
    }
    m = top;
  }
  if (at4 == 0) sm[team] = m, sl[team] = l;
  *reinterpret_cast<float4*>(&sy[team][at4]) = y;
  __syncthreads();
  float best = sm[0];
#pragma unroll
  for (int w = 1; w < kTeams; ++w) best = fmaxf(best, sm[w]);
  if (best == -CUDART_INF_F) best = 0.f;
  for (int d = threadIdx.x; d < a.D; d += JW * 32) {
    float sum = 0.f, z = 0.f;
#pragma unroll
    for (int w = 0; w < kTeams; ++w) {
      const float k = pow2(sm[w] - best);
      sum = fmaf(k, sl[w], sum);
      z = fmaf(k, sy[w][d], z);
    }
    out[d] = narrow<bf16>(sum == 0.f ? 0.f : z / sum);
  }
}

// Chunks the call has at most (the lengths are on the device; the table's width and the window bound them).
int64_t most_seen(const approxifer_attention_args& a) {
  const int64_t held = a.table_pages * a.page_size;
  return a.window && (int64_t)a.window + a.sinks < held ? (int64_t)a.window + a.sinks : held;
}
int64_t units_of(const approxifer_attention_args& a) { return (int64_t)a.batch * a.Hkv * ((a.Hq / a.Hkv + kRows - 1) / kRows); }
template <int DP, bool WHOLE>
cudaError_t launch_cluster(const approxifer_attention_args& a, const DeviceInfo& dev, int row_tiles, int page_shift, int64_t units, int split, cudaStream_t stream) {
  auto kernel = attention_token_cluster_kernel<DP, WHOLE>;
  struct Tag {};
  cudaError_t e = ensure_dynamic_smem<Tag>(kernel, dev.ordinal, smem_bytes(DP));
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, units * split, kThreads, smem_bytes(DP), split, stream, a, row_tiles, page_shift);
}

template <int DP, bool WHOLE>
cudaError_t launch_balanced(const approxifer_attention_args& a, const DeviceInfo& dev, int row_tiles, int page_shift, cudaStream_t stream) {
  auto kernel = attention_token_balanced_kernel<DP, WHOLE>;
  struct Tag {};
  cudaError_t e = ensure_dynamic_smem<Tag>(kernel, dev.ordinal, smem_bytes(DP));
  if (e != cudaSuccess) return e;
  const int ctas = dev.sms * kCtasPerSm;
  float* partial = static_cast<float*>(a.workspace);
  if ((e = launch_kernel(kernel, ctas, kThreads, smem_bytes(DP), 1, stream, a, row_tiles, page_shift, partial)) != cudaSuccess) return e;
  // a unit's share of the runs: one warp joins a few partial results, eight many
  const bool few = units_of(a) * 8 >= (int64_t)ctas * kWarps;
  return launch_kernel(few ? attention_token_join_kernel<DP, 1> : attention_token_join_kernel<DP, kJoinWarps>, (int64_t)a.batch * a.Hq,
                       few ? 32 : kJoinWarps * 32, 0, 1, stream, a, row_tiles, ctas * kWarps, partial);
}

// The balanced form from 96 K positions (times key heads) on.  Measured, cluster against balanced form, us: 8 K positions
// (one sequence of 1,024, 8 heads of 128) 6.8 / 11.3, 64 K 10.5 / 14.7; 128 K: 8 sequences of 2,048 19.9 / 19.2, one of
// 16,384 29.9 / 20.2, 64 of 256 30.7 / 21.2, one of 65,536 with 2 heads of 64 61 / 18; 512 K 82 / 56.
bool wants_balance(const approxifer_attention_args& a) { return units_of(a) * most_seen(a) >= 96 * 1024; }

}  // namespace

bool attention_token_eligible(const approxifer_attention_args& a) {
  return a.max_q == 1 && a.table_pages * a.page_size < (1LL << 31) && a.D % 8 == 0 && a.D <= 128 && aligned16(a.k_cache) && aligned16(a.v_cache) && (reinterpret_cast<uintptr_t>(a.q) & 3) == 0 &&
         (reinterpret_cast<uintptr_t>(a.out) & 3) == 0 && a.q_tstride % 2 == 0 && a.q_hstride % 2 == 0 && a.o_tstride % 2 == 0 && a.o_hstride % 2 == 0 &&
         (a.kc_pstride | a.kc_hstride | a.kc_rstride | a.vc_pstride | a.vc_hstride | a.vc_rstride) % 8 == 0;
}

int64_t attention_token_workspace(const approxifer_attention_args& a) {
  const DeviceInfo* dev;
  if (!wants_balance(a) || current_device_info(&dev) != cudaSuccess) return 0;
  return (int64_t)dev->sms * kCtasPerSm * kWarps * partial_floats(a.D <= 64 ? 64 : 128) * 4;
}

cudaError_t launch_attention_token(const approxifer_attention_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  const cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  const int row_tiles = (a.Hq / a.Hkv + kRows - 1) / kRows;
  const int dp = a.D <= 64 ? 64 : 128, keys = keys_of(dp);
  const int page_shift = exact_log2(a.page_size);  // pages of whole chunks and a power of two: one look-up a chunk
  const bool is_whole = page_shift >= 0 && a.page_size >= keys;
  const int64_t need = attention_token_workspace(a);
  if (need > 0 && a.workspace_bytes >= need && (int64_t)a.batch * a.Hq < (1LL << 31)) {
    auto launch = is_whole ? (dp == 64 ? launch_balanced<64, true> : launch_balanced<128, true>) : dp == 64 ? launch_balanced<64, false> : launch_balanced<128, false>;
    return launch(a, *dev, row_tiles, page_shift, stream);
  }
  // Until there are about four CTAs for every place on the GPU, none with less than two chunks for each warp.
  const int64_t units = units_of(a), most = most_seen(a);
  int split = 1;
  while (split < kMaxSplit && units * split < 4LL * kCtasPerSm * dev->sms && most >= (int64_t)split * 2 * kWarps * keys * 2) split *= 2;
  auto launch = is_whole ? (dp == 64 ? launch_cluster<64, true> : launch_cluster<128, true>) : dp == 64 ? launch_cluster<64, false> : launch_cluster<128, false>;
  return launch(a, *dev, row_tiles, page_shift, units, split, stream);
}

}  // namespace approxifer
