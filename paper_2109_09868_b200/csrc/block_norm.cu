// What lies between two blocks of a layer, in one pass over the tokens: norm of a block's output, gate, residual, norm before
// the next block.
//
//     u = norm_after(y),   r' = a r + b act(g) u,   x = norm_before(r')
//
// A row (token) is held in registers from its loads to its stores, in fours of neighbours that lie a CTA's width apart, so that
// each array crosses HBM once, in whole lines: its bound.  The sums of a norm are taken over the row's threads by shuffles and,
// across warps, one meeting in shared memory; the mean of a layer norm is subtracted before the squares are summed (no
// cancellation).
//
//   ring     many rows: CTAs stay and take rows in turn; the next rows are copied into shared memory (bulk copies) while this
//            one is worked on, and weights and a gate that is the same for all rows are read once for all of them
//   direct   few rows, rows that are not whole 16 bytes, or too long for two of them in shared memory: loads straight into
//            registers, a CTA (up to 256 elements a warp) to a row
//
// Measured: 16,384 tokens of 4,096, stream in fp32, gate by columns, 133 us, 6.1 TB/s, from a graph, 145 us, 5.5 TB/s, call after call;
// 1,237 tokens of 1,003 in fp32, two layer norms with biases, a gate by elements, 11 us (bound by the issue of 4-byte accesses: 53 %, and
// four meetings a row); one token of 4,096 3.9 us, two meetings after its loads.
#include "async.cuh"

namespace approxifer {

__device__ unsigned int g_block_norm_wait_timeouts = 0;

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxStages = 4;
constexpr int kHeader = 384;            // barriers, the sums' meeting place
constexpr int kRingBytes = 200 * 1024;  // of an SM's shared memory, for all its CTAs

// Four elements of type T, as they are loaded.
template <typename T>
struct Four;
template <>
struct Four<bf16> {
  uint2 u;
  __device__ __forceinline__ float at(int i) const {
    const uint32_t w = i < 2 ? u.x : u.y;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ __forceinline__ void pin() { asm volatile("" : "+r"(u.x), "+r"(u.y)); }  // (keeps the compiler from widening it ahead of a loop)
};
template <>
struct Four<float> {
  float4 u;
  __device__ __forceinline__ float at(int i) const { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }
  __device__ __forceinline__ void pin() {}
};

// VEC: four neighbours.  Else: four elements `step` apart, of which `count` are there.
template <bool VEC, typename T>
__device__ __forceinline__ Four<T> load4(const T* p, int step, int count) {
  Four<T> v;
  if constexpr (VEC) {
    using Raw = decltype(v.u);
    v.u = Raw{};
    if (count > 0) v.u = *reinterpret_cast<const Raw*>(p);
  } else {
    T x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < count ? p[(int64_t)i * step] : narrow<T>(0.f);
    if constexpr (sizeof(T) == 2) {
      const auto bits = [](bf16 b) { return (uint32_t)__bfloat16_as_ushort(b); };
      v.u = make_uint2(bits(x[0]) | bits(x[1]) << 16, bits(x[2]) | bits(x[3]) << 16);
    } else {
      v.u = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
  return v;
}
template <bool VEC, typename T>
__device__ __forceinline__ void store4(T* p, int step, int count, const float (&v)[4]) {
  if constexpr (VEC) {
    if (count <= 0) return;
    if constexpr (sizeof(T) == 2) __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])));
    else __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < count) p[(int64_t)i * step] = narrow<T>(v[i]);
  }
}

__device__ __forceinline__ float gate_of(int act, float x) {
  if (act == APPROXIFER_GATE_SIGMOID) return __fdividef(1.f, 1.f + expf(-x));  // (a division of two units' error; 1 / infinity is 0)
  if (act == APPROXIFER_GATE_TANH) return tanhf(x);
  return x;
}

// Sum over the row's threads.  `room`: two sets of a float a warp, used in turn, so that one meeting a sum is enough.
struct Row {
  float* room;
  int set, warps;
  __device__ __forceinline__ float sum(float v) {
    v = warp_sum(v);
    if (warps == 1) return v;
    const int lane = threadIdx.x % 32;
    float* at = room + (set ^= 32);
    if (lane == 0) at[threadIdx.x / 32] = v;
    __syncthreads();
    return warp_sum(lane < warps ? at[lane] : 0.f);
  }
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

enum GateKind { kGateNone, kGateColumns, kGateRows };  // one row for all tokens; a row, or a value, for each

// Q fours of elements a thread.  Elements that are not there are zero and stay out of the sums.
template <typename S, typename T, int Q, bool VEC, bool RING, GateKind GATE, int MOST>
__global__ void __launch_bounds__(MOST, MOST == kMaxThreads ? 1 : 10) block_norm_kernel(const __grid_constant__ approxifer_block_norm_args a, int stages) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr bool kHold = RING;  // weights and gate stay in registers
  const int L = blockDim.x, lane = threadIdx.x;  // threads to a row
  Row row{reinterpret_cast<float*>(smem + 128), 0, L / 32};
  volatile int* abort = reinterpret_cast<volatile int*>(smem + 120);
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const T* G = static_cast<const T*>(a.gate);
  // this thread's fours: the first element, how many there are
  const int mine = VEC ? 0 : (a.N - lane + L - 1) / L;
  auto first = [&](int q) { return VEC ? (q * L + lane) * 4 : q * 4 * L + lane; };
  auto there = [&](int q) { return VEC ? a.N - first(q) : mine - 4 * q; };
  const float inv_n = 1.f / (float)a.N;
  // (ring) a stage: a row of R, of Y, of the gate
  const uint32_t r_bytes = a.N * sizeof(S), y_bytes = a.Y ? a.N * sizeof(T) : 0, g_bytes = GATE == kGateRows && a.g_cstride ? a.N * sizeof(T) : 0;
  const uint32_t stage_bytes = r_bytes + y_bytes + g_bytes, bars = smem_addr(smem);
  unsigned char* ring = smem + kHeader;
  auto copy_row = [&](int s, int64_t t) {
    const uint32_t to = smem_addr(ring) + s * stage_bytes, bar = bars + 8 * s;
    bar_expect(bar, stage_bytes);
    bulk_copy(to, static_cast<const S*>(a.R) + t * a.r_rstride, r_bytes, bar);
    if (y_bytes) bulk_copy(to + r_bytes, static_cast<const T*>(a.Y) + t * a.y_rstride, y_bytes, bar);
    if (g_bytes) bulk_copy(to + r_bytes + y_bytes, G + t * a.g_rstride, g_bytes, bar);
  };
  let_next_start();
  if constexpr (RING) {
    if (threadIdx.x == 0) {
      for (int s = 0; s < stages; ++s) bar_init(bars + 8 * s, 1);
      *abort = 0;
      bar_init_done();
    }
    __syncthreads();
  }
  wait_for_inputs();
  if (RING && threadIdx.x == 0)
    for (int s = 0; s < stages && t + s * step < a.T; ++s) copy_row(s, t + s * step);

  Four<T> aw[Q], bw[Q];
  float gate[Q][4];
  auto vector4 = [&](const void* p, int q) { return load4<VEC, T>(static_cast<const T*>(p) + first(q), L, there(q)); };
  if constexpr (kHold) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (a.after_weight) aw[q] = vector4(a.after_weight, q);
      if (a.before_weight) bw[q] = vector4(a.before_weight, q);
      if constexpr (GATE == kGateColumns) {
        const Four<T> v = vector4(G, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) gate[q][i] = gate_of(a.gate_activation, v.at(i));
      }
    }
  }
  if constexpr (!RING) {
    // What is needed only after the first sums is asked for now, into the cache: a row's time is that of its loads after each other.
    auto ask = [&](const void* p, int64_t at) {
      const T* from = static_cast<const T*>(p) + at;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < (VEC ? 1 : 4); ++i)
          if (there(q) > i) asm volatile("prefetch.global.L1 [%0];" ::"l"(from + first(q) + i * L));
    };
    if (t < a.T) {
      if (GATE != kGateNone && a.g_cstride) ask(G, t * a.g_rstride);
      if (a.after_weight) ask(a.after_weight, 0);
      if (a.after_bias) ask(a.after_bias, 0);
      if (a.before_weight) ask(a.before_weight, 0);
      if (a.before_bias) ask(a.before_bias, 0);
    }
  }
  int turn = 0, s = 0;
  auto one_row = [&]() {
    float x[Q][4], res[Q][4], one = 1.f;
    {
      const S* R = static_cast<const S*>(a.R) + t * a.r_rstride;
      const T *Y = static_cast<const T*>(a.Y) + t * a.y_rstride, *g = G + t * a.g_rstride;
      if constexpr (RING) {
        bar_wait(bars + 8 * s, turn & 1, abort, &g_block_norm_wait_timeouts);
        R = reinterpret_cast<const S*>(ring + s * stage_bytes);
        Y = reinterpret_cast<const T*>(ring + s * stage_bytes + r_bytes), g = reinterpret_cast<const T*>(ring + s * stage_bytes + r_bytes + y_bytes);
      }
      Four<S> rv[Q];
      Four<T> yv[Q], gv[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        rv[q] = load4<VEC, S>(R + first(q), L, there(q));
        if (a.Y) yv[q] = load4<VEC, T>(Y + first(q), L, there(q));
        if constexpr (GATE == kGateRows && RING)
          if (a.g_cstride) gv[q] = load4<VEC, T>(g + first(q), L, there(q));
      }
      if constexpr (GATE == kGateRows) {
        if (!a.g_cstride) one = gate_of(a.gate_activation, widen(G[t * a.g_rstride]));
        if constexpr (RING) {
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) gate[q][i] = a.g_cstride ? gate_of(a.gate_activation, gv[q].at(i)) : one;
        }
      }
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) res[q][i] = rv[q].at(i), x[q][i] = a.Y ? yv[q].at(i) : 0.f;
      if constexpr (RING) {
        __syncthreads();  // the stage has been read
        if (threadIdx.x == 0 && t + stages * step < a.T) copy_row(s, t + stages * step);
        if (++s == stages) s = 0, ++turn;
      }
    }
    auto norm = [&](int kind, float (&x)[Q][4], const void* w, Four<T> (&held)[Q], const void* b) {
      if (kind == APPROXIFER_NORM_NONE) return;
      if (kind == APPROXIFER_NORM_LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += x[q][i];
        const float mean = row.sum(sum) * inv_n;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[q][i] = i < there(q) ? x[q][i] - mean : 0.f;
      }
      float sq = 0.f;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) sq = fmaf(x[q][i], x[q][i], sq);
      const float k = rsqrtf(row.sum(sq) * inv_n + a.eps);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[q][i] *= k;
        if (w) {
          if (!kHold) held[q] = vector4(w, q);
          held[q].pin();
#pragma unroll
          for (int i = 0; i < 4; ++i) x[q][i] *= held[q].at(i);
        }
        if (b) {
          const Four<T> v = vector4(b, q);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[q][i] += v.at(i);
        }
      }
    };
    if (a.Y) {
      norm(a.after, x, a.after_weight, aw, a.after_bias);
      S* out = static_cast<S*>(a.R_out) + t * a.ro_rstride;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if constexpr (GATE != kGateNone && !RING) {
          if (a.g_cstride) {
            const Four<T> v = vector4(G + t * a.g_rstride, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) gate[q][i] = gate_of(a.gate_activation, v.at(i));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) gate[q][i] = one;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = GATE == kGateNone ? x[q][i] : x[q][i] * gate[q][i];
          res[q][i] = i < there(q) ? fmaf(a.block_scale, u, a.residual_scale * res[q][i]) : 0.f;
        }
        store4<VEC, S>(out + first(q), L, there(q), res[q]);
      }
    }
    if (a.before != APPROXIFER_NORM_NONE) {
      norm(a.before, res, a.before_weight, bw, a.before_bias);
      T* out = static_cast<T*>(a.X) + t * a.x_rstride;
#pragma unroll
      for (int q = 0; q < Q; ++q) store4<VEC, T>(out + first(q), L, there(q), res[q]);
    }
  };
  if constexpr (!RING) {
    if (t < a.T) one_row();
  } else {
    for (; t < a.T; t += step) one_row();
    __syncthreads();
    drain_if_aborted(abort);
  }
}

// (Narrow rows: registers for ten CTAs of 128 threads on an SM.)
template <typename S, typename T, int Q, bool VEC, bool RING, int MOST = kMaxThreads>
cudaError_t launch_kind(const approxifer_block_norm_args& a, const DeviceInfo& dev, int64_t ctas, dim3 block, int smem, int stages, cudaStream_t stream) {
  auto launch = [&](auto kernel, auto tag) {
    const cudaError_t e = ensure_dynamic_smem<decltype(tag)>(kernel, dev.ordinal, smem);
    return e != cudaSuccess ? e : launch_kernel(kernel, dim3((unsigned)ctas), block, smem, 1, stream, a, stages);
  };
  struct None {};
  struct Columns {};
  struct Rows {};
  if (a.gate == nullptr) return launch(block_norm_kernel<S, T, Q, VEC, RING, kGateNone, MOST>, None{});
  if (a.g_rstride == 0 && a.g_cstride == 1) return launch(block_norm_kernel<S, T, Q, VEC, RING, kGateColumns, MOST>, Columns{});
  return launch(block_norm_kernel<S, T, Q, VEC, RING, kGateRows, MOST>, Rows{});
}

template <typename S, typename T>
cudaError_t launch_types(const approxifer_block_norm_args& a, const DeviceInfo& dev, cudaStream_t stream) {
  auto whole = [](const void* p, int64_t stride, int size) { return aligned16(p) && stride % (16 / size) == 0; };
  const bool each = a.gate && a.g_cstride != 0;  // a gate by elements
  const bool vec = a.N % 8 == 0 && whole(a.R, a.r_rstride, sizeof(S)) && whole(a.Y, a.Y ? a.y_rstride : 0, sizeof(T)) &&
                   (!each || whole(a.gate, a.g_rstride, sizeof(T))) && aligned16(a.after_weight) && aligned16(a.after_bias) && aligned16(a.before_weight) &&
                   aligned16(a.before_bias) && whole(a.R_out, a.Y ? a.ro_rstride : 0, sizeof(S)) && whole(a.X, a.before ? a.x_rstride : 0, sizeof(T));
  // eight elements a thread as long as a CTA has the threads for it
  const int fours = a.N <= 8 * kMaxThreads ? 2 : 4;
  const int threads = ((a.N + 4 * fours - 1) / (4 * fours) + 31) / 32 * 32;
  if (vec && fours == 2 && threads > 32) {
    const int64_t stage = (int64_t)a.N * (sizeof(S) + (a.Y ? sizeof(T) : 0) + (each && a.g_rstride != 0 ? sizeof(T) : 0));
    const int by_threads = kMaxThreads / threads;  // (64 registers a thread)
    const int stages = (int)(kRingBytes / by_threads / stage < kMaxStages ? kRingBytes / by_threads / stage : kMaxStages);
    const int64_t fit = (int64_t)dev.sms * by_threads, turns = (a.T + fit - 1) / fit;
    if (stages >= 2 && turns >= 2)
      return launch_kind<S, T, 2, true, true>(a, dev, (a.T + turns - 1) / turns, dim3(threads), kHeader + (int)(stages * stage), stages, stream);  // (turns of equal length)
  }
  const int rows = threads == 32 ? 4 : 1;
  const dim3 block(threads, rows);
  const int64_t ctas = (a.T + rows - 1) / rows;
  if (fours == 2 && threads * rows <= 128)
    return vec ? launch_kind<S, T, 2, true, false, 128>(a, dev, ctas, block, kHeader, 0, stream) : launch_kind<S, T, 2, false, false, 128>(a, dev, ctas, block, kHeader, 0, stream);
  if (fours == 2) return vec ? launch_kind<S, T, 2, true, false>(a, dev, ctas, block, kHeader, 0, stream) : launch_kind<S, T, 2, false, false>(a, dev, ctas, block, kHeader, 0, stream);
  return vec ? launch_kind<S, T, 4, true, false>(a, dev, ctas, block, kHeader, 0, stream) : launch_kind<S, T, 4, false, false>(a, dev, ctas, block, kHeader, 0, stream);
}

}  // namespace

cudaError_t read_block_norm_wait_timeouts(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_block_norm_wait_timeouts, sizeof(*out)); }
cudaError_t reset_block_norm_wait_timeouts() {
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_block_norm_wait_timeouts, &zero, sizeof(zero));
}

cudaError_t launch_block_norm(const approxifer_block_norm_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  const cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  if (a.stream_type == APPROXIFER_TYPE_F32) return a.type == APPROXIFER_TYPE_F32 ? launch_types<float, float>(a, *dev, stream) : launch_types<float, bf16>(a, *dev, stream);
  return a.type == APPROXIFER_TYPE_F32 ? launch_types<bf16, float>(a, *dev, stream) : launch_types<bf16, bf16>(a, *dev, stream);
}

}  // namespace approxifer
