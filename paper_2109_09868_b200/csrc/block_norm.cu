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
// 1,237 tokens of 1,003 in fp32, two layer norms with biases, a gate by elements, 9.7 us (half of it instruction issue, and four meetings a
// row, nearly at the same time in all of them: one row by itself takes 3.5); one token of 4,096 2.9 us.
#include "async.cuh"

namespace approxifer {

__device__ unsigned int g_block_norm_wait_timeouts = 0;

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxStages = 4;
constexpr int kHeader = 384;            // barriers, the sums' meeting place
constexpr int kStaged = 2;              // fours a thread where weights, biases and the gate are copied ahead by the direct form
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

template <int BYTES>
__device__ __forceinline__ void copy_ahead(uint32_t dst, const void* src, int there) {  // `there` bytes of it, then zeros
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there) : "memory");
}
__device__ __forceinline__ void copies_done() {  // (of the warp)
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
}

// How a thread's fours lie in the rows.
enum Access {
  kWhole,     // four neighbours, a row beginning with the first of four at a whole address
  kShifted,   // four neighbours at a whole address in the tokens' rows, which begin anywhere, all arrays' alike: at both ends there may be
              // fewer.  (In weights, and in a gate that is the same for all rows, the four then lie anywhere.)
  kElements,  // four elements a CTA's width apart
};

// The elements `first` (+ 0 .. 3, or + 0 .. 3 times `step`) of a row or of the weights, those that are there: in kElements `count` of them.
template <Access A, bool OF_ROW, typename T>
__device__ __forceinline__ Four<T> load4(const T* p, int first, int step, int count) {
  Four<T> v;
  using Raw = decltype(v.u);
  p += first;
  if constexpr (A == kWhole) {
    v.u = Raw{};
    if (count > 0) v.u = *reinterpret_cast<const Raw*>(p);
  } else {
    T x[4];
    if constexpr (A == kShifted) {
      if (first >= 0 && count >= 4) {
        if constexpr (OF_ROW) {
          v.u = *reinterpret_cast<const Raw*>(p);
          return v;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = p[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < count && first + i >= 0 ? p[i] : narrow<T>(0.f);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = i < count ? p[(int64_t)i * step] : narrow<T>(0.f);
    }
    if constexpr (sizeof(T) == 2) {
      const auto bits = [](bf16 b) { return (uint32_t)__bfloat16_as_ushort(b); };
      v.u = make_uint2(bits(x[0]) | bits(x[1]) << 16, bits(x[2]) | bits(x[3]) << 16);
    } else {
      v.u = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
  return v;
}
// Starts copying them (whole warps) to the thread's own place in shared memory, 16 bytes or, of whole fours of bfloat16, 8.  (Copies are of 4 bytes or
// more: of bfloat16 that lies anywhere the two whole fours that hold the four, which are put together when they are read.)
template <Access A, typename T>
constexpr bool can_copy = sizeof(T) == 4 || A != kElements;
template <Access A, typename T>
constexpr int place_bytes = sizeof(T) == 2 && A == kWhole ? 8 : 16;
template <Access A, bool OF_ROW, typename T>
__device__ __forceinline__ void copy4(unsigned char* place, const T* p, int first, int step, int count) {
  const uint32_t dst = smem_addr(place);
  if (A == kWhole ? count > 0 : A == kShifted && OF_ROW && first >= 0 && count >= 4) {
    copy_ahead<4 * sizeof(T)>(dst, p + first, 4 * sizeof(T));
  } else if constexpr (A == kShifted && OF_ROW) {
    *reinterpret_cast<Four<T>*>(place) = load4<A, OF_ROW, T>(p, first, step, count);
  } else if constexpr (A == kShifted && sizeof(T) == 4) {  // (a warp's fours lie side by side, here and there: its lanes copy neighbours)
    const int lane = threadIdx.x % 32, n = first + count;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int on = 32 * i - 3 * lane, at = first + on;
      const bool there = at >= 0 && at < n;
      copy_ahead<4>(dst + 4 * on, there ? p + at : p, there ? 4 : 0);
    }
  } else if constexpr (A == kElements && sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) copy_ahead<4>(dst + 4 * i, i < count ? p + first + (int64_t)i * step : p, i < count ? 4 : 0);
  } else if constexpr (A == kShifted) {
    const int from = first & ~3, n = first + count;
    if (from >= 0 && from + 8 <= n) {
      copy_ahead<8>(dst, p + from, 8);
      copy_ahead<8>(dst + 8, p + from + 4, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) reinterpret_cast<T*>(place)[i] = from + i >= 0 && from + i < n ? p[from + i] : narrow<T>(0.f);
    }
  }
}
template <Access A, bool OF_ROW, typename T>
__device__ __forceinline__ Four<T> copied4(const unsigned char* place, int first) {
  Four<T> v;
  if constexpr (A == kShifted && !OF_ROW && sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(place);
    const bool far = first & 2;
    const uint32_t x = far ? u.y : u.x, y = far ? u.z : u.y, z = far ? u.w : u.z;
    v.u = make_uint2(__funnelshift_r(x, y, (first & 1) * 16), __funnelshift_r(y, z, (first & 1) * 16));
  } else {
    v.u = *reinterpret_cast<const decltype(v.u)*>(place);
  }
  return v;
}
template <Access A, typename T>
__device__ __forceinline__ void store4(T* p, int first, int step, int count, const float (&v)[4]) {
  p += first;
  if (A == kWhole ? count > 0 : A == kShifted && first >= 0 && count >= 4) {
    if constexpr (sizeof(T) == 2) __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])));
    else __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  } else if constexpr (A != kWhole) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < count && (A == kElements || first + i >= 0)) p[A == kElements ? (int64_t)i * step : i] = narrow<T>(v[i]);
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
template <typename S, typename T, int Q, Access A, bool RING, GateKind GATE, int MOST>
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
  const int mine = A == kElements ? (a.N - lane + L - 1) / L : 0;
  const int shift = A == kShifted ? (int)(reinterpret_cast<uintptr_t>(static_cast<const S*>(a.R) + t * a.r_rstride) / sizeof(S) % 4) : 0;
  auto first = [&](int q) { return A == kElements ? q * 4 * L + lane : (q * L + lane) * 4 - shift; };
  auto there = [&](int q) { return A == kElements ? mine - 4 * q : a.N - first(q); };
  auto holds = [&](int q, int i) { return i < there(q) && (A != kShifted || first(q) + i >= 0); };
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
  auto vector4 = [&](const void* p, int q) { return load4<A, false, T>(static_cast<const T*>(p), first(q), L, there(q)); };
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
  // What is needed only after the first sums is copied to this thread's place in shared memory meanwhile (a row's time is that of its
  // loads after each other), or, where it cannot be, asked for into the cache.
  enum Array { kGateRow, kAfterWeight, kAfterBias, kBeforeWeight, kBeforeBias };
  constexpr bool kStage = !RING && Q == kStaged, kCopy = kStage && can_copy<A, T>;
  auto place = [&](int array, int q) {
    return smem + kHeader + ((array * Q + q) * (blockDim.x * blockDim.y) + threadIdx.y * blockDim.x + threadIdx.x) * place_bytes<A, T>;
  };
  if constexpr (!RING) {
    auto ask = [&](auto of_row, int array, const T* from) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if constexpr (kCopy) {
          copy4<A, decltype(of_row)::value, T>(place(array, q), from, first(q), L, there(q));
        } else {
#pragma unroll
          for (int i = 0; i < (A == kElements ? 4 : 1); ++i)
            if (holds(q, i)) asm volatile("prefetch.global.L1 [%0];" ::"l"(from + first(q) + i * L));
        }
      }
    };
    auto rest = [&](int array, const void* p) {
      if (p) ask(std::false_type{}, array, static_cast<const T*>(p));
    };
    if (t < a.T) {
      if (GATE != kGateNone && a.g_cstride) ask(std::bool_constant<GATE == kGateRows>{}, kGateRow, G + t * a.g_rstride);
      rest(kAfterWeight, a.after_weight), rest(kAfterBias, a.after_bias), rest(kBeforeWeight, a.before_weight), rest(kBeforeBias, a.before_bias);
    }
  }
  // Of weights and biases.
  auto again = [&](int array, const void* p, int q) {
    if constexpr (kCopy) return copied4<A, false, T>(place(array, q), first(q));
    else return vector4(p, q);
  };
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
        rv[q] = load4<A, true, S>(R, first(q), L, there(q));
        if (a.Y) yv[q] = load4<A, true, T>(Y, first(q), L, there(q));
        if constexpr (GATE == kGateRows && RING)
          if (a.g_cstride) gv[q] = load4<A, true, T>(g, first(q), L, there(q));
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
    auto norm = [&](int kind, float (&x)[Q][4], int weights, const void* w, Four<T> (&held)[Q], const void* b) {
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
          for (int i = 0; i < 4; ++i) x[q][i] = holds(q, i) ? x[q][i] - mean : 0.f;
      }
      float sq = 0.f;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) sq = fmaf(x[q][i], x[q][i], sq);
      const float k = rsqrtf(row.sum(sq) * inv_n + a.eps);
      if constexpr (kCopy) copies_done();
#pragma unroll
      for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[q][i] *= k;
        if (w) {
          if (!kHold) held[q] = again(weights, w, q);
          held[q].pin();
#pragma unroll
          for (int i = 0; i < 4; ++i) x[q][i] *= held[q].at(i);
        }
        if (b) {
          const Four<T> v = again(weights + 1, b, q);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[q][i] += v.at(i);
        }
      }
    };
    if (a.Y) {
      norm(a.after, x, kAfterWeight, a.after_weight, aw, a.after_bias);
      S* out = static_cast<S*>(a.R_out) + t * a.ro_rstride;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if constexpr (GATE != kGateNone && !RING) {
          if (a.g_cstride) {
            Four<T> v;
            if constexpr (kCopy) copies_done(), v = copied4<A, GATE == kGateRows, T>(place(kGateRow, q), first(q));
            else v = load4<A, GATE == kGateRows, T>(G + t * a.g_rstride, first(q), L, there(q));
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
          res[q][i] = holds(q, i) ? fmaf(a.block_scale, u, a.residual_scale * res[q][i]) : 0.f;
        }
        store4<A, S>(out, first(q), L, there(q), res[q]);
      }
    }
    if (a.before != APPROXIFER_NORM_NONE) {
      norm(a.before, res, kBeforeWeight, a.before_weight, bw, a.before_bias);
      T* out = static_cast<T*>(a.X) + t * a.x_rstride;
#pragma unroll
      for (int q = 0; q < Q; ++q) store4<A, T>(out, first(q), L, there(q), res[q]);
    }
  };
  if constexpr (!RING) {
    if (t < a.T) one_row();
    if constexpr (kCopy) copies_done();  // (weights of a norm that is not asked for)
  } else {
    for (; t < a.T; t += step) one_row();
    __syncthreads();
    drain_if_aborted(abort);
  }
}

// (Narrow rows: registers for ten CTAs of 128 threads on an SM.)
template <typename S, typename T, int Q, Access A, bool RING, int MOST = kMaxThreads>
cudaError_t launch_kind(const approxifer_block_norm_args& a, const DeviceInfo& dev, int64_t ctas, dim3 block, int smem, int stages, cudaStream_t stream) {
  auto launch = [&](auto kernel, auto tag) {
    const cudaError_t e = ensure_dynamic_smem<decltype(tag)>(kernel, dev.ordinal, smem);
    return e != cudaSuccess ? e : launch_kernel(kernel, dim3((unsigned)ctas), block, smem, 1, stream, a, stages);
  };
  struct None {};
  struct Columns {};
  struct Rows {};
  if (a.gate == nullptr) return launch(block_norm_kernel<S, T, Q, A, RING, kGateNone, MOST>, None{});
  if (a.g_rstride == 0 && a.g_cstride == 1) return launch(block_norm_kernel<S, T, Q, A, RING, kGateColumns, MOST>, Columns{});
  return launch(block_norm_kernel<S, T, Q, A, RING, kGateRows, MOST>, Rows{});
}

template <typename S, typename T>
cudaError_t launch_types(const approxifer_block_norm_args& a, const DeviceInfo& dev, cudaStream_t stream) {
  auto whole = [](const void* p, int64_t stride, int size) { return aligned16(p) && stride % (16 / size) == 0; };
  const bool each = a.gate && a.g_cstride != 0;  // a gate by elements
  const bool vec = a.N % 8 == 0 && whole(a.R, a.r_rstride, sizeof(S)) && whole(a.Y, a.Y ? a.y_rstride : 0, sizeof(T)) &&
                   (!each || whole(a.gate, a.g_rstride, sizeof(T))) && aligned16(a.after_weight) && aligned16(a.after_bias) && aligned16(a.before_weight) &&
                   aligned16(a.before_bias) && whole(a.R_out, a.Y ? a.ro_rstride : 0, sizeof(S)) && whole(a.X, a.before ? a.x_rstride : 0, sizeof(T));
  // rows of other lengths or strides: those of all arrays as far from a whole address, and a thread to each four that they touch
  auto shift = [&](const void* p, int64_t t, int64_t stride, int size) { return (reinterpret_cast<uintptr_t>(p) / size + t * (uint64_t)stride) % 4; };
  auto alike = [&](const void* p, int64_t stride, int size) {
    return p == nullptr || (shift(p, 0, stride, size) == shift(a.R, 0, a.r_rstride, sizeof(S)) && (a.T == 1 || shift(p, 1, stride, size) == shift(a.R, 1, a.r_rstride, sizeof(S))));
  };
  // (weights, and a gate that is the same for all rows: 8 bytes of bfloat16 are copied at a time)
  auto copies = [&](const void* p) { return sizeof(T) == 4 || aligned8(p); };
  const bool weights = copies(a.after_weight) && copies(a.after_bias) && copies(a.before_weight) && copies(a.before_bias) && (!each || a.g_rstride != 0 || copies(a.gate));
  const bool shifted = !vec && weights && a.N + 3 <= 16 * kMaxThreads && alike(a.Y, a.y_rstride, sizeof(T)) && alike(a.Y ? a.R_out : nullptr, a.ro_rstride, sizeof(S)) &&
                       alike(a.before ? a.X : nullptr, a.x_rstride, sizeof(T)) && (!each || a.g_rstride == 0 || alike(a.gate, a.g_rstride, sizeof(T)));
  const int width = shifted ? a.N + 3 : a.N;
  // Eight elements a thread as long as a CTA has the threads for it; of more rows than SMs that do not go over the ring sixteen, for
  // more and smaller CTAs to an SM.  Measured, eight against sixteen, us: 9,000 rows of 4,099, fp32, layer norms, a gate, 348 / 184, of 5,003
  // in bfloat16 393 / 188, of 2,051 115 / 98; 20 rows of 4,099 6.4 / 7.6.
  const int fours = width <= (vec || a.T <= dev.sms ? 8 * kMaxThreads : 8 * 256) ? 2 : 4;
  const int threads = ((width + 4 * fours - 1) / (4 * fours) + 31) / 32 * 32;
  if (vec && fours == 2 && threads > 32) {
    const int64_t stage = (int64_t)a.N * (sizeof(S) + (a.Y ? sizeof(T) : 0) + (each && a.g_rstride != 0 ? sizeof(T) : 0));
    const int by_threads = kMaxThreads / threads;  // (64 registers a thread)
    const int stages = (int)(kRingBytes / by_threads / stage < kMaxStages ? kRingBytes / by_threads / stage : kMaxStages);
    const int64_t fit = (int64_t)dev.sms * by_threads, turns = (a.T + fit - 1) / fit;
    // The ring's start costs what two or three rows do.  Narrow rows, of which an SM holds many CTAs, hide their loads without it, all
    // the more where a gate by elements takes its registers.  Measured, ring against direct, us: 300 rows of 4,096 (2 turns), rms norms,
    // 5.9 / 5.3, 600 with a gate by columns (3 turns) 9.3 / 10.0, 16,384 133 / 218; 300 of 8,192 7.9 / 9.6; of 1,024, layer norms and a gate by
    // elements, 1,300 (2 turns) 10.3 / 7.1, 30,000 119 / 104, rms norms and a gate by columns 62 / 81; 5,000 of 264 (3 turns) 8.9 / 7.3.
    const bool narrow = threads <= 128;
    const int64_t least = threads > 512 ? 2 : narrow ? 8 : 3;
    if (stages >= 2 && turns >= least && !(narrow && each))
      return launch_kind<S, T, 2, kWhole, true>(a, dev, (a.T + turns - 1) / turns, dim3(threads), kHeader + (int)(stages * stage), stages, stream);  // (turns of equal length)
  }
  const int rows = threads == 32 ? 4 : 1;
  const dim3 block(threads, rows);
  const int64_t ctas = (a.T + rows - 1) / rows;
  auto direct = [&](auto access) {
    constexpr Access A = decltype(access)::value;
    const int smem = kHeader + (fours == kStaged && can_copy<A, T> ? 5 * kStaged * place_bytes<A, T> * threads * rows : 0);
    if (fours == 2 && threads * rows <= 128) return launch_kind<S, T, 2, A, false, 128>(a, dev, ctas, block, smem, 0, stream);
    return fours == 2 ? launch_kind<S, T, 2, A, false>(a, dev, ctas, block, smem, 0, stream) : launch_kind<S, T, 4, A, false>(a, dev, ctas, block, smem, 0, stream);
  };
  return vec ? direct(std::integral_constant<Access, kWhole>{}) : shifted ? direct(std::integral_constant<Access, kShifted>{}) : direct(std::integral_constant<Access, kElements>{});
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
