// Matrix product with bias, activation and residual for many tiles: persistent pairs of CTAs, each pair one 256 x 256 tile
// of Y at a time (tcgen05 with cta_group::2: every CTA keeps 128 rows of X and half of the tile's rows of Wt in shared
// memory, the two tensor cores read both halves), accumulators double-buffered in tensor memory, so that the epilogue of a
// tile runs under the products of the next.
//
//   warp 0      one lane: tensor-map copies of this CTA's operands, five stages of 64 columns (32 KB) in flight
//   warp 1      of the pair's first CTA: tcgen05.mma for the pair; allocates the tensor memory
//   warps 2, 3  idle (the accumulator's lanes belong to warps by their index modulo 4)
//   warps 4-11  epilogue: two warps to each quarter of the lanes, half of the columns each; bias, activation, residual,
//               one rounding.  A thread has one row of the accumulator; through 4 KB of shared memory a warp turns 32 of
//               its columns so that eight lanes write, or read of the residual, a row's piece together (a store of 32
//               rows takes 32 passes; with short K the epilogue is all that is seen)
//
// Bound by the tensor cores, for seconds on end by the power limit.  Measured: 8,192 x 16,384 x 4,096 with bias and gelu
// 709 us, 1,551 TFLOP/s (1,619 is what a library product of 8,192^3 reaches); repeated for a second 817 to 872 us, 1.26 to 1.35
// PFLOP/s, with the SM clock.  With K = 64 (130 us) the epilogue is what is left.
#include "async.cuh"

namespace approxifer {

__device__ unsigned int g_linear_pair_wait_timeouts = 0;

namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kTileM = 256, kTileN = 256, kDepth = 64;
constexpr int kStages = 5;
constexpr int kTurnBytes = 32 * 32 * 4;           // of an epilogue warp
constexpr int kHalfBytes = 128 * kDepth * 2;      // one operand of one CTA per stage
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kHeader = 1024;
constexpr int kSmemBytes = kHeader + 1024 + kStages * kStageBytes + kEpilogueWarps * kTurnBytes;
constexpr int kTmemCols = 512;
constexpr int kGroupM = 8;  // rows of tiles that are walked together: their X stays in L2 while Wt streams by

struct PairArgs {
  int32_t M, N, K, steps, tiles_m, tiles_n, tiles;
  const bf16* bias;
  const void* R;
  void* Y;
  int64_t r_rstride, y_rstride;
  int32_t vec;  // Y and R can be accessed four elements at a time
};

// Tiles in bands of kGroupM rows of tiles, down a band's columns of tiles.
__device__ __forceinline__ void place(const PairArgs& a, int tile, int* m0, int* n0) {
  const int per_band = kGroupM * a.tiles_n, band = tile / per_band, in = tile - band * per_band;
  const int rows = min(kGroupM, a.tiles_m - band * kGroupM);
  *m0 = (band * kGroupM + in % rows) * kTileM;
  *n0 = (in / rows) * kTileN;
}

// Rows m0 .. m0+31 and columns n .. n+31: v is this lane's row of the accumulator.
template <typename Out, int ACT>
__device__ __forceinline__ void finish32(const PairArgs& a, int m0, int n, const uint32_t (&v)[32], float4* turn, int lane) {
  __syncwarp();  // the last piece has been read
#pragma unroll
  for (int j = 0; j < 8; ++j)
    turn[lane * 8 + (j ^ (lane & 7))] =
        make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3]));
  __syncwarp();
  const int col = n + (lane % 8) * 4;
  if (col >= a.N) return;
  const bool vec = a.vec && col + 4 <= a.N;
  float b[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < a.N) b[i] = widen(a.bias[col + i]);
  }
  const int left = a.M - m0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = i * 4 + lane / 8;
    if (row >= left) break;
    const float4 x = turn[row * 8 + ((lane % 8) ^ (row & 7))];
    float z[4] = {activate<ACT, Out>(x.x + b[0]), activate<ACT, Out>(x.y + b[1]), activate<ACT, Out>(x.z + b[2]), activate<ACT, Out>(x.w + b[3])};
    Out* y = static_cast<Out*>(a.Y) + (int64_t)(m0 + row) * a.y_rstride + col;
    const Out* r = a.R ? static_cast<const Out*>(a.R) + (int64_t)(m0 + row) * a.r_rstride + col : nullptr;
    if (vec) {
      if constexpr (sizeof(Out) == 2) {
        if (r) {
          const uint2 q = *reinterpret_cast<const uint2*>(r);
          z[0] += __uint_as_float(q.x << 16), z[1] += __uint_as_float(q.x & 0xffff0000u), z[2] += __uint_as_float(q.y << 16), z[3] += __uint_as_float(q.y & 0xffff0000u);
        }
        *reinterpret_cast<uint2*>(y) = make_uint2(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]));
      } else {
        if (r) {
          const float4 q = *reinterpret_cast<const float4*>(r);
          z[0] += q.x, z[1] += q.y, z[2] += q.z, z[3] += q.w;
        }
        *reinterpret_cast<float4*>(y) = make_float4(z[0], z[1], z[2], z[3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.N) y[e] = narrow<Out>(r ? z[e] + widen(r[e]) : z[e]);
    }
  }
}

template <typename Out, int ACT>
__global__ void __launch_bounds__(kThreads, 1)
    linear_pair_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ PairArgs a) {
  extern __shared__ unsigned char raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(base);  // full[stages], empty[stages], ready[2], free[2]
  volatile int* abort = reinterpret_cast<volatile int*>(base + 512);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base + 516);
  const uint32_t stages = smem_addr(base + kHeader);
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, drained = ready + 16;
  const int warp = warp_index(), lane = threadIdx.x % 32;
  const int rank = (int)cluster_rank();
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  unsigned int* count = &g_linear_pair_wait_timeouts;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) bar_init(full + 8 * s, 1), bar_init(empty + 8 * s, 1);
    for (int s = 0; s < 2; ++s) bar_init(ready + 8 * s, 1), bar_init(drained + 8 * s, 2 * kEpilogueWarps);
    *abort = 0;
    bar_init_done();
    prefetch_map(&x_map);
    prefetch_map(&w_map);
  }
  if (warp == 1) tmem_alloc_pair(smem_addr(tmem_slot), kTmemCols);
  tmem_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers stand before any is signalled from the other
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  let_next_start();  // not before: the tensor memory is held
  wait_for_inputs();

  if (warp == 0 && lane == 0) {
    int it = 0;
    bool ok = true;
    for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
      int m0, n0;
      place(a, tile, &m0, &n0);
      m0 += rank * 128, n0 += rank * 128;
      for (int k = 0; k < a.steps; ++k, ++it) {
        const int s = it % kStages, turn = it / kStages;
        if (turn > 0 && !(ok = bar_wait(empty + 8 * s, (turn - 1) & 1, abort, count))) break;
        if (rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);  // both CTAs' copies count on the first one's barrier
        const uint32_t bar = peer_smem(full + 8 * s, 0), dst = stages + s * kStageBytes;
        tma_2d_pair(dst, &x_map, k * kDepth, m0, bar);
        tma_2d_pair(dst + kHalfBytes, &w_map, k * kDepth, n0, bar);
      }
    }
  } else if (warp == 1 && rank == 0) {
    int it = 0, n = 0;
    bool ok = true;
    for (int tile = pair; tile < a.tiles && ok; tile += pairs, ++n) {
      const int acc = n & 1;
      if (n >= 2 && !(ok = warp_wait(drained + 8 * acc, (n / 2 - 1) & 1, abort, count))) break;
      tmem_fence_after();
      for (int k = 0; k < a.steps; ++k, ++it) {
        const int s = it % kStages, turn = it / kStages;
        if (!(ok = warp_wait(full + 8 * s, turn & 1, abort, count))) break;
        tmem_fence_after();
        const uint32_t src = stages + s * kStageBytes;
        const uint64_t da = desc_k_major(src), db = desc_k_major(src + kHalfBytes);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < kDepth / 16; ++j) mma_ss_pair(tmem + acc * kTileN, da + 2 * j, db + 2 * j, mma_shape(kTileM, kTileN), k > 0 || j > 0);
          mma_commit_pair(empty + 8 * s);
        }
        __syncwarp();
      }
      if (ok && elect_one()) mma_commit_pair(ready + 8 * acc);
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int q = warp % 4, half = (warp - 4) / 4;
    int n = 0;
    for (int tile = pair; tile < a.tiles; tile += pairs, ++n) {
      const int acc = n & 1;
      int m0, n0;
      place(a, tile, &m0, &n0);
      if (!warp_wait(ready + 8 * acc, (n / 2) & 1, abort, count)) break;
      tmem_fence_after();
      float4* turn = reinterpret_cast<float4*>(base + kHeader + kStages * kStageBytes + (warp - 4) * kTurnBytes);
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + acc * kTileN + half * (kTileN / 2);
#pragma unroll 1
      for (int c = 0; c < kTileN / 2; c += 32) {
        uint32_t v[32];
        tmem_ld32(from + c, v);
        tmem_wait_ld(v);
        if (c + 32 == kTileN / 2) {  // the accumulator has been read
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(peer_smem(drained + 8 * acc, 0));
        }
        finish32<Out, ACT>(a, m0 + rank * 128 + q * 32, n0 + half * (kTileN / 2) + c, v, turn, lane);
      }
    }
  }
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  drain_if_aborted(abort);
  cluster_sync();  // neither CTA leaves while the other's copies, products or arrivals may still reach it
  tmem_fence_after();
  if (warp == 1) tmem_free_pair(tmem, kTmemCols);
}

template <typename Out, int ACT>
cudaError_t launch_act(const PairArgs& t, const CUtensorMap& x, const CUtensorMap& w, const DeviceInfo& dev, cudaStream_t stream) {
  auto kernel = linear_pair_kernel<Out, ACT>;
  struct Tag {};
  const cudaError_t e = ensure_dynamic_smem<Tag>(kernel, dev.ordinal, kSmemBytes);
  if (e != cudaSuccess) return e;
  const int pairs = t.tiles < dev.sms / 2 ? t.tiles : dev.sms / 2;
  return launch_kernel(kernel, 2 * pairs, kThreads, kSmemBytes, 2, stream, x, w, t);
}

template <typename Out>
cudaError_t launch_out(int act, const PairArgs& t, const CUtensorMap& x, const CUtensorMap& w, const DeviceInfo& dev, cudaStream_t stream) {
  switch (act) {
    case APPROXIFER_ACT_RELU: return launch_act<Out, APPROXIFER_ACT_RELU>(t, x, w, dev, stream);
    case APPROXIFER_ACT_GELU: return launch_act<Out, APPROXIFER_ACT_GELU>(t, x, w, dev, stream);
    case APPROXIFER_ACT_GELU_TANH: return launch_act<Out, APPROXIFER_ACT_GELU_TANH>(t, x, w, dev, stream);
    case APPROXIFER_ACT_SILU: return launch_act<Out, APPROXIFER_ACT_SILU>(t, x, w, dev, stream);
    default: return launch_act<Out, APPROXIFER_ACT_NONE>(t, x, w, dev, stream);
  }
}

}  // namespace

cudaError_t read_linear_pair_wait_timeouts(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_linear_pair_wait_timeouts, sizeof(*out)); }
cudaError_t reset_linear_pair_wait_timeouts() {
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_linear_pair_wait_timeouts, &zero, sizeof(zero));
}

cudaError_t launch_linear_pair(const approxifer_linear_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  PairArgs t{};
  t.M = (int32_t)a.M, t.N = (int32_t)a.N, t.K = (int32_t)a.K;
  t.steps = (int32_t)((a.K + kDepth - 1) / kDepth);
  const int64_t tm = (a.M + kTileM - 1) / kTileM, tn = (a.N + kTileN - 1) / kTileN;
  if (tm * tn > 0x3fffffffLL || tn > (1 << 27)) return cudaErrorInvalidConfiguration;
  t.tiles_m = (int32_t)tm, t.tiles_n = (int32_t)tn, t.tiles = (int32_t)(tm * tn);
  t.bias = reinterpret_cast<const bf16*>(a.bias), t.R = a.R, t.Y = a.Y, t.r_rstride = a.r_rstride, t.y_rstride = a.y_rstride;
  const int quad = a.out_type == APPROXIFER_TYPE_F32 ? 16 : 8;
  auto fits = [&](const void* p) { return reinterpret_cast<uintptr_t>(p) % quad == 0; };
  t.vec = fits(a.Y) && a.y_rstride % 4 == 0 && (!a.R || (fits(a.R) && a.r_rstride % 4 == 0));
  const uint64_t xe[2] = {(uint64_t)a.K, (uint64_t)a.M}, xs[2] = {1, (uint64_t)a.x_rstride}, we[2] = {(uint64_t)a.K, (uint64_t)a.N}, ws[2] = {1, (uint64_t)a.w_rstride};
  const uint32_t box[2] = {(uint32_t)kDepth, 128};
  CUtensorMap x, w;
  if ((e = make_tensor_map(&x, a.X, 2, xe, xs, box)) != cudaSuccess || (e = make_tensor_map(&w, a.Wt, 2, we, ws, box)) != cudaSuccess) return e;
  return a.out_type == APPROXIFER_TYPE_F32 ? launch_out<float>(a.activation, t, x, w, *dev, stream) : launch_out<bf16>(a.activation, t, x, w, *dev, stream);
}

}  // namespace approxifer
