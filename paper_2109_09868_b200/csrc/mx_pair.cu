// Product of 4-bit microscaled operands for many tiles: persistent pairs of CTAs, each pair one 256 x 192 tile of Y at a time
// (tcgen05 with cta_group::2 and kind::mxf4: every CTA keeps 128 rows of X and half of the tile's rows of Wt in shared memory, the
// two tensor cores read both halves).
//
// Tensor memory holds two accumulators, so that the epilogue of a tile runs under the products of the next, and beside them the
// scales of five stages: 24 columns each, two blocks (128 x 128 elements) of the CTA's rows of X and two times two of the tile's rows
// of Wt, of which each CTA needs all.  That is why a tile has 192 columns and not 256.  A tile then starts at a block's first row or
// in its middle: its scales two columns further on.  A stage's scales are copied before the first of its products is issued: between
// products such a copy waits for those before it (copies between every two: 674 us with gelu_tanh where this order took 450).
//
//   warp 0      one lane: tensor-map copies of this CTA's operands and scales, 256 columns (31 KB) a stage, five in flight
//   warp 1      of the pair's first CTA: copies of scales and tcgen05.mma for the pair; allocates the tensor memory
//   warps 2, 3  idle (the accumulator's lanes belong to warps by their index modulo 4)
//   warps 4-15  epilogue: three warps to each quarter of the lanes, 64 columns each; a thread has one row.  Bias, activation,
//               residual and the one rounding in registers, then through 2 KB of shared memory a warp by tensor-map stores.
//
// Bound by the way of the operands into the SM (with one product of a stage's four left out it takes as long; some 54 bytes a cycle
// arrive, the tensor cores could use 83), and, repeated, by the power limit (1.6 GHz).  Measured: 8,192 x 16,384 x 4,096 236 us, 4.65
// PFLOP/s, with gelu_tanh 246 us, with K = 256 82 us.  Tried and not faster: tiles of 256 columns whose accumulators share 64 columns
// of tensor memory, read first by the epilogue (230 us, with gelu_tanh 256 us, with K = 1,024 114 against 99 us: a tile waits for those
// reads).
#include "mx.cuh"

namespace approxifer {

__device__ unsigned int g_mx_pair_wait_timeouts = 0;

namespace {

constexpr int kEpilogueWarps = 12;
constexpr int kThreads = (4 + kEpilogueWarps) * 32;
constexpr int kTileM = 256, kTileN = 192;
constexpr int kRowBytes = 128;  // of a stage: 256 columns
constexpr int kStages = 5;
constexpr int kXBytes = 128 * kRowBytes, kWBytes = kTileN / 2 * kRowBytes, kOperandBytes = kXBytes + kWBytes;
constexpr int kStageBytes = kOperandBytes + 6 * kMxBlock;
constexpr int kRoomBytes = 32 * 64;  // of an epilogue warp: 32 rows of 64 bytes
constexpr int kHeader = 1024;
constexpr int kSmemBytes = kHeader + 1024 + kStages * kStageBytes + kEpilogueWarps * kRoomBytes;
constexpr int kTmemCols = 512, kScaleCols = 24;
static_assert(2 * kTileN + kStages * kScaleCols <= kTmemCols, "the scales exceed the tensor memory");
static_assert(kStageBytes % 1024 == 0 && kSmemBytes <= 227 * 1024, "shared memory");
constexpr int kGroupM = 8;  // rows of tiles that are walked together: their X stays in L2 while Wt streams by

struct PairArgs {
  int32_t M, N, steps, products;  // stages, and products (64 columns), of K
  int32_t blocks;                 // of scales, of K
  int32_t tiles_m, tiles_n, tiles;
  const bf16* bias;
  const void* R;
  void* Y;
  int64_t r_rstride, y_rstride;
  int32_t bias_whole, whole;      // the bias; Y and R: 16 bytes at a time, Y by tensor-map stores but for the end of ragged rows
};

// Tiles in bands of kGroupM rows of tiles, down a band's columns of tiles.
__device__ __forceinline__ void place(const PairArgs& a, int tile, int* m0, int* n0) {
  const int per_band = kGroupM * a.tiles_n, band = tile / per_band, in = tile - band * per_band;
  const int rows = min(kGroupM, a.tiles_m - band * kGroupM);
  *m0 = (band * kGroupM + in % rows) * kTileM;
  *n0 = (in / rows) * kTileN;
}

__device__ __forceinline__ void store_tile(const CUtensorMap* map, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(from) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void stores_have_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Adds N neighbours (of which `count` are there) from p on.
template <int N, typename T>
__device__ __forceinline__ void add_row(const T* p, bool whole, int count, float (&z)[N]) {
  constexpr int kAt = 16 / sizeof(T);
  if (whole && count >= N) {
#pragma unroll
    for (int i = 0; i < N; i += kAt) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + i);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) z[i + 2 * e] += __uint_as_float(w[e] << 16), z[i + 2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
        else z[i + e] += __uint_as_float(w[e]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < count) z[i] += widen(p[i]);
  }
}

// 64 bytes of the thread's row m0 + lane, from column n on: z is what the accumulator holds.
template <typename Out, int ACT, int N>
__device__ __forceinline__ void finish(const PairArgs& a, const CUtensorMap* y_map, int m0, int n, float (&z)[N], unsigned char* room, int lane) {
  static_assert(N * sizeof(Out) == 64, "64 bytes of a row");
  const int m = m0 + lane, left = a.N - n;
  if (a.bias) add_row<N, bf16>(a.bias + n, a.bias_whole, left, z);
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = mx_activate<ACT, Out>(z[i]);
  auto place16 = [&](int row, int i) { return room + row * 64 + ((i ^ ((row >> 1) & 3)) << 4); };  // the i-th 16 bytes of a row (the 64-byte swizzle)
  // (A tensor-map store leaves out what lies beyond a row's end by whole 16 bytes, no less: where the row ends within 16, its last piece
  // goes the other way.)
  if (a.whole && (left >= N || a.N % (16 / (int)sizeof(Out)) == 0)) {
    if (a.R && m < a.M) add_row<N, Out>(static_cast<const Out*>(a.R) + (int64_t)m * a.r_rstride + n, true, left, z);
    if (lane == 0) stores_have_read();  // the last piece has left
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 u;
      if constexpr (sizeof(Out) == 2)
        u = make_uint4(pack_bf16x2(z[8 * i], z[8 * i + 1]), pack_bf16x2(z[8 * i + 2], z[8 * i + 3]), pack_bf16x2(z[8 * i + 4], z[8 * i + 5]), pack_bf16x2(z[8 * i + 6], z[8 * i + 7]));
      else
        u = make_uint4(__float_as_uint(z[4 * i]), __float_as_uint(z[4 * i + 1]), __float_as_uint(z[4 * i + 2]), __float_as_uint(z[4 * i + 3]));
      *reinterpret_cast<uint4*>(place16(lane, i)) = u;
    }
    async_proxy_fence();
    __syncwarp();
    if (lane == 0 && m0 < a.M && left > 0) store_tile(y_map, smem_addr(room), n, m0);
    return;
  }
  // Rows that are not whole 16 bytes: sixteen columns at a time through shared memory in fp32, so that neighbouring lanes write, and
  // read of the residual, neighbours of a row.
  if (a.whole && lane == 0) stores_have_read();  // the last piece has left
#pragma unroll
  for (int c = 0; c < N; c += 16) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(place16(lane, i)) = make_float4(z[c + 4 * i], z[c + 4 * i + 1], z[c + 4 * i + 2], z[c + 4 * i + 3]);
    __syncwarp();
    const int col = n + c + lane % 16, rows = col < a.N ? a.M - m0 - lane / 16 : 0;  // (of every second row from this lane's first on)
    float r[16];
    if (a.R) {
      const Out* from = static_cast<const Out*>(a.R) + (int64_t)(m0 + lane / 16) * a.r_rstride + col;
#pragma unroll
      for (int i = 0; i < 16; ++i) r[i] = 2 * i < rows ? widen(from[2 * i * a.r_rstride]) : 0.f;
    }
    Out* to = static_cast<Out*>(a.Y) + (int64_t)(m0 + lane / 16) * a.y_rstride + col;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float y = reinterpret_cast<const float*>(place16(2 * i + lane / 16, lane % 16 / 4))[lane % 4];
      if (a.R) y += r[i];
      if (2 * i < rows) to[2 * i * a.y_rstride] = narrow<Out>(y);
    }
  }
}

template <typename Out, int ACT>
__global__ void __launch_bounds__(kThreads, 1)
    mx_pair_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_scales,
                   const __grid_constant__ CUtensorMap w_scales, const __grid_constant__ CUtensorMap y_map, const __grid_constant__ PairArgs a) {
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
  unsigned int* count = &g_mx_pair_wait_timeouts;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) bar_init(full + 8 * s, 1), bar_init(empty + 8 * s, 1);
    for (int s = 0; s < 2; ++s) bar_init(ready + 8 * s, 1), bar_init(drained + 8 * s, 2 * kEpilogueWarps);
    *abort = 0;
    bar_init_done();
    prefetch_map(&x_map), prefetch_map(&w_map), prefetch_map(&x_scales), prefetch_map(&w_scales);
    if (a.whole) prefetch_map(&y_map);
  }
  if (warp == 1) tmem_alloc_pair(smem_addr(tmem_slot), kTmemCols);
  tmem_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers stand before any is signalled from the other
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  let_next_start();  // not before: the tensor memory is held
  wait_for_inputs();

  // (The ring's place and phase are counted, not divided out: a stage's products last some 400 cycles, and the warp that issues them
  // has little time beside.)
  if (warp == 0 && lane == 0) {
    int s = 0;
    uint32_t phase = 1;  // of `empty`: the first turn finds every place free
    bool ok = true;
    for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
      int m0, n0;
      place(a, tile, &m0, &n0);
      m0 += rank * 128;
      const int w0 = n0 + rank * (kTileN / 2), x_block = m0 / kMxRows, w_block = n0 / kMxRows;
      for (int k = 0; k < a.steps; ++k) {
        if (!(ok = bar_wait(empty + 8 * s, phase, abort, count))) break;
        if (rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);  // both CTAs' copies count on the first one's barrier
        const uint32_t bar = peer_smem(full + 8 * s, 0), dst = stages + s * kStageBytes;
        tma_2d_pair(dst, &x_map, k * 64, m0, bar);
        tma_2d_pair(dst + kXBytes, &w_map, k * 64, w0, bar);
        tma_3d_pair(dst + kOperandBytes, &x_scales, 0, 2 * k, x_block, bar);
        tma_3d_pair(dst + kOperandBytes + 2 * kMxBlock, &w_scales, 0, 2 * k, w_block, bar);
        if (++s == kStages) s = 0, phase ^= 1;
      }
    }
  } else if (warp == 1 && rank == 0) {
    int s = 0, n = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = pair; tile < a.tiles && ok; tile += pairs, ++n) {
      const int acc = n & 1;
      int m0, n0;
      place(a, tile, &m0, &n0);
      const uint32_t skip = n0 % kMxRows / 32, d = tmem + acc * kTileN;
      if (n >= 2 && !(ok = warp_wait(drained + 8 * acc, (n / 2 - 1) & 1, abort, count))) break;
      tmem_fence_after();
      for (int k = 0; k < a.steps; ++k) {
        if (!(ok = warp_wait(full + 8 * s, phase, abort, count))) break;
        tmem_fence_after();
        const uint32_t src = stages + s * kStageBytes, from = src + kOperandBytes, sx = tmem + 2 * kTileN + s * kScaleCols, sw = sx + 8;
        const uint64_t da = desc_k_major(src), db = desc_k_major(src + kXBytes);
        const int left = a.products - 4 * k;
        if (elect_one()) {
          copy_scales_pair(sx, from);
          copy_scales_pair(sw, from + 2 * kMxBlock);
          copy_scales_pair(sw + 4, from + 4 * kMxBlock);
          if (left > 2) {
            copy_scales_pair(sx + 4, from + kMxBlock);
            copy_scales_pair(sw + 8, from + 3 * kMxBlock);
            copy_scales_pair(sw + 12, from + 5 * kMxBlock);
          }
          mma_mx_pair(d, da, db, mx_shape(kTileM, kTileN, 0), sx, sw + skip, k > 0);
          if (left >= 4) {
            mma_mx_pair(d, da + 2, db + 2, mx_shape(kTileM, kTileN, 1), sx, sw + skip, true);
            mma_mx_pair(d, da + 4, db + 4, mx_shape(kTileM, kTileN, 0), sx + 4, sw + 8 + skip, true);
            mma_mx_pair(d, da + 6, db + 6, mx_shape(kTileM, kTileN, 1), sx + 4, sw + 8 + skip, true);
          } else {  // (what lies beyond K's last 64 columns is not used: it need not be zero, nor its scales there)
            if (left > 1) mma_mx_pair(d, da + 2, db + 2, mx_shape(kTileM, kTileN, 1), sx, sw + skip, true);
            if (left > 2) mma_mx_pair(d, da + 4, db + 4, mx_shape(kTileM, kTileN, 0), sx + 4, sw + 8 + skip, true);
          }
          mma_commit_pair(empty + 8 * s);
          if (k + 1 == a.steps) mma_commit_pair(ready + 8 * acc);
        }
        __syncwarp();
        if (++s == kStages) s = 0, phase ^= 1;
      }
    }
  } else if (warp >= 4) {
    const int q = warp % 4, part = (warp - 4) / 4;
    unsigned char* room = base + kHeader + kStages * kStageBytes + (warp - 4) * kRoomBytes;
    int n = 0;
    for (int tile = pair; tile < a.tiles; tile += pairs, ++n) {
      const int acc = n & 1;
      int m0, n0;
      place(a, tile, &m0, &n0);
      m0 += rank * 128 + q * 32, n0 += part * 64;
      if (!warp_wait(ready + 8 * acc, (n / 2) & 1, abort, count)) break;
      tmem_fence_after();
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + acc * kTileN + part * 64;
      constexpr int kAt = 64 / sizeof(Out);  // columns at a time
#pragma unroll
      for (int c = 0; c < 64; c += kAt) {
        float z[kAt];
        if constexpr (kAt == 32) tmem_ld32(from + c, *reinterpret_cast<uint32_t(*)[kAt]>(z));
        else tmem_ld16(from + c, *reinterpret_cast<uint32_t(*)[kAt]>(z));
        tmem_wait_ld(*reinterpret_cast<uint32_t(*)[kAt]>(z));
        if (c + kAt == 64) {  // the accumulator has been read
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(peer_smem(drained + 8 * acc, 0));
        }
        finish<Out, ACT, kAt>(a, &y_map, m0, n0 + c, z, room, lane);
      }
    }
    if (lane == 0) stores_done();
  }
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  drain_if_aborted(abort);
  cluster_sync();  // neither CTA leaves while the other's copies, products or arrivals may still reach it
  tmem_fence_after();
  if (warp == 1) tmem_free_pair(tmem, kTmemCols);
}

struct Maps {
  CUtensorMap x, w, x_scales, w_scales, y;
};

template <typename Out, int ACT>
cudaError_t launch_act(const PairArgs& t, const Maps& m, const DeviceInfo& dev, cudaStream_t stream) {
  auto kernel = mx_pair_kernel<Out, ACT>;
  struct Tag {};
  const cudaError_t e = ensure_dynamic_smem<Tag>(kernel, dev.ordinal, kSmemBytes);
  if (e != cudaSuccess) return e;
  const int pairs = t.tiles < dev.sms / 2 ? t.tiles : dev.sms / 2;
  return launch_kernel(kernel, 2 * pairs, kThreads, kSmemBytes, 2, stream, m.x, m.w, m.x_scales, m.w_scales, m.y, t);
}

template <typename Out>
cudaError_t launch_out(int act, const PairArgs& t, const Maps& m, const DeviceInfo& dev, cudaStream_t stream) {
  switch (act) {
    case APPROXIFER_ACT_RELU: return launch_act<Out, APPROXIFER_ACT_RELU>(t, m, dev, stream);
    case APPROXIFER_ACT_GELU: return launch_act<Out, APPROXIFER_ACT_GELU>(t, m, dev, stream);
    case APPROXIFER_ACT_GELU_TANH: return launch_act<Out, APPROXIFER_ACT_GELU_TANH>(t, m, dev, stream);
    case APPROXIFER_ACT_SILU: return launch_act<Out, APPROXIFER_ACT_SILU>(t, m, dev, stream);
    default: return launch_act<Out, APPROXIFER_ACT_NONE>(t, m, dev, stream);
  }
}

}  // namespace

cudaError_t read_mx_pair_wait_timeouts(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_mx_pair_wait_timeouts, sizeof(*out)); }
cudaError_t reset_mx_pair_wait_timeouts() {
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_mx_pair_wait_timeouts, &zero, sizeof(zero));
}

cudaError_t launch_mx_pair(const approxifer_mx_linear_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  const bool f32 = a.out_type == APPROXIFER_TYPE_F32;
  const int size = f32 ? 4 : 2;
  PairArgs t{};
  t.M = (int32_t)a.M, t.N = (int32_t)a.N;
  t.steps = (int32_t)((a.K + 255) / 256), t.products = (int32_t)((a.K + 63) / 64), t.blocks = (int32_t)((a.K + kMxCols - 1) / kMxCols);
  const int64_t tm = (a.M + kTileM - 1) / kTileM, tn = (a.N + kTileN - 1) / kTileN;
  if (tm * tn > 0x3fffffffLL || tn > (1 << 27)) return cudaErrorInvalidConfiguration;
  t.tiles_m = (int32_t)tm, t.tiles_n = (int32_t)tn, t.tiles = (int32_t)(tm * tn);
  t.bias = reinterpret_cast<const bf16*>(a.bias), t.R = a.R, t.Y = a.Y, t.r_rstride = a.r_rstride, t.y_rstride = a.y_rstride;
  t.bias_whole = aligned16(a.bias);
  t.whole = aligned16(a.Y) && a.y_rstride * size % 16 == 0 && a.y_rstride < (1LL << 37) && (!a.R || (aligned16(a.R) && a.r_rstride * size % 16 == 0));
  Maps m{};
  const uint64_t xe[2] = {(uint64_t)a.K / 4, (uint64_t)a.M}, xs[2] = {1, (uint64_t)a.x_rstride / 2}, we[2] = {(uint64_t)a.K / 4, (uint64_t)a.N}, ws[2] = {1, (uint64_t)a.w_rstride / 2};
  const uint32_t x_box[2] = {64, 128}, w_box[2] = {64, kTileN / 2};
  if ((e = make_tensor_map(&m.x, a.X, 2, xe, xs, x_box)) != cudaSuccess || (e = make_tensor_map(&m.w, a.Wt, 2, we, ws, w_box)) != cudaSuccess ||
      (e = make_scales_map(&m.x_scales, a.x_scales, (a.M + kMxRows - 1) / kMxRows, t.blocks, 1)) != cudaSuccess ||
      (e = make_scales_map(&m.w_scales, a.w_scales, (a.N + kMxRows - 1) / kMxRows, t.blocks, 2)) != cudaSuccess)
    return e;
  if (t.whole && (e = make_store_map(&m.y, a.Y, f32, a.M, a.N, a.y_rstride)) != cudaSuccess) return e;
  return f32 ? launch_out<float>(a.activation, t, m, *dev, stream) : launch_out<bf16>(a.activation, t, m, *dev, stream);
}

}  // namespace approxifer
