// Matrix product with bias, activation and residual, on the tensor cores: one output tile per cluster, the product's long
// axis split over the CTAs of the cluster.
//
//   Y = act(X Wt^T + bias) + R, fp32 accumulators in tensor memory (an fp32 output shows their sums: error against 64
//   bits 3.6e-7 at 300 x 1,000 x 784, 1.0e-6 at 300 x 1,000 x 4,096, where elementary fp32 operations err by 2.1e-7 and
//   6.1e-7; a bfloat16 output hides it).
//
// A CTA forms a 128 x BN tile.  The operand whose rows become the 128 lanes of the accumulator is X, or -- SWAP, for few
// rows of X, where the call is bound by reading Wt -- Wt: the tile is then the transposed one and BN needs only to cover
// the rows of X.  A cluster of S CTAs shares a tile, each with its own part of K (few tiles still fill the GPU, with no
// workspace and no second launch); the partial tiles meet in shared memory, and every CTA sums S of them in rank order
// over its share of the tile (the same order every time) and applies the epilogue to it.
//
//   warp 0     one lane: tensor-map copies, 64 columns of both operands per stage, 6 to 10 stages in flight
//   warp 1     tcgen05.mma; allocates the tensor memory
//   warps 2-5  accumulator -> shared memory; all warps: sum, epilogue, stores
//
// Few rows are bound by reading Wt, small products by the chain of a start, one copy, one product and the joining (5 to
// 8 us).  Measured: 20 rows, 4,096 -> 16,384 with bias and gelu 26 us, 5.1 TB/s; 1,280 rows, 784 -> 10 5.5 us.
#include "async.cuh"

namespace approxifer {

__device__ unsigned int g_linear_tile_wait_timeouts = 0;

namespace {

constexpr int kThreads = 192;
constexpr int kLanes = 128;   // rows of the first operand per tile ...
constexpr int kMinLanes = 96; // ... and the fewest worth having (with less a copy is too short to keep HBM busy)
constexpr int kDepth = 64;    // columns of both operands per stage: one 128-byte swizzle row
constexpr int kHeader = 1024; // mbarriers, flags; keeps the stages 1,024-byte aligned

constexpr int stage_bytes(int bn) { return (kLanes + bn) * kDepth * 2; }
constexpr int stages_of(int bn) { return 196 * 1024 / stage_bytes(bn); }
constexpr int smem_bytes(int bn) { return kHeader + 1024 + stages_of(bn) * stage_bytes(bn); }
constexpr int tmem_cols(int bn) { return bn < 32 ? 32 : bn; }

struct TileArgs {
  int32_t M, N, K;
  int32_t steps;  // stages of K in all
  int32_t tiles_cols;
  int32_t lanes;  // rows of the first operand per tile: a multiple of 8, up to 128 (the accumulator's other lanes are not used)
  const bf16* bias;
  const void* R;
  void* Y;
  int64_t r_rstride, y_rstride;
  int32_t activation;
  int32_t vec, bias_vec;  // rows of Y and R, the bias, can be accessed four elements at a time
};

template <typename Out>
__device__ __forceinline__ float4 load4(const Out* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <>
__device__ __forceinline__ float4 load4<bf16>(const bf16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(bf16* p, float4 v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)); }

// Four consecutive columns from p on, of which the first `count` are there.
template <typename Out>
__device__ __forceinline__ float4 read4(const Out* p, bool vec, int count) {
  if (vec && count >= 4) return load4<Out>(p);
  return make_float4(count > 0 ? widen(p[0]) : 0.f, count > 1 ? widen(p[1]) : 0.f, count > 2 ? widen(p[2]) : 0.f, count > 3 ? widen(p[3]) : 0.f);
}
template <typename Out>
__device__ __forceinline__ void write4(Out* p, float4 v, bool vec, int count) {
  if (vec && count >= 4) {
    store4(p, v);
    return;
  }
  if (count > 0) p[0] = narrow<Out>(v.x);
  if (count > 1) p[1] = narrow<Out>(v.y);
  if (count > 2) p[2] = narrow<Out>(v.z);
  if (count > 3) p[3] = narrow<Out>(v.w);
}

template <int BN, bool SWAP, typename Out>
__global__ void __launch_bounds__(kThreads, 1) linear_tile_kernel(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap cols_map,
                                                               const __grid_constant__ TileArgs a) {
  constexpr int kStages = stages_of(BN);
  extern __shared__ unsigned char raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(base);  // full[stages], empty[stages], done
  volatile int* abort = reinterpret_cast<volatile int*>(base + 512);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base + 516);
  unsigned char* stages = base + kHeader;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages;
  const int warp = warp_index(), lane = threadIdx.x % 32;

  const int S = (int)cluster_size(), rank = (int)cluster_rank();
  const int tile = blockIdx.x / S;
  const int row0 = (tile / a.tiles_cols) * a.lanes, col0 = (tile % a.tiles_cols) * BN;
  const int step0 = (int)((int64_t)a.steps * rank / S), step1 = (int)((int64_t)a.steps * (rank + 1) / S);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) bar_init(full + 8 * s, 1), bar_init(empty + 8 * s, 1);
    bar_init(done, 1);
    *abort = 0;
    bar_init_done();
    prefetch_map(&rows_map);
    prefetch_map(&cols_map);
  }
  if (warp == 1) tmem_alloc(smem_addr(tmem_slot), tmem_cols(BN));
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  let_next_start();  // not before: the tensor memory is held
  wait_for_inputs();

  if (warp == 0 && lane == 0) {
    for (int i = step0; i < step1; ++i) {
      const int s = (i - step0) % kStages, turn = (i - step0) / kStages;
      if (turn > 0 && !bar_wait(empty + 8 * s, (turn - 1) & 1, abort, &g_linear_tile_wait_timeouts)) break;
      const uint32_t dst = smem_addr(stages) + s * stage_bytes(BN);
      bar_expect(full + 8 * s, (a.lanes + BN) * kDepth * 2);
      tma_2d(dst, &rows_map, i * kDepth, row0, full + 8 * s);
      tma_2d(dst + kLanes * kDepth * 2, &cols_map, i * kDepth, col0, full + 8 * s);
    }
  } else if (warp == 1) {
    for (int i = step0; i < step1; ++i) {
      const int s = (i - step0) % kStages, turn = (i - step0) / kStages;
      if (!warp_wait(full + 8 * s, turn & 1, abort, &g_linear_tile_wait_timeouts)) break;
      tmem_fence_after();
      const uint32_t src = smem_addr(stages) + s * stage_bytes(BN);
      const uint64_t da = desc_k_major(src), db = desc_k_major(src + kLanes * kDepth * 2);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kDepth / 16; ++k) mma_ss(tmem, da + 2 * k, db + 2 * k, mma_shape(kLanes, BN), i > step0 || k > 0);
        mma_commit(empty + 8 * s);
      }
      __syncwarp();
    }
    if (elect_one()) mma_commit(done);
  }
  __syncwarp();
  // Accumulator -> shared memory, in the order of the output: [m][n], n contiguous.  (`done` also says that every copy has
  // been consumed, so the stages can be written over.)
  constexpr int kPitch = SWAP ? kLanes : BN + 4;
  float* part = reinterpret_cast<float*>(stages);
  if (warp >= 2) {
    const bool ok = warp_wait(done, 0, abort, &g_linear_tile_wait_timeouts);
    tmem_fence_after();
    const int q = warp % 4, l = q * 32 + lane;
    if (ok) {
      constexpr int kAt = BN < 32 ? 16 : 32;  // columns at a time
#pragma unroll 2
      for (int c = 0; c < BN; c += kAt) {
        uint32_t v[kAt];
        const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + c;
        if constexpr (kAt == 16) tmem_ld16(from, v);
        else tmem_ld32(from, v);
        tmem_wait_ld(v);
        if (step0 == step1) {  // (more CTAs than stages of K: this one has nothing to add)
#pragma unroll
          for (int j = 0; j < kAt; ++j) v[j] = 0;
        }
        if constexpr (SWAP) {
#pragma unroll
          for (int j = 0; j < kAt; ++j) part[(c + j) * kPitch + l] = __uint_as_float(v[j]);
        } else {
#pragma unroll
          for (int j = 0; j < kAt; j += 4) *reinterpret_cast<uint4*>(part + l * kPitch + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
      }
    }
    tmem_fence_before();
  }
  __syncthreads();
  drain_if_aborted(abort);
  if (warp == 1) {
    tmem_fence_after();
    tmem_free(tmem, tmem_cols(BN));
  }
  if (S > 1) cluster_sync();
  // This CTA's share of the tile's rows, a warp to a row of up to 128 columns (or several shorter ones), a lane to four
  // columns, kAhead rows' loads side by side.
  const int m0 = SWAP ? col0 : row0, n0 = SWAP ? row0 : col0;
  const int rows_here = min(SWAP ? BN : a.lanes, a.M - m0);
  const int m_from = rows_here * rank / S, m_to = rows_here * (rank + 1) / S;
  constexpr int kQuads = SWAP ? 32 : BN / 4, kSide = 32 / kQuads, kAhead = 4, kWarps = kThreads / 32;
  const int n = (lane % kQuads) * 4, count = a.N - (n0 + n);
  if (n < (SWAP ? a.lanes : BN) && count > 0) {
    const uint32_t part_addr = smem_addr(part) + n * 4;
    const float4 b = a.bias ? read4<bf16>(a.bias + n0 + n, a.bias_vec, count) : make_float4(0.f, 0.f, 0.f, 0.f);
    const Out* R = static_cast<const Out*>(a.R) + n0 + n;
    Out* Y = static_cast<Out*>(a.Y) + n0 + n;
    for (int m = m_from + warp * kSide + lane / kQuads; m < m_to; m += kWarps * kSide * kAhead) {
      float4 v[kAhead], r[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int mi = m + i * kWarps * kSide;
        v[i] = r[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mi >= m_to) continue;
        if (S == 1) v[i] = *reinterpret_cast<const float4*>(part + mi * kPitch + n);
        if (a.R) r[i] = read4<Out>(R + (int64_t)(m0 + mi) * a.r_rstride, a.vec, count);
      }
      if (S > 1) {
#pragma unroll 2
        for (int s = 0; s < S; ++s) {
          const uint32_t peer = peer_smem(part_addr, s);
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const int mi = m + i * kWarps * kSide;
            if (mi >= m_to) continue;
            const float4 u = peer_load(peer + mi * kPitch * 4);
            v[i].x += u.x, v[i].y += u.y, v[i].z += u.z, v[i].w += u.w;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int mi = m + i * kWarps * kSide;
        if (mi >= m_to) continue;
        float4 z = make_float4(v[i].x + b.x, v[i].y + b.y, v[i].z + b.z, v[i].w + b.w);
        if (a.activation != APPROXIFER_ACT_NONE)
          z = make_float4(activate<Out>(a.activation, z.x), activate<Out>(a.activation, z.y), activate<Out>(a.activation, z.z), activate<Out>(a.activation, z.w));
        write4<Out>(Y + (int64_t)(m0 + mi) * a.y_rstride, make_float4(z.x + r[i].x, z.y + r[i].y, z.z + r[i].z, z.w + r[i].w), a.vec, count);
      }
    }
  }
  if (S > 1) cluster_sync();  // (a CTA's shared memory stays until all have read it)
}

template <int BN, bool SWAP, typename Out>
cudaError_t launch_one(const TileArgs& t, const CUtensorMap& rows, const CUtensorMap& cols, int64_t tiles, int split, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  auto kernel = linear_tile_kernel<BN, SWAP, Out>;
  struct Tag {};
  if ((e = ensure_dynamic_smem<Tag>(kernel, dev->ordinal, smem_bytes(BN))) != cudaSuccess) return e;
  return launch_kernel(kernel, tiles * split, kThreads, smem_bytes(BN), split, stream, rows, cols, t);
}

template <int BN, bool SWAP>
cudaError_t launch_out(const approxifer_linear_args& a, const TileArgs& t, const CUtensorMap& rows, const CUtensorMap& cols, int64_t tiles, int split,
                       cudaStream_t stream) {
  return a.out_type == APPROXIFER_TYPE_F32 ? launch_one<BN, SWAP, float>(t, rows, cols, tiles, split, stream)
                                           : launch_one<BN, SWAP, bf16>(t, rows, cols, tiles, split, stream);
}

cudaError_t operand_map(CUtensorMap* map, const uint16_t* base, int64_t rows, int64_t cols, int64_t rstride, int box_rows) {
  if (rows == 1) rstride = (cols + 7) / 8 * 8;  // (of a single row the stride says nothing)
  const uint64_t extent[2] = {(uint64_t)cols, (uint64_t)rows}, stride[2] = {1, (uint64_t)rstride};
  const uint32_t box[2] = {(uint32_t)kDepth, (uint32_t)box_rows};
  return make_tensor_map(map, base, 2, extent, stride, box);
}

}  // namespace

cudaError_t read_linear_tile_wait_timeouts(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_linear_tile_wait_timeouts, sizeof(*out)); }
cudaError_t reset_linear_tile_wait_timeouts() {
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_linear_tile_wait_timeouts, &zero, sizeof(zero));
}

bool linear_tile_eligible(const approxifer_linear_args& a) {
  return aligned16(a.X) && aligned16(a.Wt) && (a.M == 1 || a.x_rstride % 8 == 0) && (a.N == 1 || a.w_rstride % 8 == 0) && a.x_rstride < (1LL << 38) &&
         a.w_rstride < (1LL << 38);
}

cudaError_t launch_linear_tile(const approxifer_linear_args& a, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  // Up to 128 rows of X the product is bound by reading Wt, whose rows then become the 128 lanes, and the tile is only as
  // wide as X has rows.  Beyond, X's rows are the lanes and the tile as wide as N needs, up to 128.  (From 65 rows on, where
  // both tiles are 128 wide, the two ways measure the same within 2 %.)
  const bool swap = a.M <= 128;
  const int64_t across = swap ? a.M : a.N;
  const int bn = across <= 16 ? 16 : across <= 32 ? 32 : across <= 64 ? 64 : 128;
  const int64_t lanes = swap ? a.N : a.M;
  const int64_t tiles_cols = (across + bn - 1) / bn;
  TileArgs t{};
  t.M = (int32_t)a.M, t.N = (int32_t)a.N, t.K = (int32_t)a.K;
  t.steps = (int32_t)((a.K + kDepth - 1) / kDepth);
  t.tiles_cols = (int32_t)tiles_cols;
  t.bias = reinterpret_cast<const bf16*>(a.bias), t.R = a.R, t.Y = a.Y, t.r_rstride = a.r_rstride, t.y_rstride = a.y_rstride;
  t.activation = a.activation;
  const int size = a.out_type == APPROXIFER_TYPE_F32 ? 4 : 2, quad = 4 * size;
  auto fits = [](const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; };
  t.vec = fits(a.Y, quad) && a.y_rstride % 4 == 0 && (!a.R || (fits(a.R, quad) && a.r_rstride % 4 == 0));
  t.bias_vec = fits(a.bias, 8);
  // CTAs to a tile (each with four stages of K or more), and rows to a tile: full tiles, or as many fewer as give every SM
  // one of the same size.  A CTA's time is that of reading its rows over its part of K, plus some eight stages' worth for
  // its start and its end (with the cluster's meeting, ten); what counts is how many of those follow each other on an SM.
  int split = 1, per_tile = kLanes;
  int64_t tiles = 0;
  double best = 0;
  for (int s = 1; s <= 8 && (s == 1 || t.steps >= 4 * s); s *= 2) {
    // (a cluster sits within one GPC: of its SMs some are left over, more the larger the cluster)
    const int usable = s == 1 ? dev->sms : s == 2 ? dev->sms - 4 : s == 4 ? dev->sms * 7 / 8 : dev->sms * 3 / 4;
    const int64_t places = usable / s / tiles_cols;  // tiles along the rows that run at once
    const int64_t even = places > 0 ? ((lanes + places - 1) / places + 7) / 8 * 8 : kLanes;
    for (const int64_t rows : {(int64_t)kLanes, even}) {
      if (rows > kLanes || rows < kMinLanes) continue;
      const int64_t n = (lanes + rows - 1) / rows * tiles_cols, turns = (n * s + usable - 1) / usable;
      const double time = turns * ((double)rows / kLanes * ((t.steps + s - 1) / s) + (s == 1 ? 8 : 10));
      if (tiles == 0 || time < best) best = time, split = s, per_tile = (int)rows, tiles = n;
    }
  }
  t.lanes = per_tile;
  if (tiles * split > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  CUtensorMap rows, cols;
  if ((e = operand_map(&rows, swap ? a.Wt : a.X, lanes, a.K, swap ? a.w_rstride : a.x_rstride, per_tile)) != cudaSuccess) return e;
  if ((e = operand_map(&cols, swap ? a.X : a.Wt, across, a.K, swap ? a.x_rstride : a.w_rstride, bn)) != cudaSuccess) return e;
  if (swap) {
    switch (bn) {
      case 16: return launch_out<16, true>(a, t, rows, cols, tiles, split, stream);
      case 32: return launch_out<32, true>(a, t, rows, cols, tiles, split, stream);
      case 64: return launch_out<64, true>(a, t, rows, cols, tiles, split, stream);
      default: return launch_out<128, true>(a, t, rows, cols, tiles, split, stream);
    }
  }
  switch (bn) {
    case 16: return launch_out<16, false>(a, t, rows, cols, tiles, split, stream);
    case 32: return launch_out<32, false>(a, t, rows, cols, tiles, split, stream);
    case 64: return launch_out<64, false>(a, t, rows, cols, tiles, split, stream);
    default: return launch_out<128, false>(a, t, rows, cols, tiles, split, stream);
  }
}

}  // namespace approxifer
