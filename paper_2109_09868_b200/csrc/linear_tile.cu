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
//
// The same with both operands 4-bit microscaled (two elements to a byte: a stage is 256 columns; their scales go from shared into
// tensor memory before a stage's products).  Coded X, weights from HBM, from a graph: 1 x 4,096 x 4,096 6.0 us (the two ends of the
// call, a cluster's meeting among them: reading Wt takes 1.4), 20 x 16,384 x 4,096 9.8 us, 3.7 TB/s, 1 x 1,000 x 1,024 3.2 us; X in
// bfloat16 0.5 to 2.5 us more.
#include "mx.cuh"

namespace approxifer {

__device__ unsigned int g_linear_tile_wait_timeouts = 0;

namespace {

// What the operands are: bfloat16; both 4-bit microscaled (256 columns, and two blocks of each operand's scales, a stage); the same
// with X in bfloat16, brought into the 4-bit form on its way into shared memory, where all of this CTA's part of it stays.
enum Kind { kBf16, kMx, kMxRaw };
constexpr int kRawWarps = 16;  // at most, that do so, after the first two
constexpr int kRawSteps = 16;  // stages of K that there is room for
constexpr int threads_of(Kind kind) { return kind == kMxRaw ? (2 + kRawWarps) * 32 : 192; }  // (at most)
constexpr int kLanes = 128;   // rows of the first operand per tile ...
constexpr int kMinLanes = 96; // ... and the fewest worth having (with less a copy is too short to keep HBM busy)
constexpr int kDepth = 64;    // columns of both operands per stage: one 128-byte swizzle row
constexpr int kHeader = 1024; // mbarriers, flags; keeps the stages 1,024-byte aligned

constexpr int rows_bytes(Kind kind) { return kLanes * kDepth * 2 + (kind == kBf16 ? 0 : 2 * kMxBlock); }
constexpr int cols_bytes(int bn, Kind kind) { return bn * kDepth * 2 + (kind == kBf16 ? 0 : 2 * kMxBlock); }
constexpr int raw_bytes(int bn, Kind kind) { return kind == kMxRaw ? kRawSteps * cols_bytes(bn, kind) : 0; }
constexpr int stage_bytes(int bn, Kind kind) { return rows_bytes(kind) + (kind == kMxRaw ? 0 : cols_bytes(bn, kind)); }
constexpr int stages_of(int bn, Kind kind) { return (196 * 1024 - raw_bytes(bn, kind)) / stage_bytes(bn, kind); }
constexpr int smem_bytes(int bn, Kind kind) { return kHeader + 1024 + stages_of(bn, kind) * stage_bytes(bn, kind) + raw_bytes(bn, kind); }
constexpr int acc_cols(int bn) { return bn < 32 ? 32 : bn; }
// (4 bits: behind the accumulator sixteen columns of scales a stage)
constexpr int tmem_cols(int bn, Kind kind) { return kind == kBf16 ? acc_cols(bn) : 256; }
static_assert(acc_cols(16) + 16 * stages_of(16, kMx) <= 256 && acc_cols(32) + 16 * stages_of(32, kMx) <= 256 && acc_cols(64) + 16 * stages_of(64, kMx) <= 256 &&
                  acc_cols(128) + 16 * stages_of(128, kMx) <= 256,
              "the scales exceed the tensor memory");

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
  int32_t mx_blocks;      // (4 bits) blocks of 128 columns
  const bf16* raw;        // (kMxRaw) X
  int64_t raw_rstride;
  int32_t raw_columns, raw_whole;  // ... its columns; 16 bytes at a time
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

// (kMxRaw) This warp's share of X's columns of stages step0 .. step1-1, brought into the 4-bit form.  Half a warp takes a row's 128
// columns (one of the stage's two blocks) at a time, rows and then stages in turn, with the other warps; the
// loads of the next four are in flight meanwhile.
template <int BN>
__device__ __forceinline__ void bring_raw(const TileArgs& a, unsigned char* to, uint32_t landed, int step0, int step1, int warps, int warp, int lane) {
  constexpr int kAhead = 4;
  struct Place {
    int stage, row;
    __device__ __forceinline__ void next(int stages_on, int rows_on, int rows) {
      stage += stages_on, row += rows_on;
      if (row >= rows) row -= rows, ++stage;
    }
  };
  const int M = a.M, half = lane / 16, at = lane % 16 * 8, stages = step1 - step0, stages_on = warps / M, rows_on = warps % M;
  const bf16* from = a.raw + (int64_t)step0 * 4 * kDepth + half * kMxCols + at;
  const int columns = a.raw_columns - step0 * 4 * kDepth - half * kMxCols - at;  // from there on
  Place get{warp / M, warp % M}, use = get;
  MxRow<bf16> v[kAhead];
  auto load = [&](MxRow<bf16>& x) {
    x.none();
    const int col = get.stage * 4 * kDepth;
    if (get.stage < stages && col < columns) {
      const bf16* p = from + get.row * a.raw_rstride + col;
      if (a.raw_whole) x.load<true>(p);
      else x.load<false>(p);
    }
    get.next(stages_on, rows_on, M);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load(v[i]);
  unsigned char* codes_to = to + ((half * kMxCols + at) / 32 << 4) + at / 2 % 16;
  unsigned char* scales_to = to + BN * 128 + half * kMxBlock + at / 32;
  int told = 0;  // stages that this warp has said to be there
  while (told < stages) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      uint32_t byte;
      const uint32_t codes = mx_quantize8(v[i].widened(), &byte);
      load(v[i]);
      if (use.stage < stages) {
        const int offset = use.stage * cols_bytes(BN, kMxRaw);
        *reinterpret_cast<uint32_t*>(to + offset + use.row * 128 + ((int)(codes_to - to) ^ ((use.row & 7) << 4))) = codes;  // (the 128-byte swizzle)
        if (lane % 4 == 0) scales_to[offset + use.row * 16] = (unsigned char)byte;
      }
      use.next(stages_on, rows_on, M);
      const int whole = min(use.stage, stages);
      if (told < whole) {
        async_proxy_fence();
        __syncwarp();
        if (lane == 0)
          for (int x = told; x < whole; ++x) bar_arrive(landed + 8 * x);
        told = whole;
      }
    }
  }
}

// (4 bits) One choice of the activation for all values that a thread has in hand: with one for each, the instructions fetched lie
// scattered over the code of all activations, and in a small product those fetches are waited for; nor has any of these activations a
// division's long way, which the zeros beyond a tile's rows took.  Measured, 115 x 272 x 224 with gelu_tanh 8.9 -> 5.6 us, with rows of
// 273 13.3 -> 6.1 us (without an activation 4.3 and 4.6).
template <typename Out, int N>
__device__ __forceinline__ void activate_all(int act, float4 (&v)[N]) {
  auto each = [&](auto code) {
    constexpr int ACT = decltype(code)::value;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = make_float4(mx_activate<ACT, Out>(v[i].x), mx_activate<ACT, Out>(v[i].y), mx_activate<ACT, Out>(v[i].z), mx_activate<ACT, Out>(v[i].w));
  };
  switch (act) {
    case APPROXIFER_ACT_RELU: return each(std::integral_constant<int, APPROXIFER_ACT_RELU>{});
    case APPROXIFER_ACT_GELU: return each(std::integral_constant<int, APPROXIFER_ACT_GELU>{});
    case APPROXIFER_ACT_GELU_TANH: return each(std::integral_constant<int, APPROXIFER_ACT_GELU_TANH>{});
    case APPROXIFER_ACT_SILU: return each(std::integral_constant<int, APPROXIFER_ACT_SILU>{});
    default: return;
  }
}

template <int BN, bool SWAP, typename Out, Kind KIND>
__global__ void __launch_bounds__(threads_of(KIND), 1) linear_tile_kernel(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap cols_map,
                                                               const __grid_constant__ CUtensorMap row_scales, const __grid_constant__ CUtensorMap col_scales,
                                                               const __grid_constant__ TileArgs a) {
  const int warps = KIND == kMxRaw ? (int)blockDim.x / 32 : threads_of(KIND) / 32;
  constexpr int kStages = stages_of(BN, KIND), kStageBytes = stage_bytes(BN, KIND);
  extern __shared__ unsigned char raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(base);  // full[stages], empty[stages], done, (kMxRaw) landed[steps]
  volatile int* abort = reinterpret_cast<volatile int*>(base + 512);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base + 516);
  unsigned char* stages = base + kHeader;
  unsigned char* raw_at = stages + kStages * kStageBytes;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, landed = done + 8;
  const int warp = warp_index(), lane = threadIdx.x % 32;

  const int S = (int)cluster_size(), rank = (int)cluster_rank();
  const int tile = blockIdx.x / S;
  const int row0 = (tile / a.tiles_cols) * a.lanes, col0 = (tile % a.tiles_cols) * BN;
  const int step0 = (int)((int64_t)a.steps * rank / S), step1 = (int)((int64_t)a.steps * (rank + 1) / S);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) bar_init(full + 8 * s, 1), bar_init(empty + 8 * s, 1);
    bar_init(done, 1);
    for (int s = 0; KIND == kMxRaw && s < kRawSteps; ++s) bar_init(landed + 8 * s, warps - 2);
    *abort = 0;
    bar_init_done();
    prefetch_map(&rows_map);
    if constexpr (KIND != kMxRaw) prefetch_map(&cols_map);
    if constexpr (KIND != kBf16) prefetch_map(&row_scales);
    if constexpr (KIND == kMx) prefetch_map(&col_scales);
  }
  if (warp == 1) tmem_alloc(smem_addr(tmem_slot), tmem_cols(BN, KIND));
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
      const uint32_t dst = smem_addr(stages) + s * kStageBytes;
      bar_expect(full + 8 * s, kStageBytes - (kLanes - a.lanes) * kDepth * 2);
      tma_2d(dst, &rows_map, i * kDepth, row0, full + 8 * s);
      if constexpr (KIND != kMxRaw) tma_2d(dst + rows_bytes(KIND), &cols_map, i * kDepth, col0, full + 8 * s);
      if constexpr (KIND != kBf16) tma_3d(dst + kLanes * kDepth * 2, &row_scales, 0, 2 * i, row0 / kMxRows, full + 8 * s);
      if constexpr (KIND == kMx) tma_3d(dst + rows_bytes(KIND) + BN * kDepth * 2, &col_scales, 0, 2 * i, col0 / kMxRows, full + 8 * s);
    }
  } else if (warp == 1) {
    for (int i = step0; i < step1; ++i) {
      const int s = (i - step0) % kStages, turn = (i - step0) / kStages;
      if (KIND == kMxRaw && !warp_wait(landed + 8 * (i - step0), 0, abort, &g_linear_tile_wait_timeouts)) break;
      if (!warp_wait(full + 8 * s, turn & 1, abort, &g_linear_tile_wait_timeouts)) break;
      tmem_fence_after();
      const uint32_t src = smem_addr(stages) + s * kStageBytes;
      const uint32_t cols = KIND == kMxRaw ? smem_addr(raw_at) + (i - step0) * cols_bytes(BN, KIND) : src + rows_bytes(KIND);
      const uint64_t da = desc_k_major(src), db = desc_k_major(cols);
      if (elect_one()) {
        if constexpr (KIND != kBf16) {
          // (what a block of scales holds beyond K's last 64 columns is not used: it need not be there)
          const uint32_t sa = tmem + acc_cols(BN) + s * 16, sb = sa + 8, first = sb + col0 % kMxRows / 32;
          // (a tile that starts within a block of scales starts in its middle, two columns on: an odd column is a misaligned address)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (2 * i + k < a.mx_blocks) {
              copy_scales(sa + 4 * k, src + kLanes * kDepth * 2 + k * kMxBlock);
              copy_scales(sb + 4 * k, cols + BN * kDepth * 2 + k * kMxBlock);
            }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (i * 4 + k < (a.K + 15) / 16) mma_mx(tmem, da + 2 * k, db + 2 * k, mx_shape(kLanes, BN, k % 2), sa + k / 2 * 4, first + k / 2 * 4, i > step0 || k > 0);
          }
        } else {
#pragma unroll
          for (int k = 0; k < kDepth / 16; ++k) mma_ss(tmem, da + 2 * k, db + 2 * k, mma_shape(kLanes, BN), i > step0 || k > 0);
        }
        mma_commit(empty + 8 * s);
      }
      __syncwarp();
    }
    if (elect_one()) mma_commit(done);
  } else if (KIND == kMxRaw && warp >= 2) {
    bring_raw<BN>(a, raw_at, landed, step0, step1, warps - 2, warp - 2, lane);
  }
  __syncwarp();
  // Accumulator -> shared memory, in the order of the output: [m][n], n contiguous.  (`done` also says that every copy has
  // been consumed, so the stages can be written over.)
  constexpr int kPitch = SWAP ? kLanes : BN + 4;
  float* part = reinterpret_cast<float*>(stages);
  if (warp >= 2 && warp < 6) {
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
    tmem_free(tmem, tmem_cols(BN, KIND));
  }
  if (S > 1) cluster_sync();
  // This CTA's share of the tile's rows, a warp to a row of up to 128 columns (or several shorter ones), a lane to four
  // columns, kAhead rows' loads side by side.
  const int m0 = SWAP ? col0 : row0, n0 = SWAP ? row0 : col0;
  const int rows_here = min(SWAP ? BN : a.lanes, a.M - m0);
  const int m_from = rows_here * rank / S, m_to = rows_here * (rank + 1) / S;
  constexpr int kQuads = SWAP ? 32 : BN / 4, kSide = 32 / kQuads, kAhead = 4;
  const int n = (lane % kQuads) * 4, count = a.N - (n0 + n);
  if (n < (SWAP ? a.lanes : BN) && count > 0) {
    const uint32_t part_addr = smem_addr(part) + n * 4;
    const float4 b = a.bias ? read4<bf16>(a.bias + n0 + n, a.bias_vec, count) : make_float4(0.f, 0.f, 0.f, 0.f);
    const Out* R = static_cast<const Out*>(a.R) + n0 + n;
    Out* Y = static_cast<Out*>(a.Y) + n0 + n;
    for (int m = m_from + warp * kSide + lane / kQuads; m < m_to; m += warps * kSide * kAhead) {
      float4 v[kAhead], r[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int mi = m + i * warps * kSide;
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
            const int mi = m + i * warps * kSide;
            if (mi >= m_to) continue;
            const float4 u = peer_load(peer + mi * kPitch * 4);
            v[i].x += u.x, v[i].y += u.y, v[i].z += u.z, v[i].w += u.w;
          }
        }
      }
      if constexpr (KIND != kBf16) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = make_float4(v[i].x + b.x, v[i].y + b.y, v[i].z + b.z, v[i].w + b.w);
        activate_all<Out>(a.activation, v);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int mi = m + i * warps * kSide;
        if (mi >= m_to) continue;
        float4 z = v[i];
        if constexpr (KIND == kBf16) {
          z = make_float4(v[i].x + b.x, v[i].y + b.y, v[i].z + b.z, v[i].w + b.w);
          if (a.activation != APPROXIFER_ACT_NONE)
            z = make_float4(activate<Out>(a.activation, z.x), activate<Out>(a.activation, z.y), activate<Out>(a.activation, z.z), activate<Out>(a.activation, z.w));
        }
        write4<Out>(Y + (int64_t)(m0 + mi) * a.y_rstride, make_float4(z.x + r[i].x, z.y + r[i].y, z.z + r[i].z, z.w + r[i].w), a.vec, count);
      }
    }
  }
  if (S > 1) cluster_sync();  // (a CTA's shared memory stays until all have read it)
}

struct Maps {
  CUtensorMap rows, cols, row_scales, col_scales;
};

template <int BN, bool SWAP, typename Out, Kind KIND>
cudaError_t launch_one(const TileArgs& t, const Maps& m, int64_t tiles, int split, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  auto kernel = linear_tile_kernel<BN, SWAP, Out, KIND>;
  struct Tag {};
  if ((e = ensure_dynamic_smem<Tag>(kernel, dev->ordinal, smem_bytes(BN, KIND))) != cudaSuccess) return e;
  // (X in bfloat16: sixteen warps for more than eight rows.  Eight against sixteen, us: 1 x 4,096 x 4,096 6.5 / 7.0, 16 x 16,384 x 4,096
  // 16.0 / 12.9)
  const int threads = KIND == kMxRaw && t.M <= 8 ? threads_of(KIND) - 256 : threads_of(KIND);
  return launch_kernel(kernel, tiles * split, threads, smem_bytes(BN, KIND), split, stream, m.rows, m.cols, m.row_scales, m.col_scales, t);
}

template <int BN, bool SWAP>
cudaError_t launch_out(const approxifer_linear_args& a, const TileArgs& t, const Maps& m, Kind kind, int64_t tiles, int split, cudaStream_t stream) {
  const bool f32 = a.out_type == APPROXIFER_TYPE_F32;
  if constexpr (SWAP && BN <= kMxRawRows)
    if (kind == kMxRaw) return f32 ? launch_one<BN, SWAP, float, kMxRaw>(t, m, tiles, split, stream) : launch_one<BN, SWAP, bf16, kMxRaw>(t, m, tiles, split, stream);
  if (kind == kMx) return f32 ? launch_one<BN, SWAP, float, kMx>(t, m, tiles, split, stream) : launch_one<BN, SWAP, bf16, kMx>(t, m, tiles, split, stream);
  return f32 ? launch_one<BN, SWAP, float, kBf16>(t, m, tiles, split, stream) : launch_one<BN, SWAP, bf16, kBf16>(t, m, tiles, split, stream);
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

namespace {

// The operand whose rows are the lanes, the tile's width and rows, the CTAs that share one.
struct TilePlan {
  bool swap;
  int bn, split, per_tile;
  int64_t lanes, across, tiles, tiles_cols;
  int steps;
};
// Of 4-bit operands (full tiles only: blocks of scales have 128 rows): also how wide a tile is, since a stage is soon through and a
// tile's end, its columns joined, activated and stored, is what small products consist of.  A CTA's time, in stages of narrow tiles
// (0.2 us): its stages, longer with the tile's width; some eight for its start (ten with a cluster's meeting); sixteen for the end of 128
// columns, shared by the cluster; clusters that follow each other find their places late.
TilePlan plan_mx_tiles(TilePlan p, int sms) {
  double best = 0;
  TilePlan chosen = p;
  for (int bn = p.bn; bn == p.bn || bn >= 64; bn /= 2) {  // (tiles side by side start at a block's first row or in its middle: see the kernel)
    const int64_t tiles_cols = (p.across + bn - 1) / bn, tiles = (p.lanes + kLanes - 1) / kLanes * tiles_cols;
    for (int s = 1; s <= 8 && (s == 1 || p.steps >= 4 * s); s *= 2) {
      const int usable = s == 1 ? sms : s == 2 ? sms - 4 : s == 4 ? sms * 7 / 8 : sms * 3 / 4;
      const int64_t turns = (tiles * s + usable - 1) / usable;
      const double time = turns * ((p.steps + s - 1) / s * (1 + bn / 160.0) + (s == 1 ? 8 : 10) + 16.0 * bn / 128 / s) + (s > 1 ? 6 * (turns - 1) : 0);
      if (best == 0 || time < best) best = time, chosen.bn = bn, chosen.split = s, chosen.per_tile = kLanes, chosen.tiles = tiles, chosen.tiles_cols = tiles_cols;
    }
  }
  return chosen;
}

TilePlan plan_tiles(const approxifer_linear_args& a, bool mx, int sms) {
  TilePlan p{};
  // Up to 128 rows of X the product is bound by reading Wt, whose rows then become the 128 lanes, and the tile is only as
  // wide as X has rows.  Beyond, X's rows are the lanes and the tile as wide as N needs, up to 128.  (From 65 rows on, where
  // both tiles are 128 wide, the two ways measure the same within 2 %.)
  p.swap = a.M <= 128;
  p.across = p.swap ? a.M : a.N;
  p.bn = p.across <= 16 ? 16 : p.across <= 32 ? 32 : p.across <= 64 ? 64 : 128;
  p.lanes = p.swap ? a.N : a.M;
  p.tiles_cols = (p.across + p.bn - 1) / p.bn;
  p.steps = (int32_t)((a.K + kDepth - 1) / kDepth);
  if (mx) return plan_mx_tiles(p, sms);
  // CTAs to a tile (each with four stages of K or more), and rows to a tile: full tiles, or as many fewer as give every SM
  // one of the same size.  A CTA's time is that of reading its rows over its part of K, plus some eight stages' worth for
  // its start and its end (with the cluster's meeting, ten); what counts is how many of those follow each other on an SM.
  p.split = 1, p.per_tile = kLanes;
  double best = 0;
  for (int s = 1; s <= 8 && (s == 1 || p.steps >= 4 * s); s *= 2) {
    // (a cluster sits within one GPC: of its SMs some are left over, more the larger the cluster)
    const int usable = s == 1 ? sms : s == 2 ? sms - 4 : s == 4 ? sms * 7 / 8 : sms * 3 / 4;
    const int64_t places = usable / s / p.tiles_cols;  // tiles along the rows that run at once
    const int64_t even = places > 0 ? ((p.lanes + places - 1) / places + 7) / 8 * 8 : kLanes;
    for (const int64_t rows : {(int64_t)kLanes, even}) {
      if (rows > kLanes || rows < kMinLanes) continue;
      const int64_t n = (p.lanes + rows - 1) / rows * p.tiles_cols, turns = (n * s + usable - 1) / usable;
      const double time = turns * ((double)rows / kLanes * ((p.steps + s - 1) / s) + (s == 1 ? 8 : 10));
      if (p.tiles == 0 || time < best) best = time, p.split = s, p.per_tile = (int)rows, p.tiles = n;
    }
  }
  return p;
}

}  // namespace

// X in bfloat16: its 4-bit form of a CTA's part of K has to fit beside the ring, and as every CTA makes it anew, it has to be little.
// Measured, in a launch of its own against within the product, us: 1 x 4,096 x 4,096 (4 stages a CTA) 8.6 / 6.5, 32 rows 10.3 / 9.4;
// 1 x 16,384 x 4,096 (16 stages a CTA) 12.2 / 9.8, 8 rows 12.3 / 11.6, 16 rows 12.4 / 13.0.
bool linear_tile_takes_raw(const approxifer_linear_args& a, int sms) {
  if (a.M > kMxRawRows) return false;
  const TilePlan p = plan_tiles(a, true, sms);
  const int steps = (p.steps + p.split - 1) / p.split;
  return steps <= kRawSteps && steps * a.M <= 192;
}

cudaError_t launch_linear_tile(const approxifer_linear_args& a, const MxScales* mx, cudaStream_t stream) {
  const DeviceInfo* dev;
  cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  const TilePlan p = plan_tiles(a, mx != nullptr, dev->sms);
  TileArgs t{};
  t.M = (int32_t)a.M, t.N = (int32_t)a.N, t.K = (int32_t)a.K;
  t.steps = p.steps, t.tiles_cols = (int32_t)p.tiles_cols, t.lanes = p.per_tile;
  t.bias = reinterpret_cast<const bf16*>(a.bias), t.R = a.R, t.Y = a.Y, t.r_rstride = a.r_rstride, t.y_rstride = a.y_rstride;
  t.activation = a.activation;
  const int size = a.out_type == APPROXIFER_TYPE_F32 ? 4 : 2, quad = 4 * size;
  auto fits = [](const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; };
  t.vec = fits(a.Y, quad) && a.y_rstride % 4 == 0 && (!a.R || (fits(a.R, quad) && a.r_rstride % 4 == 0));
  t.bias_vec = fits(a.bias, 8);
  if (p.tiles * p.split > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const Kind kind = mx == nullptr ? kBf16 : mx->x == nullptr ? kMxRaw : kMx;
  Maps m{};
  if ((e = operand_map(&m.rows, p.swap ? a.Wt : a.X, p.lanes, a.K, p.swap ? a.w_rstride : a.x_rstride, p.per_tile)) != cudaSuccess) return e;
  if (kind != kMxRaw && (e = operand_map(&m.cols, p.swap ? a.X : a.Wt, p.across, a.K, p.swap ? a.x_rstride : a.w_rstride, p.bn)) != cudaSuccess) return e;
  if (mx) {
    t.mx_blocks = (int32_t)((mx->K + kMxCols - 1) / kMxCols);
    auto scales_map = [&](CUtensorMap* map, const uint8_t* base, int64_t n) { return make_scales_map(map, base, (n + kMxRows - 1) / kMxRows, t.mx_blocks, 1); };
    if ((e = scales_map(&m.row_scales, p.swap ? mx->w : mx->x, p.lanes)) != cudaSuccess) return e;
    if (kind == kMx && (e = scales_map(&m.col_scales, p.swap ? mx->x : mx->w, p.across)) != cudaSuccess) return e;
    t.raw = reinterpret_cast<const bf16*>(a.X), t.raw_rstride = a.x_rstride, t.raw_columns = (int32_t)mx->K;
    t.raw_whole = aligned16(a.X) && a.x_rstride % 8 == 0;
  }
  if (p.swap) {
    switch (p.bn) {
      case 16: return launch_out<16, true>(a, t, m, kind, p.tiles, p.split, stream);
      case 32: return launch_out<32, true>(a, t, m, kind, p.tiles, p.split, stream);
      case 64: return launch_out<64, true>(a, t, m, kind, p.tiles, p.split, stream);
      default: return launch_out<128, true>(a, t, m, kind, p.tiles, p.split, stream);
    }
  }
  switch (p.bn) {
    case 16: return launch_out<16, false>(a, t, m, kind, p.tiles, p.split, stream);
    case 32: return launch_out<32, false>(a, t, m, kind, p.tiles, p.split, stream);
    case 64: return launch_out<64, false>(a, t, m, kind, p.tiles, p.split, stream);
    default: return launch_out<128, false>(a, t, m, kind, p.tiles, p.split, stream);
  }
}

}  // namespace approxifer
