// Arrays to their 4-bit microscaled form and back.
//
// Everything is exact but the one rounding to four bits (a scale is a power of two): the result is the same in whatever order.
// One pass, bound by HBM: half a warp has 128 neighbours of a row (16 bytes of bfloat16, 32 of fp32 a lane, four lanes to a group),
// kAhead such pieces in flight, and writes 64 bytes of codes and the four scale bytes of the row in its block together.
#include "mx.cuh"

namespace approxifer {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;
constexpr int kPieces = kThreads / 16 * kAhead;  // to a CTA

struct MxArgs {
  approxifer_mx_array_args a;
  uint32_t cols, pieces;  // pieces of 128 to a row; in all, rows up to whole blocks
};

// What a piece's lane has: row, column, where its scales go.
struct Piece {
  uint32_t row, piece;
  int64_t col;
  __device__ __forceinline__ Piece(const MxArgs& g, uint32_t x, int at) : row(x / g.cols), piece(x % g.cols), col((int64_t)piece * kMxCols + at * 8) {}
  __device__ __forceinline__ uint32_t* scales(const MxArgs& g) const {
    return reinterpret_cast<uint32_t*>(g.a.scales + ((int64_t)(row / kMxRows) * g.cols + piece) * kMxBlock + (row % 32) * 16 + (row / 32 % 4) * 4);
  }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const __grid_constant__ MxArgs g) {
  const int at = threadIdx.x % 16;
  const uint32_t x0 = blockIdx.x * kPieces + threadIdx.x / 16;
  let_next_start();
  wait_for_inputs();
  MxRow<T> v[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const uint32_t x = x0 + i * (kThreads / 16);
    const Piece p(g, x, at);
    v[i].none();
    if (x < g.pieces && p.row < g.a.M && p.col < g.a.K) v[i].template load<VEC>(static_cast<const T*>(g.a.X) + (int64_t)p.row * g.a.x_rstride + p.col);
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const uint32_t x = x0 + i * (kThreads / 16);
    const Piece p(g, x, at);
    uint32_t byte;
    const uint32_t codes = mx_quantize8(v[i].widened(), &byte);
    // the bytes of the piece's four groups, of which lane 4 k has that of group k
    uint32_t word = byte << (8 * (at / 4));
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if (x >= g.pieces) continue;
    if (at == 0) *p.scales(g) = word;
    if (p.row < g.a.M && p.col < g.a.K) *reinterpret_cast<uint32_t*>(g.a.codes + (int64_t)p.row * g.a.c_rstride + p.col / 2) = codes;
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const __grid_constant__ MxArgs g) {
  const int at = threadIdx.x % 16;
  const uint32_t x0 = blockIdx.x * kPieces + threadIdx.x / 16;
  let_next_start();
  wait_for_inputs();
  uint32_t codes[kAhead], word[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const uint32_t x = x0 + i * (kThreads / 16);
    const Piece p(g, x, at);
    codes[i] = word[i] = 0;
    if (x < g.pieces && p.row < g.a.M && p.col < g.a.K) {
      codes[i] = __ldcs(reinterpret_cast<const uint32_t*>(g.a.codes + (int64_t)p.row * g.a.c_rstride + p.col / 2));
      word[i] = __ldg(p.scales(g));
    }
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const uint32_t x = x0 + i * (kThreads / 16);
    const Piece p(g, x, at);
    if (x >= g.pieces || p.row >= g.a.M || p.col >= g.a.K) continue;
    const float k = mx_value(word[i] >> (8 * (at / 4)) & 255);
    uint32_t h[4];
    mx_halves(codes[i], h);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
      v[2 * e] = f.x * k, v[2 * e + 1] = f.y * k;
    }
    T* to = static_cast<T*>(g.a.X) + (int64_t)p.row * g.a.x_rstride + p.col;
    if constexpr (!VEC) {
#pragma unroll
      for (int e = 0; e < 8; ++e) to[e] = narrow<T>(v[e]);
    } else if constexpr (sizeof(T) == 2) {
      __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
    } else {
      __stcs(reinterpret_cast<float4*>(to), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(to) + 1, make_float4(v[4], v[5], v[6], v[7]));
    }
  }
}

cudaError_t launch(const approxifer_mx_array_args& a, bool rows_of_blocks, cudaStream_t stream, void (*whole32)(MxArgs), void (*whole16)(MxArgs), void (*any32)(MxArgs),
                   void (*any16)(MxArgs)) {
  MxArgs g{a, 0, 0};
  const int64_t cols = (a.K + kMxCols - 1) / kMxCols, rows = rows_of_blocks ? (a.M + kMxRows - 1) / kMxRows * kMxRows : a.M;
  if (rows > 0x7fffffffLL / cols) return cudaErrorInvalidConfiguration;  // (2^38 elements: more than the device holds)
  g.cols = (uint32_t)cols, g.pieces = (uint32_t)(rows * cols);
  const bool f32 = a.type == APPROXIFER_TYPE_F32, whole = aligned16(a.X) && a.x_rstride % (f32 ? 4 : 8) == 0;
  const int64_t blocks = ((int64_t)g.pieces + kPieces - 1) / kPieces;
  return launch_kernel(whole ? (f32 ? whole32 : whole16) : (f32 ? any32 : any16), blocks, kThreads, 0, 1, stream, g);
}

}  // namespace

cudaError_t launch_mx_quantize(const approxifer_mx_array_args& a, cudaStream_t stream) {
  return launch(a, true, stream, mx_quantize_kernel<float, true>, mx_quantize_kernel<bf16, true>, mx_quantize_kernel<float, false>, mx_quantize_kernel<bf16, false>);
}
cudaError_t launch_mx_dequantize(const approxifer_mx_array_args& a, cudaStream_t stream) {
  return launch(a, false, stream, mx_dequantize_kernel<float, true>, mx_dequantize_kernel<bf16, true>, mx_dequantize_kernel<float, false>, mx_dequantize_kernel<bf16, false>);
}

}  // namespace approxifer
