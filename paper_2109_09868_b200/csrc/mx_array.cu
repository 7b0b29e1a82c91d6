// Arrays to their 4-bit microscaled form and back.
//
// Everything is exact but the one rounding to four bits (a scale is a power of two): the result is the same in whatever order.
// One pass, bound by HBM and by the issue of its instructions.  There: eight lanes have 128 neighbours of a row (sixteen a lane, two
// lanes to a group), two such pieces in flight, and write 64 bytes of codes and the four scale bytes of the row in its block together.
// Back: sixteen lanes have them, four pieces in flight, so that what is written, the most, goes out in whole lines.  16,384 x 4,096 in
// bfloat16, there 28 us, 6.0 TB/s (eight elements a lane 40 us: 126 instructions for them), back 31 us, 5.5 TB/s (sixteen 36 us).
#include "mx.cuh"

namespace approxifer {
namespace {

constexpr int kThreads = 256;
constexpr int kThere = 8, kBack = 16;             // lanes to a piece
constexpr int kPieces = 64;                       // pieces of a CTA
constexpr int side(int lanes) { return kThreads / lanes; }          // side by side
constexpr int ahead(int lanes) { return kPieces / side(lanes); }    // and after each other

struct MxArgs {
  approxifer_mx_array_args a;
  uint32_t cols, rows;     // pieces of 128 to a row; rows, up to whole blocks of them where the scales are written
  uint32_t rows_on, rest;  // what side() pieces further on is: so many rows, so many pieces
};

// A piece: its row, its place in the row.  (One division a thread; from one of its pieces to the next the place is counted on.)
template <int LANES>
struct Piece {
  uint32_t row, piece;
  __device__ __forceinline__ Piece next(const MxArgs& g) const {
    const uint32_t on = piece + g.rest;
    return on >= g.cols ? Piece{row + g.rows_on + 1, on - g.cols} : Piece{row + g.rows_on, on};
  }
  __device__ __forceinline__ int64_t col(int at) const { return (int64_t)piece * kMxCols + at * (kMxCols / LANES); }
  __device__ __forceinline__ bool there(const MxArgs& g, int at) const { return row < g.a.M && col(at) < g.a.K; }
  __device__ __forceinline__ uint32_t* scales(const MxArgs& g) const {
    return reinterpret_cast<uint32_t*>(g.a.scales + ((int64_t)(row / kMxRows) * g.cols + piece) * kMxBlock + (row % 32) * 16 + (row / 32 % 4) * 4);
  }
};
template <int LANES>
__device__ __forceinline__ void find_pieces(const MxArgs& g, Piece<LANES> (&p)[ahead(LANES)]) {
  const uint32_t x = blockIdx.x * kPieces + threadIdx.x / LANES;
  p[0] = Piece<LANES>{x / g.cols, x % g.cols};
#pragma unroll
  for (int i = 1; i < ahead(LANES); ++i) p[i] = p[i - 1].next(g);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const __grid_constant__ MxArgs g) {
  constexpr int kAhead = ahead(kThere);
  const int at = threadIdx.x % kThere;
  let_next_start();
  wait_for_inputs();
  Piece<kThere> p[kAhead];
  MxRow<T> v[kAhead][2];
  find_pieces(g, p);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    v[i][0].none(), v[i][1].none();
    if (p[i].there(g, at)) {
      const T* from = static_cast<const T*>(g.a.X) + p[i].row * g.a.x_rstride + p[i].col(at);
      v[i][0].template load<VEC>(from), v[i][1].template load<VEC>(from + 8);
    }
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    MxEight lo = v[i][0].widened(), hi = v[i][1].widened();
    uint32_t top = max(lo.top, hi.top);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t byte = mx_scale(top);
    uint2 codes = make_uint2(0, 0);
    if (byte != 255) {
      const uint64_t k = pack2(mx_inverse(byte), mx_inverse(byte));
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        unpack2(mul2(pack2(lo.v[e], lo.v[e + 1]), k), lo.v[e], lo.v[e + 1]);
        unpack2(mul2(pack2(hi.v[e], hi.v[e + 1]), k), hi.v[e], hi.v[e + 1]);
      }
      codes = make_uint2(mx_codes(lo.v), mx_codes(hi.v));
    }
    // the bytes of the piece's four groups, of which lane 2 k has that of group k
    uint32_t word = byte << (8 * (at / 2));
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    if (at == 0 && p[i].row < g.rows) *p[i].scales(g) = word;
    if (p[i].there(g, at)) *reinterpret_cast<uint2*>(g.a.codes + p[i].row * g.a.c_rstride + p[i].col(at) / 2) = codes;
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const __grid_constant__ MxArgs g) {
  constexpr int kAhead = ahead(kBack);
  const int at = threadIdx.x % kBack;
  let_next_start();
  wait_for_inputs();
  Piece<kBack> p[kAhead];
  uint32_t codes[kAhead], word[kAhead];
  find_pieces(g, p);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    codes[i] = word[i] = 0;
    if (p[i].there(g, at)) {
      codes[i] = __ldcs(reinterpret_cast<const uint32_t*>(g.a.codes + p[i].row * g.a.c_rstride + p[i].col(at) / 2));
      word[i] = __ldg(p[i].scales(g));
    }
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    if (!p[i].there(g, at)) continue;
    const float k = mx_value(word[i] >> (8 * (at / 4)) & 255);
    uint32_t h[4];
    mx_halves(codes[i], h);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
      v[2 * e] = f.x * k, v[2 * e + 1] = f.y * k;
    }
    T* to = static_cast<T*>(g.a.X) + p[i].row * g.a.x_rstride + p[i].col(at);
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

cudaError_t launch(const approxifer_mx_array_args& a, bool rows_of_blocks, int lanes, cudaStream_t stream, void (*whole32)(MxArgs), void (*whole16)(MxArgs), void (*any32)(MxArgs),
                   void (*any16)(MxArgs)) {
  MxArgs g{a};
  const int64_t cols = (a.K + kMxCols - 1) / kMxCols, rows = rows_of_blocks ? (a.M + kMxRows - 1) / kMxRows * kMxRows : a.M;
  if (rows > 0x7fffffffLL / cols) return cudaErrorInvalidConfiguration;  // (2^38 elements: more than the device holds)
  g.cols = (uint32_t)cols, g.rows = (uint32_t)rows;
  g.rows_on = side(lanes) / g.cols, g.rest = side(lanes) % g.cols;
  const bool f32 = a.type == APPROXIFER_TYPE_F32, whole = aligned16(a.X) && a.x_rstride % (f32 ? 4 : 8) == 0;
  const int64_t blocks = (rows * cols + kPieces - 1) / kPieces;
  return launch_kernel(whole ? (f32 ? whole32 : whole16) : (f32 ? any32 : any16), blocks, kThreads, 0, 1, stream, g);
}

}  // namespace

cudaError_t launch_mx_quantize(const approxifer_mx_array_args& a, cudaStream_t stream) {
  return launch(a, true, kThere, stream, mx_quantize_kernel<float, true>, mx_quantize_kernel<bf16, true>, mx_quantize_kernel<float, false>, mx_quantize_kernel<bf16, false>);
}
cudaError_t launch_mx_dequantize(const approxifer_mx_array_args& a, cudaStream_t stream) {
  return launch(a, false, kBack, stream, mx_dequantize_kernel<float, true>, mx_dequantize_kernel<bf16, true>, mx_dequantize_kernel<float, false>, mx_dequantize_kernel<bf16, false>);
}

}  // namespace approxifer
