// Matrix product with bias, activation and residual for up to eight rows of X (single tokens): Wt is read once, and how soon
// the first of its bytes are asked for and the last are summed up is most of the time.
//
// A CTA takes 16 rows of Wt, its eight warps 128 columns of K each in turn (2 KB of every row side by side).  Nothing is
// staged: in mma.m16n8k16 the sum over k may be taken in any order as long as both operands agree on it, so a lane's eight
// consecutive elements of a row (one 16-byte load) serve as its share of two products -- of Wt's rows g and g + 8 as the
// first operand, of X's row g as the second (lane = 4 g + t).  The next 128 columns are on their way while these are
// multiplied.  The warps' sums meet in shared memory, in order.  (No barriers, no tensor memory to set up, and room for two
// CTAs and the next call's on an SM: a tensor-core tile that is nearly all padding would be waited for longer than it works.)
//
// Measured: 1 x 4,096 x 4,096 with residual 8.2 us, 4.1 TB/s, bound by HBM and the two ends of the call.
#include "async.cuh"

namespace approxifer {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 16;       // of Wt
constexpr int kMost = 8;        // rows of X
constexpr int kSteps = 4;       // of 32 columns, per warp and turn
constexpr int kColumns = kSteps * 32;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename Out>
__global__ void __launch_bounds__(kThreads, 2) linear_few_kernel(const __grid_constant__ approxifer_linear_args a) {
  __shared__ float sums[kWarps][kRows][kMost + 1];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  let_next_start();
  wait_for_inputs();
  const int64_t n0 = (int64_t)blockIdx.x * kRows;
  const bf16* w0 = reinterpret_cast<const bf16*>(a.Wt) + (n0 + g) * a.w_rstride;
  const bf16* w1 = w0 + 8 * a.w_rstride;
  const bf16* x = reinterpret_cast<const bf16*>(a.X) + g * a.x_rstride;
  const bool has0 = n0 + g < a.N, has1 = n0 + g + 8 < a.N, has_x = g < a.M;
  const uint4 none = make_uint4(0, 0, 0, 0);
  struct Turn {
    uint4 w0[kSteps], w1[kSteps], x[kSteps];
  };
  auto load = [&](Turn& v, int64_t k0) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int64_t k = k0 + s * 32 + t * 8;
      const bool in = k < a.K;
      v.w0[s] = in && has0 ? __ldcs(reinterpret_cast<const uint4*>(w0 + k)) : none;
      v.w1[s] = in && has1 ? __ldcs(reinterpret_cast<const uint4*>(w1 + k)) : none;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int64_t k = k0 + s * 32 + t * 8;
      v.x[s] = k < a.K && has_x ? __ldg(reinterpret_cast<const uint4*>(x + k)) : none;
    }
  };
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  Turn now, next;
  int64_t k0 = (int64_t)warp * kColumns;
  load(now, k0);
  for (; k0 < a.K; k0 += kWarps * kColumns) {
    load(next, k0 + kWarps * kColumns);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      mma16816(acc, now.w0[s].x, now.w1[s].x, now.w0[s].y, now.w1[s].y, now.x[s].x, now.x[s].y);
      mma16816(acc, now.w0[s].z, now.w1[s].z, now.w0[s].w, now.w1[s].w, now.x[s].z, now.x[s].w);
    }
    now = next;
  }
  sums[warp][g][2 * t] = acc[0], sums[warp][g][2 * t + 1] = acc[1];
  sums[warp][g + 8][2 * t] = acc[2], sums[warp][g + 8][2 * t + 1] = acc[3];
  __syncthreads();
  const int row = threadIdx.x % kRows, m = threadIdx.x / kRows;
  const int64_t n = n0 + row;
  if (m >= a.M || n >= a.N) return;
  float y = sums[0][row][m];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) y += sums[w][row][m];
  if (a.bias) y += widen(reinterpret_cast<const bf16*>(a.bias)[n]);
  y = activate<Out>(a.activation, y);
  if (a.R) y += widen(static_cast<const Out*>(a.R)[m * a.r_rstride + n]);
  static_cast<Out*>(a.Y)[m * a.y_rstride + n] = narrow<Out>(y);
}

}  // namespace

// Where all CTAs run at once and K is not so long that eight warps are too few to read it.  Measured, tile kernel against this
// one, us, one row of X: 10 x 784 4.6 / 2.1, 1,000 x 1,024 4.7 / 2.7, 4,096 x 4,096 10.3 / 8.2, 4,096 x 8,192 15.2 / 14.2,
// 4,600 x 4,096 11.5 / 8.8; beyond: 1,000 x 16,384 12 / 18, 8,192 x 4,096 14.6 / 16.4, 16,384 x 4,096 24 / 30.
bool linear_few_wanted(const approxifer_linear_args& a, int sms) { return a.M <= kMost && a.K % 8 == 0 && a.K <= 8192 && a.N <= 2LL * sms * kRows; }

cudaError_t launch_linear_few(const approxifer_linear_args& a, cudaStream_t stream) {
  const int64_t blocks = (a.N + kRows - 1) / kRows;
  return a.out_type == APPROXIFER_TYPE_F32 ? launch_kernel(linear_few_kernel<float>, blocks, kThreads, 0, 1, stream, a)
                                           : launch_kernel(linear_few_kernel<bf16>, blocks, kThreads, 0, 1, stream, a);
}

}  // namespace approxifer
