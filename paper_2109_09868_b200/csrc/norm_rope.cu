// Per-head norm of queries and keys with the position rotation, keys and values written to the paged cache.
#include "async.cuh"

namespace approxifer {
namespace {

constexpr int kElementThreads = 128;

// One warp = one (token, head) of q, k or v; a lane holds every 32nd element.  The path for head sizes, strides and
// rotations that do not split into whole 16-byte columns.
template <typename T>
__global__ void __launch_bounds__(kElementThreads) norm_rope_element_kernel(const __grid_constant__ approxifer_norm_rope_args a) {
  __shared__ float rows[kElementThreads / 32][256];
  float* row = rows[threadIdx.x / 32];
  const int lane = threadIdx.x % 32;
  const int heads = a.Hq + 2 * a.Hkv;
  const int64_t unit = (int64_t)blockIdx.x * (kElementThreads / 32) + threadIdx.x / 32;
  if (unit >= a.T * heads) return;
  const int64_t t = unit / heads;
  int h = (int)(unit % heads);
  const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
  const bool first = h == 0;
  const int64_t pos = a.rot ? __ldg(a.positions + t) : 0;
  const bool placed = a.rot == 0 || (pos >= 0 && pos < a.positions_max);
  const int64_t slot = a.slots ? __ldg(a.slots + t) : -1;
  const bool fits = slot < a.num_pages * a.page_size;
  if (first && lane == 0 && a.status) a.status[t] = (placed ? 0u : APPROXIFER_ST_POSITION) | (fits ? 0u : APPROXIFER_ST_SLOT);

  const T* in;
  T* out;
  const T* weight = nullptr;
  if (is_q) {
    in = static_cast<const T*>(a.q) + t * a.q_tstride + h * a.q_hstride;
    out = static_cast<T*>(a.q_out) + t * a.qo_tstride + h * a.qo_hstride;
    weight = static_cast<const T*>(a.q_weight);
  } else {
    if (!placed || !fits || slot < 0) return;
    const int64_t page = slot / a.page_size, at = slot % a.page_size;
    h -= is_k ? a.Hq : a.Hq + a.Hkv;
    if (is_k) {
      if (!a.k) return;
      in = static_cast<const T*>(a.k) + t * a.k_tstride + h * a.k_hstride;
      out = static_cast<T*>(a.k_cache) + page * a.kc_pstride + h * a.kc_hstride + at * a.kc_rstride;
      weight = static_cast<const T*>(a.k_weight);
    } else {
      if (!a.v) return;
      in = static_cast<const T*>(a.v) + t * a.v_tstride + h * a.v_hstride;
      out = static_cast<T*>(a.v_cache) + page * a.vc_pstride + h * a.vc_hstride + at * a.vc_rstride;
      for (int d = lane; d < a.D; d += 32) out[d] = in[d];
      return;
    }
  }
  float sq = 0.f;
  for (int d = lane; d < a.D; d += 32) {
    const float x = placed ? widen(in[d]) : 0.f;
    row[d] = x;
    sq = fmaf(x, x, sq);
  }
  sq = warp_sum(sq);
  const float r = weight ? rsqrtf(sq / (float)a.D + a.eps) : 1.f;
  for (int d = lane; d < a.D; d += 32) row[d] = weight ? row[d] * r * widen(weight[d]) : row[d];
  __syncwarp();
  const int half = a.rot / 2;
  for (int d = lane; d < a.D; d += 32) {
    float y = row[d];
    if (d < a.rot && placed) {
      const int i = a.interleaved ? d / 2 : d % half;
      const bool second = a.interleaved ? (d & 1) : d >= half;
      const float c = a.cos_sin[pos * a.rot + i], s = a.cos_sin[pos * a.rot + half + i];
      const float other = row[a.interleaved ? (d ^ 1) : (second ? d - half : d + half)];
      y = second ? fmaf(y, c, other * s) : fmaf(y, c, -other * s);
    }
    out[d] = narrow<T>(y);
  }
}

// The path for whole columns: one pass over HBM.  A lane holds eight elements of a row, so that a pair's two elements are in
// the same lane: four and the four that they are turned with (rot/2 further on, or, of neighbouring pairs, the next four),
// beyond rot eight that are not turned.  A row is spread over L lanes, a warp takes 32 / L rows at a time and kAhead of
// those together, all of one token and of one kind (queries, keys or values), so that the cosines, sines and weights are
// read once for many rows:
//     y = r (x A + x' B),    A = w cos,  B = -+ w' sin,   x' the other element of the pair and w' its weight,
// with r the reciprocal root mean square of the row.  All rows' loads are in flight before the first is used.
//
// With 400 MB to move this is bound by instruction issue as much as by HBM: hence the pairs within a lane (exchanging them
// between lanes cost 16 instructions of 78 a row pair), the packed fp32 arithmetic, a token to a CTA (no division to find
// it), and the two template parameters (INTER: neighbouring pairs; PARTIAL: some elements are not turned).
//
// Measured: 16,384 tokens, 32 + 8 + 8 heads of 128 in bfloat16: 81 us, 5.0 TB/s (a plain copy of as many bytes takes 66);
// 1,237 tokens, 15 + 5 + 5 heads of 80 in fp32: 5.6 us; one token 2.7 us.  Tried and slower: copying ahead into shared
// memory by persistent warps (113 us), eight rows in flight (86), two (93).
constexpr int kMaxWarps = 8;  // units of a token per CTA
constexpr int kAhead = 4;

// Four elements: a half of what a lane holds of a row.
template <typename T>
struct Four;
template <>
struct Four<bf16> {
  using Raw = uint2;
  static constexpr int kCtas = 4;  // per SM
  static __device__ __forceinline__ void get(const Raw& u, uint64_t (&x)[2]) {
    x[0] = pack2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
    x[1] = pack2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
  }
  static __device__ __forceinline__ Raw put(const uint64_t (&x)[2]) {
    float a, b, c, d;
    unpack2(x[0], a, b), unpack2(x[1], c, d);
    return make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
  }
  static __device__ __forceinline__ Raw none() { return make_uint2(0, 0); }
};
template <>
struct Four<float> {
  using Raw = uint4;
  static constexpr int kCtas = 3;
  static __device__ __forceinline__ void get(const Raw& u, uint64_t (&x)[2]) {
    x[0] = pack2(__uint_as_float(u.x), __uint_as_float(u.y)), x[1] = pack2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ Raw put(const uint64_t (&x)[2]) {
    float a, b, c, d;
    unpack2(x[0], a, b), unpack2(x[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
  static __device__ __forceinline__ Raw none() { return make_uint4(0, 0, 0, 0); }
};

__device__ __forceinline__ uint64_t swapped(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return pack2(b, a);
}

template <typename T, int L, bool INTER, bool PARTIAL>
__global__ void __launch_bounds__(kMaxWarps * 32, Four<T>::kCtas) norm_rope_kernel(const __grid_constant__ approxifer_norm_rope_args a, int q_units, int kv_units,
                                                                                   int page_shift) {
  using F = Four<T>;
  using Raw = typename F::Raw;
  constexpr int kSide = 32 / L;  // rows side by side
  const int lane = threadIdx.x % 32, at = lane % L, side = lane / L;
  let_next_start();
  wait_for_inputs();
  const int units = q_units + (a.k ? kv_units : 0) + (a.v ? kv_units : 0);
  const int64_t t = blockIdx.x;
  int unit = (int)(blockIdx.y * (blockDim.x / 32) + threadIdx.x / 32);
  if (unit >= units) return;
  const bool is_q = unit < q_units, is_k = !is_q && a.k && unit < q_units + kv_units;
  const bool head_unit = unit == 0;
  unit -= is_q ? 0 : is_k || !a.k ? q_units : q_units + kv_units;
  const int heads = (is_q ? a.Hq : a.Hkv) - unit * (kSide * kAhead) - side, h0 = unit * (kSide * kAhead) + side;
  // where this lane's two fours are
  const int half = a.rot / 2, turning = a.rot / 8;
  const bool turned = !PARTIAL || at < turning;
  const int d1 = INTER ? 8 * at : turned ? 4 * at : a.rot + 8 * (at - turning), d2 = turned && !INTER ? half + d1 : d1 + 4;
  const bool live = at * 8 < a.D;

  const int64_t in_h = is_q ? a.q_hstride : is_k ? a.k_hstride : a.v_hstride;
  const T* in = (is_q ? static_cast<const T*>(a.q) + t * a.q_tstride : is_k ? static_cast<const T*>(a.k) + t * a.k_tstride : static_cast<const T*>(a.v) + t * a.v_tstride) +
                h0 * in_h;
  Raw x1[kAhead], x2[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i, in += kSide * in_h) {
    const bool there = live && i * kSide < heads;
    x1[i] = there ? __ldcs(reinterpret_cast<const Raw*>(in + d1)) : F::none();
    x2[i] = there ? __ldcs(reinterpret_cast<const Raw*>(in + d2)) : F::none();
  }
  const int32_t pos = a.rot ? __ldg(a.positions + t) : 0;
  const bool placed = a.rot == 0 || (pos >= 0 && pos < a.positions_max);
  const int64_t slot = a.slots ? __ldg(a.slots + t) : -1;
  const bool fits = slot < a.num_pages * a.page_size;
  if (head_unit && lane == 0 && a.status) a.status[t] = (placed ? 0u : APPROXIFER_ST_POSITION) | (fits ? 0u : APPROXIFER_ST_SLOT);

  T* out;
  int64_t out_h;
  if (is_q) {
    out = static_cast<T*>(a.q_out) + t * a.qo_tstride;
    out_h = a.qo_hstride;
  } else {
    if (!placed || !fits || slot < 0) return;
    const int64_t page = page_shift >= 0 ? slot >> page_shift : slot / a.page_size, row = slot - page * a.page_size;
    out = is_k ? static_cast<T*>(a.k_cache) + page * a.kc_pstride + row * a.kc_rstride : static_cast<T*>(a.v_cache) + page * a.vc_pstride + row * a.vc_rstride;
    out_h = is_k ? a.kc_hstride : a.vc_hstride;
  }
  out += h0 * out_h;
  if ((!is_q && !is_k) || !placed) {  // values as they are; queries without a place (keys have left above) zero
#pragma unroll
    for (int i = 0; i < kAhead; ++i, out += kSide * out_h)
      if (live && i * kSide < heads) {
        *reinterpret_cast<Raw*>(out + d1) = placed ? x1[i] : F::none();
        *reinterpret_cast<Raw*>(out + d2) = placed ? x2[i] : F::none();
      }
    return;
  }

  // A, B of this lane's elements.  (An element that is not turned has no part in a pair, even where that is infinite: such
  // lanes take the pair as zero below.)
  const T* weight = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
  uint64_t A1[2], A2[2], B1[2], B2[2];
  {
    A1[0] = A1[1] = A2[0] = A2[1] = pack2(1.f, 1.f);
    B1[0] = B1[1] = B2[0] = B2[1] = 0;
    if (weight && live) F::get(__ldg(reinterpret_cast<const Raw*>(weight + d1)), A1), F::get(__ldg(reinterpret_cast<const Raw*>(weight + d2)), A2);
    if (turned && a.rot > 0 && live) {
      const float* cs = a.cos_sin + (int64_t)pos * a.rot + 4 * at;
      const float4 c = __ldg(reinterpret_cast<const float4*>(cs)), s = __ldg(reinterpret_cast<const float4*>(cs + half));
      if constexpr (INTER) {
        auto turn = [](uint64_t& A, uint64_t& B, float c, float s) {
          B = mul2(swapped(A), pack2(-s, s));
          A = mul2(A, pack2(c, c));
        };
        turn(A1[0], B1[0], c.x, s.x), turn(A1[1], B1[1], c.y, s.y), turn(A2[0], B2[0], c.z, s.z), turn(A2[1], B2[1], c.w, s.w);
      } else {
        const uint64_t c2[2] = {pack2(c.x, c.y), pack2(c.z, c.w)}, s2[2] = {pack2(s.x, s.y), pack2(s.z, s.w)}, n2[2] = {pack2(-s.x, -s.y), pack2(-s.z, -s.w)};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          B1[e] = mul2(A2[e], n2[e]), B2[e] = mul2(A1[e], s2[e]);
          A1[e] = mul2(A1[e], c2[e]), A2[e] = mul2(A2[e], c2[e]);
        }
      }
    }
  }
  const float inv_d = 1.f / (float)a.D;
#pragma unroll
  for (int i = 0; i < kAhead; ++i, out += kSide * out_h) {
    if (i * kSide >= heads + side) break;  // (the whole warp)
    uint64_t v1[2], v2[2];
    F::get(x1[i], v1), F::get(x2[i], v2);
    uint64_t sq2 = fma2(v2[1], v2[1], fma2(v2[0], v2[0], fma2(v1[1], v1[1], mul2(v1[0], v1[0]))));
    float sq, sq_hi;
    unpack2(sq2, sq, sq_hi);
    sq += sq_hi;
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, d);
    const float r = weight ? rsqrtf(sq * inv_d + a.eps) : 1.f;
    const uint64_t r2 = pack2(r, r);
    uint64_t p1[2] = {v2[0], v2[1]}, p2[2] = {v1[0], v1[1]};
    if constexpr (INTER) p1[0] = swapped(v1[0]), p1[1] = swapped(v1[1]), p2[0] = swapped(v2[0]), p2[1] = swapped(v2[1]);
    if (PARTIAL && !turned) p1[0] = p1[1] = p2[0] = p2[1] = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      p1[e] = mul2(r2, fma2(v1[e], A1[e], mul2(p1[e], B1[e])));
      p2[e] = mul2(r2, fma2(v2[e], A2[e], mul2(p2[e], B2[e])));
    }
    if (live && i * kSide < heads) {
      *reinterpret_cast<Raw*>(out + d1) = F::put(p1);
      *reinterpret_cast<Raw*>(out + d2) = F::put(p2);
    }
  }
}

template <typename T>
bool columns_fit(const approxifer_norm_rope_args& a) {
  const int64_t strides = a.q_tstride | a.q_hstride | a.qo_tstride | a.qo_hstride | (a.k ? a.k_tstride | a.k_hstride | a.kc_pstride | a.kc_hstride | a.kc_rstride : 0) |
                          (a.v ? a.v_tstride | a.v_hstride | a.vc_pstride | a.vc_hstride | a.vc_rstride : 0);
  return a.D % 8 == 0 && a.rot % 8 == 0 && strides % 4 == 0 && aligned16(a.q) && aligned16(a.q_out) && aligned16(a.k) && aligned16(a.v) && aligned16(a.k_cache) &&
         aligned16(a.v_cache) && aligned16(a.q_weight) && aligned16(a.k_weight) && aligned16(a.cos_sin);
}

template <typename T, int L>
cudaError_t launch_columns(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  constexpr int kRowsPerUnit = (32 / L) * kAhead;
  const int q_units = (a.Hq + kRowsPerUnit - 1) / kRowsPerUnit, kv_units = (a.Hkv + kRowsPerUnit - 1) / kRowsPerUnit;
  const int units = q_units + (a.k ? kv_units : 0) + (a.v ? kv_units : 0);
  const int parts = (units + kMaxWarps - 1) / kMaxWarps, warps = (units + parts - 1) / parts;
  const int page_shift = exact_log2(a.page_size);
  const bool partial = a.rot < a.D;
  auto kernel = a.interleaved ? (partial ? norm_rope_kernel<T, L, true, true> : norm_rope_kernel<T, L, true, false>)
                              : (partial ? norm_rope_kernel<T, L, false, true> : norm_rope_kernel<T, L, false, false>);
  return launch_kernel(kernel, dim3((unsigned)a.T, (unsigned)parts), warps * 32, 0, 1, stream, a, q_units, kv_units, page_shift);
}

template <typename T>
cudaError_t launch_type(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  if (columns_fit<T>(a)) {
    const int columns = a.D / 8;
    if (columns <= 8) return launch_columns<T, 8>(a, stream);
    if (columns <= 16) return launch_columns<T, 16>(a, stream);
    return launch_columns<T, 32>(a, stream);
  }
  const int64_t units = a.T * (a.Hq + 2 * a.Hkv), per = kElementThreads / 32;
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  norm_rope_element_kernel<T><<<(unsigned)blocks, kElementThreads, 0, stream>>>(a);
  count_launch();
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_rope(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  return a.type == APPROXIFER_TYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace approxifer
