// Per-head norm of queries and keys with the position rotation, keys and values written to the paged cache.
#include "hosted.cuh"

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

// The path for whole 16-byte columns: one pass over HBM.  A head's row is spread over L lanes (the power of two that holds
// its columns), a warp takes 32 / L rows at a time, kAhead of those loaded together and kBatches of these one after the
// other, all of one token and of one kind (queries, keys or values), so that the cosines, sines and weights are read once
// for many rows:
//     y_d = r (x_d A_d + x_p(d) B_d),    A_d = w_d cos,  B_d = -+ w_p(d) sin,   p(d) the other element of d's pair,
// with r the reciprocal root mean square of the row.  The pair's other element comes from another lane (halves) or from
// the lane's own column (neighbouring pairs).
constexpr int kThreads = 128;
constexpr int kAhead = 4;
constexpr int kBatches = 1;

template <typename T>
struct Column;
template <>
struct Column<bf16> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void get(const uint4& u, uint64_t (&x)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 put(const uint64_t (&x)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      unpack2(x[i], lo, hi);
      w[i] = pack_bf16x2(lo, hi);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Column<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void get(const uint4& u, uint64_t (&x)[2]) {
    x[0] = pack2(__uint_as_float(u.x), __uint_as_float(u.y)), x[1] = pack2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 put(const uint64_t (&x)[2]) {
    float a, b, c, d;
    unpack2(x[0], a, b), unpack2(x[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
};

template <typename T, int L>
__global__ void __launch_bounds__(kThreads, 8) norm_rope_kernel(const __grid_constant__ approxifer_norm_rope_args a, int q_units, int kv_units) {
  constexpr int E = Column<T>::kElems, kSide = 32 / L;  // elements of a column, rows side by side
  const int lane = threadIdx.x % 32, at = lane % L, side = lane / L;
  const int units = q_units + (a.k ? kv_units : 0) + (a.v ? kv_units : 0);
  const int64_t u = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  if (u >= a.T * units) return;
  const int64_t t = a.T < (1 << 24) && units < 128 ? (uint32_t)u / (uint32_t)units : u / units;
  int unit = (int)(u - t * units);
  const bool is_q = unit < q_units, is_k = !is_q && a.k && unit < q_units + kv_units;
  const bool head_unit = unit == 0;
  unit -= is_q ? 0 : is_k || !a.k ? q_units : q_units + kv_units;
  const int heads = is_q ? a.Hq : a.Hkv, h0 = unit * (kSide * kAhead * kBatches) + side;
  const T* in = is_q ? static_cast<const T*>(a.q) + t * a.q_tstride : is_k ? static_cast<const T*>(a.k) + t * a.k_tstride : static_cast<const T*>(a.v) + t * a.v_tstride;
  const int64_t in_h = is_q ? a.q_hstride : is_k ? a.k_hstride : a.v_hstride;
  const int d0 = at * E;
  const bool live = d0 < a.D;
  uint4 x[kAhead];
  auto load = [&](int batch) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + (batch * kAhead + i) * kSide;
      x[i] = live && h < heads ? __ldcs(reinterpret_cast<const uint4*>(in + h * in_h + d0)) : make_uint4(0, 0, 0, 0);
    }
  };
  load(0);
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
    int64_t page, row;
    if (slot < (1LL << 31)) {
      page = (uint32_t)slot / (uint32_t)a.page_size;
      row = (uint32_t)slot - (uint32_t)page * (uint32_t)a.page_size;
    } else {
      page = slot / a.page_size;
      row = slot % a.page_size;
    }
    out = is_k ? static_cast<T*>(a.k_cache) + page * a.kc_pstride + row * a.kc_rstride : static_cast<T*>(a.v_cache) + page * a.vc_pstride + row * a.vc_rstride;
    out_h = is_k ? a.kc_hstride : a.vc_hstride;
  }
  if (!is_q && !is_k) {
    for (int batch = 0; batch < kBatches; ++batch) {
      if (batch) load(batch);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + (batch * kAhead + i) * kSide;
        if (live && h < heads) *reinterpret_cast<uint4*>(out + h * out_h + d0) = x[i];
      }
    }
    return;
  }
  if (!placed) {  // (queries: keys have left above)
    for (int h = h0; h < min(heads, h0 + kAhead * kBatches * kSide); h += kSide)
      if (live) *reinterpret_cast<uint4*>(out + h * out_h + d0) = make_uint4(0, 0, 0, 0);
    return;
  }

  // A, B of this lane's elements, and the lane that holds their pairs
  const T* weight = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
  const int half = a.rot / 2;
  const bool turned = d0 < a.rot, second = d0 >= half;
  const int partner = (turned && !a.interleaved) ? (second ? d0 - half : d0 + half) : d0;
  const int from = side * L + partner / E;
  uint64_t A[E / 2], B[E / 2];
  {
    uint64_t w[E / 2], wp[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) w[e] = wp[e] = pack2(1.f, 1.f);
    if (weight && live) {
      Column<T>::get(__ldg(reinterpret_cast<const uint4*>(weight + d0)), w);
      Column<T>::get(__ldg(reinterpret_cast<const uint4*>(weight + partner)), wp);
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) A[e] = w[e], B[e] = 0;
    if (turned) {
      const float* cs = a.cos_sin + (int64_t)pos * a.rot + (a.interleaved ? d0 / 2 : second ? d0 - half : d0);
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float c = __ldg(cs + e), s = __ldg(cs + half + e);
          float x, y;
          unpack2(wp[e], x, y);
          A[e] = mul2(w[e], pack2(c, c)), B[e] = pack2(-y * s, x * s);
        }
      } else {
        const float sign = second ? 1.f : -1.f;
#pragma unroll
        for (int e = 0; e < E / 2; e += 2) {
          const float4 c = __ldg(reinterpret_cast<const float4*>(cs + 2 * e)), s = __ldg(reinterpret_cast<const float4*>(cs + half + 2 * e));
          A[e] = mul2(w[e], pack2(c.x, c.y)), A[e + 1] = mul2(w[e + 1], pack2(c.z, c.w));
          B[e] = mul2(wp[e], pack2(sign * s.x, sign * s.y)), B[e + 1] = mul2(wp[e + 1], pack2(sign * s.z, sign * s.w));
        }
      }
    }
  }
  const float inv_d = 1.f / (float)a.D;
#pragma unroll 1
  for (int batch = 0; batch < kBatches; ++batch) {
    if (batch) load(batch);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + (batch * kAhead + i) * kSide;
      if (h - side >= heads) break;  // (the whole warp)
      uint64_t v[E / 2], p[E / 2], sq2 = 0;
      Column<T>::get(x[i], v);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) sq2 = fma2(v[e], v[e], sq2);
      float sq, sq_hi;
      unpack2(sq2, sq, sq_hi);
      sq += sq_hi;
#pragma unroll
      for (int d = L / 2; d > 0; d >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, d);
      const float r = weight ? rsqrtf(sq * inv_d + a.eps) : 1.f;
      uint4 other = x[i];
      if (!a.interleaved) {
        other.x = __shfl_sync(0xffffffffu, other.x, from), other.y = __shfl_sync(0xffffffffu, other.y, from);
        other.z = __shfl_sync(0xffffffffu, other.z, from), other.w = __shfl_sync(0xffffffffu, other.w, from);
      }
      if (!turned) other = make_uint4(0, 0, 0, 0);  // (an element that is not turned has no part in a pair, even where it is infinite)
      Column<T>::get(other, p);
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          float lo, hi;
          unpack2(p[e], lo, hi);
          p[e] = pack2(hi, lo);
        }
      }
      const uint64_t r2 = pack2(r, r);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) v[e] = mul2(r2, fma2(v[e], A[e], mul2(p[e], B[e])));
      if (live && h < heads) *reinterpret_cast<uint4*>(out + h * out_h + d0) = Column<T>::put(v);
    }
  }
}

template <typename T>
bool columns_fit(const approxifer_norm_rope_args& a) {
  constexpr int E = Column<T>::kElems;
  const int64_t strides = a.q_tstride | a.q_hstride | a.qo_tstride | a.qo_hstride | (a.k ? a.k_tstride | a.k_hstride | a.kc_pstride | a.kc_hstride | a.kc_rstride : 0) |
                          (a.v ? a.v_tstride | a.v_hstride | a.vc_pstride | a.vc_hstride | a.vc_rstride : 0);
  return a.D % E == 0 && a.D / E <= 32 && (a.interleaved ? a.rot % E == 0 : a.rot % (2 * E) == 0) && strides % E == 0 && aligned16(a.q) && aligned16(a.q_out) &&
         aligned16(a.k) && aligned16(a.v) && aligned16(a.k_cache) && aligned16(a.v_cache) && aligned16(a.q_weight) && aligned16(a.k_weight) && aligned16(a.cos_sin);
}

template <typename T, int L>
cudaError_t launch_columns(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  constexpr int kRowsPerUnit = (32 / L) * kAhead * kBatches;
  const int q_units = (a.Hq + kRowsPerUnit - 1) / kRowsPerUnit, kv_units = (a.Hkv + kRowsPerUnit - 1) / kRowsPerUnit;
  const int64_t warps = a.T * (q_units + (a.k ? kv_units : 0) + (a.v ? kv_units : 0)), blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  norm_rope_kernel<T, L><<<(unsigned)blocks, kThreads, 0, stream>>>(a, q_units, kv_units);
  count_launch();
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const approxifer_norm_rope_args& a, cudaStream_t stream) {
  if (columns_fit<T>(a)) {
    const int columns = a.D / Column<T>::kElems;
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
