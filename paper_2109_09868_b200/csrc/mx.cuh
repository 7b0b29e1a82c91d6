// The 4-bit microscaled form: 32 neighbours of a row share a power of two; see approxifer_mx_quantize in approxifer.h.
#pragma once
#include "async.cuh"

namespace approxifer {

constexpr int kMxGroup = 32;               // elements that share a scale
constexpr int kMxRows = 128, kMxCols = 128;  // elements of a block of scales
constexpr int kMxBlock = 512;              // its bytes

inline int64_t mx_blocks(int64_t rows, int64_t k) { return ((rows + kMxRows - 1) / kMxRows) * ((k + kMxCols - 1) / kMxCols); }

#ifdef __CUDACC__

// The scale's byte for a group whose largest magnitude has the fp32 bits `top` (2^e <= top < 2^(e+1): e - 2 + 127, at least 0;
// an exponent field of zero is a number below 2^-126, whose scale is the smallest one anyway).
__device__ __forceinline__ uint32_t mx_scale(uint32_t top) {
  const uint32_t field = top >> 23;
  return field == 255 ? 255u : field < 2 ? 0u : field - 2;
}
// What a group's elements are multiplied with: 2^(127 - byte), exact, as is the product; of a group with an infinity or a NaN zero.
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// The value of a scale.
__device__ __forceinline__ float mx_value(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7fffffffu : byte == 0 ? 0x00400000u : byte << 23); }

// The activations of the 4-bit products.  The pair kernel's epilogues have some 3 us a tile before the next one's products are over: where
// bfloat16 is what is written (it shows 2^-8), the special-function unit's reciprocal (2^-22) takes the place of a division, and
// of gelu's erf a polynomial times an exponential: with t = 1 / (1 + c |x|), erfc(|x| / sqrt 2) / 2 = t P(t) e^(-x^2/2), P of degree four
// and c fitted (least maximum, by linear programming) so that gelu errs by at most 1.3e-7 (1 + |x|) and, as its result gets small below
// zero, by at most 5.2e-4 of it.  8,192 x 16,384 x 256 with gelu 200 -> 140 us, with gelu_tanh 126 us, with none 84 us.
// (A quotient below 2^-126 becomes zero, with an fp32 output too: results of silu and gelu_tanh below |x| 2^-126.)
__device__ __forceinline__ float mx_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <int ACT, typename Out>
__device__ __forceinline__ float mx_activate(float x) {
  if constexpr (sizeof(Out) == 2 && (ACT == APPROXIFER_ACT_SILU || ACT == APPROXIFER_ACT_GELU_TANH)) {
    // -x log2 e, or -2 sqrt(2/pi) (x + 0.044715 x^3) log2 e
    const float u = ACT == APPROXIFER_ACT_SILU ? -1.4426950409f * x : x * fmaf(-0.1029432396f, x * x, -2.3022081981f);
    return x * mx_reciprocal(1.f + pow2(u));
  }
  if constexpr (sizeof(Out) == 2 && ACT == APPROXIFER_ACT_GELU) {
    // half of erfc(|x| / sqrt 2)
    const float t = mx_reciprocal(fmaf(0.35f, fabsf(x), 1.f));
    const float h = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.098317348f, 0.27671186f), 0.018424226f), 0.16594502f), 0.13723235f) * pow2(-0.7213475204f * x * x);
    return x * (x >= 0.f ? 1.f - h : h);  // (a factor: infinity stays)
  }
  // (fp32: a division of two units' error.  It has no long way, which a correctly rounded one takes for zero and what overflows.)
  if constexpr (ACT == APPROXIFER_ACT_SILU) return __fdividef(x, 1.f + expf(-x));
  if constexpr (ACT == APPROXIFER_ACT_GELU_TANH) return __fdividef(x, 1.f + expf(-1.5957691f * (x + 0.044715f * x * x * x)));
  return activate<ACT, Out>(x);
}

// Eight values (already divided by the scale) as codes, the first in the lowest bits: nearest, ties to even, at most 6.
__device__ __forceinline__ uint32_t mx_codes(const float (&v)[8]) {
  uint32_t d;
  asm("{\n.reg .b8 a, b, c, d;\n"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      "mov.b32 %0, {a, b, c, d};\n}\n"
      : "=r"(d)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return d;
}
// The values of eight codes, two halves to a register.
__device__ __forceinline__ void mx_halves(uint32_t codes, uint32_t (&h)[4]) {
  asm("{\n.reg .b8 a, b, c, d;\n"
      "mov.b32 {a, b, c, d}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
}

// Eight neighbours of a row of bfloat16 or fp32 as they are loaded (so that many loads can be in flight), and widened, with the
// largest of their magnitudes' bits.
struct MxEight {
  float v[8];
  uint32_t top;
};
template <typename T>
struct MxRow;
template <>
struct MxRow<bf16> {
  uint4 u;
  __device__ __forceinline__ void none() { u = make_uint4(0, 0, 0, 0); }
  template <bool VEC>
  __device__ __forceinline__ void load(const bf16* p) {
    if constexpr (VEC) {
      u = __ldcs(reinterpret_cast<const uint4*>(p));
    } else {
      const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
      u = make_uint4(s[0] | (uint32_t)s[1] << 16, s[2] | (uint32_t)s[3] << 16, s[4] | (uint32_t)s[5] << 16, s[6] | (uint32_t)s[7] << 16);
    }
  }
  __device__ __forceinline__ MxEight widened() const {
    MxEight x;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.v[2 * i] = __uint_as_float(w[i] << 16), x.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      top = __vmaxu2(top, w[i] & 0x7fff7fffu);
    }
    x.top = max(top << 16, top & 0xffff0000u);
    return x;
  }
};
template <>
struct MxRow<float> {
  float4 lo, hi;
  __device__ __forceinline__ void none() { lo = hi = make_float4(0.f, 0.f, 0.f, 0.f); }
  template <bool VEC>
  __device__ __forceinline__ void load(const float* p) {
    if constexpr (VEC) lo = __ldcs(reinterpret_cast<const float4*>(p)), hi = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    else lo = make_float4(p[0], p[1], p[2], p[3]), hi = make_float4(p[4], p[5], p[6], p[7]);
  }
  __device__ __forceinline__ MxEight widened() const {
    MxEight x{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) x.top = max(x.top, __float_as_uint(x.v[i]) & 0x7fffffffu);
    return x;
  }
};

// The codes of eight values, four lanes side by side holding a group; the group's scale byte.  Whole warp.
__device__ __forceinline__ uint32_t mx_quantize8(MxEight x, uint32_t* byte) {
  uint32_t top = max(x.top, __shfl_xor_sync(0xffffffffu, x.top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  *byte = mx_scale(top);
  if (*byte == 255) return 0;
  const float k = mx_inverse(*byte);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.v[i] *= k;
  return mx_codes(x.v);
}
#endif

}  // namespace approxifer
