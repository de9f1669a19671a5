// ql_elem.h -- activations of three types (fp32, fp16, bfloat16): conversions,
// loads and stores of several neighbouring values, and fp32 / fp64 sums over a
// wave or a workgroup; used by the norm, the 4-bit products, the causal
// convolution and the selective scan.
#pragma once
#include "ql_device.h"

namespace ql {

typedef _Float16 f16;
typedef __bf16 bf16;

// N neighbouring values as fp32, whatever their alignment (the hardware takes
// 16-byte loads and stores at any element's address).  Rounding to fp16 and
// bfloat16 is to the nearest, ties to even.
template <int N, class T>
__device__ __forceinline__ void load_n(float (&v)[N], const T *p) {
  constexpr int bytes = N * (int)sizeof(T);
  constexpr int per = bytes <= 16 ? N : 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(per)));
  typedef vec any __attribute__((aligned(sizeof(T))));
#pragma unroll
  for (int k = 0; k < N / per; ++k) {
    const vec t = *reinterpret_cast<const any *>(p + k * per);
#pragma unroll
    for (int i = 0; i < per; ++i) v[k * per + i] = (float)t[i];
  }
}
template <int N, class T>
__device__ __forceinline__ void store_n(T *p, const float (&v)[N]) {
  constexpr int bytes = N * (int)sizeof(T);
  constexpr int per = bytes <= 16 ? N : 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(per)));
  typedef vec any __attribute__((aligned(sizeof(T))));
#pragma unroll
  for (int k = 0; k < N / per; ++k) {
    vec t;
#pragma unroll
    for (int i = 0; i < per; ++i) t[i] = (T)v[k * per + i];
    *reinterpret_cast<any *>(p + k * per) = t;
  }
}
// Sums over the wave, in every lane: DPP shifts within rows of 16 lanes, then row
// broadcasts, the result read from lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(dpp_i<CTRL, ROWS>(0, __float_as_int(v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v) {
  return __hiloint2double(dpp_i<CTRL, ROWS>(0, __double2hiint(v)),
                          dpp_i<CTRL, ROWS>(0, __double2loint(v)));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v += dpp_f64<kRowShr1, 0xf>(v);
  v += dpp_f64<kRowShr2, 0xf>(v);
  v += dpp_f64<kRowShr4, 0xf>(v);
  v += dpp_f64<kRowShr8, 0xf>(v);
  v += dpp_f64<kRowBcast15, 0xa>(v);
  v += dpp_f64<kRowBcast31, 0xc>(v);
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63),
                          __builtin_amdgcn_readlane(__double2loint(v), 63));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
  v += dpp_f32<kRowShr1, 0xf>(v);
  v += dpp_f32<kRowShr2, 0xf>(v);
  v += dpp_f32<kRowShr4, 0xf>(v);
  v += dpp_f32<kRowShr8, 0xf>(v);
  v += dpp_f32<kRowBcast15, 0xa>(v);
  v += dpp_f32<kRowBcast31, 0xc>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Eq. 2 in fp32 where that is certain: the fp64 product Q v decides the rounding,
// and fp32's lies within 2^-22 |Q v| of it, so a value whose fp32 product is not
// within `margin` (more than that for the whole set) of a rounding border has the
// code that fp64 gives; the others, one in some thousands, go through encode().
struct FastEncode {
  float q, z, border;  // border: 0.5 - margin
};
__device__ __forceinline__ FastEncode fast_encode(const QParams &p, float lo, float hi) {
  const float q = (float)p.q;
  const float top = fmaxf(fabsf(lo), fabsf(hi)) * q;
  return FastEncode{q, (float)p.z, 0.5f - (top + 1.0f) * 0x1p-20f};
}
// N (a multiple of 4) values -> N / 4 words of codes 0..255 (not yet in the signed
// layout).  NaN gives code 0 in either form's place; the callers' sets have none.
template <int N>
__device__ __forceinline__ void encode_words(const float (&v)[N], const QParams &p,
                                             const FastEncode &f, uint32_t (&w)[N / 4]) {
  bool sure = true;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = v[i] * f.q;
    const float r = floorf(t + 0.5f);
    sure &= fabsf(t - r) < f.border;
    const float c = __builtin_amdgcn_fmed3f(r - f.z, 0.0f, 255.0f);
    w[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(c, i % 4, i % 4 == 0 ? 0u : w[i / 4]);
  }
  if (!sure) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (uint32_t)encode(v[i], p.q, p.z);
      w[i / 4] = i % 4 == 0 ? c : w[i / 4] | c << (8 * (i % 4));
    }
  }
}
// Sum of four codes 0..255, added to s.
__device__ __forceinline__ uint32_t add_codes(uint32_t w, uint32_t s) {
  return __builtin_amdgcn_udot4(w, 0x01010101u, s, false);
}

}  // namespace ql
