// ql_elem.h -- activations of three types (fp32, fp16, bfloat16): conversions,
// loads and stores of several neighbouring values, and fp32 / fp64 sums over a
// wave or a workgroup; used by the norm, the 4-bit products, the causal
// convolution and the selective scan.
#pragma once
#include "ql_device.h"

namespace ql {

typedef _Float16 f16;
typedef __bf16 bf16;

// N neighbouring values as fp32.  p is aligned to N values (up to 16 bytes at a
// time).  Rounding to fp16 and bfloat16 is to the nearest, ties to even.
template <int N, class T>
__device__ __forceinline__ void load_n(float (&v)[N], const T *p) {
  constexpr int bytes = N * (int)sizeof(T);
  constexpr int per = bytes <= 16 ? N : 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(per)));
#pragma unroll
  for (int k = 0; k < N / per; ++k) {
    const vec t = reinterpret_cast<const vec *>(p)[k];
#pragma unroll
    for (int i = 0; i < per; ++i) v[k * per + i] = (float)t[i];
  }
}
template <int N, class T>
__device__ __forceinline__ void store_n(T *p, const float (&v)[N]) {
  constexpr int bytes = N * (int)sizeof(T);
  constexpr int per = bytes <= 16 ? N : 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(per)));
#pragma unroll
  for (int k = 0; k < N / per; ++k) {
    vec t;
#pragma unroll
    for (int i = 0; i < per; ++i) t[i] = (T)v[k * per + i];
    reinterpret_cast<vec *>(p)[k] = t;
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

}  // namespace ql
