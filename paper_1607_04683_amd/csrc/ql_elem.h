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

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

}  // namespace ql
