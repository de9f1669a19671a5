// ql_elem.h -- activations of three types (fp32, fp16, bfloat16): conversions,
// loads and stores of several neighbouring values, and fp32 / fp64 sums over a
// wave or a workgroup; used by the norm, the 4-bit products, the causal
// convolution and the selective scan.
#pragma once
#include "ql_device.h"

#include <type_traits>

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

// A row held by WAVES waves, PER values a thread in vectors of VEC: vector k of
// thread t is values (k 64 WAVES + t) VEC .. + VEC - 1.
template <int VEC, int PER, int WAVES>
struct RowSlots {
  static constexpr int kVecs = PER / VEC;
  static constexpr int kThreads = 64 * WAVES;
  static constexpr int kCols = PER * kThreads;  // the longest row
  static __device__ __forceinline__ int col(int k, int t) { return (k * kThreads + t) * VEC; }
  // The thread's values of a row of n, 0 past its end.  TAIL: n is no multiple of
  // VEC; the one vector that the end cuts comes value by value, after the others
  // are in flight.
  template <bool TAIL, class T>
  static __device__ __forceinline__ void load(float (&v)[PER], const T *p, int n, int t) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int c = col(k, t);
      float q[VEC];
      if (TAIL ? c + VEC <= n : c < n) {
        load_n<VEC>(q, p + c);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) q[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[k * VEC + i] = q[i];
    }
    if constexpr (TAIL) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int c = col(k, t);
        if (c < n && c + VEC > n)
#pragma unroll
          for (int i = 0; i < VEC - 1; ++i)
            if (c + i < n) v[k * VEC + i] = (float)p[c + i];
      }
    }
  }
  template <bool TAIL, class T>
  static __device__ __forceinline__ void store(T *p, const float (&v)[PER], int n, int t) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int c = col(k, t);
      float q[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) q[i] = v[k * VEC + i];
      if (TAIL ? c + VEC <= n : c < n) store_n<VEC>(p + c, q);
      if (TAIL && c < n && c + VEC > n)
#pragma unroll
        for (int i = 0; i < VEC - 1; ++i)
          if (c + i < n) p[c + i] = (T)q[i];
    }
  }
};

// The 8-bit codes (eq. 2) of a row held in registers, its padding [n, ld), and its
// zero point, recovery factor and code sum.  A row with a value that is not
// finite: codes and zero point 0, recovery factor NaN.
template <int VEC, int PER, int WAVES, bool TAIL>
__device__ __forceinline__ void code_row(const float (&v)[PER], int n, int t, int8_t *o, int64_t ld,
                                         int32_t *zero, float *inv_q, int32_t *sums) {
  typedef RowSlots<VEC, PER, WAVES> S;
  __shared__ float slo[16], shi[16];
  __shared__ int sbad[16], scodes[16];
  const int wave = threadIdx.x >> 6;
  float lo = INFINITY, hi = -INFINITY, nan = 0.0f;
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (S::col(e / VEC, t) + e % VEC < n) {
      lo = fminf(lo, v[e]);
      hi = fmaxf(hi, v[e]);
      nan = __builtin_fmaf(v[e], 0.0f, nan);  // NaN where one is not finite
    }
  lo = wave_min(lo);
  hi = wave_max(hi);
  bool bad = __any(nan != nan);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) slo[wave] = lo, shi[wave] = hi, sbad[wave] = bad;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      lo = fminf(lo, slo[w]);
      hi = fmaxf(hi, shi[w]);
      bad |= sbad[w] != 0;
    }
  }
  const QParams p = bad ? QParams{0.0, 0, __builtin_nanf(""), 0.0} : make_qparams(lo, hi);
  const FastEncode f = bad ? FastEncode{0.0f, 0.0f, 2.0f} : fast_encode(p, lo, hi);
  uint32_t codesum = 0;
#pragma unroll
  for (int k = 0; k < S::kVecs; ++k) {
    const int c = S::col(k, t);
    float q[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) q[i] = bad ? 0.0f : v[k * VEC + i];
    uint32_t w[VEC / 4];
    encode_words<VEC>(q, p, f, w);
    if (TAIL ? c + VEC <= n : c < n) {
      typedef uint32_t vec __attribute__((ext_vector_type(VEC / 4)));
      typedef vec any __attribute__((aligned(1)));
      vec words;
#pragma unroll
      for (int i = 0; i < VEC / 4; ++i) {
        codesum = add_codes(w[i], codesum);
        words[i] = w[i] ^ 0x80808080u;
      }
      *reinterpret_cast<any *>(o + c) = words;
    } else if (TAIL) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (c + i < n) {
          const uint32_t code = (w[i / 4] >> (8 * (i % 4))) & 255u;
          codesum += code;
          o[c + i] = (int8_t)(code ^ 0x80u);
        }
    }
  }
  for (int64_t c = n + t; c < ld; c += S::kThreads) o[c] = 0;
  int sum = wave_sum((int)codesum);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) scodes[wave] = sum;
    __syncthreads();
    sum = scodes[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += scodes[w];
  }
  if (t == 0) {
    *zero = p.z;
    *inv_q = p.inv_q;
    *sums = sum;
  }
}

// The form of a row in registers by its length: calls f with PER and WAVES as
// types; false where none holds it.
template <int N>
using Int = std::integral_constant<int, N>;
template <bool deep, class F>
static bool by_row(int64_t cols, F f) {
  if (cols <= 512)
    f(Int<8>(), Int<1>());
  else if (cols <= 1024)
    f(Int<16>(), Int<1>());
  else if (cols <= 2048)
    f(Int<deep ? 16 : 8>(), Int<deep ? 2 : 4>());
  else if (cols <= 4096)
    f(Int<deep ? 16 : 8>(), Int<deep ? 4 : 8>());
  else if (cols <= 8192)
    f(Int<deep ? 16 : 8>(), Int<deep ? 8 : 16>());
  else if (cols <= 16384)
    f(Int<16>(), Int<16>());
  else
    return false;
  return true;
}
// Whether rows to be coded take the deep form, more values a thread: what a wave does
// once a row (a square root, divisions) weighs where rows fill the chip, the longer
// chain where they do not (us deep and not, bfloat16, norm with residual into codes: 128
// x 2048 4.5 and 3.9, 512 x 2048 5.7 and 4.7, 1024 x 2048 6.3 and 6.6, 4096 x 4096 28 and
// 33, 16 x 8000 5.2 and 5.7, 4096 x 8000 52 and 66).
inline bool deep_rows(int64_t rows, int64_t cols) { return rows >= 1024 || cols > 4096; }
// A grid has fewer than 2^32 threads: the rows of one launch at `waves` waves a row.
constexpr int64_t rows_a_launch(int waves) { return ((int64_t)1 << 31) / (64 * waves); }
constexpr int block_of(int waves) { return waves == 1 ? 256 : 64 * waves; }

// Barrier of a workgroup that orders LDS accesses alone: loads from memory stay in
// flight over it (__syncthreads waits for them).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace ql
