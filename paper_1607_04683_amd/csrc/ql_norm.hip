// ql_norm.hip -- root-mean-square norm of rows with the residual's addition, its
// output as floats and / or as per-vector 8-bit codes, and its backward pass.
//
//   v = x + r (rounded to the rows' type: what the residual stream holds)
//   rstd = (float)(1 / sqrt(sum v^2 / n + eps)), in fp64
//   y = (v rstd) w, two fp32 roundings; codes: eq. 2 on the fp32 y
//
// The sum is fp64 and every fp32 operation is written out, so y and its codes
// are the same bits in any order of summation but for sums within 1e-16 of a
// rounding border: the codes equal those of ql_quantize_activations on y.
#include "ql_elem.h"
#include "ql_launch.h"

#include <algorithm>

namespace ql {

namespace {

// Sum over the workgroup (up to 16 waves) in every thread; `s` has 16 places and
// is free for the next use after the caller's next barrier.
template <class F>
__device__ __forceinline__ F block_sum(F v, F *s) {
  const int nw = blockDim.x >> 6;
  if constexpr (sizeof(F) == 8)
    v = wave_sum_f64(v);
  else
    v = wave_sum_f32(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < nw; ++w) v += s[w];
  return v;
}

}  // namespace

// One workgroup per row, the row read three times (sum of squares, range, result);
// an element is read and then written by one thread, so results may lie on
// inputs of the same layout.
template <class T>
__global__ __launch_bounds__(256) void k_rms_norm(NormArgs a) {
  __shared__ double ssum[16];
  __shared__ float slo[4], shi[4];
  __shared__ int sbad[4], scodes[4];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x, n = a.cols;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx;
  const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ldr : nullptr;
  T *sum = a.sum ? static_cast<T *>(a.sum) + row * a.lds : nullptr;
  T *y = a.y ? static_cast<T *>(a.y) + row * a.ldy : nullptr;
  const float *w = a.weight;

  double ss = 0.0;
  for (int64_t i = tid; i < n; i += 256) {
    float v = (float)x[i];
    if (r) v = (float)(T)(v + (float)r[i]);
    if (sum) sum[i] = (T)v;
    ss += (double)v * (double)v;
  }
  ss = block_sum(ss, ssum);
  const float rstd = (float)(1.0 / sqrt(ss / (double)n + a.eps));
  if (a.rstd && tid == 0) a.rstd[row] = rstd;
  auto value = [&](int64_t i) {
    float v;
    if (sum) {
      v = (float)sum[i];
    } else {
      v = (float)x[i];
      if (r) v = (float)(T)(v + (float)r[i]);
    }
    v = v * rstd;
    return w ? v * w[i] : v;
  };
  QParams p{};
  bool bad = false;
  if (a.codes) {
    float lo = INFINITY, hi = -INFINITY;
    for (int64_t i = tid; i < n; i += 256) {
      const float v = value(i);
      lo = fminf(lo, v);
      hi = fmaxf(hi, v);
      bad |= !(fabsf(v) < INFINITY);
    }
    lo = wave_min(lo);
    hi = wave_max(hi);
    const bool any = __any(bad);
    if ((tid & 63) == 0) slo[tid >> 6] = lo, shi[tid >> 6] = hi, sbad[tid >> 6] = any;
    __syncthreads();
    lo = fminf(fminf(slo[0], slo[1]), fminf(slo[2], slo[3]));
    hi = fmaxf(fmaxf(shi[0], shi[1]), fmaxf(shi[2], shi[3]));
    bad = sbad[0] | sbad[1] | sbad[2] | sbad[3];
    if (!bad) p = make_qparams(lo, hi);
  }
  int codesum = 0;
  for (int64_t i = tid; i < n; i += 256) {
    const float v = value(i);
    if (a.codes) {
      const int c = bad ? 0 : encode(v, p.q, p.z);
      codesum += c;
      a.codes[row * a.ldc + i] = (int8_t)(c ^ 0x80);
    }
    if (y) y[i] = (T)v;
  }
  if (a.codes) {
    for (int64_t i = n + tid; i < a.ldc; i += 256) a.codes[row * a.ldc + i] = 0;
    codesum = wave_sum(codesum);
    if ((tid & 63) == 0) scodes[tid >> 6] = codesum;
    __syncthreads();
    if (tid == 0) {
      a.zero[row] = bad ? 0 : p.z;
      a.inv_q[row] = bad ? __builtin_nanf("") : p.inv_q;
      a.sums[row] = scodes[0] + scodes[1] + scodes[2] + scodes[3];
    }
  }
}

// dx of one row per workgroup:
//   dx = rstd g - v rstd^3 / n sum(g v) + dsum,  g = w dy
template <class T>
__global__ __launch_bounds__(256) void k_rms_norm_dx(NormGradArgs a) {
  __shared__ float ssum[16];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x, n = a.cols;
  const T *dy = static_cast<const T *>(a.dy) + row * a.lddy;
  const T *v = static_cast<const T *>(a.v) + row * a.ldv;
  const T *ds = a.dsum ? static_cast<const T *>(a.dsum) + row * a.ldds : nullptr;
  T *dx = static_cast<T *>(a.dx) + row * a.lddx;
  float s = 0.0f;
  for (int64_t i = tid; i < n; i += 256) {
    const float g = a.weight ? a.weight[i] * (float)dy[i] : (float)dy[i];
    s = __builtin_fmaf(g, (float)v[i], s);
  }
  s = block_sum(s, ssum);
  const float rstd = a.rstd[row];
  const float c = s * rstd * rstd * rstd / (float)n;
  for (int64_t i = tid; i < n; i += 256) {
    const float g = a.weight ? a.weight[i] * (float)dy[i] : (float)dy[i];
    float d = __builtin_fmaf(g, rstd, -((float)v[i] * c));
    if (ds) d += (float)ds[i];
    dx[i] = (T)d;
  }
}

// Partial dweight of a band of rows: part[band][i] = sum dy (v rstd).
template <class T>
__global__ __launch_bounds__(256) void k_rms_norm_dw(NormGradArgs a, float *__restrict__ part,
                                                     int64_t per) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * per, r1 = r0 + per < a.rows ? r0 + per : a.rows;
  const T *dy = static_cast<const T *>(a.dy), *v = static_cast<const T *>(a.v);
  float s = 0.0f;
  for (int64_t r = r0; r < r1; ++r)
    s = __builtin_fmaf((float)dy[r * a.lddy + i], (float)v[r * a.ldv + i] * a.rstd[r], s);
  part[(int64_t)blockIdx.y * a.cols + i] = s;
}
__global__ __launch_bounds__(256) void k_rms_norm_dw_join(const float *__restrict__ part, int parts,
                                                          int64_t cols, float *__restrict__ dw) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= cols) return;
  float s = 0.0f;
  for (int p = 0; p < parts; ++p) s += part[(int64_t)p * cols + i];
  dw[i] = s;
}

// ---------------------------------------------------------------- launchers
static inline unsigned blocks_for(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

hipError_t launch_rms_norm(int type, const NormArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  auto kern = type == 0 ? k_rms_norm<float> : type == 1 ? k_rms_norm<f16> : k_rms_norm<bf16>;
  hipLaunchKernelGGL(kern, dim3((unsigned)a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Bands of rows of the partial dweight.
static int grad_parts(int64_t rows) {
  return (int)std::min<int64_t>(256, std::max<int64_t>(1, rows / 16));
}
size_t rms_norm_backward_ws(int64_t rows, int64_t cols) {
  return align_up((size_t)grad_parts(rows) * (size_t)cols * sizeof(float), 256);
}

hipError_t launch_rms_norm_backward(int type, const NormGradArgs &a, float *part, hipStream_t s) {
  if (a.dweight) {
    const int parts = grad_parts(a.rows);
    const int64_t per = (a.rows + parts - 1) / parts;
    auto kern = type == 0 ? k_rms_norm_dw<float>
                : type == 1 ? k_rms_norm_dw<f16>
                            : k_rms_norm_dw<bf16>;
    hipLaunchKernelGGL(kern, dim3(blocks_for(a.cols, 256), parts), dim3(256), 0, s, a, part, per);
    hipLaunchKernelGGL(k_rms_norm_dw_join, dim3(blocks_for(a.cols, 256)), dim3(256), 0, s, part,
                       parts, a.cols, a.dweight);
  }
  if (a.rows > 0) {
    auto kern = type == 0 ? k_rms_norm_dx<float>
                : type == 1 ? k_rms_norm_dx<f16>
                            : k_rms_norm_dx<bf16>;
    hipLaunchKernelGGL(kern, dim3((unsigned)a.rows), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace ql
