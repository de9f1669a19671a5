// ql_ssm.hip -- the selective state space layer's parts that run over time: the
// short causal convolution and the scan, for prompts and for single tokens.
//
//   conv: y_t = f(b + sum_j w_j x_{t - W + 1 + j}),  f = SiLU or none
//   scan: d = softplus(delta_t + bias);  h[n] = exp(d A[n]) h[n] + (d u_t) B_t[n]
//         y_t = (sum_n C_t[n] h[n] + D u_t) silu(z_t)
//
// Channels are the contiguous dimension of everything (A and the state lie
// [states][channels]), so a lane is a channel and its states stay in registers.
#include "ql_elem.h"
#include "ql_launch.h"

namespace ql {

namespace {
__device__ __forceinline__ float silu(float v) { return v / (1.0f + expf(-v)); }
__device__ __forceinline__ float softplus(float v) {
  return fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v)));
}
__device__ __forceinline__ int64_t clamp_len(const int32_t *lengths, int64_t b, int64_t T) {
  if (!lengths) return T;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : n > T ? T : n;
}
}  // namespace

// A thread per channel of one sequence's chunk of steps.
constexpr int kConvSteps = 16;
template <int W, class T>
__global__ __launch_bounds__(256) void k_causal_conv(ConvArgs a) {
  const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x, b = blockIdx.z;
  const int64_t t0 = (int64_t)blockIdx.y * kConvSteps;
  const int64_t len = clamp_len(a.lengths, b, a.T);
  if (d >= a.D || (t0 >= len && t0 > 0)) return;
  const T *x = static_cast<const T *>(a.x.data) + b * a.x.b_stride + d;
  T *y = static_cast<T *>(a.y) + b * a.y_b + d;
  const int64_t state = (b * (W - 1)) * a.D + d;
  float w[W], v[W];
#pragma unroll
  for (int j = 0; j < W; ++j) w[j] = a.w[j * a.D + d];
  const float bias = a.bias ? a.bias[d] : 0.0f;
  // v[j]: input of step t - W + 1 + j
  auto before = [&](int64_t t) {  // input of step t < len, from the state where t < 0
    if (t >= 0) return (float)x[t * a.x.t_stride];
    return a.state_in ? a.state_in[state + (t + W - 1) * a.D] : 0.0f;
  };
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) v[j + 1] = before(t0 - W + 1 + j);
  const int64_t t1 = t0 + kConvSteps < len ? t0 + kConvSteps : len;
  // the first chunk's thread writes the state: it has read the old one where
  // both are one buffer
  float last[W];
  if (t0 == 0 && a.state_out) {
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) last[j] = before(len - W + 1 + j);
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) a.state_out[state + j * a.D] = last[j];
  }
  for (int64_t t = t0; t < t1; ++t) {
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) v[j] = v[j + 1];
    v[W - 1] = (float)x[t * a.x.t_stride];
    float s = bias;
#pragma unroll
    for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j], v[j], s);
    y[t * a.y_t] = (T)(a.silu ? silu(s) : s);
  }
}

// A thread per channel of a sequence, its NS states in registers (states past the
// layer's have B = 0 and stay 0).
template <int NS, class T>
__global__ __launch_bounds__(64) void k_scan(ScanArgs a) {
  const int64_t d = (int64_t)blockIdx.x * 64 + threadIdx.x, b = blockIdx.y;
  if (d >= a.D) return;
  const int N = a.N;
  const int64_t len = clamp_len(a.lengths, b, a.T);
  const T *u = static_cast<const T *>(a.u.data) + b * a.u.b_stride + d;
  const T *dl = static_cast<const T *>(a.delta.data) + b * a.delta.b_stride + d;
  const T *Bm = static_cast<const T *>(a.Bm.data) + b * a.Bm.b_stride;
  const T *Cm = static_cast<const T *>(a.Cm.data) + b * a.Cm.b_stride;
  const T *z = a.z.data ? static_cast<const T *>(a.z.data) + b * a.z.b_stride + d : nullptr;
  T *y = static_cast<T *>(a.y) + b * a.y_b + d;
  const float bias = a.delta_bias ? a.delta_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
  float h[NS], A[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    A[n] = n < N ? a.A[n * a.D + d] : 0.0f;
    h[n] = n < N && a.state_in ? a.state_in[(b * N + n) * a.D + d] : 0.0f;
  }
  for (int64_t t = 0; t < len; ++t) {
    const float uv = (float)u[t * a.u.t_stride];
    float dv = (float)dl[t * a.delta.t_stride] + bias;
    if (a.softplus) dv = softplus(dv);
    const float du = dv * uv;
    float s = skip * uv;
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n < N) {
        h[n] = __builtin_fmaf(expf(dv * A[n]), h[n], du * (float)Bm[t * a.Bm.t_stride + n]);
        s = __builtin_fmaf((float)Cm[t * a.Cm.t_stride + n], h[n], s);
      }
    if (z) s *= silu((float)z[t * a.z.t_stride]);
    y[t * a.y_t] = (T)s;
  }
  if (a.state_out)
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n < N) a.state_out[(b * N + n) * a.D + d] = h[n];
}

// ---------------------------------------------------------------- launchers
static inline unsigned blocks_for(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

template <int W>
static void run_conv(int type, const ConvArgs &a, hipStream_t s) {
  const dim3 grid(blocks_for(a.D, 256), a.T ? blocks_for(a.T, kConvSteps) : 1, (unsigned)a.B);
  auto kern = type == 0 ? k_causal_conv<W, float>
              : type == 1 ? k_causal_conv<W, f16>
                          : k_causal_conv<W, bf16>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a);
}
hipError_t launch_causal_conv(int type, const ConvArgs &a, int width, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  switch (width) {
    case 1: run_conv<1>(type, a, s); break;
    case 2: run_conv<2>(type, a, s); break;
    case 3: run_conv<3>(type, a, s); break;
    case 4: run_conv<4>(type, a, s); break;
    case 5: run_conv<5>(type, a, s); break;
    case 6: run_conv<6>(type, a, s); break;
    case 7: run_conv<7>(type, a, s); break;
    default: run_conv<8>(type, a, s); break;
  }
  return hipGetLastError();
}

size_t scan_ws(int64_t D, int64_t N, int64_t T, int64_t B) { return 0; }

template <class T>
static void run_scan(const ScanArgs &a, hipStream_t s) {
  const dim3 grid(blocks_for(a.D, 64), (unsigned)a.B);
  auto kern = a.N <= 4 ? k_scan<4, T>
              : a.N <= 8 ? k_scan<8, T>
              : a.N <= 16 ? k_scan<16, T>
              : a.N <= 32 ? k_scan<32, T>
                          : k_scan<64, T>;
  hipLaunchKernelGGL(kern, grid, dim3(64), 0, s, a);
}
hipError_t launch_scan(int type, const ScanArgs &a, void *ws, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  if (type == 0)
    run_scan<float>(a, s);
  else if (type == 1)
    run_scan<f16>(a, s);
  else
    run_scan<bf16>(a, s);
  return hipGetLastError();
}

}  // namespace ql
