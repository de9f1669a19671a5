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

#include <algorithm>

namespace ql {

namespace {
__device__ __forceinline__ float silu(float v) { return v / (1.0f + expf(-v)); }
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

// ------------------------------------------------------------------- the scan
// Four lanes hold a channel, NS of its states each (state s NS + i in lane s of
// the four; states past the layer's have B = C = 0), a wave 16 channels, a
// workgroup 64.  Steps go by fours: lane j of the four prepares step t + j
// (softplus, d u, the gate, D u), each step's d and d u then reach the other
// three by a DPP broadcast, and the four partial sums over the states of four
// steps are exchanged so that lane j ends with step t + j, gates and stores
// it.  So nothing is computed twice, and there are four times the waves of one
// lane a channel.  B and C of 16 steps lie in LDS as fp32, shared by the
// workgroup; the next 16 steps' inputs are in flight while these are computed.
//
// Few sequences of few channels leave the chip idle: then time is cut into
// chunks.  A first launch runs every chunk but the last from a zero state
// (chunk 0 from the real one) and leaves its final state and sum of d; the second
// composes what lies before its chunk, H <- exp(A sum d) H + h, and runs the
// chunk.  The states are computed twice, the price of not being serial.
constexpr int kTile = 16;

// The value lane (lane ^ X) of this lane's group of four holds.
template <int X>
__device__ __forceinline__ float quad_xor(float v) {
  constexpr int ctrl = (0 ^ X) | (1 ^ X) << 2 | (2 ^ X) << 4 | (3 ^ X) << 6;
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, false));
}
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// log(1 + e) = 2 atanh(e / (2 + e)), its series to the 13th power: e / (2 + e) is at
// most 1 / 3, so what is left out is below 2^-26 of the value
__device__ __forceinline__ float softplus_fast(float x) {
  const float e = exp2_hw(-fabsf(x) * kLog2e);
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
  float p = 1.0f / 13.0f;
  p = __builtin_fmaf(p, q, 1.0f / 11.0f);
  p = __builtin_fmaf(p, q, 1.0f / 9.0f);
  p = __builtin_fmaf(p, q, 1.0f / 7.0f);
  p = __builtin_fmaf(p, q, 1.0f / 5.0f);
  p = __builtin_fmaf(p, q, 1.0f / 3.0f);
  p = __builtin_fmaf(p, q, 1.0f);
  return fmaxf(x, 0.0f) + 2.0f * s * p;
}
__device__ __forceinline__ float silu_fast(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + exp2_hw(-v * kLog2e));
}

// Where the chunks' states lie: slot 0 the initial state, slot k + 1 what chunk k
// ends with; sums of d per chunk.
struct ScanChunks {
  int64_t steps;  // a chunk's, a multiple of kTile
  int n;
  float *state;   // [B][n][N][D]
  float *dsum;    // [B][n][D]
};

template <int NS, class T, bool STATE>
__global__ __launch_bounds__(256) void k_scan(ScanArgs a, ScanChunks ch) {
  constexpr int NP = 4 * NS, kPer = NP >= 16 ? NP / 16 : 1;  // B (C) values a thread stages
  __shared__ __attribute__((aligned(16))) float bc[2][2][kTile][NP];
  const int tid = threadIdx.x, j = tid & 3;
  const int64_t D = a.D, b = blockIdx.z, c = blockIdx.y, t0 = c * ch.steps;
  const int64_t len = clamp_len(a.lengths, b, a.T);
  const int N = a.N;
  if (t0 >= len && c > 0) return;
  if (STATE && t0 + ch.steps >= len && c > 0) return;  // no chunk after it
  const int64_t own = (int64_t)blockIdx.x * 64 + (tid >> 2);
  const bool live = own < D;
  const int64_t d0 = live ? own : D - 1;
  const int64_t t1 = t0 + ch.steps < len ? t0 + ch.steps : len;

  float h[NS], A[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int n = j * NS + i;
    A[i] = n < N ? a.A[n * D + d0] * kLog2e : 0.0f;
    h[i] = 0.0f;
  }
  const float *slot = ch.state + b * ch.n * N * D + d0;  // [k][n][.]
  if (STATE || ch.n == 1) {
    if (c == 0 && a.state_in)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (j * NS + i < N) h[i] = a.state_in[(b * N + j * NS + i) * D + d0];
    if (STATE && c == 0 && live)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (j * NS + i < N) const_cast<float *>(slot)[(j * NS + i) * D] = h[i];
  } else {
    // slot 0 alone for chunk 0; else what chunk 0 ends with, and on from there
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (j * NS + i < N) h[i] = slot[((c ? 1 : 0) * N + j * NS + i) * D];
    for (int64_t k = 1; k < c; ++k) {
      const float s = ch.dsum[(b * ch.n + k) * D + d0];
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (j * NS + i < N)
          h[i] = __builtin_fmaf(exp2_hw(s * A[i]), h[i], slot[((k + 1) * N + j * NS + i) * D]);
    }
  }

  const float bias = a.delta_bias ? a.delta_bias[d0] : 0.0f;
  const float skip = !STATE && a.skip ? a.skip[d0] : 0.0f;
  const T *up = static_cast<const T *>(a.u.data) + b * a.u.b_stride + d0;
  const T *dp = static_cast<const T *>(a.delta.data) + b * a.delta.b_stride + d0;
  const T *zp = a.z.data ? static_cast<const T *>(a.z.data) + b * a.z.b_stride + d0 : nullptr;
  const T *Bp = static_cast<const T *>(a.Bm.data) + b * a.Bm.b_stride;
  const T *Cp = static_cast<const T *>(a.Cm.data) + b * a.Cm.b_stride;
  T *yp = static_cast<T *>(a.y) + b * a.y_b + d0;

  // steps past t1 are loaded from the last one and then masked
  T ru[4], rd[4], rz[4], rb[kPer], rc[kPer];
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int64_t at = t + 4 * g + j < t1 ? t + 4 * g + j : t1 - 1;
      ru[g] = up[at * a.u.t_stride];
      rd[g] = dp[at * a.delta.t_stride];
      if (!STATE && zp) rz[g] = zp[at * a.z.t_stride];
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int e = k * 256 + tid, n = e % NP;
      const int64_t at = t + e / NP;
      const bool on = e < kTile * NP && n < N && at < t1;
      rb[k] = on ? Bp[at * a.Bm.t_stride + n] : (T)0.0f;
      if (!STATE) rc[k] = on ? Cp[at * a.Cm.t_stride + n] : (T)0.0f;
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int e = k * 256 + tid;
      if (e < kTile * NP) {
        (&bc[buf][0][0][0])[e] = (float)rb[k];
        if (!STATE) (&bc[buf][1][0][0])[e] = (float)rc[k];
      }
    }
  };
  float dsum = 0.0f;
  if (t0 < t1) {
    fetch(t0);
    stage(0);
  }
  __syncthreads();
  int buf = 0;
  for (int64_t t = t0; t < t1; t += kTile, buf ^= 1) {
    float uu[4], dd[4], zz[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uu[g] = (float)ru[g];
      dd[g] = (float)rd[g];
      if (!STATE && zp) zz[g] = (float)rz[g];
    }
    if (t + kTile < t1) fetch(t + kTile);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (t + 4 * g < t1) {
        float d = dd[g] + bias;
        if (a.softplus) d = softplus_fast(d);
        const bool on = t + 4 * g + j < t1;
        d = on ? d : 0.0f;
        const float du = on ? d * uu[g] : 0.0f;
        if (STATE) dsum += d;
        float p[4];
        auto step = [&](int k, float dk, float duk) {
          float Bv[NS], Cv[NS];
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            Bv[i] = bc[buf][0][4 * g + k][j * NS + i];
            if (!STATE) Cv[i] = bc[buf][1][4 * g + k][j * NS + i];
          }
          p[k] = 0.0f;
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            h[i] = __builtin_fmaf(exp2_hw(dk * A[i]), h[i], duk * Bv[i]);
            if (!STATE) p[k] = __builtin_fmaf(Cv[i], h[i], p[k]);
          }
        };
        step(0, quad_bcast<0>(d), quad_bcast<0>(du));
        step(1, quad_bcast<1>(d), quad_bcast<1>(du));
        step(2, quad_bcast<2>(d), quad_bcast<2>(du));
        step(3, quad_bcast<3>(d), quad_bcast<3>(du));
        if (!STATE) {
          // lane j gathers step j: pairs exchange, then pairs of pairs
          const bool odd = j & 1, high = j & 2;
          const float q0 = (odd ? p[1] : p[0]) + quad_xor<1>(odd ? p[0] : p[1]);
          const float q1 = (odd ? p[3] : p[2]) + quad_xor<1>(odd ? p[2] : p[3]);
          float y = (high ? q1 : q0) + quad_xor<2>(high ? q0 : q1);
          y = __builtin_fmaf(skip, uu[g], y);
          if (zp) y *= silu_fast(zz[g]);
          if (on && live) yp[(t + 4 * g + j) * a.y_t] = (T)y;
        }
      }
    }
    if (t + kTile < t1) stage(buf ^ 1);
    __syncthreads();
  }
  if (STATE) {
    dsum += quad_xor<1>(dsum);
    dsum += quad_xor<2>(dsum);
    if (live) {
      if (j == 0) ch.dsum[(b * ch.n + c) * D + d0] = dsum;
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (j * NS + i < N) const_cast<float *>(slot)[((c + 1) * N + j * NS + i) * D] = h[i];
    }
  } else if (a.state_out && live && t0 + ch.steps >= len) {
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (j * NS + i < N) a.state_out[(b * N + j * NS + i) * D + d0] = h[i];
  }
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

// Chunks of time: enough for 2048 waves, of 32 steps at least, at most 32 (each
// chunk composes all before it).
static int scan_chunks(int64_t D, int64_t T, int64_t B) {
  const int64_t waves = (D + 63) / 64 * 4 * B;
  const int64_t want = waves >= 1024 ? 1 : (2048 + waves - 1) / waves;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, 32), T / 32));
}
size_t scan_ws(int64_t D, int64_t N, int64_t T, int64_t B) {
  if (B == 0) return 0;
  const int n = scan_chunks(D, T, B);
  return n == 1 ? 0 : (size_t)(B * n) * (size_t)((N + 1) * D) * sizeof(float);
}

template <class T>
static void run_scan(const ScanArgs &a, void *ws, hipStream_t s) {
  ScanChunks ch{};
  ch.n = scan_chunks(a.D, a.T, a.B);
  ch.steps = round_up((a.T + ch.n - 1) / ch.n, kTile);
  ch.state = static_cast<float *>(ws);
  ch.dsum = ch.state + a.B * ch.n * a.N * a.D;
  const unsigned x = blocks_for(a.D, 64);
  if (ch.n > 1) {
    auto kern = a.N <= 4 ? k_scan<1, T, true>
                : a.N <= 8 ? k_scan<2, T, true>
                : a.N <= 16 ? k_scan<4, T, true>
                : a.N <= 32 ? k_scan<8, T, true>
                            : k_scan<16, T, true>;
    hipLaunchKernelGGL(kern, dim3(x, ch.n - 1, (unsigned)a.B), dim3(256), 0, s, a, ch);
  }
  auto kern = a.N <= 4 ? k_scan<1, T, false>
              : a.N <= 8 ? k_scan<2, T, false>
              : a.N <= 16 ? k_scan<4, T, false>
              : a.N <= 32 ? k_scan<8, T, false>
                          : k_scan<16, T, false>;
  hipLaunchKernelGGL(kern, dim3(x, ch.n, (unsigned)a.B), dim3(256), 0, s, a, ch);
}
hipError_t launch_scan(int type, const ScanArgs &a, void *ws, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  if (type == 0)
    run_scan<float>(a, ws, s);
  else if (type == 1)
    run_scan<f16>(a, ws, s);
  else
    run_scan<bf16>(a, ws, s);
  return hipGetLastError();
}

}  // namespace ql
