// ql_q4.hip -- weights in 4 bits with a scale and a zero point per group of
// columns, and their products with activations in 8-bit codes.
//
// The quantizer is the paper's with S = 15 (eq. 2), one set per group of 32, 64
// or 128 columns of a row, its range widened to hold 0: the zero point z is then
// minus one of the 16 codes, and what is padded recovers to 0 exactly.
//
//   W^[n][k] = (V' + z_g) q_g,  x^[k] = (x' + zx) qx
//   Y[n] = qx sum_g q_g T_g + b[n],  T_g = sum_{k in g} (V' + z_g)(x' + zx)
//
// T_g is exact (integers, one rounding to fp32); the sum over groups is fp32.
//
// Layout of a row: runs of 128 columns, 16 words of 8 codes; word 4 q + p holds
// columns 32 p + 8 q .. + 7, so that the 16 bytes a lane loads give its share of
// every group (p: 32 columns) as operands of the matrix instructions.  Byte j of
// a word holds columns j (low half) and j + 4 (high half) as V' - 8 in two's
// complement: (word << 4) & 0xf0f0f0f0 and word & 0xf0f0f0f0 are four signed
// bytes 16 (V' - 8) each.
#include "ql_elem.h"
#include "ql_launch.h"

namespace ql {

constexpr uint32_t kHigh = 0xf0f0f0f0u;

// One wave per row, a run of 128 columns at a time, two columns a lane.
__global__ __launch_bounds__(256) void k_quantize4(const float *__restrict__ W, int64_t rows,
                                                   int64_t cols, uint8_t *__restrict__ codes,
                                                   int64_t ld, int group, int64_t ldr,
                                                   int8_t *__restrict__ zero,
                                                   float *__restrict__ inv_q) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const float *w = W + row * cols;
  for (int64_t k0 = 0; k0 < ld; k0 += 128) {
    const int64_t k = k0 + 2 * lane;
    const float a = k < cols ? w[k] : 0.0f, b = k + 1 < cols ? w[k + 1] : 0.0f;
    float lo = fminf(fminf(a, b), 0.0f), hi = fmaxf(fmaxf(a, b), 0.0f);
    for (int o = 1; o < group / 2; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o, 64));
      hi = fmaxf(hi, __shfl_xor(hi, o, 64));
    }
    const double R = (double)hi - (double)lo;
    const double q = R == 0.0 ? 1.0 : 15.0 / R;
    const int z = R == 0.0 ? 0 : (int)round_half_up(q * (double)lo);
    auto code = [&](float v) {
      int c = (int)round_half_up(q * (double)v) - z;
      c = c < 0 ? 0 : c > 15 ? 15 : c;
      return (uint32_t)(c ^ 8);
    };
    // this lane's columns are 2 (lane & 3), + 1 of its word
    const int j = 2 * (lane & 3), sh = j < 4 ? 8 * j : 8 * (j - 4) + 4;
    uint32_t word = (code(a) << sh) | (code(b) << (sh + 8));
    word |= __shfl_xor(word, 1, 64);
    word |= __shfl_xor(word, 2, 64);
    const int i = lane >> 2, p = i >> 2, qd = i & 3;
    if ((lane & 3) == 0)
      reinterpret_cast<uint32_t *>(codes + row * (ld / 2) + k0 / 2)[4 * qd + p] = word;
    if (2 * lane % group == 0) {
      const int64_t g = (k0 + 2 * lane) / group;
      zero[g * ldr + row] = (int8_t)z;
      inv_q[g * ldr + row] = R == 0.0 ? 1.0f : (float)(R / 15.0);
    }
  }
}

// Recovery: a thread per word.
__global__ __launch_bounds__(256) void k_dequantize4(const uint8_t *__restrict__ codes, int64_t ld,
                                                     int64_t rows, int64_t cols, int group,
                                                     int64_t ldr, const int8_t *__restrict__ zero,
                                                     const float *__restrict__ inv_q,
                                                     float *__restrict__ dst) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = ld / 8;
  if (i >= rows * per) return;
  const int64_t row = i / per, at = i - row * per;
  const int in = (int)(at & 15);
  const int64_t k0 = at / 16 * 128 + 32 * (in & 3) + 8 * (in >> 2);
  if (k0 >= cols) return;
  const uint32_t w = reinterpret_cast<const uint32_t *>(codes + row * (ld / 2))[at];
  const int64_t g = k0 / group * ldr + row;
  const int z = zero[g];
  const float q = inv_q[g];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = (int)((w >> (j < 4 ? 8 * j : 8 * (j - 4) + 4)) & 15u) ^ 8;
    if (k0 + j < cols) dst[row * cols + k0 + j] = (float)(c + z) * q;
  }
}

// Rows of any type quantized per vector (as k_quantize_rows does for fp32).
template <class T>
__global__ __launch_bounds__(256) void k_quantize_rows_of(const T *__restrict__ X, int64_t ldx,
                                                          int64_t m, int64_t K,
                                                          int8_t *__restrict__ codes, int64_t ld,
                                                          int32_t *__restrict__ zero,
                                                          float *__restrict__ inv_q,
                                                          int32_t *__restrict__ sums) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= m) return;
  const T *x = X + row * ldx;
  float lo = INFINITY, hi = -INFINITY;
  bool bad = false;
  for (int64_t i = lane; i < K; i += 64) {
    const float v = (float)x[i];
    lo = fminf(lo, v);
    hi = fmaxf(hi, v);
    bad |= !(fabsf(v) < INFINITY);
  }
  bad = __any(bad);
  QParams p{};
  if (!bad) p = make_qparams(wave_min(lo), wave_max(hi));
  int sum = 0;
  for (int64_t i = lane; i < ld; i += 64) {
    int c = 0x80;
    if (i < K) {
      c = bad ? 0 : encode((float)x[i], p.q, p.z);
      sum += c;
    }
    codes[row * ld + i] = (int8_t)(c ^ 0x80);
  }
  sum = wave_sum(sum);
  if (lane == 0) {
    zero[row] = p.z;
    inv_q[row] = bad ? __builtin_nanf("") : p.inv_q;
    sums[row] = sum;
  }
}

// The product.  A wave takes 16 rows of W (lane: row r = lane & 15, share
// q = lane >> 4 of the columns) and 16 MT rows of X.  Per group three products
// on the matrix units: W X (16 sum c x), W 1 (16 sum c) and 1 X (sum x), with
// c = V' - 8 and x = x' - 128; then, with z = z_g + 8 and zt = zx + 128,
//   16 T_g = W X + 16 z (1 X) + zt (W 1 + 16 z G)
// in fp32: every term but the last fma's result is an integer below 2^24.
template <int G, int MT, class TY>
__global__ __launch_bounds__(256) void k_matmul4(Q4Mat W, ActRows X, int64_t M, int64_t ncols,
                                                 const float *__restrict__ bias,
                                                 TY *__restrict__ Y) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int64_t n0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16;
  const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
  if (n0 >= W.rows) return;
  const uint8_t *w = W.codes + (n0 + r < W.rows ? n0 + r : W.rows - 1) * (W.ld / 2) + 16 * q;
  const int8_t *x[MT];
  float zt[MT];
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    const int64_t m = m0 + 16 * b + r < M ? m0 + 16 * b + r : M - 1;
    x[b] = X.codes + m * X.ld;
    zt[b] = (float)(X.zero[m] + 128);
  }
  float acc[MT][4];
#pragma unroll
  for (int b = 0; b < MT; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[b][i] = 0.0f;
  const v4i one{0x01010101, 0x01010101, 0x01010101, 0x01010101};
  const int64_t runs = W.ld / 128;
  for (int64_t k = 0; k < runs; ++k) {
    const uint4 wv = *reinterpret_cast<const uint4 *>(w + 64 * k);
    const uint32_t ww[4] = {wv.x, wv.y, wv.z, wv.w};
    int2 xv[MT][4];
#pragma unroll
    for (int b = 0; b < MT; ++b)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        // columns at and past X.ld recover to 0 in W: any codes serve
        const int64_t c = 128 * k + 32 * p + 8 * q;
        xv[b][p] = *reinterpret_cast<const int2 *>(x[b] + (c < X.ld ? c : 0));
      }
    constexpr int kParts = 128 / G;   // groups in a run
    constexpr int kWords = 4 / kParts;  // words of a lane in a group
#pragma unroll
    for (int gp = 0; gp < kParts; ++gp) {
      const int64_t g = k * kParts + gp;
      const float4 qv = *reinterpret_cast<const float4 *>(W.inv_q + g * W.ldr + n0 + 4 * q);
      const int zv = *reinterpret_cast<const int *>(W.zero + g * W.ldr + n0 + 4 * q);
      v4i wx[MT], w1{}, x1[MT];
#pragma unroll
      for (int b = 0; b < MT; ++b) wx[b] = v4i{}, x1[b] = v4i{};
      if constexpr (kWords >= 2) {
#pragma unroll
        for (int h = 0; h < kWords / 2; ++h) {
          const int p = gp * kWords + 2 * h;
          const v4i a{(int)((ww[p] << 4) & kHigh), (int)(ww[p] & kHigh),
                      (int)((ww[p + 1] << 4) & kHigh), (int)(ww[p + 1] & kHigh)};
          w1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, one, w1, 0, 0, 0);
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            const v4i bx{xv[b][p].x, xv[b][p].y, xv[b][p + 1].x, xv[b][p + 1].y};
            wx[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, bx, wx[b], 0, 0, 0);
            x1[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(one, bx, x1[b], 0, 0, 0);
          }
        }
      } else {
        auto pair = [](uint32_t lo, uint32_t hi) { return (long)(((uint64_t)hi << 32) | lo); };
        const long a = pair((ww[gp] << 4) & kHigh, ww[gp] & kHigh);
        const long one8 = 0x0101010101010101l;
        w1 = __builtin_amdgcn_mfma_i32_16x16x32_i8(a, one8, w1, 0, 0, 0);
#pragma unroll
        for (int b = 0; b < MT; ++b) {
          const long bx = pair((uint32_t)xv[b][gp].x, (uint32_t)xv[b][gp].y);
          wx[b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(a, bx, wx[b], 0, 0, 0);
          x1[b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(one8, bx, x1[b], 0, 0, 0);
        }
      }
      const float qs[4] = {qv.x, qv.y, qv.z, qv.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float z16 = (float)(16 * ((int)(int8_t)(zv >> (8 * i)) + 8));
        const float ws = __builtin_fmaf(z16, (float)G, (float)w1[i]);
#pragma unroll
        for (int b = 0; b < MT; ++b) {
          const float t = __builtin_fmaf(z16, (float)x1[b][i], (float)wx[b][i]);
          acc[b][i] = __builtin_fmaf(qs[i], __builtin_fmaf(zt[b], ws, t), acc[b][i]);
        }
      }
    }
  }
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    const int64_t m = m0 + 16 * b + r;
    if (m >= M) continue;
    const float qx = X.inv_q[m] * 0.0625f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t n = n0 + 4 * q + i;
      if (n < ncols) {
        float y = acc[b][i] * qx;
        if (bias) y += bias[n];
        Y[m * ncols + n] = (TY)y;
      }
    }
  }
}

// ---------------------------------------------------------------- launchers
static inline unsigned blocks_for(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

hipError_t launch_quantize4(const float *W, const Q4Mat &q, int64_t cols, hipStream_t s) {
  if (q.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(k_quantize4, dim3(blocks_for(q.rows, 4)), dim3(256), 0, s, W, q.rows, cols,
                     q.codes, q.ld, q.group, q.ldr, q.zero, q.inv_q);
  return hipGetLastError();
}

hipError_t launch_dequantize4(const Q4Mat &q, int64_t cols, float *dst, hipStream_t s) {
  if (q.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(k_dequantize4, dim3(blocks_for(q.rows * (q.ld / 8), 256)), dim3(256), 0, s,
                     q.codes, q.ld, q.rows, cols, q.group, q.ldr, q.zero, q.inv_q, dst);
  return hipGetLastError();
}

hipError_t launch_quantize_rows_of(int type, const void *X, int64_t ldx, int64_t m, int64_t K,
                                   int8_t *codes, int64_t ld, int32_t *zero, float *inv_q,
                                   int32_t *sums, hipStream_t s) {
  if (m == 0) return hipSuccess;
  const dim3 grid(blocks_for(m, 4)), block(256);
  if (type == 0)
    hipLaunchKernelGGL(k_quantize_rows_of<float>, grid, block, 0, s, static_cast<const float *>(X),
                       ldx, m, K, codes, ld, zero, inv_q, sums);
  else if (type == 1)
    hipLaunchKernelGGL(k_quantize_rows_of<f16>, grid, block, 0, s, static_cast<const f16 *>(X), ldx,
                       m, K, codes, ld, zero, inv_q, sums);
  else
    hipLaunchKernelGGL(k_quantize_rows_of<bf16>, grid, block, 0, s, static_cast<const bf16 *>(X),
                       ldx, m, K, codes, ld, zero, inv_q, sums);
  return hipGetLastError();
}

template <int MT, class TY>
static void run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, TY *Y,
                        hipStream_t s) {
  const dim3 grid(blocks_for(W.rows, 64), blocks_for(M, 16 * MT));
  auto kern = W.group == 32 ? k_matmul4<32, MT, TY>
              : W.group == 64 ? k_matmul4<64, MT, TY>
                              : k_matmul4<128, MT, TY>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, W, X, M, W.rows, bias, Y);
}
template <class TY>
static void run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, TY *Y,
                        hipStream_t s) {
  if (M <= 16)
    run_matmul4<1, TY>(W, X, M, bias, Y, s);
  else if (M <= 32)
    run_matmul4<2, TY>(W, X, M, bias, Y, s);
  else
    run_matmul4<4, TY>(W, X, M, bias, Y, s);
}
hipError_t launch_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, int ytype,
                          void *Y, hipStream_t s) {
  if (M == 0 || W.rows == 0) return hipSuccess;
  if (ytype == 0)
    run_matmul4(W, X, M, bias, static_cast<float *>(Y), s);
  else if (ytype == 1)
    run_matmul4(W, X, M, bias, static_cast<f16 *>(Y), s);
  else
    run_matmul4(W, X, M, bias, static_cast<bf16 *>(Y), s);
  return hipGetLastError();
}

}  // namespace ql
