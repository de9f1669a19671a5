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

// A row of any type in registers (as the norm holds it), quantized.
template <class T, int VEC, int PER, int WAVES, bool TAIL>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void k_quantize_rows_reg(
    const T *__restrict__ X, int64_t ldx, int64_t m, int n, int8_t *__restrict__ codes, int64_t ld,
    int32_t *__restrict__ zero, float *__restrict__ inv_q, int32_t *__restrict__ sums) {
  typedef RowSlots<VEC, PER, WAVES> S;
  constexpr int kRows = (WAVES == 1 ? 256 : 64 * WAVES) / S::kThreads;
  const int t = threadIdx.x % S::kThreads;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / S::kThreads;
  if (WAVES == 1 && row >= m) return;  // (no barriers in this form)
  float v[PER];
  S::template load<TAIL>(v, X + row * ldx, n, t);
  code_row<VEC, PER, WAVES, TAIL>(v, n, t, codes + row * ld, ld, zero + row, inv_q + row, sums + row);
}

// The product.  A wave takes 16 NT rows of W (lane: row r = lane & 15 of 16, share
// q = lane >> 4 of the columns) and 16 MT rows of X.  Per group three products
// on the matrix units: W X (16 sum c x), W 1 (16 sum c) and 1 X (sum x), with
// c = V' - 8 and x = x' - 128; then, with z = z_g + 8 and zt = zx + 128,
//   16 T_g = W X + [16 z, W 1 + 16 z G] . [1 X, zt]
// is one 16-bit dot product onto the first's result, exact; one conversion and one
// fma per group follow.  (Rows whose range lies so far off 0 that zt does not
// fit 16 bits: the same in fp32, every term an integer below 2^24 but the last.)
//
// The columns are split over the waves of a workgroup, `per` runs of 128 each, and
// their sums added in order: a function of the matrix alone, so that a row's
// result does not depend on the rows beside it.  The waves' weights are read
// once, straight into registers; codes of X come through the caches, which the
// workgroups share.
template <int G, int MT, int NT, bool WIDE>
__device__ __forceinline__ void mul4_runs(const Q4Mat &W, const uint8_t *const (&w)[NT],
                                          const int8_t *const (&x)[MT], int64_t ldx,
                                          const int (&zx)[MT], int64_t n0, int q, int64_t k0,
                                          int64_t k1, float (&acc)[NT][MT][4]) {
  constexpr int kParts = 128 / G;     // groups in a run
  constexpr int kWords = 4 / kParts;  // words of a lane in a group
  const v4i one{0x01010101, 0x01010101, 0x01010101, 0x01010101};
  typedef short v2s __attribute__((ext_vector_type(2)));
  for (int64_t k = k0; k < k1; ++k) {
    uint32_t ww[NT][4];
    int2 xv[MT][4];
    float4 qv[kParts][NT];
    int zv[kParts][NT];
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      const uint4 v = *reinterpret_cast<const uint4 *>(w[a] + 64 * k);
      ww[a][0] = v.x, ww[a][1] = v.y, ww[a][2] = v.z, ww[a][3] = v.w;
    }
#pragma unroll
    for (int b = 0; b < MT; ++b)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        // columns at and past ldx recover to 0 in W: any codes serve
        const int64_t c = 128 * k + 32 * p + 8 * q;
        xv[b][p] = *reinterpret_cast<const int2 *>(x[b] + (c < ldx ? c : 0));
      }
#pragma unroll
    for (int gp = 0; gp < kParts; ++gp)
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const int64_t at = (k * kParts + gp) * W.ldr + n0 + 16 * a + 4 * q;
        qv[gp][a] = *reinterpret_cast<const float4 *>(W.inv_q + at);
        zv[gp][a] = *reinterpret_cast<const int *>(W.zero + at);
      }
#pragma unroll
    for (int gp = 0; gp < kParts; ++gp) {
      v4i wx[NT][MT], w1[NT], x1[MT];
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        w1[a] = v4i{};
#pragma unroll
        for (int b = 0; b < MT; ++b) wx[a][b] = v4i{};
      }
#pragma unroll
      for (int b = 0; b < MT; ++b) x1[b] = v4i{};
      if constexpr (kWords >= 2) {
#pragma unroll
        for (int h = 0; h < kWords / 2; ++h) {
          const int p = gp * kWords + 2 * h;
          v4i bx[MT];
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            bx[b] = v4i{xv[b][p].x, xv[b][p].y, xv[b][p + 1].x, xv[b][p + 1].y};
            x1[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(one, bx[b], x1[b], 0, 0, 0);
          }
#pragma unroll
          for (int a = 0; a < NT; ++a) {
            const v4i wa{(int)((ww[a][p] << 4) & kHigh), (int)(ww[a][p] & kHigh),
                         (int)((ww[a][p + 1] << 4) & kHigh), (int)(ww[a][p + 1] & kHigh)};
            w1[a] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa, one, w1[a], 0, 0, 0);
#pragma unroll
            for (int b = 0; b < MT; ++b)
              wx[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa, bx[b], wx[a][b], 0, 0, 0);
          }
        }
      } else {
        auto pair = [](uint32_t lo, uint32_t hi) { return (long)(((uint64_t)hi << 32) | lo); };
        const long one8 = 0x0101010101010101l;
        long bx[MT];
#pragma unroll
        for (int b = 0; b < MT; ++b) {
          bx[b] = pair((uint32_t)xv[b][gp].x, (uint32_t)xv[b][gp].y);
          x1[b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(one8, bx[b], x1[b], 0, 0, 0);
        }
#pragma unroll
        for (int a = 0; a < NT; ++a) {
          const long wa = pair((ww[a][gp] << 4) & kHigh, ww[a][gp] & kHigh);
          w1[a] = __builtin_amdgcn_mfma_i32_16x16x32_i8(wa, one8, w1[a], 0, 0, 0);
#pragma unroll
          for (int b = 0; b < MT; ++b)
            wx[a][b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(wa, bx[b], wx[a][b], 0, 0, 0);
        }
      }
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const float qs[4] = {qv[gp][a].x, qv[gp][a].y, qv[gp][a].z, qv[gp][a].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int z16 = 16 * ((int)(int8_t)(zv[gp][a] >> (8 * i)) + 8);
          const int ws = w1[a][i] + z16 * G;
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            // (every row of 1 X is alike)
            float t;
            if constexpr (WIDE) {
              t = __builtin_fmaf((float)z16, (float)x1[b][0], (float)wx[a][b][i]);
              t = __builtin_fmaf((float)zx[b], (float)ws, t);
            } else {
              const v2s u{(short)z16, (short)ws}, v{(short)x1[b][0], (short)zx[b]};
              t = (float)__builtin_amdgcn_sdot2(u, v, wx[a][b][i], false);
            }
            acc[a][b][i] = __builtin_fmaf(qs[i], t, acc[a][b][i]);
          }
        }
      }
    }
  }
}

constexpr int kSlices = 8;  // waves that the columns are split over, at most
template <int G, int MT, int NT, class TY>
__global__ __launch_bounds__(64 * kSlices) void k_matmul4(Q4Mat W, ActRows X, int64_t M, int per,
                                                          const float *__restrict__ bias,
                                                          TY *__restrict__ Y) {
  extern __shared__ float4 parts[];  // [waves][NT MT][64]
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int waves = blockDim.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * NT, m0 = (int64_t)blockIdx.y * 16 * MT;
  const uint8_t *w[NT];
#pragma unroll
  for (int a = 0; a < NT; ++a) {
    const int64_t n = n0 + 16 * a + r;
    w[a] = W.codes + (n < W.rows ? n : W.rows - 1) * (W.ld / 2) + 16 * q;
  }
  const int8_t *x[MT];
  int zx[MT];
  bool wide = false;
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    const int64_t m = m0 + 16 * b + r < M ? m0 + 16 * b + r : M - 1;
    x[b] = X.codes + m * X.ld;
    zx[b] = X.zero[m] + 128;
    wide |= zx[b] != (int)(short)zx[b];
  }
  float acc[NT][MT][4];
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < MT; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[a][b][i] = 0.0f;
  const int64_t runs = W.ld / 128, k0 = (int64_t)wave * per, k1 = k0 + per < runs ? k0 + per : runs;
  if (__any(wide))
    mul4_runs<G, MT, NT, true>(W, w, x, X.ld, zx, n0, q, k0, k1, acc);
  else
    mul4_runs<G, MT, NT, false>(W, w, x, X.ld, zx, n0, q, k0, k1, acc);
  // the waves' sums, added in order
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < MT; ++b)
      parts[(wave * NT * MT + a * MT + b) * 64 + lane] =
          make_float4(acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]);
  __syncthreads();
  for (int tile = wave; tile < NT * MT; tile += waves) {
    const int64_t n = n0 + 16 * (tile / MT) + 4 * q, m = m0 + 16 * (tile % MT) + r;
    if (n >= W.rows || m >= M) continue;
    float4 s = parts[tile * 64 + lane];
    for (int p = 1; p < waves; ++p) {
      const float4 v = parts[(p * NT * MT + tile) * 64 + lane];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    const float qx = X.inv_q[m] * 0.0625f;
    float y[4] = {s.x * qx, s.y * qx, s.z * qx, s.w * qx};
    TY *o = Y + m * W.rows + n;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (bias && n + i < W.rows) y[i] += bias[n + i];
    if (n + 4 <= W.rows) {
      store_n<4>(o, y);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < W.rows) o[i] = (TY)y[i];
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

template <class T>
static void run_quantize_rows(const T *X, int64_t ldx, int64_t m, int64_t K, int8_t *codes,
                              int64_t ld, int32_t *zero, float *inv_q, int32_t *sums,
                              hipStream_t s) {
  auto go = [&](auto per, auto w) {
    constexpr int W = decltype(w)::value, VEC = 16 / sizeof(T), PER = decltype(per)::value;
    auto kern = K % VEC == 0 ? k_quantize_rows_reg<T, VEC, PER, W, false>
                             : k_quantize_rows_reg<T, VEC, PER, W, true>;
    hipLaunchKernelGGL(kern, dim3(blocks_for(m, block_of(W) / (64 * W))), dim3(block_of(W)), 0, s, X,
                       ldx, m, (int)K, codes, ld, zero, inv_q, sums);
  };
  const bool done = m >= 512 ? by_row<true>(K, go) : by_row<false>(K, go);
  if (!done)
    hipLaunchKernelGGL(k_quantize_rows_of<T>, dim3(blocks_for(m, 4)), dim3(256), 0, s, X, ldx, m, K,
                       codes, ld, zero, inv_q, sums);
}
hipError_t launch_quantize_rows_of(int type, const void *X, int64_t ldx, int64_t m, int64_t K,
                                   int8_t *codes, int64_t ld, int32_t *zero, float *inv_q,
                                   int32_t *sums, hipStream_t s) {
  if (m == 0) return hipSuccess;
  if (type == 0)
    run_quantize_rows(static_cast<const float *>(X), ldx, m, K, codes, ld, zero, inv_q, sums, s);
  else if (type == 1)
    run_quantize_rows(static_cast<const f16 *>(X), ldx, m, K, codes, ld, zero, inv_q, sums, s);
  else
    run_quantize_rows(static_cast<const bf16 *>(X), ldx, m, K, codes, ld, zero, inv_q, sums, s);
  return hipGetLastError();
}

template <int MT, int NT, class TY>
static void run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, TY *Y,
                        hipStream_t s) {
  const int runs = (int)(W.ld / 128);
  int waves = 1;
  while (waves < kSlices && 2 * waves <= runs) waves *= 2;
  const int per = (runs + waves - 1) / waves;
  const dim3 grid(blocks_for(W.rows, 16 * NT), blocks_for(M, 16 * MT));
  auto kern = W.group == 32 ? k_matmul4<32, MT, NT, TY>
              : W.group == 64 ? k_matmul4<64, MT, NT, TY>
                              : k_matmul4<128, MT, NT, TY>;
  hipLaunchKernelGGL(kern, grid, dim3(64 * waves), waves * NT * MT * 64 * sizeof(float4), s, W, X, M,
                     per, bias, Y);
}
template <class TY>
static void run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, TY *Y,
                        hipStream_t s) {
  if (M <= 16)
    run_matmul4<1, 1, TY>(W, X, M, bias, Y, s);
  else if (M <= 32)
    run_matmul4<2, 2, TY>(W, X, M, bias, Y, s);
  else
    run_matmul4<4, 2, TY>(W, X, M, bias, Y, s);
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
