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

#include <algorithm>

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
// The columns are cut into slices that the waves of a workgroup share, and the
// slices' sums added in an order that depends on the matrix alone: a row's result
// does not depend on the rows beside it.
// One run's scales and zero points of the lane's 4 NT output rows.
template <int G, int NT>
struct RunScales {
  static constexpr int kParts = 128 / G;  // groups in a run
  float4 q[kParts][NT];
  int z[kParts][NT];
  __device__ __forceinline__ void load(const Q4Mat &W, int64_t k, int64_t n) {
#pragma unroll
    for (int gp = 0; gp < kParts; ++gp)
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const int64_t at = (k * kParts + gp) * W.ldr + n + 16 * a;
        q[gp][a] = *reinterpret_cast<const float4 *>(W.inv_q + at);
        z[gp][a] = *reinterpret_cast<const int *>(W.zero + at);
      }
  }
};
// One run: the lane's 16 bytes of each 16 rows of W against its codes of X, four
// 8-byte pieces (32 columns apart) of each 16 rows.
template <int G, int MT, int NT, bool WIDE>
__device__ __forceinline__ void mul4_run(const uint4 (&wv)[NT], const int2 (&xv)[MT][4],
                                         const RunScales<G, NT> &sc, const int (&zx)[MT],
                                         float (&acc)[NT][MT][4]) {
  constexpr int kParts = 128 / G;
  constexpr int kWords = 4 / kParts;  // words of a lane in a group
  const v4i one{0x01010101, 0x01010101, 0x01010101, 0x01010101};
  typedef short v2s __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int gp = 0; gp < kParts; ++gp) {
    v4i x1[MT];
#pragma unroll
    for (int b = 0; b < MT; ++b) x1[b] = v4i{};
    auto pair = [](uint32_t lo, uint32_t hi) { return (long)(((uint64_t)hi << 32) | lo); };
    const long one8 = 0x0101010101010101l;
#pragma unroll
    for (int b = 0; b < MT; ++b) {
      if constexpr (kWords >= 2) {
#pragma unroll
        for (int p = gp * kWords; p < (gp + 1) * kWords; p += 2)
          x1[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              one, v4i{xv[b][p].x, xv[b][p].y, xv[b][p + 1].x, xv[b][p + 1].y}, x1[b], 0, 0, 0);
      } else {
        x1[b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(
            one8, pair((uint32_t)xv[b][gp].x, (uint32_t)xv[b][gp].y), x1[b], 0, 0, 0);
      }
    }
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      const uint32_t ww[4] = {wv[a].x, wv[a].y, wv[a].z, wv[a].w};
      v4i wx[MT], w1{};
#pragma unroll
      for (int b = 0; b < MT; ++b) wx[b] = v4i{};
      if constexpr (kWords >= 2) {
#pragma unroll
        for (int p = gp * kWords; p < (gp + 1) * kWords; p += 2) {
          const v4i wa{(int)((ww[p] << 4) & kHigh), (int)(ww[p] & kHigh),
                       (int)((ww[p + 1] << 4) & kHigh), (int)(ww[p + 1] & kHigh)};
          w1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa, one, w1, 0, 0, 0);
#pragma unroll
          for (int b = 0; b < MT; ++b)
            wx[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                wa, v4i{xv[b][p].x, xv[b][p].y, xv[b][p + 1].x, xv[b][p + 1].y}, wx[b], 0, 0, 0);
        }
      } else {
        const long wa = pair((ww[gp] << 4) & kHigh, ww[gp] & kHigh);
        w1 = __builtin_amdgcn_mfma_i32_16x16x32_i8(wa, one8, w1, 0, 0, 0);
#pragma unroll
        for (int b = 0; b < MT; ++b)
          wx[b] = __builtin_amdgcn_mfma_i32_16x16x32_i8(
              wa, pair((uint32_t)xv[b][gp].x, (uint32_t)xv[b][gp].y), wx[b], 0, 0, 0);
      }
      const float qs[4] = {sc.q[gp][a].x, sc.q[gp][a].y, sc.q[gp][a].z, sc.q[gp][a].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int z16 = 16 * ((int)(int8_t)(sc.z[gp][a] >> (8 * i)) + 8);
        const int ws = w1[i] + z16 * G;
#pragma unroll
        for (int b = 0; b < MT; ++b) {
          // (every row of 1 X is alike)
          float t;
          if constexpr (WIDE) {
            t = __builtin_fmaf((float)z16, (float)x1[b][0], (float)wx[b][i]);
            t = __builtin_fmaf((float)zx[b], (float)ws, t);
          } else {
            const v2s u{(short)z16, (short)ws}, v{(short)x1[b][0], (short)zx[b]};
            t = (float)__builtin_amdgcn_sdot2(u, v, wx[b][i], false);
          }
          acc[a][b][i] = __builtin_fmaf(qs[i], t, acc[a][b][i]);
        }
      }
    }
  }
}

// The columns' slices: `n` (a power of two up to kSlices, a function of the columns
// alone) of `per` runs each.  A slice is summed run by run; the sums of slices
// 2 i and 2 i + 1 are added, then those of the pairs in order, whichever kernel
// does it.
constexpr int kSlices = 8;
struct Slices {
  int n, per;
};

template <int NT, int MT>
__device__ __forceinline__ void zero_acc(float (&acc)[NT][MT][4]) {
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < MT; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[a][b][i] = 0.0f;
}
// Four neighbouring results of row m: Y[m][n ..] = s qx / 16 + bias.
template <class TY>
__device__ __forceinline__ void put4(float4 s, int64_t m, int64_t n, int64_t rows, const ActRows &X,
                                     const float *bias, TY *Y) {
  const float qx = X.inv_q[m] * 0.0625f;
  float y[4] = {s.x * qx, s.y * qx, s.z * qx, s.w * qx};
  TY *o = Y + m * rows + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (bias && n + i < rows) y[i] += bias[n + i];
  if (n + 4 <= rows) {
    store_n<4>(o, y);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < rows) o[i] = (TY)y[i];
  }
}
__device__ __forceinline__ float4 add4(float4 a, float4 b) {
  return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}

// Up to 16 rows of X: 16 rows of W a workgroup, a wave per slice.  What is read is W,
// once, straight into registers, AHEAD runs at a time in flight.
template <int G, bool WIDE, int AHEAD>
__device__ __forceinline__ void mul4_slice(const Q4Mat &W, const uint8_t *w, const int8_t *x,
                                           int64_t ldx, int zx0, int64_t n, int q, int64_t k0,
                                           int64_t k1, float (&acc)[1][1][4]) {
  const int zx[1] = {zx0};
  for (int64_t k = k0; k < k1; k += AHEAD) {
    uint4 wv[AHEAD][1];
    int2 xv[AHEAD][1][4];
    RunScales<G, 1> sc[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t ku = k + u < k1 ? k + u : k1 - 1;
      wv[u][0] = *reinterpret_cast<const uint4 *>(w + 64 * ku);
      sc[u].load(W, ku, n);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        // columns at and past ldx recover to 0 in W: any codes serve
        const int64_t c = 128 * ku + 32 * p + 8 * q;
        xv[u][0][p] = *reinterpret_cast<const int2 *>(x + (c < ldx ? c : 0));
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (k + u < k1) mul4_run<G, 1, 1, WIDE>(wv[u], xv[u], sc[u], zx, acc);
  }
}
template <int G, class TY>
__global__ __launch_bounds__(64 * kSlices) void k_matmul4_few(Q4Mat W, ActRows X, int64_t M,
                                                              Slices sl,
                                                              const float *__restrict__ bias,
                                                              TY *__restrict__ Y) {
  __shared__ float4 parts[kSlices][64];
  constexpr int kAhead = G == 32 ? 2 : 4;
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + 4 * q;
  const uint8_t *w =
      W.codes + (n0 + r < W.rows ? n0 + r : W.rows - 1) * (W.ld / 2) + 16 * q;
  const int64_t m = r < M ? r : M - 1;
  const int8_t *x = X.codes + m * X.ld;
  const int zx = X.zero[m] + 128;
  float acc[1][1][4];
  zero_acc(acc);
  const int64_t runs = W.ld / 128, k0 = (int64_t)wave * sl.per,
                k1 = k0 + sl.per < runs ? k0 + sl.per : runs;
  if (__any(zx != (int)(short)zx))
    mul4_slice<G, true, 1>(W, w, x, X.ld, zx, n, q, k0, k1, acc);
  else
    mul4_slice<G, false, kAhead>(W, w, x, X.ld, zx, n, q, k0, k1, acc);
  parts[wave][lane] = make_float4(acc[0][0][0], acc[0][0][1], acc[0][0][2], acc[0][0][3]);
  __syncthreads();
  if (wave > 0 || n >= W.rows || r >= M) return;
  float4 s = parts[0][lane];
  if (sl.n > 1) s = add4(s, parts[1][lane]);
  for (int p = 2; p < sl.n; p += 2) s = add4(s, add4(parts[p][lane], parts[p + 1][lane]));
  put4(s, r, n, W.rows, X, bias, Y);
}

// More rows of X: a workgroup takes 32 NT rows of W and 16 MT of X.  Two waves share
// the codes of a pair of slices, run by run through LDS, laid out there as the
// lanes read them (their four 8-byte pieces together); W still goes straight to
// registers.  The next run's loads are in flight while one is multiplied.
template <int G, int MT, int NT, bool WIDE>
__device__ __forceinline__ void mul4_pair(const Q4Mat &W, const ActRows &X, int64_t M,
                                          const Slices &sl, int64_t m0, int64_t n0, int pair,
                                          int half, const int (&zx)[MT], int8_t *lds,
                                          float (&tot)[NT][MT][4]) {
  constexpr int kPitch = 144;                 // bytes of a row's run in LDS: 128, and off the banks
  constexpr int kBuf = 16 * MT * kPitch;
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int64_t runs = W.ld / 128, k0 = (int64_t)pair * 2 * sl.per;
  const int count = sl.n > 1 ? 2 * sl.per : sl.per;
  const uint8_t *w[NT];
#pragma unroll
  for (int a = 0; a < NT; ++a) {
    const int64_t n = n0 + 16 * a + r;
    w[a] = W.codes + (n < W.rows ? n : W.rows - 1) * (W.ld / 2) + 16 * q;
  }
  // staging: 128 threads, a 16-byte chunk of every 16th row each
  const int th = half * 64 + lane, chunk = th & 7;
  const int8_t *src[MT];
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    const int64_t m = m0 + 16 * b + (th >> 3);
    src[b] = X.codes + (m < M ? m : M - 1) * X.ld;
  }
  int4 xr[MT];
  uint4 wn[NT];
  RunScales<G, NT> sn;
  auto fetch = [&](int64_t k) {
    const int64_t c = 128 * k + 16 * chunk;
#pragma unroll
    for (int b = 0; b < MT; ++b)
      xr[b] = *reinterpret_cast<const int4 *>(src[b] + (c < X.ld ? c : 0));
#pragma unroll
    for (int a = 0; a < NT; ++a) wn[a] = *reinterpret_cast<const uint4 *>(w[a] + 64 * k);
    sn.load(W, k, n0 + 4 * q);
  };
  auto stage = [&](int buf) {  // columns 32 p + 8 i .. + 7 of a run to i 32 + p 8
#pragma unroll
    for (int b = 0; b < MT; ++b) {
      int8_t *d = lds + buf * kBuf + (16 * b + (th >> 3)) * kPitch;
      const int e = 2 * chunk;
      *reinterpret_cast<int2 *>(d + (e & 3) * 32 + (e >> 2) * 8) = make_int2(xr[b].x, xr[b].y);
      *reinterpret_cast<int2 *>(d + ((e + 1) & 3) * 32 + (e >> 2) * 8) =
          make_int2(xr[b].z, xr[b].w);
    }
  };
  float acc[NT][MT][4];
  zero_acc(acc);
  zero_acc(tot);
  if (k0 < runs) {
    fetch(k0);
    stage(0);
  }
  __syncthreads();
  for (int i = 0; i < count; ++i) {
    const int64_t k = k0 + i;
    uint4 wv[NT];
    RunScales<G, NT> sc = sn;
#pragma unroll
    for (int a = 0; a < NT; ++a) wv[a] = wn[a];
    const bool more = i + 1 < count && k + 1 < runs;
    if (more) fetch(k + 1);
    if (k < runs) {
      int2 xv[MT][4];
      const int8_t *d = lds + (i & 1) * kBuf + r * kPitch + 32 * q;
#pragma unroll
      for (int b = 0; b < MT; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int4 v = *reinterpret_cast<const int4 *>(d + 16 * b * kPitch + 16 * h);
          xv[b][2 * h] = make_int2(v.x, v.y);
          xv[b][2 * h + 1] = make_int2(v.z, v.w);
        }
      mul4_run<G, MT, NT, WIDE>(wv, xv, sc, zx, acc);
    }
    if (i + 1 == sl.per || i + 1 == count) {  // a slice ends
#pragma unroll
      for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < MT; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) tot[a][b][e] = i + 1 == sl.per ? acc[a][b][e] : tot[a][b][e] + acc[a][b][e];
      zero_acc(acc);
    }
    if (more) stage((i + 1) & 1);
    __syncthreads();
  }
}
template <int G, int MT, int NT, class TY>
__global__ __launch_bounds__(512) void k_matmul4(Q4Mat W, ActRows X, int64_t M, Slices sl,
                                                 const float *__restrict__ bias,
                                                 TY *__restrict__ Y) {
  constexpr int kBuf = 16 * MT * 144;
  // per pair two buffers of codes; after the loop the pairs' sums
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int half = wave & 1, pair = wave >> 1, pairs = blockDim.x >> 7;
  const int64_t n0 = (int64_t)blockIdx.x * 32 * NT + 16 * NT * half;
  const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
  int zx[MT];
  bool wide = false;
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    const int64_t m = m0 + 16 * b + r < M ? m0 + 16 * b + r : M - 1;
    zx[b] = X.zero[m] + 128;
    wide |= zx[b] != (int)(short)zx[b];
  }
  // rows of W past the last: the last ones' loads, no stores (their scales' places
  // are W.ldr wide, which 16 NT rows from n0 may pass)
  const int64_t nl = n0 + 16 * NT <= W.ldr ? n0 : W.ldr - 16 * NT;
  float tot[NT][MT][4];
  if (__any(wide))  // (alike in every wave: all see the same rows of X)
    mul4_pair<G, MT, NT, true>(W, X, M, sl, m0, nl, pair, half, zx, lds + pair * 2 * kBuf, tot);
  else
    mul4_pair<G, MT, NT, false>(W, X, M, sl, m0, nl, pair, half, zx, lds + pair * 2 * kBuf, tot);
  float4 *parts = reinterpret_cast<float4 *>(lds);  // [pairs][2][NT MT][64]
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < MT; ++b)
      parts[((pair * 2 + half) * NT * MT + a * MT + b) * 64 + lane] =
          make_float4(tot[a][b][0], tot[a][b][1], tot[a][b][2], tot[a][b][3]);
  __syncthreads();
  for (int tile = pair; tile < NT * MT; tile += pairs) {
    const int64_t n = nl + 16 * (tile / MT) + 4 * q, m = m0 + 16 * (tile % MT) + r;
    if (n < n0 || n >= W.rows || m >= M) continue;
    float4 s = parts[(half * NT * MT + tile) * 64 + lane];
    for (int p = 1; p < pairs; ++p)
      s = add4(s, parts[((p * 2 + half) * NT * MT + tile) * 64 + lane]);
    put4(s, m, n, W.rows, X, bias, Y);
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
static hipError_t run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const Slices &sl,
                        const float *bias, TY *Y, hipStream_t s) {
  const int pairs = sl.n > 1 ? sl.n / 2 : 1;
  const size_t codes = (size_t)pairs * 2 * 16 * MT * 144;
  const size_t sums = (size_t)pairs * 2 * NT * MT * 64 * sizeof(float4);
  auto kern = W.group == 32 ? k_matmul4<32, MT, NT, TY>
              : W.group == 64 ? k_matmul4<64, MT, NT, TY>
                              : k_matmul4<128, MT, NT, TY>;
  const size_t lds = std::max(codes, sums);
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(blocks_for(W.rows, 32 * NT), blocks_for(M, 16 * MT)),
                     dim3(128 * pairs), lds, s, W, X, M, sl, bias, Y);
  return hipGetLastError();
}
template <class TY>
static hipError_t run_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, TY *Y,
                              hipStream_t s) {
  const int runs = (int)(W.ld / 128);
  Slices sl{1, 0};
  while (sl.n < kSlices && 2 * sl.n <= runs) sl.n *= 2;
  sl.per = (runs + sl.n - 1) / sl.n;
  if (M <= 16) {
    auto kern = W.group == 32 ? k_matmul4_few<32, TY>
                : W.group == 64 ? k_matmul4_few<64, TY>
                                : k_matmul4_few<128, TY>;
    hipLaunchKernelGGL(kern, dim3(blocks_for(W.rows, 16)), dim3(64 * sl.n), 0, s, W, X, M, sl, bias,
                       Y);
    return hipGetLastError();
  }
  if (M <= 32) return run_matmul4<2, 1, TY>(W, X, M, sl, bias, Y, s);
  if (W.ldr >= 32 && W.rows * ((M + 63) / 64) >= 64 * 256)
    return run_matmul4<4, 2, TY>(W, X, M, sl, bias, Y, s);
  return run_matmul4<4, 1, TY>(W, X, M, sl, bias, Y, s);
}
hipError_t launch_matmul4(const Q4Mat &W, const ActRows &X, int64_t M, const float *bias, int ytype,
                          void *Y, hipStream_t s) {
  if (M == 0 || W.rows == 0) return hipSuccess;
  if (ytype == 0) return run_matmul4(W, X, M, bias, static_cast<float *>(Y), s);
  if (ytype == 1) return run_matmul4(W, X, M, bias, static_cast<f16 *>(Y), s);
  return run_matmul4(W, X, M, bias, static_cast<bf16 *>(Y), s);
}

}  // namespace ql
