// The linear layer y = act(x W^T + b) + r and its gradient.
//
//   z = x W^T + b;  y = act(z) + r
//   dz = dy act'(z);  dx = dz W;  dW = dz^T x;  db = column sums of dz;  dr = dy
//
// Products and everything behind them are fp32 until the one rounding of what is stored: y from the unrounded z, and z
// itself if it is kept for the gradient.  dz is rounded to the operands' type where it enters the two products (the
// matrix cores take both operands in one type); db sums the unrounded dz.
#pragma once
#include "kernels_gemm.h"
#include "../../include/memdet.h"

namespace mdet {

// ---------------------------------------------------------------------------
// Activations.  Clamping keeps infinities out of products with zero: a z that has overflowed its 16-bit storage still
// has the slope of its side.  (Comparisons, not fmin / fmax, which would turn NaN into a number.)
// ---------------------------------------------------------------------------
constexpr float ACT_R2 = 0.70710678118654752f, ACT_R2PI = 0.39894228040143268f;
constexpr float ACT_TANH_A = 0.79788456080286536f, ACT_TANH_B = 0.044715f;

__device__ __forceinline__ float act_clamp(float z, float least, float most) {
  return z < least ? least : z > most ? most : z;
}

// 1 / (1 + exp(-t)).  For operands in fp32 without an exponential that overflows: what is small has its digits down to the least number.
template <typename T>
__device__ __forceinline__ float logistic(const float t) {
  if constexpr (sizeof(T) == 4) {
    const float e = expf(-fabsf(t));
    return (t < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
  } else return 1.0f / (1.0f + __expf(-t));
}

// Phi(z) and e = exp(-z^2 / 2), |z| <= 20.  1 - erf(x), x = |z| / sqrt(2), is exp(-x^2) times a polynomial in t = 1 / (1 + p x): a third of
// erff's instructions, which as the tail of a large product cost 10 % of its time, and no branch.
//
// For operands in 16 bits degree 5 to 1.5e-7 in all (Abramowitz and Stegun, 7.1.26).  Half of that error is 2^-23.7 of a factor that
// goes up to 1; of a small factor it is a larger part (5e-4 at z = -4, 2e-3 at -5), where rounding to 16 bits is one of up to
// 4e-3 (bf16) or 5e-4.
//
// For fp32 degree 8 to 4.4e-8 of the factor itself, however small: the best polynomial in that sense for t exp(x^2) (1 - erf(x)) over
// 0 <= x <= 14.2 (Remez exchange), p = 1/2.  erfcf in its place takes 89 us for 4096 x 8192 x 64 and 975 for 4096^3; this, 70 and 966.
template <typename T>
__device__ __forceinline__ float normal_cdf(const float z, float& e) {
  const float x = fabsf(z) * ACT_R2;
  if constexpr (sizeof(T) == 4) {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.5f * x);
    e = __expf(-0.5f * z * z);
    float q = -0.059386346489f;
    q = q * t + 0.286123484373f;
    q = q * t - 0.490405529737f;
    q = q * t + 0.281732559204f;
    q = q * t - 0.029148206115f;
    q = q * t + 0.203752472997f;
    q = q * t + 0.242835104465f;
    q = q * t + 0.282412111759f;
    q = q * t + 0.282084345818f;
    q *= 0.5f * e * t;
    return z < 0.0f ? q : 1.0f - q;
  } else {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    e = __expf(-x * x);
    const float q = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    return z < 0.0f ? q : 1.0f - q;
  }
}

// T: type of the operands.
template <typename T, int ACT>
__device__ __forceinline__ float act_value(const float z) {
  if constexpr (ACT == MDET_ACT_RELU) return z < 0.0f ? 0.0f : z;
  else if constexpr (ACT == MDET_ACT_GELU) {
    const float c = z < -20.0f ? -20.0f : z;         // the factor is zero there already
    float e;
    return c * normal_cdf<T>(c > 20.0f ? 20.0f : c, e);
  } else if constexpr (ACT == MDET_ACT_GELU_TANH) {
    const float c = z < -20.0f ? -20.0f : z;
    const float t = act_clamp(c, -20.0f, 20.0f);     // (1 + tanh(u)) / 2 = logistic(2 u)
    return c * logistic<T>(2.0f * ACT_TANH_A * (t + ACT_TANH_B * t * t * t));
  } else if constexpr (ACT == MDET_ACT_SILU) {
    const float c = z < -80.0f ? -80.0f : z;
    return c * logistic<T>(c);
  } else return z;
}

template <typename T, int ACT>
__device__ __forceinline__ float act_slope(const float z) {
  if constexpr (ACT == MDET_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
  else if constexpr (ACT == MDET_ACT_GELU) {
    const float c = act_clamp(z, -20.0f, 20.0f);
    float e;
    const float cdf = normal_cdf<T>(c, e);
    return cdf + c * e * ACT_R2PI;
  } else if constexpr (ACT == MDET_ACT_GELU_TANH) {
    const float c = act_clamp(z, -20.0f, 20.0f);
    const float q = logistic<T>(2.0f * ACT_TANH_A * (c + ACT_TANH_B * c * c * c));
    return q + 2.0f * c * q * (1.0f - q) * ACT_TANH_A * (1.0f + 3.0f * ACT_TANH_B * c * c);
  } else if constexpr (ACT == MDET_ACT_SILU) {
    const float c = act_clamp(z, -80.0f, 80.0f);
    const float q = logistic<T>(c);
    return q * (1.0f + c * (1.0f - q));
  } else return 1.0f;
}

// The activation is known at run time: `f` gets it as a constant.
template <typename F>
__device__ __forceinline__ void act_switch(const int act, F&& f) {
  switch (act) {
    case MDET_ACT_RELU: f(std::integral_constant<int, MDET_ACT_RELU>{}); break;
    case MDET_ACT_GELU: f(std::integral_constant<int, MDET_ACT_GELU>{}); break;
    case MDET_ACT_GELU_TANH: f(std::integral_constant<int, MDET_ACT_GELU_TANH>{}); break;
    case MDET_ACT_SILU: f(std::integral_constant<int, MDET_ACT_SILU>{}); break;
    default: f(std::integral_constant<int, MDET_ACT_NONE>{});
  }
}

// What happens to a sum of products on its way out.  T: type of the operands, O: of what is stored.
template <typename T, typename O>
struct LinearOut {
  O* y;
  int64_t ldy;
  const T* bias;                       // null: none
  const T* residual;                   // null: none
  int64_t ldr;
  T* z;                                // null: not kept
  int64_t ldz;
  int act;
  int64_t rows, cols;
  bool vec;                            // rows of y, bias, residual and z start where four elements can be moved at once
};

template <typename T, typename O, int ACT>
__device__ __forceinline__ void linear_put(const LinearOut<T, O>& o, const int64_t i, const int64_t j, float v) {
  if (o.bias) v += (float)o.bias[j];
  if (o.z) o.z[i * o.ldz + j] = (T)v;
  v = act_value<T, ACT>(v);
  if (o.residual) v += (float)o.residual[i * o.ldr + j];
  o.y[i * o.ldy + j] = (O)v;
}

// Four neighbours of a row, from column j on.
template <typename T, typename O, int ACT>
__device__ __forceinline__ void linear_put4(const LinearOut<T, O>& o, const int64_t i, const int64_t j, const float (&in)[4]) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  typedef O o4 __attribute__((ext_vector_type(4)));
  if (!o.vec || j + 4 > o.cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < o.cols) linear_put<T, O, ACT>(o, i, j + e, in[e]);
    return;
  }
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = in[e];
  if (o.bias) {
    const t4 b = *reinterpret_cast<const t4*>(o.bias + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += (float)b[e];
  }
  if (o.z) {
    t4 z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = (T)v[e];
    *reinterpret_cast<t4*>(o.z + i * o.ldz + j) = z;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = act_value<T, ACT>(v[e]);
  if (o.residual) {
    const t4 r = *reinterpret_cast<const t4*>(o.residual + i * o.ldr + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += (float)r[e];
  }
  o4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (O)v[e];
  *reinterpret_cast<o4*>(o.y + i * o.ldy + j) = y;
}

// Rows of a wavefront's part that go through its share of LDS at once on their way out: what lies 16 lanes apart in the
// accumulators is put side by side, whole lines leave, and the code of the activations stands once in a loop.
template <typename S>
struct LinearLds {
  static constexpr int ROWS = S::TM * 16 < 64 ? S::TM * 16 : 64, COLS = S::TN * 16, PITCH = COLS + 4;
  static constexpr int WAVE_BYTES = ROWS * PITCH * 4;
  static constexpr int BYTES = S::WAVES * WAVE_BYTES > S::NB * S::SLAB ? S::WAVES * WAVE_BYTES : S::NB * S::SLAB;
};

// Tile number t of the layer.  SPLIT: part t / tiles of the sum over k, kept in fp32 for linear_join_kernel.
template <typename T, typename O, typename S, bool ROUTER, bool COUTER, bool DIRECT, bool SPLIT>
__device__ __forceinline__ void linear_tile(const int64_t t, char* const lds, const Operand<T>& r, const Operand<T>& c, const int64_t k,
                                            const LinearOut<T, O>& out, float* const parts, const int64_t kpart) {
  typedef LinearLds<S> L;
  const int64_t down = (out.rows + S::BM - 1) / S::BM, across = (out.cols + S::BN - 1) / S::BN, tiles = down * across;
  int64_t bi, bj;
  gemm_tile_place(t % tiles, down, across, bi, bj);
  const int64_t part = t / tiles, k0 = part * kpart, kend = k0 + kpart < k ? k0 + kpart : k;
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  typename Core<T>::acc_t acc[S::TN][S::TM] = {};
  TileStream<T, S, ROUTER, COUTER, DIRECT> stream(lds);
  auto none = [] { return false; };
  stream.set(r, c, row0, col0, k0, kend);
  stream.begin(none);
  stream.run(acc, stream.slabs(k0, kend), none);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  float* const mine = reinterpret_cast<float*>(lds + wave * L::WAVE_BYTES);
  const int64_t wrow = row0 + wave / S::WN * S::TM * 16, wcol = col0 + wave % S::WN * S::TN * 16;
  constexpr int LANES = L::COLS / 4, STEP = 64 / LANES;        // lanes of a row, rows of a step
  __syncthreads();                                             // the operands are not read any more
#pragma unroll
  for (int b0 = 0; b0 < S::TM; b0 += L::ROWS / 16) {
#pragma unroll
    for (int b = 0; b < L::ROWS / 16; ++b)
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
        *reinterpret_cast<typename Core<T>::acc_t*>(mine + (16 * b + (lane & 15)) * L::PITCH + 16 * a + 4 * (lane >> 4)) = acc[a][b0 + b];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    auto rows = [&](auto&& f) {
#pragma unroll 1
      for (int s = 0; s < L::ROWS; s += STEP) {
        const int row = s + lane / LANES, col = lane % LANES * 4;
        const int64_t i = wrow + b0 * 16 + row, j = wcol + col;
        const typename Core<T>::acc_t v = *reinterpret_cast<const typename Core<T>::acc_t*>(mine + row * L::PITCH + col);
        const float in[4] = {v[0], v[1], v[2], v[3]};
        if (i < out.rows && j < out.cols) f(i, j, in);
      }
    };
    if constexpr (SPLIT) {
      float* const to = parts + part * out.rows * out.cols;
      const bool vec = out.cols % 4 == 0;
      rows([&](const int64_t i, const int64_t j, const float (&in)[4]) {
        if (vec) *reinterpret_cast<typename Core<T>::acc_t*>(to + i * out.cols + j) = typename Core<T>::acc_t{in[0], in[1], in[2], in[3]};
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j + e < out.cols) to[i * out.cols + j + e] = in[e];
      });
    } else {
      act_switch(out.act, [&](auto act) {
        rows([&](const int64_t i, const int64_t j, const float (&in)[4]) { linear_put4<T, O, decltype(act)::value>(out, i, j, in); });
      });
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// y, dx and dW.  The matrix cores bound it, in 16 bits together with the waits between slabs: 8192 x 16384 x 4096 bf16 1250
// TFLOP/s, dx and dW of 4096 x 8192 x 4096 1390 and 1350; 4096^3 fp32 143.
template <typename T, typename O, typename S, bool ROUTER, bool COUTER, bool DIRECT, bool SPLIT>
__global__ __launch_bounds__(S::THREADS) void linear_tile_kernel(const Operand<T> r, const Operand<T> c, const int64_t k, const LinearOut<T, O> out,
                                                                 const int64_t tiles, float* const parts, const int64_t kpart) {
  __shared__ __attribute__((aligned(16))) char lds[LinearLds<S>::BYTES];
  const int64_t t = gemm_tile_number(blockIdx.x, tiles);
  if (t >= 0) linear_tile<T, O, S, ROUTER, COUTER, DIRECT, SPLIT>(t, lds, r, c, k, out, parts, kpart);
}

// Both products of a small layer's gradient in one launch, which fills the device where neither would: dx = dz W by the
// first tiles, dW = dz^T x by the others.
template <typename T, typename O, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void linear_pair_kernel(const Operand<T> dzr, const Operand<T> w, const int64_t n, const LinearOut<T, T> dx,
                                                                 const Operand<T> dzc, const Operand<T> x, const int64_t m, const LinearOut<T, O> dw,
                                                                 const int64_t first, const int64_t tiles) {
  __shared__ __attribute__((aligned(16))) char lds[LinearLds<S>::BYTES];
  const int64_t t = gemm_tile_number(blockIdx.x, tiles);
  if (t < 0) return;
  if (t < first) linear_tile<T, T, S, false, true, DIRECT, false>(t, lds, dzr, w, n, dx, nullptr, n);
  else linear_tile<T, O, S, true, true, DIRECT, false>(t - first, lds, dzc, x, m, dw, nullptr, m);
}

// The parts of the sum over k, added in their order, on their way out.
template <typename T, typename O>
__global__ __launch_bounds__(256) void linear_join_kernel(const float* __restrict__ parts, const int splits, const LinearOut<T, O> out) {
  const int64_t across = (out.cols + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = id / across, j = id % across * 4;
  if (i >= out.rows) return;
  const int64_t size = out.rows * out.cols;
  const float* from = parts + i * out.cols + j;
  float v[4] = {};
  if (out.cols % 4 == 0) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    for (int s = 0; s < splits; ++s, from += size) {
      const f4 x = *reinterpret_cast<const f4*>(from);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[e];
    }
  } else {
    for (int s = 0; s < splits; ++s, from += size)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < out.cols) v[e] += from[e];
  }
  act_switch(out.act, [&](auto act) { linear_put4<T, O, decltype(act)::value>(out, i, j, v); });
}

// Up to 16 rows of x (single tokens): W is read once, 16 rows of it by a workgroup whose wavefronts share k, each piece
// straight into the registers of its product.  Bytes of W bound it, and how many are on their way: sixteen wavefronts a
// workgroup (4096 x 4096 bf16, one row: 8.7 us, 3.9 TB/s; with four 9.4, as split 32-row tiles and a join 11.4).
template <typename T, typename O, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_rows_kernel(const Operand<T> x, const Operand<T> w, const int64_t k, const LinearOut<T, O> out) {
  typedef typename Core<T>::piece_t piece_t;
  typedef typename Core<T>::acc_t acc_t;
  constexpr int VEC = Core<T>::VEC, STEP = 4 * VEC, UNROLL = 8;
  __shared__ acc_t sums[WAVES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), j = lane & 15, g = lane >> 4;
  const int64_t col0 = (int64_t)blockIdx.x * 16;
  // rows behind the last are not stored
  const T* const wp = w.p + (col0 + j < w.rows ? col0 + j : w.rows - 1) * w.stride + g * VEC;
  const T* const xp = x.p + (j < x.rows ? j : x.rows - 1) * x.stride + g * VEC;
  acc_t acc = {};
  const int64_t steps = k / STEP, each = (steps + WAVES - 1) / WAVES;
  int64_t s = wave * each;
  const int64_t end = s + each < steps ? s + each : steps;
  auto some = [&](auto count) {
    constexpr int U = decltype(count)::value;
    piece_t wf[U], xf[U];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(&wf[u], wp + (s + u) * STEP, 16);
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(&xf[u], xp + (s + u) * STEP, 16);
#pragma unroll
    for (int u = 0; u < U; ++u) Core<T>::mma(wf[u], xf[u], acc);
  };
  for (; s + UNROLL <= end; s += UNROLL) some(std::integral_constant<int, UNROLL>{});
  for (; s < end; ++s) some(std::integral_constant<int, 1>{});
  if (wave == WAVES - 1 && steps * STEP < k) {                 // what is left over, element by element
    const int64_t at = steps * STEP;
    piece_t wf = {}, xf = {};
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (at + g * VEC + e < k) {
        wf[e] = wp[at + e];
        xf[e] = xp[at + e];
      }
    Core<T>::mma(wf, xf, acc);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave == 0) {
    acc_t v = sums[0][lane];
#pragma unroll
    for (int p = 1; p < WAVES; ++p) v += sums[p][lane];
    const int64_t c = col0 + 4 * g;
    const float in[4] = {v[0], v[1], v[2], v[3]};
    if (j < out.rows && c < out.cols) act_switch(out.act, [&](auto act) { linear_put4<T, O, decltype(act)::value>(out, j, c, in); });
  }
}

// dz = dy act'(z) and the column sums of 16 EACH rows of it.  A workgroup takes 16 pieces of 16 bytes across; thread (t, c)
// every sixteenth row of piece c, all of its loads at once.  Bytes bound it (4096 x 8192 bf16 with GELU: 42 us, 4.8 TB/s).
constexpr int DZ_PIECES = 16;

template <typename T, int EACH>
__global__ __launch_bounds__(256) void linear_dz_kernel(const T* __restrict__ dy, const int64_t lddy, const T* __restrict__ z,
                                                        const int64_t ldz, T* __restrict__ dz, const int64_t lddz,
                                                        float* __restrict__ sums, const int64_t rows, const int64_t cols, const int act,
                                                        const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[16][DZ_PIECES * VEC];
  const int64_t across = (cols + DZ_PIECES * VEC - 1) / (DZ_PIECES * VEC);
  const int t = threadIdx.x / DZ_PIECES, c = threadIdx.x % DZ_PIECES * VEC;
  const int64_t id = first + blockIdx.x, strip = id / across, col0 = id % across * (DZ_PIECES * VEC), col = col0 + c, row = strip * (16 * EACH) + t;
  const bool whole = col + VEC <= cols;
  auto get = [&](const T* const p, const int64_t ld, const int64_t i) {
    piece_t x = {};
    if (i >= rows) return x;
    if (whole) __builtin_memcpy(&x, p + i * ld + col, 16);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (col + e < cols) x[e] = p[i * ld + col + e];
    return x;
  };
  piece_t y[EACH], a[EACH];
#pragma unroll
  for (int r = 0; r < EACH; ++r) y[r] = get(dy, lddy, row + 16 * r);
  if (act != MDET_ACT_NONE)
#pragma unroll
    for (int r = 0; r < EACH; ++r) a[r] = get(z, ldz, row + 16 * r);
  float sum[VEC] = {};
  act_switch(act, [&](auto which) {
    constexpr int ACT = decltype(which)::value;
#pragma unroll
    for (int r = 0; r < EACH; ++r) {
      piece_t d;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float v = (float)y[r][e];
        if constexpr (ACT != MDET_ACT_NONE) v *= act_slope<T, ACT>((float)a[r][e]);
        if (row + 16 * r < rows) sum[e] += v;
        d[e] = (T)v;
      }
      T* const to = dz + (row + 16 * r) * lddz + col;
      if (dz && row + 16 * r < rows) {
        if (whole) __builtin_memcpy(to, &d, 16);
        else
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (col + e < cols) to[e] = d[e];
      }
    }
  });
  if (!sums) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[t][c + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < DZ_PIECES * VEC && col0 + threadIdx.x < cols) {
    float v = part[0][threadIdx.x];
#pragma unroll
    for (int r = 1; r < 16; ++r) v += part[r][threadIdx.x];
    sums[strip * cols + col0 + threadIdx.x] = v;
  }
}

// db = sum of the strips' sums, sixteen threads a column, in one order.
constexpr int DB_COLS = 16;

template <typename O>
__global__ __launch_bounds__(256) void linear_db_kernel(const float* __restrict__ sums, const int64_t strips, const int64_t cols, O* __restrict__ db,
                                                        const int64_t first) {
  __shared__ float part[16][DB_COLS];
  const int t = threadIdx.x / DB_COLS, c = threadIdx.x % DB_COLS;
  const int64_t col = (first + blockIdx.x) * DB_COLS + c;
  float sum = 0.0f;
  if (col < cols)
    for (int64_t s = t; s < strips; s += 16) sum += sums[s * cols + col];
  part[t][c] = sum;
  __syncthreads();
  if (t == 0 && col < cols) {
    float v = part[0][c];
#pragma unroll
    for (int r = 1; r < 16; ++r) v += part[r][c];
    db[col] = (O)v;
  }
}

}  // namespace mdet
