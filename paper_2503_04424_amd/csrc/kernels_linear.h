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
__device__ __forceinline__ float logistic(float t) { return 1.0f / (1.0f + __expf(-t)); }

template <int ACT>
__device__ __forceinline__ float act_value(const float z) {
  if constexpr (ACT == MDET_ACT_RELU) return z < 0.0f ? 0.0f : z;
  else if constexpr (ACT == MDET_ACT_GELU) {
    const float c = z < -20.0f ? -20.0f : z;         // the factor is zero there already
    return 0.5f * c * (1.0f + erff(c * ACT_R2));
  } else if constexpr (ACT == MDET_ACT_GELU_TANH) {
    const float c = z < -20.0f ? -20.0f : z;
    const float t = act_clamp(c, -20.0f, 20.0f);     // (1 + tanh(u)) / 2 = logistic(2 u)
    return c * logistic(2.0f * ACT_TANH_A * (t + ACT_TANH_B * t * t * t));
  } else if constexpr (ACT == MDET_ACT_SILU) {
    const float c = z < -80.0f ? -80.0f : z;
    return c * logistic(c);
  } else return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(const float z) {
  if constexpr (ACT == MDET_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
  else if constexpr (ACT == MDET_ACT_GELU) {
    const float c = act_clamp(z, -20.0f, 20.0f);
    return 0.5f * (1.0f + erff(c * ACT_R2)) + c * __expf(-0.5f * c * c) * ACT_R2PI;
  } else if constexpr (ACT == MDET_ACT_GELU_TANH) {
    const float c = act_clamp(z, -20.0f, 20.0f);
    const float q = logistic(2.0f * ACT_TANH_A * (c + ACT_TANH_B * c * c * c));
    return q + 2.0f * c * q * (1.0f - q) * ACT_TANH_A * (1.0f + 3.0f * ACT_TANH_B * c * c);
  } else if constexpr (ACT == MDET_ACT_SILU) {
    const float c = act_clamp(z, -80.0f, 80.0f);
    const float q = logistic(c);
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
};

template <typename T, typename O, int ACT>
__device__ __forceinline__ void linear_put(const LinearOut<T, O>& o, const int64_t i, const int64_t j, float v) {
  if (o.bias) v += (float)o.bias[j];
  if (o.z) o.z[i * o.ldz + j] = (T)v;
  v = act_value<ACT>(v);
  if (o.residual) v += (float)o.residual[i * o.ldr + j];
  o.y[i * o.ldy + j] = (O)v;
}

template <typename T, typename O, bool ROUTER, bool COUTER>
__global__ __launch_bounds__(PLAIN_THREADS) void linear_plain_kernel(const Operand<T> r, const Operand<T> c, const int64_t k,
                                                                     const LinearOut<T, O> out) {
  __shared__ PlainLds<T> lds;
  const int64_t across = (out.cols + PLAIN_TILE - 1) / PLAIN_TILE;
  const int64_t row0 = blockIdx.x / across * PLAIN_TILE, col0 = blockIdx.x % across * PLAIN_TILE;
  typename Core<T>::acc_t acc[2][2] = {};
  plain_accumulate<T, ROUTER, COUTER>(acc, lds, r, c, row0, col0, 0, k);
  act_switch(out.act, [&](auto act) {
    plain_each<T>([&](int a, int b, int e, int i, int j) {
      if (row0 + i < out.rows && col0 + j < out.cols) linear_put<T, O, decltype(act)::value>(out, row0 + i, col0 + j, acc[a][b][e]);
    });
  });
}

// dz = dy act'(z) and the column sums of DZ_ROWS rows of it: a workgroup takes 64 columns, thread (t, c) every fourth row of
// column c.
constexpr int DZ_COLS = 64, DZ_ROWS = 64;

template <typename T>
__global__ __launch_bounds__(256) void linear_dz_kernel(const T* __restrict__ dy, const int64_t lddy, const T* __restrict__ z,
                                                        const int64_t ldz, T* __restrict__ dz, const int64_t lddz,
                                                        float* __restrict__ sums, const int64_t rows, const int64_t cols, const int act) {
  __shared__ float part[4][DZ_COLS];
  const int64_t across = (cols + DZ_COLS - 1) / DZ_COLS;
  const int64_t strip = blockIdx.x / across, col = blockIdx.x % across * DZ_COLS + (threadIdx.x & 63);
  const int t = threadIdx.x >> 6;
  float sum = 0.0f;
  if (col < cols) {
    act_switch(act, [&](auto a) {
      for (int64_t i = strip * DZ_ROWS + t; i < rows && i < (strip + 1) * DZ_ROWS; i += 4) {
        float v = (float)dy[i * lddy + col];
        if constexpr (decltype(a)::value != MDET_ACT_NONE) v *= act_slope<decltype(a)::value>((float)z[i * ldz + col]);
        if (dz) dz[i * lddz + col] = (T)v;
        sum += v;
      }
    });
  }
  part[t][threadIdx.x & 63] = sum;
  __syncthreads();
  if (sums && t == 0 && col < cols)
    sums[strip * cols + col] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

// db = sum of the strips' sums, four threads a column, in one order.
template <typename O>
__global__ __launch_bounds__(256) void linear_db_kernel(const float* __restrict__ sums, const int64_t strips, const int64_t cols, O* __restrict__ db) {
  __shared__ float part[4][64];
  const int64_t col = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int t = threadIdx.x >> 6;
  float sum = 0.0f;
  if (col < cols)
    for (int64_t s = t; s < strips; s += 4) sum += sums[s * cols + col];
  part[t][threadIdx.x & 63] = sum;
  __syncthreads();
  if (t == 0 && col < cols) db[col] = (O)((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

}  // namespace mdet
