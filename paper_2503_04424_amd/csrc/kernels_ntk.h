// Gram matrix K = J J^T of a network's Jacobian (the NTK, Sec. 2.1), without J.
//
// A dense layer z = W a + b contributes to the derivative of output r at sample i the outer product of g = df_r / dz with
// a, and g itself for b.  The inner product of two such is (a . a' + 1) (g . g'), so with the layers' inputs a_l (n x p_l)
// and gradients g_l (n d x q_l, row i d + r: sample i, output r)
//
//   K[(i, r), (j, s)] = scale sum_l (a_l,i . a_l,j + bias) (g_l,ir . g_l,js)
//
// J would have sum_l (p_l + 1) q_l columns; here a layer takes n^2 p_l + (n d)^2 q_l operations for the lower triangle,
// which is all that the log-determinant reads and all that is written.  The arithmetic is K's type: fp32 (operands in 16
// or 32 bits) or fp64.
#pragma once
#include "kernels_gemm.h"

namespace mdet {

constexpr int NTK_LAYERS = 32;         // a launch's, so that they fit the kernel's arguments

template <typename T>
struct NtkLayers {
  int count;
  int64_t p[NTK_LAYERS], q[NTK_LAYERS];
  const T* a[NTK_LAYERS];
  const T* g[NTK_LAYERS];
  int64_t lda[NTK_LAYERS], ldg[NTK_LAYERS];
};

// Element i of a matrix in type S, as a double; the conversions to fp64 are exact.
template <typename S>
__global__ __launch_bounds__(256) void ntk_widen_kernel(const S* __restrict__ from, const int64_t ld, double* __restrict__ to, const int64_t rows,
                                                        const int64_t cols, const int64_t ldto) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = id / ldto, k = id % ldto;
  if (i < rows) to[i * ldto + k] = k < cols ? (double)from[i * ld + k] : 0.0;
}

// Block number t of the lower triangle of `rows` blocks: bands of eight rows of blocks, each column by column, so that
// neighbours read the same operands; band r has 64 (r + 1) numbers.  False: above the diagonal or behind the end.
__host__ __device__ __forceinline__ int64_t ntk_numbers(const int64_t rows) {
  const int64_t bands = (rows + 7) / 8;
  return 32 * bands * (bands + 1);
}
__device__ __forceinline__ bool ntk_block(const int64_t t, const int64_t rows, int64_t& bi, int64_t& bj) {
  int64_t r = (int64_t)((sqrt(1.0 + 0.125 * (double)t) - 1.0) * 0.5);
  while (32 * r * (r + 1) > t) --r;
  while (32 * (r + 1) * (r + 2) <= t) ++r;
  const int64_t u = t - 32 * r * (r + 1);
  bi = 8 * r + (u & 7);
  bj = u >> 3;
  return bi < rows && bj <= bi;
}

// first[l] = a_l a_l^T + bias, lower triangle of n x n, for networks of several outputs: every pair of samples' product
// serves outputs^2 elements of K.
template <typename T, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void ntk_first_kernel(const NtkLayers<T> layers, const int64_t n, const typename Core<T>::acc1_t bias,
                                                               typename Core<T>::acc1_t* __restrict__ first) {
  __shared__ __attribute__((aligned(16))) char lds[2 * S::SLAB];
  const int64_t rows = (n + S::BM - 1) / S::BM, numbers = ntk_numbers(rows);
  const int64_t t = gemm_tile_number(blockIdx.x, numbers * layers.count);
  int64_t bi, bj;
  if (t < 0 || !ntk_block(t % numbers, rows, bi, bj)) return;
  const int l = (int)(t / numbers);
  const Operand<T> a{layers.a[l], layers.lda[l], n};
  typename Core<T>::acc_t acc[S::TN][S::TM] = {};
  tile_accumulate<T, S, false, false, DIRECT>(acc, lds, a, a, bi * S::BM, bj * S::BN, 0, layers.p[l]);
  typename Core<T>::acc1_t* const to = first + l * n * n;
  tile_each<T, S>([&](int a0, int b0, int e, int i, int j) {
    const int64_t I = bi * S::BM + i, J = bj * S::BN + j;
    if (I < n && J <= I) to[I * n + J] = acc[a0][b0][e] + bias;
  });
}

// A block of K.  FIRST: the first factors stand in `first`; otherwise (one output) both products are formed here, one
// after the other, and multiplied in registers.  The sum over layers stays in registers, K is written once.
template <typename T, typename S, bool DIRECT, bool FIRST>
__global__ __launch_bounds__(S::THREADS) void ntk_gram_kernel(const NtkLayers<T> layers, const int64_t n, const int d,
                                                              const typename Core<T>::acc1_t bias, const typename Core<T>::acc1_t scale,
                                                              const int accumulate, const typename Core<T>::acc1_t* __restrict__ first,
                                                              typename Core<T>::acc1_t* __restrict__ K, const int64_t ldk) {
  typedef typename Core<T>::acc_t acc_t;
  __shared__ __attribute__((aligned(16))) char lds[2 * S::SLAB];
  const int64_t N = n * d, rows = (N + S::BM - 1) / S::BM;
  const int64_t t = gemm_tile_number(blockIdx.x, ntk_numbers(rows));
  int64_t bi, bj;
  if (t < 0 || !ntk_block(t, rows, bi, bj)) return;
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  acc_t total[S::TN][S::TM] = {};
  for (int l = 0; l < layers.count; ++l) {
    acc_t second[S::TN][S::TM] = {};
    const Operand<T> g{layers.g[l], layers.ldg[l], N};
    __syncthreads();                               // the product before reads its last slab
    tile_accumulate<T, S, false, false, DIRECT>(second, lds, g, g, row0, col0, 0, layers.q[l]);
    if constexpr (FIRST) {
      const typename Core<T>::acc1_t* const from = first + l * n * n;
      tile_each<T, S>([&](int a, int b, int e, int i, int j) {
        int64_t I = row0 + i, J = col0 + j;
        if (I < N && J <= I) total[a][b][e] += from[I / d * n + J / d] * second[a][b][e];
      });
    } else {
      const Operand<T> x{layers.a[l], layers.lda[l], N};
      acc_t one[S::TN][S::TM] = {};
      __syncthreads();
      tile_accumulate<T, S, false, false, DIRECT>(one, lds, x, x, row0, col0, 0, layers.p[l]);
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int b = 0; b < S::TM; ++b) total[a][b] += (one[a][b] + bias) * second[a][b];
    }
  }
  tile_each<T, S>([&](int a, int b, int e, int i, int j) {
    const int64_t I = row0 + i, J = col0 + j;
    if (I >= N || J > I) return;
    auto v = total[a][b][e] * scale;
    if (accumulate) v += K[I * ldk + J];
    K[I * ldk + J] = v;
  });
}

}  // namespace mdet
