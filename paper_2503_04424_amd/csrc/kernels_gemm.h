// Matrix products D[i][j] = sum_k R[i][k] C[j][k] on the matrix cores, for the linear layer, its gradient and the
// Gram matrix of a network's Jacobian.  R is the row operand (its index runs along the rows of D), C the column operand.
//
// Pieces.  Every operand is handled in pieces of 16 bytes along k: 8 elements in 16 bits, 4 in fp32, 2 in fp64.  A slab
// is eight pieces (128 bytes) of k.  Lane l of a wavefront supplies piece l / 16 of row l % 16 to a product, which takes
// the four pieces of one half slab at once: one instruction of 16 x 16 x 32 in 16 bits, four of 16 x 16 x 4 in fp32, two
// in fp64 (the e-th elements of the four pieces form the e-th of them; any assignment of k's is valid as long as R and C
// use the same one).  Sums are fp32 for operands in 16 and 32 bits, fp64 for fp64.
//
// The column operand goes in as the instruction's first, so that a lane's four results are neighbours in a row of D
// (fp64: four columns apart) and leave in one store.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mdet {

constexpr int GEMM_PIECES = 8;        // pieces of a slab

template <typename T> struct Core;

template <> struct Core<__bf16> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef __bf16 piece_t __attribute__((ext_vector_type(8)));
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, r, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<_Float16> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef _Float16 piece_t __attribute__((ext_vector_type(8)));
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, r, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<float> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef float piece_t __attribute__((ext_vector_type(4)));
  static constexpr int VEC = 4;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[e], r[e], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<double> {
  typedef double acc1_t;
  typedef double acc_t __attribute__((ext_vector_type(4)));
  typedef double piece_t __attribute__((ext_vector_type(2)));
  static constexpr int VEC = 2;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
#pragma unroll
    for (int e = 0; e < 2; ++e) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(c[e], r[e], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * e + (lane >> 4); }
};

// Element (i, k) stands at p[i * stride + k], or, with k outer, at p[k * stride + i].
template <typename T>
struct Operand {
  const T* p;
  int64_t stride;
  int64_t rows;                        // i < rows
};

// ---------------------------------------------------------------------------
// The plain tile: 64 x 64 of D by four wavefronts (32 x 32 each), any strides and alignment, every element guarded.
// ---------------------------------------------------------------------------
constexpr int PLAIN_TILE = 64;
constexpr int PLAIN_THREADS = 256;

template <typename T>
struct PlainLds {
  typename Core<T>::piece_t r[PLAIN_TILE][GEMM_PIECES + 1], c[PLAIN_TILE][GEMM_PIECES + 1];
};

// One slab of one operand, rows i0 .. i0 + 63, into LDS; what lies outside of the operand is zero.
template <typename T, bool OUTER>
__device__ __forceinline__ void plain_stage(typename Core<T>::piece_t (&to)[PLAIN_TILE][GEMM_PIECES + 1], const Operand<T>& o,
                                            const int64_t i0, const int64_t k0, const int64_t kend) {
  constexpr int VEC = Core<T>::VEC;
#pragma unroll
  for (int s = 0; s < PLAIN_TILE * GEMM_PIECES / PLAIN_THREADS; ++s) {
    const int id = s * PLAIN_THREADS + (int)threadIdx.x;
    // neighbouring threads read neighbouring memory
    const int row = OUTER ? id % PLAIN_TILE : id / GEMM_PIECES, piece = OUTER ? id / PLAIN_TILE : id % GEMM_PIECES;
    const int64_t i = i0 + row, k = k0 + piece * VEC;
    typename Core<T>::piece_t v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      T x = T(0);
      if (i < o.rows && k + e < kend) x = OUTER ? o.p[(k + e) * o.stride + i] : o.p[i * o.stride + k + e];
      v[e] = x;
    }
    to[row][piece] = v;
  }
}

// acc[a][b] += columns 16 a .. + 15 times rows 16 b .. + 15 of this wavefront's part of the tile, over k0 .. kend - 1.
template <typename T, bool ROUTER, bool COUTER>
__device__ __forceinline__ void plain_accumulate(typename Core<T>::acc_t (&acc)[2][2], PlainLds<T>& lds, const Operand<T>& r,
                                                 const Operand<T>& c, const int64_t row0, const int64_t col0, const int64_t k0,
                                                 const int64_t kend) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rw = (wave >> 1) * 32 + (lane & 15), cw = (wave & 1) * 32 + (lane & 15);
  for (int64_t k = k0; k < kend; k += GEMM_PIECES * Core<T>::VEC) {
    __syncthreads();
    plain_stage<T, ROUTER>(lds.r, r, row0, k, kend);
    plain_stage<T, COUTER>(lds.c, c, col0, k, kend);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int piece = 4 * h + (lane >> 4);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) Core<T>::mma(lds.c[cw + 16 * a][piece], lds.r[rw + 16 * b][piece], acc[a][b]);
    }
  }
}

// What a lane holds of a 16 x 16 part: element e of acc[a][b] belongs to row `lane & 15` and column Core::col(lane, e).
template <typename T, typename F>
__device__ __forceinline__ void plain_each(F&& f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f(a, b, e, (wave >> 1) * 32 + 16 * b + (lane & 15), (wave & 1) * 32 + 16 * a + Core<T>::col(lane, e));
}

}  // namespace mdet
