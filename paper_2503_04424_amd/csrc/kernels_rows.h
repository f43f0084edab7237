// Rows of a matrix in pieces of 16 bytes, at any alignment of their elements.
#pragma once
#include "kernels_gemm.h"

namespace mdet {

// 16 bytes of a row from column c on; what lies behind its end is zero.
template <typename T>
__device__ __forceinline__ typename Core<T>::piece_t row_piece(const T* const row, const int64_t c, const int64_t cols) {
  typename Core<T>::piece_t x = {};
  if (c + Core<T>::VEC <= cols) __builtin_memcpy(&x, row + c, 16);
  else
#pragma unroll
    for (int e = 0; e < Core<T>::VEC - 1; ++e)
      if (c + e < cols) x[e] = row[c + e];
  return x;
}

// Likewise, but what lies behind the row's end is an element of it.
template <typename T>
__device__ __forceinline__ typename Core<T>::piece_t row_piece_filled(const T* const row, const int64_t c, const int64_t cols) {
  typename Core<T>::piece_t x;
  if (c + Core<T>::VEC <= cols) __builtin_memcpy(&x, row + c, 16);
  else {
    const T fill = row[c < cols ? c : cols - 1];
#pragma unroll
    for (int e = 0; e < Core<T>::VEC; ++e) x[e] = fill;
#pragma unroll
    for (int e = 1; e < Core<T>::VEC - 1; ++e)
      if (c + e < cols) x[e] = row[c + e];
  }
  return x;
}

// VEC values of a row from column c on, rounded.
template <typename T, typename O>
__device__ __forceinline__ void row_store(O* const row, const int64_t c, const int64_t cols, const float (&v)[Core<T>::VEC]) {
  constexpr int VEC = Core<T>::VEC;
  typedef O out_t __attribute__((ext_vector_type(VEC)));
  if (c + VEC <= cols) {
    out_t x;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = (O)v[e];
    __builtin_memcpy(row + c, &x, sizeof(x));
  } else
#pragma unroll
    for (int e = 0; e < VEC - 1; ++e)
      if (c + e < cols) row[c + e] = (O)v[e];
}

}  // namespace mdet
