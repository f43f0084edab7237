// C ABI of the layer norm and its gradient: argument checks, workspace layout and kernel launches.  A call only queues work on
// the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "kernels_norm.h"
#include "linear_cut.h"
#include "operands.h"

namespace {

using namespace mdet;

// f(threads of a workgroup, lanes of a row, pieces of a lane): lanes that hold a row in registers; false: none do.  The gradient, which also
// holds two sums for each column, has fewer pieces a lane (rows of 4096 in bf16: two pieces in 256 lanes leave room for three wavefronts, one
// in 512 for five), and in 1024 lanes no room for two pieces of 16-bit elements.
template <bool GRADIENT, int SIZE, typename F>
bool norm_shape(int64_t cols, F&& f) {
  using std::integral_constant;
  const int64_t pieces = ceil_div(cols * SIZE, 16);
  typedef integral_constant<int, 1> one;
  typedef integral_constant<int, 2> two;
  typedef integral_constant<int, 4> four;
  typedef integral_constant<int, 256> small;
  typedef integral_constant<int, 512> medium;
  typedef integral_constant<int, 1024> large;
  if (pieces <= 16) f(small{}, integral_constant<int, 16>{}, one{});
  else if (pieces <= 64) f(small{}, integral_constant<int, 64>{}, one{});
  else if (pieces <= 128) f(small{}, integral_constant<int, 64>{}, two{});
  else if (pieces <= 256) f(small{}, small{}, one{});
  else if (pieces <= 512) {
    if constexpr (GRADIENT) f(medium{}, medium{}, one{});
    else f(small{}, small{}, two{});
  } else if (pieces <= 1024) {
    if constexpr (GRADIENT) f(large{}, large{}, one{});
    else f(small{}, small{}, four{});
  } else if (pieces <= 2048 && (!GRADIENT || SIZE == 4)) {
    if constexpr (!GRADIENT || SIZE == 4) f(large{}, large{}, two{});
  } else if (pieces <= 4096 && !GRADIENT) {
    if constexpr (!GRADIENT) f(large{}, large{}, four{});
  } else return false;
  return true;
}

// Strips of rows whose sums for dw and db stand in the workspace: as many as workgroups that fill the device.
int64_t norm_strips(int64_t rows, int64_t cols, int64_t size) {
  int64_t strips = 0;
  auto held_by = [&](auto threads, auto lanes, auto) {
    const int64_t groups = threads / lanes;
    const int64_t turns = ceil_div(rows, groups), most = 262144 / threads;
    // a few rows each before there are more than compute units: 777 x 1301 in fp32, a strip a row: 30 us, of which 17 for adding the strips up
    strips = turns <= 256 ? turns : turns <= 1024 ? 256 : turns / 4 < most ? turns / 4 : most;
  };
  if (!(size == 4 ? norm_shape<true, 4>(cols, held_by) : norm_shape<true, 2>(cols, held_by))) {
    strips = 1024 / ceil_div(cols * size, 16 * NORM_THREADS);
    if (strips < 1) strips = 1;
    if (strips > rows) strips = rows;
  }
  return strips;
}

template <typename T>
int forward(const NormForward<T>& a, hipStream_t st) {
  const bool held = norm_shape<false, sizeof(T)>(a.cols, [&](auto threads, auto lanes, auto pieces) {
    constexpr int THREADS = decltype(threads)::value, LANES = decltype(lanes)::value;
    gemm_launches(ceil_div(a.rows, THREADS / LANES), THREADS, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((norm_forward_kernel<T, THREADS, LANES, decltype(pieces)::value>), grid, dim3(THREADS), 0, st, a, first);
    });
  });
  if (!held)
    gemm_launches(a.rows, 1024, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((norm_forward_long_kernel<T>), grid, dim3(1024), 0, st, a, first);
    });
  return launch_status();
}

template <typename T, typename O>
int backward(const NormBackward<T>& a, O* dw, O* db, hipStream_t st) {
  const int64_t strips = norm_strips(a.rows, a.cols, sizeof(T));
  if (a.rows > 0 && (a.dx || a.sums)) {
    const bool held = norm_shape<true, sizeof(T)>(a.cols, [&](auto threads, auto lanes, auto pieces) {
      constexpr int THREADS = decltype(threads)::value, LANES = decltype(lanes)::value;
      hipLaunchKernelGGL((norm_backward_kernel<T, THREADS, LANES, decltype(pieces)::value>), dim3((unsigned)strips), dim3(THREADS), 0, st, a);
    });
    if (!held) {
      if (a.dx)
        gemm_launches(a.rows, 1024, [&](const int64_t first, const dim3 grid) {
          hipLaunchKernelGGL((norm_backward_long_kernel<T>), grid, dim3(1024), 0, st, a, first);
        });
      if (a.sums) {
        const int64_t across = ceil_div(a.cols, Core<T>::VEC * NORM_THREADS);
        hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((unsigned)(strips * across)), dim3(NORM_THREADS), 0, st, a, strips);
      }
    }
  }
  if (dw || db)                        // without rows as well: zeros
    gemm_launches(ceil_div(a.cols, NORM_COLS), NORM_COLS * NORM_JOIN, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((norm_join_kernel<O>), grid, dim3(NORM_COLS * NORM_JOIN), 0, st, (const float*)a.sums, strips, a.cols, dw, db, first);
    });
  return launch_status();
}

// Rows so long that the workgroups of one strip would be a launch of 2^32 threads are refused.
bool norm_fits(int64_t m, int64_t n) { return sizes_fit(m, n, 1) && n <= (int64_t(1) << 32); }

}  // namespace

extern "C" {

int mdet_layernorm_workspace_query(int32_t dtype, int64_t m, int64_t n, uint64_t* bytes) {
  if (!bytes || !is_type(dtype) || !norm_fits(m, n)) return MDET_EINVAL;
  *bytes = up256((uint64_t)norm_strips(m, n, size_of(dtype)) * 2 * n * 4);
  return MDET_OK;
}

int mdet_layernorm_forward(int32_t dtype, int64_t m, int64_t n, const void* x, int64_t ldx, const void* weight, const void* bias, double eps,
                           void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
  if (!is_type(dtype) || !norm_fits(m, n) || !(eps >= 0.0) || !std::isfinite((float)eps)) return MDET_EINVAL;
  const int64_t s = size_of(dtype);
  if (!matrix_ok(x, m, n, ldx, s) || !matrix_ok(y, m, n, ldy, s) || (uintptr_t)weight % s || (uintptr_t)bias % s) return MDET_EINVAL;
  if ((uintptr_t)mean % 4 || (uintptr_t)rstd % 4) return MDET_EINVAL;
  if (m == 0 || (n == 0 && !mean && !rstd)) return MDET_OK;
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    return forward(NormForward<T>{(const T*)x, ldx, (const T*)weight, (const T*)bias, (T*)y, ldy, mean, rstd, m, n, (float)eps,
                                  n ? (float)n : 1.0f}, (hipStream_t)stream);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

int mdet_layernorm_backward(int32_t dtype, int32_t grad_dtype, int64_t m, int64_t n, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                            const float* mean, const float* rstd, const void* weight, void* dx, int64_t lddx, void* dw, void* db,
                            void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || (grad_dtype != dtype && grad_dtype != MDET_F32) || !norm_fits(m, n)) return MDET_EINVAL;
  const int64_t s = size_of(dtype), gs = size_of(grad_dtype);
  if (!matrix_ok(dy, m, n, lddy, s) || !matrix_ok(x, m, n, ldx, s) || (dx && !matrix_ok(dx, m, n, lddx, s))) return MDET_EINVAL;
  if (!vector_ok(mean, n ? m : 0, 4) || !vector_ok(rstd, n ? m : 0, 4)) return MDET_EINVAL;
  if ((uintptr_t)weight % s || (uintptr_t)dw % gs || (uintptr_t)db % gs) return MDET_EINVAL;
  uint64_t need = 0;
  if (dw || db) mdet_layernorm_workspace_query(dtype, m, n, &need);
  const int ok = workspace_ok(workspace, workspace_bytes, need);
  if (ok != MDET_OK) return ok;
  if (n == 0 || (!dx && !dw && !db)) return MDET_OK;
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    const NormBackward<T> a{(const T*)dy, (const T*)x, (const T*)weight, lddy, ldx, mean, rstd, (T*)dx, lddx, dw || db ? (float*)workspace : nullptr,
                            m, n, (float)n};
    return grad_dtype == MDET_F32 ? backward<T, float>(a, (float*)dw, (float*)db, (hipStream_t)stream)
                                  : backward<T, T>(a, (T*)dw, (T*)db, (hipStream_t)stream);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

}  // extern "C"
