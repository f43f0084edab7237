// C ABI of the linear layer and its gradient: argument checks, workspace layout and kernel launches.  A call only queues
// work on the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels_linear.h"

namespace {

using namespace mdet;

inline uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t size_of(int32_t t) { return t == MDET_F32 ? 4 : 2; }
inline bool is_type(int32_t t) { return t == MDET_F32 || t == MDET_F16 || t == MDET_BF16; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? MDET_OK : MDET_EHIP; }

// Sizes whose products and byte counts stay within 64 bits.
constexpr int64_t MOST = int64_t(1) << 40;
inline bool sizes_fit(int64_t m, int64_t n, int64_t k) {
  if (m < 0 || n < 0 || k < 0 || m > MOST || n > MOST || k > MOST) return false;
  const int64_t most = int64_t(1) << 52;
  return (!n || m <= most / n) && (!k || m <= most / k) && (!k || n <= most / k);
}

// A matrix of r rows and c columns in memory: null only where it has no elements, rows that do not overlap.
inline bool matrix_ok(const void* p, int64_t r, int64_t c, int64_t ld, int64_t size) {
  if (r == 0 || c == 0) return true;
  return p && (uintptr_t)p % size == 0 && (r == 1 || ld >= c) && ld >= 0 && ld <= MOST;
}

template <typename T, typename O, bool ROUTER, bool COUTER>
int product(const Operand<T>& r, const Operand<T>& c, int64_t k, const LinearOut<T, O>& out, hipStream_t st) {
  const int64_t tiles = ceil_div(out.rows, PLAIN_TILE) * ceil_div(out.cols, PLAIN_TILE);
  if (tiles > INT32_MAX) return MDET_EINVAL;
  hipLaunchKernelGGL((linear_plain_kernel<T, O, ROUTER, COUTER>), dim3((unsigned)tiles), dim3(PLAIN_THREADS), 0, st, r, c, k, out);
  return launch_status();
}

// Workspace of the gradient: dz, then the strips' column sums.
struct GradLayout {
  int64_t strips, lddz;
  uint64_t sums, bytes;
};
GradLayout grad_layout(int32_t dtype, int64_t m, int64_t n) {
  GradLayout g;
  g.strips = ceil_div(m, DZ_ROWS);
  g.lddz = ceil_div(n, 8) * 8;
  g.sums = up256((uint64_t)m * g.lddz * size_of(dtype));
  g.bytes = g.sums + up256((uint64_t)g.strips * n * 4);
  return g;
}

struct Grad {
  int32_t act;
  int64_t m, n, k;
  const void *dy, *z, *x, *w;
  int64_t lddy, ldz, ldx, ldw;
  void *dx, *dw, *db, *dz;
  int64_t lddx, lddw, lddz;
  char* workspace;
  hipStream_t st;
};

template <typename T, typename O>
int backward(const Grad& g) {
  const GradLayout lay = grad_layout(std::is_same<T, float>::value ? MDET_F32 : MDET_F16, g.m, g.n);
  const bool own_dz = g.dz || (g.act != MDET_ACT_NONE && (g.dx || g.dw));
  T* const dz = g.dz ? (T*)g.dz : own_dz ? (T*)g.workspace : nullptr;
  const int64_t lddz = g.dz ? g.lddz : lay.lddz;
  float* const sums = g.db ? (float*)(g.workspace + lay.sums) : nullptr;
  if ((dz || sums) && g.m > 0 && g.n > 0) {
    const int64_t blocks = lay.strips * ceil_div(g.n, DZ_COLS);
    if (blocks > INT32_MAX) return MDET_EINVAL;
    hipLaunchKernelGGL((linear_dz_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, g.st, (const T*)g.dy, g.lddy, (const T*)g.z, g.ldz,
                       dz, lddz, sums, g.m, g.n, g.act);
  }
  if (g.db && g.n > 0)
    hipLaunchKernelGGL((linear_db_kernel<O>), dim3((unsigned)ceil_div(g.n, 64)), dim3(256), 0, g.st, (const float*)sums, lay.strips, g.n,
                       (O*)g.db);
  int status = launch_status();
  const T* const d = own_dz ? dz : (const T*)g.dy;
  const int64_t ldd = own_dz ? lddz : g.lddy;
  if (status == MDET_OK && g.dx && g.m > 0 && g.k > 0) {
    const LinearOut<T, T> out{(T*)g.dx, g.lddx, nullptr, nullptr, 0, nullptr, 0, MDET_ACT_NONE, g.m, g.k};
    status = product<T, T, false, true>(Operand<T>{d, ldd, g.m}, Operand<T>{(const T*)g.w, g.ldw, g.k}, g.n, out, g.st);
  }
  if (status == MDET_OK && g.dw && g.n > 0 && g.k > 0) {
    const LinearOut<T, O> out{(O*)g.dw, g.lddw, nullptr, nullptr, 0, nullptr, 0, MDET_ACT_NONE, g.n, g.k};
    status = product<T, O, true, true>(Operand<T>{d, ldd, g.n}, Operand<T>{(const T*)g.x, g.ldx, g.k}, g.m, out, g.st);
  }
  return status;
}

}  // namespace

extern "C" {

int mdet_linear_workspace_query(int32_t dtype, int32_t backward, int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  if (!bytes || !is_type(dtype) || !sizes_fit(m, n, k)) return MDET_EINVAL;
  *bytes = backward ? grad_layout(dtype, m, n).bytes : 0;
  return MDET_OK;
}

int mdet_linear_forward(int32_t dtype, int32_t activation, int64_t m, int64_t n, int64_t k, const void* x, int64_t ldx, const void* w,
                        int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, int64_t ldz,
                        void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || activation < MDET_ACT_NONE || activation > MDET_ACT_SILU || !sizes_fit(m, n, k)) return MDET_EINVAL;
  const int64_t s = size_of(dtype);
  if (!matrix_ok(x, m, k, ldx, s) || !matrix_ok(w, n, k, ldw, s) || !matrix_ok(y, m, n, ldy, s)) return MDET_EINVAL;
  if ((residual && !matrix_ok(residual, m, n, ldr, s)) || (z && !matrix_ok(z, m, n, ldz, s)) || (uintptr_t)bias % s) return MDET_EINVAL;
  uint64_t need = 0;
  mdet_linear_workspace_query(dtype, 0, m, n, k, &need);
  if (need && !workspace) return MDET_EINVAL;
  if (workspace_bytes < need) return MDET_ENOMEM_DEVICE;
  if (m == 0 || n == 0) return MDET_OK;
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    const LinearOut<T, T> out{(T*)y, ldy, (const T*)bias, (const T*)residual, ldr, (T*)z, ldz, activation, m, n};
    return product<T, T, false, false>(Operand<T>{(const T*)x, ldx, m}, Operand<T>{(const T*)w, ldw, n}, k, out, (hipStream_t)stream);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

int mdet_linear_backward(int32_t dtype, int32_t grad_dtype, int32_t activation, int64_t m, int64_t n, int64_t k, const void* dy,
                         int64_t lddy, const void* z, int64_t ldz, const void* x, int64_t ldx, const void* w, int64_t ldw, void* dx,
                         int64_t lddx, void* dw, int64_t lddw, void* db, void* dz, int64_t lddz, void* workspace,
                         uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || (grad_dtype != dtype && grad_dtype != MDET_F32)) return MDET_EINVAL;
  if (activation < MDET_ACT_NONE || activation > MDET_ACT_SILU || !sizes_fit(m, n, k)) return MDET_EINVAL;
  const int64_t s = size_of(dtype), gs = size_of(grad_dtype);
  if (!matrix_ok(dy, m, n, lddy, s) || (activation != MDET_ACT_NONE && !matrix_ok(z, m, n, ldz, s))) return MDET_EINVAL;
  if (dx && (!matrix_ok(dx, m, k, lddx, s) || !matrix_ok(w, n, k, ldw, s))) return MDET_EINVAL;
  if (dw && (!matrix_ok(dw, n, k, lddw, gs) || !matrix_ok(x, m, k, ldx, s))) return MDET_EINVAL;
  if ((uintptr_t)db % gs || (dz && !matrix_ok(dz, m, n, lddz, s))) return MDET_EINVAL;
  uint64_t need = 0;
  mdet_linear_workspace_query(dtype, 1, m, n, k, &need);
  if (need && (!workspace || (uintptr_t)workspace % 256)) return MDET_EINVAL;
  if (workspace_bytes < need) return MDET_ENOMEM_DEVICE;
  const Grad g{activation, m, n, k, dy, z, x, w, lddy, ldz, ldx, ldw, dx, dw, db, dz, lddx, lddw, lddz, (char*)workspace, (hipStream_t)stream};
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    return grad_dtype == MDET_F32 ? backward<T, float>(g) : backward<T, T>(g);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

}  // extern "C"
