// C ABI of the linear layer and its gradient: argument checks, workspace layout and kernel launches.  A call only queues
// work on the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels_linear.h"
#include "linear_cut.h"
#include "operands.h"

namespace {

using namespace mdet;

// Whether a product of this many rows and columns goes out in one launch, which holds fewer than 2^32 threads.  A tile of 256 (128) rows and
// columns has 512 (256) threads for at least eight (four) squares of 32, the grid is rounded up by seven tiles at most, and smaller
// tiles are taken for a few hundred squares only.
inline bool tiles_fit(int64_t rows, int64_t cols) { return ceil_div(rows, 32) * ceil_div(cols, 32) <= (int64_t(1) << 26) - 1024; }

// Whether four elements at a time can be moved at this place.
template <typename T>
bool four(const void* p, int64_t ld, int64_t rows) {
  return !p || ((uintptr_t)p % (4 * sizeof(T)) == 0 && (rows == 1 || ld % 4 == 0));
}

template <typename T, typename O>
bool fours(const LinearOut<T, O>& out) {
  return four<O>(out.y, out.ldy, out.rows) && four<T>(out.bias, 0, 1) && four<T>(out.residual, out.ldr, out.rows) &&
         four<T>(out.z, out.ldz, out.rows);
}

typedef Tile<256, 256, 2, 4, 2> Big;
typedef Tile<128, 128, 2, 2, 2> Mid;
typedef Tile<64, 64, 2, 2, 2> Small;
typedef Tile<64, 64, 2, 2, 4> Ahead;
typedef Tile<32, 32, 2, 2, 4> Tiny;

template <typename T, typename O>
void rows_product(const Operand<T>& r, const Operand<T>& c, int64_t k, const LinearOut<T, O>& out, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(out.cols, 16));
  if (k * (int64_t)sizeof(T) >= 4096) hipLaunchKernelGGL((linear_rows_kernel<T, O, 16>), grid, dim3(1024), 0, st, r, c, k, out);
  else hipLaunchKernelGGL((linear_rows_kernel<T, O, 4>), grid, dim3(256), 0, st, r, c, k, out);
}

uint64_t parts_bytes(const Cut& c, int64_t rows, int64_t cols) { return c.splits > 1 ? up256((uint64_t)c.splits * rows * cols * 4) : 0; }

template <typename T, typename O, typename S, bool ROUTER, bool COUTER>
void tiles(Operand<T> r, Operand<T> c, int64_t k, const LinearOut<T, O>& out, const Cut& cut, float* parts, hipStream_t st) {
  const int64_t n = ceil_div(out.rows, S::BM) * ceil_div(out.cols, S::BN) * cut.splits;
  const dim3 grid((unsigned)(ceil_div(n, 8) * 8));
  r = gemm_operand<T, ROUTER, S::BM>(r.p, r.stride, r.rows, k);
  c = gemm_operand<T, COUTER, S::BN>(c.p, c.stride, c.rows, k);
  const bool direct = r.straight && c.straight;
  auto go = [&](auto d, auto split) {
    hipLaunchKernelGGL((linear_tile_kernel<T, O, S, ROUTER, COUTER, decltype(d)::value, decltype(split)::value>), grid, dim3(S::THREADS), 0, st, r, c, k, out,
                       n, parts, cut.kpart);
  };
  using std::false_type;
  using std::true_type;
  // sums are split for the smallest tile alone (cut_of): the others are taken where there are enough of them
  if (cut.splits > 1) {
    if constexpr (std::is_same<S, Tiny>::value) {
      if (direct) go(true_type{}, true_type{});
      else go(false_type{}, true_type{});
      const int64_t groups = ceil_div(out.rows * ceil_div(out.cols, 4), 256);
      hipLaunchKernelGGL((linear_join_kernel<T, O>), dim3((unsigned)groups), dim3(256), 0, st, (const float*)parts, cut.splits, out);
    }
  } else if (direct) go(true_type{}, false_type{});
  else if constexpr (!std::is_same<S, Ahead>::value) go(false_type{}, false_type{});
}

template <typename T, typename O, bool ROUTER, bool COUTER>
int product(Operand<T> r, Operand<T> c, int64_t k, LinearOut<T, O> out, float* parts, hipStream_t st) {
  const Cut cut = cut_of(out.rows, out.cols, k, sizeof(T), !ROUTER && !COUTER);
  out.vec = fours(out);
  if (cut.tile == 0) {
    if constexpr (!ROUTER && !COUTER) rows_product<T, O>(r, c, k, out, st);
  } else if (cut.tile == 256) {
    if constexpr (sizeof(T) == 2) tiles<T, O, Big, ROUTER, COUTER>(r, c, k, out, cut, parts, st);
  } else if (cut.tile == 128) tiles<T, O, Mid, ROUTER, COUTER>(r, c, k, out, cut, parts, st);
  else if (cut.tile == 64) {
    // three slabs on their way in 16 bits, where they last shortest, as long as all of the workgroups have room for them
    // at once (512 x 4096 x 4096 33 us with one, 28.5 with three)
    const int64_t n = ceil_div(out.rows, 64) * ceil_div(out.cols, 64);
    const bool straight = gemm_operand<T, ROUTER, 64>(r.p, r.stride, r.rows, k).straight && gemm_operand<T, COUTER, 64>(c.p, c.stride, c.rows, k).straight;
    if (sizeof(T) == 2 && n <= 512 && straight) {
      if constexpr (sizeof(T) == 2) tiles<T, O, Ahead, ROUTER, COUTER>(r, c, k, out, cut, parts, st);
    } else tiles<T, O, Small, ROUTER, COUTER>(r, c, k, out, cut, parts, st);
  }
  else tiles<T, O, Tiny, ROUTER, COUTER>(r, c, k, out, cut, parts, st);
  return launch_status();
}

// Both products of a gradient in one launch, in 16 bits, if both would be cut into small whole tiles: true if it is done.
// 256^3 bf16 with dz 12.7 -> 9.4 us, 1000^3 28.8 -> 26.2, 777 x 1301 x 515 35.4 -> 30.8.  In fp32 a product's tiles last long
// enough for their uneven numbers to count: 1000^3 69 -> 58 us, but 1500 x 700 x 900 69 -> 79 and more.
template <typename T, typename O>
bool pair(Operand<T> dzr, Operand<T> w, int64_t n, LinearOut<T, T> dx, Operand<T> dzc, Operand<T> x, int64_t m, LinearOut<T, O> dw, hipStream_t st) {
  const Cut a = cut_of(dx.rows, dx.cols, n, sizeof(T), false), b = cut_of(dw.rows, dw.cols, m, sizeof(T), false);
  if (a.tile > 64 || b.tile > 64 || a.splits > 1 || b.splits > 1) return false;
  auto tiles = [&](int64_t e) { return ceil_div(dx.rows, e) * ceil_div(dx.cols, e); };
  auto all = [&](int64_t e) { return tiles(e) + ceil_div(dw.rows, e) * ceil_div(dw.cols, e); };
  dx.vec = fours(dx);
  dw.vec = fours(dw);
  auto go = [&](auto shape) {
    typedef decltype(shape) S;
    dzr = gemm_operand<T, false, S::BM>(dzr.p, dzr.stride, dzr.rows, n);
    w = gemm_operand<T, true, S::BN>(w.p, w.stride, w.rows, n);
    dzc = gemm_operand<T, true, S::BM>(dzc.p, dzc.stride, dzc.rows, m);
    x = gemm_operand<T, true, S::BN>(x.p, x.stride, x.rows, m);
    const int64_t first = tiles(S::BM), count = all(S::BM);
    const dim3 grid((unsigned)(ceil_div(count, 8) * 8)), block(S::THREADS);
    if (dzr.straight && w.straight && dzc.straight && x.straight)
      hipLaunchKernelGGL((linear_pair_kernel<T, O, S, true>), grid, block, 0, st, dzr, w, n, dx, dzc, x, m, dw, first, count);
    else hipLaunchKernelGGL((linear_pair_kernel<T, O, S, false>), grid, block, 0, st, dzr, w, n, dx, dzc, x, m, dw, first, count);
  };
  if (all(64) >= 256) go(Small{});
  else go(Tiny{});
  return true;
}

// Workspace of the gradient: dz, then the strips' column sums, then the parts of a product that is split.
struct GradLayout {
  int64_t each, strips, lddz;
  uint64_t sums, parts, bytes;
};
GradLayout grad_layout(int32_t dtype, int64_t m, int64_t n, int64_t k) {
  GradLayout g;
  // short strips while there are too few workgroups of long ones
  g.each = m * n < (int64_t)4 << 20 ? 1 : 4;
  g.strips = ceil_div(m, 16 * g.each);
  g.lddz = ceil_div(n, 8) * 8;
  g.sums = up256((uint64_t)m * g.lddz * size_of(dtype));
  g.parts = g.sums + up256((uint64_t)g.strips * n * 4);
  const int64_t s = size_of(dtype);
  const uint64_t dx = parts_bytes(cut_of(m, k, n, s, false), m, k), dw = parts_bytes(cut_of(n, k, m, s, false), n, k);
  g.bytes = g.parts + (dx > dw ? dx : dw);
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
  const GradLayout lay = grad_layout(std::is_same<T, float>::value ? MDET_F32 : MDET_F16, g.m, g.n, g.k);
  float* const parts = (float*)(g.workspace + lay.parts);
  const bool own_dz = g.dz || (g.act != MDET_ACT_NONE && (g.dx || g.dw));
  T* const dz = g.dz ? (T*)g.dz : own_dz ? (T*)g.workspace : nullptr;
  const int64_t lddz = g.dz ? g.lddz : lay.lddz;
  float* const sums = g.db ? (float*)(g.workspace + lay.sums) : nullptr;
  if ((dz || sums) && g.m > 0 && g.n > 0) {
    const int64_t blocks = lay.strips * ceil_div(g.n, DZ_PIECES * Core<T>::VEC);
    auto go = [&](auto each) {
      gemm_launches(blocks, 256, [&](const int64_t first, const dim3 grid) {
        hipLaunchKernelGGL((linear_dz_kernel<T, decltype(each)::value>), grid, dim3(256), 0, g.st, (const T*)g.dy, g.lddy, (const T*)g.z, g.ldz, dz,
                           lddz, sums, g.m, g.n, g.act, first);
      });
    };
    if (lay.each == 1) go(std::integral_constant<int, 1>{});
    else go(std::integral_constant<int, 4>{});
  }
  if (g.db)
    gemm_launches(ceil_div(g.n, DB_COLS), 256, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((linear_db_kernel<O>), grid, dim3(256), 0, g.st, (const float*)sums, lay.strips, g.n, (O*)g.db, first);
    });
  const bool want_dx = g.dx && g.m > 0 && g.k > 0, want_dw = g.dw && g.n > 0 && g.k > 0;
  if (!want_dx && !want_dw && !(g.db && g.n > 0) && !(dz && g.m > 0 && g.n > 0)) return MDET_OK;
  int status = launch_status();
  const T* const d = own_dz ? dz : (const T*)g.dy;
  const int64_t ldd = own_dz ? lddz : g.lddy;
  if (status != MDET_OK) return status;
  const LinearOut<T, T> dx{(T*)g.dx, g.lddx, nullptr, nullptr, 0, nullptr, 0, MDET_ACT_NONE, g.m, g.k, false};
  const LinearOut<T, O> dw{(O*)g.dw, g.lddw, nullptr, nullptr, 0, nullptr, 0, MDET_ACT_NONE, g.n, g.k, false};
  const Operand<T> dzr{d, ldd, g.m, false, false}, dzc{d, ldd, g.n, false, false}, w{(const T*)g.w, g.ldw, g.k, false, false},
      x{(const T*)g.x, g.ldx, g.k, false, false};
  if constexpr (sizeof(T) == 2) {
    if (want_dx && want_dw && pair<T, O>(dzr, w, g.n, dx, dzc, x, g.m, dw, g.st)) return launch_status();
  }
  if (want_dx) status = product<T, T, false, true>(dzr, w, g.n, dx, parts, g.st);
  if (status == MDET_OK && want_dw) status = product<T, O, true, true>(dzc, x, g.m, dw, parts, g.st);
  return status;
}

}  // namespace

extern "C" {

int mdet_linear_workspace_query(int32_t dtype, int32_t backward, int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  if (!bytes || !is_type(dtype) || !sizes_fit(m, n, k)) return MDET_EINVAL;
  *bytes = backward ? grad_layout(dtype, m, n, k).bytes : parts_bytes(cut_of(m, n, k, size_of(dtype), true), m, n);
  return MDET_OK;
}

int mdet_linear_forward(int32_t dtype, int32_t activation, int64_t m, int64_t n, int64_t k, const void* x, int64_t ldx, const void* w,
                        int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, int64_t ldz,
                        void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || activation < MDET_ACT_NONE || activation > MDET_ACT_SILU || !sizes_fit(m, n, k) || !tiles_fit(m, n)) return MDET_EINVAL;
  const int64_t s = size_of(dtype);
  if (!matrix_ok(x, m, k, ldx, s) || !matrix_ok(w, n, k, ldw, s) || !matrix_ok(y, m, n, ldy, s)) return MDET_EINVAL;
  if ((residual && !matrix_ok(residual, m, n, ldr, s)) || (z && !matrix_ok(z, m, n, ldz, s)) || (uintptr_t)bias % s) return MDET_EINVAL;
  uint64_t need = 0;
  mdet_linear_workspace_query(dtype, 0, m, n, k, &need);
  if (need && (!workspace || (uintptr_t)workspace % 256)) return MDET_EINVAL;
  if (workspace_bytes < need) return MDET_ENOMEM_DEVICE;
  if (m == 0 || n == 0) return MDET_OK;
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    const LinearOut<T, T> out{(T*)y, ldy, (const T*)bias, (const T*)residual, ldr, (T*)z, ldz, activation, m, n, false};
    return product<T, T, false, false>(Operand<T>{(const T*)x, ldx, m, false, false}, Operand<T>{(const T*)w, ldw, n, false, false}, k, out, (float*)workspace, (hipStream_t)stream);
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
  if (dx && (!matrix_ok(dx, m, k, lddx, s) || !matrix_ok(w, n, k, ldw, s) || !tiles_fit(m, k))) return MDET_EINVAL;
  if (dw && (!matrix_ok(dw, n, k, lddw, gs) || !matrix_ok(x, m, k, ldx, s) || !tiles_fit(n, k))) return MDET_EINVAL;
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
