// C ABI of the softmax cross entropy of a linear layer and its gradient: argument checks, workspace layout and kernel launches.  A
// call only queues work on the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels_xent.h"
#include "linear_cut.h"
#include "operands.h"
#include "xent_cut.h"

namespace {

using namespace mdet;

typedef Tile<256, 256, 2, 4, 2> Big;
typedef Tile<128, 128, 2, 2, 2> Mid;
typedef Tile<64, 64, 2, 2, 2> Small;
typedef Tile<32, 32, 2, 2, 4> Tiny;

// f(shape) with the tile shape that a cut names.
template <typename T, typename F>
void with_tile(int tile, F&& f) {
  if (tile == 256) {
    if constexpr (sizeof(T) == 2) f(Big{});
  } else if (tile == 128) f(Mid{});
  else if (tile == 64) f(Small{});
  else f(Tiny{});
}

template <typename S>
XentUnits whole_units(int64_t rows, int64_t cols, int64_t k) {
  const int64_t down = ceil_div(rows, S::BM), across = ceil_div(cols, S::BN);
  return XentUnits{(int)down, (int)across, (int)(down * across), (int)(down * across), 1, k, k, nullptr};
}

// Workgroups for these units: a multiple of eight; for large tiles whose operands go straight to LDS, of which a compute unit holds one
// and a workgroup can take several, no more than there are of those.
template <typename S>
dim3 units_grid(const XentUnits& u, bool direct) {
  const int64_t all = ceil_div(ceil_div(u.whole, 8) * 8 + u.units - u.whole, 8) * 8;
  return dim3((unsigned)(S::BM == 256 && direct && all > 256 ? 256 : all));
}

// The places of what the forward pass leaves: in the caller's `kept`, or without the exponentials in the workspace.
template <typename T>
XentForward<T> forward_places(char* at, const XentLayout& l, bool keep) {
  XentForward<T> o{};
  o.exps = keep ? (typename XentKept<T>::type*)at : nullptr;
  o.ldexps = l.ldexps;
  char* const rest = keep ? at + l.exps_bytes : at;
  o.strips = (XentStrip*)rest;
  o.across = l.across;
  o.picked = (float*)(rest + l.strips_bytes);
  return o;
}

// A copy of rows of k elements at a distance of `ld`.
template <typename T>
void copy_rows(const T* from, int64_t ldfrom, const XentTargets& t, int64_t rows, int64_t k, T* to, int64_t ld, hipStream_t st) {
  gemm_launches(ceil_div(rows * (ld / Core<T>::VEC), 256), 256, [&](const int64_t first, const dim3 grid) {
    hipLaunchKernelGGL((xent_rows_kernel<T>), grid, dim3(256), 0, st, from, ldfrom, t, rows, k, to, ld, first);
  });
}

template <typename T>
int forward(Operand<T> x, Operand<T> w, int64_t k, XentForward<T> o, const XentLayout& l, char* copies, float* loss, float* lse,
            hipStream_t st) {
  if (o.cols > 0) {
    if (l.copies) {
      const int64_t ld = xent_pad(k);
      copy_rows<T>(x.p, x.stride, XentTargets{}, x.rows, k, (T*)copies, ld, st);
      copy_rows<T>(w.p, w.stride, XentTargets{}, w.rows, k, (T*)(copies + l.x_bytes), ld, st);
      x.p = (const T*)copies;
      w.p = (const T*)(copies + l.x_bytes);
      x.stride = w.stride = k = ld;
    }
    if (l.cut.tile == 0) {
      // Few rows of x want more of W on its way, many share their own loads out over more of it, as long as that leaves enough workgroups.  us for
      // one, two, four groups of W, rows of 4096 bf16: 4 rows over 131072 words 194, 198, 219, 8 rows 223, 212, 224, 16 rows 277, 243, 236; 16
      // rows over 5000 words 23, 19, 31.  (Tiles of 256: 261 for 5 rows, 268 for 16.)
      auto go = [&](auto groups) {
        constexpr int G = decltype(groups)::value;
        hipLaunchKernelGGL((xent_forward_rows_kernel<T, G>), dim3((unsigned)ceil_div(o.cols, 16 * G)), dim3(64 * XENT_WAVES), 0, st, x, w, k, o);
      };
      if (o.rows <= 4) go(std::integral_constant<int, 1>{});
      else if (o.rows <= 8 || o.cols < 16384) go(std::integral_constant<int, 2>{});
      else go(std::integral_constant<int, 4>{});
    } else
      with_tile<T>(l.cut.tile, [&](auto shape) {
        typedef decltype(shape) S;
        x = gemm_operand<T, false, S::BM>(x.p, x.stride, x.rows, k);
        w = gemm_operand<T, false, S::BN>(w.p, w.stride, w.rows, k);
        const bool direct = x.straight && w.straight;
        const XentUnits u = whole_units<S>(o.rows, o.cols, k);
        const dim3 grid = units_grid<S>(u, direct), block(S::THREADS);
        if (direct) hipLaunchKernelGGL((xent_forward_kernel<T, S, true>), grid, block, 0, st, x, w, o, u);
        else hipLaunchKernelGGL((xent_forward_kernel<T, S, false>), grid, block, 0, st, x, w, o, u);
      });
  }
  // a row's strips by a wavefront, or by sixteen where they are many
  if (l.across > 1024)
    gemm_launches(o.rows, 1024, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((xent_join_kernel<1024>), grid, dim3(1024), 0, st, (const XentStrip*)o.strips, l.across, o.picked, o.t, o.rows,
                         loss, lse, first);
    });
  else
    gemm_launches(ceil_div(o.rows, 4), 256, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((xent_join_kernel<64>), grid, dim3(256), 0, st, (const XentStrip*)o.strips, l.across, o.picked, o.t, o.rows,
                         loss, lse, first);
    });
  return launch_status();
}

template <typename O>
bool whole_pieces(const XentOut<O>& o) {
  return (uintptr_t)o.y % 16 == 0 && (o.rows == 1 || o.ldy * sizeof(O) % 16 == 0);
}

template <typename T, typename O, bool ROUTER>
void product(Operand<T> r, Operand<T> c, int64_t k, XentOut<O> o, float* parts, hipStream_t st) {
  const XentCut cut = xent_cut(o.rows, o.cols, k, sizeof(T));
  const XentUnits u{(int)cut.down, (int)cut.across, (int)cut.whole, (int)cut.units(), cut.splits, k, cut.kpart, parts};
  o.vec = whole_pieces(o);
  with_tile<T>(cut.tile, [&](auto shape) {
    typedef decltype(shape) S;
    r = gemm_operand<T, ROUTER, S::BM>(r.p, r.stride, r.rows, k);
    c = gemm_operand<T, true, S::BN>(c.p, c.stride, c.rows, k);
    const bool direct = r.straight && c.straight;
    const dim3 grid = units_grid<S>(u, direct), block(S::THREADS);
    if (direct) hipLaunchKernelGGL((xent_product_kernel<T, O, S, ROUTER, true>), grid, block, 0, st, r, c, o, u);
    else hipLaunchKernelGGL((xent_product_kernel<T, O, S, ROUTER, false>), grid, block, 0, st, r, c, o, u);
    if (u.units > u.whole) {
      const int tiles = u.down * u.across - u.whole;
      hipLaunchKernelGGL((xent_product_join_kernel<O, S::BM, S::BN>), dim3((unsigned)(tiles * (S::BM * S::BN / 1024))), dim3(256), 0, st, o, u);
    }
  });
}

// Numbers of the operands' type that add up to an element of e: 8 bits each in bf16, 11 in fp16, of 24.
int64_t parts_of(int32_t dtype, int32_t grad_dtype) { return dtype == MDET_F32 || grad_dtype != MDET_F32 ? 1 : dtype == MDET_BF16 ? 3 : 2; }

int64_t kept_size(int32_t dtype) { return dtype == MDET_BF16 ? 2 : 4; }

struct Grad {
  XentTargets t;
  int64_t m, n, k;
  const float *g, *lse, *loss;         // loss null: what lse says of it
  const void *x, *w, *bias;
  int64_t ldx, ldw;
  char* kept;                          // null: nothing was kept
  void *dx, *dw, *db;
  int64_t lddx, lddw;
  char* workspace;
  hipStream_t st;
};

template <typename T, typename O>
int backward(const Grad& a) {
  const XentLayout f = xent_layout(a.m, a.n, a.k, sizeof(T), sizeof(typename XentKept<T>::type));
  constexpr int parts_of_e = sizeof(T) == sizeof(O) ? 1 : std::is_same<T, _Float16>::value ? 2 : 3;
  const XentGradLayout l = xent_grad_layout(a.m, a.n, a.k, sizeof(T), parts_of_e);
  // what was kept may be rounded to 11 bits, which is not enough for more than one part
  char* const kept = parts_of_e == 1 ? a.kept : nullptr;
  const XentForward<T> was = a.kept ? forward_places<T>(a.kept, f, true) : XentForward<T>{};
  const float* const loss = a.kept ? was.picked : a.loss;
  hipStream_t st = a.st;
  T *const e = (T*)(a.workspace + l.e), *const rows = (T*)(a.workspace + l.rows);
  float *const sums = (float*)(a.workspace + l.sums), *const total = (float*)(a.workspace + l.total), *const parts = (float*)(a.workspace + l.parts);
  XentScale* scale = nullptr;
  if constexpr (sizeof(T) == 2) {
    scale = (XentScale*)(a.workspace + l.scale);
    hipLaunchKernelGGL((xent_scale_kernel<T>), dim3(1), dim3(1024), 0, st, a.g, a.t, a.m, scale);
  }
  const bool own_rows = a.k > 0 && (a.dw || (l.copies && !kept));
  for (int part = 0; own_rows && part < parts_of_e; ++part)
    copy_rows<T>((const T*)a.x, a.ldx, a.t, a.m, a.k, rows + part * a.m * l.ldrows, l.ldrows, st);
  for (int64_t v = 0; v < a.n; v += l.piece) {
    const int64_t n = a.n - v < l.piece ? a.n - v : l.piece;
    const T* w = (const T*)a.w + v * a.ldw;
    int64_t ldw = a.ldw, k = a.k;      // of the sums for e, zeros behind a row's end among them
    const bool own_w = l.copies && (a.dx || !kept);
    if (own_w) {
      copy_rows<T>(w, ldw, XentTargets{}, n, a.k, (T*)(a.workspace + l.w), l.ldrows, st);
      w = (const T*)(a.workspace + l.w);
      ldw = k = l.ldrows;
    }
    const XentSlope<T> o{a.t, a.bias ? (const T*)a.bias + v : nullptr, a.lse, a.g, loss, scale, e, l.lde, a.db ? sums : nullptr, a.m, n, v};
    int64_t strips = 0;
    if (kept) {
      strips = ceil_div(a.m, 16 * XENT_EACH);
      gemm_launches(strips * ceil_div(n, 16 * Core<T>::VEC), 256, [&](const int64_t first, const dim3 grid) {
        hipLaunchKernelGGL((xent_slope_kept_kernel<T>), grid, dim3(256), 0, st, o, was.exps, was.ldexps, (const XentStrip*)was.strips, was.across, f.strip, first);
      });
    } else
      with_tile<T>(cut_of(a.m, n, a.k, sizeof(T), false).tile, [&](auto shape) {
        typedef decltype(shape) S;
        const Operand<T> x = own_w ? gemm_operand<T, false, S::BM>(rows, l.ldrows, a.m, k) : gemm_operand<T, false, S::BM>(a.x, a.ldx, a.m, k);
        const Operand<T> c = gemm_operand<T, false, S::BN>(w, ldw, n, k);
        const bool direct = x.straight && c.straight;
        const XentUnits u = whole_units<S>(a.m, n, k);
        const dim3 grid = units_grid<S>(u, direct), block(S::THREADS);
        strips = ceil_div(a.m, S::BM) * S::WM;
        if (direct) hipLaunchKernelGGL((xent_slope_kernel<T, S, true, parts_of_e>), grid, block, 0, st, x, c, o, u);
        else hipLaunchKernelGGL((xent_slope_kernel<T, S, false, parts_of_e>), grid, block, 0, st, x, c, o, u);
      });
    if (a.db)
      gemm_launches(ceil_div(n, 16), 256, [&](const int64_t first, const dim3 grid) {
        hipLaunchKernelGGL((xent_columns_kernel<O>), grid, dim3(256), 0, st, (const float*)sums, strips, n, (O*)a.db + v, first);
      });
    if (a.dx && a.k > 0)
      product<T, T, false>(Operand<T>{e, l.lde, a.m, false, false}, Operand<T>{w, ldw, a.k, false, false}, n,
                           XentOut<T>{(T*)a.dx, a.lddx, scale, total, v == 0, v + n == a.n, a.m, a.k, false}, parts, st);
    if (a.dw && a.k > 0)
      product<T, O, true>(Operand<T>{e, l.lde, n, false, false}, Operand<T>{rows, l.ldrows, a.k, false, false}, parts_of_e * a.m,
                          XentOut<O>{(O*)a.dw + v * a.lddw, a.lddw, scale, nullptr, true, true, n, a.k, false}, parts, st);
  }
  return launch_status();
}

// A matrix without rows to sum over is zero.
template <typename O>
__global__ __launch_bounds__(256) void zero_kernel(O* to, const int64_t ld, const int64_t rows, const int64_t cols, const int64_t first) {
  const int64_t id = (first + blockIdx.x) * 256 + threadIdx.x, i = id / cols;
  if (i < rows) to[i * ld + (id - i * cols)] = (O)0.0f;
}
template <typename O>
void zero(void* to, int64_t ld, int64_t rows, int64_t cols, hipStream_t st) {
  if (!to || rows * cols == 0) return;
  gemm_launches(ceil_div(rows * cols, 256), 256, [&](const int64_t first, const dim3 grid) {
    hipLaunchKernelGGL((zero_kernel<O>), grid, dim3(256), 0, st, (O*)to, ld, rows, cols, first);
  });
}

bool is_index(int32_t bits) { return bits == 32 || bits == 64; }

// As tiles_fit of the linear layer.
bool tiles_fit(int64_t rows, int64_t cols) { return ceil_div(rows, 32) * ceil_div(cols, 32) <= (int64_t(1) << 26) - 1024; }
bool xent_fits(int64_t m, int64_t n, int64_t k) { return sizes_fit(m, n, k) && tiles_fit(m, n) && tiles_fit(m, k) && tiles_fit(n, k); }

}  // namespace

extern "C" {

int mdet_xent_workspace_query(int32_t dtype, int32_t grad_dtype, int32_t backward, int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  if (!bytes || !is_type(dtype) || (grad_dtype != dtype && grad_dtype != MDET_F32) || !xent_fits(m, n, k)) return MDET_EINVAL;
  const XentLayout l = xent_layout(m, n, k, size_of(dtype), kept_size(dtype));
  *bytes = backward ? xent_grad_layout(m, n, k, size_of(dtype), parts_of(dtype, grad_dtype)).bytes : l.workspace(false);
  return MDET_OK;
}

int mdet_xent_kept_query(int32_t dtype, int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  if (!bytes || !is_type(dtype) || !xent_fits(m, n, k)) return MDET_EINVAL;
  const XentLayout l = xent_layout(m, n, k, size_of(dtype), kept_size(dtype));
  *bytes = l.kept();
  return MDET_OK;
}

int mdet_xent_forward(int32_t dtype, int32_t index_bits, int64_t m, int64_t n, int64_t k, const void* x, int64_t ldx, const void* w, int64_t ldw,
                      const void* bias, const void* target, int64_t ignore, float* loss, float* lse, void* kept, uint64_t kept_bytes,
                      void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || !is_index(index_bits) || !xent_fits(m, n, k)) return MDET_EINVAL;
  const int64_t s = size_of(dtype);
  if (!matrix_ok(x, m, k, ldx, s) || !matrix_ok(w, n, k, ldw, s) || (uintptr_t)bias % s || !vector_ok(target, m, index_bits / 8)) return MDET_EINVAL;
  if ((uintptr_t)loss % 4 || (uintptr_t)lse % 4) return MDET_EINVAL;
  const XentLayout l = xent_layout(m, n, k, s, kept_size(dtype));
  int ok = kept ? workspace_ok(kept, kept_bytes, l.kept()) : MDET_OK;
  if (ok == MDET_OK) ok = workspace_ok(workspace, workspace_bytes, l.workspace(kept != nullptr));
  if (ok != MDET_OK) return ok;
  if (m == 0 || (!loss && !lse && !kept)) return MDET_OK;
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    XentForward<T> o = forward_places<T>(kept ? (char*)kept : (char*)workspace + l.x_bytes + l.w_bytes, l, kept != nullptr);
    o.t = XentTargets{target, index_bits, ignore, n};
    o.bias = (const T*)bias;
    o.rows = m;
    o.cols = n;
    return forward<T>(Operand<T>{(const T*)x, ldx, m, false, false}, Operand<T>{(const T*)w, ldw, n, false, false}, k, o, l, (char*)workspace, loss, lse,
                      (hipStream_t)stream);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

int mdet_xent_reduce(int32_t index_bits, int64_t m, int64_t n, const float* loss, const void* target, int64_t ignore, int32_t mean, float* out,
                     float* weights, void* stream) {
  if (!is_index(index_bits) || !xent_fits(m, n, 1) || !vector_ok(loss, m, 4) || !vector_ok(target, m, index_bits / 8)) return MDET_EINVAL;
  if (!vector_ok(out, 1, 4) || (uintptr_t)weights % 4) return MDET_EINVAL;
  hipLaunchKernelGGL(xent_reduce_kernel, dim3(1), dim3(1024), 0, (hipStream_t)stream, loss, XentTargets{target, index_bits, ignore, n}, m, mean != 0, out,
                     weights);
  return launch_status();
}

int mdet_xent_backward_with_loss(int32_t dtype, int32_t grad_dtype, int32_t index_bits, int64_t m, int64_t n, int64_t k, const float* dloss,
                                 const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, const void* target, int64_t ignore,
                                 const float* lse, const float* loss, const void* kept, uint64_t kept_bytes, void* dx, int64_t lddx, void* dw,
                                 int64_t lddw, void* db, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || (grad_dtype != dtype && grad_dtype != MDET_F32) || !is_index(index_bits) || !xent_fits(m, n, k)) return MDET_EINVAL;
  const int64_t s = size_of(dtype), gs = size_of(grad_dtype);
  if (!matrix_ok(x, m, k, ldx, s) || !matrix_ok(w, n, k, ldw, s) || (uintptr_t)bias % s || !vector_ok(target, m, index_bits / 8)) return MDET_EINVAL;
  if (!vector_ok(dloss, m, 4) || !vector_ok(lse, m, 4) || (uintptr_t)loss % 4) return MDET_EINVAL;
  if ((dx && !matrix_ok(dx, m, k, lddx, s)) || (dw && !matrix_ok(dw, n, k, lddw, gs)) || (uintptr_t)db % gs) return MDET_EINVAL;
  const XentLayout f = xent_layout(m, n, k, s, kept_size(dtype));
  int ok = kept ? workspace_ok(kept, kept_bytes, f.kept()) : MDET_OK;
  if (ok == MDET_OK) ok = workspace_ok(workspace, workspace_bytes, xent_grad_layout(m, n, k, s, parts_of(dtype, grad_dtype)).bytes);
  if (ok != MDET_OK) return ok;
  if (!dx && !dw && !db) return MDET_OK;
  hipStream_t st = (hipStream_t)stream;
  if (m == 0 || n == 0) {              // what is not empty is an empty sum
    dtype == MDET_F32 ? zero<float>(dx, lddx, m, k, st) : zero<_Float16>(dx, lddx, m, k, st);
    grad_dtype == MDET_F32 ? zero<float>(dw, lddw, n, k, st) : zero<_Float16>(dw, lddw, n, k, st);
    grad_dtype == MDET_F32 ? zero<float>(db, n, 1, n, st) : zero<_Float16>(db, n, 1, n, st);
    return launch_status();
  }
  const Grad a{XentTargets{target, index_bits, ignore, n}, m, n, k, dloss, lse, loss, x, w, bias, ldx, ldw, (char*)kept, dx, dw, db, lddx, lddw, (char*)workspace,
               st};
  auto call = [&](auto zero) {
    typedef decltype(zero) T;
    return grad_dtype == MDET_F32 ? backward<T, float>(a) : backward<T, T>(a);
  };
  return dtype == MDET_F32 ? call(0.0f) : dtype == MDET_BF16 ? call((__bf16)0.0f) : call((_Float16)0.0f);
}

int mdet_xent_backward(int32_t dtype, int32_t grad_dtype, int32_t index_bits, int64_t m, int64_t n, int64_t k, const float* dloss, const void* x,
                       int64_t ldx, const void* w, int64_t ldw, const void* bias, const void* target, int64_t ignore, const float* lse,
                       const void* kept, uint64_t kept_bytes, void* dx, int64_t lddx, void* dw, int64_t lddw, void* db, void* workspace,
                       uint64_t workspace_bytes, void* stream) {
  return mdet_xent_backward_with_loss(dtype, grad_dtype, index_bits, m, n, k, dloss, x, ldx, w, ldw, bias, target, ignore, lse, nullptr, kept, kept_bytes,
                                      dx, lddx, dw, lddw, db, workspace, workspace_bytes, stream);
}

}  // extern "C"
