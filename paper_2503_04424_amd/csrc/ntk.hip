// C ABI of the Gram matrix of a network's Jacobian: argument checks, workspace layout and kernel launches.  A call only
// queues work on the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "kernels_ntk.h"
#include "../../include/memdet.h"

namespace {

using namespace mdet;

inline uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t size_of(int32_t t) { return t == MDET_F64 ? 8 : t == MDET_F32 ? 4 : 2; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? MDET_OK : MDET_EHIP; }

constexpr int64_t MOST = INT32_MAX;
constexpr int64_t MOST_ELEMENTS = int64_t(1) << 38;      // of an operand: a terabyte or two; a launch over them fits 31 bits

// Types, sizes and strides; pointers only where `pointers` is set.
int check(int32_t dtype, int32_t out_dtype, int64_t n, int64_t outputs, const mdet_ntk_layer* layers, int32_t count, bool pointers) {
  if (dtype < MDET_F32 || dtype > MDET_BF16 || (out_dtype != MDET_F32 && out_dtype != MDET_F64)) return MDET_EINVAL;
  if (dtype == MDET_F64 && out_dtype == MDET_F32) return MDET_EINVAL;      // arithmetic narrower than the operands
  if (n < 0 || outputs < 1 || count < 0 || (count > 0 && !layers)) return MDET_EINVAL;
  if (n > MOST || outputs > MOST || (n > 0 && outputs > MOST / n)) return MDET_EINVAL;
  if (outputs > 1 && n > (int64_t(1) << 24)) return MDET_EINVAL;           // first factors of n x n
  for (int l = 0; l < count; ++l) {
    const mdet_ntk_layer& x = layers[l];
    if (x.p < 0 || x.q < 0 || x.p > MOST || x.q > MOST) return MDET_EINVAL;
    if (n > 0 && (x.p > MOST_ELEMENTS / n || x.q > MOST_ELEMENTS / (n * outputs))) return MDET_EINVAL;
    if (!pointers || n == 0) continue;
    const int64_t s = size_of(dtype);
    if (x.p > 0 && (!x.a || (uintptr_t)x.a % s || x.lda > MOST || x.lda < 0 || (n > 1 && x.lda < x.p))) return MDET_EINVAL;
    if (x.q > 0 && (!x.g || (uintptr_t)x.g % s || x.ldg > MOST || x.ldg < 0 || (n * outputs > 1 && x.ldg < x.q))) return MDET_EINVAL;
  }
  return MDET_OK;
}

// A widened operand's bytes, rows of whole pieces.
inline uint64_t wide_bytes(int64_t rows, int64_t cols) { return up256((uint64_t)rows * (ceil_div(cols, 2) * 2) * 8); }

template <typename S>
void widen(const void* from, int64_t ld, int64_t rows, int64_t cols, double* to, hipStream_t st) {
  const int64_t ldto = ceil_div(cols, 2) * 2;
  gemm_launches(ceil_div(rows * ldto, 256), 256, [&](const int64_t first, const dim3 grid) {
    hipLaunchKernelGGL(ntk_widen_kernel<S>, grid, dim3(256), 0, st, (const S*)from, ld, to, rows, cols, ldto, first);
  });
}

struct Call {
  int64_t n, d;
  double bias, scale;
  int accumulate;
  void* K;
  int64_t ldk;
  hipStream_t st;
};

typedef Tile<128, 128, 2, 4, 2> Large;
typedef Tile<64, 64, 2, 2, 2> Small;
typedef Tile<32, 32, 2, 2, 4> Tiny;

constexpr int64_t COMPUTE_UNITS = 256;

// First factors of one launch's layers, for several outputs.
inline uint64_t first_bytes(int64_t n, int64_t d, int32_t layers, int64_t size) {
  return d > 1 ? up256((uint64_t)(layers < NTK_LAYERS ? layers : NTK_LAYERS) * n * n * size) : 0;
}

// Which of the blocks a call computes, and whether a quarter at a time.
struct Range {
  int64_t begin, count;
  bool firsts;                         // and the first factors before them
};

template <typename T, typename S, bool PARTS = false>
int gram_tiles(NtkLayers<T>& list, const Call& c, int accumulate, void* first, Range range = Range{0, -1, true}) {
  typedef typename Core<T>::acc1_t A;
  // A launch goes straight to LDS where most of what it reads can go there: a last layer of one output, whose rows are
  // single elements, does not hold up the others.
  int64_t yes_a = 0, no_a = 0, yes_g = 0, no_g = 0;
  list.near_a = list.near_g = list.straight_a = list.straight_g = 0;
  for (int l = 0; l < list.count; ++l) {
    const Operand<T> a = gemm_operand<T, false, S::BM>(list.a[l], list.lda[l], c.n, list.p[l]);
    const Operand<T> g = gemm_operand<T, false, S::BM>(list.g[l], list.ldg[l], c.n * c.d, list.q[l]);
    list.near_a |= (uint32_t)a.near << l;
    list.near_g |= (uint32_t)g.near << l;
    list.straight_a |= (uint32_t)a.straight << l;
    list.straight_g |= (uint32_t)g.straight << l;
    (a.straight ? yes_a : no_a) += list.p[l];
    (g.straight ? yes_g : no_g) += list.q[l];
  }
  // In fp64 the large tile has no registers left for operands that pass through them; quarters come behind large blocks that went
  // straight.  In 16 bits large blocks, and so quarters, are for several outputs.
  constexpr bool REGISTERS = !(std::is_same<T, double>::value && (S::BM == 128 || PARTS));
  constexpr bool ONE = !(sizeof(T) == 2 && (S::BM == 128 || PARTS));
  if constexpr (!REGISTERS && !PARTS) {
    if (no_g > yes_g / 8 || (c.d > 1 && no_a > yes_a / 8) || (c.d == 1 && no_a + no_g > (yes_a + yes_g) / 8))
      return gram_tiles<T, Small>(list, c, accumulate, first);
  }
  const int64_t blocks = ntk_blocks(ceil_div(c.n * c.d, S::BM));
  // What is left over behind whole rounds of large blocks would hold up a few compute units for as long as a round takes (fp64
  // n = 8192, 2080 blocks: 3.08 ms): it goes out in quarters (2.88 ms).
  if constexpr (S::BM == 128) {
    const int64_t rest = blocks % COMPUTE_UNITS;
    if (range.count < 0 && rest > 0 && rest <= COMPUTE_UNITS / 2) {
      const int status = gram_tiles<T, S>(list, c, accumulate, first, Range{0, blocks - rest, true});
      return status != MDET_OK ? status : gram_tiles<T, Small, true>(list, c, accumulate, first, Range{blocks - rest, rest, false});
    }
  }
  if (range.count < 0) range.count = blocks;
  const int64_t all = ceil_div(range.count * (PARTS ? 4 : 1), 8) * 8;
  const int64_t firsts = c.d > 1 ? ceil_div(ntk_blocks(ceil_div(c.n, S::BM)) * list.count, 8) * 8 : 0;
  if (all > (int64_t)UINT32_MAX / S::THREADS || firsts > (int64_t)UINT32_MAX / S::THREADS) return MDET_EINVAL;    // threads of a launch
  using std::false_type;
  using std::true_type;
  auto gram = [&](auto direct, auto several) {
    hipLaunchKernelGGL((ntk_gram_kernel<T, S, decltype(direct)::value, decltype(several)::value, PARTS>), dim3((unsigned)all), dim3(S::THREADS), 0, c.st,
                       list, range.begin, range.count, c.n, (int)c.d, (A)c.bias, (A)c.scale, accumulate, (const A*)first, (A*)c.K, c.ldk);
  };
  if (c.d > 1) {
    auto firsts_of = [&](auto direct) {
      hipLaunchKernelGGL((ntk_first_kernel<T, S, decltype(direct)::value>), dim3((unsigned)firsts), dim3(S::THREADS), 0, c.st, list, c.n, (A)c.bias,
                         (A*)first);
    };
    if (list.count > 0 && range.firsts) {
      if (no_a <= yes_a / 8) firsts_of(true_type{});
      else if constexpr (REGISTERS) firsts_of(false_type{});
    }
    if (no_g <= yes_g / 8) gram(true_type{}, true_type{});
    else if constexpr (REGISTERS) gram(false_type{}, true_type{});
  } else if constexpr (ONE) {
    if (no_a + no_g <= (yes_a + yes_g) / 8) gram(true_type{}, false_type{});
    else if constexpr (REGISTERS) gram(false_type{}, false_type{});
  }
  return launch_status();
}

template <typename T>
int gram(const mdet_ntk_layer* layers, int32_t count, const Call& c, void* first) {
  int accumulate = c.accumulate;
  for (int32_t l0 = 0; l0 == 0 || l0 < count; l0 += NTK_LAYERS) {
    NtkLayers<T> list;
    list.count = count - l0 < NTK_LAYERS ? count - l0 : NTK_LAYERS;
    for (int l = 0; l < list.count; ++l) {
      const mdet_ntk_layer& x = layers[l0 + l];
      list.a[l] = (const T*)x.a, list.lda[l] = x.lda, list.p[l] = x.p;
      list.g[l] = (const T*)x.g, list.ldg[l] = x.ldg, list.q[l] = x.q;
    }
    // Several workgroups a compute unit, and so the 64 x 64 tile, are better than one large one in fp32 (n = 8192, three layers:
    // 1.48 ms, 1.65 with 128 x 128) and at small orders.  In us, 128 x 128 and 64 x 64, fp64 with three layers of 512 to 784:
    // one output order 2048 346, 305; 3000 482, 507; 4096 826, 894; 6000 1595, 1771; 8192 2866, 3200; 12000 6016, 6774; three
    // outputs 3000 294, 260; 4500 499, 494; 6000 830, 876; 9000 1730, 1863.  bf16, ten outputs of four layers: 4000 103, 80; 6000 156,
    // 147; 7000 205, 194; 8000 240, 252; 10000 366, 384; 16000 869, 932; three outputs: 3000 63, 50; 4500 88, 92; 6000 140, 142;
    // 9000 275, 303.  A few small blocks would leave most compute units without one: n = 512 in fp32 21 us with the 32 x 32 tile, 35
    // with 64 x 64, in fp64 29 and 63.
    const int64_t order = c.n * c.d;
    int status;
    if (order >= (sizeof(T) == 8 ? 4500 : 8000) && c.d != 2 && (sizeof(T) == 8 || (sizeof(T) == 2 && c.d > 1))) {
      if constexpr (sizeof(T) != 4) status = gram_tiles<T, Large>(list, c, accumulate, first);
    } else if (sizeof(T) != 2 && order < 1500) {
      if constexpr (sizeof(T) != 2) status = gram_tiles<T, Tiny>(list, c, accumulate, first);
    } else status = gram_tiles<T, Small>(list, c, accumulate, first);
    if (status != MDET_OK) return status;
    accumulate = 1;
  }
  return MDET_OK;
}

}  // namespace

extern "C" {

int mdet_ntk_workspace_query(int32_t dtype, int32_t out_dtype, int64_t n, int64_t outputs, const mdet_ntk_layer* layers, int32_t count,
                             uint64_t* bytes) {
  if (!bytes) return MDET_EINVAL;
  const int status = check(dtype, out_dtype, n, outputs, layers, count, false);
  if (status != MDET_OK) return status;
  uint64_t sum = first_bytes(n, outputs, count, size_of(out_dtype));
  if (out_dtype == MDET_F64 && dtype != MDET_F64)
    for (int l = 0; l < count; ++l) sum += wide_bytes(n, layers[l].p) + wide_bytes(n * outputs, layers[l].q);
  *bytes = sum;
  return MDET_OK;
}

int mdet_ntk_gram(int32_t dtype, int32_t out_dtype, int64_t n, int64_t outputs, const mdet_ntk_layer* layers, int32_t count, double bias,
                  double scale, int32_t accumulate, void* K, int64_t ldk, void* workspace, uint64_t workspace_bytes, void* stream) {
  int status = check(dtype, out_dtype, n, outputs, layers, count, true);
  if (status != MDET_OK) return status;
  // in the type of the arithmetic
  auto finite = [&](double x) { return out_dtype == MDET_F32 ? std::isfinite((float)x) : std::isfinite(x); };
  if (!finite(bias) || !finite(scale)) return MDET_EINVAL;
  const int64_t N = n * outputs;
  if (N == 0) return MDET_OK;
  if (!K || (uintptr_t)K % size_of(out_dtype) || (N > 1 && ldk < N) || ldk > MOST) return MDET_EINVAL;
  uint64_t need = 0;
  mdet_ntk_workspace_query(dtype, out_dtype, n, outputs, layers, count, &need);
  if (need && (!workspace || (uintptr_t)workspace % 256)) return MDET_EINVAL;
  if (workspace_bytes < need) return MDET_ENOMEM_DEVICE;
  hipStream_t st = (hipStream_t)stream;
  const Call c{n, outputs, bias, scale, accumulate, K, ldk, st};
  if (out_dtype == MDET_F32)
    return dtype == MDET_F32 ? gram<float>(layers, count, c, workspace) : dtype == MDET_BF16 ? gram<__bf16>(layers, count, c, workspace) : gram<_Float16>(layers, count, c, workspace);
  if (dtype == MDET_F64) return gram<double>(layers, count, c, workspace);
  // narrower operands: exact copies in fp64, one launch's layers after the other in the workspace
  char* at = (char*)workspace + first_bytes(n, outputs, count, 8);
  int acc = accumulate;
  for (int32_t l0 = 0; l0 == 0 || l0 < count; l0 += NTK_LAYERS) {
    mdet_ntk_layer wide[NTK_LAYERS];
    const int some = count - l0 < NTK_LAYERS ? count - l0 : NTK_LAYERS;
    for (int l = 0; l < some; ++l) {
      wide[l] = layers[l0 + l];
      auto one = [&](const void*& p, int64_t& ld, int64_t rows, int64_t cols) {
        double* const to = (double*)at;
        at += wide_bytes(rows, cols);
        if (dtype == MDET_F32) widen<float>(p, ld, rows, cols, to, st);
        else if (dtype == MDET_BF16) widen<__bf16>(p, ld, rows, cols, to, st);
        else widen<_Float16>(p, ld, rows, cols, to, st);
        p = to;
        ld = ceil_div(cols, 2) * 2;
      };
      one(wide[l].a, wide[l].lda, n, wide[l].p);
      one(wide[l].g, wide[l].ldg, N, wide[l].q);
    }
    Call part = c;
    part.accumulate = acc;
    status = gram<double>(wide, some, part, workspace);
    if (status != MDET_OK) return status;
    acc = 1;
  }
  return MDET_OK;
}

}  // extern "C"
