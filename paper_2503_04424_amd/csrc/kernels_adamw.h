// One AdamW step over many tensors.  For every element, in fp32 (m, v: running means of the gradient and of its
// square, t the number of the step):
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + ((1 - b2) g) g
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) (m / (sqrt(v) / sqrt(1 - b2^t) + eps))
//
// Every operation is rounded by itself (no fused multiply-add), so a tensor gives the same bits whatever tensors
// stand beside it, however it is aligned and whichever path takes it.
//
// States in 8 bits: ADAMW_BLOCK consecutive elements share two scales; m is code * scale with a code of -127 .. 127,
// sqrt(v) is code * scale with a code of 0 .. 255 (the root spans half the orders of magnitude that v does).  A code is
// floor(x / scale + r) with r uniform in [0, 1): rounded up with the probability of what is left over.  To nearest, v
// would never decay: with b2 = 0.999 a step changes its root by 0.05 %, far less than half a code, and the state would
// stand still until a gradient some ten times its root arrives.  r comes from a hash of the element's number, the tensor's
// and the caller's seed.  A root that is not zero has a code of at least 1: a code of 0 would divide its m by eps.
// This step's own update uses m and v before they are rounded.
//
// The mean of what is stored is the root that was rounded (from one code on).  The recurrence squares it, and the mean of the square is
// larger by the rounding's variance, so roots far below their block's largest settle too high and their steps are shorter by as much:
// with b2 = 0.999, normal gradients and 6000 steps (simulated) by 1 % at 10 % of the block's largest, 3 % at 5 %, 6 % at 2 %,
// 12 % at 1 % and 30 % at half a per cent.
//
// What bounds it: bytes.  28 a element with states, parameters and gradients in 32 bits (67 million elements: 360 us,
// 5.2 TB/s); with states in 8 bits, 16 and the two scales of a block (225 us, 4.9 TB/s), where the arithmetic is close behind.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/memdet.h"

namespace mdet {

constexpr int ADAMW_BLOCK = 256;       // elements that share a scale: one wavefront's, four a lane
constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_STEP = 1024;       // elements a workgroup takes at a time
constexpr int ADAMW_TENSORS = 48;      // a launch's, so that they fit the kernel's arguments
constexpr int64_t ADAMW_CHUNKS = (int64_t)UINT32_MAX / ADAMW_THREADS;   // a launch's, which holds fewer than 2^32 threads

struct AdamwFactors {
  float b1, a1, b2, a2, keep, rate, root, eps;
  const float* grad_scale;             // device; null: 1
  uint32_t seed;
  int first_tensor;                    // number of the launch's first tensor in the call
};

struct AdamwTensors {
  int count;
  int chunk;                           // elements a workgroup takes, whole steps
  uint32_t first[ADAMW_TENSORS + 1];   // number of each tensor's first chunk in the launch
  mdet_adamw_tensor t[ADAMW_TENSORS];
};
static_assert(sizeof(AdamwTensors) + sizeof(AdamwFactors) < 4096, "fits a kernel's arguments");

// 32 random bits of element i of tensor t: multiplications by the fractional digits of square roots and shifts.
__device__ __forceinline__ uint32_t adamw_bits(const uint32_t key, const int64_t i) {
  uint32_t h = (uint32_t)i * 0x6A09E667u + (uint32_t)((uint64_t)i >> 32) * 0x9B05688Du + key;
  h = (h ^ (h >> 16)) * 0xBB67AE85u;
  h = (h ^ (h >> 15)) * 0x3C6EF373u;
  return h ^ (h >> 16);
}

// The largest of the wavefront's, in all lanes: rows of 16 by shifts, then across rows.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(const uint32_t x) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
  return x > o ? x : o;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = dpp_max<0x111>(x);               // row_shr 1, 2, 4, 8
  x = dpp_max<0x112>(x);
  x = dpp_max<0x114>(x);
  x = dpp_max<0x118>(x);
  x = dpp_max<0x142>(x);               // row_bcast 15, 31
  x = dpp_max<0x143>(x);
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// x / d for a d that a whole block shares, correctly rounded: with y the correctly rounded reciprocal of d and q = x y, the
// remainder x - q d is exact and q + (x - q d) y rounds to the quotient (Markstein).  Three instructions in place of some
// ten.  Where d is so small or large that a step could leave the range, it is an ordinary division; a quotient too small
// for the remainder to be exact is lost beside the random number that is added to it.
struct BlockDivisor {
  float d, y;
  bool quick;
  __device__ __forceinline__ explicit BlockDivisor(const float by) : d(by), y(1.0f / by), quick(by > 0x1p-60f && by < 0x1p60f) {}
  __device__ __forceinline__ float operator()(const float x) const {
    if (!quick) return x / d;
    const float q = x * y;
    return __builtin_fmaf(__builtin_fmaf(-q, d, x), y, q);
  }
};

// Four elements from `i` on; those at n and beyond are zero.
template <typename T>
__device__ __forceinline__ void adamw_load(float (&out)[4], const T* from, const int64_t i, const int64_t n, const bool vec) {
  typedef T vec_t __attribute__((ext_vector_type(4)));
  if (vec && i + 4 <= n) {
    const vec_t v = *reinterpret_cast<const vec_t*>(from + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = i + e < n ? (float)from[i + e] : 0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void adamw_store(T* to, const float (&in)[4], const int64_t i, const int64_t n, const bool vec) {
  typedef T vec_t __attribute__((ext_vector_type(4)));
  if (vec && i + 4 <= n) {
    vec_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (T)in[e];
    *reinterpret_cast<vec_t*>(to + i) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) to[i + e] = (T)in[e];
  }
}

__device__ __forceinline__ void adamw_element(const AdamwFactors& f, const float gs, float& p, const float grad, float& m, float& v) {
#pragma clang fp contract(off)
  const float g = grad * gs;
  m = m * f.b1 + g * f.a1;
  v = v * f.b2 + (g * f.a2) * g;
  p = p * f.keep - f.rate * (m / (sqrtf(v) * f.root + f.eps));
}

// P: type of the parameters, G: of the gradients, CP: of the copy (void: none), BITS: of the states.
template <typename P, typename G, typename CP, int BITS>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwFactors f, const AdamwTensors list) {
#pragma clang fp contract(off)
  // the tensor of this chunk: the last whose first chunk is not behind it
  int lo = 0, hi = list.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list.first[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const mdet_adamw_tensor t = list.t[lo];
  const int64_t n = t.n, base = (int64_t)(blockIdx.x - list.first[lo]) * list.chunk;
  P* const p = (P*)t.p;
  const G* const g = (const G*)t.g;
  const float gs = f.grad_scale ? *f.grad_scale : 1.0f;
  const bool pv = (uintptr_t)p % (4 * sizeof(P)) == 0, gv = (uintptr_t)g % (4 * sizeof(G)) == 0;
  static_assert(ADAMW_STEP == 4 * ADAMW_THREADS, "four elements a lane");
  for (int c = 0; c < list.chunk; c += ADAMW_STEP) {
    const int64_t i = base + c + 4 * (int)threadIdx.x;
    // in whole wavefronts: the lanes of a block find its scale together
    if (base + c + 4 * (int)(threadIdx.x & ~63u) >= n) return;
    float pe[4], ge[4], me[4], ve[4];
    adamw_load(pe, p, i, n, pv);
    adamw_load(ge, g, i, n, gv);
    if constexpr (BITS == 32) {
      float* const m = (float*)t.m;
      float* const v = (float*)t.v;
      const bool mv = (uintptr_t)m % 16 == 0, vv = (uintptr_t)v % 16 == 0;
      adamw_load(me, m, i, n, mv);
      adamw_load(ve, v, i, n, vv);
#pragma unroll
      for (int e = 0; e < 4; ++e) adamw_element(f, gs, pe[e], ge[e], me[e], ve[e]);
      adamw_store(m, me, i, n, mv);
      adamw_store(v, ve, i, n, vv);
    } else {
      int8_t* const m = (int8_t*)t.m;
      uint8_t* const v = (uint8_t*)t.v;
      const bool mv = (uintptr_t)m % 4 == 0, vv = (uintptr_t)v % 4 == 0;
      float* const scales = t.scales + 2 * (i / ADAMW_BLOCK);
      const float s1 = scales[0], s2 = scales[1];
      adamw_load(me, m, i, n, mv);
      adamw_load(ve, v, i, n, vv);
      uint32_t top1 = 0, top2 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        me[e] *= s1;
        ve[e] *= s2;
        ve[e] *= ve[e];
        adamw_element(f, gs, pe[e], ge[e], me[e], ve[e]);
        ve[e] = sqrtf(ve[e]);
        // as whole numbers the magnitudes are in order, NaN above infinity: neither is lost in a maximum
        const uint32_t a = i + e < n ? __float_as_uint(me[e]) & 0x7FFFFFFFu : 0u;
        const uint32_t b = i + e < n ? __float_as_uint(ve[e]) & 0x7FFFFFFFu : 0u;
        top1 = top1 > a ? top1 : a;
        top2 = top2 > b ? top2 : b;
      }
      const float n1 = __uint_as_float(wave_max(top1)) * (1.0f / 127.0f), n2 = __uint_as_float(wave_max(top2)) * (1.0f / 255.0f);
      // comparisons that a NaN fails: a block whose scale is zero or not finite has codes of zero
      const bool ok1 = n1 > 0.0f && n1 < INFINITY, ok2 = n2 > 0.0f && n2 < INFINITY;
      const BlockDivisor by1(n1), by2(n2);
      const uint32_t key = (uint32_t)(f.first_tensor + lo) * 0xA54FF53Bu + f.seed;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t bits = adamw_bits(key, i + e);
        const float x1 = floorf(by1(me[e]) + (float)(bits & 0xFFFFu) * (1.0f / 65536.0f));
        const float x2 = floorf(by2(ve[e]) + (float)(bits >> 16) * (1.0f / 65536.0f));
        const float least = ve[e] > 0.0f ? 1.0f : 0.0f;
        me[e] = ok1 ? fminf(fmaxf(x1, -127.0f), 127.0f) : 0.0f;
        ve[e] = ok2 ? fminf(fmaxf(x2, least), 255.0f) : 0.0f;
      }
      adamw_store(m, me, i, n, mv);
      adamw_store(v, ve, i, n, vv);
      if ((threadIdx.x & 63) == 0) {
        // infinity times a code of zero is NaN: a block that met one stays visible
        scales[0] = n1;
        scales[1] = n2;
      }
    }
    adamw_store(p, pe, i, n, pv);
    if constexpr (!__is_same(CP, void)) {
      CP* const copy = (CP*)t.copy;
      adamw_store(copy, pe, i, n, (uintptr_t)copy % (4 * sizeof(CP)) == 0);
    }
  }
}

}  // namespace mdet
