// The running maximum of a softmax over scores of any size, as the attention kernels on packed tokens keep it.
//
// Exponents are of base 2: a score s has the exponent s * rc, rc = softmax_scale * log2(e).  The maximum m is kept as a score, in fp32 and exactly, and what is summed is
//   far   2^((s - m) * rc): the maximum's own exponent is 0, whatever its size;
//   near  2^(s * rc - r), r = m * rc rounded to fp32, for |r| <= kFar: one fused instruction an element instead of two.  The rounding of r is the same for all keys of a
//         row and cancels in the quotient; sums under two maxima meet with an error of half a step of r, 2^-13 of an exponent at most, which a score of that size
//         has from its own sum.  (Without the other form: from |r| = 2^31 on half a step takes the maximum out of fp32's exponents, and a row's sum to infinity or 0.)
// The kernels that are bound by the products take the near form, and the other one in a wave of which a row is far; the test is of a scalar, once a tile.
#pragma once
#include <hip/hip_runtime.h>

namespace bbm {

constexpr float kFar = 0x1p12f;
__device__ __forceinline__ bool is_far(float exponent) { return __builtin_fabsf(exponent) > kFar; }

// What sums under the maximum `from` (-infinity: of nothing) are worth under `to`, which is finite and no smaller.
__device__ __forceinline__ float weight(float from, float to, float rc) { return __builtin_amdgcn_exp2f((from - to) * rc); }

// Natural logarithm of what was summed under m.
__device__ __forceinline__ float log_sum(float m, float l, float rc) { return (m * rc + __log2f(l)) * 0.6931471805599453f; }

// The running maximum of a lane's row: m; nm, what is added to its exponents in the near form (0 if nothing was seen or the row is far); far, the wave's scalar.
struct RunningMax {
  float m = -INFINITY, nm = 0.0f;
  bool far = false;
  // What the far form takes off the row's scores (nothing of a near row, which has its nm).
  __device__ __forceinline__ float offset(float rc) const { return m != -INFINITY && is_far(m * rc) ? m : 0.0f; }
  // For scores up to mx: the maximum moves when a row of the wave exceeds its own by more than `lazy`; `rescale` gets the factor of what was summed so far.
  template <typename F>
  __device__ __forceinline__ void update(float mx, float lazy, float rc, F&& rescale) {
    if (__any(mx > m + lazy ? 1 : 0)) {
      const float m_new = fmaxf(m, mx), m_fin = m_new == -INFINITY ? 0.0f : m_new, r = m_fin * rc;
      rescale(weight(m, m_fin, rc));
      m = m_new;
      nm = is_far(r) ? 0.0f : -r;
      far = __any(is_far(r) ? 1 : 0) != 0;
    }
  }
};

}  // namespace bbm
