// Square root and quotient of the update (kernels_adamw.hip), in the bits of the correctly rounded operations for operands of moderate size: the compiler's own
// forms spend half their instructions on operands that are very large, very small or 0.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace echo {

// Magnitudes from 2^-80 to below 2^80: nothing below leaves the normal numbers, nor does a quotient by something as small as the root of the least.  0 is not
// among them.
constexpr uint32_t MODERATE_LOW = (uint32_t)(127 - 80) << 24, MODERATE_SPAN = (uint32_t)160 << 24;
// How far a magnitude lies beyond the least moderate one; as a whole number without sign, at least MODERATE_SPAN for all that are not moderate.
__device__ __forceinline__ uint32_t beyond_moderate(float x) { return (__float_as_uint(x) << 1) - MODERATE_LOW; }

// A Newton step on v_rsq_f32's estimate: r near x^-1/2, s = x r, then s + (x - s^2) r / 2 with the residual exact (Markstein, IBM J. Res. Dev. 34, 1990).  Right for every
// significand and both parities of the exponent (tests/update_sweep.hip), hence, scaling by powers of 4, for every moderate x.
__device__ __forceinline__ float moderate_sqrt(float x) {
#pragma clang fp contract(off)
  const float r = __builtin_amdgcn_rsqf(x), s = x * r;
  return fmaf(fmaf(-s, s, x), 0.5f * r, s);
}
// A Newton step on v_rcp_f32's estimate gives the correctly rounded reciprocal (every significand: tests/update_sweep.hip); with it one correction of n r by its
// exact residual is the correctly rounded quotient (Markstein, as above).
__device__ __forceinline__ float moderate_reciprocal(float d) {
#pragma clang fp contract(off)
  const float r = __builtin_amdgcn_rcpf(d);
  return fmaf(fmaf(-d, r, 1.0f), r, r);
}
__device__ __forceinline__ float moderate_quotient(float n, float d) {
#pragma clang fp contract(off)
  const float r = moderate_reciprocal(d), q = n * r;
  return fmaf(fmaf(-d, q, n), r, q);
}

}  // namespace echo
