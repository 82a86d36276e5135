// Sums of exponentials against references in natural units, for the operators on given tokens and
// lists.  The difference to the reference is formed before it is scaled, so an entry at the
// reference has the exponent 0 whatever its size, and masked entries (-inf, the type's lowest value)
// end where the exponential is zero.  References are finite from below (kLowest).
#pragma once

#include "kl_pairs.cuh"

namespace adwin {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kNil = -150.f;   // 2^kNil is zero

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// exp(a - b) for a <= b
__device__ __forceinline__ float exp_below(float a, float b) { return ex2f((a - b) * kLog2e); }

template <int U>
__device__ __forceinline__ float group_max(const uint4 (&v)[U], __nv_bfloat16*) {
  __nv_bfloat162 m = __float2bfloat162_rn(-INFINITY);
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __hmax2(m, reinterpret_cast<const __nv_bfloat162&>(w[j]));
  }
  return fmaxf(__low2float(m), __high2float(m));
}
template <int U>
__device__ __forceinline__ float group_max(const uint4 (&v)[U], float*) {
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < U; ++k)
    m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(v[k].x)), fmaxf(__uint_as_float(v[k].y), __uint_as_float(v[k].z))),
              __uint_as_float(v[k].w));
  return m;
}

}  // namespace adwin
