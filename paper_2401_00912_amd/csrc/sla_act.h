// Activations of the row operators and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

namespace sla {

enum Act { kNone = 0, kRelu = 1, kSilu = 2 };

// 1 / (1 + e^-z) for -87 <= z <= 87 from the hardware's 2^x and 1 / x (each within one step): -z log2 e in two
// terms, so that a large exponent loses nothing.  With expf and a division the activation took more time than
// the memory (240,011 x 256 bf16 values: 56 us, 47 for the bytes).
__device__ __forceinline__ float sigmoid(float z) {
  constexpr float kHi = -1.44269502f, kLo = -1.92596299e-8f;   // -log2 e
  const float t = z * kHi;
  const float r = __builtin_fmaf(z, kHi, -t) + z * kLo;
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, r * 0.693147181f, e));
}
// z between its bounds; a NaN stays one.  silu and its slope take the bounded z as their factor too: what the
// sigmoid ends at below, 1.6e-38, is none for a z of -1e38.
__device__ __forceinline__ float from_below(float z) { return __builtin_elementwise_maximum(z, -87.f); }
__device__ __forceinline__ float from_above(float z) { return __builtin_elementwise_minimum(z, 87.f); }
__device__ __forceinline__ float act(int a, float z) {
  if (a == kRelu) return z > 0.f ? z : (z != z ? z : 0.f);
  if (a == kSilu) {
    z = from_below(z);
    return z * sigmoid(from_above(z));
  }
  return z;
}
__device__ __forceinline__ float slope(int a, float z) {
  if (a == kRelu) return z > 0.f ? 1.f : 0.f;
  if (a == kSilu) {
    z = from_above(from_below(z));
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

// z / (1 + e^-z) and log(1 + e^x) where they are a small part of the work of every row, with the exponent in one
// term: e^-|x| is off by |x| 2^-23 of itself, which is what the values below 0 are off by.
__device__ __forceinline__ float quick_sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}
__device__ __forceinline__ float quick_silu(float z) {
  z = from_below(z);
  return z * quick_sigmoid(z);
}
__device__ __forceinline__ float quick_silu_slope(float z) {
  z = from_above(from_below(z));
  const float s = quick_sigmoid(z);
  return s * __builtin_fmaf(z, 1.f - s, 1.f);
}
// Of a vector, one branch for all values.
template <int N>
__device__ __forceinline__ void act_all(int a, float (&z)[N]) {
  if (a == kSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = quick_silu(z[e]);
  } else if (a == kRelu) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = act(kRelu, z[e]);
  }
}
// d times the slope at z
template <int N>
__device__ __forceinline__ void slope_all(int a, const float (&z)[N], float (&d)[N]) {
  if (a == kSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] *= quick_silu_slope(z[e]);
  } else if (a == kRelu) {
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = z[e] > 0.f ? d[e] : 0.f;
  }
}
// The larger of x and 0, and log(1 + e) of e = e^-|x| in [0, 1] as 2 atanh(s), s = e / (2 + e) <= 1 / 3, with atanh(s)
// / s a polynomial in s^2 through the Chebyshev points of [0, 1 / 9] (off by 2^-26).  A logarithm of 1 + e would lose
// the bits of a small e: step sizes of 0.001 are usual.
__device__ __forceinline__ float softplus(float x) {
  const float e = __builtin_amdgcn_exp2f(-1.44269504f * __builtin_fabsf(x));
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 0.1407889f;
  p = __builtin_fmaf(p, q, 0.13982579f);
  p = __builtin_fmaf(p, q, 0.20012298f);
  p = __builtin_fmaf(p, q, 0.3333316f);
  p = __builtin_fmaf(p, q, 1.f);
  return __builtin_fmaf(2.f * s, p, __builtin_elementwise_maximum(x, 0.f));
}

}  // namespace sla
