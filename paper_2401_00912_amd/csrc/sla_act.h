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

// log(1 + e^x) to 2^-21 of its value: the larger of x and 0, and log(1 + e) of e = e^-|x| in [0, 1] as
// 2 atanh(s), s = e / (2 + e) <= 1 / 3, by its power series (what is left out is 2^-26 of the sum at most).
// A logarithm of 1 + e would lose the bits of a small e: step sizes of 0.001 are usual.  The exponent in two
// terms, as above.
__device__ __forceinline__ float softplus(float x) {
  constexpr float kHi = -1.44269502f, kLo = -1.92596299e-8f;
  const float y = __builtin_elementwise_minimum(__builtin_fabsf(x), 128.f);
  const float t = y * kHi;
  const float r = __builtin_fmaf(y, kHi, -t) + y * kLo;
  float e = __builtin_amdgcn_exp2f(t);
  e = __builtin_fmaf(e, r * 0.693147181f, e);
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 1.f / 13.f;
  p = __builtin_fmaf(p, q, 1.f / 11.f);
  p = __builtin_fmaf(p, q, 1.f / 9.f);
  p = __builtin_fmaf(p, q, 1.f / 7.f);
  p = __builtin_fmaf(p, q, 1.f / 5.f);
  p = __builtin_fmaf(p, q, 1.f / 3.f);
  p = __builtin_fmaf(p, q, 1.f);
  return __builtin_fmaf(2.f * s, p, __builtin_elementwise_maximum(x, 0.f));
}

}  // namespace sla
