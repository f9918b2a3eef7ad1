// What the selective scan's kernels share.  For channel d with N states, of the rows t of a window,
//     dt_t = softplus(delta_t + bias) (or without the softplus),  u_t = dt_t x_t,
//     h_t[n] = exp(dt_t A[d][n]) h_{t-1}[n] + u_t B_t[n],
//     y_t = (sum_n C_t[n] h_t[n] + skip x_t) silu(z_t).
// A wave takes 64 channels of one group (the channels that share B and C), a lane a channel: h is in
// registers, and what all lanes share, the rows' B and C, comes from LDS as a broadcast into vector registers
// too: an instruction whose operands are all there takes 2.4 cycles with two waves or more on a SIMD, one
// with a scalar operand 4.2 (measured; an exponential 8.2).
//
// Windows are cut into parts of at most `per` rows that waves walk at the same time.  What a part hands on is
// a linear map of what it is given, h -> exp(A sum dt) h + S: a first launch makes S and sum dt of each part
// (from h = 0), a second joins them along each window, a third walks again, each part from its own h.
#pragma once
#include "sla_act.h"
#include "sla_rows.h"

namespace sla {
namespace scan {

constexpr float kLog2e = 1.44269504f;

struct ScanArgs {
  Windows win;
  const float *A, *skip, *bias;
  int64_t ldx, ldd, ldz, ldb, ldc, ldy;
  int32_t D, G, N;
  int32_t cg, tpg;    // channels and waves of a group
  int32_t per;        // rows of a part
  int32_t softplus;
};

// A wave's channels.
struct Tile {
  int g, c;     // group; channel of the lane (where there is none: the group's first)
  bool live;
  __device__ __forceinline__ Tile(const ScanArgs& a, int tile, int lane) {
    g = tile / a.tpg;
    const int at = (tile % a.tpg) * 64 + lane;
    live = at < a.cg;
    c = g * a.cg + (live ? at : 0);
  }
};

__device__ __forceinline__ float step_size(const ScanArgs& a, float delta, float bias) {
  const float x = delta + bias;
  return a.softplus ? softplus(x) : x;
}

// A as the exponent of two; finite, so that a step of 0 keeps the state whatever A is.
__device__ __forceinline__ float exponent(float A) {
  return __builtin_elementwise_minimum(__builtin_elementwise_maximum(A * kLog2e, -3e38f), 3e38f);
}

// NS >= N values of a channel from [N] consecutive floats; fill beyond
template <int NS>
__device__ __forceinline__ void load_states(const float* p, int N, bool vec, float (&x)[NS]) {
  if constexpr (NS % 4 == 0) {
    if (vec) {
#pragma unroll
      for (int n = 0; n < NS; n += 4) {
        const floatx4 q = n < N ? *reinterpret_cast<const floatx4*>(p + n) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 4; ++r) x[n + r] = q[r];
      }
      return;
    }
  }
#pragma unroll
  for (int n = 0; n < NS; ++n) x[n] = n < N ? p[n] : 0.f;
}
template <int NS>
__device__ __forceinline__ void store_states(float* p, int N, bool vec, const float (&x)[NS]) {
  if constexpr (NS % 4 == 0) {
    if (vec) {
#pragma unroll
      for (int n = 0; n < NS; n += 4)
        if (n < N) *reinterpret_cast<floatx4*>(p + n) = floatx4{x[n], x[n + 1], x[n + 2], x[n + 3]};
      return;
    }
  }
#pragma unroll
  for (int n = 0; n < NS; ++n)
    if (n < N) p[n] = x[n];
}
// whether a channel's N floats may be moved four at a time
__device__ __forceinline__ bool by_four(const float* p, int N) {
  return N % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

// exp(x) h where exp(x) alone may be none: in two halves, and 0 stays 0.
__device__ __forceinline__ float decayed(float x_log2, float h) {
  const float e = __builtin_amdgcn_exp2f(0.5f * x_log2);
  return h == 0.f ? 0.f : e * (e * h);
}

// Rows of a part, and the parts' results: S [slots][N][D] and sum dt [slots][D], then in place of S the state
// behind the part.
struct Parts {
  float *S, *dts;
};

// the states that a lane is built for
inline int padded_states(int N) { return N <= 1 ? 1 : N <= 4 ? 4 : N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }
template <class F>
void by_states(int N, F f) {
  switch (padded_states(N)) {
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    case 8: f(std::integral_constant<int, 8>{}); break;
    case 16: f(std::integral_constant<int, 16>{}); break;
    case 32: f(std::integral_constant<int, 32>{}); break;
    default: f(std::integral_constant<int, 64>{}); break;
  }
}

// Workgroups across the states of a window where its parts are joined: one value a thread for few windows,
// where that is latency; several for many, most of which have one part and nothing to do.
inline uint32_t carry_blocks(const ScanArgs& a) {
  const int64_t all = ((int64_t)a.N * a.D + 255) / 256;
  const int64_t some = 4096 / a.win.W;
  return (uint32_t)(all < some ? all : some < 1 ? 1 : some);
}

inline int64_t slots_of(const ScanArgs& a) { return (int64_t)a.win.n / a.per + a.win.W; }

}  // namespace scan
}  // namespace sla
