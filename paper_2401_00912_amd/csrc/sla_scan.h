// What the selective scan's kernels share.  For channel d with N states, of the rows t of a window,
//     dt_t = softplus(delta_t + bias) (or without the softplus),  u_t = dt_t x_t,
//     h_t[n] = exp(dt_t A[d][n]) h_{t-1}[n] + u_t B_t[n],
//     y_t = (sum_n C_t[n] h_t[n] + skip x_t) silu(z_t).
// A wave takes 64 channels of one group (the channels that share B and C), a lane a channel: h is in
// registers, and the only thing lanes share, the rows' B and C, comes from LDS as a broadcast.
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

template <class F>
void by_states(int N, F f) {
  if (N <= 1) f(std::integral_constant<int, 1>{});
  else if (N <= 4) f(std::integral_constant<int, 4>{});
  else if (N <= 8) f(std::integral_constant<int, 8>{});
  else if (N <= 16) f(std::integral_constant<int, 16>{});
  else if (N <= 32) f(std::integral_constant<int, 32>{});
  else f(std::integral_constant<int, 64>{});
}

inline int64_t slots_of(const ScanArgs& a) { return (int64_t)a.win.n / a.per + a.win.W; }

}  // namespace scan
}  // namespace sla
