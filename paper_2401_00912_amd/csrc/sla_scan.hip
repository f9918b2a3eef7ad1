// The selective scan over the rows of every window (the recurrence and how it is cut: sla_scan.h).
//
// Bound by the vector unit: a state and row take a product, an exponential, a product and two multiply-adds;
// the memory's part (x, delta, z in, y out) is less than half of that at 16 states.
#include "sla_scan.h"

namespace sla {
namespace {

using namespace scan;

// Rows a wave loads at once: the next ones are on their way while these are computed.
template <int NS>
constexpr int kRows = NS <= 16 ? 8 : 4;

// OUT: the walk that makes y; else the one that makes a part's map.
template <typename T, int NS, bool OUT>
__global__ __launch_bounds__(64) void k_scan(ScanArgs a, const T* __restrict__ x, const T* __restrict__ delta,
                                             const T* __restrict__ z, const T* __restrict__ B, const T* __restrict__ C,
                                             const float* __restrict__ state, T* __restrict__ y,
                                             float* __restrict__ state_out, Parts parts) {
  constexpr int U = kRows<NS>, V = OUT ? 2 * NS : NS, J = (U * V + 63) / 64;
  __shared__ __attribute__((aligned(16))) float s_bc[J * 64];
  Part part;
  if (!part_of(a.win, a.per, blockIdx.x, part)) return;
  if (!OUT && part.last) return;   // nothing follows
  const int lane = threadIdx.x;
  const Tile tile(a, blockIdx.y, lane);
  const int c = tile.c;

  float A[NS], h[NS];
  load_states<NS>(a.A + (size_t)c * a.N, a.N, by_four(a.A, a.N), A);
#pragma unroll
  for (int n = 0; n < NS; ++n) A[n] *= kLog2e;
  if (OUT && !part.first) {
    const float* p = parts.S + (size_t)(blockIdx.x - 1) * a.N * a.D + c;
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = n < a.N ? p[(size_t)n * a.D] : 0.f;
  } else if (OUT && state != nullptr && !part.last) {
    // from the copy beside the parts: state_out may be state, and another wave writes it
    const int count = (a.win.edge(part.w + 1) - part.begin - 1) / a.per;
    const float* p = parts.S + (size_t)(blockIdx.x + count) * a.N * a.D + c;
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = n < a.N ? p[(size_t)n * a.D] : 0.f;
  } else if (OUT && state != nullptr) {
    load_states<NS>(state + ((size_t)part.w * a.D + c) * a.N, a.N, by_four(state, a.N), h);
  } else {
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = 0.f;
  }
  const float bias = a.bias ? a.bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;
  float dts = 0.f;

  T xr[U], dr[U], zr[U], bc[J];
  const auto ask = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int r = p0 + i < part.end ? a.win.row(p0 + i) : -1;
      xr[i] = dr[i] = zr[i] = from_float<T>(0.f);
      if (r >= 0) {
        xr[i] = x[r * a.ldx + c];
        dr[i] = delta[r * a.ldd + c];
        if (OUT && z != nullptr) zr[i] = z[r * a.ldz + c];
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int at = lane + 64 * j, p = p0 + at / V, v = at % V, n = v % NS;
      bc[j] = from_float<T>(0.f);
      const int r = p < part.end && at < U * V && n < a.N ? a.win.row(p) : -1;
      if (r >= 0) bc[j] = v < NS ? B[r * a.ldb + tile.g * a.N + n] : C[r * a.ldc + tile.g * a.N + n];
    }
  };
  ask(part.begin);
  for (int p0 = part.begin; p0 < part.end; p0 += U) {
    T xc[U], dc[U], zc[U];
#pragma unroll
    for (int i = 0; i < U; ++i) xc[i] = xr[i], dc[i] = dr[i], zc[i] = zr[i];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < J; ++j) s_bc[lane + 64 * j] = to_float(bc[j]);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    ask(p0 + U);
    const auto row = [&](int i) __attribute__((always_inline)) {
      const float xv = to_float(xc[i]), dt = step_size(a, to_float(dc[i]), bias), u = dt * xv;
      float sum[4] = {};
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const float e = __builtin_amdgcn_exp2f(dt * A[n]);
        h[n] = __builtin_fmaf(e, h[n], u * s_bc[i * V + n]);
        if (OUT) sum[n % 4] = __builtin_fmaf(s_bc[i * V + NS + n], h[n], sum[n % 4]);
      }
      if (!OUT) {
        dts += dt;
        return;
      }
      float out = __builtin_fmaf(skip, xv, (sum[0] + sum[1]) + (sum[2] + sum[3]));
      if (z != nullptr) out *= act(kSilu, to_float(zc[i]));
      const int r = a.win.row(p0 + i);
      if (tile.live && r >= 0) y[(size_t)r * a.D + c] = from_float<T>(out);
    };
    if (p0 + U <= part.end) {
#pragma unroll
      for (int i = 0; i < U; ++i) row(i);
    } else {
#pragma unroll
      for (int i = 0; i < U - 1; ++i)
        if (p0 + i < part.end) row(i);
    }
  }
  if (!tile.live) return;
  if (OUT) {
    if (part.last && state_out != nullptr)
      store_states<NS>(state_out + ((size_t)part.w * a.D + c) * a.N, a.N, by_four(state_out, a.N), h);
  } else {
    float* p = parts.S + (size_t)blockIdx.x * a.N * a.D + c;
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n < a.N) p[(size_t)n * a.D] = h[n];
    parts.dts[(size_t)blockIdx.x * a.D + c] = dts;
  }
}

// Along the parts of every window: S becomes the state behind its part.  Windows without rows hand their
// state on.
__global__ __launch_bounds__(256) void k_scan_carry(ScanArgs a, const float* __restrict__ state,
                                                    float* __restrict__ state_out, Parts parts) {
  constexpr int kAhead = 8;
  const int w = blockIdx.x;
  const int b = a.win.edge(w), e = a.win.edge(w + 1);
  const int64_t at = (int64_t)blockIdx.y * 256 + threadIdx.x, size = (int64_t)a.N * a.D;
  if (at >= size) return;
  const int n = (int)(at / a.D), c = (int)(at % a.D);
  if (e <= b) {
    if (state_out != nullptr) {
      const size_t i = ((size_t)w * a.D + c) * a.N + n;
      state_out[i] = state != nullptr ? state[i] : 0.f;
    }
    return;
  }
  const int count = (e - b - 1) / a.per;   // parts but the last
  if (count == 0) return;
  const int64_t first = (int64_t)(b / a.per) + w;
  const float A = a.A[(size_t)c * a.N + n] * kLog2e;
  float h = state != nullptr ? state[((size_t)w * a.D + c) * a.N + n] : 0.f;
  parts.S[(first + count) * size + at] = h;   // the last part's place is free: a copy for the first part
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    float S[kAhead], d[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t s = first + min(i0 + i, count - 1);
      S[i] = parts.S[s * size + at];
      d[i] = parts.dts[s * a.D + c];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < count) {
        h = decayed(A * d[i], h) + S[i];
        parts.S[(first + i0 + i) * size + at] = h;
      }
  }
}

// Rows of a part: waves for all SIMDs, but parts long enough that joining them costs little.
int rows_per_part(int64_t n, int32_t W, int64_t tiles) {
  int64_t per = n * tiles / 4096 / 8 * 8;
  per = per < 64 ? 64 : per > 512 ? 512 : per;
  return (int)per;
}

int64_t tiles_of(int32_t D, int32_t G) { return (int64_t)G * ((D / G + 63) / 64); }

}  // namespace

size_t scan_workspace_bytes(int64_t n, int32_t W, int32_t D, int32_t G, int32_t N) {
  const int64_t slots = n / rows_per_part(n, W, tiles_of(D, G)) + W;
  return align_up((size_t)slots * D * N * 4, 256) + align_up((size_t)slots * D * 4, 256);
}

hipError_t launch_forward_scan(scan::ScanArgs a, int dtype, const void* x, const void* delta, const void* z, const void* B,
                               const void* C, const float* state_in, void* y, float* state_out, void* workspace,
                               hipStream_t stream) {
  a.cg = a.D / a.G;
  a.tpg = (a.cg + 63) / 64;
  const int64_t tiles = tiles_of(a.D, a.G);
  a.per = rows_per_part(a.win.n, a.win.W, tiles);
  const int64_t slots = slots_of(a);
  Parts parts;
  parts.S = static_cast<float*>(workspace);
  parts.dts = parts.S + align_up((size_t)slots * a.D * a.N * 4, 256) / 4;
  const dim3 grid((uint32_t)slots, (uint32_t)tiles);
  const auto run = [&](auto type) {
    using T = decltype(type);
    by_states(a.N, [&](auto ns) {
      constexpr int NS = decltype(ns)::value;
      const auto args = [&](auto kernel) {
        kernel<<<grid, 64, 0, stream>>>(a, static_cast<const T*>(x), static_cast<const T*>(delta),
                                        static_cast<const T*>(z), static_cast<const T*>(B), static_cast<const T*>(C),
                                        state_in, static_cast<T*>(y), state_out, parts);
      };
      const bool cut = a.win.n > a.per;
      if (cut) args(k_scan<T, NS, false>);
      if (cut || state_out != nullptr)
        k_scan_carry<<<dim3(a.win.W, (uint32_t)(((int64_t)a.N * a.D + 255) / 256)), 256, 0, stream>>>(a, state_in,
                                                                                                     state_out, parts);
      if (a.win.n > 0) args(k_scan<T, NS, true>);
    });
  };
  if (dtype == 0) run(float{});
  else if (dtype == 1) run(_Float16{});
  else run(bf16_t{});
  return hipGetLastError();
}

}  // namespace sla
