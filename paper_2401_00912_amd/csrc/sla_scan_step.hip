// The selective scan one row at a time, on a pool of states (the recurrence: sla_scan.h).
//
// Bound by memory: a state is read and written once where it lies, four values a lane; a channel's states are
// in neighbouring lanes, which share its row and add up its y.  256 bf16 rows of 4,096 channels and 16 states: 143 MB
// in 35 us, 4.1 TB/s; one row of 1,024 channels: 4.7 us, a launch and a chain of loads.
#include "sla_scan.h"

namespace sla {
namespace {

using namespace scan;

constexpr int kThreads = 256;

// Four states' B or C of a row, in one load where they lie so; 0 past the last.
template <typename T>
__device__ __forceinline__ void load_shared(const T* p, int count, bool vec, float (&v)[4]) {
  if (vec) {
    if (count > 0) {
      Vec<T, 4>::wide(Vec<T, 4>::load(p), v);
      return;
    }
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) v[n] = n < count ? to_float(p[n]) : 0.f;
}
template <typename T>
__device__ __forceinline__ bool shared_by_four(const T* p, int64_t ld, int N) {
  return N % 4 == 0 && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0;
}

// LN: lanes of a channel, 4 LN >= N.  CH: channels of a lane, of one group, whose states are on their way together.
template <typename T, int LN, int CH>
__global__ __launch_bounds__(kThreads) void k_scan_step(ScanArgs a, const int32_t* __restrict__ slots, int32_t num_slots,
                                                        float* __restrict__ state, const T* __restrict__ x,
                                                        const T* __restrict__ delta, const T* __restrict__ z,
                                                        const T* __restrict__ B, const T* __restrict__ C,
                                                        T* __restrict__ y) {
  constexpr int kWide = kThreads / LN;   // channels side by side
  __shared__ int s_table[2 * (kThreads / 64)];
  int b = blockIdx.x;
  const int slot = slots[b];
  if (slot < 0 || slot >= num_slots) return;   // padding: nothing is touched
  const SlotRows<kThreads / 64> rows{slots, a.win.n, s_table};
  const int k = threadIdx.x % LN, n0 = 4 * k, count = a.N - n0;
  const bool vec = by_four(state, a.N), vecA = by_four(a.A, a.N), vecB = shared_by_four(B, a.ldb, a.N),
             vecC = shared_by_four(C, a.ldc, a.N);
  float A[CH][4], h[CH][4], bias[CH], skip[CH];
  int c[CH];
  bool live[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int at = (blockIdx.y * CH + i) * kWide + threadIdx.x / LN;
    live[i] = at < a.D;
    c[i] = live[i] ? at : 0;
    load_states<4>(state + ((size_t)slot * a.D + c[i]) * a.N + n0, count, vec, h[i]);
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    load_states<4>(a.A + (size_t)c[i] * a.N + n0, count, vecA, A[i]);
#pragma unroll
    for (int n = 0; n < 4; ++n) A[i][n] = exponent(A[i][n]);
    bias[i] = a.bias ? a.bias[c[i]] : 0.f;
    skip[i] = a.skip ? a.skip[c[i]] : 0.f;
  }
  const int g = c[0] / a.cg;
  for (bool first = true;; first = false) {
    float Bv[4], Cv[4], dl[CH], xv[CH], zv[CH], sum[CH] = {};
    load_shared(B + b * a.ldb + g * a.N + n0, count, vecB, Bv);
    load_shared(C + b * a.ldc + g * a.N + n0, count, vecC, Cv);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      xv[i] = to_float(x[b * a.ldx + c[i]]);
      dl[i] = to_float(delta[b * a.ldd + c[i]]);
      zv[i] = z != nullptr ? to_float(z[b * a.ldz + c[i]]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float dt = step_size(a, dl[i], bias[i]), u = dt * xv[i];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        h[i][n] = __builtin_fmaf(__builtin_amdgcn_exp2f(dt * A[i][n]), h[i][n], u * Bv[n]);
        sum[i] = __builtin_fmaf(Cv[n], h[i][n], sum[i]);
      }
    }
    const int next = rows.next(b, slot, first);
    if (next < 0) return;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
#pragma unroll
      for (int m = 1; m < LN; m *= 2) sum[i] += __shfl_xor(sum[i], m);
      const float gate = z != nullptr ? quick_silu(zv[i]) : 1.f;
      if (live[i] && k == 0) y[(size_t)b * a.D + c[i]] = from_float<T>(__builtin_fmaf(skip[i], xv[i], sum[i]) * gate);
    }
    if (next >= a.win.n) break;
    b = next;
  }
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (live[i]) store_states<4>(state + ((size_t)slot * a.D + c[i]) * a.N + n0, count, vec, h[i]);
}

template <typename T>
void step_impl(const ScanArgs& a, const int32_t* slots, int32_t num_slots, float* state, const void* x,
               const void* delta, const void* z, const void* B, const void* C, void* y, hipStream_t stream) {
  const auto run = [&](auto lanes) {
    constexpr int LN = decltype(lanes)::value;
    const auto go = [&](auto channels) {
      constexpr int CH = decltype(channels)::value, kAcross = kThreads / LN * CH;
      const dim3 grid(a.win.n, (a.D + kAcross - 1) / kAcross);
      k_scan_step<T, LN, CH><<<grid, kThreads, 0, stream>>>(a, slots, num_slots, state, static_cast<const T*>(x),
                                                            static_cast<const T*>(delta), static_cast<const T*>(z),
                                                            static_cast<const T*>(B), static_cast<const T*>(C),
                                                            static_cast<T*>(y));
    };
    // two channels a lane where there are workgroups enough (4,096 channels of 16 states: 64 rows 10.5 us against
    // 11.6 with one, 256 rows 36.6 against 41.7; below, one: each workgroup's chain of loads is what it takes)
    if (a.G == 1 && (int64_t)a.win.n * a.D * LN >= 1 << 20) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 1>{});
  };
  if (a.N <= 4) run(std::integral_constant<int, 1>{});
  else if (a.N <= 8) run(std::integral_constant<int, 2>{});
  else if (a.N <= 16) run(std::integral_constant<int, 4>{});
  else if (a.N <= 32) run(std::integral_constant<int, 8>{});
  else run(std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t launch_step_scan(scan::ScanArgs a, int dtype, const int32_t* slots, int32_t num_slots, float* state,
                            const void* x, const void* delta, const void* z, const void* B, const void* C, void* y,
                            hipStream_t stream) {
  a.cg = a.D / a.G;
  if (dtype == 0) step_impl<float>(a, slots, num_slots, state, x, delta, z, B, C, y, stream);
  else if (dtype == 1) step_impl<_Float16>(a, slots, num_slots, state, x, delta, z, B, C, y, stream);
  else step_impl<bf16_t>(a, slots, num_slots, state, x, delta, z, B, C, y, stream);
  return hipGetLastError();
}

}  // namespace sla
