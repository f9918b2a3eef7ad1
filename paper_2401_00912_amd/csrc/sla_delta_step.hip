// The gated delta rule one row at a time, for answering: the states of many sequences lie in a
// pool, every row of the batch names its sequence's slot, and the state is updated where it lies.
//
//     S' = exp(g) S,  u = beta (v - S'^T k),  S <- S' + k u^T,  o = scale (S'^T q + (q . k) u)
//
// Bound by memory: the state (64 KB a head at 128 x 128) is read and written once, all else is a
// few rows.  A workgroup takes 32 columns of one head's state, 8 lanes of 4 columns by 32 groups of
// state rows, all of it in registers between its load and its store; S'^T k and S'^T q are summed
// in the same pass, so the row groups meet once.  256 rows, 16 heads of 128 x 128: 537 MB in 122 to
// 130 us, 4.1 to 4.4 TB/s (a copy reaches 5.2); one row, 4 heads of 64: 4.6 us, which is a launch and
// three dependent loads.
#include "sla_delta.h"

namespace sla {
namespace {

using namespace delta;

constexpr int kCols = 32, kRowGroups = 32;

struct StepArgs {
  const int32_t* slots;
  int32_t n, num_slots, Hk, H, dk, dv;
  float scale;
};

// Rows per thread DK / 32.  Rows of the batch with the same slot are one sequence's rows: the
// workgroup of the first one takes them all, in row order, and the others leave.
template <typename T, int DK>
__global__ __launch_bounds__(256) void k_delta_step(StepArgs a, float* __restrict__ state, const T* __restrict__ q,
                                                    const T* __restrict__ k, const T* __restrict__ v,
                                                    const float* __restrict__ gin, const float* __restrict__ beta,
                                                    T* __restrict__ o) {
  constexpr int NR = DK / kRowGroups;
  __shared__ floatx4 s_part[2][4][8];
  __shared__ float s_qk[4];
  __shared__ int s_next[4], s_seen[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quad = tid & 7, rg = tid >> 3;
  const int h = blockIdx.y, hk = h / (a.H / a.Hk);
  const int col = blockIdx.z * kCols + 4 * quad;
  const bool live = col < a.dv;
  int b = blockIdx.x;
  const int slot = a.slots[b];
  if (slot < 0 || slot >= a.num_slots) return;   // padding: nothing is touched

  float* st = state + (((size_t)slot * a.H + h) * a.dk) * a.dv + col;
  floatx4 S[NR];
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int d = rg + kRowGroups * j;
    S[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (live && d < a.dk) S[j] = *reinterpret_cast<const floatx4*>(st + (size_t)d * a.dv);
  }
  for (bool first = true; b < a.n; first = false) {
    // the next row of this slot, and (once) whether an earlier one has it
    int next = a.n, seen = 0;
    for (int x = first ? tid : b + 1 + tid; x < a.n; x += 256)
      if (a.slots[x] == slot) {
        if (x < b) seen = 1;
        if (x > b && x < next) next = x;
      }
    const T* qr = q + ((size_t)b * a.Hk + hk) * a.dk;
    const T* kr = k + ((size_t)b * a.Hk + hk) * a.dk;
    const size_t at = (size_t)b * a.H + h;
    const float decay = expf(gin[at]), be = beta[at];
    float qv[NR], kv[NR];
    floatx4 sk = {0.f, 0.f, 0.f, 0.f}, sq = {0.f, 0.f, 0.f, 0.f};
    float qk = 0.f;
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      const int d = rg + kRowGroups * j;
      qv[j] = d < a.dk ? load1(qr + d) : 0.f;
      kv[j] = d < a.dk ? load1(kr + d) : 0.f;
      qk += qv[j] * kv[j];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        S[j][r] *= decay;
        sk[r] += kv[j] * S[j][r];
        sq[r] += qv[j] * S[j][r];
      }
    }
    // the eight row groups of a wave, then the four waves
#pragma unroll
    for (int m = 8; m < 64; m *= 2) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sk[r] += __shfl_xor(sk[r], m);
        sq[r] += __shfl_xor(sq[r], m);
      }
      qk += __shfl_xor(qk, m);
    }
    const uint64_t sb = __ballot(seen);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int y = __shfl_xor(next, m);
      next = y < next ? y : next;
    }
    if (lane < 8) {
      s_part[0][wave][lane] = sk;
      s_part[1][wave][lane] = sq;
    }
    if (lane == 0) {
      s_qk[wave] = qk;
      s_next[wave] = next;
      s_seen[wave] = sb != 0;
    }
    __syncthreads();
    if (first && (s_seen[0] | s_seen[1] | s_seen[2] | s_seen[3])) return;
    next = min(min(s_next[0], s_next[1]), min(s_next[2], s_next[3]));
    qk = (s_qk[0] + s_qk[1]) + (s_qk[2] + s_qk[3]);
    sk = (s_part[0][0][quad] + s_part[0][1][quad]) + (s_part[0][2][quad] + s_part[0][3][quad]);
    sq = (s_part[1][0][quad] + s_part[1][1][quad]) + (s_part[1][2][quad] + s_part[1][3][quad]);
    floatx4 u = {0.f, 0.f, 0.f, 0.f}, out;
    if (live) {
#pragma unroll
      for (int r = 0; r < 4; ++r) u[r] = be * (load1(v + at * a.dv + col + r) - sk[r]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = a.scale * (sq[r] + qk * u[r]);
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[j][r] += kv[j] * u[r];
    if (live && rg == 0) store4(o + at * a.dv + col, out);
    b = next;
    if (b < a.n) __syncthreads();   // the exchange is written again
  }
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int d = rg + kRowGroups * j;
    if (live && d < a.dk) *reinterpret_cast<floatx4*>(st + (size_t)d * a.dv) = S[j];
  }
}

template <typename T>
void step_impl(const StepArgs& a, float* state, const void* q, const void* k, const void* v, const float* g,
               const float* beta, void* o, hipStream_t stream) {
  const dim3 grid(a.n, a.H, (a.dv + kCols - 1) / kCols);
  const auto run = [&](auto kernel) {
    kernel<<<grid, 256, 0, stream>>>(a, state, static_cast<const T*>(q), static_cast<const T*>(k),
                                     static_cast<const T*>(v), g, beta, static_cast<T*>(o));
  };
  switch (pad_dk(a.dk)) {
    case 32: run(k_delta_step<T, 32>); break;
    case 64: run(k_delta_step<T, 64>); break;
    default: run(k_delta_step<T, 128>); break;
  }
}

}  // namespace

hipError_t launch_step_delta(const int32_t* slots, int32_t n, int32_t num_slots, int dtype, int32_t Hk, int32_t H,
                             int32_t dk, int32_t dv, float scale, float* state, const void* q, const void* k,
                             const void* v, const float* g, const float* beta, void* o, hipStream_t stream) {
  const StepArgs a{slots, n, num_slots, Hk, H, dk, dv, scale};
  if (dtype == 0) step_impl<float>(a, state, q, k, v, g, beta, o, stream);
  else if (dtype == 1) step_impl<_Float16>(a, state, q, k, v, g, beta, o, stream);
  else step_impl<bf16_t>(a, state, q, k, v, g, beta, o, stream);
  return hipGetLastError();
}

}  // namespace sla
