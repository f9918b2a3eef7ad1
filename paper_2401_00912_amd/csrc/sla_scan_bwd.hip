// Gradients of the selective scan (the recurrence and how windows are cut: sla_scan.h).
//
// With g_t = dy_t silu(z_t), a_t = exp(dt_t A) h_{t-1}, so h_t = a_t + u_t B_t, and q_t the gradient of h_t, from
// a window's last row to its first:
//     q_t = C_t g_t + exp(dt_{t+1} A) q_{t+1},
//     dC_t = sum_d h_t g_t,  dB_t = sum_d q_t u_t,  du_t = sum_n q_t B_t,  dx_t = dt_t du_t + skip g_t,
//     ddt_t = x_t du_t + sum_n A q_t a_t,  dA = sum_t dt_t q_t a_t,
// ddelta = ddt softplus'(delta + bias), dz = dy (y before the gate) silu'(z), and the parameters' sums over rows.
//
// Four launches.  The first makes the maps of a window's parts, forward (S, sum dt) and back: what a part adds
// to the gradient of the state before it, R = sum_t exp(A sum_{s <= t} dt_s) C_t g_t.  The second joins them along
// the window both ways.  The third walks every part: forward once for the states at its tiles, then
// tile by tile from the last, forward through the tile with every row's a and decay kept in registers, and
// back.  A lane holds four states of a channel, so the sums over states go over the lane's few neighbours and
// those over channels over the wave, then over the workgroup's waves in LDS, and what is left of them (over a
// group's workgroups, and the parameters' over the parts) is added by the last launch in a fixed order.
//
// Bound by the vector unit: about 45 instructions for each state and row, 7 of them in the maps, 5 in the walk for the
// tiles' states, 15 to step a state and its gradient, the rest sums over lanes and what each row needs once.
// Measured: 16,381 bf16 rows of 2,048 channels and 16 states in 9 sequences: 180 + 36 + 650 + 14 + 10 us (maps,
// joining, walk, dB and dC, parameters), the vector unit busy for 73% of the walk; 59,837 fp16 rows of 256 channels
// and 8 states in 1,521 windows: 49 + 16 + 245 + 7 + 11 us (these calls 843 and 311 us; over an order that scatters
// the rows 1,209 and 411).  Tiles of 16 rows, without the next tile's rows on their
// way and with selects in the sums over channels: 875 us for the first walk; three workgroups a CU (168 registers,
// 64 of them spilled): 1,450; decays made again on the way back instead of kept: 971 us in all against 941.
#include <algorithm>

#include "sla_scan.h"

namespace sla {
namespace {

using namespace scan;

constexpr int kMaxTiles = 8, kThreads = 256, kWaves = 4;
// Rows of a tile: their states' a and decays are in registers, 8 for each row.
template <int NG>
constexpr int kTileOf = NG <= 8 ? 8 : 16;
constexpr float kLn2 = 0.693147181f;

struct BackArgs {
  ScanArgs a;
  int32_t cw;            // channels of a workgroup
  int32_t wpg;           // workgroups across a group's channels
  Parts fwd;             // S, sum dt
  float* R;              // [slots][N][D]
  float* bc;             // [G wpg][n][2 N]: sums over a workgroup's channels, by position
  float *pA, *pskip, *pbias;   // [slots][D N], [slots][D], [slots][D]
};

// ------------------------------------------------------------------ the parts' maps
// A wave takes 64 channels and NS of their states, as the forward does.
template <typename T, int NS>
__global__ __launch_bounds__(64) void k_scan_maps(BackArgs k, const T* __restrict__ x, const T* __restrict__ delta,
                                                  const T* __restrict__ z, const T* __restrict__ B,
                                                  const T* __restrict__ C, const T* __restrict__ dy) {
  constexpr int U = 4, V = 2 * NS, J = (U * V + 63) / 64;
  __shared__ __attribute__((aligned(16))) float s_bc[J * 64];
  const ScanArgs& a = k.a;
  Part part;
  if (!part_of(a.win, a.per, blockIdx.x, part)) return;
  if (part.first && part.last) return;   // the whole window
  const int lane = threadIdx.x, n0 = blockIdx.z * NS, N = min(a.N - n0, NS);
  const Tile tile(a, blockIdx.y, lane);
  const int c = tile.c;
  float A[NS], h[NS], P[NS], R[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    A[n] = n < N ? exponent(a.A[(size_t)c * a.N + n0 + n]) : 0.f;
    h[n] = R[n] = 0.f;
    P[n] = 1.f;
  }
  const float bias = a.bias ? a.bias[c] : 0.f;
  float dts = 0.f;
  T xr[U], dr[U], zr[U], gr[U], bc[J];
  int next_row[U], shared_row[J];
  const T* zp = z != nullptr ? z : dy;   // without a gate something that is there, and is not used
  const int64_t ldz = z != nullptr ? a.ldz : a.ldy;
  const auto ask = [&](int p0) __attribute__((always_inline)) {
    // rows past the end are the last one, and are not used
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = a.win.row(min(p0 + i, part.end - 1)), r = max(at, 0);
      next_row[i] = p0 + i < part.end ? at : -1;
      xr[i] = lane_at(x + r * a.ldx, c);
      dr[i] = lane_at(delta + r * a.ldd, c);
      gr[i] = lane_at(dy + r * a.ldy, c);
      zr[i] = lane_at(zp + r * ldz, c);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int at = lane + 64 * j, p = p0 + at / V, v = at % V, n = v % NS;
      const int r = a.win.row(min(p, part.end - 1));
      shared_row[j] = p < part.end && at < U * V && n < N ? r : -1;
      const int64_t row = max(r, 0);
      const int m = tile.g * a.N + n0 + min(n, N - 1);
      const T* src = v < NS ? B + (row * a.ldb + m) : C + (row * a.ldc + m);
      bc[j] = *src;
    }
  };
  ask(part.begin);
  for (int p0 = part.begin; p0 < part.end; p0 += U) {
    float xv[U], dt[U], zv[U], gv[U];
    int row[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      row[i] = next_row[i];
      xv[i] = to_float(xr[i]);
      dt[i] = to_float(dr[i]) + bias;
      zv[i] = to_float(zr[i]);
      gv[i] = to_float(gr[i]);
      asm volatile("" : "+v"(xv[i]), "+v"(dt[i]), "+v"(zv[i]), "+v"(gv[i]));   // the registers are the next rows'
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < J; ++j) s_bc[lane + 64 * j] = shared_row[j] >= 0 ? to_float(bc[j]) : 0.f;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    ask(p0 + U);
    if (a.softplus)
#pragma unroll
      for (int i = 0; i < U; ++i) dt[i] = softplus(dt[i]);
    if (z != nullptr)
#pragma unroll
      for (int i = 0; i < U; ++i) gv[i] *= quick_silu(zv[i]);
    // past the part's end, and where the order names no row, a row's step, input and gradient are 0, as its B and C:
    // nothing changes.  By selects: of branches on rows that the order holds the compiler dropped all but the first.
    if (p0 + U > part.end || a.win.order != nullptr)
#pragma unroll
      for (int i = 0; i < U; ++i) {
        dt[i] = row[i] >= 0 ? dt[i] : 0.f;
        xv[i] = row[i] >= 0 ? xv[i] : 0.f;
        gv[i] = row[i] >= 0 ? gv[i] : 0.f;
      }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float u = dt[i] * xv[i];
      dts += dt[i];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const float e = __builtin_amdgcn_exp2f(dt[i] * A[n]);
        h[n] = __builtin_fmaf(e, h[n], u * s_bc[i * V + n]);
        P[n] *= e;
        R[n] = __builtin_fmaf(P[n], gv[i] * s_bc[i * V + NS + n], R[n]);
      }
    }
  }
  if (!tile.live) return;
#pragma unroll
  for (int n = 0; n < NS; ++n)
    if (n < N) {
      const size_t at = ((size_t)blockIdx.x * a.N + n0 + n) * a.D + c;
      k.fwd.S[at] = h[n];
      k.R[at] = R[n];
    }
  if (n0 == 0) k.fwd.dts[(size_t)blockIdx.x * a.D + c] = dts;
}

// Along the parts of every window: S becomes the state behind its part and R the gradient of the state
// before it; the two ends' places, which are free, take copies of the window's state and of its gradient (the
// outputs may lie where these are read).  Windows without rows hand their gradient on.
__global__ __launch_bounds__(256) void k_scan_carry_back(BackArgs k, const float* __restrict__ state,
                                                         const float* __restrict__ dstate,
                                                         float* __restrict__ dstate_in) {
  const ScanArgs& a = k.a;
  const int w = blockIdx.x;
  const int b = a.win.edge(w), e = a.win.edge(w + 1);
  const int count = e > b ? (e - b - 1) / a.per : 0;   // parts but one
  if (e > b && count == 0) return;
  const int64_t size = (int64_t)a.N * a.D, first = (int64_t)(b / a.per) + w;
  for (int64_t at = (int64_t)blockIdx.y * 256 + threadIdx.x; at < size; at += (int64_t)gridDim.y * 256) {
    const int n = (int)(at / a.D), c = (int)(at % a.D);
    const size_t mine = ((size_t)w * a.D + c) * a.N + n;
    float h = state != nullptr ? state[mine] : 0.f, q = dstate != nullptr ? dstate[mine] : 0.f;
    if (e <= b) {
      if (dstate_in != nullptr) dstate_in[mine] = q;
      continue;
    }
    const float A = exponent(a.A[(size_t)c * a.N + n]);
    k.fwd.S[(first + count) * size + at] = h;
    k.R[first * size + at] = q;
    const auto join = [&](int i0, auto ahead) __attribute__((always_inline)) {
      constexpr int K = decltype(ahead)::value;
      float S[K], d[K], R[K], f[K];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int64_t s = first + min(i0 + i, count - 1), r = first + max(count - i0 - i, 1);
        S[i] = k.fwd.S[s * size + at];
        d[i] = k.fwd.dts[s * a.D + c];
        R[i] = k.R[r * size + at];
        f[i] = k.fwd.dts[r * a.D + c];
      }
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (i0 + i < count) {
          h = decayed(A * d[i], h) + S[i];
          k.fwd.S[(first + i0 + i) * size + at] = h;
          q = decayed(A * f[i], q) + R[i];
          k.R[(first + count - i0 - i) * size + at] = q;
        }
      return i0 + K;
    };
    for (int i = 0; i < count;)
      i = count - i > 8 ? join(i, std::integral_constant<int, 24>{}) : join(i, std::integral_constant<int, 8>{});
  }
}

// ------------------------------------------------------------------ sums over lanes
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// x of the lane whose number differs in bit S; below 8 in lower bits too unless EXACT (then the sum over those
// is still to come, and the pairing does not matter)
template <int S, bool EXACT>
__device__ __forceinline__ float other(float x) {
  if constexpr (S == 1) return dpp<0xb1>(x);
  else if constexpr (S == 2) return dpp<0x4e>(x);
  else if constexpr (S == 4 && !EXACT) return dpp<0x141>(x);
  else if constexpr (S == 8) return dpp<0x128>(x);
  else return __shfl_xor(x, S);
}
// Sums of pairs of lanes, a where bit S of the lane is clear, b where it is set.
template <int S, bool EXACT>
__device__ __forceinline__ float halve(float a, float b, int lane) {
  if constexpr (S == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else if constexpr (S == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    const bool up = lane & S;
    const float keep = up ? b : a, send = up ? a : b;
    return keep + other<S, EXACT>(send);
  }
}
// The same for M / 2 pairs x[k], x[k + M / 2] at once where S is 8 or 4: two additions a pair, each written to the
// banks of four lanes that it is for.  A lane's neighbour may have been written just before: two wait states.
#define SLA_PAIR(DST, SRC, SHIFT, LOW, HIGH)                                              \
  "v_add_f32_dpp " DST ", " DST ", " DST " " SHIFT " row_mask:0xf bank_mask:" LOW "\n"     \
  "v_add_f32_dpp " DST ", " SRC ", " SRC " " SHIFT " row_mask:0xf bank_mask:" HIGH "\n"
template <int M, int S>
__device__ __forceinline__ void halve_banks(float* x) {
  static_assert((M == 2 || M == 4 || M == 8) && (S == 4 || S == 8));
  if constexpr (M == 8 && S == 8)
    asm("s_nop 1\n" SLA_PAIR("%0", "%4", "row_ror:8", "0x3", "0xc") SLA_PAIR("%1", "%5", "row_ror:8", "0x3", "0xc")
        SLA_PAIR("%2", "%6", "row_ror:8", "0x3", "0xc") SLA_PAIR("%3", "%7", "row_ror:8", "0x3", "0xc")
        : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]) : "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]));
  else if constexpr (M == 8)
    asm("s_nop 1\n" SLA_PAIR("%0", "%4", "row_half_mirror", "0x5", "0xa") SLA_PAIR("%1", "%5", "row_half_mirror", "0x5", "0xa")
        SLA_PAIR("%2", "%6", "row_half_mirror", "0x5", "0xa") SLA_PAIR("%3", "%7", "row_half_mirror", "0x5", "0xa")
        : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]) : "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]));
  else if constexpr (M == 4 && S == 8)
    asm("s_nop 1\n" SLA_PAIR("%0", "%2", "row_ror:8", "0x3", "0xc") SLA_PAIR("%1", "%3", "row_ror:8", "0x3", "0xc")
        : "+v"(x[0]), "+v"(x[1]) : "v"(x[2]), "v"(x[3]));
  else if constexpr (M == 4)
    asm("s_nop 1\n" SLA_PAIR("%0", "%2", "row_half_mirror", "0x5", "0xa") SLA_PAIR("%1", "%3", "row_half_mirror", "0x5", "0xa")
        : "+v"(x[0]), "+v"(x[1]) : "v"(x[2]), "v"(x[3]));
  else if constexpr (S == 8)
    asm("s_nop 1\n" SLA_PAIR("%0", "%1", "row_ror:8", "0x3", "0xc") : "+v"(x[0]) : "v"(x[1]));
  else
    asm("s_nop 1\n" SLA_PAIR("%0", "%1", "row_half_mirror", "0x5", "0xa") : "+v"(x[0]) : "v"(x[1]));
}
#undef SLA_PAIR
// x[0 .. M - 1] summed over the lanes that differ in bits S, S / 2, .. LOW: lane bit S chooses between x[k] and
// x[k + M / 2], the next bit halves what is left, and so on; where one value is left, every lane has its sum.
template <int M, int S, int LOW, bool EXACT>
__device__ __forceinline__ void sum_lanes(float* x, int lane) {
  if constexpr (S >= LOW) {
    if constexpr (M > 8 || (M > 1 && S != 8 && (S != 4 || EXACT))) {
#pragma unroll
      for (int k = 0; k < M / 2; ++k) x[k] = halve<S, EXACT>(x[k], x[k + M / 2], lane);
      sum_lanes<M / 2, S / 2, LOW, EXACT>(x, lane);
    } else if constexpr (M > 1) {
      halve_banks<M, S>(x);
      sum_lanes<M / 2, S / 2, LOW, EXACT>(x, lane);
    } else {
      x[0] += other<S, EXACT>(x[0]);
      sum_lanes<1, S / 2, LOW, EXACT>(x, lane);
    }
  }
}

// ------------------------------------------------------------------ the walk
// NG lanes a channel, four states each; lane = ng CW + channel.  Of a tile a lane takes the rows
// j NG + ng of its channel wherever rows are taken one by one (step sizes, gates, results).
template <typename T, int NG>
__global__ __launch_bounds__(kThreads, 2) void k_scan_back(BackArgs k, const T* __restrict__ x,
                                                           const T* __restrict__ delta, const T* __restrict__ z,
                                                           const T* __restrict__ B, const T* __restrict__ C,
                                                           const float* __restrict__ state, const T* __restrict__ dy,
                                                           const float* __restrict__ dstate, T* __restrict__ dx,
                                                           T* __restrict__ ddelta, T* __restrict__ dz,
                                                           float* __restrict__ dstate_in) {
  constexpr int kTile = kTileOf<NG>, CW = 64 / NG, E = kTile / NG, NP = 4 * NG;
  constexpr int kStage = (kTile * 2 * NP + kThreads - 1) / kThreads;
  __shared__ floatx4 s_in[kWaves][kTile][CW];            // dt, u, g of the wave's channels
  __shared__ floatx4 s_start[kWaves][kMaxTiles][64];     // states before each tile
  // two of what the waves share, for tiles in turn, so that a tile has one barrier; at 64 states they would need 120 KB
  constexpr int kTurns = NG <= 8 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float s_shared[kTurns][kTile][2][NP];
  __shared__ float s_sums[kTurns][kWaves][kTile][2][NP];
  const ScanArgs& a = k.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ng = lane / CW, ch = lane % CW;
  const int g = blockIdx.y / k.wpg, at = (blockIdx.y % k.wpg) * k.cw + wave * CW + ch;
  const bool live = at < a.cg;
  const int c = g * a.cg + (live ? at : 0), n0 = 4 * ng;
  const size_t slot = blockIdx.x;
  Part part;
  if (!part_of(a.win, a.per, blockIdx.x, part)) {
    // a slot without a part: nothing to the parameters' sums
    if (live) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n0 + r < a.N) k.pA[slot * a.D * a.N + (size_t)c * a.N + n0 + r] = 0.f;
      if (ng == 0) k.pskip[slot * a.D + c] = k.pbias[slot * a.D + c] = 0.f;
    }
    return;
  }
  const int count = (a.win.edge(part.w + 1) - a.win.edge(part.w) - 1) / a.per;   // the window's parts but one
  float A[4], h[4], q[4], dA[4] = {};
  const auto from_parts = [&](const float* p, size_t s, float (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = live && n0 + r < a.N ? p[(s * a.N + n0 + r) * a.D + c] : 0.f;
  };
  const auto from_window = [&](const float* p, float (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      v[r] = p != nullptr && live && n0 + r < a.N ? p[((size_t)part.w * a.D + c) * a.N + n0 + r] : 0.f;
  };
#pragma unroll
  for (int r = 0; r < 4; ++r) A[r] = n0 + r < a.N ? exponent(a.A[(size_t)c * a.N + n0 + r]) : 0.f;
  if (!part.first) from_parts(k.fwd.S, slot - 1, h);
  else if (!part.last && state != nullptr) from_parts(k.fwd.S, slot + count, h);
  else from_window(state, h);
  if (!part.last) from_parts(k.R, slot + 1, q);
  else if (!part.first && dstate != nullptr) from_parts(k.R, slot - count, q);
  else from_window(dstate, q);
  const float bias = a.bias ? a.bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;
  float sum_skip = 0.f, sum_bias = 0.f;

  T xr[E], dr[E], zr[E] = {}, gr[E] = {}, bc[kStage];
  int row[E], shared_row[kStage];
  const T* zp = z != nullptr ? z : dy;   // without a gate something that is there, and is not used
  const int64_t ldz = z != nullptr ? a.ldz : a.ldy;
  // A tile's rows: x and delta, and with them all else that the way back needs.  Loads without conditions (row 0 for a
  // row that is none): where a register has one value or another, the compiler copies it, and waits for it, at once.
  const auto ask = [&](int p0, bool back) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int p = p0 + j * NG + ng, r = a.win.row(min(p, part.end - 1));
      row[j] = p < part.end && live ? r : -1;
      const int at = max(r, 0);
      xr[j] = x[at * a.ldx + c];
      dr[j] = delta[at * a.ldd + c];
      if (back) {
        gr[j] = dy[at * a.ldy + c];
        zr[j] = zp[at * ldz + c];
      }
    }
#pragma unroll
    for (int j = 0; j < kStage; ++j) {
      const int i = tid + kThreads * j, t = i / (2 * NP), v = i % (2 * NP), n = v % NP;
      const int r = a.win.row(min(p0 + t, part.end - 1));
      shared_row[j] = t < kTile && p0 + t < part.end && n < a.N ? r : -1;
      const int at = max(r, 0), m = g * a.N + min(n, a.N - 1);
      const T* src = v < NP ? B + (at * a.ldb + m) : C + (at * a.ldc + m);
      bc[j] = *src;
    }
  };
  float pre[E], dt[E], gate[E], xv[E], zv[E], gv[E];
  const auto stage = [&](int turn, bool back) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      xv[j] = to_float(xr[j]);
      pre[j] = to_float(dr[j]) + bias;
      zv[j] = to_float(zr[j]);
      gv[j] = to_float(gr[j]);
      asm volatile("" : "+v"(xv[j]), "+v"(pre[j]), "+v"(zv[j]), "+v"(gv[j]));   // the registers are the next rows'
      const bool real = row[j] >= 0;
      dt[j] = real ? (a.softplus ? softplus(pre[j]) : pre[j]) : 0.f;
      gate[j] = back && z != nullptr ? quick_silu(zv[j]) : 1.f;
      s_in[wave][j * NG + ng][ch] = floatx4{dt[j], real ? dt[j] * xv[j] : 0.f, real ? gv[j] * gate[j] : 0.f, 0.f};
    }
    float* flat = &s_shared[turn][0][0][0];
#pragma unroll
    for (int j = 0; j < kStage; ++j)
      if (tid + kThreads * j < kTile * 2 * NP) flat[tid + kThreads * j] = shared_row[j] >= 0 ? to_float(bc[j]) : 0.f;
  };

  const int tiles = (part.end - part.begin + kTile - 1) / kTile;
  // the states before every tile
  s_start[wave][0][lane] = floatx4{h[0], h[1], h[2], h[3]};
  if (tiles > 1) ask(part.begin, false);
  for (int i = 0; i + 1 < tiles; ++i) {
    const int turn = i % kTurns;
    if (kTurns == 1) __syncthreads();
    stage(turn, false);
    __syncthreads();
    const auto& s_bc = s_shared[turn];
    if (i + 2 < tiles) ask(part.begin + (i + 1) * kTile, false);
#pragma unroll
    for (int t = 0; t < kTile; ++t) {
      const floatx4 in = s_in[wave][t][ch], Bv = *reinterpret_cast<const floatx4*>(&s_bc[t][0][n0]);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        h[r] = __builtin_fmaf(__builtin_amdgcn_exp2f(in[0] * A[r]), h[r], in[1] * Bv[r]);
    }
    s_start[wave][i + 1][lane] = floatx4{h[0], h[1], h[2], h[3]};
  }

  // the waves' sums over their channels of the tile at p0
  const auto hand_on = [&](int p0, int turn) __attribute__((always_inline)) {
    const float* red = &s_sums[turn][0][0][0][0];
    for (int v = tid; v < kTile * 2 * NP; v += kThreads) {
      const int t = v / (2 * NP), which = v / NP % 2, n = v % NP;
      if (p0 + t < part.end && n < a.N) {
        float sum = red[v];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += red[w * kTile * 2 * NP + v];
        k.bc[((size_t)blockIdx.y * a.win.n + p0 + t) * 2 * a.N + which * a.N + n] = sum;
      }
    }
  };
  ask(part.begin + (tiles - 1) * kTile, true);
  for (int i = tiles - 1; i >= 0; --i) {
    const int p0 = part.begin + i * kTile;
    const int turn = i % kTurns;
    if (kTurns == 1) {
      __syncthreads();
      if (i + 1 < tiles) hand_on(p0 + kTile, 0);
    }
    stage(turn, true);
    int at_row[E];
#pragma unroll
    for (int j = 0; j < E; ++j) at_row[j] = row[j];
    __syncthreads();
    if (kTurns > 1 && i + 1 < tiles) hand_on(p0 + kTile, turn ^ 1);
    const auto& s_bc = s_shared[turn];
    auto& s_red = s_sums[turn];
    if (i > 0) ask(p0 - kTile, true);
    float kept[kTile][4], e[kTile][4];
    {
      const floatx4 s = s_start[wave][i][lane];
#pragma unroll
      for (int r = 0; r < 4; ++r) h[r] = s[r];
    }
#pragma unroll
    for (int t = 0; t < kTile; ++t) {
      const floatx4 in = s_in[wave][t][ch], Bv = *reinterpret_cast<const floatx4*>(&s_bc[t][0][n0]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[t][r] = __builtin_amdgcn_exp2f(in[0] * A[r]);
        kept[t][r] = e[t][r] * h[r];
        h[r] = __builtin_fmaf(in[1], Bv[r], kept[t][r]);
      }
    }
    float du[NG], dda[NG], yl[NG];
#pragma unroll
    for (int t = kTile - 1; t >= 0; --t) {
      const floatx4 in = s_in[wave][t][ch], Bv = *reinterpret_cast<const floatx4*>(&s_bc[t][0][n0]),
                    Cv = *reinterpret_cast<const floatx4*>(&s_bc[t][1][n0]);
      float shared[8];
      float s0 = 0.f, s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float ht = __builtin_fmaf(in[1], Bv[r], kept[t][r]);
        q[r] = __builtin_fmaf(Cv[r], in[2], q[r]);
        shared[r] = q[r] * in[1];
        shared[4 + r] = ht * in[2];
        s0 = __builtin_fmaf(q[r], Bv[r], s0);
        s2 = __builtin_fmaf(Cv[r], ht, s2);
        const float da = q[r] * kept[t][r];
        s1 = __builtin_fmaf(da, A[r], s1);
        dA[r] = __builtin_fmaf(da, in[0], dA[r]);
        q[r] *= e[t][r];
      }
      du[t % NG] = s0;
      dda[t % NG] = s1;
      yl[t % NG] = s2;
      sum_lanes<8, CW / 2, 1, false>(shared, lane);
      // the halvings chose: the first lane bit B or C, the next two the state
      if constexpr (CW >= 8) {
        constexpr int b0 = CW / 2, b1 = CW / 4, b2 = CW / 8;
        const int v = n0 + ((lane & b1) ? 2 : 0) + ((lane & b2) ? 1 : 0);
        if ((lane & (b2 - 1)) == 0) s_red[wave][t][(lane & b0) ? 1 : 0][v] = shared[0];
      } else {
        const int v = n0 + ((lane & 1) ? 2 : 0);
        s_red[wave][t][(lane & 2) ? 1 : 0][v] = shared[0];
        s_red[wave][t][(lane & 2) ? 1 : 0][v + 1] = shared[1];
      }
      if (t % NG == 0) {
        sum_lanes<NG, 32, CW, true>(du, lane);
        sum_lanes<NG, 32, CW, true>(dda, lane);
        sum_lanes<NG, 32, CW, true>(yl, lane);
        const int j = t / NG;
        if (at_row[j] >= 0) {
          const float g1 = gv[j] * gate[j];
          float dd = __builtin_fmaf(du[0], xv[j], dda[0] * kLn2);
          if (a.softplus) dd *= quick_sigmoid(pre[j]);
          const size_t o = (size_t)at_row[j] * a.D + c;
          dx[o] = from_float<T>(__builtin_fmaf(du[0], dt[j], g1 * skip));
          ddelta[o] = from_float<T>(dd);
          if (z != nullptr)
            dz[o] = from_float<T>(gv[j] * __builtin_fmaf(skip, xv[j], yl[0]) * quick_silu_slope(zv[j]));
          sum_skip = __builtin_fmaf(g1, xv[j], sum_skip);
          sum_bias += dd;
        }
      }
    }
  }
  __syncthreads();
  hand_on(part.begin, 0);
  float sums[1] = {sum_skip};
  sum_lanes<1, 32, CW, true>(sums, lane);
  sum_skip = sums[0];
  sums[0] = sum_bias;
  sum_lanes<1, 32, CW, true>(sums, lane);
  sum_bias = sums[0];
  if (!live) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n0 + r < a.N) {
      k.pA[slot * a.D * a.N + (size_t)c * a.N + n0 + r] = dA[r];
      if (part.first && dstate_in != nullptr) dstate_in[((size_t)part.w * a.D + c) * a.N + n0 + r] = q[r];
    }
  if (ng == 0) {
    k.pskip[slot * a.D + c] = sum_skip;
    k.pbias[slot * a.D + c] = sum_bias;
  }
}

// ------------------------------------------------------------------ the last sums
// dB and dC: over the workgroups of a group, in their order; one value a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_scan_shared(BackArgs k, T* __restrict__ dB, T* __restrict__ dC) {
  const ScanArgs& a = k.a;
  const int64_t per_row = 2 * (int64_t)a.G * a.N;
  const int first = a.win.edge(0), last = a.win.edge(a.win.W);
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < per_row * a.win.n;
       at += (int64_t)gridDim.x * kThreads) {
    const int p = (int)(at / per_row);
    const int r = p >= first && p < last ? a.win.row(p) : -1;
    if (r < 0) continue;
    const int v = (int)(at % per_row), g = v / (2 * a.N), i = v % (2 * a.N);
    const float* src = k.bc + ((size_t)g * k.wpg * a.win.n + p) * 2 * a.N + i;
    float sum = 0.f;
#pragma unroll 8
    for (int w = 0; w < k.wpg; ++w) sum += src[(size_t)w * a.win.n * 2 * a.N];
    T* out = i < a.N ? dB : dC;
    out[((size_t)r * a.G + g) * a.N + i % a.N] = from_float<T>(sum);
  }
}

// The parameters: over all parts, 64 values a workgroup, sixteen runs of parts side by side.
__global__ __launch_bounds__(1024) void k_scan_params(BackArgs k, int32_t slots, float* __restrict__ dA,
                                                      float* __restrict__ dskip, float* __restrict__ dbias) {
  __shared__ float s_sum[16][64];
  const ScanArgs& a = k.a;
  const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
  const int64_t size = (int64_t)a.D * a.N, at = (int64_t)blockIdx.x * 64 + lane;
  const float* src = nullptr;
  float* out = nullptr;
  int64_t step = a.D;
  if (at < size) src = k.pA + at, out = dA + at, step = size;
  else if (at < size + a.D) src = k.pskip + (at - size), out = dskip ? dskip + (at - size) : nullptr;
  else if (at < size + 2 * a.D) src = k.pbias + (at - size - a.D), out = dbias ? dbias + (at - size - a.D) : nullptr;
  float sum = 0.f;
  if (src != nullptr) {
    const int lo = (int)((int64_t)slots * run / 16), hi = (int)((int64_t)slots * (run + 1) / 16);
#pragma unroll 8
    for (int s = lo; s < hi; ++s) sum += src[(size_t)s * step];
  }
  s_sum[run][lane] = sum;
  __syncthreads();
  if (run || out == nullptr) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += s_sum[i][lane];
  *out = sum;
}

// Whole tiles; 1,024 workgroups, four for every CU, of which two are there at a time, but parts of eight tiles at most,
// whose states LDS holds.  Where there are windows enough, parts as long as they can be.
int rows_per_part_back(int64_t n, int32_t W, int64_t blocks, int tile) {
  int64_t per = W * blocks >= 1024 ? n : n * blocks / 1024 / tile * tile;
  per = per < 4 * tile ? 4 * tile : per > tile * kMaxTiles ? tile * kMaxTiles : per;
  return (int)per;
}

// The parts of any numbers of rows and windows up to n and W, as the forward's: parts of 4 to 7 tiles mean fewer than
// (per + tile) 1024 / blocks rows, so at most 1280 / blocks beside the windows' own.
int64_t most_parts_back(int64_t n, int32_t W, int64_t blocks, int tile) {
  return std::max(std::min(n / (4 * tile), (1280 + blocks - 1) / blocks), n / (tile * kMaxTiles)) + W;
}

int lane_groups(int32_t N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

struct BackLayout {
  int32_t ng, cw, wpg, per;
  int64_t slots;
  size_t S, dts, R, bc, pA, pskip, pbias, total;
};
// most: with the places that fewer rows or windows may need
BackLayout back_layout(int64_t n, int32_t W, int32_t D, int32_t G, int32_t N, bool most) {
  BackLayout L;
  L.ng = lane_groups(N);
  L.cw = 64 / L.ng * kWaves;
  L.wpg = (D / G + L.cw - 1) / L.cw;
  const int64_t blocks = (int64_t)G * L.wpg;
  const int tile = L.ng <= 8 ? 8 : 16;
  L.per = rows_per_part_back(n, W, blocks, tile);
  L.slots = most ? most_parts_back(n, W, blocks, tile) : n / L.per + W;
  size_t off = 0;
  const auto take = [&](size_t floats) {
    const size_t at = off;
    off = align_up(off + floats * 4, 256);
    return at;
  };
  const size_t slots = (size_t)L.slots;
  L.S = take(slots * D * N);
  L.R = take(slots * D * N);
  L.pA = take(slots * D * N);
  L.dts = take(slots * D);
  L.pskip = take(slots * D);
  L.pbias = take(slots * D);
  L.bc = take((size_t)G * L.wpg * n * 2 * N);
  L.total = off;
  return L;
}

}  // namespace

size_t scan_backward_workspace_bytes(int64_t n, int32_t W, int32_t D, int32_t G, int32_t N) {
  return back_layout(n, W, D, G, N, true).total;
}

hipError_t launch_backward_scan(scan::ScanArgs a, int dtype, const void* x, const void* delta, const void* z,
                                const void* B, const void* C, const float* state_in, const void* dy,
                                const float* dstate_out, void* dx, void* ddelta, float* dA, void* dB, void* dC,
                                float* dskip, void* dz, float* dbias, float* dstate_in, void* workspace,
                                hipStream_t stream) {
  const BackLayout L = back_layout(a.win.n, a.win.W, a.D, a.G, a.N, false);
  a.cg = a.D / a.G;
  a.tpg = (a.cg + 63) / 64;
  a.per = L.per;
  char* ws = static_cast<char*>(workspace);
  const auto at = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  BackArgs k;
  k.a = a;
  k.cw = L.cw;
  k.wpg = L.wpg;
  k.fwd.S = at(L.S);
  k.fwd.dts = at(L.dts);
  k.R = at(L.R);
  k.bc = at(L.bc);
  k.pA = at(L.pA);
  k.pskip = at(L.pskip);
  k.pbias = at(L.pbias);
  const int64_t values = (int64_t)a.D * a.N;
  const bool cut = a.win.n > a.per;
  const auto run = [&](auto type) {
    using T = decltype(type);
    const auto *xp = static_cast<const T*>(x), *dp = static_cast<const T*>(delta), *zp = static_cast<const T*>(z),
               *bp = static_cast<const T*>(B), *cp = static_cast<const T*>(C), *yp = static_cast<const T*>(dy);
    if (cut) {
      const dim3 grid((uint32_t)L.slots, (uint32_t)(a.G * a.tpg), (a.N + 15) / 16);
      const auto maps = [&](auto kernel) { kernel<<<grid, 64, 0, stream>>>(k, xp, dp, zp, bp, cp, yp); };
      if (a.N <= 4) maps(k_scan_maps<T, 4>);
      else if (a.N <= 8) maps(k_scan_maps<T, 8>);
      else maps(k_scan_maps<T, 16>);
    }
    if (cut || dstate_in != nullptr)
      k_scan_carry_back<<<dim3(a.win.W, carry_blocks(a)), 256, 0, stream>>>(k, state_in, dstate_out,
                                                                                            dstate_in);
    if (a.win.n > 0) {
      const dim3 grid((uint32_t)L.slots, (uint32_t)(a.G * L.wpg));
      const auto walk = [&](auto kernel) {
        kernel<<<grid, kThreads, 0, stream>>>(k, xp, dp, zp, bp, cp, state_in, yp, dstate_out, static_cast<T*>(dx),
                                              static_cast<T*>(ddelta), static_cast<T*>(dz), dstate_in);
      };
      switch (L.ng) {
        case 1: walk(k_scan_back<T, 1>); break;
        case 2: walk(k_scan_back<T, 2>); break;
        case 4: walk(k_scan_back<T, 4>); break;
        case 8: walk(k_scan_back<T, 8>); break;
        default: walk(k_scan_back<T, 16>); break;
      }
      const int64_t shared = 2 * (int64_t)a.win.n * a.G * a.N;
      k_scan_shared<T><<<(uint32_t)std::min<int64_t>((shared + kThreads - 1) / kThreads, 1 << 20), kThreads, 0, stream>>>(
          k, static_cast<T*>(dB), static_cast<T*>(dC));
    }
    k_scan_params<<<(uint32_t)((values + 2 * a.D + 63) / 64), 1024, 0, stream>>>(
        k, a.win.n > 0 ? (int32_t)L.slots : 0, dA, dskip, dbias);
  };
  if (dtype == 0) run(float{});
  else if (dtype == 1) run(_Float16{});
  else run(bf16_t{});
  return hipGetLastError();
}

}  // namespace sla
