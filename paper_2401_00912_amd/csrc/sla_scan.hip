// The selective scan over the rows of every window (the recurrence and how it is cut: sla_scan.h).
//
// Bound by the vector unit: a state and row take a product, an exponential, a product and two multiply-adds (one
// in the walk that makes a part's map); the memory's part (x, delta, z in, y out) is a third of that at 16 states.
// Measured: 32,768 bf16 rows of 2,048 channels and 16 states in 17 sequences: 203 + 23 + 294 us (maps, joining,
// results), some 690 cycles a row and wave where its 104 vector instructions and 19 exponentials
// and reciprocals take 570 issued one by one; 59,837 fp16 rows of 256 channels in 1,521 windows: 4.7 + 5.5 +
// 118 us, of which the longest window's 144 rows are the most; 8,191 fp32 rows of 1,024 channels in one: 32 + 17 +
// 44 us, 64 rows one after the other twice and 127 parts joined.  Over an order that scatters the rows, whose indices
// are loads that the rows' loads wait for, a call takes 778 us instead of 458 and 196 instead of 125 (the first two).
// What was not faster: B and C in scalar registers (454 -> 538 us for the results alone), matrix products for u B
// or the sum over states (fp32 ones take the vector unit's time: measured 31 ns for one with 16 products beside it,
// 14 and 16 alone), eight rows at once, workgroups of four waves (482).
#include <algorithm>

#include "sla_scan.h"

namespace sla {
namespace {

using namespace scan;

// Rows a wave takes at once: the next ones are on their way while these are computed.
constexpr int kRows = 4;

// OUT: the walk that makes y; else the one that makes a part's map.  ORDER: positions are not rows.  GATE: z is
// given.
template <typename T, int NS, bool OUT, bool ORDER, bool GATE>
__global__ __launch_bounds__(64, NS <= 16 ? 3 : 1) void k_scan(ScanArgs a, const T* __restrict__ x, const T* __restrict__ delta,
                                             const T* __restrict__ z, const T* __restrict__ B, const T* __restrict__ C,
                                             const float* __restrict__ state, T* __restrict__ y,
                                             float* __restrict__ state_out, Parts parts) {
  // a row's B and, behind it, C; J of a batch's values a lane
  constexpr int U = kRows, V = OUT ? 2 * NS : NS, J = (U * V + 63) / 64;
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
  for (int n = 0; n < NS; ++n) A[n] = exponent(A[n]);
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

  // x, delta and z of the next rows
  T xr[U], dr[U], zr[U] = {}, bc[J];
  int next_row[U], shared_row[J];
  const auto ask = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int i = (lane + 64 * j) / V, v = (lane + 64 * j) % V, n = v % NS, p = p0 + i;
      int r = min(p, part.end - 1);
      if (ORDER) r = a.win.row(r);
      shared_row[j] = i < U && n < a.N && p < part.end ? r : -1;
      const int64_t row = max(r, 0);
      const int m = tile.g * a.N + min(n, a.N - 1);
      const T* src = v < NS ? B + (row * a.ldb + m) : C + (row * a.ldc + m);
      bc[j] = *src;
    }
    // rows past the end are the last one, and are not used
    uint32_t off = c;
    asm volatile("" : "+v"(off));   // the lane's part of an address stays 32 bits beside a scalar base
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = min(p0 + i, part.end - 1), named = ORDER ? a.win.row(at) : at, r = max(named, 0);
      next_row[i] = p0 + i < part.end ? named : -1;
      xr[i] = lane_at(x + r * a.ldx, off);
      dr[i] = lane_at(delta + r * a.ldd, off);
      if (GATE) zr[i] = lane_at(z + r * a.ldz, off);
    }
  };
  // A batch's results are stored when the next one's rows are there and before those after it are asked for: loads
  // and stores end in order, and stores at the batch's end would be waited for at once.
  T late[U];
  const auto put = [&](int p0) __attribute__((always_inline)) {
    if (!tile.live) return;
    uint32_t off = c;
    asm volatile("" : "+v"(off));
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (p0 + i >= part.end) break;
      const int r = ORDER ? a.win.row(p0 + i) : p0 + i;
      if (!ORDER || r >= 0) lane_at(y + (int64_t)r * a.D, off) = late[i];
    }
  };
  ask(part.begin);
  for (int p0 = part.begin; p0 < part.end; p0 += U) {
    float xv[U], dt[U], zv[U], sum[U];
    int row_of[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      row_of[i] = next_row[i];
      xv[i] = to_float(xr[i]);
      dt[i] = to_float(dr[i]) + bias;
      zv[i] = to_float(zr[i]);
      // widened here, so that the registers are free for the next rows: a value that is still to be widened when
      // those arrive is copied at the loop's end, and that waits for them and for the stores before them
      asm volatile("" : "+v"(xv[i]), "+v"(dt[i]), "+v"(zv[i]));
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < J; ++j) s_bc[lane + 64 * j] = shared_row[j] >= 0 ? to_float(bc[j]) : 0.f;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (OUT && p0 > part.begin) put(p0 - U);
    ask(p0 + U);
    if (a.softplus)
#pragma unroll
      for (int i = 0; i < U; ++i) dt[i] = softplus(dt[i]);
    // past the part's end, and where the order names no row, a row's step and input are 0, as its B and C: h stays as
    // it is, bit for bit (by selects: k_scan_maps says why)
    if (p0 + U > part.end || ORDER)
#pragma unroll
      for (int i = 0; i < U; ++i) {
        dt[i] = row_of[i] >= 0 ? dt[i] : 0.f;
        xv[i] = row_of[i] >= 0 ? xv[i] : 0.f;
      }
    const auto row = [&](int i) __attribute__((always_inline)) {
      const float u = dt[i] * xv[i];
      float s[4] = {};
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const float e = __builtin_amdgcn_exp2f(dt[i] * A[n]);
        h[n] = __builtin_fmaf(e, h[n], u * s_bc[i * V + n]);
        if (OUT) s[n % 4] = __builtin_fmaf(s_bc[i * V + NS + n], h[n], s[n % 4]);
      }
      sum[i] = (s[0] + s[1]) + (s[2] + s[3]);
      if (!OUT) dts += dt[i];
    };
#pragma unroll
    for (int i = 0; i < U; ++i) row(i);
    if (!OUT) continue;
#pragma unroll
    for (int i = 0; i < U; ++i) sum[i] = __builtin_fmaf(skip, xv[i], sum[i]);
    if (GATE)
#pragma unroll
      for (int i = 0; i < U; ++i) sum[i] *= quick_silu(zv[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) late[i] = from_float<T>(sum[i]);
  }
  if (OUT) put(part.begin + (part.end - 1 - part.begin) / U * U);
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
  const int w = blockIdx.x;
  const int b = a.win.edge(w), e = a.win.edge(w + 1);
  const int count = e > b ? (e - b - 1) / a.per : 0;   // parts but the last
  if (e > b && count == 0) return;
  const int64_t size = (int64_t)a.N * a.D, first = (int64_t)(b / a.per) + w;
  for (int64_t at = (int64_t)blockIdx.y * 256 + threadIdx.x; at < size; at += (int64_t)gridDim.y * 256) {
    const int n = (int)(at / a.D), c = (int)(at % a.D);
    const size_t mine = ((size_t)w * a.D + c) * a.N + n;
    float h = state != nullptr ? state[mine] : 0.f;
    if (e <= b) {
      if (state_out != nullptr) state_out[mine] = h;
      continue;
    }
    const float A = exponent(a.A[(size_t)c * a.N + n]);
    parts.S[(first + count) * size + at] = h;   // the last part's place is free: a copy for the first part
    const auto join = [&](int i0, auto ahead) __attribute__((always_inline)) {
      constexpr int K = decltype(ahead)::value;
      float S[K], d[K];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int64_t s = first + min(i0 + i, count - 1);
        S[i] = parts.S[s * size + at];
        d[i] = parts.dts[s * a.D + c];
      }
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (i0 + i < count) {
          h = decayed(A * d[i], h) + S[i];
          parts.S[(first + i0 + i) * size + at] = h;
        }
      return i0 + K;
    };
    for (int i = 0; i < count;)
      i = count - i > 8 ? join(i, std::integral_constant<int, 32>{}) : join(i, std::integral_constant<int, 8>{});
  }
}

// Rows of a part, and so the order of a window's sums, by all rows and windows of the call: waves for all SIMDs,
// but parts long enough that joining them costs little (the first case above
// with at most 64 rows: 475 us, 128: 469, 256: 550, 512: 672).  Where there are waves enough without cutting, only
// windows of four times the mean are cut (the second case: 124 us; cut at twice the mean 169, at 64 rows 160: a
// map takes as long as its part's rows one after the other, however few are cut).
int rows_per_part(int64_t n, int32_t W, int64_t tiles) {
  int64_t per = n * tiles / 8192 / 8 * 8;
  per = per < 64 ? 64 : per > 128 ? 128 : per;
  if (W * tiles >= 4096) {
    const int64_t whole = 4 * n / W / 8 * 8;
    per = whole < per ? per : whole > 512 ? 512 : whole;
  }
  return (int)per;
}

// The parts of any numbers of rows and windows up to n and W, of which there are fewer where parts get longer.  Parts
// of `per` = 64 to 120 rows mean fewer than (per + 8) 8192 / tiles rows, so at most 9216 / tiles parts beside the
// windows' own; those of windows that are not cut are longer.
int64_t most_parts(int64_t n, int32_t W, int64_t tiles) {
  return std::max(std::min(n / 64, (9216 + tiles - 1) / tiles), n / 128) + W;
}

int64_t tiles_of(int32_t D, int32_t G) { return (int64_t)G * ((D / G + 63) / 64); }

}  // namespace

size_t scan_workspace_bytes(int64_t n, int32_t W, int32_t D, int32_t G, int32_t N) {
  const int64_t slots = most_parts(n, W, tiles_of(D, G));
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
      if (cut) a.win.order ? args(k_scan<T, NS, false, true, false>) : args(k_scan<T, NS, false, false, false>);
      if (cut || state_out != nullptr)
        k_scan_carry<<<dim3(a.win.W, carry_blocks(a)), 256, 0, stream>>>(a, state_in,
                                                                                                     state_out, parts);
      if (a.win.n == 0) return;
      if (z != nullptr) a.win.order ? args(k_scan<T, NS, true, true, true>) : args(k_scan<T, NS, true, false, true>);
      else a.win.order ? args(k_scan<T, NS, true, true, false>) : args(k_scan<T, NS, true, false, false>);
    });
  };
  if (dtype == 0) run(float{});
  else if (dtype == 1) run(_Float16{});
  else run(bf16_t{});
  return hipGetLastError();
}

}  // namespace sla
