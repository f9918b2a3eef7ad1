// The short causal convolution over the rows of every window, its gradients, and its form for single
// rows on a pool of states.
//
// Channel by channel, of the rows t of a window, with the width - 1 rows before the first from a state:
//     z_t = bias + sum_j w_j x_{t - K + 1 + j},   y_t = act(z_t);
// with dz_t = dy_t act'(z_t):  dx_t = sum_j w_j dz_{t + K - 1 - j},  dw_j = sum_t dz_t x_{t - K + 1 + j},
// dbias = sum_t dz_t.
//
// Bound by memory: x (and dy) in, y (dx) out, once each.  A thread takes VEC channels of a strip of rows and
// walks down it: the K - 1 rows before (and, for the gradients, the K - 1 dx still to be finished) stay in
// registers, so a row is loaded once but for the K - 1 beside a strip's ends.  The gradients make z again from x.
// The sums over rows are kept by each thread for its strip, written once for each strip, and added by a
// second launch in the order of the strips.
// Measured (a copy reaches 5.1 TB/s): forward of 65,536 rows of 2,048 bf16 channels, width 4: 112 us, 4.8 TB/s;
// gradients of 16,381 rows of 4,096: 129 + 6 us, 3.1 TB/s: taps, sums, rows before, pending dx and two batches of rows
// take 152 registers, which leaves three waves a SIMD (the some 25 instructions a value alone would take 26 to 43 us);
// single rows, 256 of 4,096 channels: 6.6 us.  The next rows asked for before these are computed: 149 -> 124 us;
// neighbouring strips on one XCD: 124, in plain order 114.  Over an order that scatters the rows each row's index is a
// load that its own loads wait for: forward 232 us, gradients 216.
#include <algorithm>

#include "sla_act.h"
#include "sla_rows.h"

namespace sla {
namespace {

// Rows that a thread loads together: the next ones are on their way while these are computed.
constexpr int kThreads = 256, kBatch = 4;

struct ConvArgs {
  Windows win;
  const float *w, *bias;
  int64_t ldx, lddy;
  int32_t C, act;
  int32_t tx;               // threads across the channels
  int32_t per, strips;      // rows of a strip, strips
  uint32_t strip_blocks;    // workgroups of strips; those behind them make the states
};

// Where a walk down the positions is.
struct Place {
  int w, begin, end, next;   // window, its bounds, where the window after it begins
  __device__ __forceinline__ void at(const Windows& win, int p) {
    w = win.find(p);
    begin = w >= 0 ? win.edge(w) : 0;
    end = w >= 0 ? win.edge(w + 1) : 0;
    next = w + 1 < win.W ? win.edge(w + 1) : INT32_MAX;
  }
  // to position p; true where another window has begun
  __device__ __forceinline__ bool to(const Windows& win, int p) {
    bool fresh = false;
    while (next <= p) {
      ++w;
      begin = next;
      end = win.edge(w + 1);
      next = w + 1 < win.W ? end : INT32_MAX;
      fresh = true;
    }
    return fresh;
  }
  __device__ __forceinline__ bool in(int p) const { return w >= 0 && p < end; }
};

template <typename T, int VEC, int K>
struct Taps {
  float w[K][VEC], b[VEC];
  __device__ __forceinline__ void load(const ConvArgs& a, int c) {
    float flat[K * VEC];
    const float* p = a.w + (size_t)c * K;
    if constexpr (VEC % 4 == 0) {
#pragma unroll
      for (int i = 0; i < K * VEC; i += 4) {
        const floatx4 q = *reinterpret_cast<const floatx4*>(p + i);
#pragma unroll
        for (int r = 0; r < 4; ++r) flat[i + r] = q[r];
      }
    } else {
#pragma unroll
      for (int i = 0; i < K * VEC; ++i) flat[i] = p[i];
    }
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[j][e] = flat[e * K + j];
#pragma unroll
    for (int e = 0; e < VEC; ++e) b[e] = a.bias ? a.bias[c + e] : 0.f;
  }
};

// The K - 1 rows before position p of window `at`: its own rows, its state's, or zero.
template <typename T, int VEC, int K>
__device__ __forceinline__ void before(const ConvArgs& a, const Place& at, int p, const T* x, const T* state, int c,
                                       float (&h)[K][VEC]) {
  using V = Vec<T, VEC>;
#pragma unroll
  for (int j = 0; j < K - 1; ++j) {
    const int q = p - (K - 1) + j;
    typename V::R r = V::zero();
    if (at.in(p)) {
      if (q >= at.begin) {
        const int row = a.win.row(q);
        if (row >= 0) r = V::load(x + row * a.ldx + c);
      } else if (state != nullptr) {
        r = V::load(state + ((size_t)at.w * (K - 1) + (q - at.begin + K - 1)) * a.C + c);
      }
    }
    V::wide(r, h[j]);
  }
}

// The same where the window begins: its state, or zero.
template <typename T, int VEC, int K>
__device__ __forceinline__ void from_state(const ConvArgs& a, int w, const T* state, int c, float (&h)[K][VEC]) {
  using V = Vec<T, VEC>;
#pragma unroll
  for (int j = 0; j < K - 1; ++j)
    V::wide(state != nullptr ? V::load(state + ((size_t)w * (K - 1) + j) * a.C + c) : V::zero(), h[j]);
}

template <typename T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_fwd(ConvArgs a, const T* __restrict__ x, const T* __restrict__ state,
                                                       T* __restrict__ y, T* __restrict__ state_out) {
  using V = Vec<T, VEC>;
  const int tx = threadIdx.x % a.tx, ty = threadIdx.x / a.tx, strips = kThreads / a.tx;
  const int c = (blockIdx.y * a.tx + tx) * VEC;
  if (c >= a.C) return;
  if (blockIdx.x >= a.strip_blocks) {
    // the last K - 1 inputs of a window: its own, or what its state held
    const int w = (int)(blockIdx.x - a.strip_blocks) * strips + ty;
    if (w >= a.win.W) return;
    const int b = a.win.edge(w), rows = max(a.win.edge(w + 1) - b, 0);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
      const int t = rows - (K - 1) + j;
      typename V::R r = V::zero();
      if (t >= 0) {
        const int row = a.win.row(b + t);
        if (row >= 0) r = V::load(x + row * a.ldx + c);
      } else if (state != nullptr) {
        r = V::load(state + ((size_t)w * (K - 1) + rows + j) * a.C + c);
      }
      *reinterpret_cast<typename V::R*>(state_out + ((size_t)w * (K - 1) + j) * a.C + c) = r;
    }
    return;
  }
  const int strip = (int)blockIdx.x * strips + ty;
  if (strip >= a.strips) return;
  const int ps = strip * a.per, pe = min(ps + a.per, a.win.n);
  Taps<T, VEC, K> taps;
  taps.load(a, c);
  Place at;
  at.at(a.win, ps);
  float h[K][VEC];
  before<T, VEC, K>(a, at, ps, x, state, c, h);
  typename V::R ahead[kBatch];
  const auto ask = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = p0 + i < pe ? a.win.row(p0 + i) : -1;
      ahead[i] = r >= 0 ? V::load(x + r * a.ldx + c) : V::zero();
    }
  };
  ask(ps);
  for (int p0 = ps; p0 < pe; p0 += kBatch) {
    typename V::R raw[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) raw[i] = ahead[i];
    ask(p0 + kBatch);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int p = p0 + i;
      if (p < pe) {
        if (at.to(a.win, p)) from_state<T, VEC, K>(a, at.w, state, c, h);
        V::wide(raw[i], h[K - 1]);
        float z[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          z[e] = taps.b[e];
#pragma unroll
          for (int j = 0; j < K; ++j) z[e] = __builtin_fmaf(taps.w[j][e], h[j][e], z[e]);
        }
        act_all(a.act, z);
        const int r = at.in(p) ? a.win.row(p) : -1;
        if (r >= 0) V::store(y + (size_t)r * a.C + c, z);
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) h[j][e] = h[j + 1][e];
      }
    }
  }
}

// part: [strips][K + 1][C], the strips' sums of dw_0 .. dw_{K-1} and dbias
template <typename T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_bwd(ConvArgs a, const T* __restrict__ x, const T* __restrict__ state,
                                                       const T* __restrict__ dy, const T* __restrict__ dstate,
                                                       T* __restrict__ dx, T* __restrict__ dstate_in,
                                                       float* __restrict__ part) {
  using V = Vec<T, VEC>;
  const int tx = threadIdx.x % a.tx, ty = threadIdx.x / a.tx, strips = kThreads / a.tx;
  const int c = (blockIdx.y * a.tx + tx) * VEC;
  if (c >= a.C) return;
  Taps<T, VEC, K> taps;
  if (blockIdx.x >= a.strip_blocks) {
    // gradients of the rows before a window: of its first K - 1 rows' dz, and of what it handed on
    const int w = (int)(blockIdx.x - a.strip_blocks) * strips + ty;
    if (w >= a.win.W) return;
    taps.load(a, c);
    const int b = a.win.edge(w), rows = max(a.win.edge(w + 1) - b, 0);
    Place at;
    at.w = w;
    at.begin = b;
    at.end = b + rows;
    float h[K][VEC], g[K][VEC] = {};
    before<T, VEC, K>(a, at, b, x, state, c, h);
#pragma unroll
    for (int t = 0; t < K - 1; ++t) {
      if (t >= rows) break;
      const int row = a.win.row(b + t);
      float dz[VEC], z[VEC];
      V::wide(row >= 0 ? V::load(x + row * a.ldx + c) : V::zero(), h[K - 1]);
      V::wide(row >= 0 ? V::load(dy + row * a.lddy + c) : V::zero(), dz);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        z[e] = taps.b[e];
#pragma unroll
        for (int j = 0; j < K; ++j) z[e] = __builtin_fmaf(taps.w[j][e], h[j][e], z[e]);
      }
      slope_all(a.act, z, dz);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (row >= 0)
#pragma unroll
          for (int j = 0; j < K - 1 - t; ++j) g[t + j][e] = __builtin_fmaf(taps.w[j][e], dz[e], g[t + j][e]);
#pragma unroll
        for (int j = 0; j < K - 1; ++j) h[j][e] = h[j + 1][e];
      }
    }
#pragma unroll
    for (int i = 0; i < K - 1; ++i) {
      if (i >= rows && dstate != nullptr) {
        float d[VEC];
        V::wide(V::load(dstate + ((size_t)w * (K - 1) + i - rows) * a.C + c), d);
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[i][e] += d[e];
      }
      V::store(dstate_in + ((size_t)w * (K - 1) + i) * a.C + c, g[i]);
    }
    return;
  }
  const int strip = (int)blockIdx.x * strips + ty;
  if (strip >= a.strips) return;
  const int ps = strip * a.per, pe = min(ps + a.per, a.win.n), last = pe + K - 1;
  taps.load(a, c);
  Place at;
  at.at(a.win, ps);
  float h[K][VEC], acc[K][VEC] = {}, dw[K][VEC] = {}, db[VEC] = {};
  uint32_t live = 0;   // bit j: position p - K + 1 + j is a row of a window
  before<T, VEC, K>(a, at, ps, x, state, c, h);
  typename V::R nx[kBatch], nd[kBatch];
  int nr[kBatch];
  const auto ask = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      nr[i] = p0 + i < min(last, a.win.n) ? a.win.row(p0 + i) : -1;
      nx[i] = nr[i] >= 0 ? V::load(x + nr[i] * a.ldx + c) : V::zero();
      nd[i] = nr[i] >= 0 ? V::load(dy + nr[i] * a.lddy + c) : V::zero();
    }
  };
  ask(ps);
  for (int p0 = ps; p0 < last; p0 += kBatch) {
    typename V::R rx[kBatch], rd[kBatch];
    int row[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) rx[i] = nx[i], rd[i] = nd[i], row[i] = nr[i];
    ask(p0 + kBatch);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int p = p0 + i;
      if (p < last) {
        if (p < a.win.n && at.to(a.win, p)) from_state<T, VEC, K>(a, at.w, state, c, h);
        // a position whose order names no row is a row of zeros that has no result, as in the forward
        const bool in = at.in(p) && row[i] >= 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[K - 1][e] = 0.f;
        live = live >> 1 | (in ? 1u << (K - 1) : 0u);
        V::wide(rx[i], h[K - 1]);
        if (in) {
          float d[VEC], z[VEC];
          V::wide(rd[i], d);
          if (dstate != nullptr && p >= at.end - (K - 1))
            V::wide(V::load(dstate + ((size_t)at.w * (K - 1) + p - (at.end - (K - 1))) * a.C + c), acc[K - 1]);
          const bool own = p < pe;
          const int t = p - at.begin;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            z[e] = taps.b[e];
#pragma unroll
            for (int j = 0; j < K; ++j) z[e] = __builtin_fmaf(taps.w[j][e], h[j][e], z[e]);
          }
          slope_all(a.act, z, d);
          if (own) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              db[e] += d[e];
#pragma unroll
              for (int j = 0; j < K; ++j) dw[j][e] = __builtin_fmaf(d[e], h[j][e], dw[j][e]);
            }
          }
#pragma unroll
          for (int j = 0; j < K; ++j)
            if (t >= K - 1 - j)
#pragma unroll
              for (int e = 0; e < VEC; ++e) acc[j][e] = __builtin_fmaf(taps.w[j][e], d[e], acc[j][e]);
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) h[j][e] = h[j + 1][e];
        const int q = p - (K - 1);
        if (q >= ps && (live & 1u)) V::store(dx + (size_t)a.win.row(q) * a.C + c, acc[0]);
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[j][e] = acc[j + 1][e];
      }
    }
  }
  float* out = part + (size_t)strip * (K + 1) * a.C + c;
  using F = Vec<float, VEC>;
#pragma unroll
  for (int j = 0; j < K; ++j) F::store(out + (size_t)j * a.C, dw[j]);
  F::store(out + (size_t)K * a.C, db);
}

// Sums of the strips, in their order: 64 values a workgroup, eight runs of strips side by side.
__global__ __launch_bounds__(512) void k_conv_sums(const float* __restrict__ part, int32_t strips, int32_t C, int32_t K,
                                                   float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float s_sum[8][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t values = (int64_t)C * (K + 1), at = (int64_t)blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (at < values) {
    const int lo = (int)((int64_t)strips * g / 8), hi = (int)((int64_t)strips * (g + 1) / 8);
#pragma unroll 8
    for (int s = lo; s < hi; ++s) sum += part[s * values + at];
  }
  s_sum[g][lane] = sum;
  __syncthreads();
  if (g || at >= values) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) sum += s_sum[i][lane];
  const int j = (int)(at / C), c = (int)(at % C);
  if (j < K) dw[(size_t)c * K + j] = sum;
  else if (db != nullptr) db[c] = sum;
}

// Single rows: a state is K - 1 rows, read, used and moved by one; bound by memory and, for few rows, by the
// launch.
template <typename T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_step(ConvArgs a, const int32_t* __restrict__ slots, int32_t num_slots,
                                                        T* __restrict__ state, const T* __restrict__ x,
                                                        T* __restrict__ y) {
  using V = Vec<T, VEC>;
  __shared__ int s_table[2 * (kThreads / 64)];
  int b = blockIdx.x;
  const int slot = slots[b];
  if (slot < 0 || slot >= num_slots) return;   // padding: nothing is touched
  const SlotRows<kThreads / 64> rows{slots, a.win.n, s_table};
  const int c = (blockIdx.y * kThreads + threadIdx.x) * VEC;
  const bool live = c < a.C;
  T* st = state + (size_t)slot * (K - 1) * a.C + c;
  typename V::R r[K];
  Taps<T, VEC, K> taps;
  if (live) {
    taps.load(a, c);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) r[j] = V::load(st + (size_t)j * a.C);
    r[K - 1] = V::load(x + b * a.ldx + c);
  }
  for (bool first = true;; first = false) {
    const int next = rows.next(b, slot, first);
    if (next < 0) return;
    if (live) {
      float z[VEC], h[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[e] = taps.b[e];
#pragma unroll
      for (int j = 0; j < K; ++j) {
        V::wide(r[j], h);
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = __builtin_fmaf(taps.w[j][e], h[e], z[e]);
      }
      act_all(a.act, z);
      V::store(y + (size_t)b * a.C + c, z);
#pragma unroll
      for (int j = 0; j < K - 1; ++j) r[j] = r[j + 1];
    }
    if (next >= a.win.n) break;
    b = next;
    if (live) r[K - 1] = V::load(x + b * a.ldx + c);
  }
  if (live)
#pragma unroll
    for (int j = 0; j < K - 1; ++j) *reinterpret_cast<typename V::R*>(st + (size_t)j * a.C) = r[j];
}

int64_t lanes_of(int32_t C, int dtype) { return dtype == 0 ? ((int64_t)C + 3) / 4 : ((int64_t)C + 7) / 8; }

int rows_per_strip(int64_t n, int32_t C, int dtype) {
  // strips for 2^17 threads (two waves a SIMD) and more, short enough that the K - 1 rows beside their ends cost
  // little (the forward above: half as many strips 152 us, twice 123; its gradients: 136, 181 at four times)
  const int64_t threads = n * lanes_of(C, dtype);
  int64_t per = (threads >> 17) / 8 * 8;
  per = per < 16 ? 16 : per > 256 ? 256 : per;
  return (int)per;
}

// The strips of any number of rows up to n, of which there are fewer where strips get longer.  A strip of `per` = 16
// to 248 rows means fewer than (per + 8) 2^17 / lanes rows, so at most 1.5 2^17 / lanes strips.
int64_t most_strips(int64_t n, int32_t C, int dtype) {
  const int64_t lanes = lanes_of(C, dtype), some = ((3 << 16) + lanes - 1) / lanes;
  return std::max(std::min((n + 15) / 16, some), (n + 255) / 256);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Vectors of 16 bytes where widths, strides and addresses allow.
template <typename T, int kVec = 16 / sizeof(T)>
bool wide_rows(int32_t C, int64_t ldx, int64_t lddy, std::initializer_list<const void*> ps) {
  if (C % kVec || ldx % kVec || lddy % kVec) return false;
  for (const void* p : ps)
    if (!aligned16(p)) return false;
  return true;
}

template <class F>
void by_width(int K, F f) {
  switch (K) {
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    case 5: f(std::integral_constant<int, 5>{}); break;
    case 6: f(std::integral_constant<int, 6>{}); break;
    case 7: f(std::integral_constant<int, 7>{}); break;
    default: f(std::integral_constant<int, 8>{}); break;
  }
}

// Threads across the channels and the grid of a call that walks strips, with a workgroup row for states.
dim3 strip_grid(ConvArgs& a, int vec, int dtype, bool states) {
  const int32_t lanes = (a.C + vec - 1) / vec;
  a.tx = 1;
  while (a.tx < lanes && a.tx < kThreads) a.tx *= 2;
  const int32_t each = kThreads / a.tx;
  a.per = rows_per_strip(a.win.n, a.C, dtype);
  a.strips = (int32_t)(((int64_t)a.win.n + a.per - 1) / a.per);
  a.strip_blocks = (uint32_t)((a.strips + each - 1) / each);
  return dim3(a.strip_blocks + (states ? (uint32_t)((a.win.W + each - 1) / each) : 0u), (lanes + a.tx - 1) / a.tx);
}

template <typename T>
void forward_impl(ConvArgs a, int dtype, int K, const void* x, const void* state, void* y, void* state_out,
                  hipStream_t stream) {
  const auto run = [&](auto vec) {
    constexpr int VEC = decltype(vec)::value;
    const dim3 grid = strip_grid(a, VEC, dtype, state_out != nullptr);
    if (grid.x == 0) return;
    by_width(K, [&](auto k) {
      k_conv_fwd<T, VEC, decltype(k)::value><<<grid, kThreads, 0, stream>>>(
          a, static_cast<const T*>(x), static_cast<const T*>(state), static_cast<T*>(y), static_cast<T*>(state_out));
    });
  };
  if (wide_rows<T>(a.C, a.ldx, 0, {x, state, y, state_out, a.w})) run(std::integral_constant<int, 16 / sizeof(T)>{});
  else run(std::integral_constant<int, 1>{});
}

template <typename T>
void backward_impl(ConvArgs a, int dtype, int K, const void* x, const void* state, const void* dy, const void* dstate,
                   void* dx, float* dw, float* db, void* dstate_in, float* part, hipStream_t stream) {
  const auto run = [&](auto vec) {
    constexpr int VEC = decltype(vec)::value;
    const dim3 grid = strip_grid(a, VEC, dtype, dstate_in != nullptr);
    if (grid.x)
      by_width(K, [&](auto k) {
        k_conv_bwd<T, VEC, decltype(k)::value><<<grid, kThreads, 0, stream>>>(
            a, static_cast<const T*>(x), static_cast<const T*>(state), static_cast<const T*>(dy),
            static_cast<const T*>(dstate), static_cast<T*>(dx), static_cast<T*>(dstate_in), part);
      });
    const uint32_t blocks = (uint32_t)(((int64_t)a.C * (K + 1) + 63) / 64);
    k_conv_sums<<<blocks, 512, 0, stream>>>(part, a.strips, a.C, K, dw, db);
  };
  if (wide_rows<T, 4>(a.C, a.ldx, a.lddy, {x, state, dy, dstate, dx, dstate_in, a.w}))
    run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 1>{});
}

template <typename T>
void step_impl(const ConvArgs& a, int K, const int32_t* slots, int32_t num_slots, void* state, const void* x, void* y,
               hipStream_t stream) {
  const auto run = [&](auto vec) {
    constexpr int VEC = decltype(vec)::value;
    const dim3 grid(a.win.n, (a.C + kThreads * VEC - 1) / (kThreads * VEC));
    by_width(K, [&](auto k) {
      k_conv_step<T, VEC, decltype(k)::value><<<grid, kThreads, 0, stream>>>(
          a, slots, num_slots, static_cast<T*>(state), static_cast<const T*>(x), static_cast<T*>(y));
    });
  };
  if (wide_rows<T>(a.C, a.ldx, 0, {x, state, y, a.w})) run(std::integral_constant<int, 16 / sizeof(T)>{});
  else run(std::integral_constant<int, 1>{});
}

}  // namespace

size_t conv_backward_workspace_bytes(int64_t n, int dtype, int32_t C, int32_t K) {
  return align_up((size_t)most_strips(n, C, dtype) * (K + 1) * C * 4 + 256, 256);
}

hipError_t launch_forward_conv(const int32_t* offsets, int32_t n, int32_t W, const int32_t* order, int dtype, int32_t C,
                               int32_t K, int activation, const void* x, int64_t ldx, const float* weight,
                               const float* bias, const void* state_in, void* y, void* state_out, hipStream_t stream) {
  const ConvArgs a{{offsets, order, n, W}, weight, bias, ldx, 0, C, activation, 0, 0, 0, 0};
  if (dtype == 0) forward_impl<float>(a, dtype, K, x, state_in, y, state_out, stream);
  else if (dtype == 1) forward_impl<_Float16>(a, dtype, K, x, state_in, y, state_out, stream);
  else forward_impl<bf16_t>(a, dtype, K, x, state_in, y, state_out, stream);
  return hipGetLastError();
}

hipError_t launch_backward_conv(const int32_t* offsets, int32_t n, int32_t W, const int32_t* order, int dtype, int32_t C,
                                int32_t K, int activation, const void* x, int64_t ldx, const float* weight,
                                const float* bias, const void* state_in, const void* dy, int64_t lddy,
                                const void* dstate_out, void* dx, float* dweight, float* dbias, void* dstate_in,
                                void* workspace, hipStream_t stream) {
  const ConvArgs a{{offsets, order, n, W}, weight, bias, ldx, lddy, C, activation, 0, 0, 0, 0};
  float* part = static_cast<float*>(workspace);
  if (dtype == 0)
    backward_impl<float>(a, dtype, K, x, state_in, dy, dstate_out, dx, dweight, dbias, dstate_in, part, stream);
  else if (dtype == 1)
    backward_impl<_Float16>(a, dtype, K, x, state_in, dy, dstate_out, dx, dweight, dbias, dstate_in, part, stream);
  else
    backward_impl<bf16_t>(a, dtype, K, x, state_in, dy, dstate_out, dx, dweight, dbias, dstate_in, part, stream);
  return hipGetLastError();
}

hipError_t launch_step_conv(const int32_t* slots, int32_t n, int32_t num_slots, int dtype, int32_t C, int32_t K,
                            int activation, void* state, const void* x, int64_t ldx, const float* weight,
                            const float* bias, void* y, hipStream_t stream) {
  const ConvArgs a{{nullptr, nullptr, n, 0}, weight, bias, ldx, 0, C, activation, 0, 0, 0, 0};
  if (dtype == 0) step_impl<float>(a, K, slots, num_slots, state, x, y, stream);
  else if (dtype == 1) step_impl<_Float16>(a, K, slots, num_slots, state, x, y, stream);
  else step_impl<bf16_t>(a, K, slots, num_slots, state, x, y, stream);
  return hipGetLastError();
}

}  // namespace sla
