// Group normalisation of rows with an activation, channels last, and its gradients.
//
// For window s and channel group j, over the m rows of the window and the cg channels of the group:
//     mean = sum x / (m cg),  rstd = 1 / sqrt(sum (x - mean)^2 / (m cg) + eps),
//     y = act(z),  z = weight xhat + bias,  xhat = (x - mean) rstd;
// without windows every row is one.  Backward, with dz = dy act'(z):
//     dweight = sum dz xhat,  dbias = sum dz  over all rows,
//     dx = rstd (weight dz - A - xhat B),  A, B the means of weight dz and weight dz xhat.
//
// Bound by memory: x is read once from HBM for the statistics and, where the window does not stay
// in registers, once more from the caches.  Three forms, by what a window is:
//   rows     every row a window: a row's vectors stay in registers between the sums and the result;
//   windows  windows of few rows (at most kShortRows on average): a workgroup goes through whole
//            windows, so one launch does (the second read of a window comes from L2);
//   long     few long windows: blocks of rows of all windows at once, their sums joined by a small
//            launch, then the results by blocks of rows.
// Measured (a copy reaches 5.2 TB/s): rows, 32,768 of 2,048 bf16 channels: 63 us, 4.3 TB/s; long, 240,011
// rows of 256 bf16 channels in 4 windows: 37 + 6 + 47 us, 2.7 TB/s of what has to move (x comes in twice);
// gradients of 59,837 rows of 128 channels: long (fp16, one window) 12 + 7 + 11 us, windows (fp32, 1,521)
// 34 + 6 us, 2.3 TB/s.
// Variances are sums of squares around a mean, never differences of sums: a thread merges its
// vectors' means and squares one by one, threads and blocks are joined around the common mean.
#include <algorithm>

#include "sla_act.h"
#include "sla_common.h"

namespace sla {
namespace {

constexpr int kThreads = 256, kWavesN = 4;
constexpr int kMaxVectors = 1024;          // channels / 4 at most

struct NormArgs {
  const int32_t* offsets;   // null: every row is a window
  const float *weight, *bias;
  int32_t n, S, C, G;
  int32_t cv, cgv;          // vectors of a row, of a group
  int32_t tpr, rp;          // threads of a row, rows of a workgroup's pass
  int32_t rows_per;         // rows of a block (long form)
  float eps;
  int32_t act;
};

struct Seg {
  int32_t begin, rows;
};
__device__ __forceinline__ Seg segment(const NormArgs& a, int s) {
  if (a.offsets == nullptr) return {s, 1};
  int b = a.offsets[s], e = a.offsets[s + 1];
  b = b < 0 ? 0 : b > a.n ? a.n : b;
  e = e < b ? b : e > a.n ? a.n : e;
  return {b, e - b};
}
// Block `slot` of the long form: window s has the blocks begin / rows_per + s and following ones
// (blocks of different windows never share a number).  False where there is none.
__device__ __forceinline__ bool block_of(const NormArgs& a, uint32_t slot, int& s, int& begin, int& rows) {
  int lo = 0, hi = a.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((uint32_t)(segment(a, mid).begin / a.rows_per) + (uint32_t)mid <= slot) lo = mid;
    else hi = mid;
  }
  const Seg g = segment(a, lo);
  const uint32_t f = (uint32_t)(g.begin / a.rows_per) + (uint32_t)lo;
  if (slot < f || (int64_t)(slot - f) * a.rows_per >= g.rows) return false;
  s = lo;
  begin = g.begin + (int)(slot - f) * a.rows_per;
  rows = min(a.rows_per, g.rows - (int)(slot - f) * a.rows_per);
  return true;
}

// ------------------------------------------------------------------ sums over a group
// Every thread's value for each of its NV vectors, summed over the threads of the vector's group;
// over all rows of the pass too unless ROW.  Where rows and groups are powers of two and one vector
// a thread does, by lane exchanges and one table over the waves; else by a table over the threads.
template <int NV>
struct GroupSum {
  float* table;   // kMaxVectors floats and kMaxVectors results
  bool fast;
  int tid, r, cv;

  // two sums at once
  template <bool ROW>
  __device__ __forceinline__ void sum(const NormArgs& a, bool live, float (&x)[NV], float (&z)[NV]) const {
    if (NV == 1 && fast) {
      const int lane = tid & 63, wave = tid >> 6;
      float y0 = live ? x[0] : 0.f, y1 = live ? z[0] : 0.f;
      const int in = a.cgv < 64 ? a.cgv : 64;
      for (int m = 1; m < in; m *= 2) y0 += __shfl_xor(y0, m), y1 += __shfl_xor(y1, m);
      if constexpr (!ROW)
        for (int m = a.tpr; m < 64; m *= 2) y0 += __shfl_xor(y0, m), y1 += __shfl_xor(y1, m);
      if (ROW ? a.cgv > 64 : true) {
        const int nw = a.tpr > 64 ? a.tpr / 64 : 1, bpg = a.cgv > 64 ? a.cgv / 64 : 1;
        const int mine = wave % nw / bpg;
        const int at = (lane % (a.tpr < 64 ? a.tpr : 64)) / in;
        __syncthreads();
        if (lane % in == 0) table[wave * 64 + at] = y0, table[256 + wave * 64 + at] = y1;
        __syncthreads();
        y0 = y1 = 0.f;
#pragma unroll
        for (int w = 0; w < kWavesN; ++w)
          if (w % nw / bpg == mine && (!ROW || w / nw == wave / nw))
            y0 += table[w * 64 + at], y1 += table[256 + w * 64 + at];
      }
      x[0] = y0;
      z[0] = y1;
      return;
    }
    sum<ROW>(a, live, x);
    sum<ROW>(a, live, z);
  }

  template <bool ROW>
  __device__ __forceinline__ void sum(const NormArgs& a, bool live, float (&x)[NV]) const {
    const int lane = tid & 63, wave = tid >> 6;
    if (NV == 1 && fast) {
      float y = live ? x[0] : 0.f;
      const int in = a.cgv < 64 ? a.cgv : 64;
      for (int m = 1; m < in; m *= 2) y += __shfl_xor(y, m);
      if constexpr (!ROW)
        for (int m = a.tpr; m < 64; m *= 2) y += __shfl_xor(y, m);
      const bool across = ROW ? a.cgv > 64 : true;
      if (across) {
        const int nw = a.tpr > 64 ? a.tpr / 64 : 1, bpg = a.cgv > 64 ? a.cgv / 64 : 1;
        const int mine = wave % nw / bpg;
        const int at = (lane % (a.tpr < 64 ? a.tpr : 64)) / in;
        __syncthreads();
        if (lane % in == 0) table[wave * 64 + at] = y;
        __syncthreads();
        y = 0.f;
#pragma unroll
        for (int w = 0; w < kWavesN; ++w)
          if (w % nw / bpg == mine && (!ROW || w / nw == wave / nw)) y += table[w * 64 + at];
      }
      x[0] = y;
      return;
    }
    // thread tid's vectors at tid + 256 j: with several vectors a thread there is one row a pass
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = tid + kThreads * j;
      if (NV == 1 || at < a.cv) table[at] = live ? x[j] : 0.f;
    }
    __syncthreads();
    float* out = table + kMaxVectors;
    const int rows = a.rp, sums = ROW ? a.G * rows : a.G;
    if (a.cgv <= 16) {
      for (int q = tid; q < sums; q += kThreads) {
        const int grp = q % a.G, row = q / a.G;
        float y = 0.f;
        for (int p = ROW ? row : 0; p < (ROW ? row + 1 : rows); ++p)
          for (int c = 0; c < a.cgv; ++c) y += table[p * a.tpr + grp * a.cgv + c];
        out[q] = y;
      }
    } else {
      for (int q = wave; q < sums; q += kWavesN) {
        const int grp = q % a.G, row = q / a.G;
        float y = 0.f;
        for (int p = ROW ? row : 0; p < (ROW ? row + 1 : rows); ++p)
          for (int c = lane; c < a.cgv; c += 64) y += table[p * a.tpr + grp * a.cgv + c];
        for (int m = 1; m < 64; m *= 2) y += __shfl_xor(y, m);
        if (lane == 0) out[q] = y;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = cv + kThreads * j;
      if (live && c < a.cv) x[j] = out[(ROW ? r * a.G : 0) + c / a.cgv];
    }
  }
};

template <int NV>
__device__ __forceinline__ GroupSum<NV> group_sum(const NormArgs& a, float* table) {
  const int tid = threadIdx.x;
  const auto pow2 = [](int x) { return (x & (x - 1)) == 0; };
  return {table, pow2(a.tpr) && pow2(a.cgv), tid, tid / a.tpr, tid % a.tpr};
}

template <typename T, int VEC>
__device__ __forceinline__ void load(const T* p, float (&x)[VEC]) {
  Frag<T, VEC>::to_f32(*reinterpret_cast<const Raw<T, VEC>*>(p), x);
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T* p, const float (&x)[VEC]) {
  *reinterpret_cast<Raw<T, VEC>*>(p) = Frag<T, VEC>::from_f32(x);
}
template <int VEC>
__device__ __forceinline__ void params(const float* w, int c, float fill, float (&x)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; e += 4) {
    const floatx4 y = w ? *reinterpret_cast<const floatx4*>(w + c + e) : floatx4{fill, fill, fill, fill};
#pragma unroll
    for (int r = 0; r < 4; ++r) x[e + r] = y[r];
  }
}

// Means and squares around them of the vectors a thread has seen: merged vector by vector, k of VEC
// values each.
template <int VEC>
struct Moments {
  float mean = 0.f, m2 = 0.f;
  __device__ __forceinline__ void add(const float (&x)[VEC], int k) {   // the k-th vector, from 0
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) s += x[e];
    const float m = s * (1.f / VEC);
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) q += (x[e] - m) * (x[e] - m);
    const float d = m - mean, f = 1.f / (float)(k + 1);
    mean += d * f;
    m2 += q + d * d * ((float)VEC * (float)k * f);
  }
};

// ------------------------------------------------------------------ rows and windows, forward
template <typename T, int VEC, int NV, bool ROWS>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(NormArgs a, const T* __restrict__ x, T* __restrict__ y,
                                                       float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_table[2 * kMaxVectors];
  const GroupSum<NV> gs = group_sum<NV>(a, s_table);
  const bool in = gs.r < a.rp;
  const int step = ROWS ? a.rp : 1;
  float w[NV][VEC], b[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = min(gs.cv + kThreads * j, a.cv - 1) * VEC;
    params<VEC>(a.weight, c, 1.f, w[j]);
    params<VEC>(a.bias, c, 0.f, b[j]);
  }
  // rows: the next row's vectors are asked for before this one's sums
  Raw<T, VEC> ahead[ROWS ? NV : 1];
  const auto ask = [&](int s) __attribute__((always_inline)) {
    if constexpr (ROWS)
#pragma unroll
      for (int j = 0; j < NV; ++j)
        ahead[j] = *reinterpret_cast<const Raw<T, VEC>*>(x + (size_t)min(s, a.S - 1) * a.C +
                                                         min(gs.cv + kThreads * j, a.cv - 1) * VEC);
  };
  ask(blockIdx.x * step + gs.r);
  for (int s0 = blockIdx.x * step; s0 < a.S; s0 += gridDim.x * step) {
    const int s = ROWS ? s0 + gs.r : s0;
    const bool live = in && (!ROWS || s < a.S);
    const Seg seg = ROWS ? Seg{min(s, a.S - 1), 1} : segment(a, s);
    if (!ROWS && seg.rows == 0) {
      for (int q = threadIdx.x; q < a.G; q += kThreads) {
        mean[(size_t)s * a.G + q] = 0.f;
        rstd[(size_t)s * a.G + q] = 1.f / sqrtf(a.eps);
      }
      continue;
    }
    const int first = ROWS ? 0 : gs.r;
    float v[NV][VEC];
    float total[NV], sq[NV];
    const float inv = 1.f / ((float)seg.rows * (float)(a.cgv * VEC));
    Moments<VEC> mo[NV];
    int k = 0;
    if constexpr (ROWS) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        Frag<T, VEC>::to_f32(ahead[j], v[j]);
        mo[j].add(v[j], 0);
      }
      k = 1;
      ask(s + gridDim.x * step);
    } else if (live) {
      for (int r = first; r < seg.rows; r += a.rp, ++k)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = gs.cv + kThreads * j;
          if (NV > 1 && c >= a.cv) continue;
          load<T, VEC>(x + (size_t)(seg.begin + r) * a.C + c * VEC, v[j]);
          mo[j].add(v[j], k);
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) total[j] = mo[j].mean * ((float)k * VEC);
    gs.template sum<ROWS>(a, live, total);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      total[j] *= inv;
      const float d = mo[j].mean - total[j];
      sq[j] = mo[j].m2 + d * d * ((float)k * VEC);
    }
    gs.template sum<ROWS>(a, live, sq);
    if (!live) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = gs.cv + kThreads * j;
      if (NV > 1 && c >= a.cv) continue;
      sq[j] = 1.f / sqrtf(sq[j] * inv + a.eps);
      if (first == 0 && c % a.cgv == 0) {
        mean[(size_t)s * a.G + c / a.cgv] = total[j];
        rstd[(size_t)s * a.G + c / a.cgv] = sq[j];
      }
    }
    for (int r = first; r < seg.rows; r += ROWS ? 1 : a.rp)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = gs.cv + kThreads * j;
        if (NV > 1 && c >= a.cv) continue;
        const size_t at = (size_t)(seg.begin + r) * a.C + c * VEC;
        if constexpr (!ROWS) load<T, VEC>(x + at, v[j]);
        float z[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = act(a.act, (v[j][e] - total[j]) * sq[j] * w[j][e] + b[j][e]);
        store<T, VEC>(y + at, z);
      }
  }
}

// ------------------------------------------------------------------ rows and windows, backward
// The workgroup's sums of dz and dz xhat by channel go to part[block][C][2] when it is done.
template <int VEC, int NV>
__device__ __forceinline__ void put_channels(const NormArgs& a, const GroupSum<NV>& gs, const float (&db)[NV][VEC],
                                             const float (&dw)[NV][VEC], float* s_rows, float* part) {
  // over the rows of the pass, 2 values of each vector slot at a time: rp x tpr threads
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (a.rp == 1) {
        const int c = gs.cv + kThreads * j;
        if (gs.r < a.rp && c < a.cv) {
          part[2 * (c * VEC + e)] = db[j][e];
          part[2 * (c * VEC + e) + 1] = dw[j][e];
        }
        continue;
      }
      __syncthreads();
      s_rows[gs.tid] = db[j][e];
      s_rows[kThreads + gs.tid] = dw[j][e];
      __syncthreads();
      if (gs.tid < 2 * a.tpr) {
        const int which = gs.tid >= a.tpr, c = gs.tid - which * a.tpr;
        float y = 0.f;
        for (int r = 0; r < a.rp; ++r) y += s_rows[which * kThreads + r * a.tpr + c];
        part[2 * (c * VEC + e) + which] = y;
      }
    }
}

template <typename T, int VEC, int NV, bool ROWS>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(NormArgs a, const T* __restrict__ x, const T* __restrict__ dy,
                                                       const float* __restrict__ mean, const float* __restrict__ rstd,
                                                       T* __restrict__ dx, float* __restrict__ part) {
  __shared__ float s_table[2 * kMaxVectors];
  const GroupSum<NV> gs = group_sum<NV>(a, s_table);
  const bool in = gs.r < a.rp;
  const int step = ROWS ? a.rp : 1;
  float w[NV][VEC], b[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = min(gs.cv + kThreads * j, a.cv - 1) * VEC;
    params<VEC>(a.weight, c, 1.f, w[j]);
    params<VEC>(a.bias, c, 0.f, b[j]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  for (int s0 = blockIdx.x * step; s0 < a.S; s0 += gridDim.x * step) {
    const int s = ROWS ? s0 + gs.r : s0;
    const bool live = in && (!ROWS || s < a.S);
    const Seg seg = ROWS ? Seg{min(s, a.S - 1), 1} : segment(a, s);
    if (!ROWS && seg.rows == 0) continue;
    const int first = ROWS ? 0 : gs.r;
    const float inv = 1.f / ((float)seg.rows * (float)(a.cgv * VEC));
    float hat[NV][VEC], dz[NV][VEC], mu[NV], rs[NV], sa[NV], sb[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = min(gs.cv + kThreads * j, a.cv - 1), q = c / a.cgv;
      mu[j] = live ? mean[(size_t)s * a.G + q] : 0.f;
      rs[j] = live ? rstd[(size_t)s * a.G + q] : 0.f;
      sa[j] = sb[j] = 0.f;
    }
    const auto row = [&](int r, int j) {   // xhat and dz of a vector
      const size_t at = (size_t)(seg.begin + r) * a.C + (gs.cv + kThreads * j) * VEC;
      load<T, VEC>(x + at, hat[j]);
      load<T, VEC>(dy + at, dz[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        hat[j][e] = (hat[j][e] - mu[j]) * rs[j];
        dz[j][e] *= slope(a.act, hat[j][e] * w[j][e] + b[j][e]);
      }
    };
    if (live)
      for (int r = first; r < seg.rows; r += ROWS ? 1 : a.rp)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          if (NV > 1 && gs.cv + kThreads * j >= a.cv) continue;
          row(r, j);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            db[j][e] += dz[j][e];
            dw[j][e] += dz[j][e] * hat[j][e];
            sa[j] += dz[j][e] * w[j][e];
            sb[j] += dz[j][e] * w[j][e] * hat[j][e];
          }
        }
    gs.template sum<ROWS>(a, live, sa, sb);
    if (!live) continue;
    for (int r = first; r < seg.rows; r += ROWS ? 1 : a.rp)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = gs.cv + kThreads * j;
        if (NV > 1 && c >= a.cv) continue;
        if constexpr (!ROWS) row(r, j);
        float z[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = rs[j] * (dz[j][e] * w[j][e] - sa[j] * inv - hat[j][e] * (sb[j] * inv));
        store<T, VEC>(dx + (size_t)(seg.begin + r) * a.C + c * VEC, z);
      }
  }
  put_channels<VEC, NV>(a, gs, db, dw, s_table, part + (size_t)blockIdx.x * 2 * a.C);
}

// ------------------------------------------------------------------ long windows
// part[slot][G][2]: mean and squares around it of a block of rows
template <typename T, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_norm_part(NormArgs a, const T* __restrict__ x, float* __restrict__ part) {
  __shared__ float s_table[2 * kMaxVectors];
  int s, begin, rows;
  if (!block_of(a, blockIdx.x, s, begin, rows)) return;
  const GroupSum<NV> gs = group_sum<NV>(a, s_table);
  const bool live = gs.r < a.rp;
  const float inv = 1.f / ((float)rows * (float)(a.cgv * VEC));
  Moments<VEC> mo[NV];
  float total[NV], sq[NV];
  int k = 0;
  if (live)
#pragma unroll 4
    for (int r = gs.r; r < rows; r += a.rp, ++k)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = gs.cv + kThreads * j;
        if (NV > 1 && c >= a.cv) continue;
        float v[VEC];
        load<T, VEC>(x + (size_t)(begin + r) * a.C + c * VEC, v);
        mo[j].add(v, k);
      }
#pragma unroll
  for (int j = 0; j < NV; ++j) total[j] = mo[j].mean * ((float)k * VEC);
  gs.template sum<false>(a, live, total);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    total[j] *= inv;
    const float d = mo[j].mean - total[j];
    sq[j] = mo[j].m2 + d * d * ((float)k * VEC);
  }
  gs.template sum<false>(a, live, sq);
  if (gs.r == 0)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = gs.cv + kThreads * j;
      if (c < a.cv && c % a.cgv == 0) {
        float* p = part + ((size_t)blockIdx.x * a.G + c / a.cgv) * 2;
        p[0] = total[j];
        p[1] = sq[j];
      }
    }
}

// A workgroup for each window and 8 groups, 32 threads a group: the blocks' means and squares joined.
__global__ __launch_bounds__(kThreads) void k_norm_join(NormArgs a, const float* __restrict__ part,
                                                        float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_sum[2][32][9];
  const int s = blockIdx.x, t = threadIdx.x & 7, q = blockIdx.y * 8 + t, l = threadIdx.x >> 3;
  const Seg seg = segment(a, s);
  const bool live = q < a.G;
  const float2* p = reinterpret_cast<const float2*>(part) + (size_t)(seg.begin / a.rows_per + s) * a.G + min(q, a.G - 1);
  const int blocks = (seg.rows + a.rows_per - 1) / a.rows_per, cg = a.C / a.G;
  const float inv = seg.rows ? 1.f / ((float)seg.rows * (float)cg) : 0.f;
  const auto total = [&](int which, float x) __attribute__((always_inline)) {
    s_sum[which][l][t] = x;
    __syncthreads();
    float y = 0.f;
#pragma unroll
    for (int r = 0; r < 32; ++r) y += s_sum[which][r][t];
    return y;
  };
  float sum = 0.f;
#pragma unroll 8
  for (int b = l; b < blocks; b += 32)
    sum += p[(size_t)b * a.G].x * (float)(min(a.rows_per, seg.rows - b * a.rows_per) * cg);
  const float m = total(0, sum) * inv;
  float sq = 0.f;
#pragma unroll 8
  for (int b = l; b < blocks; b += 32) {
    const float2 v = p[(size_t)b * a.G];
    const float d = v.x - m;
    sq += v.y + d * d * (float)(min(a.rows_per, seg.rows - b * a.rows_per) * cg);
  }
  sq = total(1, sq);
  if (l == 0 && live) {
    mean[(size_t)s * a.G + q] = m;
    rstd[(size_t)s * a.G + q] = 1.f / sqrtf(sq * inv + a.eps);
  }
}

template <typename T, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_norm_apply(NormArgs a, const T* __restrict__ x,
                                                         const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, T* __restrict__ y) {
  int s, begin, rows;
  if (!block_of(a, blockIdx.x, s, begin, rows)) return;
  const int r0 = threadIdx.x / a.tpr, cv = threadIdx.x % a.tpr;
  if (r0 >= a.rp) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = cv + kThreads * j;
    if (NV > 1 && c >= a.cv) continue;
    float w[VEC], b[VEC];
    params<VEC>(a.weight, c * VEC, 1.f, w);
    params<VEC>(a.bias, c * VEC, 0.f, b);
    const float m = mean[(size_t)s * a.G + c / a.cgv], rs = rstd[(size_t)s * a.G + c / a.cgv];
#pragma unroll 4
    for (int r = r0; r < rows; r += a.rp) {
      const size_t at = (size_t)(begin + r) * a.C + c * VEC;
      float v[VEC];
      load<T, VEC>(x + at, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = act(a.act, (v[e] - m) * rs * w[e] + b[e]);
      store<T, VEC>(y + at, v);
    }
  }
}

// part[slot][C][2]: sums of dz and dz xhat over a block of rows
template <typename T, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_part(NormArgs a, const T* __restrict__ x,
                                                            const T* __restrict__ dy, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, float* __restrict__ part) {
  __shared__ float s_table[2 * kThreads];
  int s, begin, rows;
  if (!block_of(a, blockIdx.x, s, begin, rows)) return;
  const GroupSum<NV> gs = group_sum<NV>(a, s_table);
  float dw[NV][VEC], db[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = min(gs.cv + kThreads * j, a.cv - 1);
    float w[VEC], b[VEC];
    params<VEC>(a.weight, c * VEC, 1.f, w);
    params<VEC>(a.bias, c * VEC, 0.f, b);
    const float m = mean[(size_t)s * a.G + c / a.cgv], rs = rstd[(size_t)s * a.G + c / a.cgv];
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[j][e] = db[j][e] = 0.f;
    if (gs.r < a.rp && gs.cv + kThreads * j < a.cv)
#pragma unroll 2
      for (int r = gs.r; r < rows; r += a.rp) {
        const size_t at = (size_t)(begin + r) * a.C + c * VEC;
        float h[VEC], d[VEC];
        load<T, VEC>(x + at, h);
        load<T, VEC>(dy + at, d);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          h[e] = (h[e] - m) * rs;
          d[e] *= slope(a.act, h[e] * w[e] + b[e]);
          db[j][e] += d[e];
          dw[j][e] += d[e] * h[e];
        }
      }
  }
  put_channels<VEC, NV>(a, gs, db, dw, s_table, part + (size_t)blockIdx.x * 2 * a.C);
}

// 16 columns of `count` rows of C x 2 values summed by a workgroup, 64 threads a column, each row's
// values in the same order whatever the count: to out[C x 2], or, where that is null, dbias and dweight.
__device__ __forceinline__ void sum_columns(const float* rows, int count, int C, float* out, float* dweight,
                                            float* dbias) {
  __shared__ float s_sum[64][17];
  const int t = threadIdx.x & 15, col = blockIdx.y * 16 + t, rr = threadIdx.x >> 4;
  float y = 0.f;
  if (col < 2 * C)
#pragma unroll 8
    for (int b = rr; b < count; b += 64) y += rows[(size_t)b * C * 2 + col];
  s_sum[rr][t] = y;
  __syncthreads();
  if (rr == 0 && col < 2 * C) {
    y = 0.f;
#pragma unroll
    for (int r = 0; r < 64; ++r) y += s_sum[r][t];
    if (out != nullptr) out[col] = y;
    float* to = col & 1 ? dweight : dbias;
    if (to != nullptr) to[col >> 1] = y;
  }
}
// The blocks' sums of every window, to seg[S][C][2]; with one window they are dbias and dweight too.
__global__ __launch_bounds__(1024) void k_norm_bwd_join(NormArgs a, const float* __restrict__ part,
                                                        float* __restrict__ seg, float* __restrict__ dweight,
                                                        float* __restrict__ dbias) {
  const int s = blockIdx.x;
  const Seg g = segment(a, s);
  const int blocks = (g.rows + a.rows_per - 1) / a.rows_per;
  sum_columns(part + (size_t)(g.begin / a.rows_per + s) * a.C * 2, blocks, a.C, seg + (size_t)s * a.C * 2, dweight,
              dbias);
}
__global__ __launch_bounds__(1024) void k_norm_channels(const float* __restrict__ rows, int count, int C,
                                                        float* __restrict__ dweight, float* __restrict__ dbias) {
  sum_columns(rows, count, C, nullptr, dweight, dbias);
}

// dx of a block of rows.  A and B come from the window's channel sums, summed by the block itself.
template <typename T, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_apply(NormArgs a, const T* __restrict__ x,
                                                             const T* __restrict__ dy,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd,
                                                             const float* __restrict__ seg, T* __restrict__ dx) {
  __shared__ float s_table[2 * kMaxVectors];
  int s, begin, rows;
  if (!block_of(a, blockIdx.x, s, begin, rows)) return;
  const GroupSum<NV> gs = group_sum<NV>(a, s_table);
  const Seg g = segment(a, s);
  const float inv = 1.f / ((float)g.rows * (float)(a.cgv * VEC));
  float w[NV][VEC], sa[NV], sb[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = min(gs.cv + kThreads * j, a.cv - 1);
    params<VEC>(a.weight, c * VEC, 1.f, w[j]);
    sa[j] = sb[j] = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float* p = seg + ((size_t)s * a.C + c * VEC + e) * 2;
      sa[j] += w[j][e] * p[0];
      sb[j] += w[j][e] * p[1];
    }
    if (gs.r != 0) sa[j] = sb[j] = 0.f;   // a channel's sums once
  }
  const bool live = gs.r < a.rp;
  gs.template sum<false>(a, live, sa, sb);
  if (!live) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = gs.cv + kThreads * j;
    if (NV > 1 && c >= a.cv) continue;
    float b[VEC];
    params<VEC>(a.bias, c * VEC, 0.f, b);
    const float m = mean[(size_t)s * a.G + c / a.cgv], rs = rstd[(size_t)s * a.G + c / a.cgv];
    const float A = sa[j] * inv, B = sb[j] * inv;
#pragma unroll 2
    for (int r = gs.r; r < rows; r += a.rp) {
      const size_t at = (size_t)(begin + r) * a.C + c * VEC;
      float h[VEC], d[VEC];
      load<T, VEC>(x + at, h);
      load<T, VEC>(dy + at, d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        h[e] = (h[e] - m) * rs;
        d[e] *= slope(a.act, h[e] * w[j][e] + b[e]);
        d[e] = rs * (d[e] * w[j][e] - A - h[e] * B);
      }
      store<T, VEC>(dx + at, d);
    }
  }
}

// ------------------------------------------------------------------ host
// Rows of a window on average, up to which a workgroup takes it whole; above, blocks of rows.  Windows and
// blocks, forward and gradients with the launches' host time, 59,837 rows of 256 bf16 channels: windows of
// 40 rows 21 + 41 and 44 + 164 us, 128: 28 + 47 and 39 + 91, 256: 41 + 70 and 36 + 69, 1,024: 139 + 237 and
// 34 + 54; 6,000 rows: 128: 21 + 35 and 26 + 35, 256: 34 + 59 and 26 + 33.
constexpr int kShortRows = 160;
constexpr int kGroups = 2048;      // workgroups of the rows and windows forms (8 a CU)
constexpr int kBlocks = 1024;      // blocks of rows the long form aims at (4 a CU)

enum Form { kRowsForm, kWindowsForm, kLongForm };
struct Shape {
  Form form;
  int vec, nv, grid;
  NormArgs a;
};

Shape shape_of(const int32_t* offsets, bool windows, int32_t n, int32_t S, int dtype, int32_t C, int32_t G) {
  Shape s;
  NormArgs& a = s.a;
  a = NormArgs{};
  a.offsets = offsets;
  a.n = n, a.S = S, a.C = C, a.G = G;
  // 16-byte vectors where the groups allow it, else 4 values
  s.vec = dtype != 0 && (C / G) % 8 == 0 ? 8 : 4;
  a.cv = C / s.vec;
  a.cgv = C / G / s.vec;
  a.tpr = std::min(a.cv, kThreads);
  a.rp = kThreads / a.tpr;
  const int need = (a.cv + kThreads - 1) / kThreads;
  s.nv = need <= 1 ? 1 : need <= 2 ? 2 : 4;
  s.form = !windows ? kRowsForm : (int64_t)n <= (int64_t)kShortRows * S ? kWindowsForm : kLongForm;
  a.rows_per = std::max(16, (int)((n + (int64_t)kBlocks - 1) / kBlocks));
  const int64_t units = s.form == kRowsForm ? (S + a.rp - 1) / a.rp
                        : s.form == kWindowsForm ? S
                                                 : (int64_t)n / a.rows_per + S;
  s.grid = (int)(s.form == kLongForm ? units : std::min<int64_t>(units, kGroups));
  return s;
}

template <typename T, int VEC, int NV>
void forward_impl(const Shape& s, const void* xv, void* yv, float* mean, float* rstd, float* part, hipStream_t stream) {
  const T* x = static_cast<const T*>(xv);
  T* y = static_cast<T*>(yv);
  if (s.form == kRowsForm) {
    k_norm_fwd<T, VEC, NV, true><<<s.grid, kThreads, 0, stream>>>(s.a, x, y, mean, rstd);
  } else if (s.form == kWindowsForm) {
    k_norm_fwd<T, VEC, NV, false><<<s.grid, kThreads, 0, stream>>>(s.a, x, y, mean, rstd);
  } else {
    k_norm_part<T, VEC, NV><<<s.grid, kThreads, 0, stream>>>(s.a, x, part);
    k_norm_join<<<dim3(s.a.S, (s.a.G + 7) / 8), kThreads, 0, stream>>>(s.a, part, mean, rstd);
    k_norm_apply<T, VEC, NV><<<s.grid, kThreads, 0, stream>>>(s.a, x, mean, rstd, y);
  }
}

template <typename T, int VEC, int NV>
void backward_impl(const Shape& s, const void* xv, const void* dyv, const float* mean, const float* rstd, void* dxv,
                   float* dweight, float* dbias, float* part, hipStream_t stream) {
  const T *x = static_cast<const T*>(xv), *dy = static_cast<const T*>(dyv);
  T* dx = static_cast<T*>(dxv);
  const float* rows = part;
  int count = s.grid;
  if (s.grid == 0) {
    // no row: the channels' sums below are sums over nothing
  } else if (s.form == kRowsForm) {
    k_norm_bwd<T, VEC, NV, true><<<s.grid, kThreads, 0, stream>>>(s.a, x, dy, mean, rstd, dx, part);
  } else if (s.form == kWindowsForm) {
    k_norm_bwd<T, VEC, NV, false><<<s.grid, kThreads, 0, stream>>>(s.a, x, dy, mean, rstd, dx, part);
  } else {
    float* seg = part + (size_t)s.grid * s.a.C * 2;
    k_norm_bwd_part<T, VEC, NV><<<s.grid, kThreads, 0, stream>>>(s.a, x, dy, mean, rstd, part);
    const bool one = s.a.S == 1;
    k_norm_bwd_join<<<dim3(s.a.S, (2 * s.a.C + 15) / 16), 1024, 0, stream>>>(s.a, part, seg, one ? dweight : nullptr,
                                                                            one ? dbias : nullptr);
    k_norm_bwd_apply<T, VEC, NV><<<s.grid, kThreads, 0, stream>>>(s.a, x, dy, mean, rstd, seg, dx);
    if (one) return;
    rows = seg;
    count = s.a.S;
  }
  if (dweight != nullptr || dbias != nullptr)
    k_norm_channels<<<dim3(1, (2 * s.a.C + 15) / 16), 1024, 0, stream>>>(rows, count, s.a.C, dweight, dbias);
}

template <class F>
void by_shape(const Shape& s, int dtype, F f) {
  const auto nv = [&](auto type, auto vec) {
    if (s.nv == 1) f(type, vec, std::integral_constant<int, 1>{});
    else if (s.nv == 2) f(type, vec, std::integral_constant<int, 2>{});
    else f(type, vec, std::integral_constant<int, 4>{});
  };
  const std::integral_constant<int, 4> v4;
  const std::integral_constant<int, 8> v8;
  if (dtype == 0) nv(float{}, v4);
  else if (dtype == 1) s.vec == 8 ? nv(_Float16{}, v8) : nv(_Float16{}, v4);
  else s.vec == 8 ? nv(bf16_t{}, v8) : nv(bf16_t{}, v4);
}

}  // namespace

size_t norm_workspace_bytes(bool windows, int64_t n, int32_t S, int dtype, int32_t C, int32_t G, bool backward) {
  const Shape s = shape_of(nullptr, windows, (int32_t)n, S, dtype, C, G);
  if (backward) return ((size_t)s.grid + (s.form == kLongForm ? S : 0)) * C * 2 * 4 + 256;
  return s.form == kLongForm ? (size_t)s.grid * G * 2 * 4 + 256 : 256;
}

hipError_t launch_forward_group_norm(const int32_t* offsets, int32_t n, int32_t S, int dtype, int32_t C, int32_t G,
                                     float eps, int activation, const void* x, const float* weight, const float* bias,
                                     void* y, float* mean, float* rstd, void* workspace, hipStream_t stream) {
  Shape s = shape_of(offsets, offsets != nullptr, n, S, dtype, C, G);
  s.a.weight = weight, s.a.bias = bias, s.a.eps = eps, s.a.act = activation;
  by_shape(s, dtype, [&](auto type, auto vec, auto nv) {
    if constexpr (!(std::is_same<decltype(type), float>::value && decltype(vec)::value == 8))
      forward_impl<decltype(type), decltype(vec)::value, decltype(nv)::value>(s, x, y, mean, rstd,
                                                                            static_cast<float*>(workspace), stream);
  });
  return hipGetLastError();
}

hipError_t launch_backward_group_norm(const int32_t* offsets, int32_t n, int32_t S, int dtype, int32_t C, int32_t G,
                                      int activation, const void* x, const float* weight, const float* bias,
                                      const void* dy, const float* mean, const float* rstd, void* dx, float* dweight,
                                      float* dbias, void* workspace, hipStream_t stream) {
  Shape s = shape_of(offsets, offsets != nullptr, n, S, dtype, C, G);
  s.a.weight = weight, s.a.bias = bias, s.a.act = activation;
  by_shape(s, dtype, [&](auto type, auto vec, auto nv) {
    if constexpr (!(std::is_same<decltype(type), float>::value && decltype(vec)::value == 8))
      backward_impl<decltype(type), decltype(vec)::value, decltype(nv)::value>(
          s, x, dy, mean, rstd, dx, dweight, dbias, static_cast<float*>(workspace), stream);
  });
  return hipGetLastError();
}

}  // namespace sla
