// The normalisation between two blocks, row by row, and its gradients: the norm of a block's output, its
// gate and scale, the residual sum, and the norm the next block reads, in one pass.
//
// With rms(v) = v / sqrt(mean(v^2) + eps):
//     u = rms(x) post_weight (x without one),  r' = r + scale act(gate) u,  y = rms(r') weight;
// backward, with xhat = x post_rstd and rhat = r' rstd:
//     dr = dr' + rstd (dy weight - rhat mean(dy weight rhat)),  dweight = sum dy rhat,
//     dgate = scale dr u act'(gate),  du = scale dr act(gate),  dpost_weight = sum du xhat,
//     dx = post_rstd (du post_weight - xhat mean(du post_weight xhat))  (du without a norm).
//
// Bound by memory up to 4,096 channels: every row is loaded once and stays in registers through both norms; the next
// row of a workgroup is asked for before this one's sums.  Measured (a copy reaches 5.1 TB/s): 32,768 rows of 2,048
// bf16 channels with fp32 residual rows: 197 us, 4.8 TB/s; gradients of 16,381 rows of 4,096: 210 + 5 us, 5.1 TB/s.
// Wider rows, 5,120 and 8,192 channels: forward 4.1 and 4.4 TB/s, bf16 gradients 2.8 and 3.8 (454 to 506 registers,
// one wave a SIMD), fp32 gradients 1.6 and 1.8 (194 registers spilled).  Rows that are not 16-byte aligned take 4
// values a thread up to 1,024 channels, and 32 above, with 98 to 382 registers spilled: 0.2 to 1.0 TB/s at 1,025
// and 5,001 channels.
// The gradients' sums over rows are kept by each thread for its columns, written once for each workgroup, and added
// by a second launch in a fixed order.
#include <algorithm>

#include "sla_act.h"
#include "sla_rows.h"

namespace sla {
namespace {

constexpr int kThreads = 256;

struct RnormArgs {
  int64_t n;
  int32_t C, cv;          // channels, vectors of a row
  float eps, scale;
  int32_t act;
  const float *weight, *post;
};

// Sums over a row's threads; two tables in turn, so that one barrier a sum is enough.
template <int TPR>
struct RowSum {
  float* table;   // 2 x 4 floats
  int turn = 0;
  __device__ __forceinline__ float operator()(float x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6;
      float* t = table + 4 * turn;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) t[wave] = x;
      __syncthreads();
      x = (t[0] + t[1]) + (t[2] + t[3]);
    }
    return x;
  }
  __device__ __forceinline__ float largest(float x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x = fmaxf(x, __shfl_xor(x, m));
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6;
      float* t = table + 4 * turn;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) t[wave] = x;
      __syncthreads();
      x = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
    }
    return x;
  }
};

// 1 / sqrt(mean(v^2) + eps).  Where the squares leave fp32's range, once more with the row at the power of two
// of its largest value.
template <int TPR, int VEC, int NV>
__device__ __forceinline__ float inverse_rms(const RnormArgs& a, RowSum<TPR>& sum, const float (&v)[NV][VEC]) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) s = __builtin_fmaf(v[j][e], v[j][e], s);
  s = sum(s);
  const float inv = 1.f / (float)a.C;
  const float plain = 1.f / sqrtf(__builtin_fmaf(s, inv, a.eps));
  // small squares are lost only beside an eps that is as small
  if (s < 1e37f && (s > 1e-24f || a.eps > 1e-20f)) return plain;
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) m = fmaxf(m, fabsf(v[j][e]));
  m = sum.largest(m);
  if (s != s || !(m > 0.f && m <= 3.40282347e38f)) return plain;
  // eps goes with the squares: no further up than where it would leave the range instead (there it is all that counts)
  const int k = a.eps > 0.f ? max(ilogbf(m), -62) : ilogbf(m);
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float t = ldexpf(v[j][e], -k);
      q = __builtin_fmaf(t, t, q);
    }
  q = sum(q) * inv;
  return ldexpf(1.f / sqrtf(q + ldexpf(ldexpf(a.eps, -k), -k)), -k);
}

template <int VEC, int NV>
__device__ __forceinline__ void columns(const float* w, int C, const int (&c)[NV], float (&x)[NV][VEC]) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[j][e] = w == nullptr ? 1.f : c[j] >= 0 ? w[c[j] + e] : 0.f;
}

// NV vectors of VEC values a thread, TPR threads a row; c[j] the first channel of a vector, -1 past the row.
template <int TPR, int VEC, int NV>
__device__ __forceinline__ void my_columns(const RnormArgs& a, int (&c)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int v = threadIdx.x % TPR + TPR * j;
    c[j] = v < a.cv ? v * VEC : -1;
  }
}
template <typename T, int VEC, int NV>
__device__ __forceinline__ void ask(const T* p, int64_t row, int C, const int (&c)[NV],
                                    typename Vec<T, VEC>::R (&raw)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
    raw[j] = p != nullptr && c[j] >= 0 ? Vec<T, VEC>::load(p + row * C + c[j]) : Vec<T, VEC>::zero();
}

template <typename T, typename R, int TPR, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_rnorm_fwd(RnormArgs a, const T* __restrict__ x, const R* residual,
                                                        const T* __restrict__ gate, T* __restrict__ y, R* residual_out,
                                                        float* __restrict__ rstd, float* __restrict__ post_rstd) {
  __shared__ float s_table[8];
  RowSum<TPR> sum{s_table};
  constexpr int RP = kThreads / TPR;
  int c[NV];
  my_columns<TPR, VEC, NV>(a, c);
  float w[NV][VEC], pw[NV][VEC];
  columns<VEC, NV>(a.weight, a.C, c, w);
  columns<VEC, NV>(a.post, a.C, c, pw);
  typename Vec<T, VEC>::R rx[NV], rg[NV];
  typename Vec<R, VEC>::R rr[NV];
  const int64_t step = (int64_t)gridDim.x * RP, first = (int64_t)blockIdx.x * RP + threadIdx.x / TPR;
  const auto next = [&](int64_t row) __attribute__((always_inline)) {
    if (row >= a.n) return;
    ask<T, VEC, NV>(x, row, a.C, c, rx);
    ask<R, VEC, NV>(residual, row, a.C, c, rr);
    ask<T, VEC, NV>(gate, row, a.C, c, rg);
  };
  next(first);
  for (int64_t row = first; row < a.n; row += step) {
    float v[NV][VEC], r[NV][VEC], g[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Vec<T, VEC>::wide(rx[j], v[j]);
      Vec<R, VEC>::wide(rr[j], r[j]);
      Vec<T, VEC>::wide(rg[j], g[j]);
    }
    next(row + step);
    float factor = 1.f;
    if (a.post != nullptr) {
      factor = inverse_rms<TPR, VEC, NV>(a, sum, v);
      if (threadIdx.x % TPR == 0) post_rstd[row] = factor;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float u = v[j][e] * factor * pw[j][e];
        if (gate != nullptr) u *= act(a.act, g[j][e]);
        r[j][e] = __builtin_fmaf(a.scale, u, r[j][e]);
      }
    const float rs = inverse_rms<TPR, VEC, NV>(a, sum, r);
    if (threadIdx.x % TPR == 0) rstd[row] = rs;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (c[j] >= 0) {
        Vec<R, VEC>::store(residual_out + row * a.C + c[j], r[j]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) r[j][e] = r[j][e] * rs * w[j][e];
        Vec<T, VEC>::store(y + row * a.C + c[j], r[j]);
      }
  }
}

// part: [rows of workgroups][2][C], the sums of dweight and dpost_weight
template <typename T, typename R, int TPR, int VEC, int NV>
__global__ __launch_bounds__(kThreads) void k_rnorm_bwd(RnormArgs a, const T* __restrict__ x,
                                                        const R* __restrict__ residual_out,
                                                        const T* __restrict__ gate, const float* __restrict__ rstd,
                                                        const float* __restrict__ post_rstd, const T* __restrict__ dy,
                                                        const R* dresidual_out, T* __restrict__ dx, R* dresidual,
                                                        T* __restrict__ dgate, float* __restrict__ part) {
  __shared__ float s_table[8];
  RowSum<TPR> sum{s_table};
  constexpr int RP = kThreads / TPR;
  int c[NV];
  my_columns<TPR, VEC, NV>(a, c);
  float w[NV][VEC], pw[NV][VEC], dw[NV][VEC] = {}, dpw[NV][VEC] = {};
  columns<VEC, NV>(a.weight, a.C, c, w);
  columns<VEC, NV>(a.post, a.C, c, pw);
  typename Vec<T, VEC>::R rx[NV], rg[NV], rd[NV];
  typename Vec<R, VEC>::R rr[NV], ro[NV];
  const float inv = 1.f / (float)a.C;
  const int64_t step = (int64_t)gridDim.x * RP, first = (int64_t)blockIdx.x * RP + threadIdx.x / TPR;
  float rs = 0.f, ps = 0.f;
  const auto next = [&](int64_t row) __attribute__((always_inline)) {
    if (row >= a.n) return;
    ask<R, VEC, NV>(residual_out, row, a.C, c, rr);
    ask<T, VEC, NV>(dy, row, a.C, c, rd);
    ask<R, VEC, NV>(dresidual_out, row, a.C, c, ro);
    ask<T, VEC, NV>(x, row, a.C, c, rx);
    ask<T, VEC, NV>(gate, row, a.C, c, rg);
    rs = rstd[row];
    ps = a.post != nullptr ? post_rstd[row] : 1.f;
  };
  next(first);
  for (int64_t row = first; row < a.n; row += step) {
    float v[NV][VEC], r[NV][VEC], g[NV][VEC], d[NV][VEC], o[NV][VEC];
    const float scale1 = rs, scale2 = ps;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Vec<T, VEC>::wide(rx[j], v[j]);
      Vec<R, VEC>::wide(rr[j], r[j]);
      Vec<T, VEC>::wide(rg[j], g[j]);
      Vec<T, VEC>::wide(rd[j], d[j]);
      Vec<R, VEC>::wide(ro[j], o[j]);
    }
    next(row + step);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        r[j][e] *= scale1;
        dw[j][e] = __builtin_fmaf(d[j][e], r[j][e], dw[j][e]);
        d[j][e] *= w[j][e];
        s = __builtin_fmaf(d[j][e], r[j][e], s);
      }
    s = sum(s) * inv;
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[j][e] = __builtin_fmaf(scale1, __builtin_fmaf(-s, r[j][e], d[j][e]), o[j][e]);
      if (c[j] >= 0 && dresidual != nullptr) Vec<R, VEC>::store(dresidual + row * a.C + c[j], o[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        o[j][e] *= a.scale;
        v[j][e] *= scale2;
      }
      if (gate != nullptr) {
        float dg[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          dg[e] = o[j][e] * (v[j][e] * pw[j][e]) * slope(a.act, g[j][e]);
          o[j][e] *= act(a.act, g[j][e]);
        }
        if (c[j] >= 0) Vec<T, VEC>::store(dgate + row * a.C + c[j], dg);
      }
      if (a.post != nullptr) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          dpw[j][e] = __builtin_fmaf(o[j][e], v[j][e], dpw[j][e]);
          o[j][e] *= pw[j][e];
          q = __builtin_fmaf(o[j][e], v[j][e], q);
        }
      }
    }
    if (a.post != nullptr) {
      q = sum(q) * inv;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[j][e] = scale2 * __builtin_fmaf(-q, v[j][e], o[j][e]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (c[j] >= 0) Vec<T, VEC>::store(dx + row * a.C + c[j], o[j]);
  }
  float* out = part + first * 2 * a.C;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (c[j] >= 0) {
      Vec<float, VEC>::store(out + c[j], dw[j]);
      Vec<float, VEC>::store(out + a.C + c[j], dpw[j]);
    }
}

// Sums of the workgroups' rows, in their order: 64 values a workgroup, sixteen runs side by side.
__global__ __launch_bounds__(1024) void k_rnorm_sums(const float* __restrict__ part, int32_t count, int32_t C,
                                                     float* __restrict__ dweight, float* __restrict__ dpost) {
  __shared__ float s_sum[16][64];
  const int lane = threadIdx.x & 63, run = threadIdx.x >> 6, at = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (at < 2 * C) {
    const int lo = (int)((int64_t)count * run / 16), hi = (int)((int64_t)count * (run + 1) / 16);
#pragma unroll 8
    for (int s = lo; s < hi; ++s) sum += part[(size_t)s * 2 * C + at];
  }
  s_sum[run][lane] = sum;
  __syncthreads();
  if (run || at >= 2 * C) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += s_sum[i][lane];
  if (at < C) {
    if (dweight != nullptr) dweight[at] = sum;
  } else if (dpost != nullptr) {
    dpost[at - C] = sum;
  }
}

constexpr int kBackBlocks = 512;

template <typename T, typename R>
bool wide(int32_t C, std::initializer_list<const void*> ps) {
  if (C % (16 / (int)sizeof(T))) return false;
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) & 15) return false;
  return true;
}

// run(threads of a row, values of a vector, vectors of a thread)
template <typename T, class F>
void by_row(int32_t C, bool vec, F run) {
  constexpr int VEC = 16 / sizeof(T);
  using std::integral_constant;
  const auto go = [&](auto tpr, auto v, auto nv) { run(tpr, v, nv); };
  if (vec) {
    const integral_constant<int, VEC> v{};
    const int cv = C / VEC;
    if (cv <= 64) go(integral_constant<int, 64>{}, v, integral_constant<int, 1>{});
    else if (cv <= 128) go(integral_constant<int, 64>{}, v, integral_constant<int, 2>{});
    else if (cv <= 256) go(integral_constant<int, 256>{}, v, integral_constant<int, 1>{});
    else if (cv <= 512) go(integral_constant<int, 256>{}, v, integral_constant<int, 2>{});
    else if (cv <= 1024) go(integral_constant<int, 256>{}, v, integral_constant<int, 4>{});
    else if constexpr (VEC == 4) go(integral_constant<int, 256>{}, v, integral_constant<int, 8>{});
  } else {
    const integral_constant<int, 1> v{};
    if (C <= 256) go(integral_constant<int, 64>{}, v, integral_constant<int, 4>{});
    else if (C <= 1024) go(integral_constant<int, 256>{}, v, integral_constant<int, 4>{});
    else go(integral_constant<int, 256>{}, v, integral_constant<int, 32>{});
  }
}

template <class F>
void by_types(int dtype, int rtype, F f) {
  if (dtype == 0) f(float{}, float{});
  else if (dtype == 1 && rtype == 0) f(_Float16{}, float{});
  else if (dtype == 1) f(_Float16{}, _Float16{});
  else if (rtype == 0) f(bf16_t{}, float{});
  else f(bf16_t{}, bf16_t{});
}

}  // namespace

size_t rnorm_backward_workspace_bytes(int64_t n, int32_t C) {
  // at most four rows of sums a workgroup, and those only for narrow rows
  const int64_t rows = std::min<int64_t>(n, kBackBlocks * 4);
  return align_up((size_t)(C <= 1024 ? rows + 3 : std::min<int64_t>(rows, kBackBlocks)) * 2 * C * 4 + 256, 256);
}

hipError_t launch_forward_rnorm(int64_t n, int dtype, int rtype, int32_t C, float eps, float scale, int activation,
                                const void* x, const void* residual, const void* gate, const float* post_weight,
                                const float* weight, void* y, void* residual_out, float* rstd, float* post_rstd,
                                hipStream_t stream) {
  by_types(dtype, rtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    const bool vec = wide<T, R>(C, {x, residual, gate, y, residual_out});
    by_row<T>(C, vec, [&](auto tpr, auto v, auto nv) {
      constexpr int TPR = decltype(tpr)::value, VEC = decltype(v)::value, NV = decltype(nv)::value;
      const RnormArgs a{n, C, C / VEC, eps, scale, activation, weight, post_weight};
      const int64_t blocks = (n + kThreads / TPR - 1) / (kThreads / TPR);
      k_rnorm_fwd<T, R, TPR, VEC, NV><<<(uint32_t)std::min<int64_t>(blocks, 2048), kThreads, 0, stream>>>(
          a, static_cast<const T*>(x), static_cast<const R*>(residual), static_cast<const T*>(gate), static_cast<T*>(y),
          static_cast<R*>(residual_out), rstd, post_rstd);
    });
  });
  return hipGetLastError();
}

hipError_t launch_backward_rnorm(int64_t n, int dtype, int rtype, int32_t C, float scale, int activation, const void* x,
                                 const void* residual_out, const void* gate, const float* post_weight,
                                 const float* weight, const float* rstd, const float* post_rstd, const void* dy,
                                 const void* dresidual_out, void* dx, void* dresidual, void* dgate, float* dweight,
                                 float* dpost_weight, void* workspace, hipStream_t stream) {
  float* part = static_cast<float*>(workspace);
  by_types(dtype, rtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    const bool vec = wide<T, R>(C, {x, residual_out, gate, dy, dresidual_out, dx, dresidual, dgate});
    by_row<T>(C, vec, [&](auto tpr, auto v, auto nv) {
      constexpr int TPR = decltype(tpr)::value, VEC = decltype(v)::value, NV = decltype(nv)::value;
      constexpr int RP = kThreads / TPR;
      const RnormArgs a{n, C, C / VEC, 0.f, scale, activation, weight, post_weight};
      const int blocks = (int)std::min<int64_t>((n + RP - 1) / RP, kBackBlocks);
      if (n > 0)
        k_rnorm_bwd<T, R, TPR, VEC, NV><<<blocks, kThreads, 0, stream>>>(
            a, static_cast<const T*>(x), static_cast<const R*>(residual_out), static_cast<const T*>(gate), rstd, post_rstd,
            static_cast<const T*>(dy), static_cast<const R*>(dresidual_out), static_cast<T*>(dx),
            static_cast<R*>(dresidual), static_cast<T*>(dgate), part);
      k_rnorm_sums<<<(2 * C + 63) / 64, 1024, 0, stream>>>(part, blocks * RP, C, dweight, dpost_weight);
    });
  });
  return hipGetLastError();
}

}  // namespace sla
