// Backward of the gated delta rule in chunk form.  The paper trains its linear attentions but
// writes no backward; this is the chain rule of the recurrence in sla.h.
//
// With D_ij, T, P, r, u of the forward (sla_delta.h), dS1 the gradient of the state after a chunk
// and lam_j the whole gradient of u_j:
//     du  = P^T (scale do) + exp(gam_last - gam) k dS1,
//     lam = (I + [beta_i D_ij k_i . k_j]_{j < i})^-T du,   mu = beta lam  (= dv),
//     dS0 = exp(gam_last) dS1 + scale (exp(gam) q)^T do - (exp(gam) k)^T mu,
//     dbeta_j = lam_j . r_j   (lam' . r' 2^kap / s),
//     dq_i = scale (exp(gam_i) S0 do_i + sum_{j <= i} D_ij (do_i . u_j) k_j),
//     dk_j = exp(gam_last - gam_j) dS1 u_j - exp(gam_j) S0 mu_j - sum_{i < j} D_ji (mu_j . u_i) k_i
//            - sum_{i > j} D_ij (mu_i . u_j) k_i + scale sum_{i >= j} D_ij (do_i . u_j) q_i.
// The decay's gradient needs no products of its own: dg_t is the inner product of the decayed state
// and its gradient, and from one row to the next these differ by vectors that are at hand,
//     dg_t = dg_{t+1} + o_t . do_t - v_t . dv_t,   and at a chunk's first row dg = <dS0, S0>,
// which starts the sum anew in every chunk, so that it never runs over more than 64 rows; it is fp64.  What
// is left is the error of its fp32 terms: dg is as exact as the chunk's |o . do| and |v . dv| are, however
// small it is beside them (with a fast decay it is exp(g) times as large).
//
// Four launches: T, P and their transposes (k_delta_prep); the forward walk, which keeps the states
// before every chunk, r and o . do (k_delta_walk); the walk back, which keeps lam and the gradients
// of the states after every chunk (k_delta_back); and, all chunks at once, everything that is no
// recurrence (k_delta_grad).  States are made again and not kept from the forward: they are dk / 16
// times as large as the rows.
#include "sla_delta_chunk.h"

namespace sla {
namespace {

using namespace delta;

// Workspace behind the chunk form's: byte offsets.
struct BackSpace {
  Space base;
  size_t states, dstates, resid, lam, odo, smax, dmax, start, ends, maps, back_ends, total;
};
BackSpace back_space(int64_t n, int32_t W, int dtype, int32_t Hk, int32_t H, int32_t dk, int32_t dv) {
  BackSpace s;
  s.base = space_of(n, W, dtype, Hk, H, dk, kRecordBack);
  const size_t sh = slots_of(n, W) * H, groups = dv / 16;
  size_t at = s.base.total;
  const auto take = [&](size_t floats) {
    const size_t here = at;
    at = align_up(at + floats * 4, 256);
    return here;
  };
  s.states = take(sh * pad_dk(dk) * dv);
  s.dstates = take(sh * pad_dk(dk) * dv);
  s.resid = take(sh * kChunk * dv);
  s.lam = take(sh * kChunk * dv);
  s.odo = take(sh * groups * kChunk);
  s.smax = take(sh * groups);
  s.dmax = take(sh * groups);
  s.start = take(sh * groups);
  const Args a = args_of(nullptr, n, W, nullptr, Hk, H, dk, dv, 1.f);
  s.ends = s.maps = s.back_ends = at;
  if (a.part) {
    s.ends = take(ends_halfs(a, pad_dk(dk)) / 2);
    s.maps = take(maps_halfs(a, pad_dk(dk)) / 2);
    s.back_ends = take(ends_halfs(a, pad_dk(dk)) / 2);
  }
  s.total = at;
  return s;
}

// ------------------------------------------------------------------ the walk back
// As k_delta_walk: a wave holds 16 columns of the state's gradient in registers.
// Bound by the chain like it: 16,381 bf16 rows, 9 sequences, 8 heads of 128: 147 us behind 127 for the
// parts' gradients; 1,521 fp16 windows: 85 us.
// ENDS: only the state gradients at the parts' starts, from none at their ends (the last part: from dstate).
template <typename T, int DK, int NW>
using BackStage = Stage<T, DK, NW, 0, kScalAt, kRecordBack>;

template <typename T, int DK, int NW, bool ENDS, bool AHEAD>
__global__ __launch_bounds__(64 * NW) void k_delta_back(Args a, const T* __restrict__ dout,
                                                        const float* __restrict__ dstate,
                                                        const _Float16* __restrict__ images,
                                                        const _Float16* __restrict__ records, float* ends,
                                                        const float* __restrict__ states, float* __restrict__ lam,
                                                        float* __restrict__ dstates, float* __restrict__ dmax,
                                                        float* __restrict__ start, float* __restrict__ dstate_in) {
  constexpr int NT = kTerms<T>, KB = DK / 32, IMG = kChunk * DK, ST = DK / 16;
  using SG = BackStage<T, DK, NW>;
  constexpr bool TWICE = AHEAD && kTwice<SG>;
  __shared__ SG s_a;
  __shared__ std::conditional_t<TWICE, SG, char> s_b;

  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place here = place_of(a, lane);
  const Part part = here.part;
  if (part.none || (ENDS && part.lo == 0)) return;
  const int w = part.w, h = here.h, group = a.H / a.Hk, hk = h / group;
  const int cg = blockIdx.z * NW + wave, groups = a.dv / 16;
  const bool live = cg < groups;
  const int col = 16 * cg + i;
  const Win win = window(a, w);
  const uint32_t slot0 = first_slot(win.begin, w);
  const int first = part.lo;   // the last chunk of this part's walk
  const auto rows_of = [&](int c) __attribute__((always_inline)) { return min(kChunk, win.rows - c * kChunk); };

  floatx4 S[ST];
  bool carried = true;
  // A parted window's last gradient is read once, by the walk of the ends, which keeps it where the first
  // part's would be: dstate_in, which the first part's workgroup writes, may be dstate.
  const bool kept = part.hi == part.chunks && part.lo > 0 && dstate != nullptr;
  const uint32_t from_slot = kept ? part.slot - (uint32_t)(part.lo / a.part) : part.slot + 1;
  if (ENDS || (part.hi == part.chunks && !kept)) {
    const float* from = part.hi == part.chunks ? dstate : nullptr;
    load_state(S, a, from, w, h, col, live, g);
    carried = from != nullptr;
    if (ENDS && kept && live) {
      float* to = ends + (((size_t)from_slot * a.H + h) * groups + cg) * ST * 256 + lane * 4;
#pragma unroll
      for (int t = 0; t < ST; ++t) *reinterpret_cast<floatx4*>(to + t * 256) = S[t];
    }
  } else if (live) {
    const float* from = ends + (((size_t)from_slot * a.H + h) * groups + cg) * ST * 256 + lane * 4;
#pragma unroll
    for (int t = 0; t < ST; ++t) S[t] = *reinterpret_cast<const floatx4*>(from + t * 256);
  }
  using F = Fetch<SG, T, kScalAt>;
  F fetch;
  const auto begin = [&](SG& s, int c, const Places<T>& at) __attribute__((always_inline)) {
    fetch.start(s, a, slot0 + c, hk, h, cg, live, images, records, kRecordBack, dout, at, wave, lane, rows_of(c));
  };
  Places<T> at;
  if (part.hi > first) {
    at.ask(a, win.begin + (part.hi - 1) * kChunk, rows_of(part.hi - 1), lane);
    if constexpr (TWICE) {
      begin(s_a, part.hi - 1, at);
      fetch.template jobs<0, F::kJobs>(s_a, wave);
    }
  }

  const auto work = [&](const SG& s, auto& other, int c) __attribute__((always_inline)) {
    const float* scal = reinterpret_cast<const float*>(s.rec);
    const auto jobs = [&](auto from, auto to) __attribute__((always_inline)) {
      if constexpr (TWICE)
        if (c > first) fetch.template jobs<decltype(from)::value * F::kJobs / 8, decltype(to)::value * F::kJobs / 8>(other, wave);
    };
    using std::integral_constant;
    floatx4 X[4], Y[4];
    rows_in(s.rows[wave], Y, rows_of(c), i, g);
    if constexpr (TWICE)
      if (c > first) {
        Places<T> to;
        to.take(a, scal + kPrev, lane);
        begin(other, c - 1, to);
      }
    jobs(integral_constant<int, 0>{}, integral_constant<int, 2>{});
    const size_t sh = (size_t)(slot0 + c) * a.H + h;
    const _Float16 *qi = s.img, *ki = s.img + NT * IMG;
    const _Float16 *bt = s.rec + kBackT - kScalAt, *bp = s.rec + kBackP - kScalAt;
    auto row4 = [&](int what, int tau) { return *reinterpret_cast<const floatx4*>(scal + what + 16 * tau + 4 * g); };
    const size_t sgrp = sh * (a.dv / 16) + cg;
    floatx4 s0[ENDS ? 1 : ST];   // the state before the chunk, for the end
    if constexpr (!ENDS)
#pragma unroll
      for (int t = 0; t < ST; ++t) s0[t] = *reinterpret_cast<const floatx4*>(states + sgrp * ST * 256 + t * 256 + lane * 4);
    const uint32_t top = column_max_bits(max_of(S));
    if constexpr (!ENDS) {
#pragma unroll
      for (int t = 0; t < ST; ++t) *reinterpret_cast<floatx4*>(dstates + sgrp * ST * 256 + t * 256 + lane * 4) = S[t];
      const uint32_t all = wave_max_bits(__uint_as_float(top));
      if (lane == 0) dmax[sgrp] = __uint_as_float(all);
    }
    // du = P^T do' + until k' dS
    {
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) Y[tau] *= row4(kOScale, tau);
      const Scale sy = column_scale(Y);
      const floatx4 ydown = *reinterpret_cast<const floatx4*>(scal + kBackPDown) * sy.down;
      Far Yp[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) Yp[s2] = split<Far>(Y[2 * s2], Y[2 * s2 + 1], sy.up);
      tri_times<true>(bp, bp + kTerm, Yp, X, lane);
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) X[tau] *= ydown[tau];
    }
    if (carried) {
      const Scale sc = scale_of(top);
      Pair Sp[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) Sp[kb] = split(S[2 * kb], S[2 * kb + 1], sc.up);
      floatx4 x[4];
      rows_times<NT, DK>(ki, Sp, x, i, g);
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) X[tau] += (row4(kUntil, tau) * sc.down) * x[tau];
    }
    jobs(integral_constant<int, 2>{}, integral_constant<int, 5>{});
    // lam, then -since mu in X and since do' in Y
    {
      const Scale sx = column_scale(X);
      const floatx4 xdown = *reinterpret_cast<const floatx4*>(scal + kBackTDown) * sx.down;
      Far Xp[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) Xp[s2] = split<Far>(X[2 * s2], X[2 * s2 + 1], sx.up);
      tri_times<true>(bt, bt + kTerm, Xp, X, lane);
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) {
        const floatx4 since = row4(kSince, tau);
        X[tau] *= xdown[tau];
        if constexpr (!ENDS)
#pragma unroll
          for (int r = 0; r < 4; ++r) lam[(sh * kChunk + 16 * tau + 4 * g + r) * a.dv + col] = X[tau][r];
        X[tau] *= -since * row4(kBeta, tau);
        Y[tau] *= since;
      }
    }
    jobs(integral_constant<int, 5>{}, integral_constant<int, 8>{});
    // dS = exp(gam_last) dS + q'^T (since do') - k'^T (since mu)
    {
      const Scale sc = scale_of(column_max_bits(fmaxf(max_of(X), max_of(Y))));
      Pair Xp[2], Yp[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        Xp[s2] = split(X[2 * s2], X[2 * s2 + 1], sc.up);
        Yp[s2] = split(Y[2 * s2], Y[2 * s2 + 1], sc.up);
      }
      const float last = scal[kLast];
      float dot = 0.f;
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          if constexpr (NT == 2) {
            x = mma(image_cols<DK>(ki + IMG, t >> 1, t & 1, s2, i, g), Xp[s2].hi, x);
            x = mma(image_cols<DK>(qi + IMG, t >> 1, t & 1, s2, i, g), Yp[s2].hi, x);
          }
          x = mma1(image_cols<DK>(ki, t >> 1, t & 1, s2, i, g), Xp[s2], x);
          x = mma1(image_cols<DK>(qi, t >> 1, t & 1, s2, i, g), Yp[s2], x);
        }
        S[t] = last * S[t] + sc.down * x;
        if constexpr (!ENDS)
#pragma unroll
          for (int r = 0; r < 4; ++r) dot += s0[t][r] * S[t][r];
      }
      if constexpr (!ENDS) {
#pragma unroll
        for (int m2 = 1; m2 < 64; m2 *= 2) dot += __shfl_xor(dot, m2);
        if (lane == 0) start[sgrp] = dot;
      }
      carried = true;
    }
  };

  if (!live) {   // beyond dv: a share of the moves
    for (int c = part.hi - 1; c >= first; --c) {
      barrier();
      if constexpr (TWICE) {
        if (c == first) break;
        begin(s_b, c - 1, at);
        fetch.template jobs<0, F::kJobs>(s_b, wave);
        barrier();
        if (--c == first) break;
        begin(s_a, c - 1, at);
        fetch.template jobs<0, F::kJobs>(s_a, wave);
      } else {
        begin(s_a, c, at);
        fetch.template jobs<0, F::kJobs>(s_a, wave);
        barrier();
      }
    }
    return;
  }
  if constexpr (TWICE) {
    const auto turn = [&](const SG& s, SG& other, int c) __attribute__((always_inline)) {
      barrier();   // chunk c is there, and no wave reads the other buffer any more
      work(s, other, c);
    };
    for (int c = part.hi - 1; c >= first; c -= 2) {
      turn(s_a, s_b, c);
      if (c > first) turn(s_b, s_a, c - 1);
    }
  } else {
    for (int c = part.hi - 1; c >= first; --c) {
      if (c + 1 < part.hi) at.take(a, reinterpret_cast<const float*>(s_a.rec) + kPrev, lane);
      barrier();
      begin(s_a, c, at);
      fetch.template jobs<0, F::kJobs>(s_a, wave);
      barrier();
      work(s_a, s_a, c);
    }
  }
  if constexpr (ENDS) {
    float* to = ends + (((size_t)part.slot * a.H + h) * groups + cg) * ST * 256 + lane * 4;
#pragma unroll
    for (int t = 0; t < ST; ++t) *reinterpret_cast<floatx4*>(to + t * 256) = S[t];
  } else if (part.lo == 0) {
    store_state(S, a, dstate_in, w, h, col, live, g);
  }
}

// ------------------------------------------------------------------ the rest, all chunks at once
// A workgroup per chunk and query/key head, its value heads one after the other, their dq (or dk)
// summed in registers (in head order: deterministic).  Wave w owns rows 16w .. 16w + 15, one a lane (i)
// and four lane groups over the columns, and makes the transposed tiles: a lane ends with 8
// neighbouring columns of its row.  The value columns go by in blocks of 32, the next block's loads in
// flight (not at 32 state rows, where a third workgroup a CU is worth more than they are).  dq and dk are launches of their own (FOR_K; dv, dbeta and dg come with dk): together they
// took twice the registers and waited for memory at one workgroup a CU.  Bound by the waits of the workgroups
// that a CU holds, for dk one at 128 state rows (90 KB of LDS), two at 64 and three at 32: 16,381 bf16 rows, 8
// heads of 128: 86 and 269 us; 1,521 fp16 windows, 4 heads of 32: 60 and 154 us.  Measured before the present
// operands, one launch for both: 426 and 228 us where two took 244 and 210; eight waves, four for dq and four
// for dk: 345 and 366.
//
// Computed operands (states, mu, u, the products over columns) have two fp16 terms whatever the rows'
// type: with one, 2^-11 of the largest value, small entries of dq and dk were off by many of their own
// steps, bf16's too.  Every row has powers of two of its own (a lane's own row one, the other rows' out of
// s_scale): mu' and u' of a small key are small beside its neighbours', but its dk is not.
constexpr int kBlockCols = 32;

template <int NT>
struct Op {
  half8_t t[NT];
};
template <int NA, int NB>
__device__ __forceinline__ floatx4 mma_op(const Op<NA>& a, const Op<NB>& b, floatx4 c) {
  if constexpr (NA == 2) c = mma(a.t[1], b.t[0], c);
  if constexpr (NB == 2) c = mma(a.t[0], b.t[1], c);
  return mma(a.t[0], b.t[0], c);
}
template <int NT>
__device__ __forceinline__ Op<NT> op_of(const float (&x)[8], float s) {
  Op<NT> p;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = x[e] * s;
    p.t[0][e] = (_Float16)y;
    if constexpr (NT == 2) p.t[1][e] = (_Float16)(y - (float)p.t[0][e]);
  }
  return p;
}
__device__ __forceinline__ float max8(const float (&x)[8]) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));
  return m;
}

template <typename T, int DK, bool FOR_K>
__global__ __launch_bounds__(256, DK == 32 ? 3 : 2) void k_delta_grad(Args a, const T* __restrict__ v,
                                                    const T* __restrict__ dout,
                                                    const float* __restrict__ gin,
                                                    const _Float16* __restrict__ images,
                                                    const _Float16* __restrict__ records,
                                                    const float* __restrict__ states,
                                                    const float* __restrict__ dstates, const float* __restrict__ smax,
                                                    const float* __restrict__ dmax, const float* __restrict__ resid,
                                                    const float* __restrict__ lam, const float* __restrict__ odo,
                                                    const float* __restrict__ start, int has_state, int has_dstate,
                                                    T* __restrict__ dq, T* __restrict__ dk, T* __restrict__ dv,
                                                    float* __restrict__ dg, float* __restrict__ dbeta) {
  constexpr int NT = kTerms<T>, IMG = kChunk * DK, ST = DK / 16;
  constexpr int NC = 2;   // terms of computed operands
  constexpr int kStateHalfs = ST * 256;   // one group of 16 columns, in register order
  constexpr int kStates = FOR_K ? 2 : 1;   // S0, dS1
  constexpr int kSkip = FOR_K ? 0 : NT * IMG;   // dq does not need q'
  __shared__ __attribute__((aligned(16))) _Float16 s_img[2 * NT * IMG - kSkip];
  __shared__ __attribute__((aligned(16))) _Float16 s_state[kStates][NC][2 * kStateHalfs];
  __shared__ __attribute__((aligned(16))) _Float16 s_do[FOR_K ? 4 : 1][NT][kFrag], s_mu[FOR_K ? 4 : 1][NC][kFrag];
  __shared__ __attribute__((aligned(16))) _Float16 s_u[4][NC][kFrag];
  __shared__ __attribute__((aligned(16))) float s_scale[3][kChunk];   // of do, mu', u' of every row
  __shared__ __attribute__((aligned(16))) float s_scal[kScal];
  __shared__ double s_gam[kChunk];
  __shared__ double s_dot[kChunk];

  const uint32_t slot = blockIdx.x;
  const int hk = blockIdx.y;
  const int lo = window_of(a, slot, threadIdx.x & 63);
  const Win win = window(a, lo);
  const uint32_t f = first_slot(win.begin, lo);
  if (slot < f || (int64_t)(slot - f) * kChunk >= win.rows) return;
  const int base = win.begin + (int)(slot - f) * kChunk;
  const int rows = min(kChunk, win.rows - (int)(slot - f) * kChunk);
  const bool more = (int64_t)(slot - f + 1) * kChunk < win.rows;   // the window has a chunk after this one

  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = 16 * wave + i;
  const bool real = own < rows;
  const int orig = real ? row_at(a, base + own) : 0;
  {
    const uint4* src = reinterpret_cast<const uint4*>(images + ((size_t)slot * a.Hk + hk) * 2 * NT * IMG + kSkip);
    uint4* dst = reinterpret_cast<uint4*>(s_img);
#pragma unroll 4
    for (int x = tid; x < (2 * NT * IMG - kSkip) / 8; x += 256) dst[x] = src[x];
  }
  const _Float16 *qi = s_img, *ki = s_img + (NT * IMG - kSkip);
  floatx4 D[ST];   // dq or dk, transposed
#pragma unroll
  for (int t = 0; t < ST; ++t) D[t] = floatx4{0.f, 0.f, 0.f, 0.f};

  const int group = a.H / a.Hk, groups = a.dv / 16, tid0 = tid, lane0 = lane;
  for (int hv = 0; hv < group; ++hv) {
    // the lane's numbers anew for every head: their many comparisons and addresses are made where they
    // are used, and not kept in registers over the loop
    int tid = tid0, lane = lane0;
    asm volatile("" : "+v"(tid), "+v"(lane));
    const int i = lane & 15, g = lane >> 4, own = 16 * wave + i;
    const bool real = own < rows;
    const int h = hk * group + hv;
    const size_t sh = (size_t)slot * a.H + h;
    // a block's own rows (8 columns a lane) and its two column groups of the states, as the walks left them
    constexpr int kLoads = kStates * 2 * ST * 64 / 256;
    floatx4 z[kLoads];
    Raw<T, 8> ro, rv;
    f32x8 rl, rr;
    const size_t row0 = ((size_t)orig * a.H + h) * a.dv, lam0 = (sh * kChunk + own) * a.dv;
    const auto ask = [&](int c0) __attribute__((always_inline)) {
      const int col = c0 + 8 * g < a.dv ? c0 + 8 * g : 0;   // dropped when it is used
      ro = *reinterpret_cast<const Raw<T, 8>*>(dout + row0 + col);
      rr = *reinterpret_cast<const f32x8*>(resid + lam0 + col);
      if constexpr (FOR_K) {
        rv = *reinterpret_cast<const Raw<T, 8>*>(v + row0 + col);
        rl = *reinterpret_cast<const f32x8*>(lam + lam0 + col);
      }
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int which = n >= kLoads / kStates ? 1 : 0, y = tid + 256 * (n - which * (kLoads / kStates));
        const int group2 = c0 + 16 * (y / (ST * 64)) < a.dv ? c0 / 16 + y / (ST * 64) : 0;
        z[n] = *reinterpret_cast<const floatx4*>((which ? dstates : states) +
                                                 (sh * groups + group2) * (size_t)(ST * 256) + (size_t)(y % (ST * 64)) * 4);
      }
    };
    ask(0);
    __syncthreads();
    for (int x = tid; x < kScal / 4; x += 256)
      reinterpret_cast<uint4*>(s_scal)[x] = reinterpret_cast<const uint4*>(records + sh * kRecordBack + kScalAt)[x];
    if (wave == 3) {   // the decay sums, as k_delta_prep makes them
      const bool r1 = lane < rows;
      const float g1 = r1 ? gin[(size_t)row_at(a, base + lane) * a.H + h] : 0.f;
      double gam = g1 < -104.f ? -65536.0 : (double)g1 * 1.4426950408889634;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(gam, d);
        if (lane >= d) gam += o;
      }
      s_gam[lane] = gam;
    }
    // one power of two for all of a state: the largest of its column groups
    uint32_t sbits = 0, dbits = 0;
    for (int c = 0; c < groups; ++c) {
      sbits = max(sbits, __float_as_uint(smax[sh * groups + c]));
      dbits = max(dbits, __float_as_uint(dmax[sh * groups + c]));
    }
    const Scale ss = scale_of(sbits), sd = scale_of(dbits);
    __syncthreads();
    const float since = s_scal[kSince + own], until = s_scal[kUntil + own], be = s_scal[kBeta + own];
    const float vs = s_scal[kKScale + own], write = s_scal[kWrite + own];

    // products over the value columns: M[.][j], transposed tiles with this wave's rows in the lanes.
    // dq: 0: do of own rows with u of tile j (j <= wave).  dk: 0: mu of own rows with u of tile j
    // (j <= wave) or u of own rows with mu of tile j (j > wave; at j = wave: Mw), 1: u of own rows with
    // do of tile j (j >= wave)
    floatx4 M[FOR_K ? 2 : 1][4], Mw = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < (FOR_K ? 2 : 1); ++x)
#pragma unroll
      for (int j = 0; j < 4; ++j) M[x][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    float lr = 0.f;
    double vdv = 0.;

    for (int c0 = 0; c0 < a.dv; c0 += kBlockCols) {
      if (DK == 32 && c0 > 0) ask(c0);
      const int col = c0 + 8 * g;
      const bool here = real && col < a.dv;
      float xo[8], xm[8], xu[8];
      Frag<T, 8>::to_f32(ro, xo);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xo[e] = here ? xo[e] : 0.f;
        xu[e] = here ? write * rr[e] : 0.f;
      }
      if constexpr (FOR_K) {
        float xv[8], xd[8], dot = 0.f;
        Frag<T, 8>::to_f32(rv, xv);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          xm[e] = here ? be * rl[e] : 0.f;
          lr += here ? rl[e] * rr[e] : 0.f;
          xd[e] = vs * xm[e];
          dot += here ? xv[e] * xd[e] : 0.f;
        }
        vdv += dot;
        if (here) *reinterpret_cast<Raw<T, 8>*>(dv + row0 + col) = Frag<T, 8>::from_f32(xd);
      }
      const Scale so = scale_of(column_max_bits(max8(xo))), su = scale_of(column_max_bits(max8(xu)));
      Scale sm = {1.f, 1.f};
      const Op<NT> oo = op_of<NT>(xo, so.up);
      const Op<NC> ou = op_of<NC>(xu, su.up);
      Op<NC> om;
      if constexpr (FOR_K) {
        sm = scale_of(column_max_bits(max8(xm)));
        om = op_of<NC>(xm, sm.up);
      }
      __syncthreads();   // the last block's reads are done
#pragma unroll
      for (int t = 0; t < NC; ++t) *reinterpret_cast<half8_t*>(&s_u[wave][t][lane * 8]) = ou.t[t];
      if constexpr (FOR_K) {
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<half8_t*>(&s_do[wave][t][lane * 8]) = oo.t[t];
#pragma unroll
        for (int t = 0; t < NC; ++t) *reinterpret_cast<half8_t*>(&s_mu[wave][t][lane * 8]) = om.t[t];
      }
      if (g == 0) {
        s_scale[0][own] = so.down;
        s_scale[1][own] = sm.down;
        s_scale[2][own] = su.down;
      }
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int which = n >= kLoads / kStates ? 1 : 0, y = tid + 256 * (n - which * (kLoads / kStates));
        const float up = c0 + 16 * (y / (ST * 64)) < a.dv ? (which ? sd.up : ss.up) : 0.f;
        half4_t p, l;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float u = up != 0.f ? z[n][r] * up : 0.f;
          p[r] = (_Float16)u;
          l[r] = (_Float16)(u - (float)p[r]);
        }
        *reinterpret_cast<half4_t*>(&s_state[which][0][y * 4]) = p;
        *reinterpret_cast<half4_t*>(&s_state[which][1][y * 4]) = l;
      }
      if (DK != 32 && c0 + kBlockCols < a.dv) ask(c0 + kBlockCols);
      __syncthreads();
      // rows of the block's states as operand rows: tile t's 16 state rows, contraction over 32 columns
      const auto state_rows = [&](int which, int t) __attribute__((always_inline)) {
        Op<NC> x;
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const int c = 8 * g + 4 * hh;   // the columns' place in the block
            const _Float16* at = &s_state[which][n][(((c >> 4) * ST + t) * 64 + (i & 3) * 16 + (c & 15) + (i >> 2)) * 4];
            const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) short4v*)(const_cast<_Float16*>(at)));
#pragma unroll
            for (int r = 0; r < 4; ++r) x.t[n][4 * hh + r] = __builtin_bit_cast(_Float16, (short)y[r]);
          }
        return x;
      };
      const auto rows_of = [&](auto& rows, auto& x, int j) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < (int)(sizeof(x.t) / sizeof(x.t[0])); ++n)
          x.t[n] = *reinterpret_cast<const half8_t*>(&rows[j][n][lane * 8]);
      };
      const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
      const auto scale4 = [&](int which, int j) __attribute__((always_inline)) {   // of tile j's rows
        return *reinterpret_cast<const floatx4*>(&s_scale[which][16 * j + 4 * g]);
      };
      const float fq = (a.scale * since * ss.down) * so.down;
      const float fk0 = -(vs * sm.down) * (since * ss.down), fk1 = (vs * su.down) * (until * sd.down);
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        if (t % 4 == 0) __builtin_amdgcn_sched_barrier(0);   // four tiles' operands in registers
        if constexpr (FOR_K) {
          D[t] += fk0 * mma_op(state_rows(0, t), om, zero);
          D[t] += fk1 * mma_op(state_rows(kStates - 1, t), ou, zero);
        } else {
          D[t] += fq * mma_op(state_rows(0, t), oo, zero);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // (tiles that the decays will clear are made too: fewer registers than branches)
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (FOR_K) {
          const bool before = j <= wave;
          Op<NC> x, own;
          rows_of(before ? s_u : s_mu, x, j);
          rows_of(before ? s_mu : s_u, own, wave);
          M[0][j] += (scale4(before ? 2 : 1, j) * (before ? sm.down : su.down)) * mma_op(x, own, zero);
          Op<NT> o;
          rows_of(s_do, o, j);
          M[FOR_K][j] += (scale4(0, j) * su.down) * mma_op(o, ou, zero);
        } else {
          Op<NC> u;
          rows_of(s_u, u, j);
          M[0][j] += (scale4(2, j) * so.down) * mma_op(u, oo, zero);
        }
      }
      if constexpr (FOR_K) Mw += (scale4(1, wave) * su.down) * mma_op(om, ou, zero);
    }
    // the decays between own row and the others, then the products over the chunk's rows: M[0] becomes
    // what k is multiplied with, for dk M[1] what q is
    const double go = s_gam[own];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      __builtin_amdgcn_sched_barrier(0);
      const floatx4 os = *reinterpret_cast<const floatx4*>(&s_scal[kOScale + 16 * j + 4 * g]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int o = 16 * j + 4 * g + r;   // the other row
        // decay from the other row to the own one if it is before, else from the own to the other
        const float diff = (float)(go - s_gam[o]);
        const float d = __builtin_amdgcn_exp2f(o <= own ? diff : -diff);
        if constexpr (!FOR_K) {
          const float x = a.scale * d * M[0][j][r];
          M[0][j][r] = o <= own ? x : 0.f;
        } else {
          const float x = -d * (j == wave && o > own ? Mw[r] : M[0][j][r]), y = d * M[FOR_K][j][r] * os[r];
          M[0][j][r] = o == own ? 0.f : x;
          M[FOR_K][j][r] = o >= own ? y : 0.f;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    const auto ops_of = [&](const floatx4 (&m)[4], Op<NC> (&p)[2]) __attribute__((always_inline)) {
      const Scale s = column_scale(m);
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        float x[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = m[2 * s2][r], x[4 + r] = m[2 * s2 + 1][r];
        p[s2] = op_of<NC>(x, s.up);
      }
      return s.down;
    };
    const auto add = [&](const _Float16* img, const Op<NC> (&p)[2], float f) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        if (t % 4 == 0) __builtin_amdgcn_sched_barrier(0);
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          Op<NT> c;
#pragma unroll
          for (int n = 0; n < NT; ++n) c.t[n] = image_cols<DK>(img + n * IMG, t >> 1, t & 1, s2, i, g);
          x = mma_op(c, p[s2], x);
        }
        D[t] += f * x;
      }
    };
    Op<NC> P[2];
    const float down0 = ops_of(M[0], P);
    add(ki, P, FOR_K ? vs * down0 : down0);
    if constexpr (FOR_K) {
      const float down1 = ops_of(M[FOR_K], P);
      add(qi, P, vs * down1);
    }
    if constexpr (!FOR_K) continue;
    // dbeta = lam . r and the terms of dg: sums over the lane groups
    lr += __shfl_xor(lr, 16);
    lr += __shfl_xor(lr, 32);
    vdv += __shfl_xor(vdv, 16);
    vdv += __shfl_xor(vdv, 32);
    if (g == 0) {
      if (real) dbeta[(size_t)orig * a.H + h] = lr / vs / s_scal[kVScale + own];
      double od = 0.;
      for (int c = 0; c < groups; ++c) od += real ? odo[(sh * groups + c) * kChunk + own] : 0.f;
      s_dot[own] = real ? od - vdv : 0.;
    }
    __syncthreads();
    if (wave == 0) {
      double x = s_dot[lane];
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {   // sums to the end
        const double y = __shfl_down(x, d);
        if (lane + d < 64) x += y;
      }
      double at_end = 0.;
      if (more || has_dstate) {
        const size_t from = more ? sh + a.H : sh;
        for (int c = 0; c < groups; ++c) at_end += start[from * groups + c];
        if (!more) at_end -= __shfl(x, 0);
      }
      const bool r1 = lane < rows;
      if (r1) {
        const size_t at = (size_t)row_at(a, base + lane) * a.H + h;
        // nothing to decay: a decay that forgets everything, the first row without a state
        const bool none = gin[at] < -104.f || (slot == f && lane == 0 && !has_state);
        dg[at] = none ? 0.f : (float)(x + at_end);
      }
    }
  }
  // 8 neighbouring columns of the own row from two tiles
  if (real)
#pragma unroll
    for (int t = 0; t < ST / 2; ++t) {
      const int c = 32 * t + 8 * g;
      if (c >= a.dk) continue;
      float x[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = D[2 * t][r], x[4 + r] = D[2 * t + 1][r];
      T* to = (FOR_K ? dk : dq) + ((size_t)orig * a.Hk + hk) * a.dk + c;
      *reinterpret_cast<Raw<T, 8>*>(to) = Frag<T, 8>::from_f32(x);
    }
}

struct BackArgs {
  const void *q, *k, *v, *dout;
  const float *g, *beta, *state_in, *dstate_out;
  void *dq, *dk, *dv;
  float *dg, *dbeta, *dstate_in;
};

template <typename T, int DK>
hipError_t backward_impl(const Args& a, int dtype, const BackArgs& b, void* workspace, hipStream_t stream) {
  const BackSpace sp = back_space(a.n, a.W, dtype, a.Hk, a.H, a.dk, a.dv);
  char* ws = static_cast<char*>(workspace);
  _Float16* images = reinterpret_cast<_Float16*>(ws + sp.base.images);
  _Float16* records = reinterpret_cast<_Float16*>(ws + sp.base.records);
  const auto at = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  const T *v = static_cast<const T*>(b.v), *dout = static_cast<const T*>(b.dout);
  if (a.n > 0)
    k_delta_prep<T, DK, true><<<dim3(a.slots, a.Hk), 256, 0, stream>>>(
        a, static_cast<const T*>(b.q), static_cast<const T*>(b.k), b.g, b.beta, images, records);
  _Float16* maps = reinterpret_cast<_Float16*>(ws + sp.maps);
  if (a.n > 0)
    launch_ends<T, DK>(a, v, b.state_in, images, records, kRecordBack, at(sp.ends), maps, stream);
  with_walk<T, DK>(a, [&](auto nw, auto ahead, dim3 grid) {
    constexpr int NW = decltype(nw)::value;
    if (a.n > 0)
      k_delta_walk<T, DK, kKeep, NW, decltype(ahead)::value><<<grid, 64 * NW, 0, stream>>>(
          a, v, b.state_in, images, records, kRecordBack, at(sp.ends), maps, nullptr, dout,
          WalkOut{nullptr, at(sp.states), at(sp.smax), at(sp.resid), at(sp.odo)});
    const auto back = [&](auto ends) {
      k_delta_back<T, DK, NW, decltype(ends)::value, decltype(ahead)::value><<<grid, 64 * NW, 0, stream>>>(
          a, dout, b.dstate_out, images, records, at(sp.back_ends), at(sp.states), at(sp.lam), at(sp.dstates),
          at(sp.dmax), at(sp.start), b.dstate_in);
    };
    if (a.part != 0 && a.n > 0) {
      back(std::true_type{});
      k_delta_join<DK, true><<<dim3(a.W, a.H, (a.dv / 16 + 3) / 4), 256, 0, stream>>>(a, at(sp.back_ends), maps);
    }
    back(std::false_type{});
  });
  const auto grad = [&](auto for_k) {
    k_delta_grad<T, DK, decltype(for_k)::value><<<dim3(a.slots, a.Hk), 256, 0, stream>>>(
        a, v, dout, b.g, images, records, at(sp.states), at(sp.dstates), at(sp.smax), at(sp.dmax), at(sp.resid),
        at(sp.lam), at(sp.odo), at(sp.start), b.state_in != nullptr, b.dstate_out != nullptr, static_cast<T*>(b.dq),
        static_cast<T*>(b.dk), static_cast<T*>(b.dv), b.dg, b.dbeta);
  };
  if (a.n > 0) {
    grad(std::false_type{});
    grad(std::true_type{});
  }
  return hipGetLastError();
}

template <typename T>
hipError_t backward_dk(const Args& a, int dtype, const BackArgs& b, void* workspace, hipStream_t stream) {
  switch (pad_dk(a.dk)) {
    case 32: return backward_impl<T, 32>(a, dtype, b, workspace, stream);
    case 64: return backward_impl<T, 64>(a, dtype, b, workspace, stream);
    default: return backward_impl<T, 128>(a, dtype, b, workspace, stream);
  }
}

}  // namespace

size_t delta_backward_workspace_bytes(int64_t n, int32_t W, int dtype, int32_t Hk, int32_t H, int32_t dk,
                                      int32_t dv) {
  return back_space(n, W, dtype, Hk, H, dk, dv).total;
}

hipError_t launch_backward_delta(const int32_t* offsets, int32_t n, int32_t W, const int32_t* order, int dtype,
                                 int32_t Hk, int32_t H, int32_t dk, int32_t dv, float scale, const void* q,
                                 const void* k, const void* v, const float* g, const float* beta,
                                 const float* state_in, const void* dout, const float* dstate_out, void* dq,
                                 void* dk_out, void* dv_out, float* dg, float* dbeta, float* dstate_in,
                                 void* workspace, hipStream_t stream) {
  const Args a = args_of(offsets, n, W, order, Hk, H, dk, dv, scale);
  const BackArgs b{q, k, v, dout, g, beta, state_in, dstate_out, dq, dk_out, dv_out, dg, dbeta, dstate_in};
  if (dtype == 0) return backward_dk<float>(a, dtype, b, workspace, stream);
  if (dtype == 1) return backward_dk<_Float16>(a, dtype, b, workspace, stream);
  return backward_dk<bf16_t>(a, dtype, b, workspace, stream);
}

}  // namespace sla
