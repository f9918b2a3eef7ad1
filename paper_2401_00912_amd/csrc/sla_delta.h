// Shared parts of the gated delta rule (sla_delta.hip, sla_delta_bwd.hip,
// sla_delta_step.hip): the chunk form, the workspace, operands in two 16-bit terms.
//
// Chunk form.  A window is cut into chunks of 64 rows.  With gam_i the log decays summed from
// the chunk's first row to row i, D_ij = exp(gam_i - gam_j) for j <= i, S0 the state before the
// chunk and u_j = beta_j r_j:
//     r = T (v - exp(gam) k S0),   T = (I + [D_ij (k_i . k_j) beta_j]_{j < i})^-1,
//     o = scale (exp(gam) q S0 + P u),   P_ij = D_ij (q_i . k_j) for j <= i,
//     S1 = exp(gam_last) S0 + sum_j exp(gam_last - gam_j) k_j u_j^T.
// T and P depend on no state: one kernel makes them for all chunks at once, a second one goes
// through every window's chunks in order with the state in registers.
//
// Two-term operands.  The matrix cores' 16-bit products are 16 times as fast as their fp32 ones,
// and one 16-bit rounding of a state loses what fp32 states are kept for.  So an fp32 operand is
// scaled by a power of two and split into two fp16 terms, x = hi + lo (22 bits), and a product is
// the sum of hi hi, hi lo and lo hi in fp32.  With values under 2^-16 of the largest the second term
// runs out of fp16's least steps, and one of 2^-38 is lost.  That is no loss in a sum that the largest
// one is in too.  But T, P and what they are multiplied with hold rows that have nothing to do with each
// other, early ones and a late one a billion times as large: there x = hi + 2^-11 lo, with the products
// of the second terms summed by themselves, 22 bits down to 2^-27 of the largest and none at 2^-49.
// A 16-bit input needs no second term: its row is scaled by a power of two that puts the row's largest
// value into [1, 2), and then fp16 holds fp16 and bf16 values exactly down to 2^-17 of the row's largest
// (below that, to 2^-25 of it).
// With k = 2^kap k' and q = 2^rho q' the rule reads the same for k', u' = 2^kap u, o' = 2^-rho o and
// r' = s r with any s of a row's own:
//     r' = T' (s v - t exp(gam) k' S0),   t = 2^kap s,   u' = (b / t) r',   b = 2^(2 kap) beta,
//     T' = (I + [t_i D_ij (k'_i . k'_j) b_j / t_j]_{j < i})^-1,
// so the scales cost one factor a row.  A column of r' has one power of two for its two terms, so no row
// may be large there that writes little: s = min(2^-kap, c) with c the largest min(1, b) 2^-kap of the
// chunk, which is what a row's v is worth to the state (and at least the smallest 2^-kap, where betas are
// small).  With s = 2^-kap alone a key of 1e-9 among keys of 1 put its v' 2^30 above theirs, and their r'
// were lost.  b / t is at most max(1, b), and wherever beta |k|^2 <= 2 (where the rule is stable) the
// entries of T' stay below 4 dk and those of the transposed inverse (rows with b) below 2 sqrt(4 dk).
#pragma once

#include "sla_common.h"

namespace sla {
namespace delta {

constexpr int kChunk = 64;
constexpr int kFrag = 512;            // halfs of one 16 x 32 operand: 64 lanes x 8
constexpr int kTri = 6;               // 16 x 32 operands of a lower triangular 64 x 64 matrix
constexpr int kTriHalfs = 2 * kTri * kFrag;
constexpr int kScal = 768;            // 4-byte values: 11 rows of 64, and single ones
// Rows of a chunk's scalars: exp(gam), b / t, exp(gam_last - gam), s, 2^rho scale; the original rows
// (int32) of the chunk and of its window's next and previous chunk, which are asked for while this one is in
// work; exp(gam_last); the factors that the four tile rows of T, P and their transposes are to be multiplied
// with (powers of two: rows of a growing state, g > 0, are far from each other's size, and one factor for all
// had them overflow); t exp(gam), b and 2^-kap.
enum { kSince = 0, kWrite = 64, kUntil = 128, kVScale = 192, kOScale = 256, kRow = 320, kNext = 384, kPrev = 448,
       kLast = 512, kTDown = 516, kPDown = 520, kBackTDown = 524, kBackPDown = 528, kSinceK = 576, kBeta = 640,
       kKScale = 704 };
// What a chunk has for each value head, in halfs: P's second and first terms, T's first and second,
// the scalars, and for the backward the transposed inverse and the transposed P, two terms each.
// The walk forward reads up to the scalars, the walk back from there.
constexpr int kTerm = kTriHalfs / 2;
enum { kPLo = 0, kPHi = kTerm, kTHi = 2 * kTerm, kScalAt = 4 * kTerm, kBackT = kScalAt + 2 * kScal,
       kBackP = kBackT + 2 * kTerm };
constexpr int kRecord = kBackT, kRecordBack = kBackP + 2 * kTerm;

struct Args {
  const int32_t* offsets;
  const int32_t* order;
  int32_t n, W, Hk, H, dk, dv;
  float scale;
  uint32_t slots;                     // n / 64 + W
  int32_t part;                       // chunks of a part of a window; 0: windows are not parted
};

// Workspace of the chunk form: per chunk slot and query/key head the images of q' and k', per slot and
// value head a record.
struct Space {
  size_t image, images, records, total;   // halfs of one image; byte offsets
};

__host__ __device__ inline int pad_dk(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }

__host__ __device__ inline size_t slots_of(int64_t n, int32_t W) { return (size_t)(n / kChunk + W); }

__host__ __device__ inline Space space_of(int64_t n, int32_t W, int dtype, int32_t Hk, int32_t H, int32_t dk,
                                          int record) {
  Space s;
  const size_t ns = slots_of(n, W);
  s.image = (size_t)(dtype == 0 ? 2 : 1) * kChunk * pad_dk(dk);
  s.images = 0;
  s.records = align_up(s.images + ns * Hk * 2 * s.image * 2, 256);
  s.total = align_up(s.records + ns * H * record * 2, 256);
  return s;
}

// ------------------------------------------------------------------ windows and slots
struct Win {
  int32_t begin, rows;
};
__device__ __forceinline__ Win window(const Args& a, int w) {
  int b = a.offsets[w], e = a.offsets[w + 1];
  b = b < 0 ? 0 : b > a.n ? a.n : b;
  e = e < b ? b : e > a.n ? a.n : e;
  return {b, e - b};
}
// First chunk slot of a window: chunks of different windows never share a slot, since a window of
// m rows from row b has at most floor((b + m) / 64) - floor(b / 64) + 1 chunks, and no scan over
// the windows is needed to place them.
__device__ __forceinline__ uint32_t first_slot(int begin, int w, uint32_t rows = kChunk) {
  return (uint32_t)begin / rows + (uint32_t)w;
}

// The window whose chunk `slot` is, if any is: first slots grow with the window, so each step of the
// search probes 64 windows at once (a lane each) and one of a few thousand is found in two loads.
// (Parts of `rows` rows have slots in the same way.)
__device__ __forceinline__ int window_of(const Args& a, uint32_t slot, int lane, uint32_t rows = kChunk) {
  int lo = 0, hi = a.W;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, w = lo + lane * step;
    bool at_most = false;
    if (w < hi) {
      const int b = a.offsets[w];
      at_most = first_slot(b < 0 ? 0 : b > a.n ? a.n : b, w, rows) <= slot;
    }
    const int count = __popcll(__ballot(at_most));
    lo += (count > 0 ? count - 1 : 0) * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

// Original row of position p (order: the caller's, clamped so that nothing is read out of range).
__device__ __forceinline__ int row_at(const Args& a, int p) {
  if (a.order == nullptr) return p;
  const int r = a.order[p];
  return r < 0 ? 0 : r >= a.n ? a.n - 1 : r;
}

// A row out of a chunk's record.  Where offsets are not as they should be no launch may have written that
// record, so a row is bounded here again.
__device__ __forceinline__ int kept_row(const Args& a, float x) {
  return (int)min(__float_as_uint(x), (uint32_t)a.n - 1u);
}

// ------------------------------------------------------------------ operands
struct Pair {
  half8_t hi, lo;
};
struct Far {   // second terms 2^11 times as large as what they stand for
  half8_t hi, lo;
};
struct FarSum {
  floatx4 lo = {0.f, 0.f, 0.f, 0.f}, hi = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ floatx4 all() const { return hi + lo * 0x1p-11f; }
};

__device__ __forceinline__ floatx4 mma(half8_t a, half8_t b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// products with both operands in two terms; the lo lo term is below 2^-22 of the product
__device__ __forceinline__ floatx4 mma2(const Pair& a, const Pair& b, floatx4 c) {
  c = mma(a.lo, b.hi, c);
  c = mma(a.hi, b.lo, c);
  return mma(a.hi, b.hi, c);
}
__device__ __forceinline__ void mma2(const Far& a, const Far& b, FarSum& c) {
  c.lo = mma(a.lo, b.hi, c.lo);
  c.lo = mma(a.hi, b.lo, c.lo);
  c.hi = mma(a.hi, b.hi, c.hi);
}
__device__ __forceinline__ floatx4 mma1(half8_t a, const Pair& b, floatx4 c) {
  c = mma(a, b.lo, c);
  return mma(a, b.hi, c);
}
__device__ __forceinline__ floatx4 mma1(const Pair& a, half8_t b, floatx4 c) {
  c = mma(a.lo, b, c);
  return mma(a.hi, b, c);
}

// x scaled by s as two fp16 terms, two instructions a value (Far: three): each term is one multiply-add
// that rounds to fp16, the second one's addend the first term.  (The first terms are hidden from the
// compiler once they are there: it would make them again for the second.)
template <class P = Pair>
__device__ __forceinline__ P split(const floatx4& x0, const floatx4& x1, float s) {
  typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
  P p;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float a = e < 4 ? x0[e] : x1[e - 4], b = e < 4 ? x0[e + 1] : x1[e - 3];
    half2_t h = {(_Float16)__builtin_fmaf(a, s, 0.f), (_Float16)__builtin_fmaf(b, s, 0.f)};
    uint32_t u = __builtin_bit_cast(uint32_t, h);
    asm("" : "+v"(u));
    h = __builtin_bit_cast(half2_t, u);
    p.hi[e] = h[0];
    p.hi[e + 1] = h[1];
    if constexpr (std::is_same<P, Far>::value) {
      p.lo[e] = (_Float16)__builtin_fmaf(__builtin_fmaf(a, s, -(float)h[0]), 0x1p11f, 0.f);
      p.lo[e + 1] = (_Float16)__builtin_fmaf(__builtin_fmaf(b, s, -(float)h[1]), 0x1p11f, 0.f);
    } else {
      p.lo[e] = (_Float16)__builtin_fmaf(a, s, -(float)h[0]);
      p.lo[e + 1] = (_Float16)__builtin_fmaf(b, s, -(float)h[1]);
    }
  }
  return p;
}

// Largest value of the wave of a lane's non-negative m; a lane with an infinity or a NaN does not
// count (its column is lost, the others keep their scale).
__device__ __forceinline__ uint32_t wave_max_bits(float m) {
  uint32_t b = __float_as_uint(m);
  b = b >= 0x7f800000u ? 0u : b;
  auto step = [&](int v) {
    const uint32_t o = (uint32_t)v;
    b = o > b ? o : b;
  };
  step(__builtin_amdgcn_mov_dpp((int)b, 0x128, 0xf, 0xf, false));   // row_ror:8
  step(__builtin_amdgcn_mov_dpp((int)b, 0x124, 0xf, 0xf, false));
  step(__builtin_amdgcn_mov_dpp((int)b, 0x122, 0xf, 0xf, false));
  step(__builtin_amdgcn_mov_dpp((int)b, 0x121, 0xf, 0xf, false));
  const uint32_t r0 = __builtin_amdgcn_readlane(b, 0), r1 = __builtin_amdgcn_readlane(b, 16);
  const uint32_t r2 = __builtin_amdgcn_readlane(b, 32), r3 = __builtin_amdgcn_readlane(b, 48);
  const uint32_t x = r0 > r1 ? r0 : r1, y = r2 > r3 ? r2 : r3;
  return x > y ? x : y;
}

// Largest value of the four lanes that have a column (or row) i of a tile between them, of their non-negative
// m; infinities and NaN as above.
__device__ __forceinline__ uint32_t column_max_bits(float m) {
  uint32_t b = __float_as_uint(m);
  b = b >= 0x7f800000u ? 0u : b;
  const auto x = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = x[0] > x[1] ? x[0] : x[1];
  const auto y = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return y[0] > y[1] ? y[0] : y[1];
}

// The power of two that puts a largest value with these bits into [2^13, 2^14), and its inverse.
// At 2^14 the products of 64 terms stay far inside fp32.
struct Scale {
  float up, down;
};
__device__ __forceinline__ float inverse_pow2(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }
__device__ __forceinline__ Scale scale_of(uint32_t max_bits) {
  if (max_bits == 0) return {1.f, 1.f};
  const int e = (int)(max_bits >> 23);
  const int s = 267 - e < 240 ? 267 - e : 240;
  return {__uint_as_float((uint32_t)s << 23), __uint_as_float((uint32_t)(254 - s) << 23)};
}

template <int N>
__device__ __forceinline__ float max_of(const floatx4 (&x)[N]) {
  float m = 0.f;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(x[t][r]));
  return m;
}
template <int N>
__device__ __forceinline__ Scale scale_for(const floatx4 (&x)[N]) {
  return scale_of(wave_max_bits(max_of(x)));
}
template <int N>
__device__ __forceinline__ Scale column_scale(const floatx4 (&x)[N]) {
  return scale_of(column_max_bits(max_of(x)));
}
// of the four lane groups' columns 4g .. 4g + 3, as a transposed tile has them: x of a lane's column i
__device__ __forceinline__ floatx4 across(float x, int g) {
  floatx4 y;
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = __shfl(x, 4 * g + r);
  return y;
}

// ------------------------------------------------------------------ images
// Half index of (row, column) in the image of a 64 x DK matrix: operands of 16 rows x 32 columns
// in the matrix cores' order (lane (i, g) holds row i, columns 8g .. 8g + 7), the rows of lane
// group g turned by 4g, so that the transpose reads of 4 rows x 4 column groups fall into
// different banks.
template <int DK>
__device__ __forceinline__ int image_at(int row, int kb, int g) {
  return (((row >> 4) * (DK / 32) + kb) * 64 + g * 16 + (((row & 15) + 4 * g) & 15)) * 8;
}

typedef short short4v __attribute__((ext_vector_type(4)));

// rows of tile `tau`, columns 32 kb .. + 31: contraction over columns
template <int DK>
__device__ __forceinline__ half8_t image_rows(const _Float16* img, int tau, int kb, int i, int g) {
  return *reinterpret_cast<const half8_t*>(img + image_at<DK>(16 * tau + i, kb, g));
}
// Columns as rows: operand row m stands for column 32 t + 8 (m / 4) + 4 p + m % 4 (the order in
// which the state's tiles hold their rows), contraction over rows 32 s .. 32 s + 31, element e of
// lane group g standing for row 32 s + 16 (e / 4) + 4 g + e % 4 (the order in which two 16-row
// result tiles make one operand).  Lane j of 16 addresses row j / 4 and column group j % 4 of a
// 4 x 16 block and receives column j of its four rows.
template <int DK>
__device__ __forceinline__ half8_t image_cols(const _Float16* img, int t, int p, int s, int i, int g) {
  half8_t x;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const _Float16* at = img + image_at<DK>(32 * s + 16 * h + 4 * g + (i >> 2), t, i & 3) + 4 * p;
    const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) short4v*)(const_cast<_Float16*>(at)));
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * h + r] = __builtin_bit_cast(_Float16, (short)y[r]);
  }
  return x;
}
// Number of row tile tau's operand for column block s in a triangle's term:
__device__ __forceinline__ constexpr int tri_at(int tau, int s) { return tau < 2 ? tau : 2 * tau - 2 + s; }

// ------------------------------------------------------------------ staging
// 64 x 16 bytes from every lane's address in global memory into LDS at `lds`, in lane order, without
// passing registers.  Counted with the wave's vector memory operations.
__device__ __forceinline__ void to_lds(void* lds, const void* src) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
// Barrier of the workgroup, after the wave's own LDS and vector memory operations.
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------------------ storage types
template <typename T>
using Bits = std::conditional_t<std::is_same<T, float>::value, float, unsigned short>;
template <typename T>
__device__ __forceinline__ float widen(Bits<T> x) {
  if constexpr (std::is_same<T, float>::value) return x;
  else return u16_to_f32<T>(x);
}
template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (std::is_same<T, float>::value) return *p;
  else return u16_to_f32<T>(*reinterpret_cast<const unsigned short*>(p));
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const floatx4& x) {
  if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<floatx4*>(p) = x;
  } else {
    u16x4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = f32_to_u16<T>(x[r]);
    *reinterpret_cast<u16x4*>(p) = y;
  }
}
template <typename T>
constexpr int kTerms = std::is_same<T, float>::value ? 2 : 1;

}  // namespace delta
}  // namespace sla
