// The chunk form's two forward kernels: T and P of every chunk, and the walk through a window's
// chunks.  Included by the forward and by the backward, which makes the states again.
#pragma once

#include "sla_delta.h"

namespace sla {
namespace delta {

constexpr int kLd = 68;   // floats a row of a 64 x 64 matrix in LDS: 16-byte rows, banks turned by 4

// ------------------------------------------------------------------ T and P
// Per chunk and query/key head, 256 threads: k' and q' into LDS in operand order (and into the
// workspace: the walk stages them from there as they are), k'k'^T and q'k'^T lower tiles one tile
// row per wave, then for each value head of the group the decays, the inverse and the two
// triangles.  The inverse of the unit lower triangular 64 x 64 matrix goes by 16 x 16 blocks: the
// four diagonal ones by substitution (one wave each, a column a lane), the others, diagonal after
// diagonal, as X_ij = -X_ii sum_k N_ik X_kj on the fp32 matrix cores.
//
// REV: also the transposed triangles for the reverse walk, with the inverse of
// I + [beta_i D_ij k_i . k_j], whose rows and not columns carry beta.
//
// Chunks are independent here, so a batch is bound by memory: 65,536 bf16 rows, 16 heads of 128, in
// 326 us, 1.5 GB, 4.7 TB/s (a copy reaches 5.2).  Windows of one chunk are bound by the steps between
// the barriers, some 10 us a workgroup: 1,521 fp16 windows (59,837 rows, 4 heads of 32) in 79 us, 148
// with REV.  The inverse is made here and not in the walk because there it would be part of the chain
// from chunk to chunk.
struct PrepShared {
  float n[kChunk * kLd];
  float x[kChunk * kLd];
};

__device__ __forceinline__ floatx4 mma_f32(const floatx4& a, const floatx4& b, floatx4 c) {
#pragma unroll
  for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
  return c;
}

// x = (I + n)^-1 for strictly lower n; upper blocks of x that the operands read become zero.
__device__ __forceinline__ void invert(PrepShared& s, int wave, int i, int g) {
  {
    // column i of the inverse: row after row is finished and taken out of those below it
    float col[16];
#pragma unroll
    for (int a = 0; a < 16; ++a) col[a] = a == i ? 1.f : 0.f;
#pragma unroll
    for (int b4 = 0; b4 < 4; ++b4) {
#pragma unroll
      for (int a4 = b4; a4 < 4; ++a4) {   // rows 4 a4 .. + 3 less what rows 4 b4 .. + 3 have of them
        floatx4 row[4];
#pragma unroll
        for (int a = 0; a < 4; ++a)
          row[a] = *reinterpret_cast<const floatx4*>(s.n + (16 * wave + 4 * a4 + a) * kLd + 16 * wave + 4 * b4);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            if (a4 > b4 || a > b) col[4 * a4 + a] -= row[a][b] * col[4 * b4 + b];
      }
    }
#pragma unroll
    for (int a = 0; a < 16; ++a)
      if ((a >> 2) == g) s.x[(16 * wave + a) * kLd + 16 * wave + i] = col[a];
    if ((wave & 1) == 0)
#pragma unroll
      for (int r = 0; r < 4; ++r) s.x[(16 * wave + 4 * g + r) * kLd + 16 * (wave + 1) + i] = 0.f;
  }
  __syncthreads();
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    if (wave < 4 - d) {
      const int bi = wave + d, bj = wave;
      floatx4 sum = {0.f, 0.f, 0.f, 0.f};
      for (int k = bj; k < bi; ++k) {
        const floatx4 a = *reinterpret_cast<const floatx4*>(s.n + (16 * bi + i) * kLd + 16 * k + 4 * g);
        floatx4 b;
#pragma unroll
        for (int r = 0; r < 4; ++r) b[r] = s.x[(16 * k + 4 * g + r) * kLd + 16 * bj + i];
        sum = mma_f32(a, b, sum);
      }
      floatx4 a = *reinterpret_cast<const floatx4*>(s.x + (16 * bi + i) * kLd + 16 * bi + 4 * g);
      floatx4 zero = {0.f, 0.f, 0.f, 0.f};
      sum = mma_f32(a, sum, zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) s.x[(16 * bi + 4 * g + r) * kLd + 16 * bj + i] = -sum[r];
    }
    __syncthreads();
  }
}

// The triangle's operands of tile row `tau` out of a matrix in LDS: rows as operand rows, columns
// in the order of two stacked result tiles, and to `down` the factor that belongs to the tile row.
__device__ __forceinline__ void put_tri(const float* m, _Float16* hi, _Float16* lo, float* down, int tau, int lane,
                                        int i, int g) {
  floatx4 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (j / 2 <= tau / 2) x[j] = *reinterpret_cast<const floatx4*>(m + (16 * tau + i) * kLd + 16 * j + 4 * g);
  }
  const Scale sc = scale_for(x);
  if (lane == 0) down[tau] = sc.down;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (s > tau / 2) continue;
    const Far p = split<Far>(x[2 * s], x[2 * s + 1], sc.up);
    const int at = tri_at(tau, s) * kFrag + lane * 8;
    *reinterpret_cast<half8_t*>(hi + at) = p.hi;
    *reinterpret_cast<half8_t*>(lo + at) = p.lo;
  }
}
// The transposed matrix's operands of tile row `tau`: upper triangular, kept under the mirrored
// numbers (row tile 3 - tau, column block 1 - s).
__device__ __forceinline__ void put_tri_t(const float* m, _Float16* out, float* down, int tau, int lane, int i, int g) {
  floatx4 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (j / 2 >= tau / 2)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[j][r] = m[(16 * j + 4 * g + r) * kLd + 16 * tau + i];
  }
  const Scale sc = scale_for(x);
  if (lane == 0) down[tau] = sc.down;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (s < tau / 2) continue;
    const Far p = split<Far>(x[2 * s], x[2 * s + 1], sc.up);
    _Float16* at = out + tri_at(3 - tau, 1 - s) * kFrag + lane * 8;
    *reinterpret_cast<half8_t*>(at) = p.hi;
    *reinterpret_cast<half8_t*>(at + kTri * kFrag) = p.lo;
  }
}

template <typename T, int DK, bool REV>
__global__ __launch_bounds__(256, 3) void k_delta_prep(Args a, const T* __restrict__ q, const T* __restrict__ k,
                                                    const float* __restrict__ gin, const float* __restrict__ beta,
                                                    _Float16* __restrict__ images,
                                                    _Float16* __restrict__ records) {
  constexpr int NT = kTerms<T>, KB = DK / 32, IMG = kChunk * DK;
  constexpr size_t kImages = (size_t)2 * NT * IMG * 2;
  __shared__ __attribute__((aligned(16))) char s_mem[kImages > sizeof(PrepShared) ? kImages : sizeof(PrepShared)];
  __shared__ double s_gam[2][kChunk];
  __shared__ __attribute__((aligned(16))) float s_t[2][kChunk];
  __shared__ float s_write[2][kChunk], s_b[2][kChunk], s_ks[kChunk], s_os[kChunk];
  _Float16* s_img = reinterpret_cast<_Float16*>(s_mem);
  PrepShared& sm = *reinterpret_cast<PrepShared*>(s_mem);

  const uint32_t slot = blockIdx.x;
  const int hk = blockIdx.y;
  const int lo = window_of(a, slot, threadIdx.x & 63);
  const Win win = window(a, lo);
  const uint32_t f = first_slot(win.begin, lo);
  if (slot < f || (int64_t)(slot - f) * kChunk >= win.rows) return;
  const int base = win.begin + (int)(slot - f) * kChunk;
  const int rows = min(kChunk, win.rows - (int)(slot - f) * kChunk);

  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // wave 0, a row a lane: where the rows are, and one head ahead their log decays and betas
  const int group = a.H / a.Hk;
  const bool mine = wave == 0 && lane < rows;
  int place = 0, place_next = 0, place_prev = 0;
  float g1 = 0.f, b1 = 0.f;
  const auto ask = [&](int hv) __attribute__((always_inline)) {
    const size_t at = (size_t)place * a.H + hk * group + hv;
    g1 = mine ? gin[at] : 0.f;
    b1 = mine ? beta[at] : 0.f;
  };
  if (wave == 0) {
    // a row that is none: row 0, or its chunk's first row; it is dropped when it is used
    const int p1 = base + kChunk + lane, p0 = base - kChunk + lane, end = win.begin + win.rows;
    if (mine) place = row_at(a, base + lane);
    if (base + kChunk < end) place_next = row_at(a, p1 < end ? p1 : base + kChunk);
    if (p0 >= win.begin) place_prev = row_at(a, p0);
    ask(0);
  }
  {
    const int row = tid >> 2, gg = tid & 3;
    const bool real = row < rows;
    const int r = real ? row_at(a, base + row) : 0;
#pragma unroll
    for (int which = 0; which < 2; ++which) {   // 0: q, 1: k
      const T* src = (which ? k : q) + ((size_t)r * a.Hk + hk) * a.dk;
      float x[KB][8];
      float m = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int c = 32 * kb + 8 * gg;
        Raw<T, 8> raw = Frag<T, 8>::zero();
        if (real && c < a.dk) raw = *reinterpret_cast<const Raw<T, 8>*>(src + c);
        Frag<T, 8>::to_f32(raw, x[kb]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[kb][e]));
      }
      m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0xB1, 0xf, 0xf, false)));
      m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x4E, 0xf, 0xf, false)));
      int e2 = (int)(__float_as_uint(m) >> 23) - 127;
      e2 = m == 0.f || e2 > 127 ? 0 : e2 < -60 ? -60 : e2 > 60 ? 60 : e2;
      const float down = __uint_as_float((uint32_t)(127 - e2) << 23), up = __uint_as_float((uint32_t)(127 + e2) << 23);
      _Float16* img = s_img + which * NT * IMG;
      _Float16* gimg = images + (((size_t)slot * a.Hk + hk) * 2 + which) * NT * IMG;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        half8_t h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = x[kb][e] * down;
          h[e] = (_Float16)y;
          if constexpr (NT == 2) l[e] = (_Float16)(y - (float)h[e]);
        }
        const int at = image_at<DK>(row, kb, gg);
        *reinterpret_cast<half8_t*>(img + at) = h;
        *reinterpret_cast<half8_t*>(gimg + at) = h;
        if constexpr (NT == 2) {
          *reinterpret_cast<half8_t*>(img + IMG + at) = l;
          *reinterpret_cast<half8_t*>(gimg + IMG + at) = l;
        }
      }
      if (gg == 0) {
        (which ? s_ks : s_os)[row] = up;
      }
    }
  }
  // Decay sums of head hv, in powers of two and in 64 bits: their differences are small where they are
  // large, and as an exponent a difference is exact enough in fp32 (2^t's own step is 2^-24 t).  A decay
  // that is zero in fp32 (g below -104, -infinity) counts as 2^-65536, so that no power across it is left.
  const auto sums = [&](int hv) __attribute__((always_inline)) {
    if (wave != 0) return;
    double gam = g1 < -104.f ? -65536.0 : (double)g1 * 1.4426950408889634;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double o = __shfl_up(gam, d);
      if (lane >= d) gam += o;
    }
    s_gam[hv & 1][lane] = gam;
    // the scales of r' (sla_delta.h); a beta that is no number does not count
    const float ks = s_ks[lane], b = b1 * ks * ks, worth = b == b ? fminf(1.f, fabsf(b)) * inverse_pow2(ks) : 0.f;
    const float top = __uint_as_float(wave_max_bits(lane < rows ? ks : 0.f));
    const float c = __uint_as_float((wave_max_bits(worth) + 0x7fffffu) & 0x7f800000u);   // the next power of two
    const float s = fminf(inverse_pow2(ks), fmaxf(c, inverse_pow2(top)));
    s_write[hv & 1][lane] = b1 * ks * inverse_pow2(s);
    s_t[hv & 1][lane] = s * ks;
    s_b[hv & 1][lane] = b;
    if (hv + 1 < group) ask(hv + 1);
  };
  __syncthreads();
  sums(0);

  // lower tiles of k'k'^T and q'k'^T, tile row `wave`
  floatx4 kk[4], qk[4];
  const _Float16 *qi = s_img, *ki = s_img + NT * IMG;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    kk[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    qk[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (j > wave) continue;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const half8_t kr = image_rows<DK>(ki, wave, kb, i, g), qr = image_rows<DK>(qi, wave, kb, i, g);
      const half8_t kc = image_rows<DK>(ki, j, kb, i, g);
      if constexpr (NT == 2) {
        const half8_t krl = image_rows<DK>(ki + IMG, wave, kb, i, g), qrl = image_rows<DK>(qi + IMG, wave, kb, i, g);
        const half8_t kcl = image_rows<DK>(ki + IMG, j, kb, i, g);
        kk[j] = mma(kr, kcl, mma(krl, kc, kk[j]));
        qk[j] = mma(qr, kcl, mma(qrl, kc, qk[j]));
      }
      kk[j] = mma(kr, kc, kk[j]);
      qk[j] = mma(qr, kc, qk[j]);
    }
  }
  __syncthreads();   // the images' place is the matrices' from here

  const int lane0 = lane;
  for (int hv = 0; hv < group; ++hv) {
    // the lane's numbers anew for every head, so that what follows from them takes no registers over the loop
    int lane = lane0;
    asm volatile("" : "+v"(lane));
    const int i = lane & 15, g = lane >> 4;
    const int h = hk * group + hv;
    const size_t sh = (size_t)slot * a.H + h;
    _Float16* out = records + sh * (REV ? kRecordBack : kRecord);
    float* sc = reinterpret_cast<float*>(out + kScalAt);
    const double* gam = s_gam[hv & 1];
    const float *write = s_write[hv & 1], *t = s_t[hv & 1], *b = s_b[hv & 1];
    if (wave == 0) {
      const bool real = lane < rows;
      const double gl = gam[lane], last = gam[63];
      const float kd = inverse_pow2(s_ks[lane]), since = real ? __builtin_amdgcn_exp2f((float)gl) : 0.f;
      sc[kSince + lane] = since;
      sc[kWrite + lane] = write[lane];
      sc[kUntil + lane] = real ? __builtin_amdgcn_exp2f((float)(last - gl)) : 0.f;
      sc[kVScale + lane] = t[lane] * kd;
      sc[kSinceK + lane] = t[lane] * since;
      sc[kBeta + lane] = b[lane];
      sc[kKScale + lane] = kd;
      sc[kOScale + lane] = s_os[lane] * a.scale;
      sc[kRow + lane] = __int_as_float(place);
      sc[kNext + lane] = __int_as_float(place_next);
      sc[kPrev + lane] = __int_as_float(place_prev);
      if (lane == 0) sc[kLast] = __builtin_amdgcn_exp2f((float)last);
    }
    floatx4 d[4];   // decays between the rows, zero above the diagonal
    double gr[4];
    const floatx4 tr = *reinterpret_cast<const floatx4*>(t + 16 * wave + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r) gr[r] = gam[16 * wave + 4 * g + r];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = 16 * j + i;
      d[j] = floatx4{0.f, 0.f, 0.f, 0.f};
      floatx4 n = d[j];
      if (j <= wave) {
        const double gc = gam[col];
        const float bc = write[col];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * wave + 4 * g + r;
          d[j][r] = row >= col ? __builtin_amdgcn_exp2f((float)(gr[r] - gc)) : 0.f;
          n[r] = row > col ? d[j][r] * kk[j][r] * (tr[r] * bc) : 0.f;
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) sm.n[(16 * wave + 4 * g + r) * kLd + col] = n[r];
    }
    __syncthreads();
    invert(sm, wave, i, g);
    const bool here = 16 * wave < rows;   // pieces of tile rows past the last row are not written (nor moved)
    if (here) put_tri(sm.x, out + kTHi, out + kTHi + kTerm, sc + kTDown, wave, lane, i, g);
    if constexpr (REV) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * wave + 4 * g + r, col = 16 * j + i;
          sm.n[row * kLd + col] = row > col ? d[j][r] * kk[j][r] * b[row] : 0.f;
        }
      __syncthreads();
      invert(sm, wave, i, g);
      put_tri_t(sm.x, out + kBackT, sc + kBackTDown, wave, lane, i, g);
    }
    // every wave is past its reads of n (the inverse's last barrier)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        sm.n[(16 * wave + 4 * g + r) * kLd + 16 * j + i] = d[j][r] == 0.f ? 0.f : d[j][r] * qk[j][r];
    __syncthreads();
    if (here) put_tri(sm.n, out + kPHi, out + kPLo, sc + kPDown, wave, lane, i, g);
    if constexpr (REV) put_tri_t(sm.n, out + kBackP, sc + kBackPDown, wave, lane, i, g);
    if (hv + 1 < group) sums(hv + 1);
    __syncthreads();
  }
}

// ------------------------------------------------------------------ the walk
// A wave holds 16 of the state's dv columns in registers, as result tiles: tile 2t + p, component r
// of lane (i, g) is state row 32 t + 8 g + 4 p + r, column i.  Two tiles are then an operand of the
// products with k' and q' without moving a value, and so are the chunk's r and u (16 rows a tile);
// the columns are independent of each other, so no wave waits for another but for the staging.  Each
// column (a lane's i) has powers of two of its own for the two terms of its operands, so that a large
// value in one costs the others nothing.
//
// The chunks of a window depend on each other, so their latency counts: a chunk's images, triangles,
// scalars and the waves' columns of v are moved into the second of two LDS buffers while the first
// one's chunk is worked on, with one barrier a chunk.  fp32 rows of dk = 128 do not fit twice and are
// staged between two barriers.
//
// Bound by the chain: some 5 us a chunk of 128 x 128 states with eight waves a workgroup, whatever else
// the chip does.  65,536 bf16 rows, 33 uneven sequences, 16 heads: 580 to 815 us with the sequences' lengths,
// the longest one's chunks one after the other; 12,289 rows cut into parts: 57 us behind 95 for the parts'
// states; 1,521 fp16 windows of a chunk or two: 61 us, where a workgroup waits for its only chunk.  With one
// term for bf16 rows' outputs and one power of two for 16 columns the batch's walk took 486 to 725 us.
struct WalkOut {
  float* state_out;    // final states or null
  float* states;       // the states before every chunk [slot][H][dv / 16], in register order, or null
  float* smax;         // their largest magnitudes [slot][H][dv / 16], or null
  float* resid;        // r' of every chunk row [slot][H][64][dv], or null
  float* odo;          // sums over 16 columns of o dout [slot][H][dv / 16][64], or null
};

// What a walk reads of a chunk: the images from kImgAt on and the record from kRecAt (or later) to kRecTo.
template <typename T, int DK, int NW, int kImgAt_, int kRecAt_, int kRecTo_>
struct Stage {
  static constexpr int kImages = 2 * kTerms<T> * kChunk * DK;   // halfs of both images
  static constexpr int kImgAt = kImgAt_, kRecAt = kRecAt_, kRecTo = kRecTo_, kWaves = NW;
  __attribute__((aligned(16))) _Float16 img[kImages - kImgAt];
  __attribute__((aligned(16))) _Float16 rec[kRecTo - kRecAt];
  __attribute__((aligned(16))) T rows[NW][kChunk * 16];         // 16 columns of v (or dout) a wave
};
template <class S>
constexpr bool kTwice = 2 * sizeof(S) <= 160 * 1024;

// Instructions that move a wave's 64 rows of 16 columns: 16 bytes a lane.
template <typename T>
constexpr int kMoves = sizeof(T);
// Rows whose 16 bytes this lane moves.
template <typename T>
struct Places {
  int row[kMoves<T>];
  __device__ __forceinline__ static int position(int n, int lane) { return (n * 64 + lane) / kMoves<T>; }
  // of the chunk from position `base` on: a row past its end stands for the first one
  __device__ __forceinline__ void ask(const Args& a, int base, int rows, int lane) {
#pragma unroll
    for (int n = 0; n < kMoves<T>; ++n) row[n] = row_at(a, base + (position(n, lane) < rows ? position(n, lane) : 0));
  }
  __device__ __forceinline__ void take(const Args& a, const float* rows, int lane) {
#pragma unroll
    for (int n = 0; n < kMoves<T>; ++n) row[n] = kept_row(a, rows[position(n, lane)]);
  }
};

// A chunk on its way into a buffer: kJobs moves a wave, issued in parts between the steps of the chunk
// in work (all at once, they hold up the wave that issues them, and its stores behind them).  FROM: the
// first part of the record that is wanted.
template <class S, typename T, int FROM>
struct Fetch {
  static constexpr int NW = S::kWaves, kImg = (S::kImages - S::kImgAt) * 2 / 1024, kRec = (S::kRecTo - FROM) * 2 / 1024;
  static constexpr int kImgJobs = (kImg + NW - 1) / NW, kJobs = kImgJobs + (kRec + NW - 1) / NW;
  static_assert((S::kRecTo - FROM) * 2 % 1024 == 0 && FROM >= S::kRecAt, "whole pieces");
  const char *img, *rec;
  int pieces;   // of a triangle: those with rows in them

  // rows: the wave has columns of src to move; height: the chunk's rows
  __device__ __forceinline__ void start(S& b, const Args& a, size_t slot, int hk, int h, int cg, bool rows,
                                        const _Float16* images, const _Float16* records, int record, const T* src,
                                        const Places<T>& at, int wave, int lane, int height) {
    pieces = height > 32 ? 2 * ((height + 15) / 16) - 2 : (height + 15) / 16;
    const size_t sh = slot * a.H + h;
    img = reinterpret_cast<const char*>(images + (slot * a.Hk + hk) * S::kImages + S::kImgAt) + wave * 1024 + lane * 16;
    rec = reinterpret_cast<const char*>(records + sh * record + FROM) + wave * 1024 + lane * 16;
    if (rows) {
#pragma unroll
      for (int n = 0; n < kMoves<T>; ++n)
        to_lds(b.rows[wave] + n * (1024 / sizeof(T)),
               src + ((size_t)at.row[n] * a.H + h) * a.dv + 16 * cg + (lane % kMoves<T>) * (16 / (int)sizeof(T)));
    }
  }
  template <int J0, int J1>
  __device__ __forceinline__ void jobs(S& b, int wave) const {
#pragma unroll
    for (int j = J0; j < J1; ++j) {
      if (j < kImgJobs) {
        if ((j + 1) * NW <= kImg || wave + j * NW < kImg) to_lds(b.img + (wave + j * NW) * 512, img + j * NW * 1024);
      } else {
        const int p = j - kImgJobs, q = FROM / kFrag + wave + p * NW;
        if (FROM < kScalAt && q < kScalAt / kFrag && q % kTri >= pieces) continue;
        if ((p + 1) * NW <= kRec || wave + p * NW < kRec)
          to_lds(b.rec + (FROM - S::kRecAt) + (wave + p * NW) * 512, rec + p * NW * 1024);
      }
    }
  }
};

// ------------------------------------------------------------------ parts
// The chunks of one window are a chain, and a few long windows leave most of the chip idle.  Then
// windows are cut into parts of a.part chunks.  Across a part a state is mapped linearly, S' = M S + Z,
// with M the part's walk of the unit matrix without values and Z its walk of no state: a first walk
// makes them for all parts at once (M: dk more columns), a short chain per window joins them, and the
// walk proper starts every part from its state.  The walk back does the same with M^T.
// Part slots are numbered like chunk slots, with parts of 64 a.part rows.
struct Part {
  int w, lo, hi, chunks;   // window, its part's chunks [lo, hi), all of its chunks
  uint32_t slot;           // the part's
  bool none;
};
__device__ __forceinline__ int chunks_of(const Win& win) { return (int)(((int64_t)win.rows + kChunk - 1) / kChunk); }
__device__ __forceinline__ Part part_of(const Args& a, uint32_t slot, int lane) {
  Part p;
  p.slot = slot;
  if (a.part == 0) {
    p.w = (int)slot;
    p.lo = 0;
    p.hi = p.chunks = chunks_of(window(a, p.w));
    p.none = false;
    return p;
  }
  const uint32_t rows = (uint32_t)a.part * kChunk;
  p.w = window_of(a, slot, lane, rows);
  const Win win = window(a, p.w);
  const uint32_t f = first_slot(win.begin, p.w, rows);
  p.chunks = chunks_of(win);
  const int64_t lo = (int64_t)(slot - f) * a.part;
  // a window without rows has a first part without chunks
  p.none = slot < f || (slot > f && lo >= p.chunks);
  p.lo = p.none ? 0 : (int)lo;
  p.hi = min(p.lo + a.part, p.chunks);
  return p;
}
// A walk's window (or part) and value head: grid (part slots, heads, column groups).  Where whole windows are
// walked in more workgroups than there are CUs, the longest windows' heads come first, so that none is left
// alone at the end: a lane a window, up to 64.  65,536 bf16 rows, 33 uneven sequences, 16 heads of 128: 588 us
// so, 758 in the order of the windows (measured together, before the present operands).
struct Place {
  Part part;
  int h;
};
__device__ __forceinline__ Place place_of(const Args& a, int lane) {
  if (a.part != 0 || a.W > 64 || (size_t)gridDim.x * gridDim.y * gridDim.z <= 256)
    return {part_of(a, blockIdx.x, lane), (int)blockIdx.y};
  const int rows = lane < a.W ? window(a, lane).rows : -1;
  int before = 0;   // windows that come first: with more rows, or as many and a smaller number
  for (int o = 0; o < a.W; ++o) {
    const int other = __builtin_amdgcn_readlane(rows, o);
    before += other > rows || (other == rows && o < lane) ? 1 : 0;
  }
  const int at = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  const uint64_t hit = __ballot(lane < a.W && before == at / a.H);
  return {part_of(a, (uint32_t)(__ffsll((unsigned long long)hit) - 1), lane), at % a.H};
}
__host__ __device__ inline size_t part_slots(const Args& a) {
  return a.part == 0 ? (size_t)a.W : (size_t)(a.n / (a.part * kChunk)) + a.W;
}
// Parts of 8 to 32 chunks where that gives the chip some 512 workgroups of 64 columns; none where windows have
// under 256 rows on average, or where even parts of 32 chunks would be more than those 512 (n H dv / 64 over
// 2^20).  Forward, no parts and parts of 8, 16 and 32 chunks: 7 bf16 windows with 12,289 rows in all, 8 heads
// of 128: 346 us and 165, 192, 235; 1 fp32 window of 8,191 rows, 4 heads of 64: 459 us and 88, 124, 208.  The
// aim is not sharp: one bf16 window of 16,384 rows, 16 heads of 128, with 256, 512 and 1,024 workgroups 405,
// 431 and 411 us, gradients 1,616, 1,596 and 1,537.  Both bounds know the windows by their sum alone, and few
// long windows past them are a chain that the chip waits for: 16 heads of 128 bf16 in one window, 32,768 rows
// (parts) 855 us and gradients 3,025, 32,769 rows (none) 2,267 and 7,039, with parts 717 and 2,652; 16,000 rows
// 346 and 1,384, with 100 windows of 60 rows beside them (no parts) 1,548 and 4,761.
inline int part_chunks(int64_t n, int32_t W, int32_t H, int32_t dv) {
  const int64_t blocks = (int64_t)H * ((dv + 63) / 64), most = (n * blocks + 512 * kChunk - 1) / (512 * kChunk);
  const int64_t part = most < 8 ? 8 : most;
  if (part > 32 || n < 256 * (int64_t)W || n < 2 * part * kChunk) return 0;
  return (int)part;
}
inline Args args_of(const int32_t* offsets, int64_t n, int32_t W, const int32_t* order, int32_t Hk, int32_t H,
                    int32_t dk, int32_t dv, float scale) {
  return Args{offsets, order, (int32_t)n, W, Hk, H, dk, dv, scale, (uint32_t)slots_of(n, W), part_chunks(n, W, H, dv)};
}
// Halfs of the parts' ends (dk x dv states, in register order) and of their maps: M^T as an image in two terms, and
// for each column of M the factor it is to be multiplied with, a power of two.  (Under one factor for all maps
// a part that forgets lost M's bits with the decay: at e^-15, g = -0.03 over 512 rows, all but 9 of 22.)
__host__ __device__ constexpr int map_halfs(int DK) { return 2 * DK * DK + 2 * DK; }
__host__ __device__ inline size_t ends_halfs(const Args& a, int DK) { return part_slots(a) * a.H * (size_t)DK * a.dv * 2; }
__host__ __device__ inline size_t maps_halfs(const Args& a, int DK) { return part_slots(a) * a.H * (size_t)map_halfs(DK); }
inline size_t parts_bytes(const Args& a) {
  if (a.part == 0) return 0;
  const int DK = pad_dk(a.dk);
  return align_up((ends_halfs(a, DK) + maps_halfs(a, DK)) * 2, 256);
}

// The wave's columns of a staged chunk as result tiles, rows from `rows` on zero.
template <typename T>
__device__ __forceinline__ void rows_in(const T* at, floatx4 (&x)[4], int rows, int i, int g) {
#pragma unroll
  for (int tau = 0; tau < 4; ++tau) {
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
      for (int r = 0; r < 4; ++r) x[tau][r] = at[(16 * tau + 4 * g + r) * 16 + i];
    } else {
      const unsigned short* p = reinterpret_cast<const unsigned short*>(at) + (16 * tau + 4 * g + (i >> 2)) * 16 + 4 * (i & 3);
      const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) short4v*)(const_cast<unsigned short*>(p)));
#pragma unroll
      for (int r = 0; r < 4; ++r) x[tau][r] = u16_to_f32<T>((unsigned short)y[r]);
    }
  }
  if (rows < kChunk) {
#pragma unroll
    for (int tau = 0; tau < 4; ++tau)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * tau + 4 * g + r >= rows) x[tau][r] = 0.f;
  }
}

// 16 columns of a window's state as result tiles, zero for a null pointer and beyond dk.
template <int ST>
__device__ __forceinline__ void load_state(floatx4 (&S)[ST], const Args& a, const float* state, int w, int h, int col,
                                           bool live, int g) {
#pragma unroll
  for (int t = 0; t < ST; ++t) S[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (state == nullptr || !live) return;
  const float* p = state + (((size_t)w * a.H + h) * a.dk) * a.dv + col;
#pragma unroll
  for (int t = 0; t < ST; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = 32 * (t >> 1) + 8 * g + 4 * (t & 1) + r;
      S[t][r] = p[(size_t)(d < a.dk ? d : 0) * a.dv];
    }
#pragma unroll
  for (int t = 0; t < ST; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (32 * (t >> 1) + 8 * g + 4 * (t & 1) + r >= a.dk) S[t][r] = 0.f;
}
template <int ST>
__device__ __forceinline__ void store_state(const floatx4 (&S)[ST], const Args& a, float* state, int w, int h, int col,
                                            bool live, int g) {
  if (state == nullptr || !live) return;
  float* p = state + (((size_t)w * a.H + h) * a.dk) * a.dv + col;
#pragma unroll
  for (int t = 0; t < ST; ++t) {
    const int d = 32 * (t >> 1) + 8 * g + 4 * (t & 1);   // dk is a multiple of 16
    if (d < a.dk)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[(size_t)(d + r) * a.dv] = S[t][r];
  }
}

// x[tau] = triangle times y but for the tile row's factor, lower (UPPER: the transposed triangle under its
// mirrored numbers)
template <bool UPPER>
__device__ __forceinline__ void tri_times(const _Float16* hi, const _Float16* lo, const Far (&y)[2], floatx4 (&x)[4],
                                          int lane) {
  FarSum sum[4];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int tau = 0; tau < 4; ++tau) {
      if (UPPER ? s < tau / 2 : s > tau / 2) continue;
      const int at = (UPPER ? tri_at(3 - tau, 1 - s) : tri_at(tau, s)) * kFrag + lane * 8;
      const Far t = {*reinterpret_cast<const half8_t*>(hi + at), *reinterpret_cast<const half8_t*>(lo + at)};
      mma2(t, y[s], sum[tau]);
    }
#pragma unroll
  for (int tau = 0; tau < 4; ++tau) x[tau] = sum[tau].all();
}
// x[tau] = rows of the image times the state's columns
template <int NT, int DK>
__device__ __forceinline__ void rows_times(const _Float16* img, const Pair (&S)[DK / 32], floatx4 (&x)[4], int i, int g) {
#pragma unroll
  for (int tau = 0; tau < 4; ++tau) x[tau] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kb = 0; kb < DK / 32; ++kb)
#pragma unroll
    for (int tau = 0; tau < 4; ++tau) {
      const half8_t r = image_rows<DK>(img, tau, kb, i, g);
      if constexpr (NT == 2) x[tau] = mma(image_rows<DK>(img + kChunk * DK, tau, kb, i, g), S[kb].hi, x[tau]);
      x[tau] = mma1(r, S[kb], x[tau]);
    }
}

// kOut: o and the final states; kKeep: for the backward, what WalkOut names; kEnds: the parts' Z (value
// columns) and M (dk more columns).
enum WalkKind { kOut, kKeep, kEnds };
template <typename T, int DK, int KIND, int NW>
using WalkStage = std::conditional_t<KIND == kEnds, Stage<T, DK, NW, kTerms<T> * kChunk * DK, kTHi, kRecord>,
                                     Stage<T, DK, NW, 0, 0, kRecord>>;

template <typename T, int DK, int KIND, int NW, bool AHEAD>
__global__ __launch_bounds__(64 * NW) void k_delta_walk(Args a, const T* __restrict__ v,
                                                        const float* __restrict__ state_in,
                                                        const _Float16* __restrict__ images,
                                                        const _Float16* __restrict__ records, int record,
                                                        float* ends, _Float16* __restrict__ maps,
                                                        T* __restrict__ o, const T* __restrict__ dout, WalkOut out) {
  constexpr int NT = kTerms<T>, KB = DK / 32, IMG = kChunk * DK, ST = DK / 16;
  constexpr bool KEEP = KIND == kKeep, ENDS = KIND == kEnds;
  using SG = WalkStage<T, DK, KIND, NW>;
  constexpr bool TWICE = AHEAD && kTwice<SG>;
  using F = Fetch<SG, T, ENDS ? kTHi : 0>;
  __shared__ SG s_a;
  __shared__ std::conditional_t<TWICE, SG, char> s_b;

  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place here = place_of(a, lane);
  const Part part = here.part;
  if (part.none || (ENDS && part.hi >= part.chunks)) return;
  const int w = part.w, h = here.h, group = a.H / a.Hk, hk = h / group;
  const int cg = blockIdx.z * NW + wave, groups = a.dv / 16;
  const bool map = ENDS && cg >= groups;   // columns of M
  if (ENDS && part.lo == 0 && (int)blockIdx.z * NW >= groups) return;   // a window's first part needs no M
  const bool live = ENDS ? cg < (part.lo == 0 ? groups : groups + ST) : cg < groups;
  const int col = 16 * cg + i;
  const Win win = window(a, w);
  const uint32_t slot0 = first_slot(win.begin, w);
  const int last_chunk = part.hi;   // this part's chunks end before it
  const auto rows_of = [&](int c) __attribute__((always_inline)) { return min(kChunk, win.rows - c * kChunk); };

  // o of the chunk before: stored when the next one starts, so that no barrier waits for it
  Raw<T, 4> held[4];
  int held_place[4], held_rows = 0;
  const auto put = [&]() __attribute__((always_inline)) {
    if constexpr (KIND == kOut)
#pragma unroll
      for (int tau = 0; tau < 4; ++tau)
        if (16 * tau + i < held_rows)
          *reinterpret_cast<Raw<T, 4>*>(o + ((size_t)held_place[tau] * a.H + h) * a.dv + 16 * cg + 4 * g) = held[tau];
  };

  // the state is `unit` times S, a unit a column: after a chunk S stays in the units of the products it was
  // summed with
  floatx4 S[ST];
  float unit = 1.f;
  bool carried = true;   // no products with a state that is zero
  // A parted window's first state is read once, by the walk of the ends, which keeps it where the last part's
  // end would be: state_out, which the last part's workgroup writes, may be state_in.
  const bool kept = part.lo == 0 && part.hi < part.chunks && state_in != nullptr;
  const uint32_t from_slot = kept ? part.slot + (uint32_t)((part.chunks - 1) / a.part) : part.slot - 1;
  if (map) {
#pragma unroll
    for (int t = 0; t < ST; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        S[t][r] = 32 * (t >> 1) + 8 * g + 4 * (t & 1) + r == 16 * (cg - groups) + i ? 1.f : 0.f;
  } else if (ENDS || (part.lo == 0 && !kept)) {
    const float* from = part.lo == 0 ? state_in : nullptr;
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
  F fetch;
  const auto start = [&](SG& s, int c, const Places<T>& at) __attribute__((always_inline)) {
    fetch.start(s, a, slot0 + c, hk, h, cg, live && !map, images, records, record, v, at, wave, lane, rows_of(c));
  };
  Places<T> at;
  if (part.lo < last_chunk) {
    at.ask(a, win.begin + part.lo * kChunk, rows_of(part.lo), lane);
    if constexpr (TWICE) {
      start(s_a, part.lo, at);
      fetch.template jobs<0, F::kJobs>(s_a, wave);
    }
  }

  // chunk c, staged in `s`; the next one's moves go into `other` in between
  const auto work = [&](const SG& s, auto& other, int c) __attribute__((always_inline)) {
    const int rows = rows_of(c);
    const size_t sh = (size_t)(slot0 + c) * a.H + h;
    const _Float16 *qi = s.img, *ki = s.img + (NT * IMG - SG::kImgAt);
    const auto rec = [&](int from) __attribute__((always_inline)) { return s.rec + (from - SG::kRecAt); };
    const float* scal = reinterpret_cast<const float*>(rec(kScalAt));
    auto row4 = [&](int what, int tau) { return *reinterpret_cast<const floatx4*>(scal + what + 16 * tau + 4 * g); };
    const bool next = TWICE && c + 1 < last_chunk;
    const auto jobs = [&](auto from, auto to) __attribute__((always_inline)) {
      if constexpr (TWICE)
        if (next) fetch.template jobs<decltype(from)::value * F::kJobs / 8, decltype(to)::value * F::kJobs / 8>(other, wave);
    };
    using std::integral_constant;
    floatx4 Y[4], qs[4];
    // (before any move: the compiler makes transposed reads wait for those)
    if (map) {
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) Y[tau] = floatx4{0.f, 0.f, 0.f, 0.f};
    } else {
      rows_in(s.rows[wave], Y, rows, i, g);
    }
    put();
    if constexpr (TWICE)
      if (next) {
        Places<T> to;
        to.take(a, scal + kNext, lane);
        start(other, c + 1, to);
      }
    jobs(integral_constant<int, 0>{}, integral_constant<int, 2>{});
    int place[4];   // this lane's row of every tile
#pragma unroll
    for (int tau = 0; tau < 4; ++tau) place[tau] = kept_row(a, scal[kRow + 16 * tau + i]);
    Raw<T, 4> dn[KEEP ? 4 : 1];
    if constexpr (KEEP) {
      float* to = out.states + ((sh * (a.dv / 16) + cg) * ST) * 256 + lane * 4;
#pragma unroll
      for (int t = 0; t < ST; ++t) *reinterpret_cast<floatx4*>(to + t * 256) = S[t] * unit;
      if (!carried && lane == 0) out.smax[sh * (a.dv / 16) + cg] = 0.f;
#pragma unroll
      for (int tau = 0; tau < 4; ++tau)   // row 0 where there is none
        dn[tau] = *reinterpret_cast<const Raw<T, 4>*>(dout + ((size_t)place[tau] * a.H + h) * a.dv + 16 * cg + 4 * g);
    }
    // y = s v - t exp(gam) k' S, and q' S for later
    uint32_t top = 0;   // of the state's column, in S's units
    float qdown = 0.f;
#pragma unroll
    for (int tau = 0; tau < 4; ++tau) {
      Y[tau] *= row4(kVScale, tau);
      qs[tau] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (carried) {
      top = column_max_bits(max_of(S));
      const Scale sc = scale_of(top);
      if constexpr (KEEP) {
        const uint32_t all = wave_max_bits(__uint_as_float(top) * unit);
        if (lane == 0) out.smax[sh * (a.dv / 16) + cg] = __uint_as_float(all);
      }
      Pair Sp[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) Sp[kb] = split(S[2 * kb], S[2 * kb + 1], sc.up);
      qdown = sc.down * unit;
      floatx4 x[4];
      rows_times<NT, DK>(ki, Sp, x, i, g);
      if constexpr (!ENDS)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int tau = 0; tau < 4; ++tau) {
            const half8_t qr = image_rows<DK>(qi, tau, kb, i, g);
            if constexpr (NT == 2) qs[tau] = mma(Sp[kb].hi, image_rows<DK>(qi + IMG, tau, kb, i, g), qs[tau]);
            qs[tau] = mma1(Sp[kb], qr, qs[tau]);
          }
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) Y[tau] -= (row4(kSinceK, tau) * qdown) * x[tau];
    }
    jobs(integral_constant<int, 2>{}, integral_constant<int, 5>{});
    // r = T y, u = (b / t) r; both times uunit
    floatx4 U[4];
    float uunit;
    {
      const Scale sy = column_scale(Y);
      uunit = sy.down;
      Far Yp[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) Yp[s2] = split<Far>(Y[2 * s2], Y[2 * s2 + 1], sy.up);
      tri_times<false>(rec(kTHi), rec(kTHi + kTerm), Yp, U, lane);
      const floatx4 tdown = *reinterpret_cast<const floatx4*>(scal + kTDown);
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) {
        U[tau] *= tdown[tau];
        if constexpr (KEEP) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            out.resid[(sh * kChunk + 16 * tau + 4 * g + r) * a.dv + col] = U[tau][r] * uunit;
        }
        U[tau] = 16 * tau < rows ? U[tau] * row4(kWrite, tau) : floatx4{0.f, 0.f, 0.f, 0.f};   // (what was not moved)
      }
    }
    jobs(integral_constant<int, 5>{}, integral_constant<int, 8>{});
    // o, transposed: a lane holds 4 columns of one row
    if constexpr (!ENDS) {
      const Scale su = column_scale(U);
      const floatx4 udown = across(su.down * uunit, g), sdown = across(qdown, g);
      const floatx4 pdown = *reinterpret_cast<const floatx4*>(scal + kPDown);
      FarSum y[4];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const Far up = split<Far>(U[2 * s2], U[2 * s2 + 1], su.up);
#pragma unroll
        for (int tau = 2 * s2; tau < 4; ++tau) {
          const int p = tri_at(tau, s2) * kFrag + lane * 8;
          const Far t = {*reinterpret_cast<const half8_t*>(rec(kPHi) + p),
                         *reinterpret_cast<const half8_t*>(rec(kPLo) + p)};
          mma2(up, t, y[tau]);
        }
      }
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) {
        const int p = 16 * tau + i;
        const float os = scal[kOScale + p], since = os * scal[kSince + p];
        const floatx4 z = since * (sdown * qs[tau]) + (os * pdown[tau]) * (udown * y[tau].all());
        if constexpr (!KEEP) {
          const float z4[4] = {z[0], z[1], z[2], z[3]};
          held[tau] = Frag<T, 4>::from_f32(z4);
          held_place[tau] = place[tau];
        } else {
          float d4[4], dot = 0.f;
          Frag<T, 4>::to_f32(dn[tau], d4);
#pragma unroll
          for (int r = 0; r < 4; ++r) dot += z[r] * d4[r];
          dot = p < rows ? dot : 0.f;
          dot += __shfl_xor(dot, 16);
          dot += __shfl_xor(dot, 32);
          if (g == 0) out.odo[(sh * (a.dv / 16) + cg) * kChunk + p] = dot;
        }
      }
    }
    // S = exp(gam_last) S + k'^T (until u), summed in the units of the products.  Where u is so small
    // beside the state that the state would overflow there, its units follow the state's size.
    {
#pragma unroll
      for (int tau = 0; tau < 4; ++tau) U[tau] *= row4(kUntil, tau);
      uint32_t ubits = column_max_bits(max_of(U));
      const uint32_t least = __float_as_uint(__uint_as_float(top) * unit / uunit * 0x1p-60f);
      ubits = max(ubits, min(least, 0x7f000000u));
      Scale su = scale_of(ubits);
      if (su.down * uunit < 0x1p-120f) {   // values below some 2^-100 lose their low bits, and no unit is zero
        su.down = 0x1p-120f / uunit;
        su.up = 1.f / su.down;
      }
      Pair Up[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) Up[s2] = split(U[2 * s2], U[2 * s2 + 1], su.up);
      const float newunit = su.down * uunit, keep = scal[kLast] * (unit / newunit);
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        floatx4 x = S[t] * keep;
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          if constexpr (NT == 2) x = mma(image_cols<DK>(ki + IMG, t >> 1, t & 1, s2, i, g), Up[s2].hi, x);
          x = mma1(image_cols<DK>(ki, t >> 1, t & 1, s2, i, g), Up[s2], x);
        }
        S[t] = x;
      }
      unit = newunit;
      carried = true;
    }
    held_rows = rows;
  };

  if (!live) {   // beyond the columns: a share of the moves
    for (int c = part.lo; c < last_chunk; ++c) {
      barrier();
      if constexpr (TWICE) {
        if (c + 1 >= last_chunk) break;
        start(s_b, c + 1, at);
        fetch.template jobs<0, F::kJobs>(s_b, wave);
        barrier();
        if (++c + 1 >= last_chunk) break;
        start(s_a, c + 1, at);
        fetch.template jobs<0, F::kJobs>(s_a, wave);
      } else {
        start(s_a, c, at);
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
    for (int c = part.lo; c < last_chunk; c += 2) {
      turn(s_a, s_b, c);
      if (c + 1 < last_chunk) turn(s_b, s_a, c + 1);
    }
  } else {
    for (int c = part.lo; c < last_chunk; ++c) {
      if (c > part.lo) at.take(a, reinterpret_cast<const float*>(s_a.rec + (kScalAt - SG::kRecAt)) + kNext, lane);
      barrier();
      start(s_a, c, at);
      fetch.template jobs<0, F::kJobs>(s_a, wave);
      barrier();
      work(s_a, s_a, c);
    }
  }
  put();
  if constexpr (ENDS)
    if (map) {   // a lane has a column of M: a row of the image of M^T, 8 neighbouring columns from two tiles
      _Float16* to = maps + ((size_t)part.slot * a.H + h) * map_halfs(DK);
      const int m = 16 * (cg - groups) + i;
      const Scale sc = column_scale(S);
      if (g == 0) reinterpret_cast<float*>(to + 2 * DK * DK)[m] = sc.down * unit;
#pragma unroll
      for (int t = 0; t < KB; ++t) {
        const Pair p = split(S[2 * t], S[2 * t + 1], sc.up);
        const int at2 = image_at<DK>(m, t, g);
        *reinterpret_cast<half8_t*>(to + at2) = p.hi;
        *reinterpret_cast<half8_t*>(to + DK * DK + at2) = p.lo;
      }
      return;
    }
#pragma unroll
  for (int t = 0; t < ST; ++t) S[t] *= unit;
  if constexpr (ENDS) {
    float* to = ends + (((size_t)part.slot * a.H + h) * groups + cg) * ST * 256 + lane * 4;
#pragma unroll
    for (int t = 0; t < ST; ++t) *reinterpret_cast<floatx4*>(to + t * 256) = S[t];
  } else if (part.hi == part.chunks) {
    store_state(S, a, out.state_out, w, h, col, live, g);
  }
}

// ------------------------------------------------------------------ the parts' states joined
// A wave for 16 columns of a window's states: after the first part's end, which is there, S = M S + Z part
// after part, each written over its Z.  BACK: from the last part's start to the second one's, with M^T.
// A chain of products with 64 KB of M a step (at 128 x 128), moved ahead into LDS: 34 us for 7 windows
// with 12,289 rows in all, 20 us for the 16 parts of a window at 64 x 64, 1.3 us a step.
template <int DK, bool BACK>
__global__ __launch_bounds__(256) void k_delta_join(Args a, float* ends, const _Float16* __restrict__ maps) {
  constexpr int ST = DK / 16, KB = DK / 32, kMap = 2 * DK * DK;   // halfs in LDS
  __shared__ __attribute__((aligned(16))) _Float16 s_a[kMap];
  __shared__ __attribute__((aligned(16))) _Float16 s_b[kMap];
  const int w = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), groups = a.dv / 16;
  const int cg = blockIdx.z * 4 + wave;
  const bool live = cg < groups;
  const Win win = window(a, w);
  const uint32_t f = first_slot(win.begin, w, (uint32_t)a.part * kChunk);
  const int parts = (chunks_of(win) + a.part - 1) / a.part;
  if (parts < 3) return;   // one end at most, and no map
  const auto part = [&](int n) { return f + (BACK ? parts - 1 - n : n); };   // n-th in the order of the walk
  const auto end = [&](int n) { return ends + (((size_t)part(n) * a.H + h) * groups + (live ? cg : 0)) * ST * 256 + lane * 4; };
  const auto fetch = [&](_Float16* to, int n) __attribute__((always_inline)) {
    const char* from = reinterpret_cast<const char*>(maps + ((size_t)part(n) * a.H + h) * map_halfs(DK)) + lane * 16;
#pragma unroll
    for (int j = 0; j < kMap * 2 / 4096; ++j) to_lds(to + (wave + 4 * j) * 512, from + (wave + 4 * j) * 1024);
  };
  floatx4 S[ST];
#pragma unroll
  for (int t = 0; t < ST; ++t) S[t] = *reinterpret_cast<const floatx4*>(end(0) + t * 256);
  const auto step = [&](const _Float16* m, _Float16* other, int n) __attribute__((always_inline)) {
    floatx4 Z[ST], F[ST];   // F: the factors of M's columns, in the order of the state's rows
    const float* factors = reinterpret_cast<const float*>(maps + ((size_t)part(n) * a.H + h) * map_halfs(DK) + kMap);
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      Z[t] = *reinterpret_cast<const floatx4*>(end(n) + t * 256);
      F[t] = *reinterpret_cast<const floatx4*>(factors + 32 * (t >> 1) + 8 * g + 4 * (t & 1));
    }
    barrier();
    if (n + 1 < parts - 1) fetch(other, n + 1);
    if constexpr (!BACK)
#pragma unroll
      for (int t = 0; t < ST; ++t) S[t] *= F[t];
    const Scale sc = column_scale(S);
    Pair Sp[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) Sp[kb] = split(S[2 * kb], S[2 * kb + 1], sc.up);
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Pair p;
#pragma unroll
        for (int term = 0; term < 2; ++term) {
          const _Float16* at = m + term * DK * DK;
          half8_t y;
          if constexpr (BACK) {   // rows of M^T in the order of the state's rows, contraction over columns
            y = *reinterpret_cast<const half8_t*>(at + image_at<DK>(32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3), kb, g));
          } else {                // columns as rows, contraction over rows 32 kb + 8 g + e
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              const _Float16* q = at + image_at<DK>(32 * kb + 8 * g + 4 * hh + (i >> 2), t >> 1, i & 3) + 4 * (t & 1);
              const short4v z = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) short4v*)(const_cast<_Float16*>(q)));
#pragma unroll
              for (int r = 0; r < 4; ++r) y[4 * hh + r] = __builtin_bit_cast(_Float16, (short)z[r]);
            }
          }
          if (term == 0) p.hi = y;
          else p.lo = y;
        }
        x = mma2(p, Sp[kb], x);
      }
      if constexpr (BACK) Z[t] += (sc.down * x) * F[t];
      else Z[t] += sc.down * x;
    }
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      S[t] = Z[t];
      if (live) *reinterpret_cast<floatx4*>(end(n) + t * 256) = S[t];
    }
  };
  fetch(s_a, 1);
  for (int n = 1; n < parts - 1; n += 2) {
    step(s_a, s_b, n);
    if (n + 1 < parts - 1) step(s_b, s_a, n + 1);
  }
}

// Waves of a walk's workgroup.  Eight share a chunk's staging among 128 columns, four leave a SIMD to a
// wave: eight where workgroups of four would be more than the 256 CUs.  Windows of 1,024 bf16 rows, heads
// of 128, four and eight: 64 window heads 81 and 98 us, 128: 105 and 119, 160: 166 and 132, 384: 312 and
// 274 (gradients 378 and 432, 585 and 646, 844 and 742, 1,702 and 1,622).  fp32 rows have room for four.
template <typename T>
inline int walk_waves(const Args& a) {
  const int groups = a.dv / 16;
  if (groups <= 2) return 2;
  if (groups <= 4 || sizeof(T) == 4) return 4;
  return (int64_t)part_slots(a) * a.H * ((groups + 7) / 8) > 128 ? 8 : 4;
}
// Whether the walks stage a chunk ahead.  Not where two workgroups a CU and more are there to wait for
// each other and the second buffer would keep some of them off it, which is at 32 state rows: fp16 windows of
// 256 rows, 4 heads of 32, with and without, forward and gradients: 384 workgroups 51 + 150 and 54 + 153 us,
// 512: 69 + 199 and 59 + 175, 768: 80 + 269 and 74 + 249, 1,536: 157 + 525 and 153 + 508 (fp32, 768: 117 + 382
// and 91 + 329); but 24,000 bf16 rows, 8 heads of 128: windows of 40 238 + 1,190 and 240 + 1,194, 256: 163 + 859
// and 188 + 878.
inline bool walks_ahead(dim3 grid) { return (int64_t)grid.x * grid.y * grid.z < 512; }
// f(integral_constant<waves>, bool_constant<ahead>, grid)
template <typename T, int DK, class F>
inline void with_walk(const Args& a, F f) {
  const int waves = walk_waves<T>(a);
  const dim3 grid((uint32_t)part_slots(a), a.H, (a.dv / 16 + waves - 1) / waves);
  const auto by_waves = [&](auto ahead) {
    if (waves == 2) f(std::integral_constant<int, 2>{}, ahead, grid);
    else if (waves == 4) f(std::integral_constant<int, 4>{}, ahead, grid);
    else if constexpr (sizeof(T) == 2) f(std::integral_constant<int, 8>{}, ahead, grid);
  };
  if constexpr (DK == 32)
    if (!walks_ahead(grid)) return by_waves(std::false_type{});
  by_waves(std::true_type{});
}
// The states at the parts' starts, where windows are parted.
template <typename T, int DK>
inline void launch_ends(const Args& a, const T* v, const float* state_in, const _Float16* images,
                        const _Float16* records, int record, float* ends, _Float16* maps, hipStream_t stream) {
  if (a.part == 0) return;
  const int groups = a.dv / 16 + DK / 16;
  k_delta_walk<T, DK, kEnds, 4, true><<<dim3((uint32_t)part_slots(a), a.H, (groups + 3) / 4), 256, 0, stream>>>(
      a, v, state_in, images, records, record, ends, maps, nullptr, nullptr, WalkOut{});
  k_delta_join<DK, false><<<dim3(a.W, a.H, (a.dv / 16 + 3) / 4), 256, 0, stream>>>(a, ends, maps);
}

}  // namespace delta
}  // namespace sla
