// Windows of consecutive positions and pools of states, as the operators that go through rows in
// order (the short convolution, the selective scan) meet them.
#pragma once
#include "sla_common.h"

namespace sla {

// The windows of a call.  Offsets and orders come from device memory, so they are clamped where they
// are read: whatever they hold, no access leaves the tensors.
struct Windows {
  const int32_t* offsets;   // [W + 1]
  const int32_t* order;     // [n], or null: position p is row p
  int32_t n, W;

  __device__ __forceinline__ int edge(int w) const {
    const int p = offsets[w];
    return p < 0 ? 0 : p > n ? n : p;
  }
  // the row at position p; -1 where the order names none
  __device__ __forceinline__ int row(int p) const {
    if (order == nullptr) return p;
    const int r = order[p];
    return (uint32_t)r < (uint32_t)n ? r : -1;
  }
  // the window that position p lies in: the last one that begins at p or before (-1: none does; the caller
  // looks whether it has ended)
  __device__ __forceinline__ int find(int p) const {
    int lo = -1, hi = W;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (edge(mid) <= p) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// Blocks of `per` positions of all windows: window w has the blocks edge(w) / per + w and following
// ones, so blocks of different windows never share a number, and there are fewer than n / per + W + 1.
struct Part {
  int w, begin, end;     // positions of the block
  int first, last;       // whether it begins and ends its window
};
// By whole waves: 64 windows are looked at at once, so 4,096 take two steps (one by one they were twelve loads in
// a row, a third of the time of a window of 40 rows).
__device__ __forceinline__ bool part_of(const Windows& win, int per, uint32_t slot, Part& part) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = win.W;   // the window is in [lo, hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
    const bool before = at < hi && (uint32_t)(win.edge(at) / per) + (uint32_t)at <= slot;
    const uint64_t seen = __ballot(before);
    const int last = seen ? 63 - __builtin_clzll(seen) : 0;
    lo += last * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int b = win.edge(lo), e = win.edge(lo + 1);
  const uint32_t f = (uint32_t)(b / per) + (uint32_t)lo;
  if (slot < f) return false;
  const int64_t at = (int64_t)b + (int64_t)(slot - f) * per;
  if (at >= e) return false;
  part.w = lo;
  part.begin = (int)at;
  part.end = (int)(at + per < e ? at + per : (int64_t)e);
  part.first = at == b;
  part.last = part.end == e;
  return true;
}

// Rows of a batch with the same slot are successive rows of one sequence: the workgroup of the first one
// takes them all, in row order.  next(): the row after b with b's slot (n: none), or -1 where an
// earlier one has it (asked once, `first`).  For whole workgroups of 64 x WAVES threads.
template <int WAVES>
struct SlotRows {
  const int32_t* slots;
  int32_t n;
  int* table;   // 2 WAVES ints of LDS

  __device__ __forceinline__ int next(int b, int slot, bool first) const {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int next = n, seen = 0;
    for (int x = first ? tid : b + 1 + tid; x < n; x += 64 * WAVES)
      if (slots[x] == slot) {
        if (x < b) seen = 1;
        if (x > b && x < next) next = x;
      }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int y = __shfl_xor(next, m);
      next = y < next ? y : next;
    }
    const uint64_t any = __ballot(seen);
    __syncthreads();   // the table's readers of the row before
    if (lane == 0) {
      table[wave] = next;
      table[WAVES + wave] = any != 0;
    }
    __syncthreads();
    seen = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      next = min(next, table[w]);
      seen |= table[WAVES + w];
    }
    return seen ? -1 : next;
  }
};

// Values of VEC consecutive channels in their storage format; VEC = 1 for odd widths and addresses.
template <typename T, int VEC>
struct Vec {
  using R = Raw<T, VEC>;
  static __device__ __forceinline__ R load(const T* p) { return *reinterpret_cast<const R*>(p); }
  static __device__ __forceinline__ void store(T* p, const float (&x)[VEC]) {
    *reinterpret_cast<R*>(p) = Frag<T, VEC>::from_f32(x);
  }
  static __device__ __forceinline__ R zero() { return Frag<T, VEC>::zero(); }
  static __device__ __forceinline__ void wide(R r, float (&x)[VEC]) { Frag<T, VEC>::to_f32(r, x); }
};
template <typename T>
__device__ __forceinline__ float to_float(T x) {
  if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float((uint32_t)x.bits << 16);
  else return (float)x;
}
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  if constexpr (std::is_same<T, bf16_t>::value) return bf16_t{f32_to_u16<bf16_t>(x)};
  else return (T)x;
}
template <typename T>
struct Vec<T, 1> {
  using R = T;
  static __device__ __forceinline__ R load(const T* p) { return *p; }
  static __device__ __forceinline__ void store(T* p, const float (&x)[1]) { *p = from_float<T>(x[0]); }
  static __device__ __forceinline__ R zero() { return from_float<T>(0.f); }
  static __device__ __forceinline__ void wide(R r, float (&x)[1]) { x[0] = to_float<T>(r); }
};

// p[i] of a base that all lanes share: the lane's part of the address in 32 bits, so that no lane adds 64-bit ones.
template <typename T>
__device__ __forceinline__ T& lane_at(T* p, uint32_t i) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type B;
  return *reinterpret_cast<T*>(reinterpret_cast<B*>(p) + (uint32_t)(i * (uint32_t)sizeof(T)));
}

}  // namespace sla
