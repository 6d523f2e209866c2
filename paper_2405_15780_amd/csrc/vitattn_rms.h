// Device helpers of the rms norm's forward and backward.
#pragma once

#include "vitattn_random.h"

namespace vitattn {

// As for layer norm, but rows of more than two pieces per lane take the workgroup, a
// piece per lane, in the backward and beside a wider residual: four pieces of every
// operand leave one or two waves to a SIMD (8,193 rows of 1,537, fp16 beside fp32, forward
// 40.6 -> 35.0 us, backward 74.8 -> 47.5; 32,768 of 2,048 bf16 to e4m3 100 -> 110: these
// stay with a wave each).
inline RowShape rms_shape(int D, int V, bool fwd, bool wider) {
  const RowShape s = row_shape(D, V, fwd);
  return s.lanes <= 64 && s.np > 2 && (!fwd || wider) ? RowShape{kRowThreads, 1} : s;
}

// the three indexes of row r
struct RowAt {
  int i0, i1, i2;
  __device__ __forceinline__ RowAt(const RmsArgs& a, int r) {
    const int t = a.n2 == a.rows ? 0 : r / a.n2;
    i2 = r - t * a.n2;
    i0 = t / a.n1;
    i1 = t - i0 * a.n1;
  }
  __device__ __forceinline__ long long in(const RowMap& m) const { return m.at(i0, i1, i2); }
};

// The numbers of a piece of V columns from c on (a piece of four has a half of
// their eight words).
template <int V>
struct PieceMask {
  u32x4 w;
  int first;
  __device__ __forceinline__ PieceMask(const Dropout& d, int c, uint32_t row) : w(d.words((uint32_t)c >> 3, row)), first(c & 7) {}
  template <typename O>
  __device__ __forceinline__ float add(const Dropout& d, int e, float x, float r) const {
    if constexpr (V == 8) return d.add<O>(w, e, x, r);
    const u32x4 half = first ? u32x4{w[2], w[3], 0, 0} : u32x4{w[0], w[1], 0, 0};
    return d.add<O>(half, e, x, r);
  }
};

// The wave's lanes share rows of L lanes each, NP pieces of V columns per lane, or
// (BLOCK) the workgroup a row. Lanes past D: n <= 0.
template <int V>
__device__ __forceinline__ int columns_of(int D, int c) { return min(max(D - c, 0), V); }

}  // namespace vitattn
