// Device helpers of the rms norm's forward and backward.
#pragma once

#include "vitattn_random.h"

namespace vitattn {

// V elements of type R, in as many 16-byte pieces as they take (V of a wider type
// than R's own piece: two)
template <typename R, int V>
struct Span {
  static constexpr int P = Piece<R>::V, K = V / P;
  static_assert(V % P == 0, "whole pieces");
  Piece<R> p[K];
  __device__ __forceinline__ float get(int e) const { return p[e / P].get(e % P); }
  __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float part[P];
#pragma unroll
      for (int e = 0; e < P; ++e) part[e] = x[k * P + e];
      p[k].set(part);
    }
  }
  __device__ __forceinline__ void load(const R* x, int n) {
#pragma unroll
    for (int k = 0; k < K; ++k) p[k].load(x + k * P, min(max(n - k * P, 0), P));
  }
  __device__ __forceinline__ void store(R* x, int n) const {
#pragma unroll
    for (int k = 0; k < K; ++k) p[k].store(x + k * P, min(max(n - k * P, 0), P));
  }
};

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
  __device__ __forceinline__ float add(const Dropout& d, int e, float x, float r) const {
    if constexpr (V == 8) return d.add(w, e, x, r);
    const u32x4 half = first ? u32x4{w[2], w[3], 0, 0} : u32x4{w[0], w[1], 0, 0};
    return d.add(half, e, x, r);
  }
};

// The wave's lanes share rows of L lanes each, NP pieces of V columns per lane, or
// (BLOCK) the workgroup a row. Lanes past D: n <= 0.
template <int V>
__device__ __forceinline__ int columns_of(int D, int c) { return min(max(D - c, 0), V); }

}  // namespace vitattn
