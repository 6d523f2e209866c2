// Typed 16-byte pieces of a row, shared by the row kernels (layer norm, rms norm,
// dropout, rotary positions). Elements are bf16, fp16 or fp32; a piece holds V of them. Rows
// need no alignment beyond their element's: gfx950 takes wide vector accesses
// at any address, at full rate where they are 16-byte aligned.
#pragma once

#include "vitattn_common.h"
#include "vitattn_launch.h"

namespace vitattn {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
struct Piece {
  static constexpr int V = 16 / (int)sizeof(T);
  u32x4 raw;

  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[e]);
    const uint16_t bits = (uint16_t)(raw[e >> 1] >> (16 * (e & 1)));
    if constexpr (std::is_same<T, __bf16>::value) return __uint_as_float((uint32_t)bits << 16);
    return (float)__builtin_bit_cast(_Float16, bits);
  }
  // rounds to nearest even in the 16-bit types
  __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 4) {
        raw[w] = __float_as_uint(x[w]);
      } else {
        typedef T pair __attribute__((ext_vector_type(2)));
        const pair p = {(T)x[2 * w], (T)x[2 * w + 1]};
        raw[w] = __builtin_bit_cast(uint32_t, p);
      }
    }
  }
  // the first n elements at p (0 <= n <= V; the rest are zeros)
  __device__ __forceinline__ void load(const T* p, int n) {
    if (n >= V) {
      raw = *reinterpret_cast<const u32x4_any*>(p);
      return;
    }
    raw = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) {
        if constexpr (sizeof(T) == 4)
          raw[e] = reinterpret_cast<const uint32_t*>(p)[e];
        else
          raw[e >> 1] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
      }
  }
  __device__ __forceinline__ void store(T* p, int n) const {
    if (n >= V) {
      *reinterpret_cast<u32x4_any*>(p) = raw;
      return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) {
        if constexpr (sizeof(T) == 4)
          reinterpret_cast<uint32_t*>(p)[e] = raw[e];
        else
          reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(raw[e >> 1] >> (16 * (e & 1)));
      }
  }
};

// V elements of type R, in as many 16-byte pieces as they take. Every lane loads whole
// pieces, at the row's end the 16 bytes that end with it (lanes past the row too), and
// they are put in place when all loads are on their way: read element by element, a
// last piece waits for memory before the next load.
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
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < K; ++k) p[k].raw = u32x4{0, 0, 0, 0};
  }
  // columns c .. c + V - 1 of a row of D, those past it left open until settled
  __device__ __forceinline__ void load(const R* row, int c, int D) {
    if (D >= P) {
#pragma unroll
      for (int k = 0; k < K; ++k) p[k].raw = *reinterpret_cast<const u32x4_any*>(row + min(c + k * P, D - P));
      return;
    }
    clear();
    if (c == 0)  // (a row of less than one piece)
      for (int e = D - 1; e >= 0; --e) {
        u32x4& w = p[0].raw;
        if constexpr (sizeof(R) == 4) {
          w = u32x4{reinterpret_cast<const uint32_t*>(row)[e], w[0], w[1], w[2]};
        } else {
          const uint32_t x = reinterpret_cast<const uint16_t*>(row)[e];
          w = u32x4{w[0] << 16 | x, w[1] << 16 | w[0] >> 16, w[2] << 16 | w[1] >> 16, w[3] << 16 | w[2] >> 16};
        }
      }
  }
  // puts a row's last piece in place, and zeros past it (all of it unless `on`)
  __device__ __forceinline__ void settle(int c, int D, bool on) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int m = on ? D - c - k * P : 0;
      if (!__any(m < P)) continue;
      if (m <= 0) {
        p[k].raw = u32x4{0, 0, 0, 0};
      } else if (m < P && D >= P) {
        const int by = (P - m) * 8 * (int)sizeof(R);  // bits, below 128
        uint64_t lo = (uint64_t)p[k].raw[1] << 32 | p[k].raw[0], hi = (uint64_t)p[k].raw[3] << 32 | p[k].raw[2];
        if (by >= 64) {
          lo = hi >> (by - 64);
          hi = 0;
        } else {
          lo = lo >> by | hi << (64 - by);
          hi >>= by;
        }
        p[k].raw = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
      }
    }
  }
  __device__ __forceinline__ void store(R* x, int n) const {
#pragma unroll
    for (int k = 0; k < K; ++k) p[k].store(x + k * P, min(max(n - k * P, 0), P));
  }
};

constexpr int kRowThreads = 256;  // of a workgroup of the norms

// V weights from element c on (n of them real, zeros behind), fp32 or T
template <typename T>
__device__ __forceinline__ void load_weights(const void* p, bool f32, long long c, int n, float (&w)[Piece<T>::V]) {
  constexpr int V = Piece<T>::V;
  if (f32) {
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = e < n ? static_cast<const float*>(p)[c + e] : 0.f;
  } else {
    Piece<T> x;
    x.load(static_cast<const T*>(p) + c, n);
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = x.get(e);
  }
}

// Where a thread stands: its row of the workgroup's `per` at a time (outside
// them: a wave's lanes behind its last whole row) and its lane of the row.
template <bool BLOCK>
struct Place {
  int L, lane, row, per;
  __device__ __forceinline__ explicit Place(int lanes) : L(lanes) {
    if constexpr (BLOCK) {
      lane = threadIdx.x;
      row = 0;
      per = 1;
    } else {
      const int wl = threadIdx.x & 63, rpw = 64 / L, g = wl / L;
      lane = wl - g * L;
      per = rpw * (kRowThreads / 64);
      row = g < rpw ? (int)(threadIdx.x >> 6) * rpw + g : -1;
    }
  }
  // Sum over the row's lanes (BLOCK: over the workgroup), the same in all.
  __device__ __forceinline__ float sum(float x, float* lds) const {
    if (BLOCK || (L & (L - 1)) == 0) {
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1)
        if (BLOCK || m < L) x += __shfl_xor(x, m, 64);
    } else {
      const int at = threadIdx.x & 63;
      for (int m = 32; m >= 1; m >>= 1) {
        if (m >= L) continue;
        const float y = __shfl(x, (at + m) & 63, 64);
        x += lane + m < L ? y : 0.f;
      }
      x = __shfl(x, at - lane, 64);
    }
    if constexpr (BLOCK) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
      __syncthreads();
      x = lds[0] + lds[1] + lds[2] + lds[3];
    }
    return x;
  }
  // whether it holds anywhere in the wave (BLOCK: all of which agree)
  __device__ __forceinline__ static bool any(bool x) { return BLOCK ? x : __any(x); }
};

// Lanes that share a row of a norm and pieces per lane (lanes = 0: too long for
// registers). The figures are layer norm's.
// With a piece per lane a wave sums over up to 64 lanes for 16 bytes of each; more
// pieces need fewer lanes, hence fewer steps, and are as many loads. The forward
// takes two from 4 pieces on (D = 64, 46 MB 17.6 -> 15.8 us, 400 MB 165 -> 171; 72
// 22.4 -> 19.8 and 178 -> 185; 128 19.8 -> 17.3 and 164 -> 157) and from 16 pieces on
// two or three, whichever keeps more lanes at work (D = 192 25.3 -> 17.3 and 195 ->
// 157, 768 21.3 -> 17.4 and 161 -> 152). The backward keeps dw's and db's share of
// each piece as well: one below 16 pieces (two: D = 64 35 -> 43 us), then two, or
// three where two leave a fifth of the lanes idle (D = 192 42 -> 37 and 313 -> 235,
// 384 42 -> 37 and 320 -> 230, 768, against two, 40 -> 35 and 269 -> 228). Four are
// for rows of more. These are rules on D alone: a row's bits do not depend on the
// call it is part of.
struct RowShape {
  int lanes, np;
};
inline RowShape row_shape(int D, int V, bool fwd) {
  const int pieces = (D + V - 1) / V;
  if (pieces > 256) {
    const int np = (pieces + kRowThreads - 1) / kRowThreads;
    return np > 8 ? RowShape{0, 0} : RowShape{kRowThreads, np == 7 ? 8 : np};
  }
  if (pieces < (fwd ? 4 : 16)) return {pieces, 1};
  if (pieces < 16) return {(pieces + 1) / 2, 2};
  RowShape best = {(pieces + 3) / 4, 4};
  int most = 0;
  for (int np = 2; np <= 3; ++np) {
    const int L = (pieces + np - 1) / np;
    const int used = L > 64 ? 0 : pieces * (64 / L) * 60 / np;  // of 64 * 60
    if (used <= most) continue;
    most = used;
    best = {L, np};
    if (!fwd && used >= 64 * 48) break;
  }
  return best;
}

}  // namespace vitattn
