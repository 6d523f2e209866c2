// Typed 16-byte pieces of a row, shared by the row kernels (layer norm, rotary
// positions). Elements are bf16, fp16 or fp32; a piece holds V of them. Rows
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

}  // namespace vitattn
