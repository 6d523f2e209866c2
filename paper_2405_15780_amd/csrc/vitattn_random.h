// Dropout's random numbers, formed where they are used and never stored: Philox
// 4x32 of ten rounds (Salmon, Moraes, Dror and Shaw, 2011), a bijection of a 128-bit
// counter under a 64-bit key. The key is the seed and the counter (column / 8, row,
// offset): its four words are the sixteen-bit numbers of the eight columns, the low
// half of a word first. An element is kept if its number is at least T =
// round(65536 p), so that p is taken as T / 65536, and the kept ones are multiplied
// with 65536 / (65536 - T): their mean is unchanged. (Sixteen bits and not 32: half
// of the multiplications, which bound it, for a p that is off by 2^-17 at most.)
#pragma once

#include "vitattn_rows.h"

namespace vitattn {

// DropArgs with what a device-side state adds
struct Dropout {
  uint32_t k0, k1, o0, o1, threshold;
  float up;
  __device__ __forceinline__ explicit Dropout(const DropArgs& a) {
    unsigned long long seed = a.seed, offset = a.offset;
    if (a.state) {
      seed += (unsigned long long)a.state[0];
      offset += (unsigned long long)a.state[1];
    }
    k0 = (uint32_t)seed;
    k1 = (uint32_t)(seed >> 32);
    o0 = (uint32_t)offset;
    o1 = (uint32_t)(offset >> 32);
    threshold = a.threshold;
    up = a.up;
  }
  // the numbers of columns 8 eighth .. 8 eighth + 7 of a row
  __device__ __forceinline__ u32x4 words(uint32_t eighth, uint32_t row) const {
    uint32_t c0 = eighth, c1 = row, c2 = o0, c3 = o1, a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t x = (uint64_t)c0 * 0xD2511F53u, y = (uint64_t)c2 * 0xCD9E8D57u;
      c0 = (uint32_t)(y >> 32) ^ c1 ^ a;
      c2 = (uint32_t)(x >> 32) ^ c3 ^ b;
      c1 = (uint32_t)y;
      c3 = (uint32_t)x;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
  }
  __device__ __forceinline__ bool keeps(const u32x4& w, int e) const {
    return ((e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) >= threshold;
  }
  // r + x of column e (0 .. 7) of those times up, or r whatever x is, to be rounded to O: an
  // fp32 number in every kernel. (Left to itself the compiler rounds to fp16 in the operation,
  // which is another number once in 200,000.)
  template <typename O>
  __device__ __forceinline__ float add(const u32x4& w, int e, float x, float r) const {
    float y = keeps(w, e) ? __builtin_fmaf(x, up, r) : r;
    if constexpr (sizeof(O) == 2) asm("" : "+v"(y));
    return y;
  }
};

}  // namespace vitattn
