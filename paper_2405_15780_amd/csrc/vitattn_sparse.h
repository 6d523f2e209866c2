// Device helpers of the attention over chosen key blocks.
#pragma once

#include "vitattn_common.h"
#include "vitattn_launch.h"

namespace vitattn {

// chosen blocks that are listed at a time: all that one group may choose, or (MASKED)
// some of a tile's union
constexpr int kListAll = 1024;  // VITATTN_SPARSE_MAX_TOPK
constexpr int kListUnion = 128;

// keys of sample b: the first key_lens[b] of Nk, brought into 0 .. Nk
__device__ __forceinline__ int sparse_keys(const SparseArgs& a, int b) {
  return a.key_lens ? min(max(a.key_lens[b], 0), a.Nk) : a.Nk;
}

// The rows [row0, row0 + rows) of a query tile and what their groups chose: `n`
// consecutive numbers of blocks.
struct Chosen {
  const int* at;
  int n, first_group, row0;
  __device__ __forceinline__ Chosen(const SparseArgs& a, int bh, int row, int rows) : row0(row) {
    first_group = row / a.q_block;
    const int last = (min(row + rows, a.Nq) - 1) / a.q_block;
    at = a.blocks + ((long long)bh * a.groups + first_group) * a.topk;
    n = (last - first_group + 1) * a.topk;
  }
  // the tile's rows (of 64) that chose entry e
  __device__ __forceinline__ uint64_t rows_of(const SparseArgs& a, int e) const {
    const int g = first_group + e / a.topk;
    const long long lo = max((long long)g * a.q_block - row0, 0LL), hi = min((g + 1LL) * a.q_block - row0, 64LL);
    return (hi >= 64 ? ~0ULL : (1ULL << hi) - 1) & (~0ULL << lo);
  }
};

// The blocks that any row of a query tile chose, each once and in ascending order
// whatever the order they were given in, and (MASKED) the rows that chose each. A bit
// per key block; numbers outside the sample's blocks set none.
constexpr int kNone = 0xffff;
template <bool MASKED>
struct BlockList {
  static constexpr int kCap = MASKED ? kListUnion : kListAll;
  uint32_t bits[kSparseMaxBlocks / 32];
  uint16_t before[kSparseMaxBlocks / 32];  // blocks listed before a word's
  uint16_t id[kCap + 8];               // then kNone
  uint64_t masks[MASKED ? kCap + 8 : 1];
  int total;

  // Sets the bits of entries that a row of `filter` chose; returns their number.
  template <int NT>
  __device__ __forceinline__ int build(const SparseArgs& a, const Chosen& c, int real, uint64_t filter) {
    const int words = (a.nb + 31) >> 5;
    for (int i = threadIdx.x; i < words; i += NT) bits[i] = 0;
    __syncthreads();
    for (int e = threadIdx.x; e < c.n; e += NT) {
      const int id = c.at[e];
      if ((unsigned)id >= (unsigned)real) continue;
      if (MASKED && (c.rows_of(a, e) & filter) == 0) continue;
      atomicOr(&bits[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    if (threadIdx.x < 64) {
      const int per = (words + 63) >> 6, first = threadIdx.x * per;
      int n = 0;
      for (int k = 0; k < per; ++k)
        if (first + k < words) n += __popc(bits[first + k]);
      int upto = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(upto, d, 64);
        if ((int)threadIdx.x >= d) upto += x;
      }
      int base = upto - n;
      for (int k = 0; k < per; ++k)
        if (first + k < words) {
          before[first + k] = (uint16_t)base;
          base += __popc(bits[first + k]);
        }
      if (threadIdx.x == 63) total = upto;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(total);
  }
  // How many of build's `count` blocks lie before block x. (Reads what the next build clears: a
  // barrier belongs between the two, unless fill comes between them, which ends with one.)
  __device__ __forceinline__ int below(int x, int nb, int count) const {
    if (x >= nb) return count;
    return __builtin_amdgcn_readfirstlane(before[x >> 5] + __popc(bits[x >> 5] & ((1u << (x & 31)) - 1)));
  }
  // Lists the blocks r0 .. r0 + n - 1 (n <= kCap) of those.
  template <int NT>
  __device__ __forceinline__ void fill(const SparseArgs& a, const Chosen& c, int real, uint64_t filter, int r0, int n) {
    const int words = (a.nb + 31) >> 5;
    for (int i = threadIdx.x; i < words; i += NT) {
      uint32_t m = bits[i];
      for (int r = before[i] - r0; m != 0 && r < n; ++r, m &= m - 1)
        if (r >= 0) id[r] = (uint16_t)(32 * i + __builtin_ctz(m));
    }
    if (threadIdx.x < 8) id[n + threadIdx.x] = kNone;
    if constexpr (MASKED) {
      for (int i = threadIdx.x; i < n + 8; i += NT) masks[i] = 0;
      __syncthreads();
      for (int e = threadIdx.x; e < c.n; e += NT) {
        const int x = c.at[e];
        if ((unsigned)x >= (unsigned)real) continue;
        const uint64_t rows = c.rows_of(a, e) & filter;
        const int r = before[x >> 5] + __popc(bits[x >> 5] & ((1u << (x & 31)) - 1)) - r0;
        if (rows != 0 && r >= 0 && r < n) atomicOr(reinterpret_cast<unsigned long long*>(&masks[r]), (unsigned long long)rows);
      }
    }
    __syncthreads();
  }
  // the first key of a listed block from its entry as it was read (Nk behind the last)
  __device__ __forceinline__ static int key_of(uint32_t entry, int block, int Nk) {
    const int x = __builtin_amdgcn_readfirstlane((int)entry);
    return x == kNone ? Nk : x * block;
  }
};

// A tile's place in the list: entry, and which of the block's tiles.
struct TileAt {
  int e, s;
  __device__ __forceinline__ void next(int tiles) {
    if (++s == tiles) {
      s = 0;
      ++e;
    }
  }
};

// four consecutive outputs rounded to bf16
__device__ __forceinline__ void store4_bf16(uint16_t* p, float a, float b, float c, float d) {
  const bf16x2 lo = {(__bf16)a, (__bf16)b}, hi = {(__bf16)c, (__bf16)d};
  *reinterpret_cast<uint2*>(p) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// Whether every row of a query tile of `rows` belongs to one group.
inline bool one_group(const SparseArgs& a, int rows) { return a.q_block % rows == 0 || a.q_block >= a.Nq; }
// Splits of the chosen blocks of a tile of few queries (a head's own sizes alone).
int sparse_splits(const SparseArgs& a);

}  // namespace vitattn
