// The choice of key blocks by a cheap score, for the attention over chosen blocks.
//
//   means:  m_j = mean of block j's keys, M_j = round(m_j (127 (1 / max|m_j|))) in 8 bits,
//           scale s_j = max|m_j| (1 / 127) (fp32; -1 of a block without keys)
//   choice: x_g = mean of a group's queries, X_g = round(x_g (127 (1 / max|x_g|))),
//           score_gj = fp32(X_g . M_j) * s_j; the topk blocks of highest score, ties to the
//           lowest, in ascending order, then -1
//
// (The query's own scale is positive and changes no order.) Every step is exact or
// one correctly rounded operation, so the choice is the same whatever the order in
// which a kernel adds: sums of bf16 values in fp64 (exact for values within 2^37 of each
// other), the mean and the scaling one fp64 operation each, products of whole numbers.
// A mean that is not finite counts as 0.
//
// The means are bound by reading the keys. The choice takes its scores from the matrix
// cores' 8-bit products (16 groups by 16 blocks by 64 columns an operation), 16 groups
// of one head per workgroup, and keeps them in LDS: 2,048 a group, with more blocks the
// best so far stay and compete with the next ones. A wave then takes a group at a time:
// its scores in registers as whole numbers that order alike, the topk-th largest found
// bit by bit by counting (ballots), and the chosen ones written in order.
#include "vitattn_common.h"
#include "vitattn_launch.h"

namespace vitattn {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ double finite_or_zero(double x) { return fabs(x) < 1e300 ? x : 0.; }
__device__ __forceinline__ double shfl_xor_f64(double x, int m) { return __shfl_xor(x, m, 64); }
__device__ __forceinline__ int eighth_of(double x, double by) { return (int)rint(x * by); }

// 8 whole numbers of -127 .. 127 as bytes
__device__ __forceinline__ uint2 pack_bytes(const int (&x)[8]) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(x[e] & 0xff) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void add_row(double (&s)[8], const uint16_t* p) {
  const bf16x8 x = as_bf16x8(*reinterpret_cast<const uint4*>(p));
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] += (double)(float)x[e];
}

// CH lanes take 8 columns of a row each (CH >= d / 8); a workgroup per block.
template <int CH>
__global__ __launch_bounds__(256) void means_kernel(const SelectArgs a) {
  constexpr int RG = 256 / CH;  // rows at a time
  constexpr int PER = 64 / CH;  // of them in a wave
  __shared__ double part[4][CH * 8];
  debug_poison_lds(part);
  const long long item = blockIdx.x;
  const int j = (int)(item % a.nb), bh = (int)(item / a.nb), b = bh / a.Hk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane % CH, row = threadIdx.x / CH;
  const int n = a.key_lens ? min(max(a.key_lens[b], 0), a.N) : a.N;
  const int count = min(max(n - j * a.block, 0), a.block);
  const uint16_t* const x = a.x + a.mx.head(bh, a.Hk) + (long long)j * a.block * a.mx.ld + 8 * c;
  const bool on = 8 * c < a.d;
  double s[8] = {};
  if (on)
    for (int r = row; r < count; r += RG) add_row(s, x + (long long)r * a.mx.ld);
#pragma unroll
  for (int m = CH; m < 64; m <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += shfl_xor_f64(s[e], m);
  static_assert(PER * CH == 64, "whole rows in a wave");
  if (lane < CH)
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][8 * c + e] = s[e];
  __syncthreads();
  if (wave != 0) return;
  double top = 0.;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s[e] = part[0][8 * c + e] + part[1][8 * c + e] + part[2][8 * c + e] + part[3][8 * c + e];
    s[e] = count > 0 ? finite_or_zero(s[e] / (double)count) : 0.;
    top = fmax(top, fabs(s[e]));
  }
#pragma unroll
  for (int m = 1; m < CH; m <<= 1) top = fmax(top, shfl_xor_f64(top, m));
  const double by = top > 0. ? 127. * (1. / top) : 0.;
  int q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = eighth_of(s[e], by);
  const int pitch = (a.d + 63) / 64 * 64;
  if (lane < CH && 8 * c < pitch) *reinterpret_cast<uint2*>(a.means + item * pitch + 8 * c) = pack_bytes(q);
  if (lane == 0) a.scales[item] = count > 0 ? (float)(top * (1. / 127.)) : -1.f;
}

// order-preserving whole numbers of fp32 values; 0 stands for none
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float((u & 0x80000000u) ? u ^ 0x80000000u : ~u);
}

constexpr int kTile = 16;  // groups of a workgroup

// NPL scores of a group per lane, KT 64-column steps of d, NW waves; MORE: blocks come in
// several turns, the first kSelectMax places hold the best of those before.
template <int NPL, int KT, int NW, bool MORE>
__global__ __launch_bounds__(64 * NW) void select_kernel(const SelectArgs a, int tiles) {
  constexpr int CH = KT == 1 ? 8 : KT == 2 ? 16 : 32;  // lanes of 8 columns
  constexpr int PITCH = 64 * KT;                       // means_pitch(d)
  constexpr int SP = 64 * NPL + 4;                     // a row of scores: rows four apart fall on other banks
  constexpr int FIRST = MORE ? kSelectMax : 0;
  __shared__ __attribute__((aligned(16))) int8_t qs[kTile][PITCH + 16];
  __shared__ float sc[kTile][SP];
  __shared__ int ids[MORE ? kTile : 1][MORE ? kSelectMax : 1];
  debug_poison_lds(qs, sc, ids);
  const int bh = blockIdx.x / tiles, g0 = (blockIdx.x - bh * tiles) * kTile;
  const int b = bh / a.H, head = bh - b * a.H, hk = head / (a.H / a.Hk);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  // the groups' queries: a wave per group, or 64 / CH groups of one query each
  const uint16_t* const q = a.x + a.mx.head(bh, a.H);
  const int c = lane % CH, slot = lane / CH;
  const bool single = a.q_block == 1;
  const int step = single ? 64 / CH : 1;
  for (int t = wave * step; t < kTile; t += NW * step) {
    const int local = single ? t + slot : t, g = g0 + local;
    double s[8] = {};
    const long long first = (long long)g * a.q_block;
    const int count = g < a.groups ? (int)min((long long)a.q_block, a.N - first) : 0;
    if (8 * c < a.d)
      for (int r = single ? 0 : slot; r < count; r += single ? 1 : 64 / CH) add_row(s, q + (first + r) * a.mx.ld + 8 * c);
    if (!single) {
#pragma unroll
      for (int m = CH; m < 64; m <<= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += shfl_xor_f64(s[e], m);
    }
    double top = 0.;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = count > 0 ? finite_or_zero(single ? s[e] : s[e] / (double)count) : 0.;
      top = fmax(top, fabs(s[e]));
    }
#pragma unroll
    for (int m = 1; m < CH; m <<= 1) top = fmax(top, shfl_xor_f64(top, m));
    const double by = top > 0. ? 127. * (1. / top) : 0.;
    int x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = eighth_of(s[e], by);
    if ((single || slot == 0) && 8 * c < PITCH) *reinterpret_cast<uint2*>(&qs[local][8 * c]) = pack_bytes(x);
  }
  __syncthreads();
  i32x4 qf[KT];  // A operand: group lane % 16, columns 16 (lane / 16) .. of a step
#pragma unroll
  for (int k = 0; k < KT; ++k) qf[k] = *reinterpret_cast<const i32x4*>(&qs[lane & 15][64 * k + 16 * (lane >> 4)]);

  const int8_t* const means = a.means + ((long long)b * a.Hk + hk) * a.nb * PITCH;
  const float* const scales = a.scales + ((long long)b * a.Hk + hk) * a.nb;
  constexpr int ROOM = 64 * NPL - FIRST;  // blocks of a turn
  if constexpr (MORE)
    for (int i = threadIdx.x; i < kTile * kSelectMax; i += 64 * NW) sc[i / kSelectMax][i % kSelectMax] = -INFINITY;
  for (int j0 = 0; j0 < a.nb; j0 += ROOM) {
    const int n = min(a.nb - j0, ROOM);  // of this turn
    // scores: a wave takes 16 blocks at a time, two of them in flight
    for (int j = wave * 16; j < n; j += NW * 32) {
      i32x4 m[2][KT];
      float s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int jj = j + u * NW * 16 + (lane & 15);
        const bool there = jj < n;
        s[u] = there ? scales[j0 + jj] : -1.f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
          m[u][k] = there ? *reinterpret_cast<const i32x4*>(means + (long long)(j0 + jj) * PITCH + 64 * k + 16 * (lane >> 4))
                          : i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KT; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qf[k], m[u][k], acc, 0, 0, 0);
        const int jj = j + u * NW * 16 + (lane & 15);
        if (jj < n)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[4 * (lane >> 4) + r][FIRST + jj] = s[u] < 0.f ? -INFINITY : (float)acc[r] * s[u];
      }
    }
    __syncthreads();
    const bool last = j0 + ROOM >= a.nb;
    for (int t = wave; t < kTile; t += NW) {
      const int g = g0 + t;
      if (g >= a.groups) break;
      uint32_t key[NPL];
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const int p = 64 * i + lane;
        const float x = p < FIRST + n ? sc[t][p] : -INFINITY;
        key[i] = x == -INFINITY ? 0u : ordered(x);
      }
      auto at_least = [&](uint32_t x) __attribute__((always_inline)) {
        int n_ = 0;
#pragma unroll
        for (int i = 0; i < NPL; ++i) n_ += __popcll(__ballot(key[i] >= x));
        return n_;
      };
      // the largest T that at least topk scores reach (1: fewer are there)
      uint32_t T = 0, hi = 0, lo = 0xffffffffu;
      if (at_least(1u) > a.topk) {
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
          hi = max(hi, key[i]);
          lo = min(lo, key[i]);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
          hi = max(hi, (uint32_t)__shfl_xor((int)hi, d, 64));
          lo = min(lo, (uint32_t)__shfl_xor((int)lo, d, 64));
        }
        hi = __builtin_amdgcn_readfirstlane(hi);
        lo = __builtin_amdgcn_readfirstlane(lo);
        // bits above the first in which they differ are common to all
        const uint32_t differ = hi ^ lo;
        uint32_t bit = differ ? 0x80000000u >> __builtin_clz(differ) : 0u;
        T = differ ? hi & ~(2u * bit - 1u) : hi;
        for (; bit != 0; bit >>= 1) {
          const int reach = at_least(T | bit);
          if (reach >= a.topk) T |= bit;
          if (reach == a.topk) break;
        }
      }
      if (T == 0) T = 1;
      // those above T, and as many of T's own as are left, in order
      int ties = T == 0xffffffffu ? a.topk : a.topk - at_least(T + 1), out = 0;
      int* const to = a.blocks + ((long long)bh * a.groups + g) * a.topk;
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const uint64_t above = __ballot(key[i] > T), equal = __ballot(key[i] == T);
        if ((above | equal) == 0) continue;
        const uint64_t before = (1ULL << lane) - 1;
        const bool mine = key[i] > T || (key[i] == T && (int)__popcll(equal & before) < ties);
        const uint64_t taken = __ballot(mine);
        if (mine) {
          const int p = 64 * i + lane, at = out + __popcll(taken & before);
          int id = j0 + p - FIRST;
          if (MORE && p < FIRST) id = ids[t][p];
          if (last) {
            to[at] = id;
          } else if constexpr (MORE) {  // (at <= p: read before, or in registers)
            ids[t][at] = id;
            sc[t][at] = unordered(key[i]);
          }
        }
        ties -= __popcll(taken & equal);
        out += __popcll(taken);
      }
      if (last) {
        for (int i = out + lane; i < a.topk; i += 64) to[i] = -1;
      } else if constexpr (MORE) {
        for (int i = out + lane; i < FIRST; i += 64) sc[t][i] = -INFINITY;
      }
    }
    __syncthreads();
  }
}

template <int KT>
hipError_t go(const SelectArgs& a) {
  const int tiles = (a.groups + kTile - 1) / kTile;
  const unsigned grid = (unsigned)(a.B * a.H) * tiles;
  if (a.nb <= 256) select_kernel<4, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, tiles);
  else if (a.nb <= 512) select_kernel<8, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, tiles);
  else if (a.nb <= 1024) select_kernel<16, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, tiles);
  else if (a.nb <= 2048) select_kernel<32, KT, 8, false><<<grid, 512, 0, a.stream>>>(a, tiles);
  else select_kernel<32, KT, 8, true><<<grid, 512, 0, a.stream>>>(a, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_means(const SelectArgs& a) {
  const unsigned grid = (unsigned)(a.B * a.Hk) * a.nb;
  if (a.d <= 64) means_kernel<8><<<grid, 256, 0, a.stream>>>(a);
  else if (a.d <= 128) means_kernel<16><<<grid, 256, 0, a.stream>>>(a);
  else means_kernel<32><<<grid, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_select(const SelectArgs& a) {
  return a.d <= 64 ? go<1>(a) : a.d <= 128 ? go<2>(a) : go<3>(a);
}

}  // namespace vitattn
