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
// best so far stay and compete with the next ones. A wave then takes two groups at a time,
// their scores in registers as whole numbers that order alike. The topk-th largest of the
// lanes' highest, found bit by bit by counting (ballots), is reached by topk scores and few
// more; these go to a lane each, where the same search finds the threshold.
//
// 8 heads of 32,768 groups choose 16 of 512 blocks (d = 64) in 206 us, bound by the search's
// scalar and vector instructions (80 and 71 million; the products are a twentieth, the
// bytes 16 us): taking the largest topk times over was 375 us, the search over all scores 245.
// A group of 1,024 blocks (d = 128): 8.6 us, one workgroup's latency. The means of 8 x 32,768
// keys of 64: 17 us, a launch of 2.0 TB/s.
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

// order-preserving whole numbers of fp32 values; 0 stands for none. (No score is -0: the
// scale of keys that are not all 0 is at least 2^-133 / 1024 / 127 > 2^-150, and not 0.)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}


// the value of a lane in another place: of the quad, half a row of 16 or a row mirrored,
// the neighbouring row, the other half of the wave
template <int CTRL>
__device__ __forceinline__ uint32_t lane_swap(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t row_swap(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return (threadIdx.x & 16) ? r[0] : r[1];
}
__device__ __forceinline__ uint32_t half_swap(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return (threadIdx.x & 32) ? r[0] : r[1];
}
// the largest over the wave, the same (scalar) in all
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, lane_swap<0xB1>(x));
  x = max(x, lane_swap<0x4E>(x));
  x = max(x, lane_swap<0x141>(x));
  x = max(x, lane_swap<0x140>(x));
  x = max(x, row_swap(x));
  x = max(x, half_swap(x));
  return __builtin_amdgcn_readfirstlane(x);
}
// of this mask's lanes, those before the lane
__device__ __forceinline__ int lanes_before(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

constexpr int kTile = 16;  // groups of a workgroup

// NPL scores of a group per lane, KT 64-column steps of d, NW waves; MORE: blocks come in
// several turns, the first kSelectMax places hold the best of those before.
template <int NPL, int KT, int NW, bool MORE>
__global__ __launch_bounds__(64 * NW) void select_kernel(const SelectArgs a, int per_key) {
  constexpr int CH = KT == 1 ? 8 : KT == 2 ? 16 : 32;  // lanes of 8 columns
  constexpr int PITCH = 64 * KT;                       // means_pitch(d)
  constexpr int SP = 64 * NPL + 4;                     // a row of scores: rows four apart fall on other banks
  constexpr int FIRST = MORE ? kSelectMax : 0;
  __shared__ __attribute__((aligned(16))) int8_t qs[kTile][PITCH + 16];
  __shared__ uint32_t sc[kTile][SP];  // scores as whole numbers in their order, 0: none
  __shared__ uint32_t best[NW][2][2][68];  // a wave's candidates: scores and places (behind 64: dropped)
  __shared__ int ids[MORE ? kTile : 1][MORE ? kSelectMax : 1];
  debug_poison_lds(qs, sc, best, ids);
  const int b = blockIdx.z, head = blockIdx.y, bh = b * a.H + head, hk = head / per_key, g0 = blockIdx.x * kTile;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  const int8_t* const means = a.means + ((long long)b * a.Hk + hk) * a.nb * PITCH;
  const float* const scales = a.scales + ((long long)b * a.Hk + hk) * a.nb;
  constexpr int ROOM = 64 * NPL - FIRST;  // blocks of a turn
  // Batches of four times 16 blocks per wave, the next one on its way while one is
  // multiplied, the first while the queries are.
  constexpr int TB = 4;
  struct Batch {
    i32x4 m[TB][KT];
    float s[TB];
  };
  auto load = [&](Batch& x, int j0, int j, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < TB; ++u) {
      const int jj = min(j + u * NW * 16 + (lane & 15), n - 1);  // (those past the last are not kept)
      x.s[u] = scales[j0 + jj];
#pragma unroll
      for (int k = 0; k < KT; ++k)
        x.m[u][k] = *reinterpret_cast<const i32x4*>(means + (long long)(j0 + jj) * PITCH + 64 * k + 16 * (lane >> 4));
    }
  };
  Batch next;
  load(next, 0, wave * 16, min(a.nb, ROOM));

  // the groups' queries: a wave per group, or 64 / CH groups of one query each
  const uint16_t* const q = a.x + b * a.mx.sb + head * a.mx.sh;
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

  if constexpr (MORE)
    for (int i = threadIdx.x; i < kTile * kSelectMax; i += 64 * NW) sc[i / kSelectMax][i % kSelectMax] = 0;
  for (int j0 = 0; j0 < a.nb; j0 += ROOM) {
    const int n = min(a.nb - j0, ROOM);  // of this turn
    for (int j = wave * 16; j < n; j += NW * 16 * TB) {
      const Batch x = next;
      if (j + NW * 16 * TB < n) load(next, j0, j + NW * 16 * TB, n);
#pragma unroll
      for (int u = 0; u < TB; ++u) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KT; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qf[k], x.m[u][k], acc, 0, 0, 0);
        const int j1 = j + u * NW * 16, jj = j1 + (lane & 15);
        if (MORE && j1 >= ROOM) break;
        const uint32_t there = x.s[u] < 0.f || jj >= n ? 0u : ~0u;
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[4 * (lane >> 4) + r][FIRST + jj] = ordered((float)acc[r] * x.s[u]) & there;
      }
    }
    for (int r = wave; r < kTile && n < ROOM; r += NW)  // no blocks behind the last
      for (int i = n + lane; i < ROOM; i += 64) sc[r][FIRST + i] = 0;
    if (j0 + ROOM < a.nb) load(next, j0 + ROOM, wave * 16, min(a.nb - j0 - ROOM, ROOM));
    __syncthreads();
    const bool last = j0 + ROOM >= a.nb;
    // two groups at a time, whose counts overlap
    for (int t = 2 * wave; t < kTile; t += 2 * NW) {
      if (g0 + t >= a.groups) break;
      uint32_t key[2][NPL], most[2] = {0, 0}, T[2], hi[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
          const int p = 64 * i + lane;
          key[u][i] = sc[t + u][p] & (g0 + t + u < a.groups ? ~0u : 0u);
          most[u] = max(most[u], key[u][i]);
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) hi[u] = wave_max(most[u]);
      auto at_least = [&](int u, uint32_t x) __attribute__((always_inline)) {
        int n_ = 0;
#pragma unroll
        for (int i = 0; i < NPL; ++i) n_ += (int)__popcll(__ballot(key[u][i] >= x));
        return n_;
      };
      // The largest T >= from that at least topk of the numbers counted reach, or the first
      // that topk to `enough` do: those between it and the highest share its leading bits.
      auto search = [&](auto count, const uint32_t (&from)[2], int enough) __attribute__((always_inline)) {
        uint32_t bit[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t differ = hi[u] ^ from[u];
          bit[u] = differ ? 0x80000000u >> __builtin_clz(differ) : 0u;
          T[u] = differ ? hi[u] & ~(2u * bit[u] - 1u) : hi[u];
          while (bit[u] != 0 && (T[u] | bit[u]) <= from[u]) {
            T[u] |= bit[u];
            bit[u] >>= 1;
          }
        }
        while ((bit[0] | bit[1]) != 0) {
          int reach[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) reach[u] = count(u, T[u] | bit[u]);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            T[u] = reach[u] >= a.topk ? T[u] | bit[u] : T[u];
            bit[u] = (unsigned)(reach[u] - a.topk) <= (unsigned)(enough - a.topk) ? 0 : bit[u] >> 1;
          }
        }
      };
      // What topk of the lanes' highest reach, at least topk scores do, and seldom many
      // more: these are the candidates, at most one a lane if all goes well.
      uint32_t from[2] = {0, 0};
      int found[2] = {65, 65};
      if (a.topk <= 64) {
        search([&](int u, uint32_t x) __attribute__((always_inline)) { return (int)__popcll(__ballot(most[u] >= x)); }, from, a.topk + a.topk / 4);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          from[u] = max(T[u], 1u);
          found[u] = 0;
#pragma unroll
          for (int i = 0; i < NPL; ++i) {
            const bool mine = key[u][i] >= from[u];
            const uint64_t taken = __ballot(mine);
            int at = min(found[u] + lanes_before(taken), 64);
            asm("" : "+v"(at));  // (formed by every lane, not behind a branch)
            at = mine ? at : 64;
            best[wave][u][0][at] = key[u][i];
            best[wave][u][1][at] = 64 * i + lane;
            found[u] += (int)__popcll(taken);
          }
        }
      }
      const bool few = found[0] <= 64 && found[1] <= 64;
      uint32_t cand[2] = {0, 0};
      if (few) {
#pragma unroll
        for (int u = 0; u < 2; ++u) cand[u] = lane < found[u] ? best[wave][u][0][lane] : 0u;
        search([&](int u, uint32_t x) __attribute__((always_inline)) { return (int)__popcll(__ballot(cand[u] >= x)); }, from, a.topk);
      } else {
        search(at_least, from, a.topk);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int g = g0 + t + u;
        if (g >= a.groups) break;
        const uint32_t least = max(T[u], 1u);  // (0: fewer are there)
        int* const to = a.blocks + ((long long)bh * a.groups + g) * a.topk;
        int out = 0;
        // writes the places p of the lanes with `mine`
        auto put = [&](bool mine, int p, uint32_t score) __attribute__((always_inline)) {
          const uint64_t taken = __ballot(mine);
          if (mine) {
            const int at = out + lanes_before(taken);
            int id = j0 + p - FIRST;
            if (MORE && p < FIRST) id = ids[t + u][p];
            if (last) {
              to[at] = id;
            } else if constexpr (MORE) {  // (at <= p: read before, or in registers)
              ids[t + u][at] = id;
              sc[t + u][at] = score;
            }
          }
          out += (int)__popcll(taken);
        };
        // those above the least, and as many of its own as are left, in order
        if (few) {
          const uint64_t above = __ballot(cand[u] > least), equal = __ballot(cand[u] == least);
          const bool mine = cand[u] > least || (cand[u] == least && lanes_before(equal) < a.topk - (int)__popcll(above));
          put(mine, lane < found[u] ? (int)best[wave][u][1][lane] : 0, cand[u]);
        } else {
          int ties = a.topk - (least == 0xffffffffu ? 0 : at_least(u, least + 1));
#pragma unroll
          for (int i = 0; i < NPL; ++i) {
            const uint64_t equal = __ballot(key[u][i] == least);
            const bool mine = key[u][i] > least || (key[u][i] == least && lanes_before(equal) < ties);
            ties -= (int)__popcll(equal);
            put(mine, 64 * i + lane, key[u][i]);
          }
        }
        if (last) {
          for (int i = out + lane; i < a.topk; i += 64) to[i] = -1;
        } else if constexpr (MORE) {
          for (int i = out + lane; i < FIRST; i += 64) sc[t + u][i] = 0;
        }
      }
    }
    __syncthreads();
  }
}

template <int KT>
hipError_t go(const SelectArgs& a) {
  const dim3 grid((a.groups + kTile - 1) / kTile, a.H, a.B);
  const int per_key = a.H / a.Hk;
  // A few groups (one workgroup a head): more waves read the means at once. 8 heads of 128, 1
  // and 16 groups: 768 blocks in 7.7 and 15.4 us with sixteen waves, 9.5 and 17.7 with four;
  // 1,024 in 8.2 and 15.8 (10.2 and 18.2). Not of up to 512 blocks (512: 7.6 and 14.1 with
  // sixteen, 7.3 and 12.2 with four) nor of more than 1,024 (1,025: 12.8 and 27.5 with sixteen,
  // 11.3 and 25.3 with eight; 2,048: 15.4 and 31.3, 13.9 and 28.9).
  if (a.groups <= kTile && a.nb > 512 && a.nb <= 1024) select_kernel<16, KT, 16, false><<<grid, 1024, 0, a.stream>>>(a, per_key);
  else if (a.nb <= 256) select_kernel<4, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, per_key);
  else if (a.nb <= 512) select_kernel<8, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, per_key);
  else if (a.nb <= 1024) select_kernel<16, KT, 4, false><<<grid, 256, 0, a.stream>>>(a, per_key);
  else if (a.nb <= 2048) select_kernel<32, KT, 8, false><<<grid, 512, 0, a.stream>>>(a, per_key);
  else select_kernel<32, KT, 8, true><<<grid, 512, 0, a.stream>>>(a, per_key);
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
