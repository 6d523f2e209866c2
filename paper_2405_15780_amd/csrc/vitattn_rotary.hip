// Rotary positions with several axes. Pair p of a row (a, b) at a position
// whose coordinate on the pair's axis is t turns by the angle t f_p:
//
//   a' = a cos(t f_p) - b sin(t f_p),   b' = b cos(t f_p) + a sin(t f_p)
//
// and the gradient by the opposite one. Bound by HBM (each row is read and
// written once); the angles are the work to keep small. A thread owns V pairs
// of one token: it forms their cosines and sines once and applies them to
// `group` heads of the queries and keys.
//
// Angles: the coordinate times a frequency in turns, in fp64, less the nearest
// whole number of turns. In fp32 a coordinate of 1e6 would leave 0.06 of a
// radian. What remains is at most half a turn, and fp32 holds its sine and
// cosine to about an ulp.
//
// Measured: 188,416 tokens of 16 query and 16 key heads of 64, bf16, three axes
// 321 us (1.55 GB, 4.8 TB/s; a large copy reaches 5.1); 2 x 5,003 tokens of 12 and
// 4 heads of 80, fp32, adjacent pairs 22 us (102 MB, 4.6 TB/s); one token 5.7 us,
// nearly all of it the launch. Requesting the next heads' pieces before these are
// written (U of them) took the first from 376 us to 328.
#include "vitattn_rows.h"

namespace vitattn {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double coordinate(const RotaryArgs& a, int b, int n, int axis) {
  const long long at = b * a.pos_batch + n * a.pos_row + axis * a.pos_axis;
  if (a.pos_type == 0) return (double)static_cast<const int*>(a.pos)[at];
  if (a.pos_type == 1) return (double)static_cast<const long long*>(a.pos)[at];
  return (double)static_cast<const float*>(a.pos)[at];
}

// Work item (token, piece): the row's `turned` pieces of V pairs, then (unless
// in place) its pieces of 2 V columns behind the last pair, copied as they are.
// blockIdx.y: which group of heads, blockIdx.z: batch.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, int turned, int pieces, int group) {
  constexpr int V = Piece<T>::V;
  const long long item = (long long)blockIdx.x * kThreads + threadIdx.x;
  const int n = (int)(item / pieces), piece = (int)(item - (long long)n * pieces);
  if (n >= a.N) return;
  const int b = blockIdx.z;
  const bool turn = piece < turned;
  const int R = a.pairs;
  // first and second elements: columns c0 .. and c1 .., n0 and n1 of them
  int c0, c1, n0, n1;
  float cs[V], sn[V];
  if (turn) {
    const int p0 = piece * V, np = min(R - p0, V);
    if (INTERLEAVED) {
      c0 = 2 * p0;
      c1 = c0 + V;
      n0 = min(2 * np, V);
      n1 = 2 * np - n0;
    } else {
      c0 = p0;
      c1 = R + p0;
      n0 = n1 = np;
    }
    int last = -1;
    double t = 0.;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int p = p0 + min(e, np - 1), axis = a.axis[p];
      if (axis != last) t = coordinate(a, b, n, axis);
      last = axis;
      const double turns = t * a.freq[p];
      sincospif(2.f * (float)(turns - rint(turns)), &sn[e], &cs[e]);
    }
  } else {
    c0 = 2 * R + (piece - turned) * 2 * V;
    c1 = c0 + V;
    n0 = min(a.d - c0, V);
    n1 = max(min(a.d - c1, V), 0);
  }
  const int heads = a.heads[0] + a.heads[1];
  const int h1 = min(heads, ((int)blockIdx.y + 1) * group);
  constexpr int U = 4;  // heads in flight
  for (int h0 = blockIdx.y * group; h0 < h1; h0 += U) {
    Piece<T> u[U], v[U];
    T* y[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int h = h0 + i < h1 ? h0 + i : h1 - 1;
      const int o = h >= a.heads[0];
      const int hh = o ? h - a.heads[0] : h;
      const T* x = static_cast<const T*>(a.x[o]) + a.mx[o].at(b, hh, n);
      y[i] = static_cast<T*>(a.y[o]) + a.my[o].at(b, hh, n);
      if (h0 + i < h1) {
        u[i].load(x + c0, n0);
        v[i].load(x + c1, n1);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (h0 + i >= h1) break;
      if (turn) {
        float p[V], q[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (INTERLEAVED) {  // pair e: elements 2e and 2e + 1 of the 2 V loaded
            const int k = 2 * e;
            const float first = k < V ? u[i].get(k % V) : v[i].get(k % V);
            const float second = k < V ? u[i].get(k % V + 1) : v[i].get(k % V + 1);
            const float f = first * cs[e] - second * sn[e], s = second * cs[e] + first * sn[e];
            if (k < V) {
              p[k % V] = f;
              p[k % V + 1] = s;
            } else {
              q[k % V] = f;
              q[k % V + 1] = s;
            }
          } else {
            const float first = u[i].get(e), second = v[i].get(e);
            p[e] = first * cs[e] - second * sn[e];
            q[e] = second * cs[e] + first * sn[e];
          }
        }
        u[i].set(p);
        v[i].set(q);
      }
      u[i].store(y[i] + c0, n0);
      v[i].store(y[i] + c1, n1);
    }
  }
}

template <typename T>
hipError_t go(const RotaryArgs& a) {
  constexpr int V = Piece<T>::V;
  const bool in_place = a.x[0] == a.y[0] && (a.heads[1] == 0 || a.x[1] == a.y[1]);
  const int turned = (a.pairs + V - 1) / V;
  const int rest = in_place ? 0 : (a.d - 2 * a.pairs + 2 * V - 1) / (2 * V);
  const int pieces = turned + rest;
  const int heads = a.heads[0] + a.heads[1];
  const long long blocks = ((long long)a.N * pieces + kThreads - 1) / kThreads;
  // heads per thread: as many as leave eight workgroups per CU, so that long
  // sequences form their angles once per 16 heads and short ones still fill the card
  int group = 16;
  while (group > 1 && blocks * a.B * ((heads + group - 1) / group) < 2048) group /= 2;
  const dim3 grid((unsigned)blocks, (heads + group - 1) / group, a.B);
  if (a.interleaved) rotary_kernel<T, true><<<grid, kThreads, 0, a.stream>>>(a, turned, pieces, group);
  else rotary_kernel<T, false><<<grid, kThreads, 0, a.stream>>>(a, turned, pieces, group);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a) {
  switch (a.type) {
    case kBf16: return go<__bf16>(a);
    case kFp16: return go<_Float16>(a);
    default: return go<float>(a);
  }
}

}  // namespace vitattn
