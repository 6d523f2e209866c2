// Backward of the rms norm with the residual's addition (vitattn_rms.hip): with
// n = h r and g = dy w,
//
//   dh' = r (g - n mean(g n)) + dh,  dresidual = dh',  dx = m dh',  dw = sum_rows dy n
//
// where dh is the gradient that h has from what follows it and m dropout's mask, formed
// again. dx and dresidual are both rounded from the fp32 dh'; where they would be the
// same (one type, no dropout) one is written.
//
// Bound by HBM: h, dy and dh are read once, dx and dresidual written once; a row stays
// in registers. dw as in vitattn_norm.hip: a workgroup of a grid that depends on the
// sizes alone keeps its share, writes one row of partial sums, and a second kernel adds
// those in order. Sums are fp32. No atomics. 32,768 rows of 1,024 bf16 with dropout: 62 us,
// 5.4 TB/s of what it reads and writes (h, partly from the caches), and 5 us for dw.
#include "vitattn_rms.h"

namespace vitattn {

namespace {

constexpr int kThreads = kRowThreads;

// The next long row is held as well where there are registers for it.
constexpr bool row_ahead(int np, int v) { return np * v <= 16; }

template <typename T, typename R, int NP, bool BLOCK>
__global__ __launch_bounds__(kThreads) void rms_bwd_kernel(const RmsArgs a) {
  constexpr int V = Piece<T>::V;
  constexpr bool AHEAD = BLOCK && row_ahead(NP, V);
  __shared__ float lds[4];
  __shared__ float part[BLOCK ? 1 : kThreads][V];
  debug_poison_lds(lds, part);
  const Place<BLOCK> at(a.lanes);
  const int L = at.L, lane = at.lane, per = at.per;
  const Dropout drop(a.drop);
  float w[NP][V], dw[NP][V];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i][e] = 1.f;
      dw[i][e] = 0.f;
    }
    if (a.w) load_weights<T>(a.w, a.w_f32, c, columns_of<V>(a.D, c), w[i]);
  }
  const float inv = 1.f / (float)a.D;
  struct Row {
    Span<R, V> h[NP], dh[NP];
    Span<T, V> g[NP];
    float rstd;
  };
  auto load = [&](Row& row, int r) __attribute__((always_inline)) {
    const bool on = at.row >= 0 && r < a.rows;
    const RowAt i(a, on ? r : 0);
    const R* h = static_cast<const R*>(a.h) + i.in(a.mh);
    const R* dh = static_cast<const R*>(a.dh) + (a.dh ? i.in(a.mdh) : 0);
    const T* g = static_cast<const T*>(a.dy) + i.in(a.mdy);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = (lane + k * L) * V;
      row.h[k].load(h, c, a.D);
      row.g[k].load(g, c, a.D);
      if (a.dh) row.dh[k].load(dh, c, a.D);
      else row.dh[k].clear();
    }
    row.rstd = on ? a.rstd[i.in(a.ml)] : 0.f;
  };
  Row row, next;
  const int step = gridDim.x * per;
  int r0 = blockIdx.x * per + at.row;
  if (AHEAD && r0 < a.rows) load(next, r0);
  for (; r0 - at.row < a.rows; r0 += step) {
    if constexpr (AHEAD) {
      row = next;
      if (r0 + step < a.rows) load(next, r0 + step);
    } else {
      load(row, r0);
    }
    const bool on = at.row >= 0 && r0 < a.rows;
    const float rstd = row.rstd;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V;
      row.h[i].settle(c, a.D, on);
      row.g[i].settle(c, a.D, on);
      if (a.dh) row.dh[i].settle(c, a.D, on);
    }
    // lanes past the row hold dy = 0 and add nothing to any sum
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = row.g[i].get(e), n = row.h[i].get(e) * rstd;
        s = __builtin_fmaf(d * w[i][e], n, s);
        dw[i][e] = __builtin_fmaf(d, n, dw[i][e]);
      }
    const float m = -at.sum(s, lds) * inv * rstd;
    if (!on) continue;
    const RowAt ix(a, r0);
    const uint32_t logical = (uint32_t)ix.in(a.ml);
    R* dres = static_cast<R*>(a.dres) + (a.dres ? ix.in(a.mdres) : 0);
    T* dx = static_cast<T*>(a.dx) + (a.dx ? ix.in(a.mdx) : 0);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V, n = columns_of<V>(a.D, c);
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float nv = row.h[i].get(e) * rstd;
        v[e] = __builtin_fmaf(row.g[i].get(e) * w[i][e], rstd, __builtin_fmaf(nv, m, row.dh[i].get(e)));
      }
      if (a.dres) {
        Span<R, V> o;
        o.set(v);
        o.store(dres + c, n);
      }
      if (a.dx) {
        if (a.drop_on) {
          const PieceMask<V> mask(drop, c, logical);
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = mask.template add<T>(drop, e, v[e], 0.f);
        }
        Span<T, V> o;
        o.set(v);
        o.store(dx + c, n);
      }
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (long long)blockIdx.x * a.D;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = dw[i][e];
    if constexpr (!BLOCK) {
      // the workgroup's rows, in their order
      __syncthreads();
      if (at.row >= 0)
#pragma unroll
        for (int e = 0; e < V; ++e) part[at.row * L + lane][e] = v[e];
      __syncthreads();
      if (at.row != 0) continue;
      for (int r = 1; r < per; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += part[r * L + lane][e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < a.D) out[c + e] = v[e];
  }
}

// dw from n partial rows: a workgroup takes 64 of the D columns, its 16 waves every
// 16th row each, eight loads in flight, added in a fixed order.
constexpr int kWeightWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kWeightWaves) void rms_weight_kernel(const RmsArgs a, int n) {
  __shared__ float part[kWeightWaves][64];
  debug_poison_lds(part);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < a.D) {
    const float* src = a.partial + c;
    int p = wave;
    for (; p + 7 * kWeightWaves < n; p += 8 * kWeightWaves) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = src[(long long)(p + u * kWeightWaves) * a.D];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
    for (; p < n; p += kWeightWaves) s += src[(long long)p * a.D];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= a.D) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kWeightWaves; ++w) s += part[w][lane];
  if (a.w_f32) static_cast<float*>(a.dw)[c] = s;
  else static_cast<T*>(a.dw)[c] = (T)s;
}

// Workgroups of a CU, from a lane's registers: three fp32 values per element (w, dw and
// the new gradient) and the rows as they are.
constexpr int resident(int np, int v, bool block) {
  const int regs = 3 * np * v + (block && row_ahead(np, v) ? 32 : 20) * np + 48;
  return regs <= 128 ? 4 : regs <= 170 ? 3 : regs <= 270 ? 2 : 1;
}

int rows_of(const RowShape& s) { return s.lanes > 64 ? 1 : 64 / s.lanes * (kThreads / 64); }
RowShape shape(int D, int V) {
  RowShape s = rms_shape(D, V, false, true);
  if (s.np == 5) s.np = 6;
  return s;
}

template <typename T, typename R, int NP, bool BLOCK>
hipError_t go(const RmsArgs& a, int grid) {
  rms_bwd_kernel<T, R, NP, BLOCK><<<grid, kThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

template <typename T, typename R>
hipError_t go_shape(const RmsArgs& a, const RowShape& s, int n) {
  const bool block = s.lanes > 64;
  switch (s.np) {
    case 1: return block ? go<T, R, 1, true>(a, n) : go<T, R, 1, false>(a, n);
    case 2: return block ? go<T, R, 2, true>(a, n) : go<T, R, 2, false>(a, n);
    case 3: return go<T, R, 3, true>(a, n);
    case 4: return go<T, R, 4, true>(a, n);
    case 6: return go<T, R, 6, true>(a, n);
    default: return go<T, R, 8, true>(a, n);
  }
}

template <typename T, typename R>
hipError_t bwd_t(RmsArgs a) {
  const RowShape s = shape(a.D, Piece<T>::V);
  const int n = rms_partials(a.rows, a.D, (int)sizeof(T));
  a.lanes = s.lanes;
  const hipError_t err = go_shape<T, R>(a, s, n);
  if (err != hipSuccess || !a.partial) return err;
  rms_weight_kernel<T><<<(a.D + 63) / 64, 64 * kWeightWaves, 0, a.stream>>>(a, n);
  return hipGetLastError();
}

}  // namespace

int rms_partials(int rows, int D, int elem_bytes) {
  const int V = 16 / elem_bytes;
  const RowShape s = shape(D, V);
  const int groups = (int)(((long long)rows + rows_of(s) - 1) / rows_of(s));
  return min(groups, 256 * resident(s.np, V, s.lanes > 64));
}

hipError_t launch_rms_bwd(const RmsArgs& a) {
  switch (a.type) {
    case kBf16: return a.residual_type == kFp32 ? bwd_t<__bf16, float>(a) : bwd_t<__bf16, __bf16>(a);
    case kFp16: return a.residual_type == kFp32 ? bwd_t<_Float16, float>(a) : bwd_t<_Float16, _Float16>(a);
    default: return bwd_t<float, float>(a);
  }
}

}  // namespace vitattn
