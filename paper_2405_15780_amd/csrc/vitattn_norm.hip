// Layer norm of rows of D elements, forward and backward:
//
//   mu = mean x,  r = 1/sqrt(mean (x - mu)^2 + eps),  h = (x - mu) r,  y = h w + b
//   g = dy w,  dx = r (g - mean g - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
//
// Bound by HBM: the forward reads x and writes y, the backward reads x and dy
// and writes dx, so a row is read once and kept in registers: the mean, then
// the sum of squared deviations from it (no cancellation of large squares).
// Statistics, products and sums are fp32; x, y, dy and dx are rounded once, to
// their type.
//
// L lanes share a row, each holding NP pieces of 16 bytes (pieces lane, lane +
// L, ..): a power of two of a wave's lanes for short rows, 64 / L rows per
// wave, and the four waves of a workgroup for long ones. Rows too long for
// registers (over 256 * 8 pieces) are read once per pass instead, from L2.
//
// The backward's workgroups each take a fixed run of row groups and keep their
// share of dw and db in registers; at the end the workgroup adds its lanes'
// and waves' shares in a fixed order and writes one row of partial sums, and a
// second kernel adds those in order. Their number depends on the row count
// alone, so dw and db have the same bits on any device.
#include "vitattn_rows.h"

namespace vitattn {

namespace {

constexpr int kThreads = 256;

// row r -> its three indexes
__device__ __forceinline__ void split_row(const NormArgs& a, int r, int& i0, int& i1, int& i2) {
  const int t = r / a.n2;
  i2 = r - t * a.n2;
  i0 = t / a.n1;
  i1 = t - i0 * a.n1;
}
__device__ __forceinline__ long long row_at(const NormArgs& a, const RowMap& m, int r) {
  int i0, i1, i2;
  split_row(a, r, i0, i1, i2);
  return m.at(i0, i1, i2);
}

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

// Sum over the L lanes of a row (BLOCK: over the workgroup), the same in all.
template <bool BLOCK>
__device__ __forceinline__ float row_sum(float x, int L, float* lds) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1)
    if (BLOCK || m < L) x += __shfl_xor(x, m, 64);
  if constexpr (BLOCK) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0] + lds[1] + lds[2] + lds[3];
  }
  return x;
}

template <typename T, int NP, bool BLOCK>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const int L = a.lanes;
  const int lane = threadIdx.x % L;
  const int per = kThreads / L;  // rows of a workgroup at a time
  float w[NP][V], b[NP][V];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V, n = min(max(a.D - c, 0), V);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i][e] = 1.f;
      b[i][e] = 0.f;
    }
    if (a.w) load_weights<T>(a.w, a.w_f32, c, n, w[i]);
    if (a.b) load_weights<T>(a.b, a.w_f32, c, n, b[i]);
  }
  const float inv = 1.f / (float)a.D;
  for (int r0 = blockIdx.x * per; r0 < a.rows; r0 += gridDim.x * per) {
    const int r = r0 + threadIdx.x / L;
    const bool on = r < a.rows;
    const T* x = static_cast<const T*>(a.x) + (on ? row_at(a, a.mx, r) : 0);
    Piece<T> p[NP];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V;
      p[i].load(x + c, on ? min(max(a.D - c, 0), V) : 0);
#pragma unroll
      for (int e = 0; e < V; ++e) s += p[i].get(e);
    }
    const float mean = row_sum<BLOCK>(s, L, lds) * inv;
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int n = a.D - (lane + i * L) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = p[i].get(e) - mean;
        q += e < n ? d * d : 0.f;
      }
    }
    const float rstd = rsqrtf(row_sum<BLOCK>(q, L, lds) * inv + a.eps);
    if (!on) continue;
    T* y = static_cast<T*>(a.y) + row_at(a, a.my, r);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V;
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = (p[i].get(e) - mean) * rstd * w[i][e] + b[i][e];
      Piece<T> o;
      o.set(v);
      o.store(y + c, min(max(a.D - c, 0), V));
    }
    if (lane == 0 && a.mean) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// Rows too long for registers: three passes over the row.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_fwd_long_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const float inv = 1.f / (float)a.D;
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row_at(a, a.mx, r);
    T* y = static_cast<T*>(a.y) + row_at(a, a.my, r);
    float s = 0.f, q = 0.f;
    for (int c = threadIdx.x * V; c < a.D; c += kThreads * V) {
      Piece<T> p;
      p.load(x + c, min(a.D - c, V));
#pragma unroll
      for (int e = 0; e < V; ++e) s += p.get(e);
    }
    const float mean = row_sum<true>(s, 64, lds) * inv;
    for (int c = threadIdx.x * V; c < a.D; c += kThreads * V) {
      Piece<T> p;
      p.load(x + c, min(a.D - c, V));
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = p.get(e) - mean;
        q += e < a.D - c ? d * d : 0.f;
      }
    }
    const float rstd = rsqrtf(row_sum<true>(q, 64, lds) * inv + a.eps);
    for (int c = threadIdx.x * V; c < a.D; c += kThreads * V) {
      const int n = min(a.D - c, V);
      Piece<T> p;
      p.load(x + c, n);
      float w[V], b[V], v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        w[e] = 1.f;
        b[e] = 0.f;
      }
      if (a.w) load_weights<T>(a.w, a.w_f32, c, n, w);
      if (a.b) load_weights<T>(a.b, a.w_f32, c, n, b);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = (p.get(e) - mean) * rstd * w[e] + b[e];
      p.set(v);
      p.store(y + c, n);
    }
    if (threadIdx.x == 0 && a.mean) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// dx, and this workgroup's partial sums of dw and db (a.partial: rows of 2 D
// floats, dw then db) if a.partial is set. Workgroup g takes row groups g,
// g + gridDim.x, ..
template <typename T, int NP, bool BLOCK>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  __shared__ float lds[4];
  __shared__ float part[BLOCK ? 1 : 4][BLOCK ? 1 : 64][V];
  debug_poison_lds(lds, part);
  const int L = a.lanes;
  const int lane = threadIdx.x % L;
  const int per = kThreads / L;
  float w[NP][V], dw[NP][V], db[NP][V];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V, n = min(max(a.D - c, 0), V);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i][e] = 1.f;
      dw[i][e] = db[i][e] = 0.f;
    }
    if (a.w) load_weights<T>(a.w, a.w_f32, c, n, w[i]);
  }
  const float inv = 1.f / (float)a.D;
  for (int r0 = blockIdx.x * per; r0 < a.rows; r0 += gridDim.x * per) {
    const int r = r0 + threadIdx.x / L;
    const bool on = r < a.rows;
    const T* x = static_cast<const T*>(a.x) + (on ? row_at(a, a.mx, r) : 0);
    const T* dy = static_cast<const T*>(a.dy) + (on ? row_at(a, a.mdy, r) : 0);
    const float mean = on ? a.mean[r] : 0.f, rstd = on ? a.rstd[r] : 0.f;
    Piece<T> p[NP], g[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V, n = on ? min(max(a.D - c, 0), V) : 0;
      p[i].load(x + c, n);
      g[i].load(dy + c, n);
    }
    // lanes past the row hold dy = 0 and add nothing to any sum
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = g[i].get(e), h = (p[i].get(e) - mean) * rstd, gw = d * w[i][e];
        s1 += gw;
        s2 += gw * h;
        dw[i][e] += d * h;
        db[i][e] += d;
      }
    const float m1 = row_sum<BLOCK>(s1, L, lds) * inv, m2 = row_sum<BLOCK>(s2, L, lds) * inv;
    if (!on) continue;
    T* dx = static_cast<T*>(a.y) + row_at(a, a.my, r);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V;
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (p[i].get(e) - mean) * rstd;
        v[e] = rstd * (g[i].get(e) * w[i][e] - m1 - h * m2);
      }
      Piece<T> o;
      o.set(v);
      o.store(dx + c, min(max(a.D - c, 0), V));
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (long long)blockIdx.x * 2 * a.D;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V;
    for (int k = 0; k < 2; ++k) {  // dw, then db
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = k ? db[i][e] : dw[i][e];
      if constexpr (!BLOCK) {
        // the wave's rows, then the four waves
#pragma unroll
        for (int e = 0; e < V; ++e)
          for (int m = L; m < 64; m <<= 1) v[e] += __shfl_xor(v[e], m, 64);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) part[threadIdx.x >> 6][threadIdx.x & 63][e] = v[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e)
          v[e] = part[0][threadIdx.x & 63][e] + part[1][threadIdx.x & 63][e] + part[2][threadIdx.x & 63][e] +
                 part[3][threadIdx.x & 63][e];
        if ((int)threadIdx.x >= L) continue;
      }
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (c + e < a.D) out[(long long)k * a.D + c + e] = v[e];
    }
  }
}

// dx of rows too long for registers: two passes over x and dy.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_bwd_long_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const float inv = 1.f / (float)a.D;
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row_at(a, a.mx, r);
    const T* dy = static_cast<const T*>(a.dy) + row_at(a, a.mdy, r);
    T* dx = static_cast<T*>(a.y) + row_at(a, a.my, r);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f, m1 = 0.f, m2 = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int c = threadIdx.x * V; c < a.D; c += kThreads * V) {
        const int n = min(a.D - c, V);
        Piece<T> p, g;
        p.load(x + c, n);
        g.load(dy + c, n);
        float w[V], v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = 1.f;
        if (a.w) load_weights<T>(a.w, a.w_f32, c, n, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (p.get(e) - mean) * rstd, gw = g.get(e) * w[e];
          s1 += gw;
          s2 += gw * h;
          v[e] = rstd * (gw - m1 - h * m2);
        }
        if (pass) {
          p.set(v);
          p.store(dx + c, n);
        }
      }
      if (!pass) {
        m1 = row_sum<true>(s1, 64, lds) * inv;
        m2 = row_sum<true>(s2, 64, lds) * inv;
      }
    }
  }
}

// Partial sums of dw and db for such rows: workgroup (column block, row run),
// a thread per column.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_bwd_columns_kernel(const NormArgs a) {
  const long long c = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.D) return;
  float dw = 0.f, db = 0.f;
  for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float x = (float)static_cast<const T*>(a.x)[row_at(a, a.mx, r) + c];
    const float d = (float)static_cast<const T*>(a.dy)[row_at(a, a.mdy, r) + c];
    dw += d * (x - a.mean[r]) * a.rstd[r];
    db += d;
  }
  float* out = a.partial + (long long)blockIdx.y * 2 * a.D;
  out[c] = dw;
  out[a.D + c] = db;
}

// dw and db from n partial rows: a workgroup takes 64 of the 2 D columns, its
// waves a quarter of the rows each, added in a fixed order.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_weights_kernel(const NormArgs a, int n) {
  __shared__ float part[4][64];
  debug_poison_lds(part);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long c = (long long)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < 2LL * a.D)
    for (int p = wave; p < n; p += 4) s += a.partial[(long long)p * 2 * a.D + c];
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= 2LL * a.D) return;
  s = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
  void* out = c < a.D ? a.dw : a.db;
  if (!out) return;
  const long long at = c < a.D ? c : c - a.D;
  if (a.w_f32) static_cast<float*>(out)[at] = s;
  else static_cast<T*>(out)[at] = (T)s;
}

// pieces of a row, lanes that share it, pieces per lane; lanes = 0: too long
struct Shape {
  int lanes, np;
};
Shape shape_of(int D, int V) {
  const int pieces = (D + V - 1) / V;
  if (pieces <= 256) {
    int L = 1;
    while (L < 64 && L < pieces) L *= 2;
    const int np = (pieces + L - 1) / L;
    return {L, np <= 2 ? np : 4};
  }
  const int np = (pieces + kThreads - 1) / kThreads;
  if (np > 8) return {0, 0};
  return {kThreads, np <= 2 ? np : np <= 4 ? 4 : 8};
}

template <typename T, int NP, bool BLOCK, bool FWD>
void go(const NormArgs& a, int grid) {
  if constexpr (FWD) norm_fwd_kernel<T, NP, BLOCK><<<grid, kThreads, 0, a.stream>>>(a);
  else norm_bwd_kernel<T, NP, BLOCK><<<grid, kThreads, 0, a.stream>>>(a);
}

template <typename T, bool FWD>
hipError_t go_shape(const NormArgs& a, const Shape& s, int grid) {
  if (s.lanes <= 64) {
    if (s.np == 1) go<T, 1, false, FWD>(a, grid);
    else if (s.np == 2) go<T, 2, false, FWD>(a, grid);
    else go<T, 4, false, FWD>(a, grid);
  } else {
    if (s.np == 2) go<T, 2, true, FWD>(a, grid);
    else if (s.np == 4) go<T, 4, true, FWD>(a, grid);
    else go<T, 8, true, FWD>(a, grid);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t fwd_t(NormArgs a) {
  const Shape s = shape_of(a.D, Piece<T>::V);
  if (s.lanes == 0) {
    norm_fwd_long_kernel<T><<<min(a.rows, 2048), kThreads, 0, a.stream>>>(a);
    return hipGetLastError();
  }
  a.lanes = s.lanes;
  const int per = kThreads / s.lanes;
  return go_shape<T, true>(a, s, min((a.rows + per - 1) / per, 2048));
}

template <typename T>
hipError_t bwd_t(NormArgs a) {
  const Shape s = shape_of(a.D, Piece<T>::V);
  const int n = norm_partials(a.rows, a.D, (int)sizeof(T));
  hipError_t err;
  if (s.lanes == 0) {
    norm_bwd_long_kernel<T><<<min(a.rows, 2048), kThreads, 0, a.stream>>>(a);
    if ((err = hipGetLastError()) != hipSuccess || !a.partial) return err;
    norm_bwd_columns_kernel<T><<<dim3((a.D + kThreads - 1) / kThreads, n), kThreads, 0, a.stream>>>(a);
    err = hipGetLastError();
  } else {
    a.lanes = s.lanes;
    err = go_shape<T, false>(a, s, n);
  }
  if (err != hipSuccess || !a.partial) return err;
  norm_weights_kernel<T><<<(int)((2LL * a.D + 63) / 64), kThreads, 0, a.stream>>>(a, n);
  return hipGetLastError();
}

}  // namespace

int norm_partials(int rows, int D, int elem_bytes) {
  const Shape s = shape_of(D, 16 / elem_bytes);
  const int groups = s.lanes == 0 ? rows : (rows + kThreads / s.lanes - 1) / (kThreads / s.lanes);
  const int most = s.lanes == 0 ? 64 : 1024;
  return groups < most ? groups : most;
}

hipError_t launch_norm_fwd(const NormArgs& a) {
  switch (a.type) {
    case kBf16: return fwd_t<__bf16>(a);
    case kFp16: return fwd_t<_Float16>(a);
    default: return fwd_t<float>(a);
  }
}

hipError_t launch_norm_bwd(const NormArgs& a) {
  switch (a.type) {
    case kBf16: return bwd_t<__bf16>(a);
    case kFp16: return bwd_t<_Float16>(a);
    default: return bwd_t<float>(a);
  }
}

}  // namespace vitattn
