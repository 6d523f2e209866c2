// Layer norm of rows of D elements, forward and backward:
//
//   mu = mean x,  r = 1/sqrt(mean (x - mu)^2 + eps),  h = (x - mu) r,  y = h w + b
//   g = dy w,  dx = r (g - mean g - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
//
// Bound by HBM: the forward reads x and writes y, the backward reads x and dy
// and writes dx, so a row is read once and kept in registers: the mean, then
// the sum of squared deviations from it (no cancellation of large squares). A
// mean is off by the roundings of its sum, which matters where a row's spread is
// small beside it (constant rows): from a quarter on (is_far) the deviations'
// own mean corrects it, and the squares are summed again about the corrected one. (32,768
// rows of 1,024 bf16 forward 26 us, about a mean of 100 sigma 35; the wave or
// workgroup whose rows are none such skips it.)
// Statistics, products and sums are fp32 (a lane's sums over a row too long for
// registers, up to 65,536 values, fp64); x, y, dy and dx are rounded once, to
// their type.
//
// L lanes share a row, each holding NP pieces of 16 bytes (pieces lane, lane +
// L, ..): L of a wave's 64 lanes for short rows, 64 / L rows per wave, and the
// four waves of a workgroup for long ones. Rows too long for registers (over
// 256 * 8 pieces) are read once per pass instead, from L2.
//
// Measured (a large copy reaches 5.1 TB/s): 32,768 rows of 1,024 bf16 forward
// 26 us (134 MB, 5.1 TB/s), backward 42 us (201 MB, 4.8 TB/s) and its sums of
// partials 4; 3,125,000 rows of 64 bf16 171 and 239 us (4.7 and 5.0 TB/s); 3,062
// rows of 5,001 fp32 27 and 39 us (4.5 and 4.7 TB/s); one row of 768 5.5 us,
// nearly all of it the launch. Too long for registers: 67 million bf16 elements in
// rows of 16,392 167 us forward, 491 backward (268 and 402 MB, 1.6 and 0.8 TB/s), in
// rows of 2^24, a workgroup each, 13.5 and 17.2 ms.
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
  const int t = a.n2 == a.rows ? 0 : r / a.n2;
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
      per = rpw * (kThreads / 64);
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

// A mean that a row's spread (var about it) is small beside. Below this bound the
// mean's error of n 2^-24 |mean|, n the length of a lane's sum and the lanes' tree,
// is at most 4 n 2^-24 of a standard deviation. (Infinite and NaN ones are far.)
__device__ __forceinline__ bool is_far(float mean, float var) { return mean != 0.f && !(mean * mean < 16.f * var); }
// variance from the mean of squares q and of deviations c (NaN stays NaN)
__device__ __forceinline__ float var_of(float q, float c) {
  const float v = q - c * c;
  return v < 0.f ? 0.f : v;
}

// A row's pieces in this lane's registers.
template <typename T, int NP>
struct RowRegs {
  Piece<T> p[NP];
  __device__ __forceinline__ void load(const T* x, int lane, int L, int D, bool on) {
    constexpr int V = Piece<T>::V;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * L) * V;
      p[i].load(x + c, on ? min(max(D - c, 0), V) : 0);
    }
  }
};

// Rows of a lane in flight together: short rows give it one or two pieces each.
constexpr int rows_at_once(int np) { return np == 1 ? 4 : np == 2 ? 2 : 1; }

// The backward holds the next long row as well where there are registers for it.
constexpr bool row_ahead(int np, int v) { return np * v <= 32; }

template <typename T, int NP, bool BLOCK>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  constexpr int U = BLOCK ? 1 : rows_at_once(NP);
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const Place<BLOCK> at(a.lanes);
  const int L = at.L, lane = at.lane, per = at.per;  // rows of a workgroup at a time, U times
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
  auto load = [&](RowRegs<T, NP>& x, int r) __attribute__((always_inline)) {
    const bool on = at.row >= 0 && r < a.rows;
    x.load(static_cast<const T*>(a.x) + (on ? row_at(a, a.mx, r) : 0), lane, L, a.D, on);
  };
  RowRegs<T, NP> x[U], next;
  const int step = gridDim.x * per * U;
  int r0 = blockIdx.x * per * U + at.row;
  if (BLOCK && r0 < a.rows) load(next, r0);
  for (; r0 - at.row < a.rows; r0 += step) {
    if constexpr (BLOCK) {
      x[0] = next;
      if (r0 + step < a.rows) load(next, r0 + step);  // on its way through this row's sums
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) load(x[u], r0 + u * per);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * per;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) s += x[u].p[i].get(e);
      float mean = at.sum(s, lds) * inv;
      // this lane's sums of the deviations from m and of their squares
      auto deviations = [&](float m, float& c, float& q) __attribute__((always_inline)) {
        c = q = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int n = a.D - (lane + i * L) * V;
          if (n >= V) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float d = x[u].p[i].get(e) - m;
              c += d;
              q = __builtin_fmaf(d, d, q);
            }
          } else if (n > 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float d = e < n ? x[u].p[i].get(e) - m : 0.f;
              c += d;
              q = __builtin_fmaf(d, d, q);
            }
          }
        }
      };
      float c, q;
      deviations(mean, c, q);
      q = at.sum(q, lds);
      float rstd = rsqrtf(__builtin_fmaf(q, inv, a.eps));
      const bool far = is_far(mean, q * inv);
      if (__builtin_expect(at.any(far), 0)) {
        deviations(mean, c, q);
        const float m = mean + at.sum(c, lds) * inv;
        deviations(m, c, q);
        c = at.sum(c, lds) * inv;
        q = at.sum(q, lds) * inv;
        if (far) {
          mean = m;
          rstd = rsqrtf(var_of(q, c) + a.eps);
        }
      }
      if (at.row < 0 || r >= a.rows) continue;
      T* y = static_cast<T*>(a.y) + row_at(a, a.my, r);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (lane + i * L) * V;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf((x[u].p[i].get(e) - mean) * rstd, w[i][e], b[i][e]);
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
}

// Rows too long for registers: three passes over the row (four about a far mean).
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_fwd_long_kernel(const NormArgs a) {
  constexpr int V = Piece<T>::V;
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const float inv = 1.f / (float)a.D;
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row_at(a, a.mx, r);
    T* y = static_cast<T*>(a.y) + row_at(a, a.my, r);
    const Place<true> at(kThreads);
    double s = 0.;
    for (int c = threadIdx.x * V; c < a.D; c += kThreads * V) {
      Piece<T> p;
      p.load(x + c, min(a.D - c, V));
#pragma unroll
      for (int e = 0; e < V; ++e) s += p.get(e);
    }
    float mean = at.sum((float)s, lds) * inv, c, q;
    auto about_mean = [&]() {  // mean deviation from, and sum of squares about, `mean`
      double sd = 0., sq = 0.;
      for (int k = threadIdx.x * V; k < a.D; k += kThreads * V) {
        Piece<T> p;
        p.load(x + k, min(a.D - k, V));
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = e < a.D - k ? p.get(e) - mean : 0.f;
          sd += d;
          sq += (double)d * d;
        }
      }
      c = at.sum((float)sd, lds) * inv;
      q = at.sum((float)sq, lds);
    };
    about_mean();
    float rstd = rsqrtf(__builtin_fmaf(q, inv, a.eps));
    if (is_far(mean, q * inv)) {
      mean += c;
      about_mean();
      rstd = rsqrtf(var_of(q * inv, c) + a.eps);
    }
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
  constexpr int U = 1;  // (more rows at once leave too few registers)
  constexpr bool AHEAD = BLOCK && row_ahead(NP, V);
  __shared__ float lds[4];
  __shared__ float part[BLOCK ? 1 : kThreads][V];
  debug_poison_lds(lds, part);
  const Place<BLOCK> at(a.lanes);
  const int L = at.L, lane = at.lane, per = at.per;
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
  struct Row {
    RowRegs<T, NP> x, g;
    float mean, rstd;
  };
  auto load = [&](Row& w_, int r) __attribute__((always_inline)) {
    const bool on = at.row >= 0 && r < a.rows;
    w_.x.load(static_cast<const T*>(a.x) + (on ? row_at(a, a.mx, r) : 0), lane, L, a.D, on);
    w_.g.load(static_cast<const T*>(a.dy) + (on ? row_at(a, a.mdy, r) : 0), lane, L, a.D, on);
    w_.mean = on ? a.mean[r] : 0.f;
    w_.rstd = on ? a.rstd[r] : 0.f;
  };
  Row row[U], next;
  const int step = gridDim.x * per * U;
  int r0 = blockIdx.x * per * U + at.row;
  if (AHEAD && r0 < a.rows) load(next, r0);
  for (; r0 - at.row < a.rows; r0 += step) {
    if constexpr (AHEAD) {
      row[0] = next;
      if (r0 + step < a.rows) load(next, r0 + step);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) load(row[u], r0 + u * per);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * per;
      const float mean = row[u].mean, rstd = row[u].rstd;
      // lanes past the row hold dy = 0 and add nothing to any sum
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = row[u].g.p[i].get(e), h = (row[u].x.p[i].get(e) - mean) * rstd, gw = d * w[i][e];
          s1 += gw;
          s2 = __builtin_fmaf(gw, h, s2);
          dw[i][e] = __builtin_fmaf(d, h, dw[i][e]);
          db[i][e] += d;
        }
      const float m1 = -at.sum(s1, lds) * inv * rstd, m2 = -at.sum(s2, lds) * inv * rstd;
      if (at.row < 0 || r >= a.rows) continue;
      T* dx = static_cast<T*>(a.y) + row_at(a, a.my, r);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (lane + i * L) * V;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (row[u].x.p[i].get(e) - mean) * rstd;
          v[e] = __builtin_fmaf(row[u].g.p[i].get(e) * w[i][e], rstd, __builtin_fmaf(h, m2, m1));
        }
        Piece<T> o;
        o.set(v);
        o.store(dx + c, min(max(a.D - c, 0), V));
      }
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
    double s1 = 0., s2 = 0.;
    float m1 = 0.f, m2 = 0.f;
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
          s2 += (double)gw * h;
          v[e] = rstd * (gw - m1 - h * m2);
        }
        if (pass) {
          p.set(v);
          p.store(dx + c, n);
        }
      }
      if (!pass) {
        m1 = Place<true>(kThreads).sum((float)s1, lds) * inv;
        m2 = Place<true>(kThreads).sum((float)s2, lds) * inv;
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

// dw and db from n partial rows: a workgroup takes 64 of the 2 D columns, its 16
// waves every 16th row each, eight loads in flight, added in a fixed order.
constexpr int kWeightWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kWeightWaves) void norm_weights_kernel(const NormArgs a, int n) {
  __shared__ float part[kWeightWaves][64];
  debug_poison_lds(part);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long c = (long long)blockIdx.x * 64 + lane, width = 2LL * a.D;
  float s = 0.f;
  if (c < width) {
    const float* src = a.partial + c;
    int p = wave;
    for (; p + 7 * kWeightWaves < n; p += 8 * kWeightWaves) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = src[(p + u * kWeightWaves) * width];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
    for (; p < n; p += kWeightWaves) s += src[p * width];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= width) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kWeightWaves; ++w) s += part[w][lane];
  void* out = c < a.D ? a.dw : a.db;
  if (!out) return;
  const long long at = c < a.D ? c : c - a.D;
  if (a.w_f32) static_cast<float*>(out)[at] = s;
  else static_cast<T*>(out)[at] = (T)s;
}

// Lanes that share a row and pieces per lane (lanes = 0: too long for registers).
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
struct Shape {
  int lanes, np;
};
Shape shape_of(int D, int V, bool fwd) {
  const int pieces = (D + V - 1) / V;
  if (pieces > 256) {
    const int np = (pieces + kThreads - 1) / kThreads;
    return np > 8 ? Shape{0, 0} : Shape{kThreads, np == 7 ? 8 : np};
  }
  if (pieces < (fwd ? 4 : 16)) return {pieces, 1};
  if (pieces < 16) return {(pieces + 1) / 2, 2};
  Shape best = {(pieces + 3) / 4, 4};
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

// Workgroups of the backward that a CU holds, from the registers of a lane:
// five fp32 values per element (w, dw, db and the row's h and g), the rows as
// they are and about 48 more, at most four. The grid is this many for each of
// 256 CUs: one round, so that no workgroup waits for others to end (with the sums of
// dw and db, two, three, four and five per CU: 320,016 rows of 72 bf16 47, 39, 37 and
// 37 us, 32,768 of 1,024 47, 43, 52 and 54, 100,000 of 384 53, 67, 62 and 69).
// The number is the sizes' alone: dw and db do not depend on the device.
constexpr int bwd_resident(int np, int v, bool block) {
  const int regs = 5 * np * v + (block && row_ahead(np, v) ? 16 : 8) * np + 48;
  return regs <= 128 ? 4 : regs <= 170 ? 3 : regs <= 270 ? 2 : 1;
}

// Rows of a workgroup at a time.
int rows_of(const Shape& s, bool fwd) {
  return s.lanes > 64 ? 1 : 64 / s.lanes * (kThreads / 64) * (fwd ? rows_at_once(s.np) : 1);
}
int groups_of(const Shape& s, int rows, bool fwd) {
  return (int)(((long long)rows + rows_of(s, fwd) - 1) / rows_of(s, fwd));
}

// The forward's grid is what the device holds at once (its rows do not depend on it).
template <typename T, int NP, bool BLOCK>
hipError_t go_fwd(const NormArgs& a, int groups) {
  static ResidentCache cache;
  const int most = cache.get(reinterpret_cast<const void*>(norm_fwd_kernel<T, NP, BLOCK>), kThreads).workgroups;
  norm_fwd_kernel<T, NP, BLOCK><<<min(groups, most > 0 ? most : 1024), kThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <typename T, int NP, bool BLOCK>
hipError_t go_bwd(const NormArgs& a, int grid) {
  norm_bwd_kernel<T, NP, BLOCK><<<grid, kThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

template <typename T, bool FWD, int NP, bool BLOCK>
hipError_t go(const NormArgs& a, int n) {
  if constexpr (FWD) return go_fwd<T, NP, BLOCK>(a, n);
  else return go_bwd<T, NP, BLOCK>(a, n);
}

template <typename T, bool FWD>
hipError_t go_shape(const NormArgs& a, const Shape& s, int n) {
  const bool block = s.lanes > 64;
  switch (s.np) {
    case 1: return go<T, FWD, 1, false>(a, n);  // (long rows have two pieces per lane or more)
    case 2: return block ? go<T, FWD, 2, true>(a, n) : go<T, FWD, 2, false>(a, n);
    case 3: return block ? go<T, FWD, 3, true>(a, n) : go<T, FWD, 3, false>(a, n);
    case 4: return block ? go<T, FWD, 4, true>(a, n) : go<T, FWD, 4, false>(a, n);
    case 5: return go<T, FWD, 5, true>(a, n);
    case 6: return go<T, FWD, 6, true>(a, n);
    default: return go<T, FWD, 8, true>(a, n);
  }
}

template <typename T>
hipError_t fwd_t(NormArgs a) {
  const Shape s = shape_of(a.D, Piece<T>::V, true);
  if (s.lanes == 0) {
    norm_fwd_long_kernel<T><<<min(a.rows, 2048), kThreads, 0, a.stream>>>(a);
    return hipGetLastError();
  }
  a.lanes = s.lanes;
  return go_shape<T, true>(a, s, groups_of(s, a.rows, true));
}

template <typename T>
hipError_t bwd_t(NormArgs a) {
  const Shape s = shape_of(a.D, Piece<T>::V, false);
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
  norm_weights_kernel<T><<<(int)((2LL * a.D + 63) / 64), 64 * kWeightWaves, 0, a.stream>>>(a, n);
  return hipGetLastError();
}

}  // namespace

int norm_partials(int rows, int D, int elem_bytes) {
  const Shape s = shape_of(D, 16 / elem_bytes, false);
  if (s.lanes == 0) return rows < 64 ? rows : 64;
  return min(groups_of(s, rows, false), 256 * bwd_resident(s.np, 16 / elem_bytes, s.lanes > 64));
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
