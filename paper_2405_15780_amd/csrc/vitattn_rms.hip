// Root-mean-square norm with the residual's addition, forward:
//
//   h = residual + m x (rounded to the residual's type),  r = 1/sqrt(mean h^2 + eps),
//   y = h r w
//
// with m = 0 or 1/(1 - p), dropout's mask of vitattn_random.h (1 without dropout).
// Without a residual h is x. What is normalised is h as it is stored: the backward
// reads that, and the call gives the bits of the addition and the norm one after the
// other. The output is of x's type, or e4m3 with fp32 scales of a row or of groups of
// its columns: s = max(max |y| / 448, 2^-126) of the fp32 y, and y / s rounded once, to the
// nearest even.
//
// Bound by HBM: x and the residual are read once and h and y written once; a row stays
// in registers, in the residual's type, from the sum of squares to the output. Sums
// and r are fp32. L lanes share a row as in vitattn_norm.hip; for groups of columns L
// is rounded up so that a group's lanes are neighbours and its maximum a few
// exchanges. 32,768 rows of 1,024 bf16 with residual and dropout: 53 us, 5.05 TB/s;
// 32,768 of 2,048 to e4m3 with scales of 128 columns: 109 us, 4.3 TB/s.
#include "vitattn_rms.h"

namespace vitattn {

namespace {

constexpr int kThreads = kRowThreads;
constexpr float kE4M3Max = 448.f, kLeastScale = 0x1p-126f;

// Rows of a lane in flight together, as for layer norm but with two operands.
constexpr int rows_at_once(int np) { return np == 1 ? 2 : 1; }

// Largest over the row's lanes (BLOCK: the workgroup), the same in all.
template <bool BLOCK>
__device__ __forceinline__ float row_max(const Place<BLOCK>& at, float x, float* lds) {
  if (BLOCK || (at.L & (at.L - 1)) == 0) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
      if (BLOCK || m < at.L) x = fmaxf(x, __shfl_xor(x, m, 64));
  } else {
    const int me = threadIdx.x & 63;
    for (int m = 32; m >= 1; m >>= 1) {
      if (m >= at.L) continue;
      const float y = __shfl(x, (me + m) & 63, 64);
      x = at.lane + m < at.L ? fmaxf(x, y) : x;
    }
    x = __shfl(x, me - at.lane, 64);
  }
  if constexpr (BLOCK) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  }
  return x;
}

// V values as e4m3 bytes
template <int V>
__device__ __forceinline__ void to_e4m3(const float (&v)[V], uint32_t (&w)[V / 4]) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], x, true);
  }
}

// The bytes of y / s, rounded once. Products with a reciprocal that is 2^-21 too small and one
// that is too large (rcp is within 2^-23, the products' roundings are 2^-24) lie on both sides
// of the quotient: where they give the same bytes, so does it. Where they do not it is near the
// middle between two bytes, and goes to fp32 with its last bit set if it is not exact
// (rounded to odd), so that the rounding to e4m3 is the only one. The residuals
// fma(-q, s, |y|) are exact (q is within two fp32 steps, scales below 2^-64 are taken 2^96
// times), their sign is the quotient's place beside q. 2 x 16,384 rows of 2,048 bf16 (groups of
// 128, one element in 2,500 near a middle): 109 us; 116 with every quotient rounded to odd, and
// 103 for a product with the reciprocal, which beside a middle falls on either side of it.
template <int V>
__device__ __forceinline__ void quotient_bytes(const float (&y)[V], float scale, uint32_t (&w)[V / 4]) {
  const float back = __builtin_amdgcn_rcpf(scale), less = __builtin_fmaf(back, -0x1p-21f, back), more = __builtin_fmaf(back, 0x1p-21f, back);
  float v[V];
  uint32_t other[V / 4];
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = y[e] * less;
  to_e4m3<V>(v, w);
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = y[e] * more;
  to_e4m3<V>(v, other);
  uint32_t differ = 0;
#pragma unroll
  for (int i = 0; i < V / 4; ++i) differ |= w[i] ^ other[i];
  if (differ == 0) return;
  const float up = scale < 0x1p-64f ? 0x1p96f : 1.f, s = scale * up, inv = __builtin_amdgcn_rcpf(s);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float x = fabsf(y[e]) * up;
    float q = x * inv;
    q = __builtin_fmaf(__builtin_fmaf(-q, s, x), inv, q);
    const float r = __builtin_fmaf(-q, s, x);
    const int odd = (__float_as_int(q) + (__float_as_int(r) >> 31)) | 1;
    v[e] = copysignf(r < 0.f || r > 0.f ? __int_as_float(odd) : q, y[e]);
  }
  to_e4m3<V>(v, w);
}

// V bytes, n of them stored
template <int V>
__device__ __forceinline__ void store_bytes(uint8_t* p, const uint32_t (&w)[V / 4], int n) {
  typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(1)));
  if (n >= V) {
    words o;
    if constexpr (V == 8) o = words{w[0], w[1]};
    else o = words{w[0]};
    *reinterpret_cast<words*>(p) = o;
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
}

template <typename T, typename R, int NP, bool BLOCK>
__global__ __launch_bounds__(kThreads) void rms_fwd_kernel(const RmsArgs a) {
  constexpr int V = Piece<T>::V;
  constexpr int U = BLOCK ? 1 : rows_at_once(NP);
  __shared__ float lds[4];
  debug_poison_lds(lds);
  const Place<BLOCK> at(a.lanes);
  const int L = at.L, lane = at.lane, per = at.per;
  const Dropout drop(a.drop);
  float w[NP][V];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * L) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) w[i][e] = 1.f;
    if (a.w) load_weights<T>(a.w, a.w_f32, c, columns_of<V>(a.D, c), w[i]);
  }
  const float inv = 1.f / (float)a.D;
  struct Row {
    Span<T, V> x[NP];
    Span<R, V> h[NP];
  };
  auto load = [&](Row& row, int r) __attribute__((always_inline)) {
    const bool on = at.row >= 0 && r < a.rows;
    const RowAt i(a, on ? r : 0);
    const T* x = static_cast<const T*>(a.x) + i.in(a.mx);
    const R* res = static_cast<const R*>(a.residual) + (a.residual ? i.in(a.mr) : 0);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = (lane + k * L) * V;
      row.x[k].load(x, c, a.D);
      if (a.residual) row.h[k].load(res, c, a.D);
      else row.h[k].clear();
    }
  };
  Row row[U], next;
  const int step = gridDim.x * per * U;
  int r0 = blockIdx.x * per * U + at.row;
  if (BLOCK && r0 < a.rows) load(next, r0);
  for (; r0 - at.row < a.rows; r0 += step) {
    if constexpr (BLOCK) {
      row[0] = next;
      if (r0 + step < a.rows) load(next, r0 + step);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) load(row[u], r0 + u * per);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * per;
      const bool on = at.row >= 0 && r < a.rows;
      const RowAt ix(a, on ? r : 0);
      const long long logical = ix.in(a.ml);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        float v[V];
        row[u].x[i].settle((lane + i * L) * V, a.D, on);
        if (a.residual) row[u].h[i].settle((lane + i * L) * V, a.D, on);
        if (a.drop_on) {
          const PieceMask<V> mask(drop, (lane + i * L) * V, (uint32_t)logical);
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = mask.template add<R>(drop, e, row[u].x[i].get(e), row[u].h[i].get(e));
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = row[u].x[i].get(e) + row[u].h[i].get(e);
        }
        row[u].h[i].set(v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = row[u].h[i].get(e);
          s = __builtin_fmaf(h, h, s);
        }
      }
      const float rstd = rsqrtf(__builtin_fmaf(at.sum(s, lds), inv, a.eps));
      if (on && a.residual) {
        R* h = static_cast<R*>(a.h) + ix.in(a.mh);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = (lane + i * L) * V;
          row[u].h[i].store(h + c, columns_of<V>(a.D, c));
        }
      }
      if (on && lane == 0 && a.rstd) a.rstd[logical] = rstd;
      if (!a.scale) {
        if (!on) continue;
        T* y = static_cast<T*>(a.y) + ix.in(a.my);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = (lane + i * L) * V;
          float v[V];
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = row[u].h[i].get(e) * rstd * w[i][e];
          Span<T, V> o;
          o.set(v);
          o.store(y + c, columns_of<V>(a.D, c));
        }
        continue;
      }
      // every lane of the row stays for the exchanges
      float top[NP], most = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        top[i] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) top[i] = fmaxf(top[i], fabsf(row[u].h[i].get(e) * rstd * w[i][e]));
        most = fmaxf(most, top[i]);
      }
      const int gl = a.group / V;  // lanes of a group
      if (a.group) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
          for (int m = gl >> 1; m >= 1; m >>= 1) top[i] = fmaxf(top[i], __shfl_xor(top[i], m, 64));
      } else {
        most = row_max(at, most, lds);
#pragma unroll
        for (int i = 0; i < NP; ++i) top[i] = most;
      }
      if (!on) continue;
      uint8_t* y = static_cast<uint8_t*>(a.y) + ix.in(a.my);
      const int groups = a.group ? (a.D + a.group - 1) / a.group : 1;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (lane + i * L) * V, n = columns_of<V>(a.D, c);
        const float scale = fmaxf(top[i] / kE4M3Max, kLeastScale);
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = row[u].h[i].get(e) * rstd * w[i][e];
        uint32_t bytes[V / 4];
        quotient_bytes<V>(v, scale, bytes);
        store_bytes<V>(y + c, bytes, n);
        if (a.group ? n > 0 && lane % gl == 0 : i == 0 && lane == 0)
          a.scale[logical * groups + (a.group ? c / a.group : 0)] = scale;
      }
    }
  }
}

// Rows of a workgroup at a time.
int rows_of(const RowShape& s) { return s.lanes > 64 ? 1 : 64 / s.lanes * (kThreads / 64) * rows_at_once(s.np); }

template <typename T, typename R, int NP, bool BLOCK>
hipError_t go(const RmsArgs& a, int groups) {
  static ResidentCache cache;
  const int most = cache.get(reinterpret_cast<const void*>(rms_fwd_kernel<T, R, NP, BLOCK>), kThreads).workgroups;
  rms_fwd_kernel<T, R, NP, BLOCK><<<min(groups, most > 0 ? most : 1024), kThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

template <typename T, typename R>
hipError_t fwd_t(RmsArgs a) {
  constexpr int V = Piece<T>::V;
  RowShape s = rms_shape(a.D, V, true, sizeof(R) > sizeof(T));
  if (a.group && s.lanes <= 64) {  // (divides 64)
    const int gl = a.group / V;
    s.lanes = (s.lanes + gl - 1) / gl * gl;
  }
  a.lanes = s.lanes;
  const int n = (int)(((long long)a.rows + rows_of(s) - 1) / rows_of(s));
  const bool block = s.lanes > 64;
  switch (s.np) {
    case 1: return block ? go<T, R, 1, true>(a, n) : go<T, R, 1, false>(a, n);
    case 2: return block ? go<T, R, 2, true>(a, n) : go<T, R, 2, false>(a, n);
    case 3: return block || sizeof(R) > sizeof(T) ? go<T, R, 3, true>(a, n) : go<T, R, 3, sizeof(R) != sizeof(T)>(a, n);
    case 4: return block || sizeof(R) > sizeof(T) ? go<T, R, 4, true>(a, n) : go<T, R, 4, sizeof(R) != sizeof(T)>(a, n);
    case 5:
    case 6: return go<T, R, 6, true>(a, n);
    default: return go<T, R, 8, true>(a, n);
  }
}

}  // namespace

hipError_t launch_rms_fwd(const RmsArgs& a) {
  switch (a.type) {
    case kBf16: return a.residual_type == kFp32 ? fwd_t<__bf16, float>(a) : fwd_t<__bf16, __bf16>(a);
    case kFp16: return a.residual_type == kFp32 ? fwd_t<_Float16, float>(a) : fwd_t<_Float16, _Float16>(a);
    default: return fwd_t<float, float>(a);
  }
}

}  // namespace vitattn
