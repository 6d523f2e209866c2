// Dropout of rows of D elements, y = [residual +] m x with m = 0 or 1 / (1 - p) from
// the counter of vitattn_random.h: no mask is stored, the gradient of x is the same
// call on dy. Any strides; the sum is fp32 and rounded once, to the residual's type.
//
// Bound by HBM, or by the generator's 20 32 x 32 -> 64 bit products for every
// eight elements. A thread takes eight columns of a row, several of them in turn,
// neighbours side by side; a row's index and column come from one division of the
// workgroup's first piece (64 bits, uniform) and one of a thread's small offset
// (by a reciprocal that the host made). 4 x 8,192 rows of 4,096 bf16: 104 us, 5.2 TB/s
// (a copy reaches 5.10); 16 x 20,001 rows of 72 fp32 read sequence-major, with a
// residual: 55 us, 5.0 TB/s, and 35 without. An fp32 gradient is rounded to a 16-bit branch's
// type as it is stored: 4 x 8,192 rows of 4,096 to bf16 156 us, 5.15 TB/s (337 with a cast behind).
#include "vitattn_random.h"

namespace vitattn {

namespace {

constexpr int kDropThreads = 256;
constexpr int kDropPieces = 4;  // of a thread

template <typename T, typename R, bool ADD>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const DropoutArgs a) {
  const Dropout drop(a.drop);
  const long long first = (long long)blockIdx.x * (kDropThreads * kDropPieces);
  const long long row0 = first / a.pieces;
  const uint32_t col0 = (uint32_t)(first - row0 * a.pieces);
  Span<T, 8> x[kDropPieces];
  Span<R, 8> r[kDropPieces];
  long long at_y[kDropPieces];
  uint32_t eighth[kDropPieces], logical[kDropPieces];
  int n[kDropPieces];  // columns of the piece that are there
#pragma unroll
  for (int u = 0; u < kDropPieces; ++u) {
    const uint32_t k = col0 + u * kDropThreads + threadIdx.x;  // below 2^32: pieces < 2^28
    const uint32_t rows = a.pieces == 1 ? k : (uint32_t)(((uint64_t)k * a.recip) >> 32 >> a.shift);
    const long long row = row0 + rows;
    eighth[u] = k - rows * (uint32_t)a.pieces;
    n[u] = 0;
    if (row >= a.rows) continue;
    const int i2r = (int)row;
    const int t = a.n2 == a.rows ? 0 : i2r / a.n2, i2 = i2r - t * a.n2, i0 = t / a.n1, i1 = t - i0 * a.n1;
    const int c = (int)eighth[u] * 8;
    n[u] = min(a.D - c, 8);
    logical[u] = (uint32_t)a.ml.at(i0, i1, i2);
    x[u].load(static_cast<const T*>(a.x) + a.mx.at(i0, i1, i2), c, a.D);
    if constexpr (ADD) r[u].load(static_cast<const R*>(a.residual) + a.mr.at(i0, i1, i2), c, a.D);
    at_y[u] = a.my.at(i0, i1, i2) + c;
  }
#pragma unroll
  for (int u = 0; u < kDropPieces; ++u) {
    if (n[u] == 0) continue;
    x[u].settle((int)eighth[u] * 8, a.D, true);
    if constexpr (ADD) r[u].settle((int)eighth[u] * 8, a.D, true);
    const u32x4 w = drop.words(eighth[u], logical[u]);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = drop.add<R>(w, e, x[u].get(e), ADD ? r[u].get(e) : 0.f);
    Span<R, 8> o;
    o.set(y);
    o.store(static_cast<R*>(a.y) + at_y[u], n[u]);
  }
}

template <typename T, typename R>
hipError_t go(DropoutArgs a) {
  // k / pieces of k < 2^29 by a product: recip = ceil(2^(32 + shift) / pieces), the
  // shift one less than pieces' bits, errs by less than k 2^-(32 + shift) < 1 / pieces
  a.shift = 0;
  while ((2LL << a.shift) < a.pieces) ++a.shift;
  a.recip = (uint32_t)(((1ULL << (32 + a.shift)) + a.pieces - 1) / a.pieces);
  const long long per = kDropThreads * kDropPieces, blocks = ((long long)a.rows * a.pieces + per - 1) / per;
  if constexpr (sizeof(R) >= sizeof(T))
    if (a.residual) {
      dropout_kernel<T, R, true><<<(unsigned)blocks, kDropThreads, 0, a.stream>>>(a);
      return hipGetLastError();
    }
  dropout_kernel<T, R, false><<<(unsigned)blocks, kDropThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a) {
  switch (a.type) {
    case kBf16: return a.residual_type == kFp32 ? go<__bf16, float>(a) : go<__bf16, __bf16>(a);
    case kFp16: return a.residual_type == kFp32 ? go<_Float16, float>(a) : go<_Float16, _Float16>(a);
    default:
      return a.residual_type == kBf16 ? go<float, __bf16>(a) : a.residual_type == kFp16 ? go<float, _Float16>(a) : go<float, float>(a);
  }
}

}  // namespace vitattn
