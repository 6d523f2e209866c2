// Argument checks shared by the C entry points. They make no HIP call.
#pragma once

#include <math.h>
#include <stdint.h>

#include "../../include/vitattn.h"
#include "vitattn_launch.h"

namespace vitattn_check {

inline bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool scale_ok(float s) { return isfinite(s) && s > 0.f; }

// a dispatch's grid size in work-items is 32-bit
constexpr long long kMaxWorkItems = 1LL << 32;

// One operand's strides (elements). Rows must be 16-byte aligned and must not
// overlap (row >= d); every stride is non-negative and a multiple of
// 16 / elem_bytes elements. Operands read through buffer resources (the bf16
// inputs) must keep (N + 256) rows within 31-bit byte offsets. An output must
// not overlap itself: sorted by stride, each dimension must step past the
// span of the smaller ones. Inputs may repeat heads or batches (stride 0).
inline int check_map(const vitattn_strides& m, int B, int H, int N, int d, int elem_bytes, bool output) {
  const long long unit = 16 / elem_bytes;
  if (m.batch < 0 || m.head < 0 || m.row < d) return VITATTN_E_INVAL;
  if (m.batch % unit != 0 || m.head % unit != 0 || m.row % unit != 0) return VITATTN_E_INVAL;
  if (m.row > 0x7fffffffLL) return VITATTN_E_INVAL;
  if (elem_bytes == 2 && (long long)(N + 256) * m.row * 2 > 0x7fffffffLL) return VITATTN_E_INVAL;
  // the largest element offset must fit comfortably in 64 bits
  if ((double)(B - 1) * m.batch + (double)(H - 1) * m.head + (double)N * m.row > 4.0e18) return VITATTN_E_INVAL;
  if (output) {
    long long size[3] = {B, H, N}, stride[3] = {m.batch, m.head, m.row};
    int idx[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)  // sort the three dimensions by stride
      for (int j = i + 1; j < 3; ++j)
        if (stride[idx[j]] < stride[idx[i]]) {
          const int t = idx[i];
          idx[i] = idx[j];
          idx[j] = t;
        }
    long long span = d;  // elements covered by the dimensions taken so far (a row first)
    for (int i = 0; i < 3; ++i) {
      const int x = idx[i];
      if (size[x] == 1) continue;
      if (stride[x] < span) return VITATTN_E_INVAL;
      span += (size[x] - 1) * stride[x];
    }
  }
  return VITATTN_OK;
}

inline vitattn::Map to_map(const vitattn_strides& m) { return vitattn::Map{m.batch, m.head, (int)m.row}; }

}  // namespace vitattn_check
