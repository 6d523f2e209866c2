// What the C entry points of the operators around the attention check of their
// operands: overlaps of strided memory, rows in three dimensions. No HIP call.
#pragma once

#include "vitattn_check.h"

namespace vitattn_check {

inline bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && x < y + nb && y < x + na;
}
struct Range {
  const void* p;  // null: absent
  size_t bytes;
};
// whether one of the first n_out ranges meets any other
inline bool outputs_meet(const Range* r, int n_out, int n) {
  for (int o = 0; o < n_out; ++o)
    for (int i = o + 1; i < n; ++i)
      if (ranges_overlap(r[o].p, r[o].bytes, r[i].p, r[i].bytes)) return true;
  return false;
}

// Memory of an operand: rows of `row` bytes in up to three dimensions at byte
// strides (sizes of one: their strides do not matter).
typedef __int128 wide;
struct Memory {
  const void* p;  // null: absent
  long long row;
  int n[3];
  wide stride[3];
};
inline Memory dense_memory(const void* p, size_t bytes) { return Memory{p, (long long)bytes, {1, 1, 1}, {0, 0, 0}}; }
inline Memory strided_memory(const void* p, const vitattn_strides& s, int n0, int n1, int n2, int D, int elem_bytes) {
  return Memory{p, (long long)D * elem_bytes, {n0, n1, n2},
                {(wide)s.batch * elem_bytes, (wide)s.head * elem_bytes, (wide)s.row * elem_bytes}};
}

// A step that na of the first operand's indexes and nb of the second's take.
struct Step {
  wide stride;
  long long na, nb;
};
// Whether rows of wa bytes at i_0 s_0 + .. and rows of wb at delta + j_0 s_0 + .. meet
// (0 <= i < na, 0 <= j < nb, steps from the longest to the shortest): the two parts
// under a step can meet for few differences i_0 - j_0 alone, each of which is a
// question of the same kind about the steps that are left. Interleaved views of one
// tensor have the same steps and are settled in a few of these; out of budget
// counts as meeting.
inline bool steps_meet(const Step* s, int n, wide wa, wide wb, wide delta, int& budget) {
  if (--budget < 0) return true;
  wide la = wa, lb = wb;  // spans
  for (int i = 0; i < n; ++i) {
    la += (s[i].na - 1) * s[i].stride;
    lb += (s[i].nb - 1) * s[i].stride;
  }
  if (delta >= la || -delta >= lb) return false;
  if (n == 0) return true;
  const wide S = s[0].stride;
  la -= (s[0].na - 1) * S;
  lb -= (s[0].nb - 1) * S;
  // differences t with -lb < delta - t S < la
  auto floor_div = [](wide x, wide y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
  wide lo = floor_div(delta - la, S) + 1, hi = -floor_div(-(delta + lb), S) - 1;
  if (lo < -(s[0].nb - 1)) lo = -(s[0].nb - 1);
  if (hi > s[0].na - 1) hi = s[0].na - 1;
  for (wide t = lo; t <= hi; ++t)
    if (steps_meet(s + 1, n - 1, wa, wb, delta - t * S, budget)) return true;
  return false;
}
inline bool memories_meet(const Memory& a, const Memory& b) {
  if (a.p == nullptr || b.p == nullptr) return false;
  const wide delta = (wide) reinterpret_cast<uintptr_t>(b.p) - (wide) reinterpret_cast<uintptr_t>(a.p);
  wide la = a.row, lb = b.row;
  for (int i = 0; i < 3; ++i) {
    la += (a.n[i] - 1) * a.stride[i];
    lb += (b.n[i] - 1) * b.stride[i];
  }
  if (delta >= la || -delta >= lb) return false;  // (the usual end)
  Step s[6];
  int n = 0;
  for (int i = 0; i < 6; ++i) {
    const Memory& m = i < 3 ? a : b;
    const int size = m.n[i % 3];
    const wide stride = m.stride[i % 3];
    if (size == 1 || stride == 0) continue;
    int at = 0;
    while (at < n && s[at].stride > stride) ++at;
    if (at == n || s[at].stride != stride) {
      for (int k = n++; k > at; --k) s[k] = s[k - 1];
      s[at] = Step{stride, 1, 1};
    }
    (i < 3 ? s[at].na : s[at].nb) += size - 1;
  }
  int budget = 4096;
  return steps_meet(s, n, a.row, b.row, delta, budget);
}
// whether one of the first n_out operands meets any other
inline bool outputs_meet(const Memory* m, int n_out, int n) {
  for (int o = 0; o < n_out; ++o)
    for (int i = o + 1; i < n; ++i)
      if (memories_meet(m[o], m[i])) return true;
  return false;
}

// ------------------------------------------------------------ row kernels

inline int elem_bytes(int type) { return type == VITATTN_FP32 ? 4 : type == VITATTN_BF16 || type == VITATTN_FP16 ? 2 : 0; }
inline bool aligned_to(const void* p, int bytes) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % (unsigned)bytes == 0;
}

// Rows of D elements in three dimensions at any element strides >= 0; an
// output must not overlap itself.
inline int check_rows_map(const vitattn_strides& m, int n0, int n1, int n2, int D, bool output) {
  if (m.batch < 0 || m.head < 0 || m.row < 0) return VITATTN_E_INVAL;
  if ((double)(n0 - 1) * m.batch + (double)(n1 - 1) * m.head + (double)(n2 - 1) * m.row + D > 4.0e18)
    return VITATTN_E_INVAL;
  if (!output) return VITATTN_OK;
  const long long size[3] = {n0, n1, n2}, stride[3] = {m.batch, m.head, m.row};
  int idx[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[idx[j]] < stride[idx[i]]) {
        const int t = idx[i];
        idx[i] = idx[j];
        idx[j] = t;
      }
  long long span = D;
  for (int i = 0; i < 3; ++i) {
    const int x = idx[i];
    if (size[x] == 1) continue;
    if (stride[x] < span) return VITATTN_E_INVAL;
    span += (size[x] - 1) * stride[x];
  }
  return VITATTN_OK;
}
inline bool same_strides(const vitattn_strides& a, const vitattn_strides& b, int n0, int n1, int n2) {
  return (n0 == 1 || a.batch == b.batch) && (n1 == 1 || a.head == b.head) && (n2 == 1 || a.row == b.row);
}
inline vitattn::RowMap row_map(const vitattn_strides& m, int n0, int n1, int n2) {
  return vitattn::RowMap{n0 == 1 ? 0 : m.batch, n1 == 1 ? 0 : m.head, n2 == 1 ? 0 : m.row};
}
// elements from the first to behind the last
inline size_t span_of(const vitattn_strides& m, int n0, int n1, int n2, int D) {
  return (size_t)((n0 - 1) * m.batch + (n1 - 1) * m.head + (n2 - 1) * m.row + D);
}

// Merges row dimensions that every operand steps through as one.
inline void merge_rows(int& rows, int& rows1, int& rows2, int B, int H, int N, vitattn::RowMap* const* maps, int n_maps) {
  rows = B * H * N;
  bool inner = true, outer = true;  // (H, N) as one; (B, that) as one
  for (int i = 0; i < n_maps; ++i) inner = inner && (H == 1 || N == 1 || maps[i]->s1 == N * maps[i]->s2);
  int n1 = H, n2 = N;
  if (inner) {
    for (int i = 0; i < n_maps; ++i)
      if (N == 1) maps[i]->s2 = maps[i]->s1;
    n1 = 1;
    n2 = H * N;
    for (int i = 0; i < n_maps; ++i) outer = outer && (B == 1 || n2 == 1 || maps[i]->s0 == n2 * maps[i]->s2);
    if (outer) {
      for (int i = 0; i < n_maps; ++i)
        if (n2 == 1) maps[i]->s2 = maps[i]->s0;
      n2 *= B;
    }
  }
  rows1 = n1;
  rows2 = n2;
}

}  // namespace vitattn_check
