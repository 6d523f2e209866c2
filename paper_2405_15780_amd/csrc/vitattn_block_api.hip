// C ABI of the operators around the attention (layer norm, rotary positions)
// and of differential attention: validation, workspace sizing and status codes.
// As in vitattn_api.hip, validation makes no HIP call.
#include <exception>

#include "vitattn_check.h"

namespace {

using namespace vitattn_check;

bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && x < y + nb && y < x + na;
}
struct Range {
  const void* p;  // null: absent
  size_t bytes;
};
// whether one of the first n_out ranges meets any other
bool outputs_meet(const Range* r, int n_out, int n) {
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
Memory dense_memory(const void* p, size_t bytes) { return Memory{p, (long long)bytes, {1, 1, 1}, {0, 0, 0}}; }
Memory strided_memory(const void* p, const vitattn_strides& s, int n0, int n1, int n2, int D, int elem_bytes) {
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
bool steps_meet(const Step* s, int n, wide wa, wide wb, wide delta, int& budget) {
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
bool memories_meet(const Memory& a, const Memory& b) {
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
bool outputs_meet(const Memory* m, int n_out, int n) {
  for (int o = 0; o < n_out; ++o)
    for (int i = o + 1; i < n; ++i)
      if (memories_meet(m[o], m[i])) return true;
  return false;
}

// ------------------------------------------------------------ row kernels

int elem_bytes(int type) { return type == VITATTN_FP32 ? 4 : type == VITATTN_BF16 || type == VITATTN_FP16 ? 2 : 0; }
bool aligned_to(const void* p, int bytes) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % (unsigned)bytes == 0;
}

// Rows of D elements in three dimensions at any element strides >= 0; an
// output must not overlap itself.
int check_rows_map(const vitattn_strides& m, int n0, int n1, int n2, int D, bool output) {
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
bool same_strides(const vitattn_strides& a, const vitattn_strides& b, int n0, int n1, int n2) {
  return (n0 == 1 || a.batch == b.batch) && (n1 == 1 || a.head == b.head) && (n2 == 1 || a.row == b.row);
}
vitattn::RowMap row_map(const vitattn_strides& m, int n0, int n1, int n2) {
  return vitattn::RowMap{n0 == 1 ? 0 : m.batch, n1 == 1 ? 0 : m.head, n2 == 1 ? 0 : m.row};
}
// elements from the first to behind the last
size_t span_of(const vitattn_strides& m, int n0, int n1, int n2, int D) {
  return (size_t)((n0 - 1) * m.batch + (n1 - 1) * m.head + (n2 - 1) * m.row + D);
}

constexpr int kNormMaxWidth = 1 << 24;

int check_norm(int B, int H, int N, int D, int type, int weight_type) {
  if (B < 1 || H < 1 || N < 1 || D < 1) return VITATTN_E_INVAL;
  // a row's index plus the rows of one round of workgroups (up to 2^21, at one piece a row) stays below 2^31
  if ((double)B * H * N > 0x7fffffff - (1 << 22)) return VITATTN_E_INVAL;
  if (D > kNormMaxWidth || elem_bytes(type) == 0) return VITATTN_E_UNSUPPORTED;
  return weight_type == type || weight_type == VITATTN_FP32 ? VITATTN_OK : VITATTN_E_UNSUPPORTED;
}

// Merges row dimensions that every operand steps through as one.
void set_rows(vitattn::NormArgs& a, int B, int H, int N, vitattn::RowMap* const* maps, int n_maps) {
  a.rows = B * H * N;
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
  a.n1 = n1;
  a.n2 = n2;
}

// ------------------------------------------------------------ differential attention

int check_diff_sizes(int B, int H, int Nq, int Nk, int d, int e) {
  if (B < 1 || H < 1 || Nq < 1 || Nk < 1) return VITATTN_E_INVAL;
  if (d < 8 || d > VITATTN_DIFF_MAX_D || d % 8 != 0 || e < 8 || e > VITATTN_DIFF_MAX_E || e % 8 != 0)
    return VITATTN_E_UNSUPPORTED;
  const int N = Nq > Nk ? Nq : Nk;
  // rows of the two maps, and launches below 2^32 work-items: 4 per row, padded
  // to 128 rows, and 8 to 32 of each of 64 rows in the row pass
  if (2.0 * B * H * (N + 512.0) > 0x7fffffff || 4.0 * B * H * (N + 512.0) >= kMaxWorkItems) return VITATTN_E_INVAL;
  // 1,024 per query row where the keys are split
  if (vitattn::diff_split_keys(Nq, Nk) && 1024.0 * B * H * Nq >= kMaxWorkItems) return VITATTN_E_INVAL;
  return VITATTN_OK;
}

// check_map for rows read up to 512 past the last by tile requests
int check_diff_map(const vitattn_strides& m, int B, int H, int N, int width, bool output) {
  if (check_map(m, B, H, N, width, 2, output)) return VITATTN_E_INVAL;
  return (N + 512LL) * m.row * 2 > 0x7fffffffLL ? VITATTN_E_INVAL : VITATTN_OK;
}

int check_lam(const void* lam, int lam_type) {
  if (lam_type != VITATTN_FP32 && lam_type != VITATTN_BF16) return VITATTN_E_UNSUPPORTED;
  return aligned_to(lam, elem_bytes(lam_type)) ? VITATTN_OK : VITATTN_E_INVAL;
}

}  // namespace

extern "C" {

int vitattn_layer_norm_fwd(const void* x, vitattn_strides sx, const void* w, const void* b, void* y,
                           vitattn_strides sy, float* mean, float* rstd, int B, int H, int N, int D, float eps,
                           int type, int weight_type, void* stream) {
  try {
    const int st = check_norm(B, H, N, D, type, weight_type);
    if (st != VITATTN_OK) return st;
    const int size = elem_bytes(type), wsize = elem_bytes(weight_type);
    if (!aligned_to(x, size) || !aligned_to(y, size) || (w && !aligned_to(w, wsize)) || (b && !aligned_to(b, wsize)))
      return VITATTN_E_INVAL;
    if ((mean == nullptr) != (rstd == nullptr) || (mean && (!aligned_to(mean, 4) || !aligned_to(rstd, 4))))
      return VITATTN_E_INVAL;
    if (!isfinite(eps) || eps < 0.f) return VITATTN_E_INVAL;
    if (check_rows_map(sx, B, H, N, D, false) || check_rows_map(sy, B, H, N, D, true)) return VITATTN_E_INVAL;
    if (x == y && !same_strides(sx, sy, B, H, N)) return VITATTN_E_INVAL;
    const size_t stats = sizeof(float) * B * H * N, wbytes = (size_t)D * wsize;
    const Range ranges[] = {{y, span_of(sy, B, H, N, D) * size}, {mean, stats}, {rstd, stats},
                            {x == y ? nullptr : x, span_of(sx, B, H, N, D) * size}, {w, wbytes}, {b, wbytes}};
    if (outputs_meet(ranges, 3, 6)) return VITATTN_E_INVAL;
    vitattn::NormArgs a = {};
    a.x = x;
    a.w = w;
    a.b = b;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.mx = row_map(sx, B, H, N);
    a.my = row_map(sy, B, H, N);
    vitattn::RowMap* const maps[] = {&a.mx, &a.my};
    set_rows(a, B, H, N, maps, 2);
    a.D = D;
    a.eps = eps;
    a.type = type;
    a.w_f32 = weight_type == VITATTN_FP32;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_norm_fwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_layer_norm_bwd_workspace_bytes(int B, int H, int N, int D, int type) {
  if (check_norm(B, H, N, D, type, type) != VITATTN_OK) return 0;
  return (size_t)vitattn::norm_partials(B * H * N, D, elem_bytes(type)) * 2 * D * sizeof(float);
}

int vitattn_layer_norm_bwd(const void* x, vitattn_strides sx, const void* w, const float* mean, const float* rstd,
                           const void* dy, vitattn_strides sdy, void* dx, vitattn_strides sdx, void* dw, void* db,
                           int B, int H, int N, int D, int type, int weight_type, void* workspace,
                           size_t workspace_bytes, void* stream) {
  try {
    const int st = check_norm(B, H, N, D, type, weight_type);
    if (st != VITATTN_OK) return st;
    const int size = elem_bytes(type), wsize = elem_bytes(weight_type);
    if (!aligned_to(x, size) || !aligned_to(dy, size) || !aligned_to(dx, size) || (w && !aligned_to(w, wsize)) ||
        !aligned_to(mean, 4) || !aligned_to(rstd, 4) || (dw && !aligned_to(dw, wsize)) || (db && !aligned_to(db, wsize)))
      return VITATTN_E_INVAL;
    if (check_rows_map(sx, B, H, N, D, false) || check_rows_map(sdy, B, H, N, D, false) ||
        check_rows_map(sdx, B, H, N, D, true))
      return VITATTN_E_INVAL;
    // dx may replace dy; x is still read by rows too long for registers
    if (dy == dx && !same_strides(sdy, sdx, B, H, N)) return VITATTN_E_INVAL;
    const bool sums = dw != nullptr || db != nullptr;
    const size_t need = sums ? vitattn_layer_norm_bwd_workspace_bytes(B, H, N, D, type) : 0;
    const size_t stats = sizeof(float) * B * H * N, wbytes = (size_t)D * wsize;
    const Range ranges[] = {{dx, span_of(sdx, B, H, N, D) * size}, {dw, wbytes}, {db, wbytes},
                            {sums ? workspace : nullptr, need}, {x, span_of(sx, B, H, N, D) * size},
                            {dy == dx ? nullptr : dy, span_of(sdy, B, H, N, D) * size}, {mean, stats}, {rstd, stats},
                            {w, wbytes}};
    if (outputs_meet(ranges, 4, 9)) return VITATTN_E_INVAL;
    // the column sums of rows too long for registers read dy after dx is written
    if (dy == dx && sums && D > 256 * 8 * (16 / size)) return VITATTN_E_INVAL;
    if (sums && (!aligned16(workspace) || workspace_bytes < need)) return VITATTN_E_WORKSPACE;
    vitattn::NormArgs a = {};
    a.x = x;
    a.dy = dy;
    a.w = w;
    a.y = dx;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.dw = dw;
    a.db = db;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    a.mx = row_map(sx, B, H, N);
    a.mdy = row_map(sdy, B, H, N);
    a.my = row_map(sdx, B, H, N);
    vitattn::RowMap* const maps[] = {&a.mx, &a.mdy, &a.my};
    set_rows(a, B, H, N, maps, 3);
    a.D = D;
    a.type = type;
    a.w_f32 = weight_type == VITATTN_FP32;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_norm_bwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

int vitattn_rotary(const void* q, vitattn_strides sq, void* q_out, vitattn_strides sq_out, int Hq, const void* k,
                   vitattn_strides sk, void* k_out, vitattn_strides sk_out, int Hk, const void* positions,
                   long long pos_batch, long long pos_row, long long pos_axis, int pos_type, const int* sections,
                   int n_axes, double base, int B, int N, int d, int type, int flags, void* stream) {
  try {
    if (B < 1 || N < 1 || d < 2 || Hq < 1 || Hk < 0 || n_axes < 1 || sections == nullptr) return VITATTN_E_INVAL;
    const int size = elem_bytes(type);
    if (size == 0 || n_axes > VITATTN_ROTARY_MAX_AXES) return VITATTN_E_UNSUPPORTED;
    if ((flags & ~(VITATTN_ROTARY_INTERLEAVED | VITATTN_ROTARY_INVERSE | VITATTN_ROTARY_JOINT)) != 0) return VITATTN_E_INVAL;
    if (pos_type < VITATTN_POS_I32 || pos_type > VITATTN_POS_F32) return VITATTN_E_INVAL;
    if (!isfinite(base) || base <= 0.) return VITATTN_E_INVAL;
    long long pairs = 0;
    for (int i = 0; i < n_axes; ++i) {
      if (sections[i] < 0) return VITATTN_E_INVAL;
      pairs += sections[i];
    }
    if (pairs < 1 || 2 * pairs > d) return VITATTN_E_INVAL;
    if (pairs > VITATTN_ROTARY_MAX_PAIRS || d > 65536) return VITATTN_E_UNSUPPORTED;
    // grid limits: 16-bit second and third dimensions, below 2^32 work-items in the first
    if (B > 65535 || (long long)Hq + Hk > 65535 || (double)N * (d / 2 + 2) + 256 >= kMaxWorkItems) return VITATTN_E_INVAL;
    if (!aligned_to(q, size) || !aligned_to(q_out, size) || !aligned_to(positions, pos_type == VITATTN_POS_I64 ? 8 : 4))
      return VITATTN_E_INVAL;
    if (Hk > 0 && (!aligned_to(k, size) || !aligned_to(k_out, size))) return VITATTN_E_INVAL;
    if (pos_batch < 0 || pos_row < 0 || pos_axis < 0 ||
        (double)(B - 1) * pos_batch + (double)(N - 1) * pos_row + (double)(n_axes - 1) * pos_axis > 1.0e18)
      return VITATTN_E_INVAL;
    const void* in[2] = {q, k};
    void* out[2] = {q_out, k_out};
    const vitattn_strides si[2] = {sq, sk}, so[2] = {sq_out, sk_out};
    const int heads[2] = {Hq, Hk};
    const size_t pos_bytes = (size_t)((B - 1) * pos_batch + (N - 1) * pos_row + (n_axes - 1) * pos_axis + 1) *
                             (pos_type == VITATTN_POS_I64 ? 8 : 4);
    for (int o = 0; o < 2; ++o) {
      if (heads[o] == 0) continue;
      if (check_rows_map(si[o], B, heads[o], N, d, false) || check_rows_map(so[o], B, heads[o], N, d, true))
        return VITATTN_E_INVAL;
      const size_t bytes = span_of(so[o], B, heads[o], N, d) * size;
      if (ranges_overlap(positions, pos_bytes, out[o], bytes)) return VITATTN_E_INVAL;
      for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0 || (i == o && in[i] == out[o])) continue;
        if (ranges_overlap(in[i], span_of(si[i], B, heads[i], N, d) * size, out[o], bytes)) {
          // q and k may be interleaved views of one tensor, turned in place
          const bool both = in[0] == out[0] && in[1] == out[1] && i != o;
          if (!both) return VITATTN_E_INVAL;
        }
      }
      if (in[o] == out[o] && !same_strides(si[o], so[o], B, heads[o], N)) return VITATTN_E_INVAL;
    }
    if (Hk > 0 && memories_meet(strided_memory(q_out, sq_out, B, Hq, N, d, size), strided_memory(k_out, sk_out, B, Hk, N, d, size)))
      return VITATTN_E_INVAL;
    vitattn::RotaryArgs a = {};
    for (int o = 0; o < 2; ++o) {
      if (heads[o] == 0) continue;
      a.x[o] = in[o];
      a.y[o] = out[o];
      a.heads[o] = heads[o];
      a.mx[o] = row_map(si[o], B, heads[o], N);
      a.my[o] = row_map(so[o], B, heads[o], N);
    }
    a.pos = positions;
    a.pos_batch = pos_batch;
    a.pos_row = pos_row;
    a.pos_axis = pos_axis;
    a.pos_type = pos_type;
    a.B = B;
    a.N = N;
    a.d = d;
    a.pairs = (int)pairs;
    a.type = type;
    a.interleaved = (flags & VITATTN_ROTARY_INTERLEAVED) != 0;
    // frequencies in turns: base^(-i / n) / 2 pi over the n pairs of the axis,
    // or of all axes (JOINT)
    const double sign = (flags & VITATTN_ROTARY_INVERSE) ? -1. : 1., two_pi = 6.283185307179586476925287;
    const double log_base = log(base);
    int p = 0;
    for (int ax = 0; ax < n_axes; ++ax)
      for (int i = 0; i < sections[ax]; ++i, ++p) {
        const double t = (flags & VITATTN_ROTARY_JOINT) ? (double)p / (double)pairs : (double)i / sections[ax];
        a.freq[p] = sign * exp(-t * log_base) / two_pi;
        a.axis[p] = (unsigned char)ax;
      }
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_rotary(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_diff_fwd_workspace_bytes(int B, int H, int Nq, int Nk, int d, int e) {
  if (check_diff_sizes(B, H, Nq, Nk, d, e) != VITATTN_OK) return 0;
  return vitattn::diff_fwd_workspace_floats(B, H, Nq, Nk, e) * sizeof(float);
}

int vitattn_diff_fwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                     vitattn_strides sv, const void* lam, int lam_type, const int* key_lens, void* o,
                     vitattn_strides so, float* maps, float* lse, int B, int H, int Nq, int Nk, int d, int e, float scale,
                     void* workspace, size_t workspace_bytes, void* stream) {
  try {
    int st = check_diff_sizes(B, H, Nq, Nk, d, e);
    if (st != VITATTN_OK) return st;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || (maps && !aligned16(maps)) ||
        (lse && !aligned16(lse)) || (key_lens && !aligned_to(key_lens, 4)))
      return VITATTN_E_INVAL;
    if (!scale_ok(scale)) return VITATTN_E_INVAL;
    if ((st = check_lam(lam, lam_type)) != VITATTN_OK) return st;
    if (check_diff_map(sq, B, 2 * H, Nq, d, false) || check_diff_map(sk, B, 2 * H, Nk, d, false) ||
        check_diff_map(sv, B, H, Nk, e, false) || check_diff_map(so, B, H, Nq, e, true))
      return VITATTN_E_INVAL;
    const size_t need = vitattn_diff_fwd_workspace_bytes(B, H, Nq, Nk, d, e);
    if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return VITATTN_E_WORKSPACE;
    const size_t rows = (size_t)2 * B * H * Nq;
    const Memory used[] = {strided_memory(o, so, B, H, Nq, e, 2), dense_memory(maps, rows * e * 4), dense_memory(lse, rows * 4),
                           dense_memory(need > 0 ? workspace : nullptr, need), strided_memory(q, sq, B, 2 * H, Nq, d, 2),
                           strided_memory(k, sk, B, 2 * H, Nk, d, 2), strided_memory(v, sv, B, H, Nk, e, 2),
                           dense_memory(lam, (size_t)H * elem_bytes(lam_type)), dense_memory(key_lens, (size_t)B * 4)};
    if (outputs_meet(used, 4, 9)) return VITATTN_E_INVAL;
    vitattn::DiffArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.lam = lam;
    a.key_lens = key_lens;
    a.o = static_cast<uint16_t*>(o);
    a.maps = maps;
    a.lse = lse;
    a.work = static_cast<float*>(workspace);
    a.mq = to_map(sq);
    a.mk = to_map(sk);
    a.mv = to_map(sv);
    a.mo = to_map(so);
    a.B = B;
    a.H = H;
    a.Nq = Nq;
    a.Nk = Nk;
    a.d = d;
    a.e = e;
    a.scale = scale;
    a.lam_bf16 = lam_type == VITATTN_BF16;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_diff_fwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_diff_bwd_workspace_bytes(int B, int H, int Nq, int Nk, int d, int e) {
  if (check_diff_sizes(B, H, Nq, Nk, d, e) != VITATTN_OK) return 0;
  return vitattn::diff_bwd_workspace_floats(B, H, Nq, Nk, d) * sizeof(float);
}

int vitattn_diff_bwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                     vitattn_strides sv, const void* lam, int lam_type, const int* key_lens, const float* maps,
                     const float* lse, const void* dout, vitattn_strides sdo, void* dq, vitattn_strides sdq, void* dk,
                     vitattn_strides sdk, void* dv, vitattn_strides sdv, void* dlam, int B, int H, int Nq, int Nk, int d,
                     int e, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    int st = check_diff_sizes(B, H, Nq, Nk, d, e);
    if (st != VITATTN_OK) return st;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(maps) || !aligned16(lse) || !aligned16(dout) ||
        !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || (key_lens && !aligned_to(key_lens, 4)))
      return VITATTN_E_INVAL;
    if (!scale_ok(scale)) return VITATTN_E_INVAL;
    if ((st = check_lam(lam, lam_type)) != VITATTN_OK) return st;
    if (dlam && !aligned_to(dlam, elem_bytes(lam_type))) return VITATTN_E_INVAL;
    if (check_diff_map(sq, B, 2 * H, Nq, d, false) || check_diff_map(sk, B, 2 * H, Nk, d, false) ||
        check_diff_map(sv, B, H, Nk, e, false) ||
        check_diff_map(sdo, B, H, Nq, e, false) || check_diff_map(sdq, B, 2 * H, Nq, d, true) ||
        check_diff_map(sdk, B, 2 * H, Nk, d, true) || check_diff_map(sdv, B, H, Nk, e, true))
      return VITATTN_E_INVAL;
    const size_t need = vitattn_diff_bwd_workspace_bytes(B, H, Nq, Nk, d, e), rows = (size_t)2 * B * H * Nq;
    if (!aligned16(workspace) || workspace_bytes < need) return VITATTN_E_WORKSPACE;
    const size_t lam_bytes = (size_t)H * elem_bytes(lam_type);
    const Memory used[] = {strided_memory(dq, sdq, B, 2 * H, Nq, d, 2), strided_memory(dk, sdk, B, 2 * H, Nk, d, 2),
                           strided_memory(dv, sdv, B, H, Nk, e, 2), dense_memory(dlam, lam_bytes),
                           dense_memory(workspace, need), strided_memory(q, sq, B, 2 * H, Nq, d, 2),
                           strided_memory(k, sk, B, 2 * H, Nk, d, 2), strided_memory(v, sv, B, H, Nk, e, 2),
                           strided_memory(dout, sdo, B, H, Nq, e, 2), dense_memory(maps, rows * e * 4),
                           dense_memory(lse, rows * 4), dense_memory(lam, lam_bytes), dense_memory(key_lens, (size_t)B * 4)};
    if (outputs_meet(used, 5, 13)) return VITATTN_E_INVAL;
    vitattn::DiffArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.lam = lam;
    a.key_lens = key_lens;
    a.maps = const_cast<float*>(maps);
    a.lse = const_cast<float*>(lse);
    a.dout = static_cast<const uint16_t*>(dout);
    a.dq = static_cast<uint16_t*>(dq);
    a.dk = static_cast<uint16_t*>(dk);
    a.dv = static_cast<uint16_t*>(dv);
    a.dlam = dlam;
    a.work = static_cast<float*>(workspace);
    a.mq = to_map(sq);
    a.mk = to_map(sk);
    a.mv = to_map(sv);
    a.mg = to_map(sdo);
    a.mdq = to_map(sdq);
    a.mdk = to_map(sdk);
    a.mdv = to_map(sdv);
    a.B = B;
    a.H = H;
    a.Nq = Nq;
    a.Nk = Nk;
    a.d = d;
    a.e = e;
    a.scale = scale;
    a.lam_bf16 = lam_type == VITATTN_BF16;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_diff_bwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

}  // extern "C"
