// C ABI of the rms norm with the residual's addition and of dropout: validation,
// workspace sizing and status codes. Validation makes no HIP call.
#include <exception>

#include "vitattn_operands.h"

namespace {

using namespace vitattn_check;

int check_rows(int B, int H, int N, int D) {
  if (B < 1 || H < 1 || N < 1 || D < 1) return VITATTN_E_INVAL;
  // a row's index plus the rows of one round of workgroups stays below 2^31
  return (double)B * H * N > 0x7fffffff - (1 << 22) ? VITATTN_E_INVAL : VITATTN_OK;
}

int check_rms(int B, int H, int N, int D, int type, int residual_type, int weight_type) {
  const int st = check_rows(B, H, N, D);
  if (st != VITATTN_OK) return st;
  const int size = elem_bytes(type);
  if (size == 0 || D > VITATTN_RMS_MAX_BYTES / size) return VITATTN_E_UNSUPPORTED;
  if (residual_type != type && residual_type != VITATTN_FP32) return VITATTN_E_UNSUPPORTED;
  return weight_type == type || weight_type == VITATTN_FP32 ? VITATTN_OK : VITATTN_E_UNSUPPORTED;
}

// dropout's rate and counter; null: nothing is dropped
int to_drop(const vitattn_dropout_spec* d, vitattn::DropArgs& a) {
  a = vitattn::DropArgs{0, 0, nullptr, 0, 1.f};
  if (d == nullptr) return VITATTN_OK;
  if (!(d->p >= 0. && d->p <= 1.)) return VITATTN_E_INVAL;
  if (d->state && !aligned_to(d->state, 8)) return VITATTN_E_INVAL;
  const double t = rint(d->p * 65536.);
  a.seed = d->seed;
  a.offset = d->offset;
  a.state = d->state;
  a.threshold = (uint32_t)t;
  a.up = t < 65536. ? (float)(65536. / (65536. - t)) : 0.f;
  return VITATTN_OK;
}

// An operand of rows: pointer, strides and element size (absent: null).
struct Rows {
  const void* p;
  const vitattn_strides* s;
  int bytes;
};

// Checks every operand's alignment and strides (the first n_out are written) and that
// no output shares memory with another; an output may be the input that `same` says
// (its index, or -1), at the same strides. `extra`: dense operands behind them, the
// first extra_out of them written.
int check_operands(const Rows* r, const int* same, int n_out, int n, int B, int H, int N, int D, const Range* extra,
                   int extra_out, int n_extra) {
  Memory m[16];
  for (int i = 0; i < n; ++i) {
    m[i] = Memory{};
    if (r[i].p == nullptr) continue;
    if (!aligned_to(r[i].p, r[i].bytes) || check_rows_map(*r[i].s, B, H, N, D, i < n_out)) return VITATTN_E_INVAL;
    m[i] = strided_memory(r[i].p, *r[i].s, B, H, N, D, r[i].bytes);
  }
  for (int i = 0; i < n_extra; ++i) m[n + i] = dense_memory(extra[i].p, extra[i].bytes);
  for (int i = 0; i < n + n_extra; ++i) {
    if (i >= n_out && (i < n || i >= n + extra_out)) continue;
    for (int j = 0; j < n + n_extra; ++j) {
      const bool written = j < n_out || (j >= n && j < n + extra_out);
      if (j == i || (written && j < i)) continue;
      if (i < n_out && j == same[i] && m[i].p == m[j].p) {
        if (r[i].bytes != r[j].bytes || !same_strides(*r[i].s, *r[j].s, B, H, N)) return VITATTN_E_INVAL;
        continue;
      }
      if (memories_meet(m[i], m[j])) return VITATTN_E_INVAL;
    }
  }
  return VITATTN_OK;
}

// Row dimensions in the order in which the first operand's memory has them, those
// that every operand steps through as one merged.
template <typename A>
void set_rows(A& a, int B, int H, int N, vitattn::RowMap* const* maps, int n_maps) {
  int n[3] = {B, H, N}, order[3] = {0, 1, 2};
  const long long s[3] = {maps[0]->s0, maps[0]->s1, maps[0]->s2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j) {
      const int x = order[j], y = order[j + 1];
      if (n[x] != 1 && (n[y] == 1 || s[y] > s[x])) {
        order[j] = y;
        order[j + 1] = x;
      }
    }
  for (int i = 0; i < n_maps; ++i) {
    const long long t[3] = {maps[i]->s0, maps[i]->s1, maps[i]->s2};
    *maps[i] = vitattn::RowMap{t[order[0]], t[order[1]], t[order[2]]};
  }
  merge_rows(a.rows, a.n1, a.n2, n[order[0]], n[order[1]], n[order[2]], maps, n_maps);
}

vitattn::RowMap logical_rows(int B, int H, int N) {
  return row_map(vitattn_strides{(long long)H * N, N, 1}, B, H, N);
}

int rms_fwd(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, const void* w, void* h,
            vitattn_strides sh, void* y, vitattn_strides sy, float* scale, int group, float* rstd, int B, int H, int N,
            int D, float eps, int type, int residual_type, int weight_type, const vitattn_dropout_spec* dropout,
            hipStream_t stream) {
  const int st = check_rms(B, H, N, D, type, residual_type, weight_type);
  if (st != VITATTN_OK) return st;
  const int size = elem_bytes(type), rsize = elem_bytes(residual_type), wsize = elem_bytes(weight_type);
  if (x == nullptr || y == nullptr || (residual == nullptr) != (h == nullptr)) return VITATTN_E_INVAL;
  if (residual == nullptr && residual_type != type) return VITATTN_E_INVAL;
  if ((w && !aligned_to(w, wsize)) || (rstd && !aligned_to(rstd, 4)) || (scale && !aligned_to(scale, 4)))
    return VITATTN_E_INVAL;
  if (!isfinite(eps) || eps < 0.f) return VITATTN_E_INVAL;
  vitattn::RmsArgs a = {};
  if (to_drop(dropout, a.drop) != VITATTN_OK) return VITATTN_E_INVAL;
  a.drop_on = a.drop.threshold != 0;
  if (a.drop_on && residual == nullptr) return VITATTN_E_INVAL;
  const size_t rows = (size_t)B * H * N, groups = group ? (D + (size_t)group - 1) / group : 1;
  const Rows r[] = {{y, &sy, scale ? 1 : size}, {h, &sh, rsize}, {x, &sx, size}, {residual, &sr, rsize}};
  const int same[] = {scale ? -1 : 2, 3};
  const Range extra[] = {{rstd, rows * 4}, {scale, rows * groups * 4}, {w, (size_t)D * wsize},
                         {a.drop_on ? a.drop.state : nullptr, 16}};
  if (check_operands(r, same, 2, 4, B, H, N, D, extra, 2, 4)) return VITATTN_E_INVAL;
  a.x = x;
  a.residual = residual;
  a.h = h;
  a.w = w;
  a.y = y;
  a.scale = scale;
  a.rstd = rstd;
  a.mx = row_map(sx, B, H, N);
  a.my = row_map(sy, B, H, N);
  a.mr = residual ? row_map(sr, B, H, N) : a.mx;
  a.mh = h ? row_map(sh, B, H, N) : a.mx;
  a.ml = logical_rows(B, H, N);
  vitattn::RowMap* const maps[] = {&a.mx, &a.mr, &a.mh, &a.my, &a.ml};
  set_rows(a, B, H, N, maps, 5);
  a.D = D;
  a.group = group;
  a.eps = eps;
  a.type = type;
  a.residual_type = residual_type;
  a.w_f32 = weight_type == VITATTN_FP32;
  a.stream = stream;
  return vitattn::launch_rms_fwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
}

}  // namespace

extern "C" {

int vitattn_rms_norm_fwd(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, const void* w,
                         void* h, vitattn_strides sh, void* y, vitattn_strides sy, float* rstd, int B, int H, int N,
                         int D, float eps, int type, int residual_type, int weight_type,
                         const vitattn_dropout_spec* dropout, void* stream) {
  try {
    return rms_fwd(x, sx, residual, sr, w, h, sh, y, sy, nullptr, 0, rstd, B, H, N, D, eps, type, residual_type,
                   weight_type, dropout, static_cast<hipStream_t>(stream));
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

int vitattn_rms_norm_fp8(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, const void* w,
                         void* h, vitattn_strides sh, void* y, vitattn_strides sy, float* scale, int group, int B,
                         int H, int N, int D, float eps, int type, int residual_type, int weight_type, void* stream) {
  try {
    if (group != 0 && group != 32 && group != 64 && group != 128) return VITATTN_E_UNSUPPORTED;
    if (scale == nullptr) return VITATTN_E_INVAL;
    return rms_fwd(x, sx, residual, sr, w, h, sh, y, sy, scale, group, nullptr, B, H, N, D, eps, type, residual_type,
                   weight_type, nullptr, static_cast<hipStream_t>(stream));
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_rms_norm_bwd_workspace_bytes(int B, int H, int N, int D, int type) {
  if (check_rms(B, H, N, D, type, type, type) != VITATTN_OK) return 0;
  return (size_t)vitattn::rms_partials(B * H * N, D, elem_bytes(type)) * D * sizeof(float);
}

int vitattn_rms_norm_bwd(const void* h, vitattn_strides sh, const void* w, const float* rstd, const void* dy,
                         vitattn_strides sdy, const void* dh, vitattn_strides sdh, void* dx, vitattn_strides sdx,
                         void* dres, vitattn_strides sdres, void* dw, int B, int H, int N, int D, int type,
                         int residual_type, int weight_type, const vitattn_dropout_spec* dropout, void* workspace,
                         size_t workspace_bytes, void* stream) {
  try {
    const int st = check_rms(B, H, N, D, type, residual_type, weight_type);
    if (st != VITATTN_OK) return st;
    const int size = elem_bytes(type), rsize = elem_bytes(residual_type), wsize = elem_bytes(weight_type);
    if (h == nullptr || dy == nullptr || !aligned_to(rstd, 4) || (w && !aligned_to(w, wsize)) ||
        (dw && !aligned_to(dw, wsize)))
      return VITATTN_E_INVAL;
    vitattn::RmsArgs a = {};
    if (to_drop(dropout, a.drop) != VITATTN_OK) return VITATTN_E_INVAL;
    a.drop_on = a.drop.threshold != 0;
    const size_t need = dw ? vitattn_rms_norm_bwd_workspace_bytes(B, H, N, D, type) : 0;
    if (dw && (!aligned16(workspace) || workspace_bytes < need)) return VITATTN_E_WORKSPACE;
    const Rows r[] = {{dx, &sdx, size}, {dres, &sdres, rsize}, {h, &sh, rsize}, {dy, &sdy, size}, {dh, &sdh, rsize}};
    const int same[] = {3, 4};
    const size_t wbytes = (size_t)D * wsize;
    const Range extra[] = {{dw, wbytes}, {dw ? workspace : nullptr, need}, {w, wbytes}, {rstd, (size_t)B * H * N * 4},
                           {a.drop_on ? a.drop.state : nullptr, 16}};
    if (check_operands(r, same, 2, 5, B, H, N, D, extra, 2, 5)) return VITATTN_E_INVAL;
    a.h = const_cast<void*>(h);
    a.w = w;
    a.rstd = const_cast<float*>(rstd);
    a.dy = dy;
    a.dh = dh;
    a.dx = dx;
    a.dres = dres;
    a.dw = dw;
    a.partial = dw ? static_cast<float*>(workspace) : nullptr;
    a.mh = row_map(sh, B, H, N);
    a.mdy = row_map(sdy, B, H, N);
    a.mdh = dh ? row_map(sdh, B, H, N) : a.mh;
    a.mdx = dx ? row_map(sdx, B, H, N) : a.mh;
    a.mdres = dres ? row_map(sdres, B, H, N) : a.mh;
    a.ml = logical_rows(B, H, N);
    vitattn::RowMap* const maps[] = {&a.mh, &a.mdy, &a.mdh, &a.mdx, &a.mdres, &a.ml};
    set_rows(a, B, H, N, maps, 6);
    a.D = D;
    a.type = type;
    a.residual_type = residual_type;
    a.w_f32 = weight_type == VITATTN_FP32;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_rms_bwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

int vitattn_dropout(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, void* y,
                    vitattn_strides sy, int B, int H, int N, int D, int type, int residual_type,
                    const vitattn_dropout_spec* dropout, void* stream) {
  try {
    const int st = check_rows(B, H, N, D);
    if (st != VITATTN_OK) return st;
    const int size = elem_bytes(type), rsize = elem_bytes(residual_type);
    // (fp32 rows without a residual to 16 bits: the gradient of a branch beside an fp32 residual)
    const bool narrow = residual == nullptr && type == VITATTN_FP32 && rsize == 2;
    if (size == 0 || (residual_type != type && residual_type != VITATTN_FP32 && !narrow)) return VITATTN_E_UNSUPPORTED;
    if (x == nullptr || y == nullptr || dropout == nullptr) return VITATTN_E_INVAL;
    if (residual == nullptr && residual_type != type && !narrow) return VITATTN_E_INVAL;
    vitattn::DropoutArgs a = {};
    if (to_drop(dropout, a.drop) != VITATTN_OK) return VITATTN_E_INVAL;
    a.pieces = (int)(((long long)D + 7) / 8);
    // a launch below 2^32 work-items of four pieces each
    if ((double)B * H * N * a.pieces >= 4. * (kMaxWorkItems - 4096)) return VITATTN_E_INVAL;
    const Rows r[] = {{y, &sy, rsize}, {x, &sx, size}, {residual, &sr, rsize}};
    const int same[] = {residual && y == residual ? 2 : 1};
    const Range extra[] = {{a.drop.state, 16}};
    if (check_operands(r, same, 1, 3, B, H, N, D, extra, 0, 1)) return VITATTN_E_INVAL;
    a.x = x;
    a.residual = residual;
    a.y = y;
    a.mx = row_map(sx, B, H, N);
    a.my = row_map(sy, B, H, N);
    a.mr = residual ? row_map(sr, B, H, N) : a.mx;
    a.ml = logical_rows(B, H, N);
    vitattn::RowMap* const maps[] = {&a.mx, &a.mr, &a.my, &a.ml};
    set_rows(a, B, H, N, maps, 4);
    a.D = D;
    a.type = type;
    a.residual_type = residual_type;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_dropout(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

}  // extern "C"
