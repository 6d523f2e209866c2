// C ABI of the attention over chosen key blocks and of the choice: validation,
// workspace sizing and status codes. Validation makes no HIP call.
#include <exception>

#include "vitattn_operands.h"

namespace {

using namespace vitattn_check;

// rows past the last that tile requests may ask for
constexpr long long kRowsBehind = 1280;

int check_heads(int B, int H, int Hk, int N, int d) {
  if (B < 1 || H < 1 || Hk < 1 || N < 1 || H % Hk != 0) return VITATTN_E_INVAL;
  return d < 8 || d > 160 || d % 8 != 0 ? VITATTN_E_UNSUPPORTED : VITATTN_OK;
}
int check_block(int Nk, int block) {
  if (block < 64 || block > VITATTN_SPARSE_MAX_BLOCK || block % 64 != 0) return VITATTN_E_UNSUPPORTED;
  return ((long long)Nk + block - 1) / block > VITATTN_SPARSE_MAX_BLOCKS ? VITATTN_E_UNSUPPORTED : VITATTN_OK;
}

// bf16 operands whose rows are addressed from a head's first
int check_rows(const vitattn_strides& m, int B, int H, int N, int d, bool output) {
  if (check_map(m, B, H, N, d, 2, output)) return VITATTN_E_INVAL;
  return (N + kRowsBehind) * m.row * 2 > 0x7fffffffLL ? VITATTN_E_INVAL : VITATTN_OK;
}

// sizes of the attention, into the arguments
int check_sparse(vitattn::SparseArgs& a, int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block, int topk) {
  int st = check_heads(B, H, Hk, Nq, d);
  if (st != VITATTN_OK) return st;
  if (Nk < 1 || q_block < 1 || topk < 1) return VITATTN_E_INVAL;
  if ((st = check_block(Nk, block)) != VITATTN_OK) return st;
  if (topk > VITATTN_SPARSE_MAX_TOPK || H / Hk > 2047) return VITATTN_E_UNSUPPORTED;
  if (Nq > 1 << 26) return VITATTN_E_INVAL;  // (a query tile's number has 20 bits)
  a.B = B;
  a.H = H;
  a.Hk = Hk;
  a.Nq = Nq;
  a.Nk = Nk;
  a.d = d;
  a.block = block;
  a.q_block = q_block;
  a.topk = topk;
  a.groups = (Nq - 1) / q_block + 1;
  a.nb = (Nk - 1) / block + 1;
  // launches below 2^32 work-items: 4 per row, padded to 128 rows; one per row padded to 4,096 (the map);
  // 32 splits of few queries and 192 per row where they are joined; rows below 2^31
  const double rows = (double)B * H * (Nq + 128.), keys = (double)B * Hk * ((double)a.nb * block);
  if (4. * rows >= kMaxWorkItems || (double)B * H * (Nq / 4096 + 1) * 4096. >= kMaxWorkItems || rows >= 0x7fffffff)
    return VITATTN_E_INVAL;
  if (Nq <= 256 && 192. * B * H * (Nq + 64.) >= kMaxWorkItems) return VITATTN_E_INVAL;
  if (4. * keys >= kMaxWorkItems) return VITATTN_E_INVAL;
  return VITATTN_OK;
}

int check_sparse_bwd(const vitattn::SparseArgs& a) {
  // a work item of the dK/dV kernel: 2 work-items per key of a block; int numbers
  const double items = (double)a.B * a.Hk * vitattn::sparse_bwd_items(a);
  return items * a.block * 2. >= kMaxWorkItems || items >= 0x7fffffff ? VITATTN_E_INVAL : VITATTN_OK;
}

size_t blocks_bytes(const vitattn::SparseArgs& a) { return (size_t)a.B * a.H * a.groups * a.topk * sizeof(int); }

}  // namespace

extern "C" {

int vitattn_block_means(const void* k, vitattn_strides sk, const int* key_lens, void* means, float* scales, int B,
                        int Hk, int Nk, int d, int block, void* stream) {
  try {
    int st = check_heads(B, Hk, Hk, Nk, d);
    if (st != VITATTN_OK) return st;
    if ((st = check_block(Nk, block)) != VITATTN_OK) return st;
    if (!aligned16(k) || !aligned16(means) || !aligned_to(scales, 4) || (key_lens && !aligned_to(key_lens, 4)))
      return VITATTN_E_INVAL;
    if (check_map(sk, B, Hk, Nk, d, 2, false)) return VITATTN_E_INVAL;
    const int nb = (Nk - 1) / block + 1;
    const size_t n = (size_t)B * Hk * nb;
    if ((double)n * 256. >= kMaxWorkItems) return VITATTN_E_INVAL;
    const Memory used[] = {dense_memory(means, n * vitattn::means_pitch(d)), dense_memory(scales, n * 4),
                           strided_memory(k, sk, B, Hk, Nk, d, 2), dense_memory(key_lens, (size_t)B * 4)};
    if (outputs_meet(used, 2, 4)) return VITATTN_E_INVAL;
    vitattn::SelectArgs a = {};
    a.x = static_cast<const uint16_t*>(k);
    a.mx = to_map(sk);
    a.key_lens = key_lens;
    a.means = static_cast<int8_t*>(means);
    a.scales = scales;
    a.B = B;
    a.H = a.Hk = Hk;
    a.N = Nk;
    a.d = d;
    a.nb = nb;
    a.block = block;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_means(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

int vitattn_block_select(const void* q, vitattn_strides sq, const void* means, const float* scales, int* blocks, int B,
                         int H, int Hk, int Nq, int d, int nb, int q_block, int topk, void* stream) {
  try {
    const int st = check_heads(B, H, Hk, Nq, d);
    if (st != VITATTN_OK) return st;
    if (nb < 1 || q_block < 1 || topk < 1) return VITATTN_E_INVAL;
    if (nb > VITATTN_SPARSE_MAX_BLOCKS || topk > VITATTN_SELECT_MAX) return VITATTN_E_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(means) || !aligned_to(scales, 4) || !aligned_to(blocks, 4)) return VITATTN_E_INVAL;
    if (check_map(sq, B, H, Nq, d, 2, false)) return VITATTN_E_INVAL;
    const int groups = (Nq - 1) / q_block + 1;
    // a launch's second and third dimensions have 16 bits, the first 32 of work-items
    if (B > 65535 || H > 65535 || (groups / 16 + 1.) * 1024. >= kMaxWorkItems) return VITATTN_E_INVAL;
    const size_t n = (size_t)B * Hk * nb;
    const Memory used[] = {dense_memory(blocks, (size_t)B * H * groups * topk * 4), strided_memory(q, sq, B, H, Nq, d, 2),
                           dense_memory(means, n * vitattn::means_pitch(d)), dense_memory(scales, n * 4)};
    if (outputs_meet(used, 1, 4)) return VITATTN_E_INVAL;
    vitattn::SelectArgs a = {};
    a.x = static_cast<const uint16_t*>(q);
    a.mx = to_map(sq);
    a.means = static_cast<int8_t*>(const_cast<void*>(means));
    a.scales = const_cast<float*>(scales);
    a.blocks = blocks;
    a.B = B;
    a.H = H;
    a.Hk = Hk;
    a.N = Nq;
    a.d = d;
    a.nb = nb;
    a.q_block = q_block;
    a.groups = groups;
    a.topk = topk;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_select(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_block_fwd_workspace_bytes(int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block, int topk) {
  vitattn::SparseArgs a = {};
  if (check_sparse(a, B, H, Hk, Nq, Nk, d, block, q_block, topk) != VITATTN_OK) return 0;
  return vitattn::sparse_fwd_workspace_bytes(a);
}

int vitattn_block_fwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                      vitattn_strides sv, const int* blocks, const int* key_lens, void* o, vitattn_strides so,
                      float* o32, float* lse, int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block,
                      int topk, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    vitattn::SparseArgs a = {};
    const int st = check_sparse(a, B, H, Hk, Nq, Nk, d, block, q_block, topk);
    if (st != VITATTN_OK) return st;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || (o32 && !aligned16(o32)) ||
        (lse && !aligned16(lse)) || !aligned_to(blocks, 4) || (key_lens && !aligned_to(key_lens, 4)))
      return VITATTN_E_INVAL;
    if (!scale_ok(scale)) return VITATTN_E_INVAL;
    if (check_rows(sq, B, H, Nq, d, false) || check_rows(sk, B, Hk, Nk, d, false) || check_rows(sv, B, Hk, Nk, d, false) ||
        check_rows(so, B, H, Nq, d, true))
      return VITATTN_E_INVAL;
    const size_t need = vitattn::sparse_fwd_workspace_bytes(a), rows = (size_t)B * H * Nq;
    if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return VITATTN_E_WORKSPACE;
    const Memory used[] = {strided_memory(o, so, B, H, Nq, d, 2), dense_memory(o32, rows * d * 4), dense_memory(lse, rows * 4),
                           dense_memory(need > 0 ? workspace : nullptr, need), strided_memory(q, sq, B, H, Nq, d, 2),
                           strided_memory(k, sk, B, Hk, Nk, d, 2), strided_memory(v, sv, B, Hk, Nk, d, 2),
                           dense_memory(blocks, blocks_bytes(a)), dense_memory(key_lens, (size_t)B * 4)};
    if (outputs_meet(used, 4, 9)) return VITATTN_E_INVAL;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.blocks = blocks;
    a.key_lens = key_lens;
    a.o = static_cast<uint16_t*>(o);
    a.o32 = o32;
    a.lse = lse;
    a.work = static_cast<char*>(workspace);
    a.mq = to_map(sq);
    a.mk = to_map(sk);
    a.mv = to_map(sv);
    a.mo = to_map(so);
    a.scale = scale;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_sparse_fwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

size_t vitattn_block_bwd_workspace_bytes(int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block, int topk) {
  vitattn::SparseArgs a = {};
  if (check_sparse(a, B, H, Hk, Nq, Nk, d, block, q_block, topk) != VITATTN_OK) return 0;
  return check_sparse_bwd(a) != VITATTN_OK ? 0 : vitattn::sparse_bwd_workspace_bytes(a);
}

int vitattn_block_bwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                      vitattn_strides sv, const int* blocks, const int* key_lens, const float* o32, const float* lse,
                      const void* dout, vitattn_strides sdo, void* dq, vitattn_strides sdq, void* dk,
                      vitattn_strides sdk, void* dv, vitattn_strides sdv, int B, int H, int Hk, int Nq, int Nk, int d,
                      int block, int q_block, int topk, float scale, void* workspace, size_t workspace_bytes,
                      void* stream) {
  try {
    vitattn::SparseArgs a = {};
    int st = check_sparse(a, B, H, Hk, Nq, Nk, d, block, q_block, topk);
    if (st != VITATTN_OK) return st;
    if ((st = check_sparse_bwd(a)) != VITATTN_OK) return st;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o32) || !aligned16(lse) || !aligned16(dout) ||
        !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned_to(blocks, 4) || (key_lens && !aligned_to(key_lens, 4)))
      return VITATTN_E_INVAL;
    if (!scale_ok(scale)) return VITATTN_E_INVAL;
    if (check_rows(sq, B, H, Nq, d, false) || check_rows(sk, B, Hk, Nk, d, false) || check_rows(sv, B, Hk, Nk, d, false) ||
        check_rows(sdo, B, H, Nq, d, false) || check_rows(sdq, B, H, Nq, d, true) || check_rows(sdk, B, Hk, Nk, d, true) ||
        check_rows(sdv, B, Hk, Nk, d, true))
      return VITATTN_E_INVAL;
    const size_t need = vitattn::sparse_bwd_workspace_bytes(a), rows = (size_t)B * H * Nq;
    if (!aligned16(workspace) || workspace_bytes < need) return VITATTN_E_WORKSPACE;
    const Memory used[] = {strided_memory(dq, sdq, B, H, Nq, d, 2), strided_memory(dk, sdk, B, Hk, Nk, d, 2),
                           strided_memory(dv, sdv, B, Hk, Nk, d, 2), dense_memory(workspace, need),
                           strided_memory(q, sq, B, H, Nq, d, 2), strided_memory(k, sk, B, Hk, Nk, d, 2),
                           strided_memory(v, sv, B, Hk, Nk, d, 2), strided_memory(dout, sdo, B, H, Nq, d, 2),
                           dense_memory(o32, rows * d * 4), dense_memory(lse, rows * 4), dense_memory(blocks, blocks_bytes(a)),
                           dense_memory(key_lens, (size_t)B * 4)};
    if (outputs_meet(used, 4, 12)) return VITATTN_E_INVAL;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.blocks = blocks;
    a.key_lens = key_lens;
    a.o32 = const_cast<float*>(o32);
    a.lse = const_cast<float*>(lse);
    a.dout = static_cast<const uint16_t*>(dout);
    a.dq = static_cast<uint16_t*>(dq);
    a.dk = static_cast<uint16_t*>(dk);
    a.dv = static_cast<uint16_t*>(dv);
    a.work = static_cast<char*>(workspace);
    a.mq = to_map(sq);
    a.mk = to_map(sk);
    a.mv = to_map(sv);
    a.mg = to_map(sdo);
    a.mdq = to_map(sdq);
    a.mdk = to_map(sdk);
    a.mdv = to_map(sdv);
    a.scale = scale;
    a.stream = static_cast<hipStream_t>(stream);
    return vitattn::launch_sparse_bwd(a) == hipSuccess ? VITATTN_OK : VITATTN_E_HIP;
  } catch (...) {
    return VITATTN_E_INTERNAL;
  }
}

}  // extern "C"
