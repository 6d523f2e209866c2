// dQ of the attention over chosen key blocks (vitattn_sparse_bwd.hip).
#include "vitattn_sparse_bwd.h"

namespace vitattn {

namespace {

// A workgroup of NW waves = 32 NW queries, Q and dO held; the listed blocks' K and V
// stream through a ring of four slots in tiles of 32 keys. Per tile: S^T = K Q^T, dP^T =
// V dO^T (from -D), dS^T, dQ^T += K^T dS^T.
template <int D, int KS, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, D <= 96 ? 2 : 1) void sparse_dq_kernel(const SparseArgs a, const float* __restrict__ stats, int n_qtiles, int total, float c) {
  constexpr int BM = 32 * NW, BN = 32, RING = 4, PF = 3, NT = 64 * NW;
  constexpr int NC = (KS + 1) / 2;
  constexpr int T = BN * D * 2;
  static_assert(!MASKED || BM == 64, "a bit per row");
  __shared__ __attribute__((aligned(1024))) char kbuf0[T];
  __shared__ __attribute__((aligned(1024))) char kbuf1[T];
  __shared__ __attribute__((aligned(1024))) char kbuf2[T];
  __shared__ __attribute__((aligned(1024))) char kbuf3[T];
  __shared__ __attribute__((aligned(1024))) char vbuf0[T];
  __shared__ __attribute__((aligned(1024))) char vbuf1[T];
  __shared__ __attribute__((aligned(1024))) char vbuf2[T];
  __shared__ __attribute__((aligned(1024))) char vbuf3[T];
  __shared__ BlockList<MASKED> list;
  __shared__ uint32_t bad[NW];
  char* const kbuf[RING] = {kbuf0, kbuf1, kbuf2, kbuf3};
  char* const vbuf[RING] = {vbuf0, vbuf1, vbuf2, vbuf3};
  debug_poison_lds(kbuf0, kbuf1, kbuf2, kbuf3, vbuf0, vbuf1, vbuf2, vbuf3, list, bad);

  const int work = xcd_remap(blockIdx.x, total);
  const int bh = work / n_qtiles, qt = work - bh * n_qtiles;
  const int b = bh / a.H, head = bh - b * a.H, hk = head / (a.H / a.Hk);
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qrow = qt * BM + wave * 32 + (lane & 31);
  const int Nk = sparse_keys(a, b), real = (Nk + a.block - 1) / a.block;
  const Chosen chosen(a, bh, qt * BM, BM);
  const int tiles = a.block / BN;

  const int chr = a.d >> 3;
  const int ldq = 2 * a.mq.ld, ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld, ldg = 2 * a.mg.ld;
  bf16x8 qf[KS], gf[KS];
  {
    const rsrc_t rq = make_rsrc(a.q + b * a.mq.sb + head * a.mq.sh, (unsigned)(a.Nq * ldq));
    const rsrc_t rg = make_rsrc(a.dout + b * a.mg.sb + head * a.mg.sh, (unsigned)(a.Nq * ldg));
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      qf[kk] = as_bf16x8(buffer_load16(rq, chunk_offset(qrow, 2 * kk + h, ldq, chr)));
      gf[kk] = as_bf16x8(buffer_load16(rg, chunk_offset(qrow, 2 * kk + h, ldg, chr)));
    }
  }
  const int blocks32 = (a.Nq + 31) / 32;
  const bool row_there = qrow < 32 * blocks32;
  const float* const st = stats + ((long long)bh * blocks32 + (qrow >> 5)) * kStat + (qrow & 31);
  const float nd = row_there ? st[0] : 0.f, lse2 = row_there ? st[32] : INFINITY;

  const rsrc_t rk = make_rsrc(a.k + b * a.mk.sb + hk * a.mk.sh, (unsigned)(Nk * ldk));
  const rsrc_t rv = make_rsrc(a.v + b * a.mv.sb + hk * a.mv.sh, (unsigned)(Nk * ldv));
  TileDma<D, BN, NW> dma, dmv;
  dma.init(wave, lane, ldk, chr);
  dmv.init(wave, lane, ldv, chr);
  constexpr int PW = decltype(dma)::PER_WAVE, NREQ = 2 * PW;
  auto request = [&](auto slot_tag, int key0, int r) __attribute__((always_inline)) {
    constexpr int SL = decltype(slot_tag)::value;
    if (r < PW) dma.issue_one(rk, key0, ldk, kbuf[SL], r);
    else dmv.issue_one(rv, key0, ldv, vbuf[SL], r - PW);
  };
  RowFrag<D> rf;
  TrFrag<D> tf;
  rf.init(lane);
  tf.init(lane);
  f32x16 acc[NC];  // dQ^T
  constexpr bool HELD = D <= 96;  // dP starts at -D: held where there are registers
  f32x16 start;
#pragma unroll
  for (int r = 0; r < 16; ++r) start[r] = nd;

  auto attend = [&](int n) __attribute__((always_inline)) {
    const int n_kt = n * tiles;
    TileAt ahead{0, 0};
    int keys[RING];    // first key of the tile in each slot, and its entry
    int entry[RING];
    static_for<0, PF>([&](auto SC) __attribute__((always_inline)) {
      constexpr int s = decltype(SC)::value;
      entry[s] = min(ahead.e, n);
      keys[s] = list.key_of(list.id[entry[s]], a.block, Nk) + ahead.s * BN;
      ahead.next(tiles);
#pragma unroll
      for (int r = 0; r < NREQ; ++r) request(SC, keys[s], r);
    });
    uint32_t raw_id = list.id[min(ahead.e, n)];  // of the tile that the next stage requests
    wait_vmem();
    __syncthreads();
    // Tile j's scores are in s; the stream of ops runs dP(j), the scores of tile j + 1 and
    // dQ += K(j)^T dS(j), the vector work of tile j spread over the first two.
    constexpr int NP = KS, NS = KS, NQ = 2 * NC, NOPS = NP + NS + NQ;
    constexpr auto exp_at = [](int r) { return r * (NP + NS - 2) / 16; };
    constexpr auto ds_at = [](int r) { return NP + 1 + r * (NS + NC - 2) / 16; };
    static_assert(ds_at(7) <= NP + NS - 2 && ds_at(15) <= NP + NS + NC - 2, "dS before dQ");
    static_assert(exp_at(15) <= ds_at(0) || exp_at(15) < ds_at(8), "P before dS");
    static_assert(NREQ <= NOPS, "requests fit the op stream");
    // keys past the last: P = 0
    auto cut = [&](f32x16& s, int key0) __attribute__((always_inline)) {
      if (key0 + BN > Nk)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + acc_row(r, h) >= Nk) s[r] = -INFINITY;
    };
    f32x16 sa = zero16(), sb;
#pragma unroll
    for (int i = 0; i < KS; ++i) sa = mfma32(lds_frag_row(kbuf0, rf.at(i)), qf[i], sa);
    cut(sa, keys[0]);
    bf16x8 lead[2] = {lds_frag_row(vbuf0, rf.at(0)), lds_frag_row(vbuf0, rf.at(1))};
    auto stage = [&](auto slot_tag, f32x16& s, f32x16& sn) __attribute__((always_inline)) {
      constexpr int SL = decltype(slot_tag)::value, NX = (SL + 1) % RING, RF = (SL + PF) % RING;
      // of a block that the row did not choose P = exp2(s - inf) = 0
      float lse_of = lse2;
      if constexpr (MASKED)
        if (!((reinterpret_cast<const uint32_t*>(list.masks)[2 * entry[SL] + wave] >> (lane & 31)) & 1)) lse_of = INFINITY;
      entry[RF] = min(ahead.e, n);
      keys[RF] = list.key_of(raw_id, a.block, Nk) + ahead.s * BN;
      ahead.next(tiles);
      raw_id = list.id[min(ahead.e, n)];
      f32x16 dp;
      if constexpr (!HELD)
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = nd;
      bf16x8 db[2];
      bf16x8 aq[3];
      auto load_op = [&](int i) -> bf16x8 {
        if (i >= NOPS) return lds_frag_row(vbuf[NX], rf.at(i - NOPS));
        if (i < NP) return lds_frag_row(vbuf[SL], rf.at(i));
        if (i < NP + NS) return lds_frag_row(kbuf[NX], rf.at(i - NP));
        return tf.load(kbuf[SL], 16 * ((i - NP - NS) / NC), (i - NP - NS) % NC);
      };
      aq[0] = lead[0];
      aq[1] = lead[1];
      sched_fence();
      static_for<0, NOPS>([&](auto IC) __attribute__((always_inline)) {
        constexpr int i = decltype(IC)::value;
        if constexpr (i == 0) __builtin_amdgcn_s_setprio(1);
        if constexpr (i + 2 < NOPS) aq[(i + 2) % 3] = load_op(i + 2);
        else lead[i + 2 - NOPS] = load_op(i + 2);
        if constexpr (i < NP) {
          dp = mfma32(aq[i % 3], gf[i], HELD && i == 0 ? start : dp);
        } else if constexpr (i < NP + NS) {
          if constexpr (i == NP) sn = zero16();
          sn = mfma32(aq[i % 3], qf[i - NP], sn);
        } else {
          constexpr int t = i - NP - NS;
          acc[t % NC] = mfma32(aq[i % 3], db[t / NC], acc[t % NC]);
        }
        if constexpr (i < NREQ) request(std::integral_constant<int, RF>{}, keys[RF], i);
        static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          if constexpr (exp_at(r) == i) {
            float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse_of));
            pin(x);
            s[r] = x;
          }
        });
        static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          if constexpr (ds_at(r) == i) {
            float x = s[r] * dp[r];
            pin(x);
            s[r] = x;
            if constexpr ((r & 7) == 7) db[r >> 3] = acc_to_operand(s, r >> 3);
          }
        });
        if constexpr (i == NOPS - 1) cut(sn, keys[NX]);
        sched_fence();
      });
      __builtin_amdgcn_s_setprio(0);
      wait_vmem_leave<(PF - 2) * 2 * (decltype(dma)::ALL_ACTIVE ? PW : 0)>();
      barrier_lds();
    };
    const int padded_tiles = (n_kt + RING - 1) / RING * RING;
    for (int j = 0; j < padded_tiles; j += RING) {
      stage(std::integral_constant<int, 0>{}, sa, sb);
      stage(std::integral_constant<int, 1>{}, sb, sa);
      stage(std::integral_constant<int, 2>{}, sa, sb);
      stage(std::integral_constant<int, 3>{}, sb, sa);
    }
    wait_vmem();
    __syncthreads();
  };

  uint64_t filter = ~0ULL, again = 0;
  while (filter != 0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) acc[i] = zero16();
    const int count = list.template build<NT>(a, chosen, real, filter);
    for (int r = 0; r < count; r += list.kCap) {
      const int n = min(count - r, list.kCap);
      list.template fill<NT>(a, chosen, real, filter, r, n);
      attend(n);
    }
    if (qrow < a.Nq && (!MASKED || ((filter >> (wave * 32 + (lane & 31))) & 1))) {
      uint16_t* const out = a.dq + b * a.mdq.sb + head * a.mdq.sh + (long long)qrow * a.mdq.ld;
#pragma unroll
      for (int cb = 0; cb < NC; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          if (col < a.d)
            store4_bf16(out + col, acc[cb][4 * g] * a.scale, acc[cb][4 * g + 1] * a.scale, acc[cb][4 * g + 2] * a.scale,
                        acc[cb][4 * g + 3] * a.scale);
        }
    }
    if constexpr (!MASKED) break;
    if (filter == ~0ULL) {
      float x = 0.f;
#pragma unroll
      for (int cb = 0; cb < NC; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) x = __builtin_fmaf(acc[cb][r], 0.f, x);
      const uint64_t lanes = __ballot(!(x == 0.f) && qrow < a.Nq);
      if (lane == 0) bad[wave] = (uint32_t)lanes | (uint32_t)(lanes >> 32);
      __syncthreads();
      again = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)bad[NW - 1]) << 32 |
              (uint32_t)__builtin_amdgcn_readfirstlane((int)bad[0]);
    }
    filter = again & -again;
    again &= again - 1;
  }
}

template <int D, int KS, int NW, bool MASKED>
hipError_t go(const SparseArgs& a, const SparseWork& w) {
  const int n_qtiles = (a.Nq + 32 * NW - 1) / (32 * NW), total = a.B * a.H * n_qtiles;
  sparse_dq_kernel<D, KS, NW, MASKED><<<total, 64 * NW, 0, a.stream>>>(a, w.stats, n_qtiles, total, a.scale * kLog2e);
  return hipGetLastError();
}
template <int D, int KS>
hipError_t go_tile(const SparseArgs& a, const SparseWork& w) {
  if (one_group(a, 128) && a.Nq > 64) return go<D, KS, 4, false>(a, w);
  return one_group(a, 64) ? go<D, KS, 2, false>(a, w) : go<D, KS, 2, true>(a, w);
}

}  // namespace

hipError_t launch_sparse_dq(const SparseArgs& a, const SparseWork& w) {
  switch (tile_width(a.d)) {
    case 64: return go_tile<64, 4>(a, w);
    case 96: return a.d <= 80 ? go_tile<96, 5>(a, w) : go_tile<96, 6>(a, w);
    case 128: return go_tile<128, 8>(a, w);
    default: return go_tile<160, 10>(a, w);
  }
}

}  // namespace vitattn
