// Attention of groups of queries over the key blocks that each group chose, forward.
// Row i of head h attends to the union of the blocks blocks[b][h][i / q_block][..]
// within the sample's keys:
//
//   O_i = sum_j P_ij V_j,  P_ij = exp(scale q_i . k_j - LSE_i)
//
// An online softmax as in vitattn_fwd.hip, over a list of tiles instead of all of them.
// A workgroup of NW waves owns 32 NW consecutive queries of one head. It first lists in
// LDS the blocks that any of its rows chose (BlockList), then streams their keys in
// tiles of 32 or 64 (32 * KB) through the pipeline of vitattn_fwd.hip: one stream of score ops
// (tile j + 1) then PV ops (tile j), operands read two ops ahead, exponentials, tile requests
// and the next maximum spread over it. Keys past the last arrive as zeros, their scores
// are masked.
//
// Where a tile's rows belong to one group (q_block a multiple of its rows) they share
// the list. Else (MASKED) the list is the union of what 64 rows chose, with 64 bits per
// block for the rows that did: the others subtract a maximum of +inf, so that their P is 0,
// with no work per score. A block costs the tile the same whether one row chose it or all,
// so neighbouring queries should choose alike. What a row did not choose must not reach
// it, also where it is not finite: zero times an infinite V is NaN, so a tile whose outputs are not all finite goes over its
// rows again, one at a time, each with the blocks of its own (of a split: of the split's).
//
// Bound by vector work beside the matrix cores where rows share a list: 4 heads of 188,416
// queries in groups of 128, each 16 blocks of 128 keys (d = 64), 480 us, 0.83 PFLOP/s; 8 heads
// of 32,768 in groups of 64, each 32 blocks: 227-250 us, vector units busy 57 %, matrix cores
// 37 %. Rows that choose apart (8,003 rows, 8 of 126 blocks each, 64 of them 45 together):
// 127 us, 15 of them the lists.
//
// Few queries (SPLIT): the list is split over workgroups, each writes its normalised
// outputs and LSE, and a second kernel joins them, O = sum_s exp(LSE_s - LSE) O_s. One
// query of 8 heads over 32 blocks of 128 keys (d = 128): 8.9 us in 32 splits and 4.0 for the
// join, latencies both.
//
// P is rounded to bf16 as the matrix cores' operand (its sum is of the fp32 values);
// scores, statistics and sums are fp32; o is rounded once. The backward takes the
// unrounded outputs (o32), since it subtracts dO . O from every dP.
#include "vitattn_sparse.h"

namespace vitattn {

namespace {

constexpr int kMaxSplits = 32;

// see vitattn_fwd.hip: score e of 16*KB per lane is exponentiated in slot
// e*W/(16*KB), two slots before the PV op that reads it
constexpr bool exp_fits(int NS, int CPB, int KB, int W) {
  for (int t = 0; t < 2 * KB; ++t)
    if ((8 * t + 7) * W / (16 * KB) > NS + CPB * t - 2) return false;
  return true;
}
constexpr int exp_window(int NS, int CPB, int KB, int NOPS) {
  int w = NOPS - 5;
  while (w > 1 && !exp_fits(NS, CPB, KB, w)) --w;
  return w;
}

template <int D, int KS, int KB, int NW, bool MASKED, bool SPLIT>
__global__ __launch_bounds__(64 * NW, MASKED && D > 96 ? 1 : D == 64 && (NW == 4 || (KB == 1 && !MASKED)) ? 3 : 2) void sparse_fwd_kernel(const SparseArgs a, int n_qtiles, int n_split, int total,
                                                                float c) {
  constexpr int BM = 32 * NW, BN = 32 * KB, NT = 64 * NW;
  constexpr int TILE = BN * D * 2;
  constexpr int NS = KB * KS;        // score ops per tile
  constexpr int CPB = D / 32;        // PV ops per 16-key step
  constexpr int NV = 2 * KB * CPB;   // PV ops per tile
  static_assert(!MASKED || BM == 64, "a bit per row");
  __shared__ __attribute__((aligned(1024))) char kbuf0[TILE];
  __shared__ __attribute__((aligned(1024))) char kbuf1[TILE];
  __shared__ __attribute__((aligned(1024))) char vbuf0[TILE];
  __shared__ __attribute__((aligned(1024))) char vbuf1[TILE];
  __shared__ BlockList<MASKED> list;
  __shared__ uint32_t bad[NW];
  char* const kbuf[2] = {kbuf0, kbuf1};
  char* const vbuf[2] = {vbuf0, vbuf1};
  debug_poison_lds(kbuf0, kbuf1, vbuf0, vbuf1, list, bad);

  const int work = xcd_remap(blockIdx.x, total);
  const int part = work / n_qtiles;
  const int qt = work - part * n_qtiles;
  const int bh = SPLIT ? part / n_split : part;
  const int sp = SPLIT ? part - bh * n_split : 0;
  const int b = bh / a.H, head = bh - b * a.H, hk = head / (a.H / a.Hk);
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qrow = qt * BM + wave * 32 + (lane & 31);
  const int Nk = sparse_keys(a, b), real = (Nk + a.block - 1) / a.block;
  const Chosen chosen(a, bh, qt * BM, BM);
  const int tiles = a.block / BN;  // of a block

  const int chr = a.d >> 3;  // 16-byte chunks of a row that hold data
  const int ldq = 2 * a.mq.ld, ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld;
  const rsrc_t rq = make_rsrc(a.q + b * a.mq.sb + head * a.mq.sh, (unsigned)(a.Nq * ldq));
  const rsrc_t rk = make_rsrc(a.k + b * a.mk.sb + hk * a.mk.sh, (unsigned)(Nk * ldk));
  const rsrc_t rv = make_rsrc(a.v + b * a.mv.sb + hk * a.mv.sh, (unsigned)(Nk * ldv));

  bf16x8 qf[KS];  // B operands of K Q^T
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) qf[kk] = as_bf16x8(buffer_load16(rq, chunk_offset(qrow, 2 * kk + h, ldq, chr)));

  TileDma<D, BN, NW> dma, dmv;
  dma.init(wave, lane, ldk, chr);
  dmv.init(wave, lane, ldv, chr);
  RowFrag<D> kfrag;
  kfrag.init(lane);
  TrFrag<D> vfrag;
  vfrag.init(lane);

  f32x16 oacc[CPB];
  float m_run, l_part;

  constexpr int NE = 16 * KB;
  // scores of keys past the last are -inf
  auto mask = [&](f32x16 (&s)[KB], int key0) __attribute__((always_inline)) {
    if (key0 + BN > Nk) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + kb * 32 + acc_row(r, h) >= Nk) s[kb][r] = -INFINITY;
    }
  };
  // x where the lane's row chose the block (of the wave's bits), or else what stands for it
  auto chose = [&](uint32_t rows, float x, float other) __attribute__((always_inline)) {
    return !MASKED || ((rows >> (lane & 31)) & 1) ? x : other;
  };
  // the wave's 32 bits of entry e's mask
  auto rows_of = [&](int e) __attribute__((always_inline)) -> uint32_t {
    if constexpr (MASKED) return reinterpret_cast<const uint32_t*>(list.masks)[2 * e + wave];
    else return 0xffffffffu;
  };
  auto uniform = [](uint32_t x) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
  auto max_quarter = [&](const f32x16 (&s)[KB], int q) {
    float m = -INFINITY;
#pragma unroll
    for (int e = q * NE / 4; e < (q + 1) * NE / 4; ++e) m = fmaxf(m, s[e / 16][e % 16]);
    return m;
  };
  auto fold_max = [&](float mx) __attribute__((always_inline)) {
    if (__any(mx * c > m_run)) {
      const float m_new = fmaxf(m_run, max_halves(mx) * c);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_part *= alpha;
#pragma unroll
      for (int cb = 0; cb < CPB; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[cb][r] *= alpha;
    }
  };

  // Stage j as in vitattn_fwd.hip: s holds tile j's scores, sn gets tile j + 1's (of
  // key0 k1 and the rows' bits r1); K of tile j + 2 (k2) and V of tile j + 1 are requested.
  // A wave none of whose rows chose either tile (r0, r1) has the requests alone.
  auto stage = [&](auto parity, auto has_next, f32x16 (&s)[KB], f32x16 (&sn)[KB], int k1, int k2, uint32_t r0, uint32_t r1) __attribute__((always_inline)) {
    constexpr int P = decltype(parity)::value;
    constexpr bool NEXT = decltype(has_next)::value;
    const char* ks = kbuf[1 - P];
    const char* vs = vbuf[P];
    if constexpr (MASKED && NEXT) {
      if ((r0 | r1) == 0) {
        dma.issue(rk, k2, ldk, kbuf[P]);
        dmv.issue(rv, k1, ldv, vbuf[1 - P]);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sn[kb][r] = 0.f;
        wait_vmem();
        __syncthreads();
        return;
      }
    }
    const float m_cur = chose(r0, m_run, INFINITY);  // (P = exp2(s - inf) = 0)
    float ls0 = 0.f, ls1 = 0.f;
    u32x4 pq[2 * KB];
    float xe[NE];
    auto exp_slice = [&](auto I, auto WC) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value;
      constexpr int W = decltype(WC)::value;
      static_for<0, NE>([&](auto EC) __attribute__((always_inline)) {
        constexpr int e = decltype(EC)::value;
        if constexpr (e * W / NE == i) {
          xe[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 16][e % 16], c, -m_cur));
          if constexpr ((e & 1) != 0) {
            const bf16x2 pr2 = {(__bf16)xe[e - 1], (__bf16)xe[e]};
            ls0 += xe[e - 1];
            ls1 += xe[e];
            pin(ls0);
            pin(ls1);
            constexpr int pr = e / 2;
            pq[pr / 4][pr % 4] = __builtin_bit_cast(uint32_t, pr2);
          }
        }
      });
    };
    auto pfrag = [&](int t) { return __builtin_bit_cast(bf16x8, pq[t]); };

    if constexpr (NEXT) {
      constexpr int NOPS = NS + NV;
      constexpr int W = exp_window(NS, CPB, KB, NOPS);
      static_assert(exp_fits(NS, CPB, KB, W), "probabilities must be ready before their PV op");
      constexpr int PW = decltype(dma)::PER_WAVE, NDMA = 2 * PW;
      constexpr int STEP = 2 * NDMA <= NOPS ? 2 : 1;
      static_assert(STEP * NDMA <= NOPS, "tile requests must fit the stream");
      auto load_op = [&](int i) -> bf16x8 {
        if (i < NS) return lds_frag_row(ks, (i % KB) * 32 * 2 * D + kfrag.at(i / KB));
        const int t = i - NS;
        return vfrag.load(vs, 16 * (t / CPB), t % CPB);
      };
      float mq[4];
      bf16x8 opq[3];
      opq[0] = load_op(0);
      opq[1] = load_op(1);
      sched_fence();
      static_for<0, NOPS>([&](auto IC) __attribute__((always_inline)) {
        constexpr int i = decltype(IC)::value;
        if constexpr (i == 0) __builtin_amdgcn_s_setprio(2);
        if constexpr (i == W) __builtin_amdgcn_s_setprio(1);
        if constexpr (i == W + 4) __builtin_amdgcn_s_setprio(0);
        if constexpr (i + 2 < NOPS) opq[(i + 2) % 3] = load_op(i + 2);
        if constexpr (i < NS) {
          if constexpr (i / KB == 0) sn[i % KB] = zero16();
          sn[i % KB] = mfma32(opq[i % 3], qf[i / KB], sn[i % KB]);
        } else {
          constexpr int t = i - NS;
          oacc[t % CPB] = mfma32(opq[i % 3], pfrag(t / CPB), oacc[t % CPB]);
        }
        if constexpr (i % STEP == STEP - 1 && i / STEP < NDMA) {
          constexpr int q = i / STEP;
          if constexpr (q < PW) dma.issue_one(rk, k2, ldk, kbuf[P], q);
          else dmv.issue_one(rv, k1, ldv, vbuf[1 - P], q - PW);
        }
        exp_slice(IC, std::integral_constant<int, W>{});
        if constexpr (i >= W && i < W + 4) {
          if constexpr (i == W) mask(sn, k1);
          mq[i - W] = max_quarter(sn, i - W);
          pin(mq[i - W]);
        }
        sched_fence();
      });
      l_part += ls0 + ls1;
      fold_max(chose(r1, fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])), -INFINITY));
      wait_vmem();
      __syncthreads();
    } else {
      exp_slice(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
      bf16x8 vq[3];
      vq[0] = vfrag.load(vs, 0, 0);
      vq[1] = vfrag.load(vs, 16 * (1 / CPB), 1 % CPB);
      sched_fence();
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (i + 2 < NV) vq[(i + 2) % 3] = vfrag.load(vs, 16 * ((i + 2) / CPB), (i + 2) % CPB);
        oacc[i % CPB] = mfma32(vq[i % 3], pfrag(i / CPB), oacc[i % CPB]);
        sched_fence();
      }
      l_part += ls0 + ls1;
    }
  };

  // adds the list's n blocks (n > 0) to the outputs
  auto attend = [&](int n) __attribute__((always_inline)) {
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    f32x16 sa[KB], sb[KB];
    const int n_kt = n * tiles;
    // Tile j + 3's entry is read in stage j and used in the next: a wave does not wait for
    // LDS between two stages. (Past the last block: Nk and more.)
    TileAt at{0, 0};
    auto key_of = [&](uint32_t entry, int s) __attribute__((always_inline)) { return list.key_of(entry, a.block, Nk) + s * BN; };
    const int k0 = key_of(list.id[0], 0);
    uint32_t r0 = uniform(rows_of(0)), r1, r2;
    dma.issue(rk, k0, ldk, kbuf[0]);
    dmv.issue(rv, k0, ldv, vbuf[0]);
    at.next(tiles);
    int k1 = key_of(list.id[at.e], at.s), k2;
    r1 = uniform(rows_of(at.e));
    dma.issue(rk, k1, ldk, kbuf[1]);
    at.next(tiles);
    k2 = key_of(list.id[at.e], at.s);
    r2 = uniform(rows_of(at.e));
    wait_vmem();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (i % KS == 0) sa[i / KS] = zero16();
      sa[i / KS] = mfma32(lds_frag_row(kbuf[0], (i / KS) * 32 * 2 * D + kfrag.at(i % KS)), qf[i % KS], sa[i / KS]);
    }
    mask(sa, k0);
    fold_max(chose(r0, fmaxf(fmaxf(max_quarter(sa, 0), max_quarter(sa, 1)), fmaxf(max_quarter(sa, 2), max_quarter(sa, 3))), -INFINITY));
    __syncthreads();  // kbuf[0] is refilled by the first stage
    uint32_t raw_id, raw_rows;
    auto peek = [&]() __attribute__((always_inline)) {
      at.next(tiles);
      raw_id = list.id[at.e];
      raw_rows = rows_of(at.e);
    };
    // the next stage's tiles
    auto step = [&]() __attribute__((always_inline)) {
      k1 = k2;
      r0 = r1;
      r1 = r2;
      k2 = key_of(raw_id, at.s);
      r2 = uniform(raw_rows);
    };
    int j = 0;
    for (; j + 2 < n_kt; j += 2) {
      peek();
      stage(P0{}, std::true_type{}, sa, sb, k1, k2, r0, r1);
      step();
      peek();
      stage(P1{}, std::true_type{}, sb, sa, k1, k2, r0, r1);
      step();
    }
    if (j + 1 < n_kt) {
      stage(P0{}, std::true_type{}, sa, sb, k1, k2, r0, r1);
      stage(P1{}, std::false_type{}, sb, sa, 0, 0, r1, 0);
    } else {
      stage(P0{}, std::false_type{}, sa, sb, 0, 0, r0, 0);
    }
    __syncthreads();  // before another list's tiles
  };

  // Of a split: the blocks lo .. hi - 1, which all of the tile's rows keep to.
  int lo = 0, hi = 0;
  // The outputs of the rows of `filter` from the blocks that they chose.
  auto rows = [&](uint64_t filter) __attribute__((always_inline)) {
#pragma unroll
    for (int cb = 0; cb < CPB; ++cb) oacc[cb] = zero16();
    m_run = -3.0e38f;  // (finite, so that a tile of scores -inf leaves zeros and not NaN)
    l_part = 0.f;
    const int count = list.template build<NT>(a, chosen, real, filter);
    const bool first = filter == ~0ULL;
    const int r0 = !SPLIT ? 0 : first ? (int)((long long)count * sp / n_split) : list.below(lo, a.nb, count);
    const int r1 = !SPLIT ? count : first ? (int)((long long)count * (sp + 1) / n_split) : list.below(hi, a.nb, count);
    // A row that chose nothing of the split goes on to the next one's build, which clears what
    // the other wave still reads here.
    if (SPLIT && !first) __syncthreads();
    if constexpr (MASKED) {
      for (int r = r0; r < r1; r += list.kCap) {
        const int n = min(r1 - r, list.kCap);
        list.template fill<NT>(a, chosen, real, filter, r, n);
        if (SPLIT && first) {
          if (r == r0) lo = __builtin_amdgcn_readfirstlane((int)list.id[0]);
          hi = __builtin_amdgcn_readfirstlane((int)list.id[n - 1]) + 1;
        }
        attend(n);
      }
    } else if (r1 > r0) {  // (one group's are never more)
      list.template fill<NT>(a, chosen, real, filter, r0, r1 - r0);
      attend(r1 - r0);
    }
    const float l = sum_halves(l_part);
    // (a row without keys, or whose scores are all -inf: zeros and an LSE of -inf)
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const float lse = (m_run + __log2f(l)) * kLn2;
    if (qrow < a.Nq && (!MASKED || ((filter >> (wave * 32 + (lane & 31))) & 1))) {
      const long long row = SPLIT ? ((long long)bh * n_split + sp) * a.Nq + qrow : (long long)bh * a.Nq + qrow;
      float* const share = reinterpret_cast<float*>(a.work);
      float* const o32 = SPLIT ? share + row * a.d : a.o32 ? a.o32 + row * a.d : nullptr;
      float* const ol = SPLIT ? share + (long long)a.B * a.H * n_split * a.Nq * a.d + row : a.lse ? a.lse + row : nullptr;
      uint16_t* const orow = a.o + b * a.mo.sb + head * a.mo.sh + (long long)qrow * a.mo.ld;
#pragma unroll
      for (int cb = 0; cb < CPB; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          if (col >= a.d) continue;
          const float4 x = make_float4(oacc[cb][4 * g] * inv, oacc[cb][4 * g + 1] * inv, oacc[cb][4 * g + 2] * inv,
                                       oacc[cb][4 * g + 3] * inv);
          if (o32) *reinterpret_cast<float4*>(o32 + col) = x;
          if (!SPLIT) store4_bf16(orow + col, x.x, x.y, x.z, x.w);
        }
      if (h == 0 && ol) *ol = lse;
    }
  };

  if constexpr (!MASKED) {
    rows(~0ULL);
  } else {
    uint64_t filter = ~0ULL, again = 0;
    while (filter != 0) {
      rows(filter);
      if (filter == ~0ULL) {
        float x = 0.f;  // NaN if any output is not finite
#pragma unroll
        for (int cb = 0; cb < CPB; ++cb)
#pragma unroll
          for (int r = 0; r < 16; ++r) x = __builtin_fmaf(oacc[cb][r], 0.f, x);
        const uint64_t lanes = __ballot(!(x == 0.f) && qrow < a.Nq);
        if (lane == 0) bad[wave] = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        __syncthreads();
        again = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)bad[1]) << 32 |
                (uint32_t)__builtin_amdgcn_readfirstlane((int)bad[0]);
      }
      filter = again & -again;
      again &= again - 1;
    }
  }
}

// Joins the splits (at most kMaxSplits) of one query row: a wave per row and 64 columns,
// all of its loads on their way at once.
__global__ __launch_bounds__(64) void sparse_join_kernel(const SparseArgs a, int n_split) {
  const long long row = blockIdx.x, rows = (long long)a.B * a.H * a.Nq;
  const int lane = threadIdx.x, col = 64 * blockIdx.y + lane;
  const long long bh = row / a.Nq;
  const int i = (int)(row - bh * a.Nq), b = (int)(bh / a.H), head = (int)(bh - (long long)b * a.H);
  const float* const share = reinterpret_cast<const float*>(a.work);
  const float* const outs = share + (bh * n_split * a.Nq + i) * a.d + min(col, a.d - 1);
  const float* const lses = share + rows * n_split * a.d + bh * n_split * a.Nq + i;
  const float mine = lane < n_split ? lses[(long long)lane * a.Nq] : -INFINITY;
  float x[kMaxSplits];
#pragma unroll
  for (int s = 0; s < kMaxSplits; ++s) x[s] = outs[(long long)min(s, n_split - 1) * a.Nq * a.d];
  float top = mine;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const float ref = top == -INFINITY ? 0.f : top;
  const float weight = mine == -INFINITY ? 0.f : expf(mine - ref);  // of the lane's split
  const uint32_t there = (uint32_t)__ballot(mine != -INFINITY);
  float o = 0.f, sum = 0.f;
#pragma unroll
  for (int s = 0; s < kMaxSplits; ++s) {
    const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), s));
    sum += w;
    o += (there >> s) & 1 ? w * x[s] : 0.f;
  }
  if (lane == 0 && blockIdx.y == 0 && a.lse) a.lse[row] = top == -INFINITY ? -INFINITY : ref + logf(sum);
  if (col >= a.d) return;
  const float y = sum == 0.f ? 0.f : o / sum;
  if (a.o32) a.o32[row * a.d + col] = y;
  a.o[b * a.mo.sb + head * a.mo.sh + (long long)i * a.mo.ld + col] = __builtin_bit_cast(uint16_t, (__bf16)y);
}

template <int D, int KS, int KB, int NW, bool MASKED, bool SPLIT>
hipError_t go(const SparseArgs& a, int n_split) {
  const int n_qtiles = (a.Nq + 32 * NW - 1) / (32 * NW);
  const int total = a.B * a.H * n_split * n_qtiles;
  sparse_fwd_kernel<D, KS, KB, NW, MASKED, SPLIT><<<total, 64 * NW, 0, a.stream>>>(a, n_qtiles, n_split, total, a.scale * kLog2e);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || !SPLIT) return err;
  sparse_join_kernel<<<dim3(a.B * a.H * a.Nq, (a.d + 63) / 64), 64, 0, a.stream>>>(a, n_split);
  return hipGetLastError();
}

template <int D, int KS, int KB4, int KB2>
hipError_t go_tile(const SparseArgs& a) {
  const int n_split = sparse_splits(a);
  if (n_split > 1)
    return one_group(a, 64) ? go<D, KS, KB2, 2, false, true>(a, n_split) : go<D, KS, KB2, 2, true, true>(a, n_split);
  if (one_group(a, 128) && a.Nq > 64) return go<D, KS, KB4, 4, false, false>(a, 1);
  return one_group(a, 64) ? go<D, KS, KB2, 2, false, false>(a, 1) : go<D, KS, KB2, 2, true, false>(a, 1);
}

}  // namespace

// Up to 256 queries: at least two tiles of 64 keys for each split of a tile's list,
// at most kMaxSplits.
int sparse_splits(const SparseArgs& a) {
  if (a.Nq > 256) return 1;
  const int in_tile = one_group(a, 64) ? 1 : (min(a.Nq, 64) + a.q_block - 1) / a.q_block + 1;
  const long long most = min((long long)in_tile * a.topk, (long long)a.nb) * (a.block / 64);
  return (int)max(1LL, min((long long)kMaxSplits, most / 2));
}

size_t sparse_fwd_workspace_bytes(const SparseArgs& a) {
  const int s = sparse_splits(a);
  return s > 1 ? (size_t)a.B * a.H * s * a.Nq * (a.d + 1) * sizeof(float) : 0;
}

hipError_t launch_sparse_fwd(const SparseArgs& a) {
  switch (tile_width(a.d)) {
    case 64: return go_tile<64, 4, 2, 1>(a);
    case 96: return a.d <= 80 ? go_tile<96, 5, 2, 1>(a) : go_tile<96, 6, 2, 1>(a);
    case 128: return go_tile<128, 8, 2, 1>(a);
    default: return go_tile<160, 10, 1, 1>(a);
  }
}

}  // namespace vitattn
