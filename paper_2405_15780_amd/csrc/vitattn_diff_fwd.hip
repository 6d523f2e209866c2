// Forward pass of differential attention for gfx950. Per (b, h), over the
// first key_lens[b] keys:
//
//   O_m = softmax(scale Q_m K_m^T) V  (m = 1, 2),   O = O_1 - lam O_2
//
// Two softmaxes with statistics of their own over one V: each map is an online
// softmax (running max and sum) as in vitattn_fwd.hip, and the difference is
// taken in fp32 at the end. A workgroup of 2 QW waves owns 32 QW queries of
// one (b, h); waves w and w + QW share 32 of them and take one map each, so
// the tiles of V (and both maps' K) are fetched once for the two maps and both
// land on the same SIMD (QW = 4), where one wave's exponentials run beside the
// other's matrix ops. K_1, K_2 and V stream through LDS in tiles of 32 KB keys
// (R slots each, K one tile ahead of V), rows past the sample's keys read as
// zeros. The pipeline within a tile is vitattn_fwd.hip's: one stream of
// score ops (tile j + 1) then PV ops (tile j), operands read two ops ahead,
// exponentials, tile requests and the next maximum spread over it.
//
// P is rounded to bf16 as the matrix cores' operand (its sum is of the fp32
// values); scores, statistics, sums and the difference are fp32; o is rounded
// once, at the end. What the backward needs is kept in fp32: it subtracts dO .
// O_m from every dP, and where values share a mean these cancel to a small part
// (kept in bf16, dQ was 1.1 % off at 32,768 keys).
//
// Few queries over many keys (SPLIT): the grid also splits the keys, each
// workgroup writes its maps' normalised outputs and LSE to the workspace, and
// a second kernel joins them, O_m = sum_s exp(LSE_s - LSE) O_s. The split
// depends on Nq and Nk alone, so a head's bits do not depend on the call it is
// part of.
//
// Bound by the vector work beside the matrix cores and the power limit for long
// sequences: 4 heads, 32,768 keys, d = 64, e = 128 3.1 ms, 3.3 TFLOP at 1.06
// PFLOP/s, where a large matrix product runs at 1.35; by one and a third rounds of
// workgroups at 64 heads of 1,024, d = 32 (48 us); by HBM for one query: 8 heads
// over 131,072 keys 106 us with the join (537 MB, 5.1 TB/s), 256 heads over 32,768
// 722 us (5.9 TB/s).
#include "vitattn_diff.h"

namespace vitattn {

namespace {

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

template <int DQ, int QS, int DV, int KB, int QW, int R, bool SPLIT>
__global__ __launch_bounds__(128 * QW, QW == 1 && R == 4 ? 1 : 2) void diff_fwd_kernel(const DiffArgs a, int n_qtiles, int n_split,
                                                               int split_keys, int total, float c) {
  constexpr int NW = 2 * QW;
  constexpr int BM = 32 * QW, BN = 32 * KB;
  constexpr int KT = BN * DQ * 2, VT = BN * DV * 2;  // bytes of a K and a V tile
  constexpr int NS = KB * QS;                        // score ops per tile
  constexpr int CPB = DV / 32;                       // PV ops per 16-key step
  constexpr int NV = 2 * KB * CPB;                   // PV ops per tile
  __shared__ __attribute__((aligned(1024))) char kbuf0[2 * KT];  // K_1, then K_2
  __shared__ __attribute__((aligned(1024))) char kbuf1[2 * KT];
  __shared__ __attribute__((aligned(1024))) char kbuf2[R > 2 ? 2 * KT : 1];
  __shared__ __attribute__((aligned(1024))) char kbuf3[R > 2 ? 2 * KT : 1];
  __shared__ __attribute__((aligned(1024))) char vbuf0[VT];
  __shared__ __attribute__((aligned(1024))) char vbuf1[VT];
  __shared__ __attribute__((aligned(1024))) char vbuf2[R > 2 ? VT : 1];
  __shared__ __attribute__((aligned(1024))) char vbuf3[R > 2 ? VT : 1];
  // The second map's outputs, 32 columns at a time: over the K tiles where these
  // are large enough (no wave reads K in the last stage), which leaves a CU room
  // for another workgroup.
  constexpr bool OVER_K = 2 * KT >= QW * 4096;
  __shared__ float xown[OVER_K ? 1 : QW][16][64];
  static_assert(R == 2 || R == 4, "slots, a multiple of the two score buffers");
  // (selected at compile time: a table of them would be one of generic addresses)
  auto kbuf = [&](auto I) __attribute__((always_inline)) -> char* {
    constexpr int i = decltype(I)::value % R;
    if constexpr (i == 0) return kbuf0;
    else if constexpr (i == 1) return kbuf1;
    else if constexpr (i == 2) return kbuf2;
    else return kbuf3;
  };
  auto vbuf = [&](auto I) __attribute__((always_inline)) -> char* {
    constexpr int i = decltype(I)::value % R;
    if constexpr (i == 0) return vbuf0;
    else if constexpr (i == 1) return vbuf1;
    else if constexpr (i == 2) return vbuf2;
    else return vbuf3;
  };
  debug_poison_lds(kbuf0, kbuf1, kbuf2, kbuf3, vbuf0, vbuf1, vbuf2, vbuf3, xown);
  float(*const xbuf)[16][64] = OVER_K ? reinterpret_cast<float(*)[16][64]>(kbuf0) : xown;

  const int work = work_item(a.key_lens, total);
  const int part = work / n_qtiles;
  const int qt = work - part * n_qtiles;
  const int bh = SPLIT ? part / n_split : part;
  const int sp = SPLIT ? part - bh * n_split : 0;
  const int b = bh / a.H, head = bh - b * a.H;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qw = wave % QW, map = wave / QW;
  const int qrow = qt * BM + qw * 32 + (lane & 31);

  // this workgroup's keys: [key_first, key_first + Nk)
  const int all = keys_of(a.key_lens, b, a.Nk);
  const int key_first = SPLIT ? min(sp * split_keys, all) : 0;
  const int Nk = SPLIT ? min(all - key_first, split_keys) : all;
  // SPLIT: rows of the workspace, [bh][split][map][query] of DV columns (a.e
  // of them used), then as many LSE
  const long long wrow = SPLIT ? (((long long)bh * n_split + sp) * 2 + map) * a.Nq + qrow : 0;
  float* const wo = a.work + wrow * a.e;
  float* const wl = a.work + (long long)a.B * a.H * n_split * 2 * a.Nq * a.e + wrow;
  uint16_t* const orow = a.o + b * a.mo.sb + head * a.mo.sh + (long long)qrow * a.mo.ld;
  float* const mrow = a.maps ? a.maps + (((long long)bh * 2 + map) * a.Nq + qrow) * a.e : nullptr;
  float* const lrow = a.lse ? a.lse + ((long long)bh * 2 + map) * a.Nq + qrow : nullptr;

  if (Nk == 0) {  // the whole workgroup: nothing to attend to, the output is zero
    if (qrow < a.Nq) {
      if (!SPLIT)
        for (int col = 4 * h; col < a.e; col += 8) {
          if (map == 0) put4_bf16(orow + col, 0.f, 0.f, 0.f, 0.f);
          if (mrow) *reinterpret_cast<float4*>(mrow + col) = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      if (h == 0) {
        if (SPLIT) *wl = -INFINITY;  // its outputs are not read
        else if (lrow) *lrow = -INFINITY;
      }
    }
    return;
  }

  const int chr = a.d >> 3, chv = a.e >> 3;  // 16-byte chunks of a row that hold data
  const int ldq = 2 * a.mq.ld, ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld;
  const rsrc_t rq = make_rsrc(a.q + map_head(a.mq, b, head, map), (unsigned)(a.Nq * ldq));
  const rsrc_t rk1 = make_rsrc(a.k + map_head(a.mk, b, head, 0) + (long long)key_first * a.mk.ld, (unsigned)(Nk * ldk));
  const rsrc_t rk2 = make_rsrc(a.k + map_head(a.mk, b, head, 1) + (long long)key_first * a.mk.ld, (unsigned)(Nk * ldk));
  const rsrc_t rv = make_rsrc(a.v + b * a.mv.sb + head * a.mv.sh + (long long)key_first * a.mv.ld, (unsigned)(Nk * ldv));

  bf16x8 qf[QS];  // B operands of K Q^T
#pragma unroll
  for (int kk = 0; kk < QS; ++kk) qf[kk] = as_bf16x8(buffer_load16(rq, chunk_offset(qrow, 2 * kk + h, ldq, chr)));

  TileDma<DQ, BN, NW> dma;
  TileDma<DV, BN, NW> dmv;
  dma.init(wave, lane, ldk, chr);
  dmv.init(wave, lane, ldv, chv);
  RowFrag<DQ> kfrag;
  kfrag.init(lane);
  TrFrag<DV> vfrag;
  vfrag.init(lane);
  // a stage's requests: K_1, K_2 (tile j + R), V (tile j + R - 1)
  constexpr int PK = decltype(dma)::PER_WAVE, PV = decltype(dmv)::PER_WAVE, NDMA = 2 * PK + PV;

  f32x16 oacc[CPB];
#pragma unroll
  for (int cb = 0; cb < CPB; ++cb) oacc[cb] = zero16();
  float m_run = -INFINITY;  // running max of scaled logits, log2 units
  float l_part = 0.f;

  // (tiles past the last are zeros whose scores are masked)
  const int tiles = (Nk + BN - 1) / BN, n_kt = R == 2 ? tiles : (tiles + R - 1) / R * R;
  dma.issue(rk1, 0, ldk, kbuf0);
  dma.issue(rk2, 0, ldk, kbuf0 + KT);
  static_for<1, R>([&](auto T) __attribute__((always_inline)) {
    constexpr int t = decltype(T)::value;
    dma.issue(rk1, t * BN, ldk, kbuf(T));
    dma.issue(rk2, t * BN, ldk, kbuf(T) + KT);
    dmv.issue(rv, (t - 1) * BN, ldv, vbuf(std::integral_constant<int, t - 1>{}));
  });
  wait_vmem_leave<(R - 2) * NDMA>();
  barrier_lds();

  constexpr int NE = 16 * KB;
  auto mask_ragged = [&](f32x16 (&s)[KB], int tile) {
    const int key0 = tile * BN;
    if (key0 + BN > Nk) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + kb * 32 + acc_row(r, h) >= Nk) s[kb][r] = -INFINITY;
    }
  };
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

  f32x16 sa[KB], sb[KB];
  const int koff = map * KT;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    if (i % QS == 0) sa[i / QS] = zero16();
    sa[i / QS] = mfma32(lds_frag_row(kbuf0 + koff, (i / QS) * 32 * 2 * DQ + kfrag.at(i % QS)), qf[i % QS], sa[i / QS]);
  }
  mask_ragged(sa, 0);
  // (finite, so that a first tile of scores -inf leaves zeros and not NaN)
  m_run = fmaxf(max_halves(fmaxf(fmaxf(max_quarter(sa, 0), max_quarter(sa, 1)), fmaxf(max_quarter(sa, 2), max_quarter(sa, 3)))) * c,
                -3.0e38f);
  barrier_lds();  // kbuf0 is refilled by the first stage

  auto stage = [&](auto parity, auto has_next, f32x16 (&s)[KB], f32x16 (&sn)[KB], int j) __attribute__((always_inline)) {
    constexpr int P = decltype(parity)::value;
    constexpr bool NEXT = decltype(has_next)::value;
    const char* ks = kbuf(std::integral_constant<int, P + 1>{}) + koff;
    const char* vs = vbuf(parity);
    const float m_cur = m_run;
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
      // requests on the odd ops where they fit there, else on every op
      constexpr int STEP = 2 * NDMA <= NOPS ? 2 : 1;
      static_assert(STEP * NDMA <= NOPS, "tile requests must fit the stream");
      auto load_op = [&](int i) -> bf16x8 {
        if (i < NS) return lds_frag_row(ks, (i % KB) * 32 * 2 * DQ + kfrag.at(i / KB));
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
          if constexpr (q < PK) dma.issue_one(rk1, (j + R) * BN, ldk, kbuf(parity), q);
          else if constexpr (q < 2 * PK) dma.issue_one(rk2, (j + R) * BN, ldk, kbuf(parity) + KT, q - PK);
          else dmv.issue_one(rv, (j + R - 1) * BN, ldv, vbuf(std::integral_constant<int, P + R - 1>{}), q - 2 * PK);
        }
        exp_slice(IC, std::integral_constant<int, W>{});
        if constexpr (i >= W && i < W + 4) {
          if constexpr (i == W) mask_ragged(sn, j + 1);
          mq[i - W] = max_quarter(sn, i - W);
          pin(mq[i - W]);
        }
        sched_fence();
      });
      l_part += ls0 + ls1;
      fold_max(fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])));
      wait_vmem_leave<(R - 2) * NDMA>();
      barrier_lds();
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

  int j = 0;
  for (; j + R < n_kt; j += R) {
    static_for<0, R / 2>([&](auto IC) __attribute__((always_inline)) {
      constexpr int p = 2 * decltype(IC)::value;
      stage(std::integral_constant<int, p>{}, std::true_type{}, sa, sb, j + p);
      stage(std::integral_constant<int, p + 1>{}, std::true_type{}, sb, sa, j + p + 1);
    });
  }
  if (R > 2 || j + 1 < n_kt) {
    static_for<0, R / 2>([&](auto IC) __attribute__((always_inline)) {
      constexpr int p = 2 * decltype(IC)::value;
      stage(std::integral_constant<int, p>{}, std::true_type{}, sa, sb, j + p);
      stage(std::integral_constant<int, p + 1>{}, std::bool_constant<(p + 2 < R)>{}, sb, sa, j + p + 1);
    });
  } else {
    stage(std::integral_constant<int, 0>{}, std::false_type{}, sa, sb, j);
  }
  wait_vmem();  // requests past the last tile still write LDS

  const float l = sum_halves(l_part);
  // (l is at least 1 but for a query whose scores are all -inf, which has zeros and an
  // LSE of -inf, as a sample without keys has and as the join makes of such splits)
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const float lse = (m_run + __log2f(l)) * kLn2;
  if constexpr (SPLIT) {
    if (qrow < a.Nq) {
#pragma unroll
      for (int cb = 0; cb < CPB; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          if (col < a.e)
            *reinterpret_cast<float4*>(wo + col) = make_float4(oacc[cb][4 * g] * inv, oacc[cb][4 * g + 1] * inv,
                                                               oacc[cb][4 * g + 2] * inv, oacc[cb][4 * g + 3] * inv);
        }
      if (h == 0) *wl = lse;
    }
  } else {
    // the second map's wave hands its outputs over, 32 columns at a time
    const float lam = lam_of(a.lam, a.lam_bf16, head);
#pragma unroll
    for (int cb = 0; cb < CPB; ++cb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[cb][r] *= inv;
      if (map == 1) {
#pragma unroll
        for (int r = 0; r < 16; ++r) xbuf[qw][r][lane] = oacc[cb][r];
      }
      if (mrow && qrow < a.Nq) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          if (col < a.e)
            *reinterpret_cast<float4*>(mrow + col) =
                make_float4(oacc[cb][4 * g], oacc[cb][4 * g + 1], oacc[cb][4 * g + 2], oacc[cb][4 * g + 3]);
        }
      }
      __syncthreads();
      if (map == 0 && qrow < a.Nq) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = oacc[cb][4 * g + e] - lam * xbuf[qw][4 * g + e][lane];
          if (col < a.e) put4_bf16(orow + col, x[0], x[1], x[2], x[3]);
        }
      }
      __syncthreads();
    }
    if (lrow && qrow < a.Nq && h == 0) *lrow = lse;
  }
}

// Joins the splits of one query row (bh, query), a workgroup per row and 64
// columns: Q waves for each map, each of which takes a Q-th of the splits. The
// outputs of U splits are requested beside their LSE, the first U before the
// maximum is known, and added in split order, then the waves' in order.
template <int Q>
__global__ __launch_bounds__(128 * Q) void diff_join_kernel(const DiffArgs a, int n_split) {
  constexpr int U = 16;
  __shared__ float tops[2 * Q], sums[2 * Q], acc[2][Q][64];
  debug_poison_lds(tops, sums, acc);
  const long long row = blockIdx.x, rows = (long long)a.B * a.H * a.Nq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = wave / Q, share = wave % Q, col = 64 * blockIdx.y + lane;
  const long long bh = row / a.Nq;
  const int i = (int)(row - bh * a.Nq);
  const int b = (int)(bh / a.H), head = (int)(bh - (long long)b * a.H);
  const long long base = (bh * n_split * 2 + m) * a.Nq + i, step = 2LL * a.Nq;
  const float* lses = a.work + rows * n_split * 2 * a.e + base;
  const float* outs = a.work + base * a.e;
  // this wave's splits
  const int s0 = (int)((long long)n_split * share / Q), s1 = (int)((long long)n_split * (share + 1) / Q);
  float lse[U], x[U];
  auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      lse[u] = -INFINITY;
      x[u] = 0.f;
      if (s + u < s1) {
        lse[u] = lses[(s + u) * step];
        if (col < a.e) x[u] = outs[(s + u) * step * a.e + col];
      }
    }
  };
  load(s0);
  float top = -INFINITY;
  for (int s = s0 + lane; s < s1; s += 64) top = fmaxf(top, lses[s * step]);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < Q; ++w) top = fmaxf(top, tops[m * Q + w]);
  const float ref = top == -INFINITY ? 0.f : top;  // no keys at all
  float o = 0.f, sum = 0.f;
  for (int s = s0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool any = lse[u] != -INFINITY;  // an empty split wrote no outputs
      const float w = any ? expf(lse[u] - ref) : 0.f;
      sum += w;
      o += any ? w * x[u] : 0.f;
    }
    s += U;
    if (s >= s1) break;
    load(s);
  }
  if (lane == 0) sums[wave] = sum;
  acc[m][share][lane] = o;
  __syncthreads();
  float l[2];
#pragma unroll
  for (int mm = 0; mm < 2; ++mm) {
    l[mm] = 0.f;
#pragma unroll
    for (int w = 0; w < Q; ++w) l[mm] += sums[mm * Q + w];
  }
  if (lane == 0 && share == 0 && blockIdx.y == 0 && a.lse)
    a.lse[(bh * 2 + m) * a.Nq + i] = top == -INFINITY ? -INFINITY : ref + logf(m ? l[1] : l[0]);
  const float lam = lam_of(a.lam, a.lam_bf16, head);
  if (wave == 0 && col < a.e) {
    float y[2];
#pragma unroll
    for (int mm = 0; mm < 2; ++mm) {
      const float inv = l[mm] > 0.f || l[mm] != l[mm] ? 1.f / l[mm] : 0.f;
      y[mm] = 0.f;
#pragma unroll
      for (int w = 0; w < Q; ++w) y[mm] += acc[mm][w][lane];
      y[mm] *= inv;
      if (a.maps) a.maps[((bh * 2 + mm) * a.Nq + i) * a.e + col] = y[mm];
    }
    a.o[b * a.mo.sb + head * a.mo.sh + (long long)i * a.mo.ld + col] =
        __builtin_bit_cast(uint16_t, (__bf16)(y[0] - lam * y[1]));
  }
}

template <int DQ, int QS, int DV, int KB, int QW, int R, bool SPLIT>
hipError_t go(const DiffArgs& a, int split_keys, int n_split) {
  const int n_qtiles = (a.Nq + 32 * QW - 1) / (32 * QW);
  const int total = a.B * a.H * n_split * n_qtiles;
  diff_fwd_kernel<DQ, QS, DV, KB, QW, R, SPLIT>
      <<<total, 128 * QW, 0, a.stream>>>(a, n_qtiles, n_split, split_keys, total, a.scale * kLog2e);
  return hipGetLastError();
}

// Query waves of a workgroup, four (128 queries) or two. Of two of the wider tiles
// two workgroups fit on a CU: they take 1.0-1.06 of the wide one's time, and one
// alone 0.75-0.85 (N = 256 .. 16,384), so two are taken where they are one per CU
// or fill the last round better. Of e <= 64 three fit, and take 0.75-1.07 (0.82-
// 0.97 over many rounds up to N = 4,096, 0.97-1.03 at 16,384): always two there.
// A row's operations are the same in both.
template <int DQ, int QS, int DV, int KB>
bool two_query_waves(const DiffArgs& a) {
  if (a.Nq <= 64) return true;
  static ResidentCache cache;
  const int cus = cache.get(reinterpret_cast<const void*>(diff_fwd_kernel<DQ, QS, DV, KB, 4, 2, false>), 512).cus;
  if (cus <= 0) return false;
  const long long wide = (long long)a.B * a.H * ((a.Nq + 127) / 128), narrow = (long long)a.B * a.H * ((a.Nq + 63) / 64);
  const long long left = narrow % (2 * cus);
  const double two = 1.04 * (narrow / (2 * cus)) + (left == 0 ? 0. : left <= cus ? 0.8 : 1.04);
  return two < (double)((wide + cus - 1) / cus);
}

// Split keys, each workgroup a few KB of its own: bound by the latency of the tile
// requests. Up to 32 queries take one wave per map, tiles of 32 keys and four slots,
// three tiles ahead (d = 64, e = 128, one query, against two waves, 64 keys and two
// slots: 131,072 keys 1 head 33.2 -> 28.8 us, 32,768 keys 4 heads 26.0 -> 23.3, 32
// heads 103 -> 101). Of two slots twice as many workgroups fit: taken where all of
// the grid is resident then and would not be with four (8 heads, 131,072 keys 115 ->
// 106 us; twice the grid 101 -> 109). The bits are the same. The 96-wide tile keeps
// its shape (its four slots leave one workgroup per CU: 115.2 us against 115.7).
template <int DQ, int QS, int DV, int KB>
hipError_t go_split(const DiffArgs& a, int split_keys, int n_split) {
  if constexpr (DQ < 96) {
    if (a.Nq <= 32) {
      static ResidentCache two, four;
      const int n2 = two.get(reinterpret_cast<const void*>(diff_fwd_kernel<DQ, QS, DV, 1, 1, 2, true>), 128).workgroups;
      const int n4 = four.get(reinterpret_cast<const void*>(diff_fwd_kernel<DQ, QS, DV, 1, 1, 4, true>), 128).workgroups;
      const long long grid = (long long)a.B * a.H * n_split;
      if (grid > n4 && grid <= n2) return go<DQ, QS, DV, 1, 1, 2, true>(a, split_keys, n_split);
      return go<DQ, QS, DV, 1, 1, 4, true>(a, split_keys, n_split);
    }
  }
  return go<DQ, QS, DV, KB, 2, 2, true>(a, split_keys, n_split);
}

template <int DQ, int QS, int DV, int KB>
hipError_t go_tile(const DiffArgs& a) {
  const int split_keys = diff_split_keys(a.Nq, a.Nk);
  if (split_keys == 0) {
    if constexpr (DV > 64)
      if (!two_query_waves<DQ, QS, DV, KB>(a)) return go<DQ, QS, DV, KB, 4, 2, false>(a, 0, 1);
    return go<DQ, QS, DV, KB, 2, 2, false>(a, 0, 1);
  }
  const int n_split = (a.Nk + split_keys - 1) / split_keys;
  const hipError_t err = go_split<DQ, QS, DV, KB>(a, split_keys, n_split);
  if (err != hipSuccess) return err;
  // (one query of 8 heads in 128 splits: eight waves per map 117 us for both kernels,
  // one 123; 64 queries 161 and 151)
  const dim3 grid(a.B * a.H * a.Nq, (a.e + 63) / 64);
  if (n_split > 32 && a.Nq <= 16) diff_join_kernel<8><<<grid, 1024, 0, a.stream>>>(a, n_split);
  else diff_join_kernel<1><<<grid, 128, 0, a.stream>>>(a, n_split);
  return hipGetLastError();
}

}  // namespace

// Up to 128 splits of 512 keys or more for one workgroup's queries, up to 32 of
// 4,096 or more for four of them. (Splits write and read 8 e bytes per query: 256
// heads of 256 queries over 4,096 keys in two splits took 384 us against 239, so
// these wait for longer keys: 8 heads of 128 queries over 32,768 took 72 us in
// eight splits against 417, 256 heads of 256 over 8,192 in two 593 against 460.)
int diff_split_keys(int Nq, int Nk) {
  if (Nq > 256 || Nk < (Nq > 64 ? 8192 : 1024)) return 0;
  const int least = Nq > 64 ? 4096 : 512, most = Nq > 64 ? 32 : 128;
  const int keys = ((Nk + most - 1) / most + 63) / 64 * 64;
  return keys > least ? keys : least;
}

size_t diff_fwd_workspace_floats(int B, int H, int Nq, int Nk, int e) {
  const int s = diff_split_keys(Nq, Nk);
  return s ? (size_t)B * H * ((Nk + s - 1) / s) * 2 * Nq * (e + 1) : 0;
}

hipError_t launch_diff_fwd(const DiffArgs& a) {
  const DiffTile t = diff_tile(a.d, a.e);
  if (t.dq == 96) return go_tile<96, 5, 160, 1>(a);
  if (t.dv == 128) return go_tile<64, 4, 128, 2>(a);
  return t.dq == 32 ? go_tile<32, 2, 64, 2>(a) : go_tile<64, 4, 64, 2>(a);
}

}  // namespace vitattn
