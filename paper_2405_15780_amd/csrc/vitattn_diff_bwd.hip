// Backward pass of differential attention for gfx950, P recomputed from q, k
// and the saved LSE of each map. Per (b, h), with O = O_1 - lam O_2:
//
//   dP = dO V^T (one product for both maps),  D_m = dO . O_m,
//   dS_1 = P_1 o (dP - D_1),  dS_2 = P_2 o (dP - D_2)  (times -lam at the end),
//   dQ_m = scale dS_m K_m,  dK_m = scale dS_m^T Q_m,  dV = (P_1 - lam P_2)^T dO,
//   dlam = - sum_i D_2.
//
//   1. row pass: -D_1, D_1 - D_2 and LSE_m * log2(e) per query, and a partial sum of
//      D_2 per workgroup (HBM-bound; O_1 and O_2 in fp32, see the forward).
//   2. dK/dV kernel: a workgroup per 32 KBW keys; two waves per 32 keys split the
//      work (as in vitattn_bwd.hip): role V holds K_1, K_2, forms both maps' P
//      and accumulates dV from P_1 - lam P_2, role K holds V, takes the P it is
//      handed through LDS, forms both dS and accumulates dK_1 and dK_2. At
//      e = 2 d both have 16 matrix ops per 32 x 32 block.
//   3. dQ kernel: 32 queries per wave, four waves, Q_1, Q_2 and dO held; streams
//      K_1, K_2 and V. Few queries over many keys: the keys are split over
//      workgroups as in the forward, and a fourth kernel adds the shares in order.
//
// P_1 - lam P_2 and dS are rounded to bf16 as matrix-core operands, and P to
// bf16 where role V hands it over: with fp32's range of exponents, since dK of a
// key that every query gives little weight is a sum of small P alone (fp16 has
// three bits more, dK 2.4e-3 off in norm and not 2.9e-3, and even with a factor
// 2^14 made such rows coarse below P = 2^-28 and zero below 2^-39). Everything
// else is fp32 until the outputs are rounded once. One of the two differences dP - D
// comes from the matrix cores, whose accumulator starts at -D_1; the other is that
// plus D_1 - D_2. No atomics: the sums of dlam's partials are added in a fixed
// order, and each output row by one workgroup.
//
// Bound as the forward is. 4 heads of 32,768 tokens, d = 64, e = 128: dK/dV 4.3 ms
// (4.4 TFLOP, 1.02 PFLOP/s), dQ 3.0 (3.3 TFLOP, 1.1), rows 0.03, the board at its
// power limit (a large matrix product runs at 1.35 PFLOP/s there). 64 heads of 1,024,
// d = 32, e = 64: 67, 40 and 9 us, in one and a third rounds of workgroups. Four heads
// of 5,003, two samples, d = 72, e = 144: dK/dV 230 + 132 us, wide and narrow
// workgroups in turn, dQ 221. The wide dK/dV workgroups of d = 64, e = 128 and of d = 72
// fill 256 registers; two and one more are written to scratch before the loop and read
// after it.
#include "vitattn_diff.h"

namespace vitattn {

namespace {

// Workspace: the shares of dQ where the keys are split, fp32 [bh][split][map]
// [query][d]; then per (b, h) and block of 32 queries 128 floats, [-D_1 | D_1 - D_2 |
// LSE_1 log2 e | LSE_2 log2 e] of 32 each; then the partial sums of D_2,
// [bh][row-pass workgroup]. Rows past the last query hold zeros and an LSE of
// +inf, which makes their P zero; so do rows without keys.
constexpr int kStat = 128;
constexpr int kRowBlock = 64;  // query rows of a row-pass workgroup
constexpr int kKeyBlock = 128;  // keys of a wide dK/dV workgroup, or of two narrow ones

__host__ __device__ constexpr int query_blocks(int Nq) { return (Nq + 31) / 32; }
__host__ __device__ constexpr int row_groups(int Nq) { return (Nq + kRowBlock - 1) / kRowBlock; }

// LPR lanes per row take 8 columns each.
template <int LPR>
__global__ __launch_bounds__(256) void diff_rowdot_kernel(const DiffArgs a, float* __restrict__ stats,
                                                          float* __restrict__ partial, int groups) {
  constexpr int RPP = 256 / LPR;  // rows at a time
  __shared__ float sums[4];
  debug_poison_lds(sums);
  const int bh = blockIdx.x / groups, group = blockIdx.x - bh * groups;
  const int b = bh / a.H, head = bh - b * a.H;
  const int col = 8 * (threadIdx.x % LPR);
  const float* const o1 = a.maps + 2LL * bh * a.Nq * a.e;
  const float* const o2 = o1 + (long long)a.Nq * a.e;
  const uint16_t* const g = a.dout + b * a.mg.sb + head * a.mg.sh;
  float* const st = stats + (long long)bh * query_blocks(a.Nq) * kStat;
  float total = 0.f;
  for (int r0 = 0; r0 < kRowBlock; r0 += RPP) {
    const int row = group * kRowBlock + r0 + threadIdx.x / LPR;
    float d1 = 0.f, d2 = 0.f;
    if (row < a.Nq && col < a.e) {
      const bf16x8 gv = as_bf16x8(*reinterpret_cast<const uint4*>(g + (long long)row * a.mg.ld + col));
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(o1 + (long long)row * a.e + col + i);
        const float4 y = *reinterpret_cast<const float4*>(o2 + (long long)row * a.e + col + i);
        const float g0 = (float)gv[i], g1 = (float)gv[i + 1], g2 = (float)gv[i + 2], g3 = (float)gv[i + 3];
        d1 += g0 * x.x + g1 * x.y + g2 * x.z + g3 * x.w;
        d2 += g0 * y.x + g1 * y.y + g2 * y.z + g3 * y.w;
      }
    }
#pragma unroll
    for (int m = LPR / 2; m >= 1; m >>= 1) {
      d1 += __shfl_xor(d1, m, 64);
      d2 += __shfl_xor(d2, m, 64);
    }
    if (col == 0) total += d2;
    if (col == 0 && row < 32 * query_blocks(a.Nq)) {
      float l1 = INFINITY, l2 = INFINITY;
      if (row < a.Nq) {
        l1 = a.lse[(2LL * bh) * a.Nq + row] * kLog2e;
        l2 = a.lse[(2LL * bh + 1) * a.Nq + row] * kLog2e;
        if (l1 == -INFINITY) l1 = INFINITY;
        if (l2 == -INFINITY) l2 = INFINITY;
      }
      float* s = st + (row >> 5) * kStat + (row & 31);
      s[0] = -d1;
      s[32] = d1 - d2;
      s[64] = l1;
      s[96] = l2;
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) total += __shfl_xor(total, m, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// Widest window of ops that a block's 16 rows of vector work may ride on (row r
// on op r W / 16): rows 0..7 complete two ops before op NS, the first that
// reads them, rows 8..15 two before op NS + half.
constexpr int row_window(int NS, int half) {
  int w = NS + half;
  while (w > 1 && !(7 * w / 16 <= NS - 2 && 15 * w / 16 <= NS + half - 2)) --w;
  return w;
}

// ------------------------------------------------------------------ dK / dV
//
// Steps of 32 queries. In step j role V turns S_m(j) into P_m(j), which it hands
// to its partner, while the matrix cores run dV += (P_1 - lam P_2)(j-1)^T dO(j-1)
// and the scores of block j + 1. Role K turns the P(j-1) it was handed and
// dP(j-1) into dS_m(j-1), while they run dK_m += dS_m(j-LAG)^T Q_m(j-LAG) and
// dP(j). With a ring of six LAG is 2, and the vector work of a step feeds only
// the next step's ops; a ring of four (the widest tile) holds one block less, so
// dP(j) goes first there and dK follows with this step's dS. The stream of ops
// runs through the barriers: the first two operands of a step are of blocks that
// the step before may read already, and are read before the barrier.
// Blocks below 0 and past the last are zeros (P is then 0 or 1, and dO, dS and Q
// are zero): they add nothing, and the steps group by the ring depth, so that
// every slot is a compile-time constant.
// (four-wave workgroups of the wider tiles have a CU's LDS, and its registers, alone)
template <int DQ, int QS, int DV, int RING, int KBW>
__global__ __launch_bounds__(128 * KBW, KBW == 2 && DV > 64 ? 1 : 2) void diff_dkdv_kernel(const DiffArgs a,
                                                                       const float* __restrict__ stats, int n_ktiles,
                                                                       int first, int total, float c) {
  constexpr int NW = 2 * KBW, BQ = 32;
  constexpr int PARTS = kKeyBlock / (32 * KBW);  // workgroups of a block of keys
  constexpr int VS = DV / 16, NCV = DV / 32;
  constexpr int NCQ = (QS + 1) / 2;  // 32-column blocks of d that may hold data
  constexpr int QT = BQ * DQ * 2, GT = BQ * DV * 2;
  static_assert(RING == 4 || RING == 6, "ring depth");
  __shared__ __attribute__((aligned(1024))) char qbuf0[2 * QT];  // Q_1, then Q_2
  __shared__ __attribute__((aligned(1024))) char qbuf1[2 * QT];
  __shared__ __attribute__((aligned(1024))) char qbuf2[2 * QT];
  __shared__ __attribute__((aligned(1024))) char qbuf3[2 * QT];
  __shared__ __attribute__((aligned(1024))) char qbuf4[RING > 4 ? 2 * QT : 16];
  __shared__ __attribute__((aligned(1024))) char qbuf5[RING > 4 ? 2 * QT : 16];
  __shared__ __attribute__((aligned(1024))) char gbuf0[GT];
  __shared__ __attribute__((aligned(1024))) char gbuf1[GT];
  __shared__ __attribute__((aligned(1024))) char gbuf2[GT];
  __shared__ __attribute__((aligned(1024))) char gbuf3[GT];
  __shared__ __attribute__((aligned(1024))) char gbuf4[RING > 4 ? GT : 16];
  __shared__ __attribute__((aligned(1024))) char gbuf5[RING > 4 ? GT : 16];
  __shared__ __attribute__((aligned(16))) float sbuf0[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf1[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf2[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf3[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf4[RING > 4 ? kStat : 4];
  __shared__ __attribute__((aligned(16))) float sbuf5[RING > 4 ? kStat : 4];
  __shared__ __attribute__((aligned(16))) uint4 xbuf0[KBW][2][2][64];  // P of even blocks: [pair][map][step][lane]
  __shared__ __attribute__((aligned(16))) uint4 xbuf1[KBW][2][2][64];  // of odd ones
  char* const qbuf[6] = {qbuf0, qbuf1, qbuf2, qbuf3, qbuf4, qbuf5};
  char* const gbuf[6] = {gbuf0, gbuf1, gbuf2, gbuf3, gbuf4, gbuf5};
  float* const sbuf[6] = {sbuf0, sbuf1, sbuf2, sbuf3, sbuf4, sbuf5};
  debug_poison_lds(qbuf0, qbuf1, qbuf2, qbuf3, qbuf4, qbuf5, gbuf0, gbuf1, gbuf2, gbuf3, gbuf4, gbuf5, sbuf0, sbuf1,
                   sbuf2, sbuf3, sbuf4, sbuf5, xbuf0, xbuf1);

  const int work = work_item(a.key_lens, total), block = first + work / PARTS;
  const int bh = block / n_ktiles, key_first = (block - bh * n_ktiles) * kKeyBlock + (work % PARTS) * 32 * KBW;
  const int b = bh / a.H, head = bh - b * a.H;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = wave % KBW;
  const bool role_v = wave < KBW;
  const int key = key_first + kb * 32 + (lane & 31);
  const int Nk = keys_of(a.key_lens, b, a.Nk);
  const float lam = lam_of(a.lam, a.lam_bf16, head);

  // held operands (this wave's 32 keys): K_1 and K_2, or V
  constexpr int NH = 2 * QS > VS ? 2 * QS : VS;
  bf16x8 hf[NH];
  const int chr = a.d >> 3, chv = a.e >> 3;
  const int ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld, ldq = 2 * a.mq.ld, ldg = 2 * a.mg.ld;
  if (role_v) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const rsrc_t r = make_rsrc(a.k + map_head(a.mk, b, head, m), (unsigned)(Nk * ldk));
#pragma unroll
      for (int kk = 0; kk < QS; ++kk) hf[m * QS + kk] = as_bf16x8(buffer_load16(r, chunk_offset(key, 2 * kk + h, ldk, chr)));
    }
  } else {
    const rsrc_t r = make_rsrc(a.v + b * a.mv.sb + head * a.mv.sh, (unsigned)(Nk * ldv));
#pragma unroll
    for (int kk = 0; kk < VS; ++kk) hf[kk] = as_bf16x8(buffer_load16(r, chunk_offset(key, 2 * kk + h, ldv, chv)));
  }

  // Streamed blocks. Half of the waves fetch Q_1, the others Q_2; all fetch dO;
  // waves 0 and 1 the statistics.
  const int qmap = wave / KBW;
  const rsrc_t rq = make_rsrc(a.q + map_head(a.mq, b, head, qmap), (unsigned)(a.Nq * ldq));
  const rsrc_t rg = make_rsrc(a.dout + b * a.mg.sb + head * a.mg.sh, (unsigned)(a.Nq * ldg));
  const int nb = query_blocks(a.Nq);
  const rsrc_t rs = make_rsrc(stats + (long long)bh * nb * kStat, (unsigned)nb * kStat * 4);
  TileDma<DQ, BQ, KBW> dmq;
  TileDma<DV, BQ, NW> dmg;
  dmq.init(wave % KBW, lane, ldq, chr);
  dmg.init(wave, lane, ldg, chv);
  constexpr int PQ = decltype(dmq)::PER_WAVE, PG = decltype(dmg)::PER_WAVE;
  constexpr int NREQ = PQ + PG + 1;
  auto request = [&](auto slot_tag, int blk, int r) __attribute__((always_inline)) {
    constexpr int SL = decltype(slot_tag)::value;
    if (r < PQ)
      dmq.issue_one(rq, blk * BQ, ldq, qbuf[SL] + qmap * QT, r);
    else if (r < PQ + PG)
      dmg.issue_one(rg, blk * BQ, ldg, gbuf[SL], r - PQ);
    else if (wave < 2)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)(sbuf[SL] + 64 * wave), 4,
                                               (blk * kStat + 64 * wave + lane) * 4, 0, 0, 0);
  };

  RowFrag<DQ> rfq;
  RowFrag<DV> rfg;
  TrFrag<DQ> tfq;
  TrFrag<DV> tfg;
  rfq.init(lane);
  rfg.init(lane);
  tfq.init(lane);
  tfg.init(lane);

  constexpr int NACC = NCV > 2 * NCQ ? NCV : 2 * NCQ;
  f32x16 acc[NACC];  // dV^T, or dK_1^T then dK_2^T
#pragma unroll
  for (int i = 0; i < NACC; ++i) acc[i] = zero16();

  constexpr int LAG = RING > 4 ? 2 : 1;
  constexpr int PF = RING - 1 - LAG;  // blocks fetched ahead
  auto end_step = [&]() __attribute__((always_inline)) {
    // requests of the last PF - 2 steps may stay in flight
    wait_vmem_leave<(PF - 2) * ((decltype(dmq)::ALL_ACTIVE ? PQ : 0) + (decltype(dmg)::ALL_ACTIVE ? PG : 0))>();
    barrier_lds();
  };

  if (key_first < Nk) {  // else every key of this workgroup is past the sample's last: zeros
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    using S2 = std::integral_constant<int, 2>;
    using S3 = std::integral_constant<int, 3>;
    using S4 = std::integral_constant<int, 4>;
    using S5 = std::integral_constant<int, 5>;
    static_for<0, PF>([&](auto T) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < NREQ; ++r) request(T, decltype(T)::value, r);
    });
    // blocks -1 and -LAG: zero rows (as those of block nb are) and P = 0
    static_for<0, NREQ>([&](auto R) __attribute__((always_inline)) {
      request(std::integral_constant<int, RING - 1>{}, nb, decltype(R)::value);
      if constexpr (LAG > 1) request(std::integral_constant<int, RING - LAG>{}, nb, decltype(R)::value);
    });
    if (!role_v)
#pragma unroll
      for (int i = 0; i < 4; ++i) xbuf1[kb][i >> 1][i & 1][lane] = make_uint4(0, 0, 0, 0);
    wait_vmem();
    __syncthreads();
    const int n_pad = (nb + LAG + RING - 1) / RING * RING;  // LAG steps past the last block

    if (role_v) {
      f32x16 sa[2], sb[2];  // scores of the current and the next block, per map
#pragma unroll
      for (int i = 0; i < 2 * QS; ++i) {
        if (i < 2) sa[i] = zero16();
        sa[i & 1] = mfma32(lds_frag_row(qbuf[0] + (i & 1) * QT, rfq.at(i >> 1)), hf[(i & 1) * QS + (i >> 1)], sa[i & 1]);
      }
      bf16x8 ob[2] = {};          // P_1 - lam P_2 of the block before
      bf16x8 lead[2];             // the next step's first two operands
      auto load_v = [&](const char* g, int t) -> bf16x8 { return tfg.load(g, 16 * (t / NCV), t % NCV); };
      lead[0] = load_v(gbuf[RING - 1], 0);
      lead[1] = load_v(gbuf[RING - 1], 1);
      auto step = [&](auto slot_tag, f32x16 (&cur)[2], f32x16 (&nxt)[2], int j) __attribute__((always_inline)) {
        constexpr int SL = decltype(slot_tag)::value;
        constexpr int PR = (SL + RING - 1) % RING, NX = (SL + 1) % RING, RF = (SL + PF) % RING;
        constexpr int NS = 2 * QS, NV = 2 * NCV, NOPS = NV + NS;
        constexpr int STEP = 2 * NREQ <= NOPS ? 2 : 1;
        static_assert(STEP * NREQ <= NOPS, "requests fit the op stream");
        const float* st = sbuf[SL];
        uint4(*xb)[2][64] = (SL & 1) ? xbuf1[kb] : xbuf0[kb];
        bf16x8 on[2];
        float4 l1[4], l2[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          l1[g] = *reinterpret_cast<const float4*>(st + 64 + 8 * g + 4 * h);
          l2[g] = *reinterpret_cast<const float4*>(st + 96 + 8 * g + 4 * h);
        }
        f32x16 wv;
        auto row = [&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[0][r], c, -l1[r >> 2][r & 3]));
          const float p2 = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[1][r], c, -l2[r >> 2][r & 3]));
          float w = __builtin_fmaf(-lam, p2, p1);
          pin(w);
          cur[0][r] = p1;
          cur[1][r] = p2;
          wv[r] = w;
          if constexpr ((r & 7) == 7) {
            xb[0][r >> 3][lane] = __builtin_bit_cast(uint4, acc_to_operand(cur[0], r >> 3));
            xb[1][r >> 3][lane] = __builtin_bit_cast(uint4, acc_to_operand(cur[1], r >> 3));
            on[r >> 3] = acc_to_operand(wv, r >> 3);
          }
        };
        auto load_op = [&](int i) -> bf16x8 {
          if (i < NV) return load_v(gbuf[PR], i);
          if (i < NOPS) return lds_frag_row(qbuf[NX] + ((i - NV) & 1) * QT, rfq.at((i - NV) >> 1));
          return load_v(gbuf[SL], i - NOPS);
        };
        bf16x8 aq[3];
        aq[0] = lead[0];
        aq[1] = lead[1];
        sched_fence();
        static_for<0, NOPS>([&](auto IC) __attribute__((always_inline)) {
          constexpr int i = decltype(IC)::value;
          if constexpr (i == 0) __builtin_amdgcn_s_setprio(1);
          if constexpr (i + 2 < NOPS) aq[(i + 2) % 3] = load_op(i + 2);
          else lead[i + 2 - NOPS] = load_op(i + 2);
          if constexpr (i < NV) {
            acc[i % NCV] = mfma32(aq[i % 3], ob[i / NCV], acc[i % NCV]);
          } else {
            constexpr int t = i - NV;
            if constexpr (t < 2) nxt[t] = zero16();
            nxt[t & 1] = mfma32(aq[i % 3], hf[(t & 1) * QS + (t >> 1)], nxt[t & 1]);
          }
          if constexpr (i % STEP == STEP - 1 && i / STEP < NREQ) request(std::integral_constant<int, RF>{}, j + PF, i / STEP);
          static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
            if constexpr (decltype(RC)::value * NOPS / 16 == i) row(RC);
          });
          sched_fence();
        });
        __builtin_amdgcn_s_setprio(0);
        ob[0] = on[0];
        ob[1] = on[1];
        end_step();
      };
      for (int j = 0; j < n_pad; j += RING) {
        step(S0{}, sa, sb, j);
        step(S1{}, sb, sa, j + 1);
        step(S2{}, sa, sb, j + 2);
        step(S3{}, sb, sa, j + 3);
        if constexpr (RING > 4) {
          step(S4{}, sa, sb, j + 4);
          step(S5{}, sb, sa, j + 5);
        }
      }
    } else {
      f32x16 da, db = zero16();  // dP of the current (j - 1) and the next block
      bf16x8 ob[2][2] = {};      // dS, [map][step], of the block before
      bf16x8 lead[2];
      // dK op t: contraction step t / (2 NCQ), map, column block
      auto load_k = [&](const char* q, int t) -> bf16x8 {
        const int u = t % (2 * NCQ);
        return tfq.load(q + (u / NCQ) * QT, 16 * (t / (2 * NCQ)), u % NCQ);
      };
#pragma unroll
      for (int t = 0; t < 2; ++t) lead[t] = LAG > 1 ? load_k(qbuf[RING - LAG], t) : lds_frag_row(gbuf[0], rfg.at(t));
      auto step = [&](auto slot_tag, f32x16& cur, f32x16& nxt, int j) __attribute__((always_inline)) {
        constexpr int SL = decltype(slot_tag)::value;  // of block j
        constexpr int PR = (SL + RING - 1) % RING, KR = (SL + RING - LAG) % RING, RF = (SL + PF) % RING;
        constexpr int NS = VS, NK = 4 * NCQ, NOPS = NS + NK;
        constexpr int K0 = LAG > 1 ? 0 : NS, P0 = LAG > 1 ? NK : 0;  // first dK and dP op
        constexpr int STEP = 2 * NREQ <= NOPS ? 2 : 1;
        static_assert(STEP * NREQ <= NOPS, "requests fit the op stream");
        uint4(*xb)[2][64] = (SL & 1) ? xbuf0[kb] : xbuf1[kb];  // of block j - 1
        bf16x8 on[2][2];
        uint4 pm[2][2];
        float4 dd[4];  // D_1 - D_2
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int m = 0; m < 2; ++m) pm[m][s] = xb[m][s][lane];
#pragma unroll
        for (int g = 0; g < 4; ++g) dd[g] = *reinterpret_cast<const float4*>(sbuf[PR] + 32 + 8 * g + 4 * h);
        f32x16 s1, s2;
        auto row = [&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          auto p_of = [&](int m) {
            const uint32_t w = __builtin_bit_cast(u32x4, pm[m][r >> 3])[(r & 7) >> 1];
            return __uint_as_float((r & 1) ? (w & 0xffff0000u) : (w << 16));
          };
          float x1 = p_of(0) * cur[r];
          float x2 = p_of(1) * (cur[r] + dd[r >> 2][r & 3]);
          pin(x1);
          pin(x2);
          s1[r] = x1;
          s2[r] = x2;
          if constexpr ((r & 7) == 7) {
            on[0][r >> 3] = acc_to_operand(s1, r >> 3);
            on[1][r >> 3] = acc_to_operand(s2, r >> 3);
          }
        };
        // the op on which row r rides: over the whole step behind the first two
        // ops, whose time the handed P needs, or as ROW_W says
        constexpr auto op_of = [](int r) { return LAG > 1 ? 2 + r * (NOPS - 2) / 16 : r * row_window(NS, 2 * NCQ) / 16; };
        auto load_op = [&](int i) -> bf16x8 {
          if (i >= NOPS) return LAG > 1 ? load_k(qbuf[PR], i - NOPS) : lds_frag_row(gbuf[(SL + 1) % RING], rfg.at(i - NOPS));
          return i >= K0 && i < K0 + NK ? load_k(qbuf[KR], i - K0) : lds_frag_row(gbuf[SL], rfg.at(i - P0));
        };
        bf16x8 aq[3];
        aq[0] = lead[0];
        aq[1] = lead[1];
        sched_fence();
        static_for<0, NOPS>([&](auto IC) __attribute__((always_inline)) {
          constexpr int i = decltype(IC)::value;
          if constexpr (i == 0) __builtin_amdgcn_s_setprio(1);
          if constexpr (i + 2 < NOPS) aq[(i + 2) % 3] = load_op(i + 2);
          else lead[i + 2 - NOPS] = load_op(i + 2);
          if constexpr (i >= K0 && i < K0 + NK) {
            constexpr int t = i - K0, u = t % (2 * NCQ);
            if constexpr (LAG > 1) acc[u] = mfma32(aq[i % 3], ob[u / NCQ][t / (2 * NCQ)], acc[u]);
            else acc[u] = mfma32(aq[i % 3], on[u / NCQ][t / (2 * NCQ)], acc[u]);
          } else {
            constexpr int t = i - P0;
            if constexpr (t == 0) {  // starts at -D_1 of its rows
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const float4 x = *reinterpret_cast<const float4*>(sbuf[SL] + 8 * g + 4 * h);
                nxt[4 * g] = x.x;
                nxt[4 * g + 1] = x.y;
                nxt[4 * g + 2] = x.z;
                nxt[4 * g + 3] = x.w;
              }
            }
            nxt = mfma32(aq[i % 3], hf[t], nxt);
          }
          if constexpr (i % STEP == STEP - 1 && i / STEP < NREQ) request(std::integral_constant<int, RF>{}, j + PF, i / STEP);
          static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
            if constexpr (op_of(decltype(RC)::value) == i) row(RC);
          });
          sched_fence();
        });
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int x = 0; x < 2; ++x) ob[m][x] = on[m][x];
        end_step();
      };
      for (int j = 0; j < n_pad; j += RING) {
        step(S0{}, db, da, j);
        step(S1{}, da, db, j + 1);
        step(S2{}, db, da, j + 2);
        step(S3{}, da, db, j + 3);
        if constexpr (RING > 4) {
          step(S4{}, db, da, j + 4);
          step(S5{}, da, db, j + 5);
        }
      }
    }
    wait_vmem();  // requests past the last block must land before this LDS is reassigned
  }

  if (key >= a.Nk) return;
  const bool real = key < Nk;
  if (role_v) {
    uint16_t* out = a.dv + b * a.mdv.sb + head * a.mdv.sh + (long long)key * a.mdv.ld;
#pragma unroll
    for (int cb = 0; cb < NCV; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * cb + 8 * g + 4 * h;
        if (col < a.e)
          put4_bf16(out + col, real ? acc[cb][4 * g] : 0.f, real ? acc[cb][4 * g + 1] : 0.f,
                    real ? acc[cb][4 * g + 2] : 0.f, real ? acc[cb][4 * g + 3] : 0.f);
      }
  } else {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float f = m ? -lam * a.scale : a.scale;
      uint16_t* out = a.dk + map_head(a.mdk, b, head, m) + (long long)key * a.mdk.ld;
#pragma unroll
      for (int cb = 0; cb < NCQ; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * cb + 8 * g + 4 * h;
          const f32x16& x = acc[m * NCQ + cb];
          if (col < a.d)
            put4_bf16(out + col, real ? x[4 * g] * f : 0.f, real ? x[4 * g + 1] * f : 0.f, real ? x[4 * g + 2] * f : 0.f,
                      real ? x[4 * g + 3] * f : 0.f);
        }
    }
  }
}

// ------------------------------------------------------------------ dQ
//
// One workgroup = NW waves = 32 NW queries of one (b, h). K_1, K_2 and V stream
// through a ring of LDS slots in tiles of 32 keys. Per tile:
//   S_m^T = K_m Q_m^T, dP^T = V dO^T;  dS_m^T;  dQ_m^T += K_m^T dS_m^T
// Keys past the sample's last have P = 0 (their scores are of zero rows, and an
// LSE far below zero would make exp overflow). The (first) workgroup of query tile
// 0 of sample 0 also adds its head's partial sums of dlam.
template <int DQ, int QS, int DV, int RING, int NW, bool SPLIT>
__global__ __launch_bounds__(64 * NW, DV > 128 ? 1 : 2) void diff_dq_kernel(const DiffArgs a, const float* __restrict__ stats,
                                                                  const float* __restrict__ partial, int groups,
                                                                  int n_qtiles, int n_split, int split_keys, int total,
                                                                  float c) {
  constexpr int BM = 32 * NW, BN = 32;
  constexpr int VS = DV / 16;
  constexpr int NCQ = (QS + 1) / 2;
  constexpr int KT = BN * DQ * 2, VT = BN * DV * 2;
  static_assert(RING == 4, "one variable per slot");
  __shared__ __attribute__((aligned(1024))) char kbuf0[2 * KT];
  __shared__ __attribute__((aligned(1024))) char kbuf1[2 * KT];
  __shared__ __attribute__((aligned(1024))) char kbuf2[2 * KT];
  __shared__ __attribute__((aligned(1024))) char kbuf3[2 * KT];
  __shared__ __attribute__((aligned(1024))) char vbuf0[VT];
  __shared__ __attribute__((aligned(1024))) char vbuf1[VT];
  __shared__ __attribute__((aligned(1024))) char vbuf2[VT];
  __shared__ __attribute__((aligned(1024))) char vbuf3[VT];
  __shared__ float sums[NW];
  char* const kbuf[RING] = {kbuf0, kbuf1, kbuf2, kbuf3};
  char* const vbuf[RING] = {vbuf0, vbuf1, vbuf2, vbuf3};
  debug_poison_lds(kbuf0, kbuf1, kbuf2, kbuf3, vbuf0, vbuf1, vbuf2, vbuf3, sums);

  const int work = work_item(a.key_lens, total);
  const int part = work / n_qtiles, qt = work - part * n_qtiles;
  const int bh = SPLIT ? part / n_split : part, sp = SPLIT ? part - bh * n_split : 0;
  const int b = bh / a.H, head = bh - b * a.H;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qrow = qt * BM + wave * 32 + (lane & 31);
  // this workgroup's keys: [key_first, key_first + Nk)
  const int all = keys_of(a.key_lens, b, a.Nk);
  const int key_first = SPLIT ? min(sp * split_keys, all) : 0;
  const int Nk = SPLIT ? min(all - key_first, split_keys) : all;
  const float lam = lam_of(a.lam, a.lam_bf16, head);

  if (b == 0 && qt == 0 && sp == 0 && a.dlam) {
    float s = 0.f;
    for (int i = threadIdx.x; i < a.B * groups; i += 64 * NW) {
      const int bb = i / groups;
      s += partial[((long long)bb * a.H + head) * groups + (i - bb * groups)];
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      s = 0.f;
      for (int w = 0; w < NW; ++w) s += sums[w];
      if (a.lam_bf16) static_cast<__bf16*>(a.dlam)[head] = (__bf16)-s;
      else static_cast<float*>(a.dlam)[head] = -s;
    }
  }

  const int chr = a.d >> 3, chv = a.e >> 3;
  const int ldq = 2 * a.mq.ld, ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld, ldg = 2 * a.mg.ld;
  bf16x8 qf[2][QS], gf[VS];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const rsrc_t r = make_rsrc(a.q + map_head(a.mq, b, head, m), (unsigned)(a.Nq * ldq));
#pragma unroll
    for (int kk = 0; kk < QS; ++kk) qf[m][kk] = as_bf16x8(buffer_load16(r, chunk_offset(qrow, 2 * kk + h, ldq, chr)));
  }
  const rsrc_t rg = make_rsrc(a.dout + b * a.mg.sb + head * a.mg.sh, (unsigned)(a.Nq * ldg));
#pragma unroll
  for (int kk = 0; kk < VS; ++kk) gf[kk] = as_bf16x8(buffer_load16(rg, chunk_offset(qrow, 2 * kk + h, ldg, chv)));
  const int nqb = query_blocks(a.Nq);
  const rsrc_t rs = make_rsrc(stats + (long long)bh * nqb * kStat, (unsigned)nqb * kStat * 4);
  auto stat = [&](int which) {  // of this lane's query; zeros past the last block
    return __builtin_bit_cast(
        float, __builtin_amdgcn_raw_buffer_load_b32(rs, ((qrow >> 5) * kStat + 32 * which + (qrow & 31)) * 4, 0, 0));
  };
  const float l1 = stat(2), l2 = stat(3), dd = stat(1);
  const float nd1 = stat(0);
  constexpr bool START = DV < 160;  // dP starts at -D_1 (the widest tile has no registers to hold that)
  f32x16 start;
  if constexpr (START) {
#pragma unroll
    for (int r = 0; r < 16; ++r) start[r] = nd1;
  } else {
    start = zero16();
  }

  const rsrc_t rk1 = make_rsrc(a.k + map_head(a.mk, b, head, 0) + (long long)key_first * a.mk.ld, (unsigned)(Nk * ldk));
  const rsrc_t rk2 = make_rsrc(a.k + map_head(a.mk, b, head, 1) + (long long)key_first * a.mk.ld, (unsigned)(Nk * ldk));
  const rsrc_t rv = make_rsrc(a.v + b * a.mv.sb + head * a.mv.sh + (long long)key_first * a.mv.ld, (unsigned)(Nk * ldv));
  TileDma<DQ, BN, NW> dma;
  TileDma<DV, BN, NW> dmv;
  dma.init(wave, lane, ldk, chr);
  dmv.init(wave, lane, ldv, chv);
  constexpr int PK = decltype(dma)::PER_WAVE, PV = decltype(dmv)::PER_WAVE, NREQ = 2 * PK + PV;
  auto request = [&](auto slot_tag, int tile, int r) __attribute__((always_inline)) {
    constexpr int SL = decltype(slot_tag)::value;
    if (r < PK) dma.issue_one(rk1, tile * BN, ldk, kbuf[SL], r);
    else if (r < 2 * PK) dma.issue_one(rk2, tile * BN, ldk, kbuf[SL] + KT, r - PK);
    else dmv.issue_one(rv, tile * BN, ldv, vbuf[SL], r - 2 * PK);
  };
  RowFrag<DQ> rfk;
  RowFrag<DV> rfv;
  TrFrag<DQ> tfk;
  rfk.init(lane);
  rfv.init(lane);
  tfk.init(lane);

  f32x16 acc[2 * NCQ];  // dQ_1^T, then dQ_2^T
#pragma unroll
  for (int i = 0; i < 2 * NCQ; ++i) acc[i] = zero16();

  const int n_kt = (Nk + BN - 1) / BN;
  constexpr int PF = RING - 1;  // tiles fetched ahead
  static_for<0, PF>([&](auto T) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < NREQ; ++r) request(T, decltype(T)::value, r);
  });
  wait_vmem();
  __syncthreads();

  // Tile j in slot SL; tile j + PF is requested into the slot of tile j - 1. One
  // stream of ops: the scores, dP beside the exponentials, then dQ in four groups
  // (map, contraction step), each beside the vector work of the next group's dS.
  // Operands are read two ops ahead, through the barrier: the barrier before stage
  // j waited for tile j + 1.
  constexpr int NS = 2 * QS + VS, NQ = 4 * NCQ, AH = 2;
  auto load_op = [&](auto slot_tag, int i) __attribute__((always_inline)) -> bf16x8 {
    constexpr int SL = decltype(slot_tag)::value, NX = (SL + 1) % RING;
    if (i >= NS + NQ) return lds_frag_row(kbuf[NX] + ((i - NS - NQ) & 1) * KT, rfk.at((i - NS - NQ) >> 1));
    if (i < 2 * QS) return lds_frag_row(kbuf[SL] + (i & 1) * KT, rfk.at(i >> 1));
    if (i < NS) return lds_frag_row(vbuf[SL], rfv.at(i - 2 * QS));
    const int g = (i - NS) / NCQ;
    return tfk.load(kbuf[SL] + (g >> 1) * KT, 16 * (g & 1), (i - NS) % NCQ);
  };
  bf16x8 lead[AH];
#pragma unroll
  for (int i = 0; i < AH; ++i) lead[i] = load_op(std::integral_constant<int, 0>{}, i);
  auto stage = [&](auto slot_tag, int j) __attribute__((always_inline)) {
    constexpr int SL = decltype(slot_tag)::value;
    constexpr int RF = (SL + PF) % RING;
    f32x16 s[2], dp;
    bf16x8 ob[4];
    bf16x8 aq[AH + 1];
#pragma unroll
    for (int i = 0; i < AH; ++i) aq[i] = lead[i];
    // dS of row r of group g
    auto row = [&](int g, int r) __attribute__((always_inline)) {
      const int m = g >> 1;
      if (!START && m == 0) dp[r] += nd1;
      float x = s[m][r] * (m ? dp[r] + dd : dp[r]);
      pin(x);
      s[m][r] = x;
      if ((r & 7) == 7) ob[g] = acc_to_operand(s[m], g & 1);
    };
    sched_fence();
    static_for<0, NS + NQ>([&](auto IC) __attribute__((always_inline)) {
      constexpr int i = decltype(IC)::value;
      if constexpr (i + AH < NS + NQ) aq[(i + AH) % (AH + 1)] = load_op(slot_tag, i + AH);
      else lead[i + AH - NS - NQ] = load_op(slot_tag, i + AH);
      if constexpr (i < 2 * QS) {
        if constexpr (i < 2) s[i] = zero16();
        s[i & 1] = mfma32(aq[i % (AH + 1)], qf[i & 1][i >> 1], s[i & 1]);
      } else if constexpr (i < NS) {
        dp = mfma32(aq[i % (AH + 1)], gf[i - 2 * QS], i == 2 * QS ? start : dp);
        static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          if constexpr (r * VS / 16 == i - 2 * QS) {
            float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], c, -l1));
            float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[1][r], c, -l2));
            pin(x);
            pin(y);
            s[0][r] = x;
            s[1][r] = y;
          }
        });
      } else {
        constexpr int t = i - NS, g = t / NCQ, u = t % NCQ;
        if constexpr (t == 0) {
          if ((j + 1) * BN > Nk)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (j * BN + acc_row(r, h) >= Nk) s[0][r] = s[1][r] = 0.f;
#pragma unroll
          for (int r = 0; r < 8; ++r) row(0, r);
        }
        acc[(g >> 1) * NCQ + u] = mfma32(aq[i % (AH + 1)], ob[g], acc[(g >> 1) * NCQ + u]);
        if constexpr (g < 3)
          static_for<0, 8>([&](auto RC) __attribute__((always_inline)) {
            constexpr int r = decltype(RC)::value;
            if constexpr (r * NCQ / 8 == u) row(g + 1, 8 * ((g + 1) & 1) + r);
          });
      }
      if constexpr (i < NREQ) request(std::integral_constant<int, RF>{}, j + PF, i);
      sched_fence();
    });
    // tile j + 2 was requested in stage j + 2 - PF
    wait_vmem_leave<(PF - 2) * ((decltype(dma)::ALL_ACTIVE ? 2 * PK : 0) + (decltype(dmv)::ALL_ACTIVE ? PV : 0))>();
    barrier_lds();
  };
  const int n_iter = (n_kt + RING - 1) / RING * RING;  // tiles past the last have P = 0
  for (int j = 0; j < n_iter; j += RING) {
    stage(std::integral_constant<int, 0>{}, j);
    stage(std::integral_constant<int, 1>{}, j + 1);
    stage(std::integral_constant<int, 2>{}, j + 2);
    stage(std::integral_constant<int, 3>{}, j + 3);
  }
  wait_vmem();  // requests past the last tile must land before this LDS is reassigned

  if (qrow >= a.Nq) return;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float f = m ? -lam * a.scale : a.scale;
    uint16_t* out = a.dq + map_head(a.mdq, b, head, m) + (long long)qrow * a.mdq.ld;
    float* share = a.work + ((((long long)bh * n_split + sp) * 2 + m) * a.Nq + qrow) * a.d;
#pragma unroll
    for (int cb = 0; cb < NCQ; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * cb + 8 * g + 4 * h;
        const f32x16& x = acc[m * NCQ + cb];
        if (col >= a.d) continue;
        if (SPLIT) *reinterpret_cast<float4*>(share + col) = make_float4(x[4 * g] * f, x[4 * g + 1] * f, x[4 * g + 2] * f, x[4 * g + 3] * f);
        else put4_bf16(out + col, x[4 * g] * f, x[4 * g + 1] * f, x[4 * g + 2] * f, x[4 * g + 3] * f);
      }
  }
}

// Adds the shares of dQ in split order, eight in flight (one query over 131,072 keys,
// 8 heads: the whole backward 3,069 us unsplit, 617 split): a wave per (bh, map,
// query) row, a column per lane and 64 more.
__global__ __launch_bounds__(256) void diff_dq_join_kernel(const DiffArgs a, int n_split) {
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = 2LL * a.B * a.H * a.Nq;
  if (row >= rows) return;
  const long long bhm = row / a.Nq, bh = bhm >> 1;
  const int i = (int)(row - bhm * a.Nq), m = (int)(bhm & 1), b = (int)(bh / a.H), head = (int)(bh - (long long)b * a.H);
  const long long step = 2LL * a.Nq * a.d;
  const float* src = a.work + ((bh * n_split * 2 + m) * a.Nq + i) * a.d;
  uint16_t* out = a.dq + map_head(a.mdq, b, head, m) + (long long)i * a.mdq.ld;
  for (int col = threadIdx.x & 63; col < a.d; col += 64) {
    float s = 0.f;
    for (int s0 = 0; s0 < n_split; s0 += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = s0 + u < n_split ? src[(s0 + u) * step + col] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
    out[col] = __builtin_bit_cast(uint16_t, (__bf16)s);
  }
}

// `parts` workgroups for each of n blocks of keys from `first` on
template <int DQ, int QS, int DV, int RING, int KBW>
hipError_t go_dkdv(const DiffArgs& a, const float* stats, int first, int n) {
  if (n == 0) return hipSuccess;
  const int total = n * (kKeyBlock / (32 * KBW));
  diff_dkdv_kernel<DQ, QS, DV, RING, KBW><<<total, 128 * KBW, 0, a.stream>>>(
      a, stats, (a.Nk + kKeyBlock - 1) / kKeyBlock, first, total, a.scale * kLog2e);
  return hipGetLastError();
}

// One wide workgroup is on a CU at a time. A narrow one (64 keys) takes 0.74-0.85
// of its time alone on a CU, and 1.0-1.4 of it for two (N = 256 .. 16,384, every
// tile): blocks left over by whole rounds go to narrow workgroups if these are at
// most one per CU. Of the narrowest tile three fit on a CU, and take 0.83-1.08
// (0.86-1.0 over many rounds): all of its blocks go to them. Each key's operations
// are the same in both.
template <int DQ, int QS, int DV, int RING>
hipError_t launch_dkdv(const DiffArgs& a, const float* stats) {
  const int n = a.B * a.H * ((a.Nk + kKeyBlock - 1) / kKeyBlock);
  if constexpr (DQ == 32) {
    return go_dkdv<DQ, QS, DV, 4, 2>(a, stats, 0, n);
  } else {
    static ResidentCache cache;
    const int cus = cache.get(reinterpret_cast<const void*>(diff_dkdv_kernel<DQ, QS, DV, RING, 4>), 512).cus;
    int narrow = cus > 0 ? n % cus : 0;
    if (2 * narrow > cus || n - narrow > 8 * cus) narrow = 0;
    const hipError_t err = go_dkdv<DQ, QS, DV, RING, 4>(a, stats, 0, n - narrow);
    return err != hipSuccess ? err : go_dkdv<DQ, QS, DV, 4, 2>(a, stats, n - narrow, narrow);
  }
}

template <int DQ, int QS, int DV, int RING>
hipError_t go_tile(const DiffArgs& a, const float* stats, const float* partial, int groups) {
  const hipError_t err = launch_dkdv<DQ, QS, DV, RING>(a, stats);
  if (err != hipSuccess) return err;
  // workgroups of four waves: 0.44-1.02 of the time of eight (N = 256 .. 16,384)
  constexpr int NW = 4;
  const int n_qtiles = (a.Nq + 32 * NW - 1) / (32 * NW), total = a.B * a.H * n_qtiles;
  const int split_keys = diff_split_keys(a.Nq, a.Nk);
  if (split_keys == 0) {
    diff_dq_kernel<DQ, QS, DV, 4, NW, false>
        <<<total, 64 * NW, 0, a.stream>>>(a, stats, partial, groups, n_qtiles, 1, 0, total, a.scale * kLog2e);
    return hipGetLastError();
  }
  const int n_split = (a.Nk + split_keys - 1) / split_keys;
  diff_dq_kernel<DQ, QS, DV, 4, NW, true><<<total * n_split, 64 * NW, 0, a.stream>>>(
      a, stats, partial, groups, n_qtiles, n_split, split_keys, total * n_split, a.scale * kLog2e);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  diff_dq_join_kernel<<<(unsigned)((2LL * a.B * a.H * a.Nq + 3) / 4), 256, 0, a.stream>>>(a, n_split);
  return hipGetLastError();
}

}  // namespace

static size_t dq_share_floats(int B, int H, int Nq, int Nk, int d) {
  const int s = diff_split_keys(Nq, Nk);
  return s ? (size_t)B * H * ((Nk + s - 1) / s) * 2 * Nq * d : 0;  // (d: a multiple of 8)
}

size_t diff_bwd_workspace_floats(int B, int H, int Nq, int Nk, int d) {
  const size_t bh = (size_t)B * H;
  return dq_share_floats(B, H, Nq, Nk, d) + bh * query_blocks(Nq) * kStat + bh * row_groups(Nq);
}

hipError_t launch_diff_bwd(const DiffArgs& a) {
  float* const stats = a.work + dq_share_floats(a.B, a.H, a.Nq, a.Nk, a.d);
  float* const partial = stats + (size_t)a.B * a.H * query_blocks(a.Nq) * kStat;
  const int groups = row_groups(a.Nq);
  const unsigned grid = (unsigned)(a.B * a.H) * groups;
  if (a.e <= 64) diff_rowdot_kernel<8><<<grid, 256, 0, a.stream>>>(a, stats, partial, groups);
  else if (a.e <= 128) diff_rowdot_kernel<16><<<grid, 256, 0, a.stream>>>(a, stats, partial, groups);
  else diff_rowdot_kernel<32><<<grid, 256, 0, a.stream>>>(a, stats, partial, groups);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const DiffTile t = diff_tile(a.d, a.e);
  if (t.dq == 96) return go_tile<96, 5, 160, 4>(a, stats, partial, groups);
  if (t.dv == 128) return go_tile<64, 4, 128, 6>(a, stats, partial, groups);
  return t.dq == 32 ? go_tile<32, 2, 64, 6>(a, stats, partial, groups) : go_tile<64, 4, 64, 6>(a, stats, partial, groups);
}

}  // namespace vitattn
