// dK and dV of the attention over chosen key blocks (vitattn_sparse_bwd.hip).
//
// Steps of 32 queries: a wave holds its 32 keys' K and V and sums dK and dV. In step j
// the matrix cores run dP(j) = dO(j) V^T (starting at -D) and the scores of step j + 1
// beside the exponentials of step j, then dV += P(j)^T dO(j) beside dS(j), then
// dK += dS(j)^T Q(j). Blocks of 32 queries arrive in a ring of four slots, three steps
// ahead. Steps past the last read zeros: P is 1 there, and dO and Q are zero; so do the
// places that a step of gathered rows (MASKED) leaves empty. (Of a key with an infinite
// element P is NaN there, as dK and dV of that key then are, and of no other.)
#include "vitattn_sparse_bwd.h"

namespace vitattn {

namespace {

constexpr int kRunList = 128;   // query tiles that an item lists at a time
constexpr int kRunRows = 32;    // the same where each row chose its own

template <int D, int KS, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, D == 64 ? 2 : 1) void sparse_dkdv_kernel(const SparseArgs a, const SparseWork w, int words, int run, int n_items, int subs, float c) {
  constexpr int BQ = 32, RING = 4, PF = 3;
  constexpr int NC = (KS + 1) / 2;  // 32-column blocks of d that may hold data
  constexpr int T = BQ * D * 2;
  __shared__ __attribute__((aligned(1024))) char qbuf0[T];
  __shared__ __attribute__((aligned(1024))) char qbuf1[T];
  __shared__ __attribute__((aligned(1024))) char qbuf2[T];
  __shared__ __attribute__((aligned(1024))) char qbuf3[T];
  __shared__ __attribute__((aligned(1024))) char gbuf0[T];
  __shared__ __attribute__((aligned(1024))) char gbuf1[T];
  __shared__ __attribute__((aligned(1024))) char gbuf2[T];
  __shared__ __attribute__((aligned(1024))) char gbuf3[T];
  __shared__ __attribute__((aligned(16))) float sbuf0[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf1[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf2[kStat];
  __shared__ __attribute__((aligned(16))) float sbuf3[kStat];
  constexpr int LIST = MASKED ? kRunRows : kRunList;
  __shared__ int list[LIST];  // query tiles: head of the group << 20 | tile
  __shared__ uint64_t rows[MASKED ? LIST : 1];       // of each tile, those that chose the block
  __shared__ int place[MASKED ? LIST : 1];           // and where the first of them is in ids
  __shared__ uint16_t ids[MASKED ? 64 * LIST : 1];   // rows that chose the block, 32 a step, of one head's 65,536
  __shared__ uint2 steps[MASKED ? 2 * LIST : 1];     // head << 10 | which 65,536; how many of the 32
  __shared__ int n_steps;
  char* const qbuf[RING] = {qbuf0, qbuf1, qbuf2, qbuf3};
  char* const gbuf[RING] = {gbuf0, gbuf1, gbuf2, gbuf3};
  float* const sbuf[RING] = {sbuf0, sbuf1, sbuf2, sbuf3};
  debug_poison_lds(qbuf0, qbuf1, qbuf2, qbuf3, gbuf0, gbuf1, gbuf2, gbuf3, sbuf0, sbuf1, sbuf2, sbuf3, list, rows, place, ids, steps, n_steps);

  // the item: a block, a run of its query tiles, and 32 NW of its keys
  // (each XCD takes a run of them, whose blocks share queries in its L2, unless samples
  // differ in length)
  const unsigned work = a.key_lens ? blockIdx.x : (unsigned)xcd_remap((int)blockIdx.x, (int)gridDim.x);
  const unsigned at = work / (unsigned)subs;
  const int sub = (int)(work - at * subs);
  const int bhk = (int)(at / (unsigned)n_items);
  const int item = (int)(at - bhk * n_items);
  const int total = w.first[(long long)bhk * (a.nb + 1) + a.nb];
  const int4 rec = w.items[(long long)bhk * n_items + item];
  if (item >= total) return;  // (the whole workgroup; what it read was never written)
  const int j = rec.x, n_runs = rec.z;
  const int rank0 = rec.y * run, n_tiles = min(rec.w - rank0, run);
  const int b = bhk / a.Hk, hk = bhk - b * a.Hk, G = a.H / a.Hk;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int in_block = sub * 32 * NW + wave * 32 + (lane & 31);
  const int key = j * a.block + in_block;
  const int Nk = sparse_keys(a, b);
  const int blocks32 = (a.Nq + 31) / 32;

  const int chr = a.d >> 3;
  const int ldq = 2 * a.mq.ld, ldk = 2 * a.mk.ld, ldv = 2 * a.mv.ld, ldg = 2 * a.mg.ld;
  bf16x8 kf[KS], vf[KS];  // B operands of this wave's keys
  {
    const rsrc_t rk = make_rsrc(a.k + b * a.mk.sb + hk * a.mk.sh, (unsigned)(Nk * ldk));
    const rsrc_t rv = make_rsrc(a.v + b * a.mv.sb + hk * a.mv.sh, (unsigned)(Nk * ldv));
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      kf[kk] = as_bf16x8(buffer_load16(rk, chunk_offset(key, 2 * kk + h, ldk, chr)));
      vf[kk] = as_bf16x8(buffer_load16(rv, chunk_offset(key, 2 * kk + h, ldv, chr)));
    }
  }
  TileDma<D, BQ, NW> dmq, dmg;
  dmq.init(wave, lane, ldq, chr);
  dmg.init(wave, lane, ldg, chr);
  constexpr int PW = decltype(dmq)::PER_WAVE, NREQ = 2 * PW + 1;

  // 32 queries on their way: their head and first row, or (MASKED) the 65,536 rows that
  // they are of, how many there are, and which rows this lane requests.
  struct Step {
    int head, row, count;
    uint32_t id[MASKED ? PW + 1 : 1];
  };
  struct Raw {  // as it is read from LDS
    uint2 x;
    uint32_t id[MASKED ? PW + 1 : 1];
  };
  int row_in[MASKED ? PW : 1];    // of the tile, that this lane requests a chunk of
  unsigned col[MASKED ? PW : 1];  // the chunk's offset in the row
  if constexpr (MASKED)
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int pos = decltype(dmq)::instr(wave, i) * 64 + lane;
      row_in[i] = pos / (D / 8);
      col[i] = (unsigned)chunk_offset(0, (pos % (D / 8)) ^ swz<D>(row_in[i]), 0, chr);
    }
  // Step s of n; past the last: rows past the end.
  auto peek = [&](int s, int n) __attribute__((always_inline)) -> Raw {
    s = min(s, n - 1);
    Raw r;
    if constexpr (MASKED) {
      r.x = steps[s];
#pragma unroll
      for (int i = 0; i < PW; ++i) r.id[i] = ids[32 * s + row_in[i]];
      r.id[PW] = ids[32 * s + (lane & 31)];
    } else {
      r.x = make_uint2((uint32_t)list[s >> 1], 0);
    }
    return r;
  };
  auto step_of = [&](const Raw& raw, int s, int n) __attribute__((always_inline)) {
    const uint32_t x = (uint32_t)__builtin_amdgcn_readfirstlane((int)raw.x.x);
    Step st;
    if constexpr (MASKED) {
      const int count = __builtin_amdgcn_readfirstlane((int)raw.x.y);
      st.head = (int)(x >> 10);
      st.row = (int)(x & 1023) << 16;
      st.count = s < n ? count : 0;
#pragma unroll
      for (int i = 0; i <= PW; ++i) st.id[i] = raw.id[i];
    } else {
      st.head = s < n ? (int)(x >> 20) : 0;
      st.row = s < n ? (int)(x & 0xfffff) * kTileRows + 32 * (s & 1) : 32 * blocks32;
    }
    return st;
  };
  auto request = [&](auto slot_tag, const Step& st, int r) __attribute__((always_inline)) {
    constexpr int SL = decltype(slot_tag)::value;
    const int hq = hk * G + st.head;
    if (r < 2 * PW) {
      const bool is_q = r < PW;
      const auto& dma = is_q ? dmq : dmg;
      const int i = is_q ? r : r - PW, ld = is_q ? ldq : ldg;
      const Map& m = is_q ? a.mq : a.mg;
      const rsrc_t rs = make_rsrc((is_q ? a.q : a.dout) + b * m.sb + hq * m.sh, (unsigned)(a.Nq * ld));
      char* const to = is_q ? qbuf[SL] : gbuf[SL];
      if constexpr (!MASKED) {
        dma.issue_one(rs, st.row, ld, to, i);
      } else {
        if (!decltype(dmq)::ALL_ACTIVE && !dma.active) return;
        const unsigned off = row_in[i] < st.count ? (unsigned)((st.row + (int)st.id[i]) * ld) + col[i] : kOobOffset;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)dma.lds_slot(to, i), 16, (int)off, 0, 0, 0);
      }
    } else if (wave == 0) {
      const long long bh = (long long)b * a.H + hq;
      const rsrc_t rs = make_rsrc(w.stats + bh * blocks32 * kStat, (unsigned)blocks32 * kStat * 4);
      unsigned off = (unsigned)((st.row >> 5) * kStat + lane) * 4;
      if constexpr (MASKED) {
        const int row = st.row + (int)st.id[PW];
        off = (lane & 31) < st.count ? (unsigned)((row >> 5) * kStat + (row & 31) + (lane & 32)) * 4 : kOobOffset;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)sbuf[SL], 4, (int)off, 0, 0, 0);
    }
  };

  RowFrag<D> rf;
  TrFrag<D> tf;
  rf.init(lane);
  tf.init(lane);
  f32x16 dk[NC], dv[NC];  // dK^T and dV^T
#pragma unroll
  for (int i = 0; i < NC; ++i) dk[i] = dv[i] = zero16();

  // Lists tiles r0 .. r0 + n - 1 of the block's (ranks over all heads of the group);
  // returns the steps.
  auto fill = [&](int r0, int n) __attribute__((always_inline)) -> int {
    if constexpr (MASKED) {
      const long long slot = ((long long)bhk * n_items + item) * run + r0 - rank0;
      for (int e = threadIdx.x; e < n; e += 64 * NW) {
        list[e] = w.tiles[slot + e];
        rows[e] = w.rows[slot + e];
      }
      __syncthreads();
      // Their places: one after the other, a new step where the head (or the 65,536) ends.
      if (wave == 0) {
        int base = 0, key_before = -1;
        for (int i0 = 0; i0 < n; i0 += 64) {
          const int e = i0 + lane, mine = e < n ? (int)__popcll(rows[e]) : 0, key_of = e < n ? list[e] >> 10 : -1;
          int upto = mine;
#pragma unroll
          for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(upto, d, 64);
            if (lane >= d) upto += x;
          }
          uint64_t left = __ballot(e < n);
          while (left != 0) {
            const int f = __builtin_ctzll(left), of = __shfl(key_of, f, 64);
            const uint64_t same = __ballot(key_of == of) & left;
            const int l = 63 - __builtin_clzll(same), before = f > 0 ? __shfl(upto, f - 1, 64) : 0, here = __shfl(upto, l, 64) - before;
            if (of != key_before) base = (base + 31) & ~31;
            key_before = of;
            if ((same >> lane) & 1) place[e] = base + upto - mine - before;
            for (int t = base / 32 + lane; 32 * t < base + here; t += 64) steps[t] = make_uint2((uint32_t)of, (uint32_t)min(32, base + here - 32 * t));
            base += here;
            left &= ~same;
          }
        }
        if (lane == 0) n_steps = (base + 31) / 32;
      }
      __syncthreads();
      for (int e = wave; e < n; e += NW) {
        const uint64_t m = rows[e];
        if ((m >> lane) & 1) ids[place[e] + (int)__popcll(m & ((1ULL << lane) - 1))] = (uint16_t)((list[e] & 1023) * kTileRows + lane);
      }
      __syncthreads();
      return __builtin_amdgcn_readfirstlane(n_steps);
    }
    if (wave == 0) {
      int base = 0;
      for (int i0 = 0; i0 < G * words && base < r0 + n; i0 += 64) {
        const int i = i0 + lane, g = i / words, word = i - g * words;
        uint64_t m = i < G * words ? w.map[(((long long)b * a.H + hk * G + g) * words + word) * a.nb + j] : 0;
        const int mine = __popcll(m);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int x = __shfl_up(upto, d, 64);
          if (lane >= d) upto += x;
        }
        for (int r = base + upto - mine - r0; m != 0 && r < n; ++r, m &= m - 1)
          if (r >= 0) list[r] = g << 20 | (word * kMapTiles + __builtin_ctzll(m));
        base += __shfl(upto, 63, 64);
      }
    }
    __syncthreads();
    return 2 * n;
  };

  // adds the n steps listed (n > 0: a listed tile has a row that chose the block)
  auto attend = [&](int n) __attribute__((always_inline)) {
    static_for<0, PF>([&](auto SC) __attribute__((always_inline)) {
      const Step st = step_of(peek(decltype(SC)::value, n), decltype(SC)::value, n);
#pragma unroll
      for (int r = 0; r < NREQ; ++r) request(SC, st, r);
    });
    wait_vmem();
    __syncthreads();
    f32x16 sa = zero16(), sb;
#pragma unroll
    for (int i = 0; i < KS; ++i) sa = mfma32(lds_frag_row(qbuf0, rf.at(i)), kf[i], sa);
    bf16x8 lead[2] = {lds_frag_row(gbuf0, rf.at(0)), lds_frag_row(gbuf0, rf.at(1))};  // the next step's first operands
    f32x16 dpn;                                                                       // -D of its rows
    auto start_of = [&](const float* st) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = *reinterpret_cast<const float4*>(st + 8 * g + 4 * h);
        dpn[4 * g] = x.x;
        dpn[4 * g + 1] = x.y;
        dpn[4 * g + 2] = x.z;
        dpn[4 * g + 3] = x.w;
      }
    };
    start_of(sbuf0);
    Raw raw = peek(PF, n);  // of the step that the next one requests
    auto step = [&](auto slot_tag, f32x16& s, f32x16& sn, int i0) __attribute__((always_inline)) {
      constexpr int SL = decltype(slot_tag)::value, NX = (SL + 1) % RING, RF = (SL + PF) % RING;
      constexpr int NP = KS, NS = KS, NV = 2 * NC, NOPS = NP + NS + 2 * NV;
      // Vector work on the ops, evenly: row r's exponential before the dV op that reads
      // it, two ops ahead, then its dS before the dK op.
      constexpr auto exp_at = [](int r) { return r * (NP + NS + NC - 1) / 16; };
      constexpr auto ds_at = [](int r) { return NP + 2 + r * (NS + NV + NC - 3) / 16; };
      static_assert(exp_at(7) <= NP + NS - 2 && exp_at(15) <= NP + NS + NC - 2, "P before dV");
      static_assert(ds_at(0) > exp_at(7) && ds_at(8) > exp_at(15), "P is handed over before dS takes its place");
      static_assert(ds_at(7) <= NP + NS + NV - 2 && ds_at(15) <= NP + NS + NV + NC - 2, "dS before dK");
      static_assert(NREQ <= NOPS, "requests fit the op stream");
      const Step ahead = step_of(raw, i0 + PF, n);
      raw = peek(i0 + PF + 1, n);
      f32x16 dp = dpn;
      f32x16 l;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = *reinterpret_cast<const float4*>(sbuf[SL] + 32 + 8 * g + 4 * h);
        l[4 * g] = x.x;
        l[4 * g + 1] = x.y;
        l[4 * g + 2] = x.z;
        l[4 * g + 3] = x.w;
      }
      bf16x8 pb[2], db[2];
      auto load_op = [&](int i) -> bf16x8 {
        if (i >= NOPS) return lds_frag_row(gbuf[NX], rf.at(i - NOPS));
        if (i < NP) return lds_frag_row(gbuf[SL], rf.at(i));
        if (i < NP + NS) return lds_frag_row(qbuf[NX], rf.at(i - NP));
        const int t = (i - NP - NS) % NV;
        return tf.load(i < NP + NS + NV ? gbuf[SL] : qbuf[SL], 16 * (t / NC), t % NC);
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
        if constexpr (i < NP) {
          dp = mfma32(aq[i % 3], vf[i], dp);
        } else if constexpr (i < NP + NS) {
          if constexpr (i == NP) sn = zero16();
          sn = mfma32(aq[i % 3], kf[i - NP], sn);
        } else if constexpr (i < NP + NS + NV) {
          constexpr int t = i - NP - NS;
          dv[t % NC] = mfma32(aq[i % 3], pb[t / NC], dv[t % NC]);
        } else {
          constexpr int t = i - NP - NS - NV;
          dk[t % NC] = mfma32(aq[i % 3], db[t / NC], dk[t % NC]);
        }
        if constexpr (i < NREQ) request(std::integral_constant<int, RF>{}, ahead, i);
        if constexpr (i == NOPS - 2) start_of(sbuf[NX]);
        static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          if constexpr (exp_at(r) == i) {
            float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -l[r]));
            pin(x);
            s[r] = x;
            if constexpr ((r & 7) == 7) pb[r >> 3] = acc_to_operand(s, r >> 3);
          }
          if constexpr (ds_at(r) == i) {
            float x = s[r] * dp[r];
            pin(x);
            s[r] = x;
            if constexpr ((r & 7) == 7) db[r >> 3] = acc_to_operand(s, r >> 3);
          }
        });
        sched_fence();
      });
      __builtin_amdgcn_s_setprio(0);
      // this wave's requests of the step before last have landed
      wait_vmem_leave<(PF - 2) * 2 * (decltype(dmq)::ALL_ACTIVE ? PW : 0)>();
      barrier_lds();
    };
    const int padded_steps = (n + RING - 1) / RING * RING;
    for (int i = 0; i < padded_steps; i += RING) {
      step(std::integral_constant<int, 0>{}, sa, sb, i);
      step(std::integral_constant<int, 1>{}, sb, sa, i + 1);
      step(std::integral_constant<int, 2>{}, sa, sb, i + 2);
      step(std::integral_constant<int, 3>{}, sb, sa, i + 3);
    }
    wait_vmem();  // requests past the last step must land before this LDS is reassigned
    __syncthreads();
  };

  for (int r = 0; r < n_tiles; r += LIST) {
    const int n = min(n_tiles - r, LIST);
    attend(fill(rank0 + r, n));
  }

  const bool there = key < Nk;  // (of the sample's keys)
  if (n_runs > 1) {
    float* const share = w.shares + ((((long long)bhk * n_items + item) * 2) * a.block + in_block) * a.d;
#pragma unroll
    for (int cb = 0; cb < NC; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * cb + 8 * g + 4 * h;
        if (col >= a.d) continue;
        *reinterpret_cast<float4*>(share + col) = make_float4(dk[cb][4 * g], dk[cb][4 * g + 1], dk[cb][4 * g + 2], dk[cb][4 * g + 3]);
        *reinterpret_cast<float4*>(share + (long long)a.block * a.d + col) =
            make_float4(dv[cb][4 * g], dv[cb][4 * g + 1], dv[cb][4 * g + 2], dv[cb][4 * g + 3]);
      }
    return;
  }
  if (key >= a.Nk) return;
  uint16_t* const ok = a.dk + b * a.mdk.sb + hk * a.mdk.sh + (long long)key * a.mdk.ld;
  uint16_t* const ov = a.dv + b * a.mdv.sb + hk * a.mdv.sh + (long long)key * a.mdv.ld;
#pragma unroll
  for (int cb = 0; cb < NC; ++cb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * cb + 8 * g + 4 * h;
      if (col >= a.d) continue;
      float x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = there ? dk[cb][4 * g + e] * a.scale : 0.f;
        y[e] = there ? dv[cb][4 * g + e] : 0.f;
      }
      store4_bf16(ok + col, x[0], x[1], x[2], x[3]);
      store4_bf16(ov + col, y[0], y[1], y[2], y[3]);
    }
}

template <int D, int KS, int NW, bool MASKED>
hipError_t go(const SparseArgs& a, const SparseWork& w, const SparsePlan& p) {
  const int subs = a.block / (32 * NW);
  const long long grid = (long long)a.B * a.Hk * p.items * subs;
  sparse_dkdv_kernel<D, KS, NW, MASKED><<<(unsigned)grid, 64 * NW, 0, a.stream>>>(a, w, p.words, p.run, (int)p.items, subs, a.scale * kLog2e);
  return hipGetLastError();
}
template <int D, int KS>
hipError_t go_tile(const SparseArgs& a, const SparseWork& w, const SparsePlan& p) {
  const bool whole = one_group(a, 64);
  if (a.block % 128 == 0) return whole ? go<D, KS, 4, false>(a, w, p) : go<D, KS, 4, true>(a, w, p);
  return whole ? go<D, KS, 2, false>(a, w, p) : go<D, KS, 2, true>(a, w, p);
}

}  // namespace

hipError_t launch_sparse_dkdv(const SparseArgs& a, const SparseWork& w, const SparsePlan& p) {
  switch (tile_width(a.d)) {
    case 64: return go_tile<64, 4>(a, w, p);
    case 96: return a.d <= 80 ? go_tile<96, 5>(a, w, p) : go_tile<96, 6>(a, w, p);
    case 128: return go_tile<128, 8>(a, w, p);
    default: return go_tile<160, 10>(a, w, p);
  }
}

}  // namespace vitattn
