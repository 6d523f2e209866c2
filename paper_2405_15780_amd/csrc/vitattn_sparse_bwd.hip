// Backward of the attention over chosen key blocks (vitattn_sparse_fwd.hip), P
// recomputed from q, k and the saved LSE:
//
//   D_i = dO_i . O_i,  dS = P o (dO V^T - D),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
//   1. row pass: -D and LSE log2(e) per query (HBM-bound; O in fp32), and zeroed counts.
//   2. map: for each key block the query tiles (of 64) that chose it, a bit each, and how
//      many. A workgroup per 64 tiles and head collects them in LDS, so nothing global is
//      cleared or merged but the counts (integers: their order does not matter).
//   3. plan: each key block's tiles are cut into runs of at most `run`, a work item each:
//      a block that every query chose does not keep one workgroup for all of them. A
//      prefix sum over the blocks gives the items their places.
//   4. dK/dV: an item's run of query tiles for 32 NW keys, a wave per 32 keys. The grid is
//      the largest number of items that the sizes allow; those past the last end at once.
//      Items of a block of several runs write fp32 shares.
//   5. a block of several runs adds its shares in their order.
//   6. dQ: as the forward walks its list of key tiles.
//
// P and dS are rounded to bf16 as matrix-core operands; everything else is fp32 until the
// outputs are rounded once. No atomics on results: each output row is one workgroup's, or
// a sum in fixed order. Of grouped heads (H > Hk) an item's run goes over the query tiles
// of all heads that share the keys.
//
// Where a query tile's rows chose apart (MASKED) its other rows arrive as zeros: Q, dO and
// their statistics are read past the buffer's end, and P dO and dS Q add nothing, whatever
// the rows hold. dQ's rows share the keys they read; there a tile whose dQ is not finite
// goes over its rows one at a time, as the forward does.
#include "vitattn_sparse.h"

namespace vitattn {

namespace {

constexpr int kTileRows = 64;   // of a query tile
constexpr int kMapTiles = 64;   // query tiles of a map word
constexpr int kMapRows = kTileRows * kMapTiles;
constexpr int kRowBlock = 64;   // query rows of a row-pass workgroup
constexpr int kRunList = 128;   // query tiles that an item lists at a time
constexpr int kStat = 64;       // floats per 32 queries: -D, then LSE log2(e)

struct Plan {  // sizes of the backward's workspace
  int tiles, words;   // query tiles of a head, map words of a key block
  int run;            // query tiles of an item
  long long items;    // items of a key head, at most
};
Plan plan_of(const SparseArgs& a) {
  Plan p;
  p.tiles = (a.Nq + kTileRows - 1) / kTileRows;
  p.words = (p.tiles + kMapTiles - 1) / kMapTiles;
  // blocks that a tile's rows can choose
  const long long groups = a.q_block >= kTileRows ? (a.q_block % kTileRows == 0 ? 1 : 2)
                                                  : min((long long)kTileRows / a.q_block + 2, (long long)min(a.Nq, kTileRows));
  const long long pairs = (long long)(a.H / a.Hk) * p.tiles * min(groups * a.topk, (long long)a.nb);
  // runs of 64 tiles, of 32 where there are few blocks to fill the card with, and longer
  // ones where the shares of as many items would outgrow eight times the keys
  p.run = (int)max(a.nb < 256 ? 32LL : 64LL, min(4096LL, (pairs + 8LL * a.nb - 1) / (8LL * a.nb)));
  p.items = a.nb + pairs / p.run;  // sum over the blocks of max(1, ceil(count / run))
  return p;
}

// workspace
struct Work {
  float* stats;      // [BH][32-query blocks][kStat]
  uint64_t* map;     // [BH][words][nb]
  int* counts;       // [B Hk][nb]
  int* first;        // [B Hk][nb + 1]: a block's first item; the number of items
  int4* items;       // [B Hk][items]: an item's block, its run, the block's runs and query tiles
  float* shares;     // [B Hk][items][2][block][d]
  size_t bytes;
};
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
Work work_of(const SparseArgs& a, const Plan& p) {
  Work w;
  const size_t bh = (size_t)a.B * a.H, bhk = (size_t)a.B * a.Hk;
  char* at = a.work;
  size_t n = 0;
  auto take = [&](size_t bytes) {
    char* x = at + n;
    n += padded(bytes);
    return x;
  };
  w.stats = reinterpret_cast<float*>(take(bh * ((a.Nq + 31) / 32) * kStat * 4));
  w.map = reinterpret_cast<uint64_t*>(take(bh * p.words * a.nb * 8));
  w.counts = reinterpret_cast<int*>(take(bhk * a.nb * 4));
  w.first = reinterpret_cast<int*>(take(bhk * (a.nb + 1) * 4));
  w.items = reinterpret_cast<int4*>(take(bhk * p.items * sizeof(int4)));
  w.shares = reinterpret_cast<float*>(take(p.items > a.nb ? bhk * p.items * 2 * a.block * a.d * 4 : 0));
  w.bytes = n;
  return w;
}

// LPR lanes per row take 8 columns each.
template <int LPR>
__global__ __launch_bounds__(256) void sparse_rowdot_kernel(const SparseArgs a, float* __restrict__ stats, int* counts, int n_counts, int groups) {
  constexpr int RPP = 256 / LPR;  // rows at a time
  const int bh = blockIdx.x / groups, group = blockIdx.x - bh * groups;
  const int b = bh / a.H, head = bh - b * a.H;
  const int col = 8 * (threadIdx.x % LPR);
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n_counts; i += gridDim.x * 256) counts[i] = 0;
  const float* const o = a.o32 + (long long)bh * a.Nq * a.d;
  const uint16_t* const g = a.dout + b * a.mg.sb + head * a.mg.sh;
  const int blocks = (a.Nq + 31) / 32;
  float* const st = stats + (long long)bh * blocks * kStat;
#pragma unroll
  for (int r0 = 0; r0 < kRowBlock; r0 += RPP) {
    const int row = group * kRowBlock + r0 + threadIdx.x / LPR;
    float d = 0.f;
    if (row < a.Nq && col < a.d) {
      const bf16x8 gv = as_bf16x8(*reinterpret_cast<const uint4*>(g + (long long)row * a.mg.ld + col));
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(o + (long long)row * a.d + col + i);
        d += (float)gv[i] * x.x + (float)gv[i + 1] * x.y + (float)gv[i + 2] * x.z + (float)gv[i + 3] * x.w;
      }
    }
#pragma unroll
    for (int m = LPR / 2; m >= 1; m >>= 1) d += __shfl_xor(d, m, 64);
    if (col == 0 && row < 32 * blocks) {
      // rows past the last, and those without keys: P = exp2(s - inf) = 0
      float l = row < a.Nq ? a.lse[(long long)bh * a.Nq + row] * kLog2e : INFINITY;
      if (l == -INFINITY) l = INFINITY;
      float* s = st + (row >> 5) * kStat + (row & 31);
      s[0] = -d;
      s[32] = l;
    }
  }
}

// The query tiles that chose each key block: bit t of map[bh][word][j] for tile 64 word + t.
constexpr int kMapChunk = 4096;  // key blocks at a time
__global__ __launch_bounds__(1024) void sparse_map_kernel(const SparseArgs a, uint64_t* __restrict__ map, int* __restrict__ counts, int words) {
  __shared__ unsigned long long bits[kMapChunk];
  debug_poison_lds(bits);
  const int bh = blockIdx.x / words, word = blockIdx.x - bh * words;
  const int b = bh / a.H, head = bh - b * a.H, hk = head / (a.H / a.Hk);
  const int Nk = sparse_keys(a, b), real = (Nk + a.block - 1) / a.block;
  const long long row0 = (long long)word * kMapRows;
  const int first_group = (int)(row0 / a.q_block);
  const int last = (int)((min(row0 + kMapRows, (long long)a.Nq) - 1) / a.q_block);
  const long long n = (long long)(last - first_group + 1) * a.topk;
  const int* const chosen = a.blocks + ((long long)bh * a.groups + first_group) * a.topk;
  for (int j0 = 0; j0 < a.nb; j0 += kMapChunk) {
    const int here = min(a.nb - j0, kMapChunk);
    for (int i = threadIdx.x; i < here; i += 1024) bits[i] = 0;
    __syncthreads();
    for (long long e = threadIdx.x; e < n; e += 1024) {
      const int id = chosen[e];
      if ((unsigned)id >= (unsigned)real || id < j0 || id >= j0 + here) continue;
      const long long g = first_group + e / a.topk;
      // the group's rows [lo, hi) of this word's
      const long long lo = max(g * a.q_block - row0, 0LL), hi = min(min((g + 1) * a.q_block, (long long)a.Nq) - row0, (long long)kMapRows);
      const int t0 = (int)(lo / kTileRows), t1 = (int)((hi - 1) / kTileRows);
      const unsigned long long m = (t1 == 63 ? ~0ULL : (2ULL << t1) - 1) & (~0ULL << t0);
      atomicOr(&bits[id - j0], m);
    }
    __syncthreads();
    uint64_t* const out = map + ((long long)bh * words + word) * a.nb + j0;
    int* const count = counts + ((long long)b * a.Hk + hk) * a.nb + j0;
    for (int i = threadIdx.x; i < here; i += 1024) {
      const uint64_t m = bits[i];
      out[i] = m;
      if (m) atomicAdd(&count[i], __popcll(m));
    }
    __syncthreads();
  }
}

// Items of each key block, max(1, ceil(count / run)), and their places: a workgroup per
// key head.
__global__ __launch_bounds__(1024) void sparse_plan_kernel(const SparseArgs a, const int* __restrict__ counts, int* __restrict__ first, int4* __restrict__ items, int run,
                                                           long long n_items) {
  __shared__ int sums[16];
  debug_poison_lds(sums);
  const long long bhk = blockIdx.x;
  const int per = (a.nb + 1023) / 1024, j0 = threadIdx.x * per;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  counts += bhk * a.nb;
  first += bhk * (a.nb + 1);
  items += bhk * n_items;
  auto of = [&](int j) { return max(1, (counts[j] + run - 1) / run); };
  int n = 0;
  for (int j = j0; j < min(j0 + per, a.nb); ++j) n += of(j);
  int upto = n;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(upto, d, 64);
    if (lane >= d) upto += x;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int at = upto - n;
  for (int w = 0; w < wave; ++w) at += sums[w];
  for (int j = j0; j < min(j0 + per, a.nb); ++j) {
    first[j] = at;
    const int m = of(j);
    for (int i = 0; i < m; ++i) items[at + i] = make_int4(j, i, m, counts[j]);
    at += m;
  }
  if (threadIdx.x == 1023) first[a.nb] = at;
}

// ------------------------------------------------------------------ dK / dV
//
// Steps of 32 queries: a wave holds its 32 keys' K and V and sums dK and dV. In step j
// the matrix cores run dP(j) = dO(j) V^T (starting at -D) and the scores of step j + 1
// beside the exponentials of step j, then dV += P(j)^T dO(j) beside dS(j), then
// dK += dS(j)^T Q(j). Blocks of 32 queries arrive in a ring of four slots, three steps
// ahead. Steps past the last read zeros: P is 1 there, and dO and Q are zero.
template <int D, int KS, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, D == 64 ? 2 : 1) void sparse_dkdv_kernel(const SparseArgs a, const Work w, int words, int run, int n_items, int subs, float c) {
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
  __shared__ int list[kRunList];  // query tiles: head of the group << 20 | tile
  __shared__ uint64_t rows[MASKED ? kRunList : 1];  // of each tile, those that chose the block
  __shared__ uint2 steps[MASKED ? 2 * kRunList : 1];  // halves that any did: head << 21 | half, rows
  __shared__ int n_halves;
  char* const qbuf[RING] = {qbuf0, qbuf1, qbuf2, qbuf3};
  char* const gbuf[RING] = {gbuf0, gbuf1, gbuf2, gbuf3};
  float* const sbuf[RING] = {sbuf0, sbuf1, sbuf2, sbuf3};
  debug_poison_lds(qbuf0, qbuf1, qbuf2, qbuf3, gbuf0, gbuf1, gbuf2, gbuf3, sbuf0, sbuf1, sbuf2, sbuf3, list, rows, steps, n_halves);

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

  // 32 queries on their way: where they are, and (MASKED) the rows that chose the block
  struct Step {
    int head, row;
    uint32_t mine;
  };
  // Step s of n, as it is read from LDS and (later) where it is; past the last: rows past
  // the end.
  auto peek = [&](int s, int n) __attribute__((always_inline)) -> uint2 {
    s = min(s, n - 1);
    if constexpr (MASKED) return steps[s];
    else return make_uint2((uint32_t)list[s >> 1], 0xffffffffu);
  };
  auto step_of = [&](uint2 raw, int s, int n) __attribute__((always_inline)) {
    const uint32_t x = (uint32_t)__builtin_amdgcn_readfirstlane((int)raw.x);
    const uint32_t mine = MASKED ? (uint32_t)__builtin_amdgcn_readfirstlane((int)raw.y) : 0xffffffffu;
    if (s >= n) return Step{0, 32 * blocks32, 0xffffffffu};
    if (MASKED) return Step{(int)(x >> 21), (int)(x & 0x1fffff) * 32, mine};
    return Step{(int)(x >> 20), (int)(x & 0xfffff) * kTileRows + 32 * (s & 1), mine};
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
        // rows that did not choose the block are read past the end: zeros
        if (!decltype(dmq)::ALL_ACTIVE && !dma.active) return;
        const int row = ((decltype(dmq)::instr(wave, i)) * 64 + lane) / (D / 8);
        const unsigned off = (st.mine >> row) & 1 ? (unsigned)(st.row * ld) + dma.voff[i] : kOobOffset;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)dma.lds_slot(to, i), 16, (int)off, 0, 0, 0);
      }
    } else if (wave == 0) {
      const long long bh = (long long)b * a.H + hq;
      const rsrc_t rs = make_rsrc(w.stats + bh * blocks32 * kStat, (unsigned)blocks32 * kStat * 4);
      const unsigned off = (unsigned)((st.row >> 5) * kStat + lane) * 4;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)sbuf[SL], 4, (int)(!MASKED || ((st.mine >> (lane & 31)) & 1) ? off : kOobOffset), 0, 0, 0);
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
    if constexpr (MASKED) {
      // a wave per tile, a lane per row: whether its group chose the block
      for (int e = wave; e < n; e += NW) {
        const int x = list[e], row = (x & 0xfffff) * kTileRows + lane;
        bool mine = false;
        if (row < a.Nq) {
          const int* const chosen = a.blocks + (((long long)b * a.H + hk * G + (x >> 20)) * a.groups + row / a.q_block) * a.topk;
          for (int i = 0; i < a.topk; ++i) mine = mine || chosen[i] == j;
        }
        const uint64_t bits = __ballot(mine);
        if (lane == 0) rows[e] = bits;
      }
      __syncthreads();
      if (wave == 0) {
        int found = 0;
        for (int i0 = 0; i0 < 2 * n; i0 += 64) {
          const int i = i0 + lane;
          const uint32_t mine = i < 2 * n ? reinterpret_cast<const uint32_t*>(rows)[i] : 0u;
          const uint64_t taken = __ballot(mine != 0);
          if (mine != 0) {
            const int x = list[i >> 1];
            steps[found + (int)__popcll(taken & ((1ULL << lane) - 1))] = make_uint2((uint32_t)(x >> 20) << 21 | (uint32_t)(2 * (x & 0xfffff) + (i & 1)), mine);
          }
          found += (int)__popcll(taken);
        }
        if (lane == 0) n_halves = found;
      }
      __syncthreads();
      return __builtin_amdgcn_readfirstlane(n_halves);
    }
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
    uint2 raw = peek(PF, n);  // of the step that the next one requests
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

  for (int r = 0; r < n_tiles; r += kRunList) {
    const int n = min(n_tiles - r, kRunList);
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

// Adds the shares of a key block of several runs in their order: a workgroup per block,
// four columns per thread.
__global__ __launch_bounds__(256) void sparse_share_kernel(const SparseArgs a, const Work w, long long n_items) {
  const int bhk = blockIdx.x / a.nb, j = blockIdx.x - bhk * a.nb;
  const int* const first = w.first + (long long)bhk * (a.nb + 1);
  const int i0 = first[j], n = first[j + 1] - i0;
  if (n <= 1) return;
  const int b = bhk / a.Hk, hk = bhk - b * a.Hk, Nk = sparse_keys(a, b);
  const long long size = (long long)a.block * a.d;
  const float* const src = w.shares + ((long long)bhk * n_items + i0) * 2 * size;
  for (int at = 4 * threadIdx.x; at < 2 * size; at += 4 * 256) {
    const int of = at >= size, in = at - of * (int)size, row = in / a.d, col = in - row * a.d, key = j * a.block + row;
    if (key >= a.Nk) continue;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (key < Nk)
      for (int i = 0; i < n; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(src + i * 2 * size + at);
        s = make_float4(s.x + x.x, s.y + x.y, s.z + x.z, s.w + x.w);
      }
    const float f = of ? 1.f : a.scale;
    const Map& m = of ? a.mdv : a.mdk;
    store4_bf16((of ? a.dv : a.dk) + b * m.sb + hk * m.sh + (long long)key * m.ld + col, s.x * f, s.y * f, s.z * f, s.w * f);
  }
}

// ------------------------------------------------------------------ dQ
//
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
      uint32_t mine = 0xffffffffu;
      if constexpr (MASKED) mine = reinterpret_cast<const uint32_t*>(list.masks)[2 * entry[SL] + wave];
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
            float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
            pin(x);
            s[r] = x;
          }
        });
        static_for<0, 16>([&](auto RC) __attribute__((always_inline)) {
          constexpr int r = decltype(RC)::value;
          if constexpr (ds_at(r) == i) {
            float x = s[r] * dp[r];
            if constexpr (MASKED) x = (mine >> (lane & 31)) & 1 ? x : 0.f;  // (of a block that the row did not choose)
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
hipError_t go_dkdv(const SparseArgs& a, const Work& w, const Plan& p) {
  const int subs = a.block / (32 * NW);
  const long long grid = (long long)a.B * a.Hk * p.items * subs;
  sparse_dkdv_kernel<D, KS, NW, MASKED><<<(unsigned)grid, 64 * NW, 0, a.stream>>>(a, w, p.words, p.run, (int)p.items, subs, a.scale * kLog2e);
  return hipGetLastError();
}

template <int D, int KS, int NW, bool MASKED>
hipError_t go_dq(const SparseArgs& a, const Work& w) {
  const int n_qtiles = (a.Nq + 32 * NW - 1) / (32 * NW), total = a.B * a.H * n_qtiles;
  sparse_dq_kernel<D, KS, NW, MASKED><<<total, 64 * NW, 0, a.stream>>>(a, w.stats, n_qtiles, total, a.scale * kLog2e);
  return hipGetLastError();
}

template <int D, int KS>
hipError_t go_tile(const SparseArgs& a, const Work& w, const Plan& p) {
  const bool whole = one_group(a, 64);
  hipError_t err;
  if (a.block % 128 == 0) err = whole ? go_dkdv<D, KS, 4, false>(a, w, p) : go_dkdv<D, KS, 4, true>(a, w, p);
  else err = whole ? go_dkdv<D, KS, 2, false>(a, w, p) : go_dkdv<D, KS, 2, true>(a, w, p);
  if (err != hipSuccess) return err;
  if (p.items > a.nb) {
    sparse_share_kernel<<<(unsigned)(a.B * a.Hk) * a.nb, 256, 0, a.stream>>>(a, w, p.items);
    if ((err = hipGetLastError()) != hipSuccess) return err;
  }
  if (one_group(a, 128) && a.Nq > 64) return go_dq<D, KS, 4, false>(a, w);
  return whole ? go_dq<D, KS, 2, false>(a, w) : go_dq<D, KS, 2, true>(a, w);
}

}  // namespace

long long sparse_bwd_items(const SparseArgs& a) { return plan_of(a).items; }

size_t sparse_bwd_workspace_bytes(const SparseArgs& a) { return work_of(a, plan_of(a)).bytes; }

hipError_t launch_sparse_bwd(const SparseArgs& a) {
  const Plan p = plan_of(a);
  const Work w = work_of(a, p);
  const int groups = (a.Nq + kRowBlock - 1) / kRowBlock, n_counts = a.B * a.Hk * a.nb;
  const unsigned grid = (unsigned)(a.B * a.H) * groups;
  if (a.d <= 64) sparse_rowdot_kernel<8><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  else if (a.d <= 128) sparse_rowdot_kernel<16><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  else sparse_rowdot_kernel<32><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  sparse_map_kernel<<<(unsigned)(a.B * a.H) * p.words, 1024, 0, a.stream>>>(a, w.map, w.counts, p.words);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  sparse_plan_kernel<<<a.B * a.Hk, 1024, 0, a.stream>>>(a, w.counts, w.first, w.items, p.run, p.items);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  switch (tile_width(a.d)) {
    case 64: return go_tile<64, 4>(a, w, p);
    case 96: return a.d <= 80 ? go_tile<96, 5>(a, w, p) : go_tile<96, 6>(a, w, p);
    case 128: return go_tile<128, 8>(a, w, p);
    default: return go_tile<160, 10>(a, w, p);
  }
}

}  // namespace vitattn
