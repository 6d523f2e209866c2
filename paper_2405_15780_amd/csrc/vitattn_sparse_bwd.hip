// Backward of the attention over chosen key blocks (vitattn_sparse_fwd.hip), P
// recomputed from q, k and the saved LSE:
//
//   D_i = dO_i . O_i,  dS = P o (dO V^T - D),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
//   1. row pass: -D and LSE log2(e) per query (HBM-bound; O in fp32), and zeroed counts.
//   2. map: for each key block the query tiles (of 64) that chose it, a bit each, and how
//      many. A workgroup per 16 tiles and head collects them in LDS, so nothing global is
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
// Where a query tile's rows chose apart (MASKED), dK/dV gathers those that chose the block,
// 32 a step, from wherever they are: no other row is read. Two more passes list them: the
// rank of each word's first tile among a block's, then a workgroup per tile collects which
// rows chose what, as the forward does, and puts a tile and its 64 bits in their item's place. dQ's rows share the keys they
// read; there a tile whose dQ is not finite goes over its rows one at a time, as the
// forward does.
//
// Heads of 64, 8 of them, 32,768 queries in groups of 64 of 32 blocks of 64 keys each: row pass
// 17 us (5.0 TB/s), map 6, plan 5, dK/dV 369-397 (0.69 PFLOP/s; matrix cores busy 51-53 %, LDS
// 41 %), shares 17, dQ 233-260. 2 samples of 4 heads (2 of keys) of 72, 8,003 queries of 8 blocks
// each: 8, 8, 5, 82, 14 and 183 us, and 14 for the rows' lists. There dK/dV took 266 us reading
// every half tile that any row chose from, and 139 where each item looked through its tiles'
// choices itself.

#include "vitattn_sparse_bwd.h"

namespace vitattn {

namespace {

constexpr int kRowBlock = 64;   // query rows of a row-pass workgroup

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
constexpr int kMapPart = 16;     // query tiles of a workgroup: a quarter of a word
__global__ __launch_bounds__(1024) void sparse_map_kernel(const SparseArgs a, uint64_t* __restrict__ map, int* __restrict__ counts, int words, int parts) {
  __shared__ uint32_t bits[kMapChunk];
  debug_poison_lds(bits);
  constexpr int ROWS = kMapPart * kTileRows, PARTS = kMapTiles / kMapPart;
  const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts;
  const int b = bh / a.H, head = bh - b * a.H, hk = head / (a.H / a.Hk);
  const int Nk = sparse_keys(a, b), real = (Nk + a.block - 1) / a.block;
  const long long row0 = (long long)part * ROWS;
  const int first_group = (int)min(row0 / a.q_block, (long long)a.groups);
  const int last = (int)((min(row0 + ROWS, (long long)a.Nq) - 1) / a.q_block);
  // (at most 1,024 groups of 1,024; none where the part of a last word lies behind the rows)
  const int n = row0 < a.Nq ? (last - first_group + 1) * a.topk : 0;
  const int* const chosen = a.blocks + ((long long)bh * a.groups + first_group) * a.topk;
  uint16_t* const out = reinterpret_cast<uint16_t*>(map + ((long long)bh * words + part / PARTS) * a.nb) + part % PARTS;
  int* const count = counts + ((long long)b * a.Hk + hk) * a.nb;
  for (int j0 = 0; j0 < a.nb; j0 += kMapChunk) {
    const int here = min(a.nb - j0, kMapChunk);
    for (int i = threadIdx.x; i < here; i += 1024) bits[i] = 0;
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += 1024) {
      const int id = chosen[e];
      if ((unsigned)id >= (unsigned)real || id < j0 || id >= j0 + here) continue;
      const long long g = first_group + e / a.topk;
      // the group's rows [lo, hi) of these
      const int lo = (int)max(g * a.q_block - row0, 0LL), hi = (int)min(min((g + 1) * a.q_block, (long long)a.Nq) - row0, (long long)ROWS);
      const int t0 = lo / kTileRows, t1 = (hi - 1) / kTileRows;
      atomicOr(&bits[id - j0], (2u << t1) - (1u << t0));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < here; i += 1024) {
      const uint32_t m = bits[i];
      out[(long long)(j0 + i) * PARTS] = (uint16_t)m;
      if (m) atomicAdd(&count[j0 + i], __popc(m));
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

// Of query tiles whose rows choose apart, where each block's begin in the words of the map:
// a thread per block.
__global__ __launch_bounds__(256) void sparse_rank_kernel(const SparseArgs a, const SparseWork w, int words, int groups) {
  const int bhk = blockIdx.x / groups, j = 256 * (blockIdx.x - bhk * groups) + threadIdx.x;
  if (j >= a.nb) return;
  const long long at = (long long)bhk * (a.H / a.Hk) * words * a.nb + j;
  int n = 0;
#pragma unroll 4
  for (int i = 0; i < a.H / a.Hk * words; ++i) {
    w.ranks[at + (long long)i * a.nb] = n;
    n += __popcll(w.map[at + (long long)i * a.nb]);
  }
}

// And the rows of each that chose its blocks, to the items' places: a workgroup per tile.
__global__ __launch_bounds__(128) void sparse_rows_kernel(const SparseArgs a, const SparseWork w, int words, int tiles, int run, long long n_items) {
  __shared__ BlockList<true> list;
  debug_poison_lds(list);
  const int bh = blockIdx.x / tiles, t = blockIdx.x - bh * tiles;
  const int b = bh / a.H, head = bh - b * a.H, G = a.H / a.Hk;
  const long long bhk = (long long)b * a.Hk + head / G;
  const int Nk = sparse_keys(a, b), real = (Nk + a.block - 1) / a.block;
  const Chosen chosen(a, bh, t * kTileRows, kTileRows);
  const int left = a.Nq - t * kTileRows;
  const uint64_t there = left >= 64 ? ~0ULL : (1ULL << left) - 1;
  const int* const first = w.first + bhk * (a.nb + 1);
  const long long word = ((long long)bh * words + t / kMapTiles) * a.nb;
  const int count = list.build<128>(a, chosen, real, ~0ULL);
  for (int r = 0; r < count; r += list.kCap) {
    const int n = min(count - r, list.kCap);
    list.fill<128>(a, chosen, real, ~0ULL, r, n);
    for (int i = threadIdx.x; i < n; i += 128) {
      const int j = list.id[i];
      const int rank = w.ranks[word + j] + __popcll(w.map[word + j] & ((1ULL << (t % kMapTiles)) - 1));
      const long long slot = (bhk * n_items + first[j]) * run + rank;
      w.rows[slot] = list.masks[i] & there;
      w.tiles[slot] = (head % G) << 20 | t;
    }
    __syncthreads();  // before another list
  }
}

// Adds the shares of a key block of several runs in their order: four columns per thread.
__global__ __launch_bounds__(256) void sparse_share_kernel(const SparseArgs a, const SparseWork w, long long n_items) {
  const int bhk = blockIdx.x / a.nb, j = blockIdx.x - bhk * a.nb;
  const int* const first = w.first + (long long)bhk * (a.nb + 1);
  const int i0 = first[j], n = first[j + 1] - i0;
  if (n <= 1) return;
  const int b = bhk / a.Hk, hk = bhk - b * a.Hk, Nk = sparse_keys(a, b);
  const int size = a.block * a.d, at = 4 * (256 * blockIdx.y + threadIdx.x);
  if (at >= 2 * size) return;
  const float* const src = w.shares + ((long long)bhk * n_items + i0) * 2 * size + at;
  const int of = at >= size, in = at - of * size, row = in / a.d, col = in - row * a.d, key = j * a.block + row;
  if (key >= a.Nk) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (key < Nk) {
    constexpr int U = 4;
    for (int i = 0; i < n; i += U) {
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const float4*>(src + (long long)min(i + u, n - 1) * 2 * size);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < n) s = make_float4(s.x + x[u].x, s.y + x[u].y, s.z + x[u].z, s.w + x[u].w);
    }
  }
  const float f = of ? 1.f : a.scale;
  const Map& m = of ? a.mdv : a.mdk;
  store4_bf16((of ? a.dv : a.dk) + b * m.sb + hk * m.sh + (long long)key * m.ld + col, s.x * f, s.y * f, s.z * f, s.w * f);
}

}  // namespace

long long sparse_bwd_items(const SparseArgs& a) { return plan_of(a).items; }

size_t sparse_bwd_workspace_bytes(const SparseArgs& a) { return work_of(a, plan_of(a)).bytes; }

hipError_t launch_sparse_bwd(const SparseArgs& a) {
  const SparsePlan p = plan_of(a);
  const SparseWork w = work_of(a, p);
  const int groups = (a.Nq + kRowBlock - 1) / kRowBlock, n_counts = a.B * a.Hk * a.nb;
  const unsigned grid = (unsigned)(a.B * a.H) * groups;
  if (a.d <= 64) sparse_rowdot_kernel<8><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  else if (a.d <= 128) sparse_rowdot_kernel<16><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  else sparse_rowdot_kernel<32><<<grid, 256, 0, a.stream>>>(a, w.stats, w.counts, n_counts, groups);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int parts = p.words * (kMapTiles / kMapPart);
  sparse_map_kernel<<<(unsigned)(a.B * a.H) * parts, 1024, 0, a.stream>>>(a, w.map, w.counts, p.words, parts);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  sparse_plan_kernel<<<a.B * a.Hk, 1024, 0, a.stream>>>(a, w.counts, w.first, w.items, p.run, p.items);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  if (!one_group(a, kTileRows)) {
    const int parts_of_blocks = (a.nb + 255) / 256;
    sparse_rank_kernel<<<(unsigned)(a.B * a.Hk) * parts_of_blocks, 256, 0, a.stream>>>(a, w, p.words, parts_of_blocks);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    sparse_rows_kernel<<<(unsigned)(a.B * a.H) * p.tiles, 128, 0, a.stream>>>(a, w, p.words, p.tiles, p.run, p.items);
    if ((err = hipGetLastError()) != hipSuccess) return err;
  }
  if ((err = launch_sparse_dkdv(a, w, p)) != hipSuccess) return err;
  if (p.items > a.nb) {
    sparse_share_kernel<<<dim3((unsigned)(a.B * a.Hk) * a.nb, (2 * a.block * a.d + 1023) / 1024), 256, 0, a.stream>>>(a, w, p.items);
    if ((err = hipGetLastError()) != hipSuccess) return err;
  }
  return launch_sparse_dq(a, w);
}

}  // namespace vitattn
