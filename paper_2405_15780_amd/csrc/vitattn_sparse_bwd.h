// What the kernels of the sparse attention's backward share.
#pragma once

#include "vitattn_sparse.h"

namespace vitattn {

constexpr int kTileRows = 64;   // of a query tile
constexpr int kMapTiles = 64;   // query tiles of a map word
constexpr int kStat = 64;       // floats per 32 queries: -D, then LSE log2(e)

struct SparsePlan {  // sizes of the backward's workspace
  int tiles, words;   // query tiles of a head, map words of a key block
  int run;            // query tiles of an item
  long long items;    // items of a key head, at most
};
inline SparsePlan plan_of(const SparseArgs& a) {
  SparsePlan p;
  p.tiles = (a.Nq + kTileRows - 1) / kTileRows;
  p.words = (p.tiles + kMapTiles - 1) / kMapTiles;
  // blocks that a tile's rows can choose
  const long long groups = a.q_block >= kTileRows ? (a.q_block % kTileRows == 0 ? 1 : 2)
                                                  : min((long long)kTileRows / a.q_block + 2, (long long)min(a.Nq, kTileRows));
  const long long pairs = (long long)(a.H / a.Hk) * p.tiles * min(groups * a.topk, (long long)a.nb);
  // Runs of 64 tiles, of 32 where there are few blocks to fill the card with (126 blocks of
  // 4 key heads: dK/dV and shares 98 us with 32, 105 with 64, 118 with 128; 512 blocks of 8:
  // 399, 396, 442), and longer ones where the shares of as many items would outgrow eight
  // times the keys.
  p.run = (int)max(a.nb < 256 ? 32LL : 64LL, min(4096LL, (pairs + 8LL * a.nb - 1) / (8LL * a.nb)));
  p.items = a.nb + pairs / p.run;  // sum over the blocks of max(1, ceil(count / run))
  return p;
}

// workspace
struct SparseWork {
  float* stats;      // [BH][32-query blocks][kStat]
  uint64_t* map;     // [BH][words][nb]
  int* counts;       // [B Hk][nb]
  int* first;        // [B Hk][nb + 1]: a block's first item; the number of items
  int4* items;       // [B Hk][items]: an item's block, its run, the block's runs and query tiles
  // where a query tile's rows choose apart (not one_group(a, 64)):
  int* ranks;        // [BH][words][nb]: tiles that chose the block before the word's, of all heads that share keys
  uint64_t* rows;    // [B Hk][items][run]: of an item's query tiles, the rows that chose the block
  int* tiles;        // [B Hk][items][run]: and which they are, head of the group << 20 | tile
  float* shares;     // [B Hk][items][2][block][d]
  size_t bytes;
};
inline size_t padded(size_t n) { return (n + 255) / 256 * 256; }
inline SparseWork work_of(const SparseArgs& a, const SparsePlan& p) {
  SparseWork w;
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
  const size_t apart = one_group(a, kTileRows) ? 0 : 1, slots = apart * bhk * p.items * p.run;
  w.ranks = reinterpret_cast<int*>(take(apart * bh * p.words * a.nb * 4));
  w.rows = reinterpret_cast<uint64_t*>(take(slots * 8));
  w.tiles = reinterpret_cast<int*>(take(slots * 4));
  w.shares = reinterpret_cast<float*>(take(p.items > a.nb ? bhk * p.items * 2 * a.block * a.d * 4 : 0));
  w.bytes = n;
  return w;
}


hipError_t launch_sparse_dkdv(const SparseArgs& a, const SparseWork& w, const SparsePlan& p);
hipError_t launch_sparse_dq(const SparseArgs& a, const SparseWork& w);

}  // namespace vitattn
