// Device helpers of the differential attention kernels.
#pragma once

#include "vitattn_common.h"
#include "vitattn_launch.h"

namespace vitattn {

__device__ __forceinline__ float lam_of(const void* lam, bool bf16, int h) {
  return bf16 ? (float)static_cast<const __bf16*>(lam)[h] : static_cast<const float*>(lam)[h];
}
// keys of sample b: the first key_lens[b] of Nk, brought into 0 .. Nk
__device__ __forceinline__ int keys_of(const int* key_lens, int b, int Nk) {
  return key_lens ? min(max(key_lens[b], 0), Nk) : Nk;
}
// This workgroup's work item: each XCD takes a run of consecutive ones, which
// share keys in its L2, unless samples differ in length. Then the runs would too
// (a padded batch's short samples on some XCDs), and items go to the XCDs in turn.
__device__ __forceinline__ int work_item(const int* key_lens, int total) {
  return key_lens ? (int)blockIdx.x : xcd_remap(blockIdx.x, total);
}
// head of map m of (b, h) in a tensor of 2 H heads
__device__ __forceinline__ long long map_head(const Map& m, int b, int h, int map) {
  return b * m.sb + (2LL * h + map) * m.sh;
}
// four consecutive outputs rounded to bf16
__device__ __forceinline__ void put4_bf16(uint16_t* p, float a, float b, float c, float d) {
  const bf16x2 lo = {(__bf16)a, (__bf16)b}, hi = {(__bf16)c, (__bf16)d};
  *reinterpret_cast<uint2*>(p) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// Tile widths: of q and k, contracted over their QS 16-column steps that may
// hold data, and of v. Head dims past them are refused.
struct DiffTile {
  int dq, qs, dv;
};
inline DiffTile diff_tile(int d, int e) {
  if (d <= 32 && e <= 64) return {32, 2, 64};
  if (d <= 64 && e <= 64) return {64, 4, 64};
  if (d <= 64 && e <= 128) return {64, 4, 128};
  return {96, 5, 160};
}

}  // namespace vitattn
