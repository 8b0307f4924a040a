// What the kernels of the decode steps share: reductions, partial results, who takes which key range (not part of the ABI).
#pragma once

#include "wkv_device.h"

namespace wkv {

// Sum over the LPK (8, 16 or 32) adjacent lanes that hold one row; every lane gets the total.
template <int LPK>
__device__ __forceinline__ float row_lanes_sum(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false));  // quad_perm [1,0,3,2]
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false));  // quad_perm [2,3,0,1]
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false)); // row_half_mirror
  if (LPK >= 16)
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x140, 0xF, 0xF, false)); // row_mirror
  if (LPK >= 32) x += __shfl_xor(x, 16);
  return x;
}

__device__ __forceinline__ float row_lanes_max8(float x) {
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false)));  // quad_perm [1,0,3,2]
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false)));  // quad_perm [2,3,0,1]
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false)));      // row_half_mirror
}

// Sum and maximum over the wave, in every lane: DPP steps inside rows of 16 lanes, then two permlane swaps.
__device__ __forceinline__ float wave_sum(float x) { return quads_sum(row16_sum(x)); }
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false)));  // quad_perm [1,0,3,2]
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false)));  // quad_perm [2,3,0,1]
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false))); // row_half_mirror
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x140, 0xF, 0xF, false))); // row_mirror
  return quads_max(x);
}

// Partial results in the workspace: the outputs [B*Hkv][splits][G][D] of every key range (only of ranges that
// hold rows), then their (m, l) [B*Hkv][splits][G].  A range past the end of a row has m = -inf; m of range 0
// is NaN where the cache cannot take the new row.
// (Byte offsets fit 32 bits: at most 65535 heads of one range each, or 1536 ranges, times eight query heads of 130 floats.  A launch runs
// through its code once, at some 7 cycles an instruction, and products of 64 bits are a dozen of them.)
__device__ __forceinline__ uint32_t part_index(const DecodeShape &s, int bh, int split, int g) {
  return ((uint32_t)bh * s.n_splits + split) * s.G + g;
}
__device__ __forceinline__ float2 &part_stats(const DecodeShape &s, float *part, uint32_t at) {
  return *(float2 *)((char *)part + (s.stats_at + at * 8u));
}
__device__ __forceinline__ const float2 &part_stats(const DecodeShape &s, const float *part, uint32_t at) {
  return *(const float2 *)((const char *)part + (s.stats_at + at * 8u));
}

// Which range of which cache this workgroup takes, and the rows of that cache.  It looks at the count of its own cache alone: a caller may
// write the counts of other sequences meanwhile (a slot of the batch that is being filled anew).  Ranges dealt out by all counts, whole ones first,
// would leave ranges of the others to nobody when a count changes between the start of two workgroups; they took, us a layer, own count / all: mixed
// batches of 32q/8kv heads, 8 up to 8000 rows 27.6 / 26.5, 24 up to 4000 45.1 / 38.4, 64 up to 2000 59.5 / 55.1; 64 of 4128 167.5 / 168.3, 16 48.7 / 49.4.
struct KeyRange {
  int head, range, n;
  __device__ __forceinline__ KeyRange(const DecodeShape &s, const int32_t *__restrict__ n_valid) {
    const RangeOf it(blockIdx.x, blockIdx.y, s.B * s.Hkv, s.heads_magic);
    head = it.head; range = it.range; n = load_scalar(n_valid + head);
  }
};

}  // namespace wkv
