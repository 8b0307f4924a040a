// What the attention kernels share: key and value tiles that reach LDS by DMA, the reference of a row's softmax (not part of the ABI).
#pragma once

#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// KEYS_: keys of a tile.
template <int D_, int DT, int WAVES_, int KEYS_ = att_tile_keys(DT == DT_F32)>
struct Att {
  static constexpr int D = D_, ES = DT == DT_F32 ? 4 : 2;
  static constexpr int WAVES = WAVES_, NT = WAVES * 64;
  static constexpr int KEYS = KEYS_;
  static constexpr int KT = KEYS / 32;
  static constexpr int ROWB = D * ES, PPR = ROWB / 16;      // bytes and 16-byte pieces of a row
  static constexpr int KS = PPR / 2;                      // contraction steps over the channels, two pieces each
  static constexpr int VT = D / 32;                       // channel tiles of the output
  static constexpr int TILE = KEYS * ROWB, STAGE = 2 * TILE, STAGES = 2;
  static constexpr int RPI = 64 / PPR;                    // rows of a DMA instruction
  static constexpr int LPT = TILE / 1024 / WAVES;         // DMA instructions of a wave per tile of keys (of values)
  static constexpr int OFFS = 16 / (RPI * WAVES) > 1 ? 16 / (RPI * WAVES) : 1;      // of them with key offsets of their own
  // Where piece p of row r lies within its row's slot.  Keys are read by 32 lanes of as many rows, a piece each: rows 16 apart share a
  // place.  Values: 16-bit types by four rows of 64 bytes at a time, fp32 by two rows, four apart, of 128 bytes.
  static __device__ __forceinline__ int key_slot(int r, int p) { return p ^ (PPR == 8 ? (r >> 1) & 7 : r & 15); }
  static __device__ __forceinline__ int value_slot(int r, int p) {
    return p ^ (ES == 4 ? (r >> 2 & 1) * 8 : PPR == 8 ? (r >> 1 & 1) * 4 : (r & 3) * 4);
  }
};

// A DMA instruction of a wave, from base + off bytes of each lane.  STREAM: past the memory-side cache.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool STREAM = false>
__device__ __forceinline__ void dma_rows(uint32_t lds, const char *base, uint32_t off) {
  if constexpr (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Two floats as a pair of 16-bit numbers, each rounded to nearest.
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  if constexpr (DT == DT_F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (h2){(_Float16)a, (_Float16)b});
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (b2){(__bf16)a, (__bf16)b});
  }
}

// A row's reference moves when a logit exceeds it by LIFT + GROW (base 2), to LIFT below that logit: the largest probability of a row is 2^LIFT to 2^(LIFT + GROW).
// For the product with the values 16-bit types round a probability to their own type, by half a step (the prompt attention; trees hold what that leaves in a second number): an fp32
// product takes eight times as long.  (Their sum, which the normaliser needs in fp32, is of the unrounded ones.)  fp16 has all its bits from 2^-14 to 2^16 alone and nothing below 2^-25, so its probabilities are held high: what
// it loses of a key is at most 2^-38 of the row's sum, and of 8192 keys, with values up to 1, no more than the rounding of an output in fp16 does.  Unlifted, a key of value zero that
// stands 17 (base e) above 4096 others left a third of the output wrong.  GROW of 0 / 1 / 2 / 4 / 8, the packed prompts of 17.4K tokens
// in fp16: 940 / 924 / 914 / 905 / 905 us.
template <int DT> struct Reference { static constexpr float LIFT = DT == DT_F16 ? 13.0f : 0.0f, GROW = DT == DT_F16 ? 2.0f : 8.0f; };

}  // namespace wkv
