// Attention over a prompt: softmax(q K^T scale) V, causal, for blocks of rows of one KV head.
//
// One pass over the keys with a running reference and sum of the softmax (both fp32).  Everything is computed transposed, so that
// a lane of the 32x32 results belongs to one row of the softmax:
//   S^T = K Q^T    keys the A operand, 32 query rows the B operand: lane l holds row l % 32 and 16 of 32 keys, the statistics of a
//                  row are sums within a lane and over its two halves
//   O^T = V^T P^T  the probabilities as they lie in the lanes are the B operand already, if the contraction takes the keys in the order in
//                  which a lane holds them; the values are read to match (16 bits: transposed, ds_read_tr; four keys of a channel)
// The rows of a block are (query, head of the group) pairs, query-major: the G heads that share a KV head share its tiles.
//
// Long prompts are bound by the matrix pipe at the clock that power leaves it: 32768 tokens of 32q/8kv heads with 128 channels in bf16 take 7.4 to 8.0 ms from chip to chip =
// 1100-1190 TFLOP/s (a library product of 8192^3 1202-1275; the same call on zeros 5.8 ms): by the counters 56 % of the matrix cycles at 1.9 to 2.0 GHz.  Short ones are bound by a
// wave's chain of products, statistics and products, 1.2 us a tile.  Eight waves of 32 rows, all at the same tile, fetch it once: 7.67 ms, by workgroups of four
// 7.84 (4096 tokens 133 and 146 us).  No better: 64 rows a wave with a SIMD for itself, so that a fragment from LDS feeds two products (9.07; with the next tile's
// logits computed beside this one's exponentials the registers do not suffice); a reference that moves when a tile's sum overflows, without
// maxima (+2 %); 128 keys to a barrier (+4 %); three or four tiles in LDS (+1 %); wave priorities (the same).
#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <int D_, int DT, int WAVES_>
struct Att {
  static constexpr int D = D_, ES = DT == DT_F32 ? 4 : 2;
  static constexpr int WAVES = WAVES_, NT = WAVES * 64;
  static constexpr int KEYS = att_tile_keys(DT == DT_F32);      // of a tile
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

// A DMA instruction of a wave, from base + off bytes of each lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma_rows(uint32_t lds, const char *base, uint32_t off) {
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

// Which block of which (sequence, KV head) work item `item` is, and what follows for the keys.
template <int ROWS>
struct Block {
  AttentionSeq sq;
  int h, block, past, n_rows, n_tiles, n_splits;
  const AttentionArgs &a;
  __device__ __forceinline__ Block(const AttentionArgs &args, int item, int tile_keys) : a(args) {
    const int lane = threadIdx.x & 63;
    const int end = lane < a.n_seqs ? a.ends[lane] : 0x7fffffff;
    const int seg = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__ballot(item >= end)));
    const int rel = item - (seg ? a.ends[seg - 1] : 0);
    const int level_items = (seg + 1) * a.Hkv;
    const int level = (int)((uint32_t)rel / (uint32_t)level_items), at = rel - level * level_items;
    const int si = (int)((uint32_t)at / (uint32_t)a.Hkv);
    h = at - si * a.Hkv;
    sq = a.seq[si];
    block = a.seq[seg].blocks - 1 - level;
    past = sq.k_len - sq.q_len;
    n_rows = sq.q_len * a.G;
    n_tiles = n_rows ? (sees(min((block + 1) * ROWS, n_rows) - 1) + tile_keys - 1) / tile_keys : 0;
    n_splits = a.splits == 1 ? 1 : max((n_tiles + a.chunk - 1) / a.chunk, 1);
  }
  __device__ __forceinline__ int query(int r) const { return divide((uint32_t)r, a.g_magic); }
  __device__ __forceinline__ int sees(int r) const { return min(max(query(r) + past + 1, 0), sq.k_len); }      // keys that row r sees
};

// Natural logarithm of a row's sum, from its base-2 reference; no key weighs anything: -inf.
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.0f ? -INFINITY : (m + fast_log2(l)) * 0.69314718055994531f; }

// A row's reference moves when a logit exceeds it by LIFT + GROW (base 2), to LIFT below that logit: the largest probability of a row is 2^LIFT to 2^(LIFT + GROW).
// For the product with the values 16-bit types round a probability to their own type, by half a step: an fp32 product takes eight times as long.  (Their sum, which the
// normaliser needs in fp32, is of the unrounded ones.)  fp16 has all its bits from 2^-14 to 2^16 alone and nothing below 2^-25, so its probabilities are held high: what
// it loses of a key is at most 2^-38 of the row's sum, and of 8192 keys, with values up to 1, no more than the rounding of an output in fp16 does.  Unlifted, a key of value zero that
// stands 17 (base e) above 4096 others left a third of the output wrong.  GROW of 0 / 1 / 2 / 4 / 8, the packed prompts of 17.4K tokens
// in fp16: 940 / 924 / 914 / 905 / 905 us.
template <int DT> struct Reference { static constexpr float LIFT = DT == DT_F16 ? 13.0f : 0.0f, GROW = DT == DT_F16 ? 2.0f : 8.0f; };

// -inf for the normalisers of rows that do not exist, by the workgroup of the first block.
template <int ROWS>
__device__ __forceinline__ void missing_normalisers(const Block<ROWS> &it, float *__restrict__ lse) {
  const AttentionArgs &a = it.a;
  for (int i = threadIdx.x; i < (a.lse_rows - it.sq.q_len) * a.G; i += blockDim.x) {
    const int r = i / a.G, g = i - r * a.G;
    lse[((int64_t)it.sq.b * a.Hq + it.h * a.G + g) * a.lse_rows + r] = -INFINITY;
  }
}

// The results of a wave's 32 rows, from row `first` of the block on: normalised, or as they are for join_kernel.
template <int D, int DT, int ROWS>
__device__ __forceinline__ void write_rows(const Block<ROWS> &it, int part_of, int first, int seen, const f32x16 (&o)[D / 32], float m, float l,
                                           char *__restrict__ out, float *__restrict__ lse, float *__restrict__ part, float2 *__restrict__ stats) {
  const AttentionArgs &a = it.a;
  const int lane = threadIdx.x & 63, half = lane >> 5, in_block = first + (lane & 31), row = it.block * ROWS + in_block;
  l = add_halves(l, l);
  if (it.n_splits > 1) {
    const int64_t at = (int64_t)part_of * ROWS + in_block;
    if (row < it.n_rows && half == 0) stats[at] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (row < it.n_rows) *(float4 *)(part + at * D + i * 32 + e * 2 + half * 4) = make_float4(o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]);
    return;
  }
  const int qi = it.query(min(row, it.n_rows - 1)), g = min(row, it.n_rows - 1) - qi * a.G, lse_first = it.sq.q_len - a.lse_rows;
  if (row < it.n_rows && half == 0 && qi >= lse_first) lse[((int64_t)it.sq.b * a.Hq + it.h * a.G + g) * a.lse_rows + (qi - lse_first)] = row_lse(m, l);
  const float inv = seen > 0 ? 1.0f / l : 0.0f;
  char *op = out + (it.sq.b * a.o_sb + (int64_t)(it.h * a.G + g) * a.o_sh + (it.sq.q_start + qi) * a.o_st);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const f32x16 &x = o[i];
    if constexpr (DT == DT_F32) {
#pragma unroll
      for (int e = 0; e < 16; e += 4)       // channels i * 32 + e * 2 + half * 4 ..
        if (row < it.n_rows) *(float4 *)(op + (i * 32 + e * 2 + half * 4) * 4) = make_float4(x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += 8) {     // the halves exchange four channels each: 16 bytes of a row to a lane
        const auto y0 = __builtin_amdgcn_permlane32_swap(pack_pair<DT>(x[e] * inv, x[e + 1] * inv), pack_pair<DT>(x[e + 4] * inv, x[e + 5] * inv), false, false);
        const auto y1 = __builtin_amdgcn_permlane32_swap(pack_pair<DT>(x[e + 2] * inv, x[e + 3] * inv), pack_pair<DT>(x[e + 6] * inv, x[e + 7] * inv), false, false);
        if (row < it.n_rows) *(uint4 *)(op + (i * 32 + e * 2 + half * 8) * 2) = make_uint4(y0[0], y1[0], y0[1], y1[1]);
      }
    }
  }
}

// Which item a workgroup takes.  Longest first; but where two start on a compute unit at once, the second ones the other way round (whole turns over
// the XCDs at a time), so that a unit's two take as long as another's: the second half of 257 to 512 blocks of 128 rows, and the second, fourth, ..
// parts of blocks that are cut (2048 tokens of 32q/8kv heads in fp32 372 -> 280 us).
__device__ __forceinline__ int item_of(const AttentionArgs &a) {
  const int x = blockIdx.x, from = blockIdx.y & 1 ? a.fold_parts : a.fold_from;
  return x < from ? x : ((gridDim.x - 1 - x + from) & ~7) | (x & 7);
}

// A wave takes 32 rows, a workgroup 32 * WAVES.
template <int D, int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void prefill_kernel(AttentionArgs a, const char *__restrict__ q, const char *__restrict__ k,
                                                                const char *__restrict__ v, char *__restrict__ out, float *__restrict__ lse,
                                                                float *__restrict__ part, float2 *__restrict__ stats) {
  using C = Att<D, DT, WAVES>;
  constexpr int KS = C::KS, KT = C::KT, VT = C::VT, ROWS = WAVES * 32;
  __shared__ __attribute__((aligned(1024))) char ring[C::STAGES * C::STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;

  // ---- which block of which KV head, and which of its key tiles
  const int item = item_of(a);
  const Block<ROWS> it(a, item, C::KEYS);
  const AttentionSeq &sq = it.sq;
  const int h = it.h, k_len = sq.k_len, n_rows = it.n_rows, split = blockIdx.y;
  if (split >= it.n_splits) return;
  if (it.block == 0 && split == 0) missing_normalisers(it, lse);
  if (n_rows == 0) return;
  const int t_begin = split ? split * a.chunk : 0, t_end = it.n_splits == 1 ? it.n_tiles : min(t_begin + a.chunk, it.n_tiles);

  // ---- this lane's row
  const int wave_row = it.block * ROWS + wave * 32, row = min(wave_row + col, n_rows - 1);
  const int qi = it.query(row), g = row - qi * a.G;
  const int seen = it.sees(row), wave_least = it.sees(min(wave_row, n_rows - 1));
  const int wave_most = wave_row < n_rows ? it.sees(min(wave_row + 31, n_rows - 1)) : 0;

  // ---- the key and value stream
  const char *kb = k + (sq.b * a.kv_sb + h * a.kv_sh + sq.k_start * a.kv_st);
  const char *vb = v + (sq.b * a.kv_sb + h * a.kv_sh + sq.k_start * a.kv_st);
  const uint32_t st = (uint32_t)a.kv_st;
  const int my_row = wave * C::RPI + lane / C::PPR, my_piece = lane % C::PPR;      // of this lane's first DMA instruction
  uint32_t k_off[C::OFFS];
#pragma unroll
  for (int i = 0; i < C::OFFS; ++i) k_off[i] = my_row * st + C::key_slot(my_row + i * C::RPI * WAVES, my_piece) * 16;
  const uint32_t v_off = my_row * st + C::value_slot(my_row, my_piece) * 16;
  const uint32_t ring_at = lds_address(ring) + wave * 1024;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    const uint32_t dst = ring_at + (t % C::STAGES) * C::STAGE;
    const int j0 = t * C::KEYS;
    if (j0 + C::KEYS <= k_len) {
#pragma unroll
      for (int i = 0; i < C::LPT; ++i)
        dma_rows(dst + i * (WAVES * 1024), kb + (int64_t)(j0 + i * (C::RPI * WAVES)) * a.kv_st, k_off[i % C::OFFS]);
#pragma unroll
      for (int i = 0; i < C::LPT; ++i)
        dma_rows(dst + C::TILE + i * (WAVES * 1024), vb + (int64_t)(j0 + i * (C::RPI * WAVES)) * a.kv_st, v_off);
    } else {                              // rows past the sequence: its last one again
#pragma unroll
      for (int i = 0; i < C::LPT; ++i) {
        const int64_t r = min(j0 + i * (C::RPI * WAVES) + my_row, k_len - 1);
        dma_to_lds(dst + i * (WAVES * 1024), kb + r * a.kv_st + (k_off[i % C::OFFS] - my_row * st));
        dma_to_lds(dst + C::TILE + i * (WAVES * 1024), vb + r * a.kv_st + (v_off - my_row * st));
      }
    }
  };
  if (t_begin < t_end) fetch(t_begin);

  // ---- queries: B fragments
  bf16x8 qf[KS];
  {
    const char *qp = q + (sq.b * a.q_sb + (int64_t)(h * a.G + g) * a.q_sh + (sq.q_start + qi) * a.q_st) + half * 16;
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[i] = *(const bf16x8 *)(qp + i * 32);
    // (waited for here, once: left to itself the compiler waits for them in every turn of the loop, behind the next tile's requests)
#pragma unroll
    for (int i = 0; i < KS; ++i) asm volatile("" : "+v"(qf[i]));
  }

  f32x16 o[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;           // reference and this lane's part of the sum, base 2

  auto attend = [&](const char *ks, const char *vs, int j0) __attribute__((always_inline)) {
    // S^T
    f32x16 s[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.0f;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const bf16x8 kf = *(const bf16x8 *)(ks + (kt * 32 + col) * C::ROWB + C::key_slot(col, 2 * i + half) * 16);
        if constexpr (DT == DT_F32) {
          const f32x4 x = __builtin_bit_cast(f32x4, kf), y = __builtin_bit_cast(f32x4, qf[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[kt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], s[kt], 0, 0, 0);
        } else {
          s[kt] = mfma_step<DT, 32>(kf, qf[i], s[kt]);
        }
      }
    }
    // element e of a lane is key kt * 32 + e / 4 * 8 + half * 4 + e % 4
    if (j0 + C::KEYS > wave_least) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + kt * 32 + e / 4 * 8 + half * 4 + e % 4 >= seen) s[kt][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kt][e]);
    {
      const Pair p = swap_halves(top, top);
      top = fmaf(fmaxf(p.a, p.b), a.c1, -Reference<DT>::LIFT);
    }
    // The reference moves only when a row's logits outgrow it, which a few tiles of a long row do.
    if (__any(top > m + Reference<DT>::GROW)) {
      const float to = fmaxf(m, top), corr = to == -INFINITY ? 1.0f : fast_exp2(m - to);
      m = to;
      l *= corr;
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= corr;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kt][e] = fast_exp2(fmaf(s[kt][e], a.c1, -ref));
        l += s[kt][e];
      }

    // O^T
    if constexpr (DT == DT_F32) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = kt * 32 + e / 4 * 8 + e % 4 + half * 4;
#pragma unroll
          for (int i = 0; i < VT; ++i) {
            const int c = i * 32 + col;
            const float x = *(const float *)(vs + key * C::ROWB + C::value_slot(half * 4, c / 4) * 16 + c % 4 * 4);
            o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[kt][e], o[i], 0, 0, 0);
          }
        }
    } else {
      const int tl = lane & 15, at = lane >> 4 & 1, y = half * 4 + tl / 4;      // transposed reads: 16 lanes take four rows of 16 channels
#pragma unroll
      for (int x = 0; x < KT * 2; ++x) {
        const f32x16 &p = s[x / 2];
        const int e = x % 2 * 8;
        const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pack_pair<DT>(p[e], p[e + 1]), pack_pair<DT>(p[e + 2], p[e + 3]),
                                                                pack_pair<DT>(p[e + 4], p[e + 5]), pack_pair<DT>(p[e + 6], p[e + 7])));
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const char *vp = vs + (x * 16 + y) * C::ROWB + C::value_slot(y, i * 4 + at * 2 + tl % 4 / 2) * 16 + tl % 2 * 8;
          typedef __attribute__((address_space(3))) s16x4 lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)vp);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)(vp + 8 * C::ROWB));
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          o[i] = mfma_step<DT, 32>(vf, pf, o[i]);
        }
      }
    }
  };

  for (int t = t_begin; t < t_end; ++t) {
    // the tile is in LDS (each wave waits for its own requests, the barrier for all), and everyone is done with the place of the next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < t_end) fetch(t + 1);
    const char *ks = ring + (t % C::STAGES) * C::STAGE;
    if (t * C::KEYS < wave_most) attend(ks, ks + C::TILE, t * C::KEYS);
  }
  write_rows<D, DT, ROWS>(it, item * a.splits + split, wave * 32, seen, o, m, l, out, lse, part, stats);
}

// The rows of blocks that several workgroups shared: D / 4 threads take four channels each, of every GROUPS-th partial result.
constexpr int JOIN_THREADS = 256;
template <int D, int DT, int ROWS, int GROUPS>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(AttentionArgs a, const float *__restrict__ part, const float2 *__restrict__ stats,
                                                            char *__restrict__ out, float *__restrict__ lse) {
  constexpr int COLS = D / 4, AHEAD = 4, SLOTS = JOIN_THREADS / COLS, AT_ONCE = SLOTS / GROUPS, ES = DT == DT_F32 ? 4 : 2;
  __shared__ float4 o_s[GROUPS > 1 ? SLOTS : 1][COLS];
  __shared__ float2 ml_s[GROUPS > 1 ? SLOTS : 1];
  const Block<ROWS> it(a, blockIdx.x, att_tile_keys(DT == DT_F32));
  const int slot = threadIdx.x / COLS, col = threadIdx.x % COLS, group = slot % GROUPS;
  const int r = blockIdx.y * AT_ONCE + slot / GROUPS, row = it.block * ROWS + r;
  if (it.n_splits == 1) return;
  const bool exists = row < it.n_rows;
  const int64_t at = (int64_t)blockIdx.x * a.splits * ROWS + r;
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto merge = [&](const float2 (&ml)[AHEAD], const float4 (&x)[AHEAD]) __attribute__((always_inline)) {
    float to = m;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) to = fmaxf(to, ml[u].x);
    const float ref = to == -INFINITY ? 0.0f : to, old = fast_exp2(m - ref);
    m = to;
    l *= old; o.x *= old; o.y *= old; o.z *= old; o.w *= old;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float w = fast_exp2(ml[u].x - ref);
      l = fmaf(ml[u].y, w, l);
      o.x = fmaf(x[u].x, w, o.x); o.y = fmaf(x[u].y, w, o.y); o.z = fmaf(x[u].z, w, o.z); o.w = fmaf(x[u].w, w, o.w);
    }
  };
  for (int s0 = group; exists && s0 < it.n_splits; s0 += AHEAD * GROUPS) {
    float2 ml[AHEAD];
    float4 x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      ml[u] = make_float2(-INFINITY, 0.0f);
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s0 + u * GROUPS < it.n_splits) {
        const int64_t from = at + (int64_t)(s0 + u * GROUPS) * ROWS;
        ml[u] = stats[from];
        x[u] = *(const float4 *)(part + from * D + col * 4);
      }
    }
    merge(ml, x);
  }
  if constexpr (GROUPS > 1) {
    o_s[slot][col] = o;
    if (col == 0) ml_s[slot] = make_float2(m, l);
    __syncthreads();
    if (group != 0) return;
    m = -INFINITY; l = 0.0f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
    static_assert(GROUPS % AHEAD == 0, "the groups of a row, AHEAD at a time");
#pragma unroll
    for (int g0 = 0; g0 < GROUPS; g0 += AHEAD) {
      float2 ml[AHEAD];
      float4 x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) { ml[u] = ml_s[slot + g0 + u]; x[u] = o_s[slot + g0 + u][col]; }
      merge(ml, x);
    }
  }
  if (!exists) return;
  const int qi = it.query(row), g = row - qi * a.G, first = it.sq.q_len - a.lse_rows;
  if (col == 0 && qi >= first) lse[((int64_t)it.sq.b * a.Hq + it.h * a.G + g) * a.lse_rows + (qi - first)] = row_lse(m, l);
  const float inv = it.sees(row) > 0 ? 1.0f / l : 0.0f;
  char *op = out + (it.sq.b * a.o_sb + (int64_t)(it.h * a.G + g) * a.o_sh + (it.sq.q_start + qi) * a.o_st + col * 4 * ES);
  if constexpr (DT == DT_F32) *(float4 *)op = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else *(uint2 *)op = make_uint2(pack_pair<DT>(o.x * inv, o.y * inv), pack_pair<DT>(o.z * inv, o.w * inv));
}

template <int D, int DT, int ROWS>
hipError_t launch_blocks(const AttentionPlan &plan, const void *q, const void *k, const void *v, void *out, float *lse, void *ws, hipStream_t stream) {
  const AttentionArgs &a = plan.args;
  float *part = (float *)ws;
  float2 *stats = (float2 *)((char *)ws + plan.stats_at);
  hipLaunchKernelGGL((prefill_kernel<D, DT, ROWS / 32>), dim3((uint32_t)plan.items, (uint32_t)a.splits), dim3(ROWS * 2), 0, stream, a, (const char *)q,
                     (const char *)k, (const char *)v, (char *)out, lse, part, stats);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  // one trip to memory up to 4 partial results, or 32 by eight groups of threads (one token over 32768, 64 of them: 33.2 us the call by one group, 28.1 so)
  constexpr int SLOTS = JOIN_THREADS / (D / 4);
#define WKV_JOIN(GROUPS) \
  hipLaunchKernelGGL((join_kernel<D, DT, ROWS, GROUPS>), dim3((uint32_t)plan.items, (uint32_t)((plan.most_rows + SLOTS / GROUPS - 1) / (SLOTS / GROUPS))), \
                     dim3(JOIN_THREADS), 0, stream, a, part, stats, (char *)out, lse)
  if (a.splits > 8) WKV_JOIN(8);
  else WKV_JOIN(1);
#undef WKV_JOIN
  return hipGetLastError();
}
template <int D, int DT>
hipError_t launch_d(const AttentionPlan &plan, const void *q, const void *k, const void *v, void *out, float *lse, void *ws, hipStream_t stream) {
  if constexpr (DT != DT_F32)
    if (plan.rows == ATT_ROWS) return launch_blocks<D, DT, ATT_ROWS>(plan, q, k, v, out, lse, ws, stream);
  return plan.rows == ATT_ROWS_FEW ? launch_blocks<D, DT, ATT_ROWS_FEW>(plan, q, k, v, out, lse, ws, stream) : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_attention(const AttentionPlan &plan, const void *q, const void *k, const void *v, void *out, float *lse, void *ws, hipStream_t stream) {
#define WKV_ATT_TYPE(DT) return plan.args.d == 128 ? launch_d<128, DT>(plan, q, k, v, out, lse, ws, stream) : launch_d<64, DT>(plan, q, k, v, out, lse, ws, stream)
  if (plan.args.dtype == WKV_BF16) WKV_ATT_TYPE(DT_BF16);
  if (plan.args.dtype == WKV_F16) WKV_ATT_TYPE(DT_F16);
  WKV_ATT_TYPE(DT_F32);
#undef WKV_ATT_TYPE
}

}  // namespace wkv
