// Attention over a prompt: softmax(q K^T scale) V, causal, for blocks of rows of one KV head.
//
// One pass over the keys with a running reference and sum of the softmax (both fp32).  Everything is computed transposed, so that
// a lane of the 32x32 results belongs to one row of the softmax:
//   S^T = K Q^T    keys the A operand, 32 query rows the B operand: lane l holds row l % 32 and 16 of 32 keys, the statistics of a
//                  row are sums within a lane and over its two halves
//   O^T = V^T P^T  the probabilities as they lie in the lanes are the B operand already, if the contraction takes the keys in the order in
//                  which a lane holds them; the values are read to match (16 bits: transposed, ds_read_tr; four keys of a channel)
// The rows of a block are (query, head of the group) pairs, query-major: the G heads that share a KV head share its tiles.
#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <int D_, int DT>
struct Att {
  static constexpr int D = D_, ES = DT == DT_F32 ? 4 : 2;
  static constexpr int WAVES = 4, NT = WAVES * 64;
  static constexpr int KEYS = DT == DT_F32 ? 32 : 64;     // of a tile
  static constexpr int KT = KEYS / 32;
  static constexpr int ROWB = D * ES, PPR = ROWB / 16;      // bytes and 16-byte pieces of a row
  static constexpr int KS = PPR / 2;                      // contraction steps over the channels, two pieces each
  static constexpr int VT = D / 32;                       // channel tiles of the output
  static constexpr int TILE = KEYS * ROWB, STAGE = 2 * TILE, STAGES = 2;
  static constexpr int RPI = 64 / PPR;                    // rows of a DMA instruction
  static constexpr int LPT = TILE / 1024 / WAVES;         // DMA instructions of a wave per tile of keys (of values)
  static constexpr int OFFS = 16 / (RPI * WAVES) > 1 ? 16 / (RPI * WAVES) : 1;      // of them with key offsets of their own
  static_assert(WAVES * 32 == ATT_ROWS, "a block of rows");
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
    n_tiles = n_rows ? (sees(min((block + 1) * ATT_ROWS, n_rows) - 1) + tile_keys - 1) / tile_keys : 0;
    n_splits = a.splits == 1 ? 1 : max((n_tiles + a.chunk - 1) / a.chunk, 1);
  }
  __device__ __forceinline__ int query(int r) const { return divide((uint32_t)r, a.g_magic); }
  __device__ __forceinline__ int sees(int r) const { return min(max(query(r) + past + 1, 0), sq.k_len); }      // keys that row r sees
};

// Natural logarithm of a row's sum, from its base-2 reference; no key weighs anything: -inf.
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.0f ? -INFINITY : (m + fast_log2(l)) * 0.69314718055994531f; }

constexpr float ATT_GROW = 8.0f;      // a row's reference moves when a logit exceeds it by this (base 2): probabilities up to 2^8

template <int D, int DT>
__global__ __launch_bounds__(256, 2) void prefill_kernel(AttentionArgs a, const char *__restrict__ q, const char *__restrict__ k,
                                                         const char *__restrict__ v, char *__restrict__ out, float *__restrict__ lse,
                                                         float *__restrict__ part, float2 *__restrict__ stats) {
  using C = Att<D, DT>;
  constexpr int KS = C::KS, KT = C::KT, VT = C::VT;
  __shared__ __attribute__((aligned(1024))) char ring[C::STAGES * C::STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;

  // ---- which block of which KV head, and which of its key tiles
  const Block it(a, blockIdx.x, C::KEYS);
  const AttentionSeq &sq = it.sq;
  const int h = it.h, block = it.block, q_len = sq.q_len, k_len = sq.k_len, n_rows = it.n_rows, split = blockIdx.y;
  if (split >= it.n_splits) return;
  if (block == 0 && split == 0)          // normalisers of rows that do not exist
    for (int i = threadIdx.x; i < (a.lse_rows - q_len) * a.G; i += C::NT) {
      const int r = i / a.G, g = i - r * a.G;
      lse[((int64_t)sq.b * a.Hq + h * a.G + g) * a.lse_rows + r] = -INFINITY;
    }
  if (n_rows == 0) return;
  const int t_begin = split ? split * a.chunk : 0, t_end = it.n_splits == 1 ? it.n_tiles : min(t_begin + a.chunk, it.n_tiles);

  // ---- this lane's row
  const int first_row = block * ATT_ROWS;
  const int row = min(first_row + wave * 32 + col, n_rows - 1);
  const int qi = it.query(row), g = row - qi * a.G;
  const int seen = it.sees(row), wave_least = it.sees(min(first_row + wave * 32, n_rows - 1));
  const int wave_most = first_row + wave * 32 < n_rows ? it.sees(min(first_row + wave * 32 + 31, n_rows - 1)) : 0;

  // ---- the key and value stream
  const char *kb = k + (sq.b * a.kv_sb + h * a.kv_sh + sq.k_start * a.kv_st);
  const char *vb = v + (sq.b * a.kv_sb + h * a.kv_sh + sq.k_start * a.kv_st);
  const uint32_t st = (uint32_t)a.kv_st;
  const int my_row = wave * C::RPI + lane / C::PPR, my_piece = lane % C::PPR;      // of this lane's first DMA instruction
  uint32_t k_off[C::OFFS];
#pragma unroll
  for (int i = 0; i < C::OFFS; ++i) k_off[i] = my_row * st + C::key_slot(my_row + i * C::RPI * C::WAVES, my_piece) * 16;
  const uint32_t v_off = my_row * st + C::value_slot(my_row, my_piece) * 16;
  const uint32_t ring_at = lds_address(ring) + wave * 1024;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    const uint32_t dst = ring_at + (t % C::STAGES) * C::STAGE;
    const int j0 = t * C::KEYS;
    if (j0 + C::KEYS <= k_len) {
#pragma unroll
      for (int i = 0; i < C::LPT; ++i)
        dma_rows(dst + i * (C::WAVES * 1024), kb + (int64_t)(j0 + i * (C::RPI * C::WAVES)) * a.kv_st, k_off[i % C::OFFS]);
#pragma unroll
      for (int i = 0; i < C::LPT; ++i)
        dma_rows(dst + C::TILE + i * (C::WAVES * 1024), vb + (int64_t)(j0 + i * (C::RPI * C::WAVES)) * a.kv_st, v_off);
    } else {                              // rows past the sequence: its last one again
#pragma unroll
      for (int i = 0; i < C::LPT; ++i) {
        const int64_t r = min(j0 + i * (C::RPI * C::WAVES) + my_row, k_len - 1);
        dma_to_lds(dst + i * (C::WAVES * 1024), kb + r * a.kv_st + (k_off[i % C::OFFS] - my_row * st));
        dma_to_lds(dst + C::TILE + i * (C::WAVES * 1024), vb + r * a.kv_st + (v_off - my_row * st));
      }
    }
  };
  if (t_begin < t_end) fetch(t_begin);

  // ---- queries: B fragments
  bf16x8 qf[KS];
  {
    const char *qp = q + (sq.b * a.q_sb + (int64_t)(h * a.G + g) * a.q_sh + (sq.q_start + qi) * a.q_st) + half * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const bf16x8 *)(qp + s * 32);
  }

  f32x16 o[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;           // reference and this lane's part of the sum, base 2

  for (int t = t_begin; t < t_end; ++t) {
    // the tile is in LDS (each wave waits for its own requests, the barrier for all), and everyone is done with the place of the next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < t_end) fetch(t + 1);
    const int j0 = t * C::KEYS;
    if (j0 >= wave_most) continue;
    const char *ks = ring + (t % C::STAGES) * C::STAGE, *vs = ks + C::TILE;

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
      top = fmaxf(p.a, p.b) * a.c1;
    }
    // The reference moves only when a row's logits outgrow it, which a few tiles of a long row do.
    if (__any(top > m + ATT_GROW)) {
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
      const int tl = lane & 15, part = lane >> 4 & 1;      // transposed reads: 16 lanes take four rows of 16 channels
#pragma unroll
      for (int x = 0; x < KT * 2; ++x) {
        uint4 pw;
        pw.x = pack_pair<DT>(s[x / 2][x % 2 * 8 + 0], s[x / 2][x % 2 * 8 + 1]);
        pw.y = pack_pair<DT>(s[x / 2][x % 2 * 8 + 2], s[x / 2][x % 2 * 8 + 3]);
        pw.z = pack_pair<DT>(s[x / 2][x % 2 * 8 + 4], s[x / 2][x % 2 * 8 + 5]);
        pw.w = pack_pair<DT>(s[x / 2][x % 2 * 8 + 6], s[x / 2][x % 2 * 8 + 7]);
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const int r = half * 4 + tl / 4;                 // row of the first four of each eight
          const char *vp = vs + (x * 16 + r) * C::ROWB + C::value_slot(r, i * 4 + part * 2 + tl % 4 / 2) * 16 + tl % 2 * 8;
          typedef __attribute__((address_space(3))) s16x4 lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)vp);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)(vp + 8 * C::ROWB));
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          o[i] = mfma_step<DT, 32>(vf, pf, o[i]);
        }
      }
    }
  }

  // ---- normalise and write
  l = add_halves(l, l);
  const bool exists = first_row + wave * 32 + col < n_rows;
  if (it.n_splits > 1) {                  // joined by join_kernel
    const int64_t r = ((int64_t)blockIdx.x * a.splits + split) * ATT_ROWS + wave * 32 + col;
    if (exists && half == 0) stats[r] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < VT; ++i)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (exists) *(float4 *)(part + r * D + i * 32 + e * 2 + half * 4) = make_float4(o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]);
    return;
  }
  if (exists && half == 0 && qi >= q_len - a.lse_rows)
    lse[((int64_t)sq.b * a.Hq + h * a.G + g) * a.lse_rows + (qi - (q_len - a.lse_rows))] =
        row_lse(m, l);
  const float inv = seen > 0 ? 1.0f / l : 0.0f;
  char *op = out + (sq.b * a.o_sb + (int64_t)(h * a.G + g) * a.o_sh + (sq.q_start + qi) * a.o_st);
#pragma unroll
  for (int i = 0; i < VT; ++i) {
    if constexpr (DT == DT_F32) {
#pragma unroll
      for (int e = 0; e < 16; e += 4)       // channels i * 32 + e * 2 + half * 4 ..
        if (exists) *(float4 *)(op + (i * 32 + e * 2 + half * 4) * 4) = make_float4(o[i][e] * inv, o[i][e + 1] * inv, o[i][e + 2] * inv, o[i][e + 3] * inv);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += 8) {     // the halves exchange four channels each: 16 bytes of a row to a lane
        const uint32_t a0 = pack_pair<DT>(o[i][e] * inv, o[i][e + 1] * inv), a1 = pack_pair<DT>(o[i][e + 2] * inv, o[i][e + 3] * inv);
        const uint32_t b0 = pack_pair<DT>(o[i][e + 4] * inv, o[i][e + 5] * inv), b1 = pack_pair<DT>(o[i][e + 6] * inv, o[i][e + 7] * inv);
        const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        if (exists) *(uint4 *)(op + (i * 32 + e * 2 + half * 8) * 2) = make_uint4(x[0], y[0], x[1], y[1]);
      }
    }
  }
}

// The rows of blocks that several workgroups shared: D / 4 threads a row, four channels each.
constexpr int JOIN_THREADS = 256;
template <int D, int DT>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(AttentionArgs a, const float *__restrict__ part, const float2 *__restrict__ stats,
                                                            char *__restrict__ out, float *__restrict__ lse) {
  using C = Att<D, DT>;
  constexpr int COLS = D / 4, ROWS = JOIN_THREADS / COLS, AHEAD = 4;
  const Block it(a, blockIdx.x, C::KEYS);
  const int r = blockIdx.y * ROWS + threadIdx.x / COLS, c = threadIdx.x % COLS * 4, row = it.block * ATT_ROWS + r;
  if (it.n_splits == 1 || row >= it.n_rows) return;
  const int64_t at = (int64_t)blockIdx.x * a.splits * ATT_ROWS + r;
  const int last = it.n_splits - 1;
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 <= last; s0 += AHEAD) {
    float2 ml[AHEAD];
    float4 x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t from = at + (int64_t)min(s0 + u, last) * ATT_ROWS;
      ml[u] = stats[from];
      x[u] = *(const float4 *)(part + from * D + c);
    }
    float to = m;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) to = fmaxf(to, ml[u].x);
    const float ref = to == -INFINITY ? 0.0f : to, old = fast_exp2(m - ref);
    m = to;
    l *= old; o.x *= old; o.y *= old; o.z *= old; o.w *= old;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float w = s0 + u <= last ? fast_exp2(ml[u].x - ref) : 0.0f;
      l = fmaf(ml[u].y, w, l);
      o.x = fmaf(x[u].x, w, o.x); o.y = fmaf(x[u].y, w, o.y); o.z = fmaf(x[u].z, w, o.z); o.w = fmaf(x[u].w, w, o.w);
    }
  }
  const int qi = it.query(row), g = row - qi * a.G, first = it.sq.q_len - a.lse_rows;
  if (c == 0 && qi >= first)
    lse[((int64_t)it.sq.b * a.Hq + it.h * a.G + g) * a.lse_rows + (qi - first)] = row_lse(m, l);
  const float inv = it.sees(row) > 0 ? 1.0f / l : 0.0f;
  char *op = out + (it.sq.b * a.o_sb + (int64_t)(it.h * a.G + g) * a.o_sh + (it.sq.q_start + qi) * a.o_st + c * C::ES);
  if constexpr (DT == DT_F32) *(float4 *)op = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else *(uint2 *)op = make_uint2(pack_pair<DT>(o.x * inv, o.y * inv), pack_pair<DT>(o.z * inv, o.w * inv));
}

template <int D, int DT>
hipError_t launch_d(const AttentionPlan &plan, const void *q, const void *k, const void *v, void *out, float *lse, void *ws, hipStream_t stream) {
  const AttentionArgs &a = plan.args;
  float *part = (float *)ws;
  float2 *stats = (float2 *)((char *)ws + plan.stats_at);
  hipLaunchKernelGGL((prefill_kernel<D, DT>), dim3((uint32_t)plan.items, (uint32_t)a.splits), dim3(Att<D, DT>::NT), 0, stream, a, (const char *)q,
                     (const char *)k, (const char *)v, (char *)out, lse, part, stats);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL((join_kernel<D, DT>), dim3((uint32_t)plan.items, ATT_ROWS / (JOIN_THREADS / (D / 4))), dim3(JOIN_THREADS), 0, stream, a, part, stats,
                     (char *)out, lse);
  return hipGetLastError();
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
