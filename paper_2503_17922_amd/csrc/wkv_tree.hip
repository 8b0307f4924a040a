// Attention for a tree of drafted tokens over a cache, and the acceptance of one of its paths.
//
// The rows of a block are (node, head of the group) pairs of one KV head, node-major: all of them see every row of the cache, and of the nodes' own rows those
// on the way to the top, a 64-bit mask a node.  One pass over the keys with a running reference and sum, transposed as in wkv_attention.hip:
//   S^T = K Q^T    keys the A operand, 32 rows the B operand: lane l holds row l % 32 and half of the tile's keys
//   O^T = V^T P^T  the probabilities as they lie in the lanes are the B operand, the values are read transposed
// 16-bit types take a probability as two numbers, its upper bits and what they leave (8 + 8 bits, 11 + 11), each a product of its own with the same values: nothing but the output
// is rounded to the type, as at a decode step.  With the upper part alone, rounded, outputs were 0.0024 (bf16; 0.00026 in fp16) of their root mean square off, more than the rounding of
// an output, 0.0017 (0.0002).  It costs, a call: one sequence of 4128 rows and 16 nodes 15.6 -> 16.0 us, 64 of them 170 -> 173, eleven of mixed lengths and 64 nodes, 28q/4kv heads in fp16, 66 -> 77,
// 64 of 2000 rows and 64 nodes 180 -> 225.  The lower products behind all upper ones of 16 keys: the same.
// Key and value tiles reach LDS by DMA, a tile ahead.  A cache is read once for up to 256 rows, so a few nodes are bound by the stream of the cache and many by
// the matrix pipe.  Where a wave's 32 rows are all there are, or half of them, the waves of a workgroup share the keys of a tile instead and join their results in LDS.
//
// bf16, 32q/8kv heads of 128 channels, 16 nodes over caches of 4128 rows: 64 sequences 175 us = 6.2 TB/s.
//
// How many rows a cache has is on the device: the ranges divide its capacity, and those behind its rows return at once.  The nodes' own tile, read from
// the new rows, is a range of its own where there are several.  They are put into the cache at the end or by the second launch: nobody reads its rows from n on.
#include "wkv_attention_tile.h"
#include "wkv_generation.h"

namespace wkv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The nodes of a sequence, one to a lane.
struct Nodes {
  uint64_t family, all;          // this lane's node: itself and those it hangs below (0: it does not exist); which nodes exist
  __device__ __forceinline__ Nodes(const TreeArgs &a, const int32_t *__restrict__ parent, int b) {
    const int lane = threadIdx.x & 63;
    int up = -2;                                   // a node on the way up, -1: the top was reached, -2: the way ends at no node
    if (lane < a.T) {
      up = parent[(int64_t)b * a.T + lane];
      if (up < -1 || up >= lane) up = -2;
    }
    family = 1ull << lane;
    // ways of 2^k steps from ways of 2^(k-1)
#pragma unroll
    for (int k = 0; k < 6; ++k) {
      const int at = max(up, 0);
      const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)family, at), hi = (uint32_t)__shfl((int)(uint32_t)(family >> 32), at);
      const int further = __shfl(up, at);
      if (up >= 0) { family |= (uint64_t)hi << 32 | lo; up = further; }
    }
    all = __ballot(up == -1);
    if (up != -1) family = 0;
  }
  __device__ __forceinline__ uint64_t of(int t) const {
    return (uint64_t)(uint32_t)__shfl((int)(uint32_t)(family >> 32), t) << 32 | (uint32_t)__shfl((int)(uint32_t)family, t);
  }
};

// Two floats as pairs of 16-bit numbers whose sums they are, but for what the second pair cannot hold: the upper bits, cut off, and what is left over of them.
struct Parts { uint32_t upper, lower; };
template <int DT>
__device__ __forceinline__ Parts split_pair(float a, float b) {
  if constexpr (DT == DT_F16) {
    const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
    return {__builtin_bit_cast(uint32_t, h), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a - (float)h[0], b - (float)h[1]))};
  } else {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    return {__builtin_amdgcn_perm(y, x, 0x07060302u), pack_pair<DT>(a - __uint_as_float(x & 0xffff0000u), b - __uint_as_float(y & 0xffff0000u))};
  }
}

// Whether 16 bytes of a tensor are finite numbers.
template <int DT>
__device__ __forceinline__ bool all_finite(const uint4 &x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool ok = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == DT_F32) ok &= (w[i] & 0x7f800000u) != 0x7f800000u;
    else {
      constexpr uint32_t E = DT == DT_BF16 ? 0x7f80u : 0x7c00u;
      ok &= (w[i] & E) != E && (w[i] >> 16 & E) != E;
    }
  }
  return ok;
}

// The new rows of the nodes that exist (`all`) into the cache, by NT threads.
template <int PPR, int NT>
__device__ __forceinline__ void copy_rows(const TreeArgs &a, uint64_t all, int b, int h, int n, const char *__restrict__ kn, const char *__restrict__ vn,
                                          char *__restrict__ kc, char *__restrict__ vc) {
  constexpr int AHEAD = 4;
  const int64_t from = b * a.n_sb + h * a.n_sh, to = b * a.c_sb + h * a.c_sh + n * a.c_st;
  for (int i0 = threadIdx.x; i0 < 2 * a.T * PPR; i0 += AHEAD * NT) {
    u32x4 x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = min(i0 + k * NT, 2 * a.T * PPR - 1), r = i / PPR;
      x[k] = *(const u32x4 *)((r & 1 ? vn : kn) + from + (r >> 1) * a.n_st + i % PPR * 16);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + k * NT, r = i / PPR;
      if (i < 2 * a.T * PPR && all >> (r >> 1) & 1) *(u32x4 *)((r & 1 ? vc : kc) + to + (r >> 1) * a.c_st + i % PPR * 16) = x[k];
    }
  }
}

// ROW_WAVES times 32 rows, KEY_WAVES waves to each.
template <int D, int DT, int ROW_WAVES, int KEY_WAVES>
struct Shares {
  static constexpr int WAVES = ROW_WAVES * KEY_WAVES, NT = WAVES * 64, ROWS = ROW_WAVES * 32;
  static constexpr int KW = tree_wave_keys(DT == DT_F32, KEY_WAVES), KEYS = KW * KEY_WAVES;
  using Tile = Att<D, DT, WAVES, KEYS>;
  static constexpr int SLOTS = 5, LDS = SLOTS * Tile::TILE;          // tiles of keys and of values in turn: two in use, three under way
  // of a SIMD; two at least where the LDS of a compute unit has room for as many workgroups
  static constexpr int LEAST_WAVES = 160 * 1024 / LDS * WAVES >= 8 ? 2 : 1;
};

template <int D, int DT, int ROW_WAVES, int KEY_WAVES, bool STREAM>
__global__ __launch_bounds__((ROW_WAVES * KEY_WAVES * 64), (Shares<D, DT, ROW_WAVES, KEY_WAVES>::LEAST_WAVES)) void tree_kernel(TreeArgs a, const char *__restrict__ q, const char *__restrict__ kn,
                                                                             const char *__restrict__ vn, const int32_t *__restrict__ parent,
                                                                             char *__restrict__ kc, char *__restrict__ vc,
                                                                             const int32_t *__restrict__ n_valid, char *__restrict__ out,
                                                                             float *__restrict__ part, float2 *__restrict__ stats) {
  using S = Shares<D, DT, ROW_WAVES, KEY_WAVES>;
  using C = typename S::Tile;
  constexpr int KS = C::KS, VT = C::VT, WAVES = S::WAVES, KW = S::KW, KT = KW / 32, KEYS = S::KEYS, ROWS = S::ROWS, ES = C::ES;
  __shared__ __attribute__((aligned(1024))) char ring[S::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, row_wave = wave / KEY_WAVES, key_wave = wave % KEY_WAVES;

  // where there are several ranges, y == 0 are the nodes, whose way is longest, and range y - 1 the others
  const int y = blockIdx.y;
  const bool whole = a.splits == 1, of_nodes = y == 0;
  const RangeOf it(blockIdx.x, y, a.heads, a.heads_magic);
  const int bh = it.head, split = whole ? 0 : y - 1, block = blockIdx.z, b = divide(bh, a.kv_magic), h = bh - b * a.Hkv;
  const int n = load_scalar(n_valid + bh);
  const bool fits = n >= 0 && n <= a.capacity - a.T;
  const int own = of_nodes && fits ? (a.T + KEYS - 1) / KEYS : 0;          // tiles of new rows
  const int t_begin = split * a.chunk, t_end = fits && split >= 0 ? min(t_begin + a.chunk, (n + KEYS - 1) / KEYS) : t_begin;
  const int n_tiles = own + max(t_end - t_begin, 0);
  if (n_tiles == 0 && !of_nodes) return;

  // ---- this lane's row
  const int wave_row = block * ROWS + row_wave * 32, row = min(wave_row + col, a.n_rows - 1);
  const int node = divide((uint32_t)row, a.g_magic), g = row - node * a.G;

  // ---- the key and value stream: tile i < own of the new rows, then those of the cache
  const int64_t c_at = b * a.c_sb + h * a.c_sh, n_at = b * a.n_sb + h * a.n_sh;
  const char *kb = kc + c_at, *vb = vc + c_at, *knb = kn + n_at, *vnb = vn + n_at;
  const int my_row = wave * C::RPI + lane / C::PPR, my_piece = lane % C::PPR;      // of this lane's first DMA instruction
  uint32_t k_slot[C::OFFS];
#pragma unroll
  for (int i = 0; i < C::OFFS; ++i) k_slot[i] = C::key_slot(my_row + i * C::RPI * WAVES, my_piece) * 16;
  const uint32_t v_slot = C::value_slot(my_row, my_piece) * 16;
  const uint32_t ring_at = lds_address(ring) + wave * 1024;
  // Tile i of keys or of values, number 2 * i (+ 1) of the ring; of rows past the last one, it again.
  auto fetch = [&](int i, bool is_v) __attribute__((always_inline)) {
    const uint32_t dst = ring_at + (2 * i + is_v) % S::SLOTS * C::TILE;
    const bool is_new = i < own;
    const int j0 = (is_new ? i : t_begin + i - own) * KEYS, last = min((is_new ? a.T : n) - 1 - j0, KEYS - 1);
    const int64_t by = is_new ? a.n_st : a.c_st;
    const char *from = (is_new ? (is_v ? vnb : knb) : is_v ? vb : kb) + j0 * by;
    const uint32_t st = (uint32_t)by, most = last * st, at = my_row * st;
#pragma unroll
    for (int x = 0; x < C::LPT; ++x)
      dma_rows<STREAM>(dst + x * (WAVES * 1024), from, min(at + x * (C::RPI * WAVES) * st, most) + (is_v ? v_slot : k_slot[x % C::OFFS]));
  };
  if (n_tiles > 0) { fetch(0, false); fetch(0, true); }
  if (n_tiles > 1) fetch(1, false);

  // ---- queries: B fragments; this row's part of the tree
  bf16x8 qf[KS];
  {
    const char *qp = q + (b * a.q_sb + (int64_t)(h * a.G + g) * a.q_sh + node * a.q_st) + half * 16;
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[i] = *(const bf16x8 *)(qp + i * 32);
    // (waited for here, once)
#pragma unroll
    for (int i = 0; i < KS; ++i) asm volatile("" : "+v"(qf[i]));
  }
  uint64_t family = 0, not_finite = 0, all = 0;     // of this row's node; of all nodes: those whose values are not all finite, those that exist
  if (of_nodes) {
    const Nodes nodes(a, parent, b);
    family = nodes.of(node);
    all = nodes.all;
    constexpr int AHEAD = 4;
    for (int t0 = 0; t0 < a.T; t0 += AHEAD * C::RPI) {
      uint4 x[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) x[k] = *(const uint4 *)(vnb + min(t0 + k * C::RPI + lane / C::PPR, a.T - 1) * a.n_st + lane % C::PPR * 16);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const uint64_t wrong = __ballot(!all_finite<DT>(x[k]));
        if (wrong)
          for (int r = 0; r < C::RPI; ++r)
            if (wrong >> (r * C::PPR) & ((1ull << C::PPR) - 1)) not_finite |= 1ull << min(t0 + k * C::RPI + r, a.T - 1);
      }
    }
  }
  f32x16 o[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;           // reference and this lane's part of the sum, base 2

  // (masked: key kt * 32 + half * 4 + x of the tile counts where bit kt * 32 + x of `seen` is set)
  auto attend = [&](const char *ks, const char *vs, bool masked, uint64_t seen) __attribute__((always_inline)) {
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
    if (masked) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!((uint32_t)(seen >> (kt * 32)) >> (e / 4 * 8 + e % 4) & 1u)) s[kt][e] = -INFINITY;
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
    if (__any(top > m + Reference<DT>::GROW)) {
      // (each row's moves by its own logits alone: what the rows beside it hold, padding among them, does not show in its roundings)
      const float to = top > m + Reference<DT>::GROW ? top : m, corr = to == -INFINITY ? 1.0f : fast_exp2(m - to);
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
        const Parts w0 = split_pair<DT>(p[e], p[e + 1]), w1 = split_pair<DT>(p[e + 2], p[e + 3]), w2 = split_pair<DT>(p[e + 4], p[e + 5]),
                    w3 = split_pair<DT>(p[e + 6], p[e + 7]);
        const bf16x8 upper = __builtin_bit_cast(bf16x8, make_uint4(w0.upper, w1.upper, w2.upper, w3.upper));
        const bf16x8 lower = __builtin_bit_cast(bf16x8, make_uint4(w0.lower, w1.lower, w2.lower, w3.lower));
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const char *vp = vs + (x * 16 + y) * C::ROWB + C::value_slot(y, i * 4 + at * 2 + tl % 4 / 2) * 16 + tl % 2 * 8;
          typedef __attribute__((address_space(3))) s16x4 lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)vp);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(__attribute__((address_space(3))) char *)(vp + 8 * C::ROWB));
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          o[i] = mfma_step<DT, 32>(vf, upper, o[i]);
          o[i] = mfma_step<DT, 32>(vf, lower, o[i]);
        }
      }
    }
  };

  for (int i = 0; i < n_tiles; ++i) {
    // the tiles are in LDS (each wave waits for its own requests but the next keys, the barrier for all), and everyone is done with the two before
    if (i + 1 < n_tiles) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(C::LPT) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (i + 1 < n_tiles) fetch(i + 1, true);
    if (i + 2 < n_tiles) fetch(i + 2, false);
    const char *ks = ring + 2 * i % S::SLOTS * C::TILE + key_wave * KW * C::ROWB, *vs = ring + (2 * i + 1) % S::SLOTS * C::TILE + key_wave * KW * C::ROWB;
    if (i < own && not_finite) {
      // A probability of zero times an infinity is a NaN: values that are not finite, of padding too, are taken out of the tile, and the rows that see them are
      // told at the end.
      char *tile = ring + (2 * i + 1) % S::SLOTS * C::TILE;
      for (int x = threadIdx.x; x < KEYS * C::PPR; x += S::NT)
        if (not_finite >> min(i * KEYS + x / C::PPR, a.T - 1) & 1) *(uint4 *)(tile + x * 16) = make_uint4(0, 0, 0, 0);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (wave_row >= a.n_rows) continue;
    const int j0 = (i < own ? i : t_begin + i - own) * KEYS + key_wave * KW, at = j0 + half * 4;
    uint64_t seen;
    if (i < own) seen = at < 64 ? family >> at : 0;
    else seen = at + 64 <= n ? ~0ull : at < n ? (1ull << (n - at)) - 1 : 0;
    attend(ks, vs, i < own || j0 + KW > n, seen);
  }

  if (family & not_finite) l = __uint_as_float(0x7fc00000u);

  if (whole && block == 0 && fits) copy_rows<C::PPR, S::NT>(a, all, b, h, n, kn, vn, kc, vc);

  // ---- the waves that share rows
  if constexpr (KEY_WAVES > 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");          // (the tiles are done with)
    constexpr int QUADS = VT * 4;
    static_assert((WAVES - ROW_WAVES) * 64 * (QUADS * 16 + 8) <= S::LDS, "room for the results of the waves that hand them over");
    float4 *o_s = (float4 *)ring;
    float2 *ml_s = (float2 *)(ring + (WAVES - ROW_WAVES) * 64 * QUADS * 16);
    const int slot = row_wave * (KEY_WAVES - 1) - 1;          // + key_wave: where a wave's results lie
    if (key_wave > 0) {
      const int at = slot + key_wave;
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) o_s[(at * QUADS + i * 4 + e / 4) * 64 + lane] = make_float4(o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]);
      ml_s[at * 64 + lane] = make_float2(m, l);
    }
    __syncthreads();
    if (key_wave > 0) return;
    float2 other[KEY_WAVES - 1];
    float to = m;
#pragma unroll
    for (int k = 1; k < KEY_WAVES; ++k) {
      other[k - 1] = ml_s[(slot + k) * 64 + lane];
      to = fmaxf(to, other[k - 1].x);
    }
    const float ref = to == -INFINITY ? 0.0f : to, by = fast_exp2(m - ref);
    m = to;
    l *= by;
#pragma unroll
    for (int i = 0; i < VT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] *= by;
#pragma unroll
    for (int k = 1; k < KEY_WAVES; ++k) {
      const float w = fast_exp2(other[k - 1].x - ref);
      l = fmaf(other[k - 1].y, w, l);
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const float4 x = o_s[((slot + k) * QUADS + i * 4 + e / 4) * 64 + lane];
          o[i][e] = fmaf(x.x, w, o[i][e]); o[i][e + 1] = fmaf(x.y, w, o[i][e + 1]);
          o[i][e + 2] = fmaf(x.z, w, o[i][e + 2]); o[i][e + 3] = fmaf(x.w, w, o[i][e + 3]);
        }
    }
  }

  // ---- results: of this range, for join_tree_kernel, or of the row
  l = add_halves(l, l);
  const bool exists = wave_row + col < a.n_rows;
  const bool counts = !of_nodes || family != 0;          // (a node that is none leaves its row as it is, and says so by a negative sum)
  if (a.splits > 1) {
    const int64_t at = (((int64_t)bh * a.blocks + block) * (a.splits + 1) + y) * ROWS + row_wave * 32 + col;
    if (exists && half == 0) stats[at] = counts ? make_float2(m, fits ? l : __uint_as_float(0x7fc00000u)) : make_float2(-INFINITY, -1.0f);
    if (!fits) return;
#pragma unroll
    for (int i = 0; i < VT; ++i)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (exists) *(float4 *)(part + at * D + i * 32 + e * 2 + half * 4) = make_float4(o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]);
    return;
  }
  const float inv = fits ? 1.0f / l : __uint_as_float(0x7fc00000u);
  char *op = out + (b * a.o_sb + (int64_t)(h * a.G + g) * a.o_sh + node * a.o_st);
#pragma unroll
  for (int i = 0; i < VT; ++i) {
    const f32x16 &x = o[i];
    if constexpr (DT == DT_F32) {
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (exists && counts) *(float4 *)(op + (i * 32 + e * 2 + half * 4) * ES) = make_float4(x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += 8) {     // the halves exchange four channels each: 16 bytes of a row to a lane
        const auto y0 = __builtin_amdgcn_permlane32_swap(pack_pair<DT>(x[e] * inv, x[e + 1] * inv), pack_pair<DT>(x[e + 4] * inv, x[e + 5] * inv), false, false);
        const auto y1 = __builtin_amdgcn_permlane32_swap(pack_pair<DT>(x[e + 2] * inv, x[e + 3] * inv), pack_pair<DT>(x[e + 6] * inv, x[e + 7] * inv), false, false);
        if (exists && counts) *(uint4 *)(op + (i * 32 + e * 2 + half * 8) * ES) = make_uint4(y0[0], y1[0], y0[1], y1[1]);
      }
    }
  }
}

// The rows of a block whose keys several workgroups shared: D / 4 threads take four channels each, of every GROUPS-th partial result.
constexpr int JOIN_THREADS = 256;
template <int D, int DT, int GROUPS>
__global__ __launch_bounds__(JOIN_THREADS) void join_tree_kernel(TreeArgs a, int rows_of_block, int keys_of_tile, const int32_t *__restrict__ n_valid,
                                                                 const float *__restrict__ part, const float2 *__restrict__ stats, char *__restrict__ out,
                                                                 const char *__restrict__ kn, const char *__restrict__ vn, const int32_t *__restrict__ parent,
                                                                 char *__restrict__ kc, char *__restrict__ vc) {
  constexpr int COLS = D / 4, AHEAD = 4, SLOTS = JOIN_THREADS / COLS, AT_ONCE = SLOTS / GROUPS, ES = DT == DT_F32 ? 4 : 2;
  __shared__ float4 o_s[GROUPS > 1 ? SLOTS : 1][COLS];
  __shared__ float2 ml_s[GROUPS > 1 ? SLOTS : 1];
  const int bh = blockIdx.x, b = divide(bh, a.kv_magic), h = bh - b * a.Hkv;
  const int n = load_scalar(n_valid + bh);
  const bool fits = n >= 0 && n <= a.capacity - a.T;
  if (blockIdx.y == 0) {                     // the new rows go into the cache
    if (fits) copy_rows<D * ES / 16, JOIN_THREADS>(a, Nodes(a, parent, b).all, b, h, n, kn, vn, kc, vc);
    return;
  }
  const int slot = threadIdx.x / COLS, col = threadIdx.x % COLS, group = slot % GROUPS;
  const int row = (blockIdx.y - 1) * AT_ONCE + slot / GROUPS, block = row / rows_of_block;
  const bool exists = row < a.n_rows;
  // the nodes', then the ranges that hold rows
  const int tiles = fits ? (n + keys_of_tile - 1) / keys_of_tile : 0, splits = (tiles + a.chunk - 1) / a.chunk + 1;
  const int64_t at = ((int64_t)bh * a.blocks + block) * (a.splits + 1) * rows_of_block + (row - block * rows_of_block);
  float m = -INFINITY, l = 0.0f, first = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (exists) first = stats[at].y;
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
  for (int s0 = group; exists && fits && s0 < splits; s0 += AHEAD * GROUPS) {
    float2 ml[AHEAD];
    float4 x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      ml[u] = make_float2(-INFINITY, 0.0f);
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s0 + u * GROUPS < splits) {
        const int64_t from = at + (int64_t)(s0 + u * GROUPS) * rows_of_block;
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
  if (!exists || first < 0.0f) return;
  const int node = divide((uint32_t)row, a.g_magic), g = row - node * a.G;
  const float inv = fits ? 1.0f / l : __uint_as_float(0x7fc00000u);
  char *op = out + (b * a.o_sb + (int64_t)(h * a.G + g) * a.o_sh + node * a.o_st + col * 4 * ES);
  if constexpr (DT == DT_F32) *(float4 *)op = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else *(uint2 *)op = make_uint2(pack_pair<DT>(o.x * inv, o.y * inv), pack_pair<DT>(o.z * inv, o.w * inv));
}

template <int D, int DT, int ROW_WAVES, int KEY_WAVES>
hipError_t launch_shares(const TreePlan &plan, const void *q, const void *kn, const void *vn, const int32_t *parent, void *kc, void *vc,
                         const int32_t *n_valid, void *out, void *ws, hipStream_t stream) {
  using S = Shares<D, DT, ROW_WAVES, KEY_WAVES>;
  const TreeArgs &a = plan.args;
  float *part = (float *)ws;
  float2 *stats = (float2 *)((char *)ws + plan.stats_at);
  const dim3 grid((uint32_t)a.heads, (uint32_t)(a.splits == 1 ? 1 : a.splits + 1), (uint32_t)a.blocks);
#define WKV_TREE(STREAM) \
  hipLaunchKernelGGL((tree_kernel<D, DT, ROW_WAVES, KEY_WAVES, STREAM>), grid, dim3(S::NT), 0, stream, a, (const char *)q, (const char *)kn, (const char *)vn, \
                     parent, (char *)kc, (char *)vc, n_valid, (char *)out, part, stats)
  if (plan.streams) WKV_TREE(true);
  else WKV_TREE(false);
#undef WKV_TREE
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  constexpr int SLOTS = JOIN_THREADS / (D / 4);
#define WKV_JOIN(GROUPS) \
  hipLaunchKernelGGL((join_tree_kernel<D, DT, GROUPS>), dim3((uint32_t)a.heads, (uint32_t)((a.n_rows + SLOTS / GROUPS - 1) / (SLOTS / GROUPS)) + 1), \
                     dim3(JOIN_THREADS), 0, stream, a, S::ROWS, S::KEYS, n_valid, part, stats, (char *)out, (const char *)kn, \
                     (const char *)vn, parent, (char *)kc, (char *)vc)
  // The ranges of a row by one group of threads / by eight, us a call, 16 nodes, 32q/8kv heads of 128 channels in bf16: five ranges (eight sequences of 4128 rows) 40.5 / 43.5, eight (four of
  // them) 22.9 / 23.9, 14 (two) 18.3 / 18.0, 23 (one) 17.8 / 16.0; 64 nodes 14 ranges 24.2 / 24.3; 8q/1kv heads, three nodes, 60 ranges 24.3 / 17.7.
  if (a.splits > 8) WKV_JOIN(8);
  else WKV_JOIN(1);
#undef WKV_JOIN
  return hipGetLastError();
}

template <int D, int DT>
hipError_t launch_d(const TreePlan &plan, const void *q, const void *kn, const void *vn, const int32_t *parent, void *kc, void *vc, const int32_t *n_valid,
                    void *out, void *ws, hipStream_t stream) {
#define WKV_SHARES(R, K) \
  if (plan.row_waves == R && plan.key_waves == K) return launch_shares<D, DT, R, K>(plan, q, kn, vn, parent, kc, vc, n_valid, out, ws, stream)
  WKV_SHARES(2, 2);
  WKV_SHARES(4, 1);
  if constexpr (DT != DT_F32) WKV_SHARES(8, 1);
#undef WKV_SHARES
  return hipErrorInvalidValue;
}

// ---- acceptance ------------------------------------------------------------------------------------
// How many nodes of sequence b's path are kept: as far as it ascends within the tree.  Lane i of a wave gets node i of the path.
__device__ __forceinline__ int accepted(const TreeArgs &a, const int32_t *__restrict__ path, const int32_t *__restrict__ n_accept, int b, int &node) {
  const int lane = threadIdx.x & 63, want = n_accept[b];
  const int32_t *p = path + (int64_t)b * a.T;
  node = lane < a.T ? p[lane] : -1;
  const int before = lane > 0 && lane < a.T ? p[lane - 1] : -1;
  const uint64_t wrong = __ballot(!(lane < want && lane < a.T && node >= 0 && node < a.T && node > before));
  return wrong ? __builtin_ctzll(wrong) : 64;
}

constexpr int ACCEPT_THREADS = 256;
// Rows n + path[i] of one tensor and (sequence, KV head) into rows n + i.  All nodes' rows are asked for before the path is known, and every thread finds out
// where its own go: two trips to memory instead of three.  64 sequences with 16 nodes, 8 KV heads of 128 channels, bf16: 4.9 us; with the rows in an array under
// conditions, which the compiler keeps outside the registers, 16.5.
template <int PPR>
__global__ __launch_bounds__(ACCEPT_THREADS) void accept_kernel(TreeArgs a, EvictLayers layers, const int32_t *__restrict__ path,
                                                                const int32_t *__restrict__ n_accept, const int32_t *__restrict__ n_valid) {
  constexpr int ROWS = ACCEPT_THREADS / PPR, TURNS = WKV_MAX_NODES / ROWS;
  __shared__ int place_s[WKV_MAX_NODES];          // of a node's row
  const int bh = blockIdx.x, b = divide(bh, a.kv_magic), h = bh - b * a.Hkv, layer = blockIdx.y >> 1;
  char *cache = (char *)(blockIdx.y & 1 ? layers.v[layer] : layers.k[layer]);
  const int n = load_scalar(n_valid + bh);
  if (n < 0 || n > a.capacity - a.T) return;
  char *rows = cache + (b * a.c_sb + h * a.c_sh + (int64_t)n * a.c_st) + threadIdx.x % PPR * 16;
  const int my_node = threadIdx.x / PPR;
  u32x4 x[TURNS];
#pragma unroll
  for (int k = 0; k < TURNS; ++k)
    x[k] = *(const u32x4 *)(rows + min(k * ROWS + my_node, a.T - 1) * a.c_st);          // (without a condition, under which an array leaves the registers)
  if (threadIdx.x < 64) {
    place_s[threadIdx.x] = -1;
    int node;
    const int count = accepted(a, path, n_accept, b, node);
    if ((int)threadIdx.x < count) place_s[node] = threadIdx.x;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < TURNS; ++k) {
    const int t = k * ROWS + my_node, to = place_s[t];
    if (to >= 0 && to != t) *(u32x4 *)(rows + to * a.c_st) = x[k];
  }
}

// (a launch of its own: the workgroups above read the counts)
__global__ __launch_bounds__(ACCEPT_THREADS) void advance_kernel(TreeArgs a, const int32_t *__restrict__ path, const int32_t *__restrict__ n_accept,
                                                                 int32_t *__restrict__ n_valid) {
  const int bh = blockIdx.x * (ACCEPT_THREADS / 64) + (threadIdx.x >> 6);
  if (bh >= a.heads) return;
  int node;
  const int count = accepted(a, path, n_accept, divide(bh, a.kv_magic), node), n = n_valid[bh];
  if (n >= 0 && n <= a.capacity - a.T && (threadIdx.x & 63) == 0) n_valid[bh] = n + count;
}

}  // namespace

hipError_t launch_tree(const TreePlan &plan, const void *q, const void *kn, const void *vn, const int32_t *parent, void *kc, void *vc,
                       const int32_t *n_valid, void *out, void *ws, hipStream_t stream) {
#define WKV_TREE_TYPE(DT) \
  return plan.args.d == 128 ? launch_d<128, DT>(plan, q, kn, vn, parent, kc, vc, n_valid, out, ws, stream) : launch_d<64, DT>(plan, q, kn, vn, parent, kc, vc, n_valid, out, ws, stream)
  if (plan.args.dtype == WKV_BF16) WKV_TREE_TYPE(DT_BF16);
  if (plan.args.dtype == WKV_F16) WKV_TREE_TYPE(DT_F16);
  WKV_TREE_TYPE(DT_F32);
#undef WKV_TREE_TYPE
}

hipError_t launch_accept(const TreeArgs &a, const EvictLayers &layers, int32_t n_layers, const int32_t *path, const int32_t *n_accept,
                         int32_t *n_valid, bool keep_count, hipStream_t stream) {
  const dim3 grid((uint32_t)a.heads, (uint32_t)n_layers * 2);
#define WKV_ACCEPT(PPR) hipLaunchKernelGGL((accept_kernel<PPR>), grid, dim3(ACCEPT_THREADS), 0, stream, a, layers, path, n_accept, n_valid)
  const int64_t pieces = a.d * elem_bytes(a.dtype) / 16;
  if (pieces == 32) WKV_ACCEPT(32);
  else if (pieces == 16) WKV_ACCEPT(16);
  else WKV_ACCEPT(8);
#undef WKV_ACCEPT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || keep_count) return e;
  hipLaunchKernelGGL(advance_kernel, dim3((uint32_t)((a.heads + ACCEPT_THREADS / 64 - 1) / (ACCEPT_THREADS / 64))), dim3(ACCEPT_THREADS), 0, stream, a, path, n_accept, n_valid);
  return hipGetLastError();
}

}  // namespace wkv
