// The decode step over caches in 8 and 4 bits: softmax(q K^T scale) V over rows that are codes with a power of two for every 32 channels.
//
// Bound by the stream of codes, half or a quarter of a 16-bit cache's, beside which the conversions count.  A pair of codes with its scale becomes a
// pair of bfloat16 by one instruction, exactly, so both products run on the matrix pipe:
//   S = K Q^T      16 cache rows the A operand, in operand layout as they arrive; the query heads the B operand
//   O^T = V^T P^T  a lane fetches eight channels of the eight rows whose scores it holds, and transposes them among its registers: channel tile c of the A operand
//                  is channel c of every lane, the probabilities are the B operand as they lie
// The 16 columns of the B operand hold up to eight heads and parts of their numbers: a query or a probability is the sum of two or three bfloat16,
// eight bits each, in columns of their own, and nothing is rounded to 16 bits (a 32-bit result would show it).  Up to four heads the three parts fit the columns;
// five heads and more take a second product for the third part.
//
// Caches of 4128 rows, 32q/8kv heads of 128 channels, 8 bits: one sequence 7.0 us, 64 of them 87 us = 6.4 TB/s (103 before the codes came by nontemporal loads and scalar
// addresses, 90 with 1536 ranges).  44 of 96 to 4500 rows, 28q/4kv, 4 bits, 19.4 us = 2.8 TB/s (20.0).  Blocks fetched two or three ahead: nothing or worse (with 1536 ranges 94 us for the 64, 20.8 and 24.3 for the
// 44).  The merge is 4 to 5 us more.
//
// Partial results and their merge are those of the decode step over plain caches (wkv_decode.hip); the key ranges are fewer (plan_quantized).
#include "wkv_decode_parts.h"
#include "wkv_few_bits.h"

namespace wkv {

namespace {

constexpr int DQ_THREADS = 256, DQ_WAVES = DQ_THREADS / 64, BLOCK = 32;      // rows of a block, a wave's
constexpr int PARTS = 3;

// How a row of codes is read.
template <int FORMAT, int D>
struct Row {
  static constexpr int BYTES = code_bytes<FORMAT>(D), SB = D / SCALE_GROUP;
  static constexpr int K_LOAD = BYTES >= 64 ? 16 : 8;                        // bytes of a load on the key side: 4 lanes take 4 * K_LOAD neighbouring ones
  static constexpr int K_LOADS = BYTES / (4 * K_LOAD), K_CH = K_LOAD * D / BYTES;      // loads, channels of one
  static constexpr int STEPS = K_CH / 8;                                     // contraction steps of a load
  static constexpr int V_LOAD = BYTES / 16, V_CH = D / 16;                   // bytes and channels of a lane on the value side
};
template <int BYTES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

// STREAM: a nontemporal load, which puts nothing into the memory-side cache.
typedef const __attribute__((address_space(1))) char *global_ptr;
template <bool STREAM, typename T>
__device__ __forceinline__ T load(global_ptr base, uint32_t offset) {
  typedef const __attribute__((address_space(1))) T *P;
  if constexpr (STREAM) return __builtin_nontemporal_load((P)(base + offset));
  else return *(P)(base + offset);
}

// Word w of a load.
template <typename T>
__device__ __forceinline__ uint32_t word(const T &x, int w) {
  if constexpr (sizeof(T) <= 4) return (uint32_t)x;
  else return x[w];
}

typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, (b16x2){(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ float low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Parts `first` and on of two numbers, `which` of them in this lane: the nearest bfloat16, the nearest of what is left, ..
template <int N>
__device__ __forceinline__ uint32_t part_of(float a, float b, int which) {
  uint32_t p = pack_bf16(a, b), got = p;
#pragma unroll
  for (int k = 1; k < N; ++k) {
    a -= low(p); b -= high(p);
    p = pack_bf16(a, b);
    got = which == k ? p : got;
  }
  return which < N ? got : 0u;
}

// A number's upper eight bits.
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// The sum over the columns of a head, in all of them: lanes COLUMNS apart within 16.
template <int COLUMNS>
__device__ __forceinline__ float columns_sum(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xF, 0xF, false));      // row_ror:8
  if (COLUMNS == 4) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x124, 0xF, 0xF, false));      // row_ror:4
  return x;
}

// COLUMNS: 4 or 8 heads at most, in this many columns; 16 / COLUMNS parts of a number fit beside each other.
template <int DT, int D, int FORMAT, int COLUMNS, bool STREAM>
__global__ __launch_bounds__(DQ_THREADS, 2) void decode_quantized_kernel(DecodeShape s, const char *__restrict__ q_new, const char *__restrict__ k_codes,
                                                                        const uint8_t *__restrict__ k_scales, const char *__restrict__ v_codes,
                                                                        const uint8_t *__restrict__ v_scales, const int32_t *__restrict__ n_valid,
                                                                        float *__restrict__ part) {
  using R = Row<FORMAT, D>;
  constexpr int FIT = 16 / COLUMNS, ES = DT == DT_F32 ? 4 : 2;
  constexpr int Q_PARTS = DT == DT_BF16 ? 1 : DT == DT_F16 ? 2 : 3;          // bf16 is itself, 11 bits are two parts, 24 three
  constexpr int Q_SETS = (Q_PARTS + FIT - 1) / FIT, P_SETS = (PARTS + FIT - 1) / FIT;
  constexpr int QS = R::K_LOADS * R::STEPS;                                  // contraction steps of a row
  __shared__ float wave_state[DQ_WAVES][COLUMNS][D + 2];

  const KeyRange item(s, n_valid);
  const int bh = item.head, b = divide(bh, s.kv_magic), h = bh - b * s.Hkv, split = item.range;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4, head = col % COLUMNS, which = col / COLUMNS;
  const int n = item.n, c0 = split * s.chunk, cend = min(c0 + s.chunk, n < s.capacity ? n : 0);
  if (c0 >= cend) {                          // a range without rows says so, and the first whether the cache cannot take another
    if (threadIdx.x < s.G)
      part_stats(s, part, part_index(s, bh, split, threadIdx.x)) =
          make_float2(split == 0 && (n < 0 || n >= s.capacity) ? __uint_as_float(0x7fc00000u) : -INFINITY, 0.0f);
    return;
  }
  const int64_t cache = (int64_t)b * s.sb + (int64_t)h * s.sh;
  const uint32_t st = (uint32_t)s.st;
  const char *kc = k_codes + cache, *vc = v_codes + cache;
  const uint8_t *ks = k_scales + (int64_t)bh * s.capacity * R::SB, *vs = v_scales + (int64_t)bh * s.capacity * R::SB;

  struct Raw {
    typename Word<R::K_LOAD>::type k[2][R::K_LOADS];
    typename Word<R::V_LOAD>::type v[8];
    uint32_t k_scale[2], v_scale[2];
  };
  const uint32_t k_row = col * st, v_row = quad * 4 * st, ks_row = col * R::SB, vs_row = (quad * 4 + (col & 3)) * R::SB;
  const uint32_t k_lane = quad * R::K_LOAD, v_lane = col * R::V_LOAD, vs_lane = col * R::V_CH / SCALE_GROUP;
  auto request = [&](Raw &x, int j0) __attribute__((always_inline)) {
    typedef typename Word<R::K_LOAD>::type KW;
    typedef typename Word<R::V_LOAD>::type VW;
    typedef typename Word<R::SB>::type SW;
    global_ptr kb = (global_ptr)(kc + (int64_t)j0 * s.st), vb = (global_ptr)(vc + (int64_t)j0 * s.st);
    global_ptr ksb = (global_ptr)(ks + (int64_t)j0 * R::SB), vsb = (global_ptr)(vs + (int64_t)j0 * R::SB);
    // (a scalar address and an offset of 32 bits each: left to itself the compiler keeps 64 bits a load and lane)
    asm("" : "+s"(kb));
    asm("" : "+s"(vb));
    asm("" : "+s"(ksb));
    asm("" : "+s"(vsb));
    const uint32_t last = min(cend - 1 - j0, BLOCK - 1), most = last * st;          // rows past the range: its last one again
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t at = min(k_row + t * 16 * st, most) + k_lane;
#pragma unroll
      for (int l = 0; l < R::K_LOADS; ++l) x.k[t][l] = load<STREAM, KW>(kb, at + l * 4 * R::K_LOAD);
      x.k_scale[t] = load<false, SW>(ksb, min(ks_row + t * 16 * R::SB, last * R::SB));
      // a quad of lanes has the scales of its channels in four rows
      x.v_scale[t] = load<false, uint8_t>(vsb, min(vs_row + t * 16 * R::SB, last * R::SB) + vs_lane);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = load<STREAM, VW>(vb, min(v_row + (i / 4 * 16 + i % 4) * st, most) + v_lane);
  };
  Raw next;
  if (c0 + wave * BLOCK < cend) request(next, c0 + wave * BLOCK);

  // ---- queries: B fragments
  bf16x8 qf[Q_SETS][QS];
#pragma unroll
  for (int l = 0; l < R::K_LOADS; ++l)
#pragma unroll
    for (int u = 0; u < R::STEPS; ++u) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = 0.0f;
      if (head < s.G) {
        const char *qp = q_new + (((int64_t)bh * s.G + head) * D + (l * 4 + quad) * R::K_CH + u * 8) * ES;
        widen<DT>(*(const uint4 *)qp, f);
        if constexpr (DT == DT_F32) widen<DT>(*(const uint4 *)(qp + 16), f + 4);
      }
#pragma unroll
      for (int set = 0; set < Q_SETS; ++set) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = part_of<Q_PARTS>(f[2 * e], f[2 * e + 1], set * FIT + which);
        qf[set][l * R::STEPS + u] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }

  // COLUMNS == 4: parts 0, 1, 2 of a probability, and its third part's rest, which is nothing; 8: parts 0 and 1, then part 2 in the first eight columns
  const float takes_first = which >= 1 ? 1.0f : 0.0f, takes_second = which >= 2 ? 1.0f : 0.0f, takes_third = which == 0 ? 1.0f : 0.0f;
  const float nothing = COLUMNS == 4 && which == 3 ? -INFINITY : 0.0f;          // added to a logit
  f32x4 o[R::V_CH];                          // o[c][i]: channel (quad * 4 + i) * V_CH + c, of this column
#pragma unroll
  for (int c = 0; c < R::V_CH; ++c) o[c] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;             // reference and this lane's part of the sum, base 2

  for (int j0 = c0 + wave * BLOCK; j0 < cend; j0 += DQ_WAVES * BLOCK) {
    const Raw x = next;
    if (j0 + DQ_WAVES * BLOCK < cend) request(next, j0 + DQ_WAVES * BLOCK);
    // ---- logits of 32 rows: element i of tile t is row t * 16 + quad * 4 + i
    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ld = 0; ld < R::K_LOADS; ++ld) {
        const float scale = scale_of(x.k_scale[t] >> ((ld * 4 + quad) * R::K_CH / SCALE_GROUP * 8) & 255u);
#pragma unroll
        for (int u = 0; u < R::STEPS; ++u) {
          uint32_t w[4];
          if constexpr (FORMAT == E4M3) {
            w[0] = bf16_pair<FORMAT, 0>(word(x.k[t][ld], 2 * u), scale); w[1] = bf16_pair<FORMAT, 1>(word(x.k[t][ld], 2 * u), scale);
            w[2] = bf16_pair<FORMAT, 0>(word(x.k[t][ld], 2 * u + 1), scale); w[3] = bf16_pair<FORMAT, 1>(word(x.k[t][ld], 2 * u + 1), scale);
          } else {
            w[0] = bf16_pair<FORMAT, 0>(word(x.k[t][ld], u), scale); w[1] = bf16_pair<FORMAT, 1>(word(x.k[t][ld], u), scale);
            w[2] = bf16_pair<FORMAT, 2>(word(x.k[t][ld], u), scale); w[3] = bf16_pair<FORMAT, 3>(word(x.k[t][ld], u), scale);
          }
          const bf16x8 kf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
          for (int set = 0; set < Q_SETS; ++set) sc[t] = mfma_16x16x32<false>(kf, qf[set][ld * R::STEPS + u], sc[t]);
        }
      }
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = columns_sum<COLUMNS>(sc[i / 4][i % 4]);
    if (j0 + BLOCK > cend) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (j0 + i / 4 * 16 + quad * 4 + i % 4 >= cend) p[i] = -INFINITY;
    }
    float top = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, p[i]);
    // (the reference is the same in all lanes of a column, and moves when a logit is 2^8 times as much)
    top = quads_max(top) * s.c1;
    if (__any(top > m + 8.0f)) {
      const float to = fmaxf(m, top), corr = to == -INFINITY ? 1.0f : fast_exp2(m - to);
      m = to;
      l *= corr;
#pragma unroll
      for (int c = 0; c < R::V_CH; ++c) o[c] *= corr;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = fast_exp2(fmaf(p[i], s.c1, nothing - ref));
      l += p[i];
    }
    // Three parts of a probability, its upper eight bits, the next eight and the last: cut off, so that their sum is the number itself.  Every lane goes as far as its part.
    bf16x8 pf[P_SETS];
    {
      float x0[8], x1[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (COLUMNS == 4) {
          x0[i] = fmaf(-takes_first, upper(p[i]), p[i]);
          x0[i] = fmaf(-takes_second, upper(x0[i]), x0[i]);
        } else {
          const float rest = p[i] - upper(p[i]);
          x0[i] = which ? rest : p[i];
          x1[i] = (rest - upper(rest)) * takes_third;
        }
      }
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(x0[2 * i + 1]), __float_as_uint(x0[2 * i]), 0x07060302u);
      pf[0] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      if constexpr (P_SETS == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(x1[2 * i + 1]), __float_as_uint(x1[2 * i]), 0x07060302u);
        pf[1] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
    // ---- values: pairs of channels of a row, then pairs of rows of a channel
    uint32_t vf[R::V_CH][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint32_t pair[2][R::V_CH / 2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = 2 * r + k;
        // row i's scale lies in lane i % 4 of every quad
        const int from = (int)x.v_scale[i / 4];
        uint32_t byte;
        switch (i % 4) {
          case 0: byte = __builtin_amdgcn_mov_dpp(from, 0x00, 0xF, 0xF, true); break;
          case 1: byte = __builtin_amdgcn_mov_dpp(from, 0x55, 0xF, 0xF, true); break;
          case 2: byte = __builtin_amdgcn_mov_dpp(from, 0xAA, 0xF, 0xF, true); break;
          default: byte = __builtin_amdgcn_mov_dpp(from, 0xFF, 0xF, 0xF, true); break;
        }
        const float scale = scale_of(byte);
        if constexpr (FORMAT == E4M3) {
#pragma unroll
          for (int c = 0; c < R::V_CH / 4; ++c) {
            pair[k][2 * c] = bf16_pair<FORMAT, 0>(word(x.v[i], c), scale);
            pair[k][2 * c + 1] = bf16_pair<FORMAT, 1>(word(x.v[i], c), scale);
          }
        } else {
          pair[k][0] = bf16_pair<FORMAT, 0>(word(x.v[i], 0), scale);
          pair[k][1] = bf16_pair<FORMAT, 1>(word(x.v[i], 0), scale);
          if constexpr (R::V_CH == 8) {
            pair[k][2] = bf16_pair<FORMAT, 2>(word(x.v[i], 0), scale);
            pair[k][3] = bf16_pair<FORMAT, 3>(word(x.v[i], 0), scale);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < R::V_CH / 2; ++c) {
        vf[2 * c][r] = __builtin_amdgcn_perm(pair[1][c], pair[0][c], 0x05040100u);
        vf[2 * c + 1][r] = __builtin_amdgcn_perm(pair[1][c], pair[0][c], 0x07060302u);
      }
    }
#pragma unroll
    for (int c = 0; c < R::V_CH; ++c)
#pragma unroll
      for (int set = 0; set < P_SETS; ++set)
        o[c] = mfma_16x16x32<false>(__builtin_bit_cast(bf16x8, make_uint4(vf[c][0], vf[c][1], vf[c][2], vf[c][3])), pf[set], o[c]);
  }

  // ---- the parts of a head together, then the waves
  l = quads_sum(l);
#pragma unroll
  for (int c = 0; c < R::V_CH; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[c][i] = columns_sum<COLUMNS>(o[c][i]);
  if (col < COLUMNS)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < R::V_CH; ++c) wave_state[wave][col][(quad * 4 + i) * R::V_CH + c] = o[c][i];
  if (quad == 0 && col < COLUMNS) { wave_state[wave][col][D] = m; wave_state[wave][col][D + 1] = l; }
  __syncthreads();
  for (int i = threadIdx.x; i < s.G * D; i += DQ_THREADS) {
    const int g = i / D, c = i % D;
    float mm = wave_state[0][g][D];
#pragma unroll
    for (int w = 1; w < DQ_WAVES; ++w) mm = fmaxf(mm, wave_state[w][g][D]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    float ll = 0.0f, oo = 0.0f;
#pragma unroll
    for (int w = 0; w < DQ_WAVES; ++w) {
      const float a = fast_exp2(wave_state[w][g][D] - ref);
      ll = fmaf(wave_state[w][g][D + 1], a, ll);
      oo = fmaf(wave_state[w][g][c], a, oo);
    }
    const uint32_t at = part_index(s, bh, split, g);
    part[at * D + c] = oo;
    if (c == 0) part_stats(s, part, at) = make_float2(mm, ll);
  }
}

// A workgroup per (sequence, KV head) and query head: the new token's rows as the caches will hold them (head 0's workgroup puts them there), its logit, and the
// merge of the key ranges.
template <int DT, int D, int FORMAT>
__global__ __launch_bounds__(DQ_THREADS) void merge_quantized_kernel(DecodeShape s, const char *__restrict__ q_new, const char *__restrict__ k_new,
                                                                     const char *__restrict__ v_new, char *__restrict__ k_codes,
                                                                     uint8_t *__restrict__ k_scales, char *__restrict__ v_codes,
                                                                     uint8_t *__restrict__ v_scales, const float *__restrict__ part,
                                                                     int32_t *__restrict__ n_valid, float *__restrict__ out) {
  using R = Row<FORMAT, D>;
  constexpr int ES = DT == DT_F32 ? 4 : 2, COLS = D / 4, GROUPS = DQ_THREADS / COLS;
  __shared__ float weight_s[DQ_THREADS], wave_m[DQ_WAVES], wave_l[DQ_WAVES], new_v[D], logit_s;
  __shared__ __attribute__((aligned(16))) float acc_s[GROUPS][D];
  __shared__ float first_s;
  const int bh = blockIdx.x, g = blockIdx.y, b = divide(bh, s.kv_magic), h = bh - b * s.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // statistics of the ranges, one a thread
  float2 ml = make_float2(-INFINITY, 0.0f);
  if (tid < s.n_splits) ml = part_stats(s, part, part_index(s, bh, tid, g));
  // the new rows: wave 0 the key, wave 1 the value, two channels a lane
  const int c = 2 * lane;
  if (wave < 2) {
    auto two = [&](const char *row) __attribute__((always_inline)) {
      if constexpr (DT == DT_F32) return *(const float2 *)(row + c * ES);
      else {
        const uint32_t w = *(const uint32_t *)(row + c * ES);
        if constexpr (DT == DT_BF16) return make_float2(low(w), high(w));
        else { typedef _Float16 f16x2 __attribute__((ext_vector_type(2))); const f16x2 x = __builtin_bit_cast(f16x2, w); return make_float2((float)x[0], (float)x[1]); }
      }
    };
    const bool in = c < D;
    float2 x = make_float2(0.0f, 0.0f), q = x;
    if (in) x = two((wave ? v_new : k_new) + (int64_t)bh * D * ES);
    if (in && wave == 0) q = two(q_new + ((int64_t)bh * s.G + g) * D * ES);
    // 16 lanes share a scale
    uint32_t largest = max(__float_as_uint(x.x) & 0x7fffffffu, __float_as_uint(x.y) & 0x7fffffffu);
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x128, 0xF, 0xF, false));      // row_ror:8, 4, 2, 1
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x124, 0xF, 0xF, false));
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x122, 0xF, 0xF, false));
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x121, 0xF, 0xF, false));
    const uint32_t byte = (uint32_t)scale_byte<FORMAT>(largest);
    const float scale = scale_of(byte);
    uint32_t code = to_codes<FORMAT, 0>(0, x.x, x.y, scale);
    if (byte == NO_SCALE) code = 0;
    x = float_pair<FORMAT, 0>(code, scale);
    if (wave == 0) {
      const float dot = wave_sum(in ? fmaf(q.x, x.x, q.y * x.y) : 0.0f);
      if (lane == 0) logit_s = dot * s.c1;
    } else if (in) {
      new_v[c] = x.x; new_v[c + 1] = x.y;
    }
    if (g == 0 && in) {
      const int n = n_valid[bh];              // (of this workgroup alone, which raises it at the end)
      if (n >= 0 && n < s.capacity) {
        char *to = (wave ? v_codes : k_codes) + ((int64_t)b * s.sb + (int64_t)h * s.sh + (int64_t)n * s.st);
        if constexpr (FORMAT == E4M3) *(uint16_t *)(to + lane * 2) = (uint16_t)code;
        else *(uint8_t *)(to + lane) = (uint8_t)code;
        if (lane % 16 == 0) (wave ? v_scales : k_scales)[((int64_t)bh * s.capacity + n) * R::SB + lane / 16] = (uint8_t)byte;
      }
    }
  }
  const float top = wave_max(ml.x);
  if (lane == 0) wave_m[wave] = top;
  if (tid == 0) first_s = ml.x;              // NaN: the cache cannot take the row
  __syncthreads();
  float m = logit_s;
#pragma unroll
  for (int w = 0; w < DQ_WAVES; ++w) m = fmaxf(m, wave_m[w]);
  const float ref = m == -INFINITY ? 0.0f : m;
  const float a = fast_exp2(ml.x - ref);     // a range without rows: 0
  const float sum = wave_sum(ml.x == -INFINITY ? ml.y : ml.y * a);          // (its sum is 0, or NaN where all its logits are)
  if (lane == 0) wave_l[wave] = sum;
  weight_s[tid] = a;
  __syncthreads();
  const float w_new = fast_exp2(logit_s - ref);
  float l = w_new;
#pragma unroll
  for (int w = 0; w < DQ_WAVES; ++w) l += wave_l[w];
  // (outputs of a range without rows are whatever memory held: not read)
  const int group = tid / COLS, at = tid % COLS;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int sp = group; sp < s.n_splits; sp += GROUPS) {
    const float w = weight_s[sp];
    if (w == 0.0f) continue;
    const float4 x = *(const float4 *)(part + (int64_t)part_index(s, bh, sp, g) * D + at * 4);
    o.x = fmaf(x.x, w, o.x); o.y = fmaf(x.y, w, o.y); o.z = fmaf(x.z, w, o.z); o.w = fmaf(x.w, w, o.w);
  }
  *(float4 *)&acc_s[group][at * 4] = o;
  __syncthreads();
  if (tid < D) {
    float x = w_new * new_v[tid];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) x += acc_s[i][tid];
    out[((int64_t)bh * s.G + g) * D + tid] = first_s != first_s ? first_s : x / l;
  }
  if (g == 0 && tid == 0 && !s.keep_count) {
    const int n = n_valid[bh];
    if (n >= 0 && n < s.capacity) n_valid[bh] = n + 1;      // (behind the barriers: the waves that append have read it)
  }
}

template <int DT, int D, int FORMAT>
hipError_t launch_as(const DecodeShape &s, const void *q, const void *kn, const void *vn, void *kc, void *ks, void *vc, void *vs, int32_t *n_valid, float *out,
                     float *part, hipStream_t stream) {
  const dim3 grid(s.B * s.Hkv, s.n_splits);
  // what exceeds the memory-side cache is not found there at the next token
  const bool streams = 2 * (int64_t)s.B * s.Hkv * s.capacity * (code_bytes<FORMAT>(D) + D / SCALE_GROUP) > MEMORY_CACHE_BYTES;
#define WKV_DQ(COLUMNS, STREAM) \
  hipLaunchKernelGGL((decode_quantized_kernel<DT, D, FORMAT, COLUMNS, STREAM>), grid, dim3(DQ_THREADS), 0, stream, s, (const char *)q, (const char *)kc, \
                     (const uint8_t *)ks, (const char *)vc, (const uint8_t *)vs, n_valid, part)
  if (s.G <= 4) { if (streams) WKV_DQ(4, true); else WKV_DQ(4, false); }
  else { if (streams) WKV_DQ(8, true); else WKV_DQ(8, false); }
#undef WKV_DQ
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  static_assert(DEC_MAX_SPLITS <= DQ_THREADS, "one thread per range");
  hipLaunchKernelGGL((merge_quantized_kernel<DT, D, FORMAT>), dim3(s.B * s.Hkv, s.G), dim3(DQ_THREADS), 0, stream, s, (const char *)q, (const char *)kn,
                     (const char *)vn, (char *)kc, (uint8_t *)ks, (char *)vc, (uint8_t *)vs, part, n_valid, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_quantized(const DecodeShape &s, int32_t format, const void *q_new, const void *k_new, const void *v_new, void *k_codes,
                                   void *k_scales, void *v_codes, void *v_scales, int32_t *n_valid, float *out, float *part, hipStream_t stream) {
#define WKV_DQ_AS(DT, D, FORMAT) return launch_as<DT, D, FORMAT>(s, q_new, k_new, v_new, k_codes, k_scales, v_codes, v_scales, n_valid, out, part, stream)
#define WKV_DQ_TYPE(DT) \
  if (format == E4M3) { if (s.d == 128) WKV_DQ_AS(DT, 128, E4M3); else WKV_DQ_AS(DT, 64, E4M3); } \
  else { if (s.d == 128) WKV_DQ_AS(DT, 128, E2M1); else WKV_DQ_AS(DT, 64, E2M1); }
  if (s.dtype == WKV_BF16) { WKV_DQ_TYPE(DT_BF16) }
  if (s.dtype == WKV_F16) { WKV_DQ_TYPE(DT_F16) }
  WKV_DQ_TYPE(DT_F32)
#undef WKV_DQ_TYPE
#undef WKV_DQ_AS
}

}  // namespace wkv
