// Eviction by accumulated attention weight: which rows of a (sequence, KV head) stay, and the moves that close the gaps.
//
//   select kernel   a workgroup per (sequence, KV head).  The keep-th largest of order-preserving keys by digits of the range they span, then
//                   walks in row order: every wave takes a range of rows, so the ranks of kept, dropped and equal rows need one
//                   scan over the waves and ballots inside them.  Kept rows from `keep` on move into the dropped places
//                   below it, the r-th into the r-th: sources and targets are disjoint, so the caches are compacted in
//                   place, and one row too many costs one row's copy instead of half a cache's.
//   move kernel     copies the rows of every layer's keys and values.
// The selection reads 8 bytes a row and is a chain of scans, bound by their latency (4097 rows: 20.6 us with the weights read anew in every
// step and fixed digits, 9 to 10 so); the copies by memory, in pieces of a row here and there (5 TB/s).
#include <algorithm>

#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

namespace {

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64;
constexpr int EV_BINS = 2048;

// Larger weight, larger key; NaN below every number, both zeros the same.  0 and the greatest key are no weight's.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 1u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Sum of `x` over the waves before this one, and over all (x uniform within a wave).
__device__ __forceinline__ uint32_t before_this_wave(uint32_t x, uint32_t *waves_s, int wave, uint32_t &all) {
  if ((threadIdx.x & 63) == 0) waves_s[wave] = x;
  __syncthreads();
  uint32_t sum = 0, before = 0;
#pragma unroll
  for (int w = 0; w < EV_WAVES; ++w) {
    before += w < wave ? waves_s[w] : 0u;
    sum += waves_s[w];
  }
  all = sum;
  return before;
}

struct EvictLds {
  uint32_t bins[EV_BINS];
  uint32_t waves[8][EV_WAVES];              // one array a reduction: no second synchronisation before the next
  uint32_t bin, above, count;
};

// The key of the last row that stays, by digits of the range [lo, hi] that the keys span (digits from the top of the word would put nearly
// all weights into a few bins and serialise the counters); until what still fits is a whole bin or a bin is one key wide.  count(lo, hi, shift): adds up
// the rows with keys from lo to hi in bins, (key - lo) >> shift.  `counted`: that has been done for the first range.
struct Bound {
  uint32_t key, take_eq;                    // keys above it stay, and the first take_eq rows that have it
};
__device__ __forceinline__ int digit_shift(uint32_t lo, uint32_t hi) { return max(32 - __clz((int)((hi - lo) | 1u)) - 11, 0); }
template <class F>
__device__ __forceinline__ Bound last_that_stays(EvictLds &lds, uint32_t remaining, uint32_t lo, uint32_t hi, bool counted, F &&count) {
  const int tid = threadIdx.x, wave = tid >> 6;
  while (remaining > 0) {
    const int shift = digit_shift(lo, hi);
    if (!counted) {
      count(lo, hi, shift);
      __syncthreads();
    }
    counted = false;
    const int b0 = EV_BINS - 1 - 2 * tid;              // two bins a thread, the largest digit first
    const uint32_t c0 = lds.bins[b0], c1 = lds.bins[b0 - 1], upto = wave_sums(c0 + c1);
    uint32_t all, above = before_this_wave(last_lane(upto), lds.waves[6], wave, all) + upto - c0 - c1;
    if (above < remaining && above + c0 >= remaining) { lds.bin = b0; lds.above = above; lds.count = c0; }
    above += c0;
    if (above < remaining && above + c1 >= remaining) { lds.bin = b0 - 1; lds.above = above; lds.count = c1; }
    lds.bins[b0] = 0; lds.bins[b0 - 1] = 0;
    __syncthreads();
    remaining -= lds.above;
    const uint32_t bin_lo = lo + (lds.bin << shift);
    if (shift == 0) return {bin_lo, remaining};
    if (lds.count == remaining) return {bin_lo - 1, 0};           // (bin_lo > 0: 0 is no weight's key)
    hi = bin_lo + min((1u << shift) - 1u, hi - bin_lo);
    lo = bin_lo;
  }
  return {0xfffffffeu, 0};                             // only the rows that are not selected from
}

// Keys of rows that always stay (protected ones, where they all fit) and that never do (the others, where not).
constexpr uint32_t ALWAYS = 0xffffffffu, NEVER = 0u;

// Rows are dealt to the waves in ranges, in row order, a lane every 64th of its wave's range.  A bit a turn tells which of a thread's rows stay.
struct Range {
  int from, to, turns;
  __device__ __forceinline__ Range(int n, int wave) {
    const int per_wave = ((n + EV_WAVES - 1) / EV_WAVES + 63) / 64 * 64;
    from = min(wave * per_wave, n); to = min(from + per_wave, n); turns = (to - from + 63) / 64;
  }
};

// Up to ROWS rows: their keys lie in LDS.  (In registers, a thread's rows unrolled, the code is four times as long, and a launch fetches it anew: 4097 rows
// 11.2 us, 9.9 so.)
template <int ROWS>
__device__ __forceinline__ int evict_rows(const EvictArgs &a, EvictLds &lds, uint32_t *keys, int32_t *toks, int n, int stay, float *w, int32_t *tok, int2 *mv) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Range r(n, wave);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  constexpr int AHEAD = 4;

  // ---- 1. the last position, whose `recent` rows are protected, and the range of the weights
  uint32_t last = 0, lo = 0xffffffffu, hi = 0;
  for (int i = 0; i < r.turns; i += AHEAD) {
    float x[AHEAD];
    int32_t t[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) { const int j = min(r.from + (i + u) * 64 + lane, r.to - 1); x[u] = w[j]; t[u] = tok[j]; }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {                  // (past the end: the last row again)
      const int j = min(r.from + (i + u) * 64 + lane, r.to - 1);
      const uint32_t key = weight_key(x[u]);
      keys[j] = key; toks[j] = t[u];
      last = max(last, (uint32_t)t[u] ^ 0x80000000u);               // signed order to unsigned
      lo = min(lo, key); hi = max(hi, key);
    }
  }
  last = wave_largest(last); lo = ~wave_largest(~lo); hi = wave_largest(hi);
  if (lane == 0) { lds.waves[0][wave] = last; lds.waves[1][wave] = lo; lds.waves[2][wave] = hi; }
  for (int i = tid; i < EV_BINS; i += EV_THREADS) lds.bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) { last = max(last, lds.waves[0][i]); lo = min(lo, lds.waves[1][i]); hi = max(hi, lds.waves[2][i]); }
  const int64_t old = (int64_t)(int32_t)(last ^ 0x80000000u) - a.recent;        // positions up to this one are not protected

  // ---- 2. the protected rows, and the first digit of the others
  uint32_t fresh = 0, n_fresh;
  const int shift = digit_shift(lo, hi);
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    const bool in = j < r.to, f = in && toks[j] > old;
    fresh += __builtin_popcountll(__ballot(f));
    if (f) keys[j] = ALWAYS;
    else if (in) atomicAdd(&lds.bins[(keys[j] - lo) >> shift], 1u);
  }
  before_this_wave(fresh, lds.waves[3], wave, n_fresh);
  const bool crowded = (int)n_fresh > stay;
  if (crowded) {                             // they do not all fit: they alone are selected from, by weight
    for (int i = tid; i < EV_BINS; i += EV_THREADS) lds.bins[i] = 0;
    __syncthreads();
    for (int j = r.from + lane; j < r.to; j += 64) {
      const uint32_t key = toks[j] > old ? weight_key(w[j]) : NEVER;
      keys[j] = key;
      if (key != NEVER) atomicAdd(&lds.bins[(key - lo) >> shift], 1u);
    }
    __syncthreads();
  }
  const Bound bound = last_that_stays(lds, crowded ? stay : stay - n_fresh, lo, hi, true, [&](uint32_t lo, uint32_t hi, int shift) {
    for (int j = r.from + lane; j < r.to; j += 64)
      if (keys[j] >= lo && keys[j] <= hi) atomicAdd(&lds.bins[(keys[j] - lo) >> shift], 1u);
  });

  // ---- 3. which rows stay; dropped ones below `stay` and kept ones from there on: their numbers, then their ranks
  uint32_t stays = 0, rank = 0, n_holes = 0, n_late = 0, all;
  if (bound.take_eq > 0) {
    uint32_t equal = 0;
    for (int i = 0; i < r.turns; ++i) {
      const int j = r.from + i * 64 + lane;
      equal += __builtin_popcountll(__ballot(j < r.to && keys[j] == bound.key));
    }
    rank = before_this_wave(equal, lds.waves[4], wave, all);
  }
  static_assert(ROWS <= 32 * EV_THREADS, "a bit a turn");
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    const bool in = j < r.to;
    const uint32_t key = in ? keys[j] : NEVER;
    bool kept = key > bound.key;
    if (bound.take_eq > 0) {                           // (uniform)
      const uint64_t same = __ballot(in && key == bound.key);
      kept |= (same >> lane & 1) && rank + __builtin_popcountll(same & below) < bound.take_eq;
      rank += __builtin_popcountll(same);
    }
    stays |= (uint32_t)kept << i;
    n_holes += __builtin_popcountll(__ballot(in && !kept && j < stay));
    n_late += __builtin_popcountll(__ballot(kept && j >= stay));
  }
  if (lane == 0) lds.waves[5][wave] = n_late;
  uint32_t hole = before_this_wave(n_holes, lds.waves[7], wave, all), late = 0;
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) late += i < wave ? lds.waves[5][i] : 0u;
  int32_t *holes = toks;                     // (nobody looks at the positions any more)
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    const uint64_t open = __ballot(j < min(r.to, stay) && !(stays >> i & 1));
    if (open >> lane & 1) holes[hole + __builtin_popcountll(open & below)] = j;
    hole += __builtin_popcountll(open);
  }
  __syncthreads();
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    const uint64_t comes = __ballot(j >= stay && (stays >> i & 1));
    if (comes >> lane & 1) {
      const int at = late + __builtin_popcountll(comes & below), to = holes[at];
      mv[at] = make_int2(j, to);
      w[to] = w[j];
      tok[to] = tok[j];
    }
    late += __builtin_popcountll(comes);
  }
  return (int)all;
}

// Any number of rows: the same steps, with the weights read in each, and the first digit over all keys.  (What fits LDS goes the way above: eight sequences of 8 heads,
// 2 layers, a tenth of 16384 rows dropped 64 us the call, of 32768 222, so; two of 131072 456.)
__device__ __forceinline__ int evict_long(const EvictArgs &a, EvictLds &lds, int n, int stay, float *w, int32_t *tok, int2 *mv) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Range r(n, wave);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  uint32_t last = 0, all;
  for (int j = r.from + lane; j < r.to; j += 64) last = max(last, (uint32_t)tok[j] ^ 0x80000000u);
  last = wave_largest(last);
  if (lane == 0) lds.waves[0][wave] = last;
  for (int i = tid; i < EV_BINS; i += EV_THREADS) lds.bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) last = max(last, lds.waves[0][i]);
  const int64_t old = (int64_t)(int32_t)(last ^ 0x80000000u) - a.recent;
  uint32_t fresh = 0, n_fresh;
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    fresh += __builtin_popcountll(__ballot(j < r.to && tok[j] > old));
  }
  before_this_wave(fresh, lds.waves[3], wave, n_fresh);
  const bool crowded = (int)n_fresh > stay;
  auto key_of = [&](int j) __attribute__((always_inline)) {
    const bool f = tok[j] > old;
    return f != crowded ? (f ? ALWAYS : NEVER) : weight_key(w[j]);
  };
  const Bound bound = last_that_stays(lds, crowded ? stay : stay - n_fresh, 1u, 0xfffffffeu, false, [&](uint32_t lo, uint32_t hi, int shift) {
    for (int j = r.from + lane; j < r.to; j += 64) {
      const uint32_t key = key_of(j);
      if (key >= lo && key <= hi) atomicAdd(&lds.bins[(key - lo) >> shift], 1u);
    }
  });
  uint32_t equal = 0;
  for (int i = 0; i < r.turns; ++i) {
    const int j = r.from + i * 64 + lane;
    equal += __builtin_popcountll(__ballot(j < r.to && key_of(j) == bound.key));
  }
  const uint32_t equal_before = before_this_wave(equal, lds.waves[4], wave, all);
  auto walk = [&](uint32_t &holes, uint32_t &late, bool emit) __attribute__((always_inline)) {
    uint32_t rank = equal_before;
    for (int i = 0; i < r.turns; ++i) {
      const int j = r.from + i * 64 + lane;
      const bool in = j < r.to;
      const uint32_t key = in ? key_of(j) : NEVER;
      const uint64_t same = __ballot(in && key == bound.key);
      const bool kept = in && (key > bound.key || ((same >> lane & 1) && rank + __builtin_popcountll(same & below) < bound.take_eq));
      rank += __builtin_popcountll(same);
      const uint64_t open = __ballot(in && !kept && j < stay), comes = __ballot(kept && j >= stay);
      if (emit && (open >> lane & 1)) mv[holes + __builtin_popcountll(open & below)].y = j;
      if (emit && (comes >> lane & 1)) mv[late + __builtin_popcountll(comes & below)].x = j;
      holes += __builtin_popcountll(open);
      late += __builtin_popcountll(comes);
    }
  };
  uint32_t holes = 0, late = 0, n_moves;
  walk(holes, late, false);
  holes = before_this_wave(holes, lds.waves[5], wave, n_moves);
  late = before_this_wave(late, lds.waves[7], wave, all);
  walk(holes, late, true);
  __syncthreads();
  for (int i = tid; i < (int)n_moves; i += EV_THREADS) {
    const int2 m = mv[i];
    w[m.y] = w[m.x];
    tok[m.y] = tok[m.x];
  }
  return (int)n_moves;
}

// LONG: caches may have more than ROWS rows.
template <int ROWS, bool LONG>
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a, float *weights, int32_t *tok_idx, int32_t *n_valid,
                                                                  const int32_t *__restrict__ keep, int32_t *__restrict__ counts,
                                                                  int2 *__restrict__ moves) {
  __shared__ EvictLds lds;
  __shared__ uint32_t keys[ROWS];
  __shared__ int32_t toks[ROWS];
  const int row = blockIdx.x, n = n_valid[row], stay = keep[row];
  int n_moves = 0;
  if (stay >= 0 && n <= a.capacity && n > stay) {
    float *w = weights + (int64_t)row * a.capacity;
    int32_t *tok = tok_idx + (int64_t)row * a.capacity;
    int2 *mv = moves + (int64_t)row * a.max_moves;
    if (!LONG || n <= ROWS) n_moves = evict_rows<ROWS>(a, lds, keys, toks, n, stay, w, tok, mv);
    else n_moves = evict_long(a, lds, n, stay, w, tok, mv);
    if (threadIdx.x == 0) n_valid[row] = stay;         // (every thread has read it: there was a synchronisation since)
  }
  if (threadIdx.x == 0) counts[row] = n_moves;
}

// Workgroups over the moves of a (sequence, KV head), of every tensor.
constexpr int MOVE_THREADS = 256, MOVE_AHEAD = 8;      // of a thread at once
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int LPR>                      // lanes of 16 bytes to a row
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictArgs a, EvictLayers layers, const int32_t *__restrict__ counts,
                                                                  const int2 *__restrict__ moves) {
  constexpr int ROWS = MOVE_THREADS / LPR, AHEAD = MOVE_AHEAD;
  const int row = blockIdx.y, b = divide((uint32_t)row, a.hkv_magic), h = row - b * a.Hkv;
  const i32x2 *mv = (const i32x2 *)moves + (int64_t)row * a.max_moves;
  const int step = gridDim.x * ROWS;
  int i = blockIdx.x * ROWS + threadIdx.x / LPR;
  i32x2 m[AHEAD];
  auto request = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) m[u] = mv[min(i + u * step, a.max_moves - 1)];
  };
  request();                               // (together with their number; entries past it are not used)
  const int n = counts[row];
  char *base = (char *)(blockIdx.z & 1 ? layers.v[blockIdx.z >> 1] : layers.k[blockIdx.z >> 1]) + (b * a.sb + h * a.sh + threadIdx.x % LPR * 16);
  while (i < n) {
    u32x4 x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i + u * step < n) x[u] = __builtin_nontemporal_load((const u32x4 *)(base + m[u].x * a.st));
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i + u * step < n) __builtin_nontemporal_store(x[u], (u32x4 *)(base + m[u].y * a.st));
    i += AHEAD * step;
    if (i < n) request();
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, const EvictLayers &layers, int32_t n_layers, float *weights, int32_t *tok_idx, int32_t *n_valid,
                        const int32_t *keep, int32_t *counts, int2 *moves, hipStream_t stream) {
#define WKV_SELECT(ROWS, LONG) \
  hipLaunchKernelGGL((evict_select_kernel<ROWS, LONG>), dim3(a.rows), dim3(EV_THREADS), 0, stream, a, weights, tok_idx, n_valid, keep, counts, moves)
  if (a.capacity <= 6144) WKV_SELECT(6144, false);          // (two workgroups a compute unit)
  else WKV_SELECT(16384, true);
#undef WKV_SELECT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Workgroups for as many moves as there can be, one round of a thread's each: how many there are is on the device (eight sequences, 4 layers, 236 MB to move:
  // 66.0 us; with a quarter of them, four rounds each, 69.2; moves two at a time 66.5).  But not many more than the chip starts in some 6 us, since most calls of a serving
  // loop find little or nothing to move.  At most 65536 / 20480 / 8192 of them, us: nothing to drop, 64 sequences of 8 heads, 4 layers 18.9 / 11.9 / 6.8, 32 layers 31 / 17 / 17, 32
  // sequences 11.1 / 10.3 / 6.6; one row too many in each of 64 51.5 / 33 / 28.5; sixteen cut from 8192 rows to 4096 211 / 216 / 224; the eight sequences 63.8 / 63.8 / 66.
  // (16384, rows of all workgroups a power of two apart: 65; a workgroup's moves side by side instead of one of each stretch 70 to 102.)
  // Nontemporal: plain stores leave their write-back to the next kernel (71.6).
  const int lpr = a.row_bytes / 16, rows_at_once = MOVE_THREADS / lpr;
  const int64_t most = (a.max_moves + MOVE_AHEAD * rows_at_once - 1) / (MOVE_AHEAD * rows_at_once), pairs = (int64_t)a.rows * n_layers * 2;
  const int64_t want = std::min(most, std::max<int64_t>(20480 / pairs, 1));
  const dim3 grid((uint32_t)want, a.rows, n_layers * 2);
#define WKV_MOVE(LPR) hipLaunchKernelGGL((evict_move_kernel<LPR>), grid, dim3(MOVE_THREADS), 0, stream, a, layers, counts, moves)
  if (lpr == 8) WKV_MOVE(8);
  else if (lpr == 16) WKV_MOVE(16);
  else WKV_MOVE(32);
#undef WKV_MOVE
  return hipGetLastError();
}

}  // namespace wkv
