// Eviction by accumulated attention weight: which rows of a (sequence, KV head) stay, and the moves that close the gaps.
//
//   select kernel   a workgroup per (sequence, KV head).  The keep-th largest of order-preserving keys by digits of the range they span, then
//                   walks in row order: every wave takes a range of rows, so the ranks of kept, dropped and equal rows need one
//                   scan over the waves and ballots inside them.  Kept rows from `keep` on move into the dropped places
//                   below it, the r-th into the r-th: sources and targets are disjoint, so the caches are compacted in
//                   place, and one row too many costs one row's copy instead of half a cache's.
//   move kernel     copies the rows of every layer's keys and values.
// The selection reads 8 bytes a row and is a chain of scans, bound by their latency (4097 rows: 20.6 us with the weights read anew in every
// step and fixed digits, 11.2 so); the copies by memory, in pieces of a row here and there (5 TB/s).
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

// Rows are dealt to the waves in ranges, in row order, a lane every 64th of its wave's range.  HELD: a thread keeps its weights and
// positions in registers (ranges of up to HELD * 64 rows); 0: they are read again in every step.
template <int HELD>
__device__ __forceinline__ void evict_rows(const EvictArgs &a, EvictLds &lds, int32_t *holes, int n, int stay, float *w, int32_t *tok, int2 *mv, int &n_moves) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per_wave = ((n + EV_WAVES - 1) / EV_WAVES + 63) / 64 * 64;
  const int from = min(wave * per_wave, n), to = min(from + per_wave, n), iters = (to - from + 63) / 64;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  constexpr int N = HELD ? HELD : 1;
  float own_w[N];
  int32_t own_tok[N];
  if constexpr (HELD > 0) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) { const int j = min(from + i * 64 + lane, n - 1); own_w[i] = w[j]; own_tok[i] = tok[j]; }
  }
  // f(i, row, is a row, its weight, its position) for every row of the thread, all lanes of a wave together
  auto each = [&](auto &&f) __attribute__((always_inline)) {
    if constexpr (HELD > 0) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i < iters) f(i, from + i * 64 + lane, from + i * 64 + lane < to, own_w[i], own_tok[i]);
    } else {
      for (int i = 0; i < iters; ++i) {
        const int j = from + i * 64 + lane, at = min(j, n - 1);
        f(i, j, j < to, w[at], tok[at]);
      }
    }
  };

  // ---- 1. the last position; rows within `recent` of it are protected
  uint32_t last = 0;
  each([&](int, int, bool in, float, int32_t t) { last = max(last, in ? (uint32_t)t ^ 0x80000000u : 0u); });      // signed order to unsigned
  last = wave_largest(last);
  if (lane == 0) lds.waves[0][wave] = last;
  for (int i = tid; i < EV_BINS; i += EV_THREADS) lds.bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) last = max(last, lds.waves[0][i]);
  const int64_t old = (int64_t)(int32_t)(last ^ 0x80000000u) - a.recent;        // positions up to this one are not protected

  // ---- 2. how many are, and the range of the weights of either kind
  uint32_t fresh = 0, least[2] = {0xffffffffu, 0xffffffffu}, most[2] = {0, 0};
  each([&](int, int, bool in, float x, int32_t t) {
    const bool f = t > old;
    const uint32_t key = weight_key(x);
    fresh += __builtin_popcountll(__ballot(in && f));
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (in && f == (c == 1)) { least[c] = min(least[c], key); most[c] = max(most[c], key); }
  });
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t lo = ~wave_largest(~least[c]), hi = wave_largest(most[c]);
    if (lane == 0) { lds.waves[1 + 2 * c][wave] = lo; lds.waves[2 + 2 * c][wave] = hi; }
  }
  uint32_t n_fresh;
  before_this_wave(fresh, lds.waves[5], wave, n_fresh);
  // Protected rows come first; where they do not all fit, they alone are selected from, by weight.
  const bool crowded = (int)n_fresh > stay;
  uint32_t remaining = crowded ? stay : stay - n_fresh;                  // of the rows that are selected from
  uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) { lo = min(lo, lds.waves[crowded ? 3 : 1][i]); hi = max(hi, lds.waves[crowded ? 4 : 2][i]); }

  // ---- 3. the key of the last row that stays, by digits of the range that the keys span (digits from the top of the word would put nearly
  // all weights into a few bins and serialise the counters); until what still fits is a whole bin or a bin is one key wide
  uint32_t bound = 0xffffffffu, take_eq = 0;           // keys above `bound` stay, and the first take_eq rows that have it
  while (remaining > 0) {
    const int bits = 32 - __clz((int)((hi - lo) | 1u)), shift = max(bits - 11, 0);
    each([&](int, int, bool in, float x, int32_t t) {
      const uint32_t key = weight_key(x);
      if (in && (t > old) == crowded && key >= lo && key <= hi) atomicAdd(&lds.bins[(key - lo) >> shift], 1u);
    });
    __syncthreads();
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
    if (shift == 0) { bound = bin_lo; take_eq = remaining; break; }
    if (lds.count == remaining) { bound = bin_lo - 1; break; }           // (bin_lo > 0: 0 is no weight's key)
    hi = bin_lo + min((1u << shift) - 1u, hi - bin_lo);
    lo = bin_lo;
  }

  // ---- 4. dropped rows below `stay`, and kept rows from there on: their numbers, then their ranks
  uint32_t rank = 0, all;
  auto keeps = [&](bool in, float x, int32_t t) __attribute__((always_inline)) {
    const bool f = t > old;
    const uint32_t key = weight_key(x);
    bool kept = in && (f != crowded ? f : key > bound);
    if (take_eq > 0) {                                 // (uniform)
      const uint64_t same = __ballot(in && f == crowded && key == bound);
      kept |= (same >> lane & 1) && rank + __builtin_popcountll(same & below) < take_eq;
      rank += __builtin_popcountll(same);
    }
    return kept;
  };
  uint32_t equal_before = 0;
  if (take_eq > 0) {
    uint32_t equal = 0;
    each([&](int, int, bool in, float x, int32_t t) { equal += __builtin_popcountll(__ballot(in && (t > old) == crowded && weight_key(x) == bound)); });
    equal_before = before_this_wave(equal, lds.waves[7], wave, all);
  }
  rank = equal_before;
  uint32_t n_holes = 0, n_late = 0;
  each([&](int, int j, bool in, float x, int32_t t) {
    const bool kept = keeps(in, x, t);
    n_holes += __builtin_popcountll(__ballot(in && !kept && j < stay));
    n_late += __builtin_popcountll(__ballot(kept && j >= stay));
  });
  uint32_t hole = before_this_wave(n_holes, lds.waves[0], wave, all), late = before_this_wave(n_late, lds.waves[1], wave, all);
  n_moves = (int)all;
  rank = equal_before;
  each([&](int, int j, bool in, float x, int32_t t) {
    const uint64_t open = __ballot(in && !keeps(in, x, t) && j < stay);
    if (open >> lane & 1) {
      const uint32_t r = hole + __builtin_popcountll(open & below);
      if (HELD) holes[r] = j; else mv[r].y = j;
    }
    hole += __builtin_popcountll(open);
  });
  __syncthreads();
  rank = equal_before;
  each([&](int, int j, bool in, float x, int32_t t) {
    const uint64_t comes = __ballot(keeps(in, x, t) && j >= stay);
    if (comes >> lane & 1) {
      const uint32_t r = late + __builtin_popcountll(comes & below);
      const int32_t dst = HELD ? holes[r] : mv[r].y;
      mv[r] = make_int2(j, dst);
      if (HELD) { w[dst] = x; tok[dst] = t; }
    }
    late += __builtin_popcountll(comes);
  });
  if constexpr (HELD == 0) {                           // (nobody reads the rows below `stay` any more)
    __syncthreads();
    for (int i = tid; i < n_moves; i += EV_THREADS) {
      const int2 m = mv[i];
      w[m.y] = w[m.x];
      tok[m.y] = tok[m.x];
    }
  }
}

// HELD * 1024 rows or fewer (LONG: where there are more, their weights are read in every step).
template <int HELD, bool LONG>
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a, float *weights, int32_t *tok_idx, int32_t *n_valid,
                                                                  const int32_t *__restrict__ keep, int32_t *__restrict__ counts,
                                                                  int2 *__restrict__ moves) {
  __shared__ EvictLds lds;
  __shared__ int32_t holes[HELD * EV_THREADS / 2];     // at most min(stay, n - stay)
  const int row = blockIdx.x, n = n_valid[row], stay = keep[row];
  int n_moves = 0;
  if (stay >= 0 && n <= a.capacity && n > stay) {
    float *w = weights + (int64_t)row * a.capacity;
    int32_t *tok = tok_idx + (int64_t)row * a.capacity;
    int2 *mv = moves + (int64_t)row * a.max_moves;
    if (!LONG || n <= HELD * EV_THREADS) evict_rows<HELD>(a, lds, holes, n, stay, w, tok, mv, n_moves);
    else if constexpr (LONG) evict_rows<0>(a, lds, holes, n, stay, w, tok, mv, n_moves);
    __syncthreads();                       // (every thread has read the count)
    if (threadIdx.x == 0) n_valid[row] = stay;
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
#define WKV_SELECT(HELD, LONG) \
  hipLaunchKernelGGL((evict_select_kernel<HELD, LONG>), dim3(a.rows), dim3(EV_THREADS), 0, stream, a, weights, tok_idx, n_valid, keep, counts, moves)
  if (a.capacity <= 2 * EV_THREADS) WKV_SELECT(2, false);
  else if (a.capacity <= 5 * EV_THREADS) WKV_SELECT(5, false);
  else WKV_SELECT(12, true);
#undef WKV_SELECT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Workgroups for as many moves as there can be, one round of a thread's each: how many there are is on the device, and a workgroup without any
  // costs little (eight sequences, 4 layers, 236 MB to move: 66.0 us; with a quarter of them, four rounds each, 69.2; moves two at a time
  // 66.5).  Nontemporal: plain stores leave their write-back to the next kernel (71.6).
  const int lpr = a.row_bytes / 16, rows_at_once = MOVE_THREADS / lpr;
  const int64_t most = (a.max_moves + MOVE_AHEAD * rows_at_once - 1) / (MOVE_AHEAD * rows_at_once), pairs = (int64_t)a.rows * n_layers * 2;
  const int64_t want = std::min(most, std::max<int64_t>(65536 / pairs, 1));
  const dim3 grid((uint32_t)want, a.rows, n_layers * 2);
#define WKV_MOVE(LPR) hipLaunchKernelGGL((evict_move_kernel<LPR>), grid, dim3(MOVE_THREADS), 0, stream, a, layers, counts, moves)
  if (lpr == 8) WKV_MOVE(8);
  else if (lpr == 16) WKV_MOVE(16);
  else WKV_MOVE(32);
#undef WKV_MOVE
  return hipGetLastError();
}

}  // namespace wkv
