// Eviction by accumulated attention weight: which rows of a (sequence, KV head) stay, and the moves that close the gaps.
//
//   select kernel   a workgroup per (sequence, KV head).  The keep-th largest of order-preserving keys by digits (11, 11 and 10
//                   bits), then one walk in row order: every wave takes a range of rows, so the ranks of kept, dropped and equal
//                   rows need one scan over the waves and ballots inside them.  Kept rows from `keep` on move into the
//                   dropped places below it, the r-th into the r-th: sources and targets are disjoint, so the caches are
//                   compacted in place, and one row too many costs one row's copy instead of half a cache's.
//   move kernel     copies the rows of every layer's keys and values.
// The selection reads 8 bytes a row and is a chain of scans, bound by their latency; the copies by memory.
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
  __syncthreads();
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

__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a, float *weights, int32_t *tok_idx, int32_t *n_valid,
                                                                  const int32_t *__restrict__ keep, int32_t *__restrict__ counts,
                                                                  int2 *__restrict__ moves) {
  __shared__ uint32_t bins[EV_BINS];
  __shared__ uint32_t waves_s[EV_WAVES];
  __shared__ uint32_t found[2];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = n_valid[row], stay = keep[row];
  if (stay < 0 || n < 0 || n > a.capacity || n <= stay) {
    if (tid == 0) counts[row] = 0;
    return;
  }
  float *w = weights + (int64_t)row * a.capacity;
  int32_t *tok = tok_idx + (int64_t)row * a.capacity;
  int2 *mv = moves + (int64_t)row * a.max_moves;

  // rows of this wave: [from, to), 64 at a time
  const int per_wave = ((n + EV_WAVES - 1) / EV_WAVES + 63) / 64 * 64;
  const int from = min(wave * per_wave, n), to = min(from + per_wave, n);

  // the last position
  int32_t last = INT32_MIN;
  for (int j = from + lane; j < to; j += 64) last = max(last, tok[j]);
  // (as keys of the scan: signed order to unsigned order)
  const uint32_t wave_last = wave_largest((uint32_t)last ^ 0x80000000u);
  if (lane == 0) waves_s[wave] = wave_last;
  __syncthreads();
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < EV_WAVES; ++i) top = max(top, waves_s[i]);
  const int64_t old = (int64_t)(int32_t)(top ^ 0x80000000u) - a.recent;        // positions up to this one are not protected
  // Protected rows come first; where they do not all fit, they alone are selected from, by weight.
  uint32_t fresh = 0, n_fresh;
  for (int j0 = from; j0 < to; j0 += 64) fresh += __builtin_popcountll(__ballot(j0 + lane < to && (int64_t)tok[j0 + lane] > old));
  before_this_wave(fresh, waves_s, wave, n_fresh);
  const bool crowded = (int)n_fresh > stay;
  auto key_of = [&](int j) __attribute__((always_inline)) {
    const bool is_fresh = (int64_t)tok[j] > old;
    return is_fresh != crowded ? (is_fresh ? 0xffffffffu : 0u) : weight_key(w[j]);
  };

  // ---- the stay-th largest key, digit by digit; `left`: how many of the rows that share the digits so far stay
  uint32_t prefix = 0, mask = 0;
  int left = stay;
  constexpr int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
  if (stay > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = shifts[pass], n_bins = 1 << widths[pass];
      for (int i = tid; i < EV_BINS; i += EV_THREADS) bins[i] = 0;
      __syncthreads();
      for (int j = from + lane; j < to; j += 64) {
        const uint32_t key = key_of(j);
        if ((key & mask) == prefix) atomicAdd(&bins[key >> shift & (n_bins - 1)], 1u);
      }
      __syncthreads();
      // two bins a thread, the largest digit first
      const int b0 = EV_BINS - 1 - 2 * tid;
      const uint32_t c0 = bins[b0], c1 = bins[b0 - 1], mine = c0 + c1;
      const uint32_t upto = wave_sums(mine);
      uint32_t all;
      const uint32_t before = before_this_wave(last_lane(upto), waves_s, wave, all) + upto - mine;
      if ((int)before < left && left <= (int)(before + mine)) {
        const bool second = (int)(before + c0) < left;
        found[0] = second ? b0 - 1 : b0;
        found[1] = left - before - (second ? c0 : 0);
      }
      __syncthreads();
      prefix |= found[0] << shift;
      left = (int)found[1];
      mask |= (uint32_t)(n_bins - 1) << shift;
    }
  }
  const uint32_t bound = stay > 0 ? prefix : 0xffffffffu;      // of rows with exactly this key the first `left` stay
  if (stay == 0) left = 0;

  // ---- ranks of the rows with that key, then of the dropped rows below `stay` and of the kept rows from there on
  uint32_t equal = 0, all;
  for (int j0 = from; j0 < to; j0 += 64) equal += __builtin_popcountll(__ballot(j0 + lane < to && key_of(j0 + lane) == bound));
  const uint32_t equal_before = before_this_wave(equal, waves_s, wave, all);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  auto walk = [&](uint32_t holes, uint32_t late, bool emit) __attribute__((always_inline)) {
    uint32_t rank = equal_before;
    for (int j0 = from; j0 < to; j0 += 64) {
      const int j = j0 + lane;
      const uint32_t key = j < to ? key_of(j) : 0u;
      const uint64_t same = __ballot(j < to && key == bound);
      const bool kept = j < to && (key > bound || (key == bound && (int)(rank + __builtin_popcountll(same & below)) < left));
      rank += __builtin_popcountll(same);
      const bool hole = j < to && j < stay && !kept, comes = j >= stay && kept;
      const uint64_t hole_b = __ballot(hole), comes_b = __ballot(comes);
      if (emit) {
        if (hole) mv[holes + __builtin_popcountll(hole_b & below)].y = j;
        if (comes) mv[late + __builtin_popcountll(comes_b & below)].x = j;
      }
      holes += __builtin_popcountll(hole_b);
      late += __builtin_popcountll(comes_b);
    }
    return make_uint2(holes, late);
  };
  const uint2 mine = walk(0, 0, false);
  uint32_t n_moves;
  const uint32_t holes_before = before_this_wave(mine.x, waves_s, wave, n_moves);
  const uint32_t late_before = before_this_wave(mine.y, waves_s, wave, all);
  walk(holes_before, late_before, true);
  __syncthreads();
  for (int i = tid; i < (int)n_moves; i += EV_THREADS) {
    const int2 m = mv[i];
    w[m.y] = w[m.x];
    tok[m.y] = tok[m.x];
  }
  if (tid == 0) { counts[row] = (int)n_moves; n_valid[row] = stay; }
}

// Workgroups over the moves of a (sequence, KV head), of every tensor.
constexpr int MOVE_THREADS = 256;
template <int LPR>                      // lanes of 16 bytes to a row
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictArgs a, EvictLayers layers, const int32_t *__restrict__ counts,
                                                                  const int2 *__restrict__ moves) {
  constexpr int ROWS = MOVE_THREADS / LPR, AHEAD = 4;
  const int row = blockIdx.y, n = counts[row];
  int i = blockIdx.x * ROWS + threadIdx.x / LPR;
  if (blockIdx.x * ROWS >= n) return;
  const int b = divide((uint32_t)row, a.hkv_magic), h = row - b * a.Hkv;
  char *base = (char *)(blockIdx.z & 1 ? layers.v[blockIdx.z >> 1] : layers.k[blockIdx.z >> 1]) + (b * a.sb + h * a.sh + threadIdx.x % LPR * 16);
  const int2 *mv = moves + (int64_t)row * a.max_moves;
  const int step = gridDim.x * ROWS;
  for (; i < n; i += AHEAD * step) {
    int2 m[AHEAD];
    uint4 x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) m[u] = mv[min((int64_t)i + (int64_t)u * step, (int64_t)n - 1)];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = *(const uint4 *)(base + m[u].x * a.st);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) *(uint4 *)(base + m[u].y * a.st) = x[u];        // (past the end: the last move again)
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, const EvictLayers &layers, int32_t n_layers, float *weights, int32_t *tok_idx, int32_t *n_valid,
                        const int32_t *keep, int32_t *counts, int2 *moves, hipStream_t stream) {
  hipLaunchKernelGGL(evict_select_kernel, dim3(a.rows), dim3(EV_THREADS), 0, stream, a, weights, tok_idx, n_valid, keep, counts, moves);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int lpr = a.row_bytes / 16, rows_at_once = MOVE_THREADS / lpr;
  const int64_t most = (a.max_moves + rows_at_once - 1) / rows_at_once, want = 4096 / ((int64_t)a.rows * n_layers * 2);
  const dim3 grid((uint32_t)(want < 1 ? 1 : want < most ? want : most), a.rows, n_layers * 2);
#define WKV_MOVE(LPR) hipLaunchKernelGGL((evict_move_kernel<LPR>), grid, dim3(MOVE_THREADS), 0, stream, a, layers, counts, moves)
  if (lpr == 8) WKV_MOVE(8);
  else if (lpr == 16) WKV_MOVE(16);
  else WKV_MOVE(32);
#undef WKV_MOVE
  return hipGetLastError();
}

}  // namespace wkv
