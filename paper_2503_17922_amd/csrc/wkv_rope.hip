// Rotary positions: pairs of channels of queries and keys turned by position * inv_freq.
//
// Two floats in, two out, four multiplications: bound by memory, which every element crosses once each way.  The angle is kept as a
// fraction of a turn in 64-bit fixed point (position * turns modulo 2^64 is one integer product, exact however far the position), whose
// top 32 bits become the argument of sincospi; a thread takes eight pairs of a token and turns them in up to five heads at
// once, all loads ahead of the sines and of the first store.  32768 tokens of 32q/8kv heads, 128 channels, bf16: 130 us head by head,
// 123 so, 120 (5.6 TB/s) with the sines behind the loads.  With 1, 4 or 32 heads of a token side by side instead of 8 10 to 40 us more.
// How many heads a thread takes at once matters little from four on, whatever their number.  us with 1 / 3 / 4 / 5 / 6 / 8: 32 + 8 heads 144 / 121 / 119 / 118 / 118 / 119, 64 + 8 249 / 229 /
// 227 / 225 / 224 / 223, 28 + 4 116 / 101 / 100 / 100 / 100 / 100, 12 + 2 57 / 45 / 44 / 44 / 46 / 45, 32 + 32 219 / 196 / 192 / 198 / 192 / 190; 4096 tokens of 32 + 8
// 19.6 / 15.3 / 15.4 / 15.4 / 15.4 / 15.2.
#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

namespace {

constexpr int ROPE_THREADS = 256;

template <int DT> struct RopeElement;
template <> struct RopeElement<DT_BF16> { typedef __bf16 type; };
template <> struct RopeElement<DT_F16> { typedef _Float16 type; };
template <> struct RopeElement<DT_F32> { typedef float type; };

// Workgroup (x, y): tokens x * TOKENS .., heads in groups of HEADS from y * `groups` on.  A head's row is P pieces of 16 bytes, taken by
// LPH = d / 16 lanes, neighbouring pieces by neighbouring lanes: whole lines in every load and store (interleaved pairs by
// 32 neighbouring bytes a lane: three sequences, 17027 tokens, 28q/4kv heads, 64 of 128 channels 67.8 us, 62.6 so, 54.2
// with the sines behind the loads).
//   by halves     lane p takes slots p, p + LPH, ..: piece j and its partner rotary / 2 channels on, E pairs
//   interleaved   lane p takes pieces p, p + LPH, ..: E / 2 pairs each
// Pieces past the rotary channels are copied.
constexpr int HEADS = 8, ROPE_U = 5;
template <int DT, int D, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(RopeArgs a, int32_t groups) {
  typedef typename RopeElement<DT>::type T;
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  constexpr int E = 16 / sizeof(T), P = D / E, LPH = D / 16, N = P / LPH, TOKENS = ROPE_THREADS / LPH / HEADS;
  const int p = threadIdx.x % LPH, unit = threadIdx.x / LPH;
  const int64_t token = (int64_t)blockIdx.x * TOKENS + unit / HEADS;
  if (token >= (int64_t)a.batch * a.n_tokens) return;
  const int32_t pos = a.positions[token];
  if (pos < 0) return;
  const int32_t b = (int32_t)((uint32_t)token / (uint32_t)a.n_tokens), t = (int32_t)token - b * a.n_tokens;

  // this lane's pieces, two for every run of PAIRS angles
  constexpr int RUNS = INTERLEAVED ? N : N / 2, PAIRS = 8 / RUNS;
  int at[N];
  bool turns[RUNS];
  float c[RUNS][PAIRS], s[RUNS][PAIRS];
  const int turned = a.rotary / E;               // pieces that turn
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    const int j = p + k * LPH;
    if constexpr (INTERLEAVED) {
      at[k] = j * 16;
      turns[k] = j < turned;
    } else {
      turns[k] = j < turned / 2;
      at[2 * k] = (turns[k] ? j : j + turned / 2) * 16;
      at[2 * k + 1] = at[2 * k] + (turns[k] ? turned / 2 : P / 2 - turned / 2) * 16;
    }
  }
  const int heads = min(a.q_heads + a.kv_heads, (int)(blockIdx.y + 1) * groups * HEADS);
  int first = blockIdx.y * groups * HEADS + unit % HEADS;
  vec v[ROPE_U][N];
  char *to[ROPE_U];
  auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < ROPE_U; ++u) {
      const int head = first + u * HEADS;
      if (head >= heads) break;
      const bool is_q = head < a.q_heads;
      const RopeTensor &x = is_q ? a.q : a.k;
      const int64_t h = is_q ? head : head - a.q_heads;
      const char *in = (const char *)x.in + b * x.in_b + h * x.in_h + t * x.in_t;
      to[u] = (char *)x.out + b * x.out_b + h * x.out_h + t * x.out_t;
#pragma unroll
      for (int i = 0; i < N; ++i) v[u][i] = *(const vec *)(in + at[i]);
    }
  };
  load();
  // (while the first rows are under way)
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
    if (turns[k]) {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const int32_t part = (int32_t)(uint32_t)((uint64_t)(uint32_t)pos * a.turns[(p + k * LPH) * PAIRS + i] >> 32);      // signed: -1/2 .. 1/2 turn
        sincospif((float)part * 0x1p-31f, &s[k][i], &c[k][i]);
        c[k][i] *= a.amplitude;
        s[k][i] *= a.inverse ? -a.amplitude : a.amplitude;
      }
    }
  for (;;) {
#pragma unroll
    for (int u = 0; u < ROPE_U; ++u) {
      if (first + u * HEADS >= heads) break;
#pragma unroll
      for (int k = 0; k < RUNS; ++k)
        if (turns[k]) {
#pragma unroll
          for (int i = 0; i < PAIRS; ++i) {
            T &e0 = ((T *)&v[u][INTERLEAVED ? k : 2 * k])[INTERLEAVED ? 2 * i : i], &e1 = ((T *)&v[u][INTERLEAVED ? k : 2 * k + 1])[INTERLEAVED ? 2 * i + 1 : i];
            const float x0 = (float)e0, x1 = (float)e1;
            e0 = (T)(x0 * c[k][i] - x1 * s[k][i]);
            e1 = (T)(x1 * c[k][i] + x0 * s[k][i]);
          }
        }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (STREAM) __builtin_nontemporal_store(v[u][i], (vec *)(to[u] + at[i]));
        else *(vec *)(to[u] + at[i]) = v[u][i];
      }
    }
    first += ROPE_U * HEADS;
    if (first >= heads) break;
    load();
  }
}

template <int DT, int D>
hipError_t launch_rope_d(const RopeArgs &a, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.batch * a.n_tokens;
  constexpr int TOKENS = ROPE_THREADS / (D / 16) / HEADS;
  const int64_t x = (tokens + TOKENS - 1) / TOKENS;
  const int32_t groups = (a.q_heads + a.kv_heads + HEADS - 1) / HEADS;
  // With few tokens a thread takes a single head, and the heads spread over the device.
  const bool few = x * groups <= 4096;
  const dim3 grid((uint32_t)x, (uint32_t)(few ? groups : 1));
  // What exceeds the memory-side cache is not found there by whoever reads it next.
  const bool streams = tokens * (a.q_heads + a.kv_heads) * D * elem_bytes(a.dtype) > MEMORY_CACHE_BYTES;
#define WKV_ROPE(INTERLEAVED, STREAM) \
  hipLaunchKernelGGL((rope_kernel<DT, D, INTERLEAVED, STREAM>), grid, dim3(ROPE_THREADS), 0, stream, a, few ? 1 : groups)
  if (a.interleaved) { if (streams) WKV_ROPE(true, true); else WKV_ROPE(true, false); }
  else { if (streams) WKV_ROPE(false, true); else WKV_ROPE(false, false); }
#undef WKV_ROPE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream) {
#define WKV_ROPE_TYPE(DT) return a.d == 128 ? launch_rope_d<DT, 128>(a, stream) : launch_rope_d<DT, 64>(a, stream)
  if (a.dtype == WKV_BF16) WKV_ROPE_TYPE(DT_BF16);
  if (a.dtype == WKV_F16) WKV_ROPE_TYPE(DT_F16);
  WKV_ROPE_TYPE(DT_F32);
#undef WKV_ROPE_TYPE
}

}  // namespace wkv
