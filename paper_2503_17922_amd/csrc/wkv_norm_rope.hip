// Queries and keys normalised a head at a time and turned by their positions, of one axis or several.
//
//   y = x * w / sqrt(mean(x^2) + eps),   pairs of y turned by position[axis] * inv_freq   (computed in fp32, rounded once)
//
// Bound by memory, which every element crosses once each way.  The LPH = d / 16 lanes that hold a head's row add up its squares by DPP
// steps; a lane keeps the weights of its 16 channels, of queries and of keys, in registers.  Everything else (whole lines in every load and store, five heads
// of a token at once, fixed-point angles) is as for the rotation alone, wkv_rope.hip.
// bf16, 32q/8kv heads of 128 channels: 64 tokens 4.5 us, a launch; 32768 tokens 115 us = 5.8 TB/s.  f16, 28q/4kv, 17027 tokens of three axes, interleaved, 58 us = 4.8 TB/s.
// Fewer instructions (the root by the hardware's estimate, sine and cosine by a series of their own, weights selected in pairs) left all three times as they are.
#include "wkv_device.h"
#include "wkv_generation.h"

namespace wkv {

namespace {

constexpr int NR_THREADS = 256;
constexpr float TINY = 0x1p-100f;          // below it an eps is next to none

template <int DT> struct Element;
template <> struct Element<DT_BF16> { typedef __bf16 type; };
template <> struct Element<DT_F16> { typedef _Float16 type; };
template <> struct Element<DT_F32> { typedef float type; };

// Sum over the LPH (4 or 8) adjacent lanes of a head's row, in all of them.
template <int LPH>
__device__ __forceinline__ float lanes_sum(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false));  // quad_perm [1,0,3,2]
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false));  // quad_perm [2,3,0,1]
  if (LPH == 8)
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false)); // row_half_mirror
  return x;
}

// Workgroup (x, y): tokens x * TOKENS .., heads in groups of HEADS from y * `groups` on; which pieces of a row a lane takes is as in rope_kernel:
//   by halves     lane p takes slots p, p + LPH, ..: piece j and its partner rotary / 2 channels on, E pairs
//   interleaved   lane p takes pieces p, p + LPH, ..: E / 2 pairs each
// Pieces past the rotary channels are normalised alone.
// At once, two heads / five: the interleaved call above 57 / 62 us (96 and 134 registers), the one by halves of 32768 tokens 119 / 115.  In fp32 the same: interleaved with three axes (the call
// above) 100 / 104, by halves 32768 tokens 258 / 253 = 5.3 TB/s, 16000 tokens with three axes 121 / 117; but 6000 by halves 50 / 53.
constexpr int HEADS = 8;
// SMALL: a call with an eps below TINY.
template <int DT, int D, bool INTERLEAVED, bool AXES, bool STREAM, bool SMALL>
__global__ __launch_bounds__(NR_THREADS) void norm_rope_kernel(NormRopeArgs a, int32_t groups) {
  typedef typename Element<DT>::type T;
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  constexpr int AT_ONCE = INTERLEAVED ? 2 : 5;
  constexpr int E = 16 / sizeof(T), P = D / E, LPH = D / 16, N = P / LPH, TOKENS = NR_THREADS / LPH / HEADS;
  const int p = threadIdx.x % LPH, unit = threadIdx.x / LPH;
  const int64_t token = (int64_t)blockIdx.x * TOKENS + unit / HEADS;
  if (token >= (int64_t)a.batch * a.n_tokens) return;
  int32_t pos[AXES ? WKV_ROPE_MAX_AXES : 1];
  if constexpr (AXES) {
    int32_t least = 0;
#pragma unroll
    for (int i = 0; i < WKV_ROPE_MAX_AXES; ++i) {
      pos[i] = i < a.n_axes ? a.positions[token * a.n_axes + i] : 0;
      least = min(least, pos[i]);
    }
    if (least < 0) return;
  } else {
    pos[0] = a.positions[token];
    if (pos[0] < 0) return;
  }
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
  vec v[AT_ONCE][N], w[2][N];
  char *to[AT_ONCE];
  auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int head = first + u * HEADS;
      if (head >= heads) break;
      const bool is_q = head < a.q_heads;
      const RopeTensor &x = is_q ? a.q : a.k;
      const int64_t h = is_q ? head : head - a.q_heads;
      const char *in = (const char *)x.in + b * x.in_b + h * x.in_h + t * x.in_t;
      to[u] = (char *)x.out + b * x.out_b + h * x.out_h + t * x.out_t;
#pragma unroll
      for (int i = 0; i < N; ++i) v[u][i] = STREAM ? __builtin_nontemporal_load((const vec *)(in + at[i])) : *(const vec *)(in + at[i]);
    }
  };
  load();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const char *from = (const char *)(x ? a.k_weight : a.q_weight);
    if (from)
#pragma unroll
      for (int i = 0; i < N; ++i) w[x][i] = *(const vec *)(from + at[i]);
  }
  // (while the first rows are under way)
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
    if (turns[k]) {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const int pair = (p + k * LPH) * PAIRS + i;
        int32_t where = pos[0];
        if constexpr (AXES) {
          const int axis = a.axis[pair];
#pragma unroll
          for (int x = 1; x < WKV_ROPE_MAX_AXES; ++x) where = axis == x ? pos[x] : where;
        }
        const int32_t part = (int32_t)(uint32_t)((uint64_t)(uint32_t)where * a.turns[pair] >> 32);      // signed: -1/2 .. 1/2 turn
        sincospif((float)part * 0x1p-31f, &s[k][i], &c[k][i]);
        c[k][i] *= a.amplitude;
        s[k][i] *= a.amplitude;
      }
    }
  for (;;) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int head = first + u * HEADS;
      if (head >= heads) break;
      const bool is_q = head < a.q_heads, norms = is_q ? a.q_weight != nullptr : a.k_weight != nullptr;
      float x[N][E];
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) x[i][e] = (float)v[u][i][e];
      if (norms) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) sum = fmaf(x[i][e], x[i][e], sum);
        sum = lanes_sum<LPH>(sum);
        float eps = a.eps;
        // With no eps, or next to none, a row counts whose squares leave fp32's normal numbers: again, of the row times 2^100 (all its numbers are below 2^-50).  In a kernel
        // of its own: where interleaved it takes 105 registers instead of 96, and the call above 59 us instead of 57.
        if (SMALL && sum < TINY) {
          sum = 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              x[i][e] *= 1.0f / TINY;
              sum = fmaf(x[i][e], x[i][e], sum);
            }
          sum = lanes_sum<LPH>(sum);
          eps = eps * (1.0f / TINY) * (1.0f / TINY);
        }
        const float by = 1.0f / sqrtf(fmaf(sum, 1.0f / D, eps));
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) x[i][e] *= by * (float)(is_q ? w[0][i][e] : w[1][i][e]);
      }
#pragma unroll
      for (int k = 0; k < RUNS; ++k)
        if (turns[k]) {
#pragma unroll
          for (int i = 0; i < PAIRS; ++i) {
            float &e0 = x[INTERLEAVED ? k : 2 * k][INTERLEAVED ? 2 * i : i], &e1 = x[INTERLEAVED ? k : 2 * k + 1][INTERLEAVED ? 2 * i + 1 : i];
            const float x0 = e0, x1 = e1;
            e0 = x0 * c[k][i] - x1 * s[k][i];
            e1 = x1 * c[k][i] + x0 * s[k][i];
          }
        }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        vec y;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = (T)x[i][e];
        if constexpr (STREAM) __builtin_nontemporal_store(y, (vec *)(to[u] + at[i]));
        else *(vec *)(to[u] + at[i]) = y;
      }
    }
    first += AT_ONCE * HEADS;
    if (first >= heads) break;
    load();
  }
}

template <int DT, int D>
hipError_t launch_d(const NormRopeArgs &a, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.batch * a.n_tokens;
  constexpr int TOKENS = NR_THREADS / (D / 16) / HEADS;
  const int64_t x = (tokens + TOKENS - 1) / TOKENS;
  const int32_t groups = (a.q_heads + a.kv_heads + HEADS - 1) / HEADS;
  // With few tokens a thread takes a single head, and the heads spread over the device.  A head / all heads to a thread, us, 32q/8kv heads of 128 channels in bf16: 16 tokens 4.6 / 6.1,
  // 256 5.3 / 6.7, 700 6.8 / 7.0, 800 (1000 workgroups) 7.0 / 7.2, 900 8.5 / 7.4, 1024 8.8 / 7.8, 1200 9.3 / 9.8, 2048 13.3 / 11.4, 3276 18.3 / 15.3.  Of 64 channels 1600 tokens 6.9 / 7.2;
  // 64q/8kv heads in fp32 400 tokens 9.6 / 11.1; interleaved, 28q/4kv, fp16 500 5.7 / 7.0, 800 7.6 / 7.3.
  const bool few = x * groups <= 1024;
  const dim3 grid((uint32_t)x, (uint32_t)(few ? groups : 1));
  // What exceeds the memory-side cache is not found there by whoever reads it next, and is read and written past it: the 32K prompt 115 us, by plain loads 121.
  const bool streams = tokens * (a.q_heads + a.kv_heads) * D * elem_bytes(a.dtype) > MEMORY_CACHE_BYTES;
#define WKV_NR(INTERLEAVED, AXES, STREAM, SMALL) \
  hipLaunchKernelGGL((norm_rope_kernel<DT, D, INTERLEAVED, AXES, STREAM, SMALL>), grid, dim3(NR_THREADS), 0, stream, a, few ? 1 : groups)
#define WKV_NR_AXES(INTERLEAVED, STREAM, SMALL) \
  if (a.n_axes > 1) WKV_NR(INTERLEAVED, true, STREAM, SMALL); \
  else WKV_NR(INTERLEAVED, false, STREAM, SMALL)
  const bool small = a.eps < TINY;          // (all of them by plain loads)
  if (a.interleaved) {
    if (small) { WKV_NR_AXES(true, false, true); } else if (streams) { WKV_NR_AXES(true, true, false); } else { WKV_NR_AXES(true, false, false); }
  } else {
    if (small) { WKV_NR_AXES(false, false, true); } else if (streams) { WKV_NR_AXES(false, true, false); } else { WKV_NR_AXES(false, false, false); }
  }
#undef WKV_NR_AXES
#undef WKV_NR
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs &a, hipStream_t stream) {
#define WKV_NR_TYPE(DT) return a.d == 128 ? launch_d<DT, 128>(a, stream) : launch_d<DT, 64>(a, stream)
  if (a.dtype == WKV_BF16) WKV_NR_TYPE(DT_BF16);
  if (a.dtype == WKV_F16) WKV_NR_TYPE(DT_F16);
  WKV_NR_TYPE(DT_F32);
#undef WKV_NR_TYPE
}

}  // namespace wkv
