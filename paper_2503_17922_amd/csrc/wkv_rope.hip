// Rotary positions: pairs of channels of queries and keys turned by position * inv_freq.
//
// Two floats in, two out, four multiplications: bound by memory, which every element crosses once each way.  What could get in
// the way is the angle.  It is kept as a fraction of a turn in 64-bit fixed point (position * turns modulo 2^64 is one integer
// product, exact however far the position), whose top 32 bits become the argument of sincospi; a thread takes eight pairs of a
// token and turns them in many heads, so that the sine and cosine cost little.
#include "wkv_device.h"
#include "wkv_operators.h"

namespace wkv {

namespace {

constexpr int ROPE_THREADS = 256;

template <int DT> struct RopeElement;
template <> struct RopeElement<DT_BF16> { typedef __bf16 type; };
template <> struct RopeElement<DT_F16> { typedef _Float16 type; };
template <> struct RopeElement<DT_F32> { typedef float type; };

// 16 elements of a row, 8 at `a` and 8 at `b`.
template <int DT>
struct Sixteen {
  typedef typename RopeElement<DT>::type T;
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  static constexpr int E = 16 / sizeof(T), N = 8 / E;      // elements of a 16-byte piece, pieces of eight elements
  vec lo[N], hi[N];
  __device__ __forceinline__ void load(const char *a, const char *b) {
#pragma unroll
    for (int i = 0; i < N; ++i) { lo[i] = *(const vec *)(a + i * 16); hi[i] = *(const vec *)(b + i * 16); }
  }
  __device__ __forceinline__ void store(char *a, char *b) const {
#pragma unroll
    for (int i = 0; i < N; ++i) { *(vec *)(a + i * 16) = lo[i]; *(vec *)(b + i * 16) = hi[i]; }
  }
  __device__ __forceinline__ float get(int i) const { return i < 8 ? (float)lo[i / E][i % E] : (float)hi[(i - 8) / E][(i - 8) % E]; }
  __device__ __forceinline__ void set(int i, float x) { if (i < 8) lo[i / E][i % E] = (T)x; else hi[(i - 8) / E][(i - 8) % E] = (T)x; }
};

// Workgroup (x, y): 256 / LPH / HEADS tokens side by side, heads y, y + gridDim.y, ... HEADS at a time.  LPH = d / 16 lanes take a
// head's row, 16 channels each: the first rotary / 16 of them eight pairs, the others a copy.
template <int DT, int D, bool INTERLEAVED>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(RopeArgs a, int32_t heads_at_once) {
  constexpr int ES = DT == DT_F32 ? 4 : 2, LPH = D / 16;
  const int lane_of_head = threadIdx.x % LPH, unit = threadIdx.x / LPH;
  const int tokens_at_once = ROPE_THREADS / LPH / heads_at_once;
  const int64_t token = (int64_t)blockIdx.x * tokens_at_once + unit / heads_at_once;
  if (token >= (int64_t)a.batch * a.n_tokens) return;
  const int32_t pos = a.positions[token];
  if (pos < 0) return;
  const int32_t b = (int32_t)((uint32_t)token / (uint32_t)a.n_tokens), t = (int32_t)token - b * a.n_tokens;

  const int half = a.rotary / 2, p = lane_of_head;
  const bool turns = p < a.rotary / 16;
  // (channels past the rotary ones: two neighbouring groups of eight)
  const int at0 = (!turns || INTERLEAVED ? 16 * p : 8 * p) * ES;
  const int at1 = (!turns || INTERLEAVED ? 16 * p + 8 : half + 8 * p) * ES;
  float c[8], s[8];
  if (turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int32_t part = (int32_t)(uint32_t)((uint64_t)(uint32_t)pos * a.turns[8 * p + i] >> 32);      // signed: -1/2 .. 1/2 turn
      sincospif((float)part * 0x1p-31f, &s[i], &c[i]);
      c[i] *= a.amplitude;
      s[i] *= a.inverse ? -a.amplitude : a.amplitude;
    }
  }
  const int heads = a.q_heads + a.kv_heads;
  for (int head = blockIdx.y * heads_at_once + unit % heads_at_once; head < heads; head += gridDim.y * heads_at_once) {
    const bool is_q = head < a.q_heads;
    const RopeTensor &x = is_q ? a.q : a.k;
    const int64_t h = is_q ? head : head - a.q_heads;
    const char *in = (const char *)x.in + b * x.in_b + h * x.in_h + t * x.in_t;
    char *out = (char *)x.out + b * x.out_b + h * x.out_h + t * x.out_t;
    Sixteen<DT> v;
    v.load(in + at0, in + at1);
    if (turns) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : 8 + i;
        const float x0 = v.get(i0), x1 = v.get(i1);
        v.set(i0, x0 * c[i] - x1 * s[i]);
        v.set(i1, x1 * c[i] + x0 * s[i]);
      }
    }
    v.store(out + at0, out + at1);
  }
}

template <int DT, int D>
hipError_t launch_rope_d(const RopeArgs &a, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.batch * a.n_tokens;
  const int32_t heads = a.q_heads + a.kv_heads, at_once = 8;
  const int32_t tokens_at_once = ROPE_THREADS / (D / 16) / at_once;
  const int64_t x = (tokens + tokens_at_once - 1) / tokens_at_once;
  const int32_t groups = (heads + at_once - 1) / at_once;
  const int32_t y = x >= 2048 ? 1 : groups;
  const dim3 grid((uint32_t)x, (uint32_t)y);
  if (a.interleaved) hipLaunchKernelGGL((rope_kernel<DT, D, true>), grid, dim3(ROPE_THREADS), 0, stream, a, at_once);
  else hipLaunchKernelGGL((rope_kernel<DT, D, false>), grid, dim3(ROPE_THREADS), 0, stream, a, at_once);
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
