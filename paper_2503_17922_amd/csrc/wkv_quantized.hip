// Cache rows into 8 and 4 bits and back: bound by memory, which every row crosses once each way.
//
// A lane takes eight channels; four lanes share a scale, whose largest magnitude is found by two DPP steps.  The lanes of a row put its scales
// together, so that they leave in one store.  A workgroup takes rows of one (sequence, KV head), whose counts are scalars then, or, where there are
// few rows to each, all rows of several: a token a sequence fills workgroups as well as a long prompt does.
//
// The 4128 kept rows a KV head of the 32K benchmark's prompt, four layers (102 MB), picked one by one from eight times as many, into 8 bits: 37 us with each row's lookups
// before its loads, 31 with all of a lane's lookups at once, 29.5 with the lookups as scalars and no load under a condition, 22.3 = 4.6 TB/s with the plain rows, which are read
// once, by nontemporal loads (a ragged batch into 4 bits 27.4 and 21.5, a token for each of 64 sequences 3.5 both).  Back 16.7 us = 6.1 TB/s.
#include "wkv_few_bits.h"

namespace wkv {

namespace {

// Rows of a lane at once.  Two / four / eight, us, by workgroups of 128 before the nontemporal loads: a token for each of 64 sequences, four layers, 3.4 / 4.4 / 5.9 into 8 bits and
// 3.2 / 3.8 / 4.7 back; the long call above 29.4 / 31.2 / 32.3 and 17.8 / 17.2 / 17.4; a ragged batch in 4 bits 27.4 / 27.8 / 29.2 and 21.3 / 19.2 / 20.2.  Two at once by workgroups
// of 64 / 128 / 256: within 0.3 us of each other, but for the ragged batch: 26.7 / 27.4 / 27.4 and 25.9 / 21.3 / 21.1 back.
constexpr int QZ_THREADS = 256, AT_ONCE = 2;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false); }

// Where the rows of a lane lie, every UNITS-th of the workgroup's: its (sequence, KV head), its own number r, its place in the cache, and whether there is such a row at all.
// (No number of a row that is not there leaves its range, so that nothing is loaded under a condition: behind one the compiler waits for each load by itself, which
// costs a trip to memory a row.)
// MANY: `group` (sequence, KV head) pairs to a workgroup.
template <int UNITS, bool MANY>
struct RowsOf {
  int bh[AT_ONCE], r[AT_ONCE], place[AT_ONCE];
  bool there[AT_ONCE];
  __device__ __forceinline__ RowsOf(const QuantizedArgs &a, int unit) {
    int first[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int v = u * UNITS + unit;
      if constexpr (MANY) {
        const int at = divide((uint32_t)v, a.rows_magic);
        there[u] = at < a.group && (int)blockIdx.y * a.group + at < a.heads;
        bh[u] = min((int)blockIdx.y * a.group + at, a.heads - 1);
        r[u] = v - at * a.n_rows;
      } else {
        bh[u] = blockIdx.y;
        r[u] = a.first_row + (int)blockIdx.x * (UNITS * AT_ONCE) + v;
        there[u] = r[u] < a.n_rows;
        r[u] = min(r[u], a.n_rows - 1);
      }
    }
    of(a.first, 0, first);
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int64_t at = (int64_t)first[u] + r[u];
      there[u] = there[u] && at >= 0 && at < a.capacity;
      place[u] = (int)min(max(at, (int64_t)0), (int64_t)a.capacity - 1);
    }
  }
  // A number of each (sequence, KV head), `otherwise` where there are none.
  __device__ __forceinline__ void of(const int32_t *p, int otherwise, int (&x)[AT_ONCE]) const {
    if (!p) {
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) x[u] = otherwise;
    } else if constexpr (MANY) {
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) x[u] = p[bh[u]];
    } else {
      const int all = load_scalar(p + blockIdx.y);
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) x[u] = all;
    }
  }
};

template <int DT, int D, int FORMAT, bool MANY>
__global__ __launch_bounds__(QZ_THREADS) void quantize_kernel(QuantizedArgs a, QuantizedLayers layers) {
  constexpr int LPR = D / 8, UNITS = QZ_THREADS / LPR, PIECES = DT == DT_F32 ? 2 : 1, SB = D / SCALE_GROUP;
  const int layer = blockIdx.z >> 1, is_v = blockIdx.z & 1;
  const char *plain = (const char *)layers.plain[is_v][layer];
  char *codes = (char *)layers.codes[is_v][layer], *scales = (char *)layers.scales[is_v][layer];
  const int lane = threadIdx.x % LPR, unit = threadIdx.x / LPR;

  if (!MANY && a.n_keep && a.first_row + (int)blockIdx.x * (UNITS * AT_ONCE) >= load_scalar(a.n_keep + blockIdx.y)) return;
  RowsOf<UNITS, MANY> rows(a, unit);
  int keep[AT_ONCE], from[AT_ONCE];
  rows.of(a.n_keep, a.n_rows, keep);
  if (a.tok_idx) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) from[u] = a.tok_idx[(int64_t)rows.bh[u] * a.n_rows + rows.r[u]];
  } else {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) from[u] = rows.r[u];
  }
  u32x4 x[AT_ONCE][PIECES];
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u) {
    rows.there[u] = rows.there[u] && rows.r[u] < keep[u] && from[u] >= 0 && from[u] < a.row_capacity;
    const int b = divide((uint32_t)rows.bh[u], a.kv_magic), h = rows.bh[u] - b * a.Hkv;
    const char *in = plain + (b * a.r_sb + h * a.r_sh + min(max(from[u], 0), a.row_capacity - 1) * a.r_st) + lane * (16 * PIECES);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) x[u][k] = __builtin_nontemporal_load((const u32x4 *)(in + k * 16));
  }
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u) {
    if (!rows.there[u]) continue;                // (the same in all lanes of a row)
    float f[8];
    widen<DT>(__builtin_bit_cast(uint4, x[u][0]), f);
    if constexpr (PIECES == 2) widen<DT>(__builtin_bit_cast(uint4, x[u][1]), f + 4);
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(f[e]) & 0x7fffffffu);
    largest = max(largest, dpp<0xB1>(largest));                  // quad_perm [1,0,3,2]
    largest = max(largest, dpp<0x4E>(largest));                  // quad_perm [2,3,0,1]
    const uint32_t byte = (uint32_t)scale_byte<FORMAT>(largest);
    const float scale = scale_of(byte);
    const int b = divide((uint32_t)rows.bh[u], a.kv_magic), h = rows.bh[u] - b * a.Hkv;
    char *to = codes + (b * a.c_sb + h * a.c_sh + rows.place[u] * a.c_st);
    if constexpr (FORMAT == E4M3) {
      uint32_t lo = to_codes<FORMAT, 1>(to_codes<FORMAT, 0>(0, f[0], f[1], scale), f[2], f[3], scale);
      uint32_t hi = to_codes<FORMAT, 1>(to_codes<FORMAT, 0>(0, f[4], f[5], scale), f[6], f[7], scale);
      if (byte == NO_SCALE) lo = hi = 0;
      *(u32x2 *)(to + lane * 8) = (u32x2){lo, hi};
    } else {
      uint32_t w = to_codes<FORMAT, 1>(to_codes<FORMAT, 0>(0, f[0], f[1], scale), f[2], f[3], scale);
      w = to_codes<FORMAT, 3>(to_codes<FORMAT, 2>(w, f[4], f[5], scale), f[6], f[7], scale);
      if (byte == NO_SCALE) w = 0;
      *(uint32_t *)(to + lane * 4) = w;
    }
    uint32_t all = byte << (lane / 4 * 8);
    char *sc = scales + ((int64_t)rows.bh[u] * a.capacity + rows.place[u]) * SB;
    if constexpr (D == 128) {
      all |= dpp<0x124>(all);                                    // row_ror:4
      all |= dpp<0x128>(all);                                    // row_ror:8
      if (lane == 0) *(uint32_t *)sc = all;
    } else {
      all |= dpp<0x141>(all);                                    // row_half_mirror
      if (lane == 0) *(uint16_t *)sc = (uint16_t)all;
    }
  }
}

template <int DT, int D, int FORMAT, bool MANY>
__global__ __launch_bounds__(QZ_THREADS) void dequantize_kernel(QuantizedArgs a, QuantizedLayers layers) {
  constexpr int LPR = D / 8, UNITS = QZ_THREADS / LPR, SB = D / SCALE_GROUP, WORDS = FORMAT == E4M3 ? 2 : 1;
  const int layer = blockIdx.z >> 1, is_v = blockIdx.z & 1;
  char *plain = (char *)layers.plain[is_v][layer];
  const char *codes = (const char *)layers.codes[is_v][layer];
  const uint8_t *scales = (const uint8_t *)layers.scales[is_v][layer];
  const int lane = threadIdx.x % LPR, unit = threadIdx.x / LPR;

  if (!MANY && a.n_keep && (int64_t)(a.first ? load_scalar(a.first + blockIdx.y) : 0) + a.first_row + (int)blockIdx.x * (UNITS * AT_ONCE) >= load_scalar(a.n_keep + blockIdx.y)) return;
  RowsOf<UNITS, MANY> rows(a, unit);
  int valid[AT_ONCE];
  rows.of(a.n_keep, a.capacity, valid);
  uint32_t x[AT_ONCE][WORDS], byte[AT_ONCE];
  char *to[AT_ONCE];
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u) {
    rows.there[u] = rows.there[u] && rows.place[u] < valid[u];
    const int b = divide((uint32_t)rows.bh[u], a.kv_magic), h = rows.bh[u] - b * a.Hkv;
    const char *in = codes + (b * a.c_sb + h * a.c_sh + rows.place[u] * a.c_st) + lane * (WORDS * 4);
    if constexpr (WORDS == 2) { const u32x2 w = *(const u32x2 *)in; x[u][0] = w[0]; x[u][1] = w[1]; }
    else x[u][0] = *(const uint32_t *)in;
    byte[u] = scales[((int64_t)rows.bh[u] * a.capacity + rows.place[u]) * SB + lane / 4];
    to[u] = plain + (b * a.r_sb + h * a.r_sh + rows.r[u] * a.r_st) + lane * (DT == DT_F32 ? 32 : 16);
  }
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u) {
    if (!rows.there[u]) continue;
    const float scale = scale_of(byte[u]);
    if constexpr (DT == DT_BF16) {
      u32x4 y;
      if constexpr (FORMAT == E4M3)
        y = (u32x4){bf16_pair<FORMAT, 0>(x[u][0], scale), bf16_pair<FORMAT, 1>(x[u][0], scale), bf16_pair<FORMAT, 0>(x[u][1], scale), bf16_pair<FORMAT, 1>(x[u][1], scale)};
      else
        y = (u32x4){bf16_pair<FORMAT, 0>(x[u][0], scale), bf16_pair<FORMAT, 1>(x[u][0], scale), bf16_pair<FORMAT, 2>(x[u][0], scale), bf16_pair<FORMAT, 3>(x[u][0], scale)};
      *(u32x4 *)to[u] = y;
    } else {
      float2 f[4];
      f[0] = float_pair<FORMAT, 0>(x[u][0], scale);
      f[1] = float_pair<FORMAT, 1>(x[u][0], scale);
      f[2] = float_pair<FORMAT, FORMAT == E4M3 ? 0 : 2>(x[u][WORDS - 1], scale);
      f[3] = float_pair<FORMAT, FORMAT == E4M3 ? 1 : 3>(x[u][WORDS - 1], scale);
      if constexpr (DT == DT_F32) {
        ((float4 *)to[u])[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
        ((float4 *)to[u])[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
      } else {
        // past the largest number of the type: that one (a value may have been rounded up to 2^16); NaN stays
        auto half = [](float v) { return (_Float16)(v > 65504.0f ? 65504.0f : v < -65504.0f ? -65504.0f : v); };
        typedef _Float16 f16x8v __attribute__((ext_vector_type(8)));
        *(f16x8v *)to[u] = (f16x8v){half(f[0].x), half(f[0].y), half(f[1].x), half(f[1].y), half(f[2].x), half(f[2].y), half(f[3].x), half(f[3].y)};
      }
    }
  }
}

template <int DT, int D, int FORMAT>
hipError_t launch_as(bool back, QuantizedArgs a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream) {
  constexpr int ROWS = QZ_THREADS / (D / 8) * AT_ONCE;
  const bool many = a.n_rows <= ROWS / 2;
  a.group = many ? ROWS / a.n_rows : 1;
  a.rows_magic = division_magic(a.n_rows);          // (of numbers below ROWS)
  const int64_t groups = many ? 1 : ((int64_t)a.n_rows + ROWS - 1) / ROWS;
  for (int64_t at = 0; at < groups; at += MOST_ROW_GROUPS) {
    a.first_row = (int32_t)(at * ROWS);
    const dim3 grid((uint32_t)(groups - at < MOST_ROW_GROUPS ? groups - at : MOST_ROW_GROUPS), (uint32_t)((a.heads + a.group - 1) / a.group), (uint32_t)n_layers * 2);
#define WKV_QZ(KERNEL, MANY) hipLaunchKernelGGL((KERNEL<DT, D, FORMAT, MANY>), grid, dim3(QZ_THREADS), 0, stream, a, layers)
    if (back) { if (many) WKV_QZ(dequantize_kernel, true); else WKV_QZ(dequantize_kernel, false); }
    else { if (many) WKV_QZ(quantize_kernel, true); else WKV_QZ(quantize_kernel, false); }
#undef WKV_QZ
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int DT>
hipError_t launch_type(bool back, const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream) {
  if (a.format == E4M3) return a.d == 128 ? launch_as<DT, 128, E4M3>(back, a, layers, n_layers, stream) : launch_as<DT, 64, E4M3>(back, a, layers, n_layers, stream);
  return a.d == 128 ? launch_as<DT, 128, E2M1>(back, a, layers, n_layers, stream) : launch_as<DT, 64, E2M1>(back, a, layers, n_layers, stream);
}
hipError_t launch_rows(bool back, const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream) {
  if (a.dtype == WKV_BF16) return launch_type<DT_BF16>(back, a, layers, n_layers, stream);
  if (a.dtype == WKV_F16) return launch_type<DT_F16>(back, a, layers, n_layers, stream);
  return launch_type<DT_F32>(back, a, layers, n_layers, stream);
}

}  // namespace

hipError_t launch_quantize(const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream) {
  return launch_rows(false, a, layers, n_layers, stream);
}
hipError_t launch_dequantize(const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream) {
  return launch_rows(true, a, layers, n_layers, stream);
}

}  // namespace wkv
