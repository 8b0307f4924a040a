// Drives the host half of the operators of generation (validation, sizes, launch plans) over a sweep of shapes, with launchers that check
// the plan they get instead of launching.
#include <cstdio>
#include <cstring>
#include <algorithm>

#include "wkv_generation.h"

static int failures = 0, launches = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s (last error: %s)\n", __LINE__, #cond, wkv_last_error()); ++failures; } } while (0)

namespace wkv {
// (of the operators that are linked but not driven here)
hipError_t launch_rope(const RopeArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttentionPlan &, const void *, const void *, const void *, void *, float *, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_weighted(const DecodeShape &, const void *, const void *, const void *, void *, void *, int32_t *, const DecodeWeights &,
                                  float *, float *, hipStream_t) { return hipSuccess; }
hipError_t launch_evict(const EvictArgs &, const EvictLayers &, int32_t, float *, int32_t *, int32_t *, const int32_t *, int32_t *, int2 *, hipStream_t) { return hipSuccess; }

hipError_t launch_norm_rope(const NormRopeArgs &a, hipStream_t) {
  ++launches;
  for (int i = 0; i < a.rotary / 2; ++i) EXPECT(a.axis[i] < a.n_axes);
  return hipSuccess;
}
hipError_t launch_quantize(const QuantizedArgs &a, const QuantizedLayers &, int32_t, hipStream_t) { ++launches; EXPECT((int64_t)a.heads * a.n_rows <= 1 << 30); return hipSuccess; }
hipError_t launch_dequantize(const QuantizedArgs &a, const QuantizedLayers &, int32_t, hipStream_t) { ++launches; EXPECT((int64_t)a.heads * a.n_rows <= 1 << 30); return hipSuccess; }
hipError_t launch_decode_quantized(const DecodeShape &s, int32_t, const void *, const void *, const void *, void *, void *, void *, void *, int32_t *, float *, float *, hipStream_t) {
  ++launches;
  EXPECT((int64_t)s.n_splits * s.chunk >= s.capacity && s.chunk % 64 == 0 && s.n_splits <= DEC_MAX_SPLITS && s.st * 32 <= 0x7fffffff);
  return hipSuccess;
}
hipError_t launch_tree(const TreePlan &plan, const void *, const void *, const void *, const int32_t *, void *, void *, const int32_t *, void *, void *, hipStream_t) {
  ++launches;
  const TreeArgs &a = plan.args;
  const int rows = plan.row_waves * 32;
  const int64_t keys = (int64_t)tree_wave_keys(a.dtype == WKV_F32, plan.key_waves) * plan.key_waves;
  // every row has a block and every key a range; a grid and 32-bit row numbers that hold them; room for the partial results
  EXPECT(a.blocks * rows >= a.n_rows && (a.blocks - 1) * rows < a.n_rows);
  EXPECT(a.splits >= 1 && (int64_t)a.splits * a.chunk * keys >= a.capacity && (int64_t)(a.splits - 1) * a.chunk * keys < a.capacity);
  EXPECT((int64_t)a.splits * a.chunk <= 0x7fffffff && a.splits < 65535 && a.heads <= 65535);
  EXPECT(a.splits == 1 || (int64_t)a.heads * a.blocks * a.splits <= 2048);
  if (a.splits > 1) EXPECT(plan.ws_bytes >= (size_t)a.heads * a.blocks * (a.splits + 1) * rows * (a.d * 4 + 8));
  // (head numbers by multiplication: heads + 9 a range stay within what the divider is exact for)
  for (int y : {0, a.splits == 1 ? 0 : a.splits})          // (the last: the nodes)
    for (int x : {0, 1, a.heads / 2, a.heads - 1}) {
      const RangeOf it(x, y, a.heads, a.heads_magic);
      EXPECT(it.head == (x + 9 * y) % a.heads && it.range == y);
    }
  EXPECT(plan.key_waves == (plan.row_waves == 2 ? 2 : 1) && (plan.row_waves == 2 || plan.row_waves == 4 || (plan.row_waves == 8 && a.dtype != WKV_F32 && a.splits == 1)));
  return hipSuccess;
}
hipError_t launch_accept(const TreeArgs &, const EvictLayers &, int32_t, const int32_t *, const int32_t *, int32_t *, bool, hipStream_t) { ++launches; return hipSuccess; }
}  // namespace wkv

int main() {
  char *dev = (char *)0x7f0000001000ull;
  auto at = [&](int i) { return (void *)(dev + ((size_t)i << 20)); };
  int32_t *ints = (int32_t *)at(20);

  // ---- trees
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int d : {64, 128})
      for (int G : {1, 3, 8})
        for (int T : {1, 4, 16, 33, 64})
          for (int capacity : {1, 63, 64, 65, 4384, 100000, 1 << 30})
            for (int heads : {1, 8, 88, 512, 4000, 65535}) {
              wkv_tree_shape s;
              std::memset(&s, 0, sizeof s);
              s.batch = heads == 65535 ? 65535 : 1; s.n_kv_heads = heads / s.batch; s.n_q_heads = s.n_kv_heads * G; s.head_dim = d; s.dtype = dtype; s.n_nodes = T;
              s.capacity = capacity;
              s.cache_stride_b = s.cache_stride_h = s.cache_stride_t = s.q_stride_h = s.q_stride_t = s.new_stride_h = s.new_stride_t = s.out_stride_h = s.out_stride_t = d;
              const size_t ws = wkv_tree_workspace_bytes(&s);
              EXPECT(ws > 0);
              EXPECT(wkv_decode_tree(&s, at(0), at(1), at(2), ints, at(3), at(4), ints, at(5), at(6), ws, nullptr) == WKV_OK);
              void *layers[2] = {at(0), at(1)};
              EXPECT(wkv_tree_accept(&s, 2, layers, layers, ints, ints, ints, nullptr) == WKV_OK);
            }

  // ---- caches in 8 and 4 bits
  for (int format = 0; format < 2; ++format)
    for (int d : {64, 128})
      for (int capacity : {1, 4384, 1 << 30})
        for (int heads : {1, 8, 512, 65535}) {
          wkv_quantized_shape s;
          std::memset(&s, 0, sizeof s);
          s.batch = heads; s.n_q_heads = 3; s.n_kv_heads = 1; s.head_dim = d; s.dtype = WKV_BF16; s.format = format; s.capacity = capacity;
          s.code_stride_b = s.code_stride_h = s.code_stride_t = 128; s.n_rows = s.row_capacity = std::min(capacity, (1 << 30) / heads);
          s.row_stride_b = s.row_stride_h = s.row_stride_t = d;
          const size_t ws = wkv_decode_quantized_workspace_bytes(&s);
          EXPECT(ws >= (size_t)heads * 3 * (d + 2) * 4);
          EXPECT(wkv_decode_step_quantized(&s, at(0), at(1), at(2), at(3), at(4), at(5), at(6), ints, (float *)at(7), at(8), ws, nullptr) == WKV_OK);
          void *l[2] = {at(0), at(1)};
          EXPECT(wkv_cache_quantize(&s, 2, l, l, ints, ints, ints, l, l, l, l, nullptr) == WKV_OK);
          EXPECT(wkv_cache_dequantize(&s, 2, l, l, l, l, ints, ints, l, l, nullptr) == WKV_OK);
        }

  // ---- norms with rotary positions
  double inv[64];
  int32_t axis[64];
  for (int i = 0; i < 64; ++i) { inv[i] = 1.0 / (i + 1); axis[i] = i % 4; }
  for (int axes : {1, 4})
    for (int rotary : {16, 128}) {
      wkv_norm_rope_shape r;
      std::memset(&r, 0, sizeof r);
      r.batch = 2; r.n_tokens = 3; r.n_q_heads = 2; r.n_kv_heads = 1; r.head_dim = 128; r.rotary_dim = rotary; r.dtype = WKV_F32; r.n_axes = axes; r.inv_freq = inv;
      r.axis_of_pair = axes > 1 ? axis : nullptr;
      r.q_stride_h = r.q_stride_t = r.q_out_stride_h = r.q_out_stride_t = r.k_stride_h = r.k_stride_t = r.k_out_stride_h = r.k_out_stride_t = 128;
      EXPECT(wkv_norm_rope(&r, ints, at(0), nullptr, at(1), at(2), at(3), at(4), nullptr) == WKV_OK);
    }
  EXPECT(launches > 2000);
  std::printf("ok (%d checks failed)\n", failures);
  return failures ? 1 : 0;
}
