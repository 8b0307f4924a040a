// Prints how wkv_decode_tree cuts its work: for every line "batch Hq Hkv d dtype n_nodes capacity" on standard input one line
// "row_waves key_waves blocks splits streams" (see plan_tree).  Host code only; the launchers are stand-ins.
#include <cstdio>
#include <cstring>

#include "wkv_generation.h"

namespace wkv {
hipError_t launch_rope(const RopeArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttentionPlan &, const void *, const void *, const void *, void *, float *, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_weighted(const DecodeShape &, const void *, const void *, const void *, void *, void *, int32_t *, const DecodeWeights &,
                                  float *, float *, hipStream_t) { return hipSuccess; }
hipError_t launch_evict(const EvictArgs &, const EvictLayers &, int32_t, float *, int32_t *, int32_t *, const int32_t *, int32_t *, int2 *, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_rope(const NormRopeArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_quantize(const QuantizedArgs &, const QuantizedLayers &, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_dequantize(const QuantizedArgs &, const QuantizedLayers &, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_quantized(const DecodeShape &, int32_t, const void *, const void *, const void *, void *, void *, void *, void *, int32_t *, float *, float *, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_tree(const TreePlan &, const void *, const void *, const void *, const int32_t *, void *, void *, const int32_t *, void *, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_accept(const TreeArgs &, const EvictLayers &, int32_t, const int32_t *, const int32_t *, int32_t *, bool, hipStream_t) { return hipSuccess; }
}  // namespace wkv

int main() {
  int B, Hq, Hkv, d, dtype, T, capacity;
  while (std::scanf("%d %d %d %d %d %d %d", &B, &Hq, &Hkv, &d, &dtype, &T, &capacity) == 7) {
    wkv_tree_shape s;
    std::memset(&s, 0, sizeof s);
    s.batch = B; s.n_q_heads = Hq; s.n_kv_heads = Hkv; s.head_dim = d; s.dtype = dtype; s.n_nodes = T; s.capacity = capacity;
    s.cache_stride_h = s.cache_stride_t = s.q_stride_h = s.q_stride_t = s.new_stride_h = s.new_stride_t = s.out_stride_h = s.out_stride_t = d;
    wkv::TreePlan plan;
    if (wkv::plan_tree(&s, &plan) != WKV_OK) { std::printf("error %s\n", wkv_last_error()); return 1; }
    std::printf("%d %d %d %d %d\n", plan.row_waves, plan.key_waves, plan.args.blocks, plan.args.splits, (int)plan.streams);
  }
  return 0;
}
