// Prints whether one workgroup takes all rows of a (sequence, KV head) in wkv_decode_step_weighted: for every line "batch Hq Hkv d dtype capacity" on
// standard input one line, 0 or 1 (see decode_takes_whole_caches).  Host code only; the launchers are stand-ins.
#include <cstdio>
#include <cstring>

#include "wkv_operators.h"

namespace wkv {
hipError_t launch_rope(const RopeArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttentionPlan &, const void *, const void *, const void *, void *, float *, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_weighted(const DecodeShape &, const void *, const void *, const void *, void *, void *, int32_t *, const DecodeWeights &,
                                  float *, float *, hipStream_t) { return hipSuccess; }
hipError_t launch_evict(const EvictArgs &, const EvictLayers &, int32_t, float *, int32_t *, int32_t *, const int32_t *, int32_t *, int2 *,
                        hipStream_t) { return hipSuccess; }
}  // namespace wkv

int main() {
  wkv_decode_shape p;
  std::memset(&p, 0, sizeof p);
  while (std::scanf("%d %d %d %d %d %d", &p.batch, &p.n_q_heads, &p.n_kv_heads, &p.head_dim, &p.dtype, &p.capacity) == 6) {
    p.cache_stride_h = (int64_t)p.capacity * p.head_dim; p.cache_stride_b = p.cache_stride_h * p.n_kv_heads; p.cache_stride_t = p.head_dim;
    wkv::Decode dc;
    if (wkv::validate_decode(&p, &dc) != WKV_OK) { std::printf("error %s\n", wkv_last_error()); return 1; }
    const wkv::DecodeShape &s = dc.shape;
    const bool whole = wkv::decode_takes_whole_caches(s);
    // the logits of a full cache, in blocks of 16 rows, and then the outputs of its waves lie in LDS
    if (whole && ((s.capacity + 15) / 16 * 16 * s.G > wkv::WHOLE_FLOATS || wkv::WHOLE_THREADS / 64 * s.G * s.d > wkv::WHOLE_FLOATS)) { std::printf("error room\n"); return 1; }
    std::printf("%d\n", whole ? 1 : 0);
  }
  return 0;
}
