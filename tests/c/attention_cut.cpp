// Prints how wkv_prefill_attention cuts its work: for every line "batch Hq Hkv d dtype, then q_len k_len of every sequence" on standard input
// one line "rows splits fold_from" (see plan_attention).  Host code only; the launchers are stand-ins.
#include <cstdio>
#include <cstring>
#include <vector>

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
  int B, Hq, Hkv, d, dtype;
  while (std::scanf("%d %d %d %d %d", &B, &Hq, &Hkv, &d, &dtype) == 5) {
    std::vector<int32_t> q(B), k(B);
    for (int b = 0; b < B; ++b)
      if (std::scanf("%d %d", &q[b], &k[b]) != 2) return 1;
    wkv_attention_shape s;
    std::memset(&s, 0, sizeof s);
    s.batch = B; s.n_q_heads = Hq; s.n_kv_heads = Hkv; s.head_dim = d; s.dtype = dtype; s.q_len = q.data(); s.k_len = k.data();
    s.q_stride_h = s.kv_stride_h = s.out_stride_h = s.q_stride_t = s.kv_stride_t = s.out_stride_t = 128;
    wkv::AttentionPlan plan;
    if (wkv::plan_attention(&s, &plan) != WKV_OK) { std::printf("error %s\n", wkv_last_error()); return 1; }
    const wkv::AttentionArgs &a = plan.args;
    // what the kernels write of the workspace: the statistics of the last part of the last block
    const size_t parts = (size_t)plan.items * a.splits * plan.rows;
    if (a.splits > 1 && (plan.stats_at < parts * d * 4 || plan.ws_bytes < plan.stats_at + parts * 8)) { std::printf("error workspace\n"); return 1; }
    std::printf("%d %d %d\n", plan.rows, a.splits, a.fold_from < plan.items ? a.fold_from : -1);
  }
  return 0;
}
