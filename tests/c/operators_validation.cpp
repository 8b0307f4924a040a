// Drives the host half of the operators around the compression (validation, sizes, launch plans) over a sweep of shapes, with
// launchers that check the plan they get instead of launching: every block of every sequence has exactly one work item.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <vector>

#include "wkv_operators.h"

static int failures = 0, launches = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s (last error: %s)\n", __LINE__, #cond, wkv_last_error()); ++failures; } } while (0)

namespace wkv {
static RopeArgs last_rope;
hipError_t launch_rope(const RopeArgs &a, hipStream_t) { last_rope = a; ++launches; return hipSuccess; }
hipError_t launch_attention(const AttentionPlan &plan, const void *, const void *, const void *, void *, float *, void *, hipStream_t) {
  ++launches;
  const AttentionArgs &a = plan.args;
  std::vector<std::vector<int>> seen((size_t)a.n_seqs * a.Hkv);
  for (int i = 0; i < a.n_seqs; ++i) for (int h = 0; h < a.Hkv; ++h) seen[(size_t)i * a.Hkv + h].assign(a.seq[i].blocks, 0);
  for (int i = 0; i + 1 < a.n_seqs; ++i) EXPECT(a.seq[i].blocks >= a.seq[i + 1].blocks);
  for (int item = 0; item < plan.items; ++item) {          // (as the kernel does it)
    int seg = 0;
    while (seg < a.n_seqs && item >= a.ends[seg]) ++seg;
    EXPECT(seg < a.n_seqs);
    if (seg >= a.n_seqs) return hipSuccess;
    const int rel = item - (seg ? a.ends[seg - 1] : 0), per_level = (seg + 1) * a.Hkv;
    const int level = rel / per_level, at = rel % per_level, si = at / a.Hkv, h = at % a.Hkv, block = a.seq[seg].blocks - 1 - level;
    EXPECT(block >= 0 && block < a.seq[si].blocks);
    if (block >= 0 && block < a.seq[si].blocks) ++seen[(size_t)si * a.Hkv + h][block];
  }
  for (const auto &rows : seen) for (int n : rows) EXPECT(n == 1);
  return hipSuccess;
}
hipError_t launch_decode_weighted(const DecodeShape &, const void *, const void *, const void *, void *, void *, int32_t *, const DecodeWeights &,
                                  float *, float *, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_evict(const EvictArgs &a, const EvictLayers &, int32_t, float *, int32_t *, int32_t *, const int32_t *, int32_t *, int2 *,
                        hipStream_t) { EXPECT(2 * (int64_t)a.max_moves + 1 >= a.capacity); ++launches; return hipSuccess; }
}  // namespace wkv

int main() {
  char *dev = (char *)0x7f0000001000ull;
  auto at = [&](int i) { return (void *)(dev + ((size_t)i << 20)); };

  // ---- attention: lengths of all kinds
  uint32_t state = 12345;
  auto random = [&](uint32_t n) { state = state * 1664525u + 1013904223u; return (int32_t)((state >> 8) % n); };
  for (int round = 0; round < 400; ++round) {
    const int B = 1 + random(round % 5 == 0 ? 64 : 7), Hkv = 1 + random(9), G = 1 + random(9);
    std::vector<int32_t> q(B), k(B);
    std::vector<int64_t> qs(B), ks(B);
    for (int b = 0; b < B; ++b) { q[b] = random(4) ? random(700) : 0; k[b] = random(3) ? q[b] + random(900) : random(300); qs[b] = random(1000); ks[b] = random(1000); }
    wkv_attention_shape s;
    std::memset(&s, 0, sizeof s);
    s.batch = B; s.n_q_heads = Hkv * G; s.n_kv_heads = Hkv; s.head_dim = round % 2 ? 64 : 128; s.dtype = round % 3; s.lse_rows = round % 4 ? random(50) : 0;
    s.q_len = q.data(); s.k_len = round % 3 ? k.data() : nullptr; s.q_start = round % 2 ? qs.data() : nullptr; s.k_start = round % 2 ? ks.data() : nullptr;
    s.q_stride_h = s.kv_stride_h = s.out_stride_h = s.q_stride_t = s.kv_stride_t = s.out_stride_t = 128;
    const size_t ws = wkv_attention_workspace_bytes(&s);
    EXPECT(ws > 0);
    EXPECT(wkv_prefill_attention(&s, at(0), at(1), at(2), at(3), (float *)at(4), at(5), ws, nullptr) == WKV_OK);
  }

  // ---- rope: the fixed-point frequencies
  double inv[64];
  for (int i = 0; i < 64; ++i) inv[i] = std::pow(1.5, i) * 1e-9 * (i % 2 ? -1 : 1);
  wkv_rope_shape r;
  std::memset(&r, 0, sizeof r);
  r.batch = 2; r.n_tokens = 3; r.n_q_heads = 2; r.n_kv_heads = 1; r.head_dim = 128; r.rotary_dim = 128; r.dtype = WKV_F32; r.inv_freq = inv;
  r.q_stride_h = r.q_stride_t = r.q_out_stride_h = r.q_out_stride_t = r.k_stride_h = r.k_stride_t = r.k_out_stride_h = r.k_out_stride_t = 128;
  EXPECT(wkv_rope(&r, (const int32_t *)at(0), at(1), at(2), at(3), at(4), nullptr) == WKV_OK);
  for (int i = 0; i < 64; ++i) {
    const long double turns = (long double)inv[i] / 6.283185307179586476925286766559L, part = turns - floorl(turns);
    const long double got = ldexpl((long double)wkv::last_rope.turns[i], -64), off = fabsl(got - part);
    // the constant 1 / (2 pi) has 64 significant bits (off by up to 1.6 * 2^-64 of the turns), the division here as many, the result a step of 2^-64
    const long double tol = 4 * (fabsl(turns) + 1) * 0x1p-64L;
    EXPECT(off < tol || 1 - off < tol);
  }
  EXPECT(wkv::last_rope.amplitude == 1.0f);

  // ---- caches
  for (int capacity : {1, 2, 3, 1000, 4128, 1 << 20, 1 << 30})
    for (int g : {1, 4, 8}) {
      wkv_decode_shape c;
      std::memset(&c, 0, sizeof c);
      c.batch = 3; c.n_q_heads = 2 * g; c.n_kv_heads = 2; c.head_dim = 64; c.dtype = WKV_BF16; c.capacity = capacity;
      c.cache_stride_b = c.cache_stride_h = c.cache_stride_t = 64;
      const size_t w1 = wkv_decode_weighted_workspace_bytes(&c), w2 = wkv_evict_workspace_bytes(&c);
      EXPECT(w1 > (size_t)6 * g * capacity * 4 && w2 > (size_t)6 * (capacity / 2) * 8);
      EXPECT(wkv_decode_step_weighted(&c, at(0), at(1), at(2), at(3), at(4), (int32_t *)at(5), (float *)at(6), nullptr, nullptr, (float *)at(7), at(8), w1, nullptr) == WKV_OK);
      void *layers[2] = {at(0), at(1)};
      EXPECT(wkv_cache_evict(&c, 2, layers, layers, (float *)at(6), (int32_t *)at(5), (int32_t *)at(7), (int32_t *)at(8), 5, at(9), w2, nullptr) == WKV_OK);
    }
  EXPECT(launches > 400);
  std::printf("ok (%d checks failed)\n", failures);
  return failures ? 1 : 0;
}
