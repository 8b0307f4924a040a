// Host side of the operators of generation: argument validation, derived sizes, launch plans and the entry points.
// Nothing in this file but the launchers' calls touches the GPU.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "wkv_generation.h"

namespace wkv {

namespace {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

wkv_status plan_norm_rope(const wkv_norm_rope_shape *p, NormRopeArgs *a) {
  set_error("");
  if (!p) return invalid("shape is NULL");
  if (p->batch < 1) { set_error("batch must be >= 1 (got %d)", p->batch); return WKV_ERR_INVALID_ARG; }
  if (p->n_tokens < 0) return invalid("n_tokens must be >= 0");
  if ((int64_t)p->batch * p->n_tokens > 1 << 25) { set_error("batch * n_tokens exceeds 2^25; split the call"); return WKV_ERR_UNSUPPORTED; }
  if (p->n_q_heads < 0 || p->n_kv_heads < 0) return invalid("numbers of heads must be >= 0");
  if (p->n_q_heads > 65535 || p->n_kv_heads > 65535) { set_error("more than 65535 heads"); return WKV_ERR_UNSUPPORTED; }
  if (!known_dtype(p->dtype)) return WKV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) { set_error("head_dim %d is not supported (64 or 128)", p->head_dim); return WKV_ERR_UNSUPPORTED; }
  if (p->rotary_dim < 1 || p->rotary_dim > p->head_dim) { set_error("rotary_dim %d outside [1, head_dim]", p->rotary_dim); return WKV_ERR_INVALID_ARG; }
  if (p->rotary_dim % 16 != 0) { set_error("rotary_dim %d is not supported (a multiple of 16)", p->rotary_dim); return WKV_ERR_UNSUPPORTED; }
  if (p->flags & ~WKV_ROPE_INTERLEAVED) { set_error("unknown bits in flags (0x%x)", p->flags); return WKV_ERR_INVALID_ARG; }
  if (p->n_axes < 1 || p->n_axes > WKV_ROPE_MAX_AXES) { set_error("n_axes %d outside [1, %d]", p->n_axes, WKV_ROPE_MAX_AXES); return WKV_ERR_INVALID_ARG; }
  if (!(p->eps >= 0.0f) || std::isinf(p->eps)) return invalid("eps must be finite and >= 0");
  if (!std::isfinite(p->amplitude) || std::fabs(p->amplitude) > 3.0e38) return invalid("amplitude must be finite (0 selects 1)");
  if (!p->inv_freq) return invalid("inv_freq must be a non-NULL host array");
  for (int32_t i = 0; i < p->rotary_dim / 2; ++i) {
    if (!std::isfinite(p->inv_freq[i])) { set_error("inv_freq[%d] is not finite", i); return WKV_ERR_INVALID_ARG; }
    if (p->axis_of_pair && (p->axis_of_pair[i] < 0 || p->axis_of_pair[i] >= p->n_axes)) {
      set_error("axis_of_pair[%d] = %d outside [0, %d)", i, p->axis_of_pair[i], p->n_axes); return WKV_ERR_INVALID_ARG;
    }
  }
  if (p->n_q_heads && (!good_strides(p->dtype, p->head_dim, p->q_stride_b, p->q_stride_h, p->q_stride_t, "q") ||
                       !good_strides(p->dtype, p->head_dim, p->q_out_stride_b, p->q_out_stride_h, p->q_out_stride_t, "q_out")))
    return WKV_ERR_INVALID_ARG;
  if (p->n_kv_heads && (!good_strides(p->dtype, p->head_dim, p->k_stride_b, p->k_stride_h, p->k_stride_t, "k") ||
                        !good_strides(p->dtype, p->head_dim, p->k_out_stride_b, p->k_out_stride_h, p->k_out_stride_t, "k_out")))
    return WKV_ERR_INVALID_ARG;
  std::memset(a, 0, sizeof(*a));
  const int64_t e = elem_bytes(p->dtype);
  a->q = {nullptr, nullptr, p->q_stride_b * e, p->q_stride_h * e, p->q_stride_t * e, p->q_out_stride_b * e, p->q_out_stride_h * e, p->q_out_stride_t * e};
  a->k = {nullptr, nullptr, p->k_stride_b * e, p->k_stride_h * e, p->k_stride_t * e, p->k_out_stride_b * e, p->k_out_stride_h * e, p->k_out_stride_t * e};
  for (int32_t i = 0; i < p->rotary_dim / 2; ++i) {
    a->turns[i] = turns_of(p->inv_freq[i]);
    a->axis[i] = (uint8_t)(p->axis_of_pair ? p->axis_of_pair[i] : 0);
  }
  a->batch = p->batch; a->n_tokens = p->n_tokens; a->q_heads = p->n_q_heads; a->kv_heads = p->n_kv_heads;
  a->d = p->head_dim; a->rotary = p->rotary_dim; a->dtype = p->dtype; a->n_axes = p->n_axes;
  a->interleaved = (p->flags & WKV_ROPE_INTERLEAVED) ? 1 : 0;
  a->amplitude = p->amplitude == 0.0 ? 1.0f : (float)p->amplitude;
  a->eps = p->eps;
  return WKV_OK;
}

// The checks of caches in 8 and 4 bits, and the decode step's key ranges: about 1280 workgroups if every cache were full, ranges of a multiple of 128 rows, a block for each of four
// waves.  With merge, us a call at 768 / 1024 / 1280 / 1536 and multiples of 64 / 2048, 32q/8kv heads of 128 channels, 8 bits: one sequence of 32768 rows 24.9 / 24.8 / 29.4 / 32.7 / 29.4, eight of 4128
// 21.9 / 21.9 / 24.5 / 24.8 / 24.6, 64 of 4128 91.6 / 92.3 / 92.0 / 96.2 / 97.7; in 4 bits 24 of mixed lengths 26.0 / 24.9 / 22.7 / 26.7 / 26.5, 28q/4kv 44 of them 27.0 / 25.4 / 22.6 / 25.5 / 26.1.  Over 30
// shapes, against the last but one: 6.1 % faster, 41 % slower at worst (16 caches of 3200 to 32000 rows) / 4.4, 19 / 3.3, 7 / - / 0.1, 20.
wkv_status plan_quantized(const wkv_quantized_shape *p, Decode *dc) {
  set_error("");
  if (!p) return invalid("shape is NULL");
  wkv_decode_shape s;
  std::memset(&s, 0, sizeof s);
  s.batch = p->batch; s.n_q_heads = p->n_q_heads; s.n_kv_heads = p->n_kv_heads; s.head_dim = p->head_dim; s.dtype = p->dtype; s.scale = p->scale;
  s.capacity = p->capacity; s.flags = p->flags;
  s.cache_stride_b = s.cache_stride_h = s.cache_stride_t = 128;                    // (the codes' own are checked below)
  const wkv_status st = validate_decode(&s, dc);
  if (st != WKV_OK) return st;
  if (p->format != WKV_CACHE_E4M3 && p->format != WKV_CACHE_E2M1) { set_error("unknown format %d", p->format); return WKV_ERR_INVALID_ARG; }
  if (p->capacity > 1 << 30) { set_error("capacity %d is not supported (at most 2^30 rows)", p->capacity); return WKV_ERR_UNSUPPORTED; }
  const int64_t row = p->format == WKV_CACHE_E4M3 ? p->head_dim : p->head_dim / 2;
  const int64_t strides[3] = {p->code_stride_b, p->code_stride_h, p->code_stride_t};
  for (const int64_t x : strides)
    if (x < 0 || x % 16 != 0 || x > MAX_STRIDE) return invalid("code strides must be non-negative multiples of 16 bytes, at most 2^48");
  if (p->code_stride_t < row || p->code_stride_h < row) { set_error("code token and head strides must be >= %lld bytes", (long long)row); return WKV_ERR_INVALID_ARG; }
  // (the rows of a block are addressed by 32-bit offsets)
  if (p->code_stride_t * 32 > 0x7fffffff) { set_error("code token stride %lld is not supported", (long long)p->code_stride_t); return WKV_ERR_UNSUPPORTED; }
  DecodeShape &c = dc->shape;
  c.sb = p->code_stride_b; c.sh = p->code_stride_h; c.st = p->code_stride_t;
  const int64_t rows = (int64_t)c.B * c.Hkv, most = std::min<int64_t>(std::max<int64_t>(1280 / rows, 1), DEC_MAX_SPLITS);
  c.chunk = (int32_t)(ceil_div(ceil_div(c.capacity, most), 128) * 128);
  c.n_splits = (int32_t)ceil_div(c.capacity, c.chunk);
  c.stats_at = (uint32_t)(rows * c.n_splits * c.G * c.d * (int64_t)sizeof(float));
  dc->ws_bytes = (size_t)rows * c.n_splits * c.G * (c.d + 2) * sizeof(float);
  return WKV_OK;
}

// Rows in and out of caches: checks, and everything of the launch but the pointers of the counts.
wkv_status plan_rows(const wkv_quantized_shape *p, int32_t n_layers, const void *const *k_plain, const void *const *v_plain, const void *const *k_codes,
                     const void *const *k_scales, const void *const *v_codes, const void *const *v_scales, QuantizedArgs *a, QuantizedLayers *layers) {
  Decode dc;
  const wkv_status st = plan_quantized(p, &dc);
  if (st != WKV_OK) return st;
  if (p->n_rows < 0) return invalid("n_rows must be >= 0");
  const DecodeShape &s = dc.shape;
  if ((int64_t)s.B * s.Hkv * p->n_rows > 1 << 30) { set_error("batch * n_kv_heads * n_rows exceeds 2^30; split the call"); return WKV_ERR_UNSUPPORTED; }
  if (!good_strides(p->dtype, p->head_dim, p->row_stride_b, p->row_stride_h, p->row_stride_t, "row")) return WKV_ERR_INVALID_ARG;
  if (n_layers < 1 || n_layers > WKV_MAX_LAYERS) { set_error("n_layers outside [1, %d]", WKV_MAX_LAYERS); return WKV_ERR_INVALID_ARG; }
  if (!k_plain || !v_plain || !k_codes || !k_scales || !v_codes || !v_scales) return invalid("an array of layers is NULL");
  std::memset(a, 0, sizeof *a);
  std::memset(layers, 0, sizeof *layers);
  for (int32_t l = 0; l < n_layers; ++l) {
    layers->plain[0][l] = k_plain[l]; layers->plain[1][l] = v_plain[l];
    layers->codes[0][l] = k_codes[l]; layers->codes[1][l] = v_codes[l];
    layers->scales[0][l] = k_scales[l]; layers->scales[1][l] = v_scales[l];
    for (int i = 0; i < 2; ++i) {
      if (!layers->plain[i][l] || !layers->codes[i][l] || !layers->scales[i][l]) { set_error("a tensor of layer %d is NULL", l); return WKV_ERR_INVALID_ARG; }
      if (misaligned(layers->plain[i][l], 16) || misaligned(layers->codes[i][l], 16)) { set_error("rows and codes of layer %d must be 16-byte aligned", l); return WKV_ERR_INVALID_ARG; }
      if (misaligned(layers->scales[i][l], 4)) { set_error("scales of layer %d must be 4-byte aligned", l); return WKV_ERR_INVALID_ARG; }
    }
  }
  const int64_t e = elem_bytes(p->dtype);
  a->heads = s.B * s.Hkv; a->Hkv = s.Hkv; a->d = s.d; a->dtype = s.dtype; a->format = p->format;
  a->capacity = s.capacity; a->n_rows = p->n_rows; a->row_capacity = p->row_capacity; a->kv_magic = s.kv_magic;
  a->c_sb = s.sb; a->c_sh = s.sh; a->c_st = s.st;
  a->r_sb = p->row_stride_b * e; a->r_sh = p->row_stride_h * e; a->r_st = p->row_stride_t * e;
  return WKV_OK;
}

}  // namespace

// How the work of a tree is cut: rows of a block and ranges of a cache, by an estimate of the time in us that takes every cache for nine tenths full.  Fitted to 34 shapes, each timed with up to
// fifteen numbers of ranges and every kind of block, before 16-bit types took a probability in two parts.  On the present kernels the cut that it takes is 4.3 % behind the best in the geometric
// mean, 15 % at worst and once 28 % (two sequences of 2000 and 1000 rows, 64 nodes, fp32: 12 ranges 68 us, 20 53); constants fitted anew 3.6 %.
//   blocks   of 64 rows (two pairs of waves, the waves of a pair share a tile's keys) where there are no more; of 128; of 256 where these fill the compute units
//            without ranges (64 sequences of 2000 rows and 64 nodes, 32q/8kv heads 221 us, by blocks of 128 251).  For 64 rows by blocks of 128: 16 nodes over 4128 rows, 64 sequences 192 us for
//            175, 32 of them 112 for 98, one the same.
//   ranges   one / two / four / eight / 16 / 32, us: 16 nodes over 4128 rows, one sequence 79 / 47 / 29 / 20 / 16.2 / 16.3, eight 81 / 51 / 39 / 41 / 48 / 55, 64 sequences
//            175 / 216 / 237 / ..
struct TreeCut {
  int32_t row_waves, key_waves, blocks, chunk, splits;
};
static TreeCut cut_tree(int64_t heads, int32_t n_rows, int32_t d, bool f32, int64_t capacity) {
  TreeCut best = {};
  double best_time = 1e300;
  for (const int32_t row_waves : {2, 4, 8}) {
    if (row_waves == 2 ? n_rows > 64 : row_waves == 4 ? n_rows <= 64 : n_rows <= 128 || f32) continue;
    TreeCut cut;
    cut.row_waves = row_waves;
    cut.key_waves = row_waves == 2 ? 2 : 1;
    cut.blocks = (int32_t)ceil_div(n_rows, row_waves * 32);
    const int64_t tiles = ceil_div(capacity, tree_wave_keys(f32, cut.key_waves) * cut.key_waves), groups = heads * cut.blocks;
    if (row_waves == 8 && groups < 256) continue;
    // workgroups at a time; a tile's time, alone on a compute unit and beside another
    const double slots = row_waves == 8 || (f32 && row_waves == 2 && d == 128) ? 256 : 512, size = d == 128 ? 1.0 : 0.62;
    const double alone = (f32 ? 3.6 : row_waves == 8 ? 2.0 : 1.25) * size, shared = (f32 ? 3.6 : row_waves == 8 ? 2.0 : 2.45) * size;
    for (const int32_t want : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      if (want > 1 && (want > tiles || groups * want > 2048 || row_waves == 8)) break;
      cut.chunk = (int32_t)ceil_div(tiles, want);
      cut.splits = (int32_t)ceil_div(tiles, cut.chunk);
      const double parts = cut.splits > 1 ? cut.splits * 0.9 + 1 : 1;          // workgroups of a block, the nodes' among them
      const double busy = std::min(std::max((groups * parts - 256) / 256, 0.0), 1.0);
      double time = std::max(groups * (tiles * 0.9 + 3.0 * parts + 3.4) * shared / slots, 5.6 + cut.chunk * (alone + (shared - alone) * busy));
      if (cut.splits > 1) time += 4.1 + (double)heads * n_rows * parts * (d * 8) / 4e6;
      if (time < best_time) { best_time = time; best = cut; }
    }
  }
  return best;
}

wkv_status plan_tree(const wkv_tree_shape *p, TreePlan *plan) {
  set_error("");
  if (!p) return invalid("shape is NULL");
  if (p->batch < 1) { set_error("batch must be >= 1 (got %d)", p->batch); return WKV_ERR_INVALID_ARG; }
  if (p->n_kv_heads < 1 || p->n_q_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) {
    set_error("n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads); return WKV_ERR_INVALID_ARG;
  }
  if ((int64_t)p->batch * p->n_kv_heads > 65535) { set_error("batch * n_kv_heads exceeds 65535 (launch grid limit); split the call"); return WKV_ERR_UNSUPPORTED; }
  const int32_t G = p->n_q_heads / p->n_kv_heads;
  if (G > 8) { set_error("n_q_heads / n_kv_heads = %d is not supported (at most 8)", G); return WKV_ERR_UNSUPPORTED; }
  if (!known_dtype(p->dtype)) return WKV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) { set_error("head_dim %d is not supported (64 or 128)", p->head_dim); return WKV_ERR_UNSUPPORTED; }
  if (!(p->scale >= 0.0f) || std::isinf(p->scale)) return invalid("scale must be finite and >= 0 (0 selects 1/sqrt(head_dim))");
  if (p->n_nodes < 1) { set_error("n_nodes must be >= 1 (got %d)", p->n_nodes); return WKV_ERR_INVALID_ARG; }
  if (p->n_nodes > WKV_MAX_NODES) { set_error("n_nodes %d exceeds WKV_MAX_NODES=%d", p->n_nodes, WKV_MAX_NODES); return WKV_ERR_UNSUPPORTED; }
  if (p->capacity < 1) return invalid("capacity must be >= 1");
  if (p->capacity > 1 << 30) { set_error("capacity %d is not supported (at most 2^30 rows)", p->capacity); return WKV_ERR_UNSUPPORTED; }
  if (p->flags & ~WKV_DECODE_KEEP_COUNT) { set_error("unknown bits in flags (0x%x)", p->flags); return WKV_ERR_INVALID_ARG; }
  if (!good_strides(p->dtype, p->head_dim, p->cache_stride_b, p->cache_stride_h, p->cache_stride_t, "cache") ||
      !good_strides(p->dtype, p->head_dim, p->q_stride_b, p->q_stride_h, p->q_stride_t, "q") ||
      !good_strides(p->dtype, p->head_dim, p->new_stride_b, p->new_stride_h, p->new_stride_t, "new") ||
      !good_strides(p->dtype, p->head_dim, p->out_stride_b, p->out_stride_h, p->out_stride_t, "out"))
    return WKV_ERR_INVALID_ARG;
  // (the rows that a wave fetches of a tile are addressed by 32-bit offsets)
  if (p->cache_stride_t * elem_bytes(p->dtype) * 64 > 0x7fffffff) { set_error("cache token stride %lld is not supported", (long long)p->cache_stride_t); return WKV_ERR_UNSUPPORTED; }
  if (p->new_stride_t * elem_bytes(p->dtype) * 64 > 0x7fffffff) { set_error("new token stride %lld is not supported", (long long)p->new_stride_t); return WKV_ERR_UNSUPPORTED; }
  std::memset(plan, 0, sizeof *plan);
  TreeArgs &a = plan->args;
  const bool f32 = p->dtype == WKV_F32;
  a.heads = p->batch * p->n_kv_heads; a.Hkv = p->n_kv_heads; a.G = G; a.d = p->head_dim; a.dtype = p->dtype; a.T = p->n_nodes; a.capacity = p->capacity;
  a.n_rows = a.T * G;
  a.heads_magic = division_magic(a.heads); a.kv_magic = division_magic(a.Hkv); a.g_magic = division_magic(G);
  const double scale = p->scale > 0.0f ? (double)p->scale : 1.0 / std::sqrt((double)p->head_dim);
  a.c1 = (float)(scale * 1.4426950408889634074);
  const int64_t e = elem_bytes(p->dtype);
  a.c_sb = p->cache_stride_b * e; a.c_sh = p->cache_stride_h * e; a.c_st = p->cache_stride_t * e;
  a.q_sb = p->q_stride_b * e; a.q_sh = p->q_stride_h * e; a.q_st = p->q_stride_t * e;
  a.n_sb = p->new_stride_b * e; a.n_sh = p->new_stride_h * e; a.n_st = p->new_stride_t * e;
  a.o_sb = p->out_stride_b * e; a.o_sh = p->out_stride_h * e; a.o_st = p->out_stride_t * e;
  const TreeCut cut = cut_tree(a.heads, a.n_rows, a.d, f32, a.capacity);
  plan->row_waves = cut.row_waves; plan->key_waves = cut.key_waves;
  a.blocks = cut.blocks; a.chunk = cut.chunk; a.splits = cut.splits;
  plan->streams = 2 * (int64_t)a.heads * a.capacity * a.d * e > MEMORY_CACHE_BYTES;
  const int32_t rows = plan->row_waves * 32;
  plan->ws_bytes = 256;
  if (a.splits > 1) {
    const size_t all = (size_t)a.heads * a.blocks * (a.splits + 1) * rows;
    plan->stats_at = all * a.d * sizeof(float);
    plan->ws_bytes = round_up(plan->stats_at + all * sizeof(float2));
  }
  return WKV_OK;
}

}  // namespace wkv

using namespace wkv;

extern "C" {

wkv_status wkv_norm_rope(const wkv_norm_rope_shape *shape, const int32_t *positions, const void *q_weight, const void *k_weight, const void *q_in,
                         void *q_out, const void *k_in, void *k_out, void *hip_stream) {
  NormRopeArgs a;
  const wkv_status st = plan_norm_rope(shape, &a);
  if (st != WKV_OK) return st;
  if (a.n_tokens == 0 || (a.q_heads == 0 && a.kv_heads == 0)) return WKV_OK;
  if (!positions) return invalid("positions is NULL");
  if (misaligned(positions, 4)) return invalid("positions must be 4-byte aligned");
  if (a.q_heads && (!q_in || !q_out)) return invalid("q_in / q_out is NULL");
  if (a.kv_heads && (!k_in || !k_out)) return invalid("k_in / k_out is NULL");
  if ((a.q_heads && (misaligned(q_in, 16) || misaligned(q_out, 16) || misaligned(q_weight, 16))) ||
      (a.kv_heads && (misaligned(k_in, 16) || misaligned(k_out, 16) || misaligned(k_weight, 16))))
    return invalid("the tensors and weights must be 16-byte aligned");
  a.q.in = q_in; a.q.out = q_out; a.k.in = k_in; a.k.out = k_out;
  for (const RopeTensor *t : {a.q_heads ? &a.q : nullptr, a.kv_heads ? &a.k : nullptr})
    if (t && t->in == t->out && (t->in_b != t->out_b || t->in_h != t->out_h || t->in_t != t->out_t))
      return invalid("in place, input and output strides must be the same");
  if (a.q_heads && a.kv_heads && q_out == k_out) return invalid("q_out and k_out are the same memory");
  a.positions = positions;
  a.q_weight = a.q_heads ? q_weight : nullptr; a.k_weight = a.kv_heads ? k_weight : nullptr;
  return launched(launch_norm_rope(a, (hipStream_t)hip_stream), "wkv_norm_rope");
}

wkv_status wkv_cache_quantize(const wkv_quantized_shape *shape, int32_t n_layers, const void *const *k_layers, const void *const *v_layers,
                              const int32_t *tok_idx, const int32_t *n_keep, const int32_t *first, void *const *k_codes, void *const *k_scales,
                              void *const *v_codes, void *const *v_scales, void *hip_stream) {
  QuantizedArgs a;
  QuantizedLayers layers;
  const wkv_status st = plan_rows(shape, n_layers, k_layers, v_layers, k_codes, k_scales, v_codes, v_scales, &a, &layers);
  if (st != WKV_OK) return st;
  if (shape->row_capacity < (tok_idx ? 0 : a.n_rows)) return invalid("row_capacity must be >= n_rows, or >= 0 with tok_idx");
  if (misaligned(tok_idx, 4) || misaligned(n_keep, 4) || misaligned(first, 4)) return invalid("tok_idx, n_keep and first must be 4-byte aligned");
  a.tok_idx = tok_idx; a.n_keep = n_keep; a.first = first;
  if (a.n_rows == 0 || a.row_capacity == 0) return WKV_OK;
  return launched(launch_quantize(a, layers, n_layers, (hipStream_t)hip_stream), "wkv_cache_quantize");
}

wkv_status wkv_cache_dequantize(const wkv_quantized_shape *shape, int32_t n_layers, const void *const *k_codes, const void *const *k_scales,
                                const void *const *v_codes, const void *const *v_scales, const int32_t *first, const int32_t *n_valid,
                                void *const *k_out, void *const *v_out, void *hip_stream) {
  QuantizedArgs a;
  QuantizedLayers layers;
  const wkv_status st = plan_rows(shape, n_layers, k_out, v_out, k_codes, k_scales, v_codes, v_scales, &a, &layers);
  if (st != WKV_OK) return st;
  if (misaligned(first, 4) || misaligned(n_valid, 4)) return invalid("first and n_valid must be 4-byte aligned");
  a.n_keep = n_valid; a.first = first;
  if (a.n_rows == 0) return WKV_OK;
  return launched(launch_dequantize(a, layers, n_layers, (hipStream_t)hip_stream), "wkv_cache_dequantize");
}

size_t wkv_decode_quantized_workspace_bytes(const wkv_quantized_shape *shape) {
  Decode dc;
  return plan_quantized(shape, &dc) == WKV_OK ? dc.ws_bytes : 0;
}

wkv_status wkv_decode_step_quantized(const wkv_quantized_shape *shape, const void *q_new, const void *k_new, const void *v_new, void *k_codes,
                                     void *k_scales, void *v_codes, void *v_scales, int32_t *n_valid, float *out, void *workspace,
                                     size_t workspace_bytes, void *hip_stream) {
  Decode dc;
  wkv_status st = plan_quantized(shape, &dc);
  if (st != WKV_OK) return st;
  if (!q_new || !k_new || !v_new || !k_codes || !k_scales || !v_codes || !v_scales || !n_valid || !out)
    return invalid("q_new / k_new / v_new / k_codes / k_scales / v_codes / v_scales / n_valid / out is NULL");
  if (misaligned(q_new, 16) || misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(k_codes, 16) || misaligned(v_codes, 16))
    return invalid("q_new, k_new, v_new and the codes must be 16-byte aligned");
  if (misaligned(k_scales, 4) || misaligned(v_scales, 4) || misaligned(n_valid, 4) || misaligned(out, 4))
    return invalid("the scales, n_valid and out must be 4-byte aligned");
  st = check_workspace(workspace, workspace_bytes, dc.ws_bytes);
  if (st != WKV_OK) return st;
  return launched(launch_decode_quantized(dc.shape, shape->format, q_new, k_new, v_new, k_codes, k_scales, v_codes, v_scales, n_valid, out,
                                          (float *)workspace, (hipStream_t)hip_stream), "wkv_decode_step_quantized");
}

size_t wkv_tree_workspace_bytes(const wkv_tree_shape *shape) {
  TreePlan plan;
  return plan_tree(shape, &plan) == WKV_OK ? plan.ws_bytes : 0;
}

wkv_status wkv_decode_tree(const wkv_tree_shape *shape, const void *q_new, const void *k_new, const void *v_new, const int32_t *parent, void *k_cache,
                           void *v_cache, const int32_t *n_valid, void *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
  TreePlan plan;
  wkv_status st = plan_tree(shape, &plan);
  if (st != WKV_OK) return st;
  if (!q_new || !k_new || !v_new || !parent || !k_cache || !v_cache || !n_valid || !out)
    return invalid("q_new / k_new / v_new / parent / k_cache / v_cache / n_valid / out is NULL");
  if (misaligned(q_new, 16) || misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(out, 16))
    return invalid("q_new, k_new, v_new, the caches and out must be 16-byte aligned");
  if (misaligned(parent, 4) || misaligned(n_valid, 4)) return invalid("parent and n_valid must be 4-byte aligned");
  if (out == q_new || out == k_new || out == v_new || out == k_cache || out == v_cache) return invalid("out must not overlap the inputs");
  st = check_workspace(workspace, workspace_bytes, plan.ws_bytes);
  if (st != WKV_OK) return st;
  return launched(launch_tree(plan, q_new, k_new, v_new, parent, k_cache, v_cache, n_valid, out, workspace, (hipStream_t)hip_stream), "wkv_decode_tree");
}

wkv_status wkv_tree_accept(const wkv_tree_shape *shape, int32_t n_layers, void *const *k_caches, void *const *v_caches, const int32_t *path,
                           const int32_t *n_accept, int32_t *n_valid, void *hip_stream) {
  TreePlan plan;
  const wkv_status st = plan_tree(shape, &plan);
  if (st != WKV_OK) return st;
  if (n_layers < 1 || n_layers > WKV_MAX_LAYERS) { set_error("n_layers outside [1, %d]", WKV_MAX_LAYERS); return WKV_ERR_INVALID_ARG; }
  if (!k_caches || !v_caches || !path || !n_accept || !n_valid) return invalid("k_caches / v_caches / path / n_accept / n_valid is NULL");
  if (misaligned(path, 4) || misaligned(n_accept, 4) || misaligned(n_valid, 4)) return invalid("path, n_accept and n_valid must be 4-byte aligned");
  EvictLayers layers;
  std::memset(&layers, 0, sizeof layers);
  for (int32_t l = 0; l < n_layers; ++l) {
    layers.k[l] = k_caches[l]; layers.v[l] = v_caches[l];
    if (!layers.k[l] || !layers.v[l]) { set_error("cache of layer %d is NULL", l); return WKV_ERR_INVALID_ARG; }
    if (misaligned(layers.k[l], 16) || misaligned(layers.v[l], 16)) { set_error("caches of layer %d must be 16-byte aligned", l); return WKV_ERR_INVALID_ARG; }
  }
  return launched(launch_accept(plan.args, layers, n_layers, path, n_accept, n_valid, (shape->flags & WKV_DECODE_KEEP_COUNT) != 0, (hipStream_t)hip_stream),
                  "wkv_tree_accept");
}

}  // extern "C"
