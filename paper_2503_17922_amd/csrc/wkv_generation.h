// Internal declarations of the operators of generation: norms with rotary positions, caches in 8 and 4 bits, trees of drafted
// tokens (not part of the ABI).
#pragma once

#include "wkv_operators.h"

namespace wkv {

// ---- norms with rotary positions ------------------------------------------------------------------
struct NormRopeArgs {
  uint64_t turns[ROPE_PAIRS];      // turns per position as a fraction of 2^64
  uint8_t axis[ROPE_PAIRS];        // whose position turns a pair
  RopeTensor q, k;
  const void *q_weight, *k_weight;
  const int32_t *positions;
  int32_t batch, n_tokens, q_heads, kv_heads, d, rotary, dtype, interleaved, n_axes;
  float amplitude, eps;
};
hipError_t launch_norm_rope(const NormRopeArgs &a, hipStream_t stream);

// ---- caches in 8 and 4 bits -----------------------------------------------------------------------
constexpr int32_t SCALE_GROUP = 32;      // channels that share a scale
struct QuantizedLayers {
  const void *plain[2][WKV_MAX_LAYERS];        // keys, values
  const void *codes[2][WKV_MAX_LAYERS], *scales[2][WKV_MAX_LAYERS];
};
struct QuantizedArgs {
  int32_t heads, Hkv, d, dtype, format;        // heads: sequences times KV heads
  int32_t capacity, n_rows, row_capacity;
  uint32_t kv_magic;                           // division_magic(Hkv)
  int64_t c_sb, c_sh, c_st, r_sb, r_sh, r_st;  // strides of codes and of plain rows in bytes
  const int32_t *tok_idx, *n_keep, *first;     // wkv_cache_dequantize: n_keep is its n_valid
  int32_t group;                               // of the launch: (sequence, KV head) pairs to a workgroup; division_magic(n_rows)
  uint32_t rows_magic;
  int32_t first_row;                           // of the launch, with rows of one pair to a workgroup
};
constexpr int32_t MOST_ROW_GROUPS = 1 << 22;   // workgroups of a launch along the rows: a grid holds fewer than 2^32 threads a dimension, so long calls are several launches
hipError_t launch_quantize(const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream);
hipError_t launch_dequantize(const QuantizedArgs &a, const QuantizedLayers &layers, int32_t n_layers, hipStream_t stream);

// The decode step: DecodeShape as for plain caches, its strides those of the codes in bytes.
hipError_t launch_decode_quantized(const DecodeShape &s, int32_t format, const void *q_new, const void *k_new, const void *v_new, void *k_codes,
                                   void *k_scales, void *v_codes, void *v_scales, int32_t *n_valid, float *out, float *part, hipStream_t stream);

// ---- trees of drafted tokens ----------------------------------------------------------------------
// A work item is a block of rows of one (sequence, KV head) and a range of its cache's key tiles: row r is node r / G for its query head r % G.  Waves
// of a workgroup: `row_waves` times 32 rows, each of them `key_waves` times, for a share of every tile.
struct TreeArgs {
  int32_t heads, Hkv, G, d, dtype, T, capacity;
  int32_t n_rows, blocks;                // T * G rows in `blocks` blocks
  int32_t chunk, splits;                 // key tiles of a range, ranges of a full cache
  uint32_t heads_magic, kv_magic, g_magic;
  float c1;                              // scale * log2(e)
  int64_t c_sb, c_sh, c_st, q_sb, q_sh, q_st, n_sb, n_sh, n_st, o_sb, o_sh, o_st;      // bytes
};
// Partial results in the workspace, with more than one range: outputs float [heads][blocks][splits + 1][rows of a block][d], the first of them those of the nodes' own
// rows, then their references and sums float2.
struct TreePlan {
  TreeArgs args;
  int32_t row_waves, key_waves;
  bool streams;                          // the caches exceed the memory-side cache
  size_t stats_at, ws_bytes;
};
constexpr int32_t tree_wave_keys(bool f32, int32_t key_waves) { return f32 || key_waves > 1 ? 32 : 64; }      // keys of a tile that a wave takes
wkv_status plan_tree(const wkv_tree_shape *p, TreePlan *plan);
hipError_t launch_tree(const TreePlan &plan, const void *q, const void *kn, const void *vn, const int32_t *parent, void *kc, void *vc,
                       const int32_t *n_valid, void *out, void *workspace, hipStream_t stream);
hipError_t launch_accept(const TreeArgs &a, const EvictLayers &layers, int32_t n_layers, const int32_t *path, const int32_t *n_accept,
                         int32_t *n_valid, bool keep_count, hipStream_t stream);

}  // namespace wkv
