// Internal declarations of the operators around the compression: rotary positions, the prompt's attention, the decode
// step that accumulates attention weights, eviction (not part of the ABI).
#pragma once

#include "wkv_internal.h"

namespace wkv {

// ---- rotary positions ---------------------------------------------------------------------------
constexpr int32_t ROPE_PAIRS = 64;        // pairs of channels of a head, at most
struct RopeTensor {
  const void *in;
  void *out;
  int64_t in_b, in_h, in_t, out_b, out_h, out_t;   // strides in bytes
};
struct RopeArgs {
  uint64_t turns[ROPE_PAIRS];      // turns per token as a fraction of 2^64: position * turns modulo 2^64 is the angle
  RopeTensor q, k;
  const int32_t *positions;
  int32_t batch, n_tokens, q_heads, kv_heads, d, rotary, dtype, interleaved, inverse;
  float amplitude;
};
wkv_status plan_rope(const wkv_rope_shape *p, RopeArgs *a);
hipError_t launch_rope(const RopeArgs &a, hipStream_t stream);

// ---- attention over a prompt --------------------------------------------------------------------
// A work item is a block of 128 or 256 rows of one (sequence, KV head): row r is query r / G of its query head r % G, so that the heads of
// a KV head share the key tiles.  (Both sides of the launch go by these: a kernel that took other blocks or tiles than the plan has would
// write past the workspace.)
constexpr int32_t ATT_ROWS = 256, ATT_ROWS_FEW = 128;
constexpr int32_t att_tile_keys(bool f32) { return f32 ? 32 : 64; }      // keys of a tile
constexpr int32_t ATT_MAX = 1 << 30;     // most rows of a (sequence, KV head), and most keys
struct AttentionSeq {
  int32_t b, q_len, k_len, blocks;       // blocks of AttentionPlan::rows rows
  int64_t q_start, k_start;
};
struct AttentionArgs {
  // Longest first: sequences in descending order of their blocks, and items by block number from the top.  Segment s holds the
  // levels at which the first s+1 sequences have a block: ends[s] is the first item after it.
  int32_t ends[WKV_MAX_BATCH];
  AttentionSeq seq[WKV_MAX_BATCH];
  int32_t n_seqs, Hq, Hkv, G, d, dtype, lse_rows;
  uint32_t g_magic;                      // division_magic(G)
  float c1;                              // scale * log2(e)
  int64_t q_sb, q_sh, q_st, kv_sb, kv_sh, kv_st, o_sb, o_sh, o_st;      // bytes
  int32_t chunk, splits;                 // key tiles of a workgroup, workgroups of a block with the most tiles (see plan_attention)
  int32_t fold_from, fold_parts;         // from these workgroups on the items go the other way round (wkv_attention.hip, item_of)
};
// Partial results in the workspace, of blocks that more than one workgroup shares: outputs float [items][splits][rows][d], then
// their references and sums float2 [items][splits][rows], both without the last items, those of sequences that have no rows.
struct AttentionPlan {
  AttentionArgs args;
  int32_t items, rows, most_rows;        // blocks, their rows, and the most that any of them has
  size_t stats_at, ws_bytes;
};
wkv_status plan_attention(const wkv_attention_shape *p, AttentionPlan *plan);
hipError_t launch_attention(const AttentionPlan &plan, const void *q, const void *k, const void *v, void *out, float *lse, void *workspace,
                            hipStream_t stream);

// ---- decode step with weights ---------------------------------------------------------------------
// Whether one workgroup takes all rows of a (sequence, KV head), whose logits stay in its LDS, instead of ranges of them: with two workgroups to a compute unit,
// 80 KB each.
constexpr int32_t WHOLE_THREADS = 512, WHOLE_FLOATS = 20224;
bool decode_takes_whole_caches(const DecodeShape &s);
// Behind the partial results in the workspace: the row counts of this step, int32 [B*Hkv], then the logits (base 2),
// float [B*Hkv][n_splits * chunk / 16][G][16].
struct DecodeWeights {
  float *weights;
  int32_t *tok_idx;
  const int32_t *position;
  int32_t *counts;
  float *logits;
  const void *k_new, *v_new;             // and these where one launch does the whole step
  int32_t *n_valid;
  float *out;
};
size_t decode_weighted_layout(const DecodeShape &s, size_t partial_bytes, size_t *counts_at, size_t *logits_at);
hipError_t launch_decode_weighted(const DecodeShape &s, const void *q_new, const void *k_new, const void *v_new, void *k_cache,
                                  void *v_cache, int32_t *n_valid, const DecodeWeights &w, float *out, float *part, hipStream_t stream);

// ---- eviction -------------------------------------------------------------------------------------
struct EvictLayers {
  void *k[WKV_MAX_LAYERS], *v[WKV_MAX_LAYERS];
};
struct EvictArgs {
  int32_t rows;              // B * Hkv
  int32_t Hkv, capacity, recent, row_bytes;
  uint32_t hkv_magic;
  int64_t sb, sh, st;        // cache strides in bytes
  int32_t max_moves;         // room of a list of moves
};
// Workspace: int32 [rows] numbers of moves, then (from, to) int2 [rows][max_moves].
size_t evict_layout(int32_t rows, int32_t max_moves, size_t *moves_at);
hipError_t launch_evict(const EvictArgs &a, const EvictLayers &layers, int32_t n_layers, float *weights, int32_t *tok_idx, int32_t *n_valid,
                        const int32_t *keep, int32_t *counts, int2 *moves, hipStream_t stream);

}  // namespace wkv
