// Host side of the operators around the compression: argument validation, derived sizes, launch plans and the entry points.
// Nothing in this file but the launchers' calls touches the GPU.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "wkv_operators.h"

namespace wkv {

namespace {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

wkv_status invalid(const char *what) { set_error("%s", what); return WKV_ERR_INVALID_ARG; }
wkv_status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return WKV_OK;
  set_error("%s launch: %s", what, hipGetErrorString(e));
  return WKV_ERR_HIP;
}
bool known_dtype(int32_t dtype) {
  if (dtype == WKV_F32 || dtype == WKV_BF16 || dtype == WKV_F16) return true;
  set_error("unknown dtype %d", dtype);
  return false;
}
// Row starts at multiples of 16 bytes, rows of head_dim channels that do not overlap.
bool good_strides(int32_t dtype, int32_t head_dim, int64_t sb, int64_t sh, int64_t st, const char *what) {
  const int64_t vec = 16 / elem_bytes(dtype);
  if (sb < 0 || sh < 0 || st < 0 || sb % vec != 0 || sh % vec != 0 || st % vec != 0) {
    set_error("%s strides must be non-negative multiples of %lld elements (16 bytes)", what, (long long)vec);
    return false;
  }
  if (std::max({sb, sh, st}) > MAX_STRIDE) { set_error("%s strides must be at most 2^48 elements", what); return false; }
  if (st < head_dim || sh < head_dim) { set_error("%s token and head strides must be >= head_dim", what); return false; }
  return true;
}
wkv_status check_workspace(const void *ws, size_t bytes, size_t needed) {
  if (!ws) { set_error("workspace is NULL"); return WKV_ERR_WORKSPACE; }
  if (misaligned(ws, 256)) { set_error("workspace must be 256-byte aligned"); return WKV_ERR_WORKSPACE; }
  if (bytes < needed) { set_error("workspace has %zu bytes, %zu needed", bytes, needed); return WKV_ERR_WORKSPACE; }
  return WKV_OK;
}

// An angular frequency as turns per token modulo one, in units of 2^-64 turns.  In integers, as 64 divisions of 80-bit floats take 3 us: a double is
// m * 2^e, and 1 / (2 pi) is TURN * 2^-66 with 64 significant bits.  (A position of 2^31 leaves an error of 2^-33 turns of
// the frequency's own 53 bits.)
uint64_t turns_of(double inv_freq) {
  constexpr uint64_t TURN = 0xa2f9836e4e441529ull;
  uint64_t bits;
  std::memcpy(&bits, &inv_freq, 8);
  const int exponent = (int)(bits >> 52 & 0x7ff);
  const uint64_t mantissa = (bits & 0xfffffffffffffull) | (exponent ? 1ull << 52 : 0);
  const int shift = 66 - 64 - ((exponent ? exponent : 1) - 1075);        // turns * 2^64 = mantissa * TURN * 2^-shift
  const unsigned __int128 product = (unsigned __int128)mantissa * TURN;
  uint64_t turns = 0;
  if (shift <= 0) turns = shift > -64 ? (uint64_t)product << -shift : 0;
  else if (shift < 128) turns = (uint64_t)(product >> shift) + (uint64_t)(product >> (shift - 1) & 1);
  return bits >> 63 ? 0 - turns : turns;
}

wkv_status plan_rope(const wkv_rope_shape *p, RopeArgs *a) {
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
  if (p->flags & ~(WKV_ROPE_INTERLEAVED | WKV_ROPE_INVERSE)) { set_error("unknown bits in flags (0x%x)", p->flags); return WKV_ERR_INVALID_ARG; }
  if (!std::isfinite(p->amplitude) || std::fabs(p->amplitude) > 3.0e38) return invalid("amplitude must be finite (0 selects 1)");
  if (!p->inv_freq) return invalid("inv_freq must be a non-NULL host array");
  for (int32_t i = 0; i < p->rotary_dim / 2; ++i)
    if (!std::isfinite(p->inv_freq[i])) { set_error("inv_freq[%d] is not finite", i); return WKV_ERR_INVALID_ARG; }
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
  for (int32_t i = 0; i < p->rotary_dim / 2; ++i) a->turns[i] = turns_of(p->inv_freq[i]);
  a->batch = p->batch; a->n_tokens = p->n_tokens; a->q_heads = p->n_q_heads; a->kv_heads = p->n_kv_heads;
  a->d = p->head_dim; a->rotary = p->rotary_dim; a->dtype = p->dtype;
  a->interleaved = (p->flags & WKV_ROPE_INTERLEAVED) ? 1 : 0;
  a->inverse = (p->flags & WKV_ROPE_INVERSE) ? 1 : 0;
  a->amplitude = p->amplitude == 0.0 ? 1.0f : (float)p->amplitude;
  return WKV_OK;
}

// How the work is cut: blocks of 128 or 256 rows, and `splits` workgroups that share the key tiles of a block where the blocks alone do not fill the device (a
// second launch joins their results).  By an estimate of the time in us, fitted to some forty shapes, of which it takes the best cut or one within a
// few percent of it (a sixth at worst): a workgroup of 256 rows has a compute unit for itself, two of 128 share one and take twice as long; every workgroup has a
// start, and every partial result is written and read.  us by blocks of 128 / 256 rows, 32q/8kv heads of 128 channels, bf16, each with its best number of
// splits: 128 tokens 7.7 / 9.9, 1024 24.1 / 28.1, 2048 47.4 / 57.7, 4096 146 / 132, 200 tokens over 20000 86 / 84, 1024 over 20000 318 / 300; whole / cut
// in its best number: one token over 20000 320 / 19.5, 512 tokens of 12q/2kv heads 14.3 / 12.6, 4096 of these 84 / 80, 2048 in fp32 278 / 315, 1024 139 / 89.
struct AttentionCut {
  int32_t rows, chunk, splits;
};
// (The key tiles of a sequence's blocks rise evenly from the first block's to the last one's, so sums over them need no loop.)
static AttentionCut cut_attention(const wkv_attention_shape *p) {
  const int64_t G = p->n_q_heads / p->n_kv_heads, Hkv = p->n_kv_heads;
  const bool f32 = p->dtype == WKV_F32;
  const int32_t keys = att_tile_keys(f32);
  constexpr double UNITS = 256.0;               // compute units
  constexpr int32_t WHOLE = 0x7fffffff;
  AttentionCut best = {f32 ? ATT_ROWS_FEW : ATT_ROWS, WHOLE, 1};
  double best_time = 1e300;
  struct { double n, least, most; } blocks[WKV_MAX_BATCH];
  for (const int32_t rows : {ATT_ROWS_FEW, ATT_ROWS}) {
    if (f32 && rows != ATT_ROWS_FEW) continue;
    const double tile = (p->head_dim == 128 ? 1.0 : 0.62) * (f32 ? 3.4 : rows == ATT_ROWS ? 1.75 : 1.15), start = rows == ATT_ROWS ? 5.0 : 4.0;
    double n_blocks = 0, total = 0;
    int64_t most = 0;
    for (int32_t b = 0; b < p->batch; ++b) {
      const int64_t q_len = p->q_len[b], k_len = p->k_len ? p->k_len[b] : q_len;
      auto tiles = [&](int64_t last) { return ceil_div(std::min(std::max<int64_t>(last / G + k_len - q_len + 1, 0), k_len), (int64_t)keys); };
      const int64_t top = q_len > 0 ? tiles(q_len * G - 1) : 0;
      blocks[b] = {(double)(ceil_div(q_len * G, rows) * Hkv), q_len > 0 ? (double)tiles(std::min<int64_t>(rows, q_len * G) - 1) : 0.0, (double)top};
      n_blocks += blocks[b].n;
      total += blocks[b].n * (blocks[b].least + blocks[b].most) / 2;
      most = std::max(most, top);
    }
    for (const int32_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (want > 1 && (want > most || n_blocks * want > 4096)) break;
      const double chunk = want == 1 ? std::max<double>((double)most, 1) : (double)ceil_div(most, want);
      double parts = 0, joined = 0, full = 0;             // workgroups, rows of partial results, workgroups with a whole chunk
      for (int32_t b = 0; b < p->batch; ++b) {
        const double n = blocks[b].n, lo = blocks[b].least, hi = blocks[b].most;
        if (hi <= chunk) { parts += n; full += lo == hi && hi == chunk ? n : 0; continue; }
        const double mean = (lo + hi) / 2 / chunk, cut = lo >= chunk ? 1.0 : (hi - chunk) / (hi - lo);     // share of the blocks that are cut
        const double pieces = lo == hi ? std::ceil(mean) : mean + 0.5;
        parts += n * pieces; joined += n * (cut * pieces) * std::min<double>(rows, (double)p->q_len[b] * (double)G); full += n * (lo == hi ? std::floor(mean) : std::max(mean - 0.5, 0.0));
      }
      double time = start + tile * std::max(chunk, total / UNITS) + 2.0 * parts / UNITS;
      if (want > 1) {
        if (rows == ATT_ROWS) time = std::max(time, start + tile * chunk * std::ceil(full / UNITS));      // (equal ones: whole rounds)
        time += 5.0 + joined * p->head_dim * 4 * 2 / 4e6 + 0.35 * tile * chunk * std::min(std::max(parts / UNITS - 1.0, 0.0), 1.0);
      }
      if (time < best_time) { best_time = time; best = {rows, want == 1 ? WHOLE : (int32_t)chunk, want == 1 ? 1 : (int32_t)ceil_div(most, (int64_t)chunk)}; }
    }
  }
  return best;
}

wkv_status plan_attention(const wkv_attention_shape *p, AttentionPlan *plan) {
  set_error("");
  if (!p) return invalid("shape is NULL");
  if (!p->q_len) return invalid("q_len must be a non-NULL host array");
  if (p->batch < 1) { set_error("batch must be >= 1 (got %d)", p->batch); return WKV_ERR_INVALID_ARG; }
  if (p->batch > WKV_MAX_BATCH) { set_error("batch %d exceeds WKV_MAX_BATCH=%d; split the call", p->batch, WKV_MAX_BATCH); return WKV_ERR_UNSUPPORTED; }
  if (p->n_kv_heads < 1 || p->n_q_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) {
    set_error("n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads); return WKV_ERR_INVALID_ARG;
  }
  if (!known_dtype(p->dtype)) return WKV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) { set_error("head_dim %d is not supported (64 or 128)", p->head_dim); return WKV_ERR_UNSUPPORTED; }
  if (!(p->scale >= 0.0f) || std::isinf(p->scale)) return invalid("scale must be finite and >= 0 (0 selects 1/sqrt(head_dim))");
  if (p->lse_rows < 0) return invalid("lse_rows must be >= 0");
  if ((int64_t)p->lse_rows * (p->n_q_heads / p->n_kv_heads) > ATT_MAX) { set_error("lse_rows %d is not supported", p->lse_rows); return WKV_ERR_UNSUPPORTED; }
  if (p->flags != 0) { set_error("unknown bits in flags (0x%x)", p->flags); return WKV_ERR_INVALID_ARG; }
  if (!good_strides(p->dtype, p->head_dim, p->q_stride_b, p->q_stride_h, p->q_stride_t, "q") ||
      !good_strides(p->dtype, p->head_dim, p->kv_stride_b, p->kv_stride_h, p->kv_stride_t, "K and V") ||
      !good_strides(p->dtype, p->head_dim, p->out_stride_b, p->out_stride_h, p->out_stride_t, "out"))
    return WKV_ERR_INVALID_ARG;
  // (the rows that a wave fetches of a tile are addressed by 32-bit offsets)
  if (p->kv_stride_t * elem_bytes(p->dtype) * 64 > 0x7fffffff) { set_error("K and V token stride %lld is not supported", (long long)p->kv_stride_t); return WKV_ERR_UNSUPPORTED; }
  AttentionArgs &a = plan->args;
  std::memset(plan, 0, sizeof(*plan));
  a.Hq = p->n_q_heads; a.Hkv = p->n_kv_heads; a.G = a.Hq / a.Hkv; a.d = p->head_dim; a.dtype = p->dtype; a.lse_rows = p->lse_rows;
  a.n_seqs = p->batch;
  const double scale = p->scale > 0.0f ? (double)p->scale : 1.0 / std::sqrt((double)p->head_dim);
  a.c1 = (float)(scale * 1.4426950408889634074);
  const int64_t e = elem_bytes(p->dtype);
  a.q_sb = p->q_stride_b * e; a.q_sh = p->q_stride_h * e; a.q_st = p->q_stride_t * e;
  a.kv_sb = p->kv_stride_b * e; a.kv_sh = p->kv_stride_h * e; a.kv_st = p->kv_stride_t * e;
  a.o_sb = p->out_stride_b * e; a.o_sh = p->out_stride_h * e; a.o_st = p->out_stride_t * e;
  for (int32_t b = 0; b < p->batch; ++b) {
    AttentionSeq &s = a.seq[b];
    s.b = b; s.q_len = p->q_len[b]; s.k_len = p->k_len ? p->k_len[b] : p->q_len[b];
    s.q_start = p->q_start ? p->q_start[b] : 0; s.k_start = p->k_start ? p->k_start[b] : 0;
    if (s.q_len < 0 || s.k_len < 0) { set_error("q_len[%d] = %d, k_len[%d] = %d: lengths must be >= 0", b, s.q_len, b, s.k_len); return WKV_ERR_INVALID_ARG; }
    if (s.q_start < 0 || s.k_start < 0) { set_error("q_start[%d] and k_start[%d] must be >= 0", b, b); return WKV_ERR_INVALID_ARG; }
    // (rows are divided by G through multiplication: row * G < 2^32)
    if ((int64_t)s.q_len * a.G > ATT_MAX || s.k_len > ATT_MAX || ((int64_t)s.q_len * a.G + ATT_ROWS) * a.G > 0xffffffffll) {
      set_error("sequence %d has too many rows or keys; split the call", b); return WKV_ERR_UNSUPPORTED;
    }
    plan->most_rows = (int32_t)std::max<int64_t>(plan->most_rows, (int64_t)s.q_len * a.G);
  }
  const AttentionCut cut = cut_attention(p);
  plan->rows = cut.rows;
  plan->most_rows = std::min(plan->most_rows, cut.rows);
  // (a sequence without rows has a block for the normalisers of rows that do not exist)
  for (int32_t b = 0; b < p->batch; ++b)
    a.seq[b].blocks = (int32_t)std::max<int64_t>(ceil_div((int64_t)a.seq[b].q_len * a.G, plan->rows), p->lse_rows > 0 ? 1 : 0);
  // (and goes last: its block leaves no partial results and has no room for any)
  std::sort(a.seq, a.seq + p->batch, [](const AttentionSeq &x, const AttentionSeq &y) {
    if (x.blocks != y.blocks) return x.blocks > y.blocks;
    return (x.q_len == 0) != (y.q_len == 0) ? y.q_len == 0 : x.b < y.b;
  });
  int64_t items = 0, idle = 0;
  for (int32_t b = 0; b < p->batch; ++b) idle += a.seq[b].q_len == 0 ? (int64_t)a.seq[b].blocks * a.Hkv : 0;
  for (int32_t i = 0; i < WKV_MAX_BATCH; ++i) {
    if (i < p->batch) items += (int64_t)(a.seq[i].blocks - (i + 1 < p->batch ? a.seq[i + 1].blocks : 0)) * (i + 1) * a.Hkv;
    if (items > 1 << 23) { set_error("more than 2^23 blocks of %d rows; split the call", plan->rows); return WKV_ERR_UNSUPPORTED; }      // (launch grid limit)
    a.ends[i] = (int32_t)items;
  }
  plan->items = (int32_t)items;
  a.g_magic = division_magic(a.G);
  a.chunk = cut.chunk; a.splits = cut.splits;
  a.fold_from = plan->rows == ATT_ROWS_FEW && a.splits == 1 && items > 256 && items <= 512 && items % 8 == 0 ? 256 : 0x7fffffff;
  a.fold_parts = items % 8 == 0 ? 0 : 0x7fffffff;
  plan->ws_bytes = 256;
  if (a.splits > 1) {
    const size_t rows = (size_t)(items - idle) * a.splits * plan->rows;        // at most 2^20: 4096 workgroups of 256 rows (cut_attention)
    plan->stats_at = rows * a.d * sizeof(float);
    plan->ws_bytes = round_up(plan->stats_at + rows * sizeof(float2));
  }
  return WKV_OK;
}

size_t decode_weighted_layout(const DecodeShape &s, size_t partial_bytes, size_t *counts_at, size_t *logits_at) {
  const size_t rows = (size_t)s.B * s.Hkv;
  *counts_at = round_up(partial_bytes);
  *logits_at = round_up(*counts_at + rows * sizeof(int32_t));
  return *logits_at + rows * s.G * s.n_splits * s.chunk * sizeof(float);
}

// Where the pairs of sequence and KV head fill the compute units, one or two to each, or their caches are short, and the logits of full caches fit into half a unit's LDS.  The
// logits make no trip through memory then (34 MB written among the rows' reads cost the launch of 64 sequences 20 of 187 us), and there is no second
// launch; but nobody takes over a long cache's rows.  us by ranges / so, 32q/8kv heads of 128 channels, 4128 rows, three sets of caches in turn: 16 sequences 60 / 66, 20 71 / 68, 28
// 97 / 81, 32 107 / 92, 34 118 / 133, 44 148 / 145, 52 168 / 160, 64 203 / 179, 128 411 / 361; 4383 rows, 65 243 / 232, 72 254 / 241, 88 309 / 260, 144 518 / 440; 1000 rows, 32
// 33.0 / 26.7, 52 48 / 42, 64 59 / 48, 65 60 / 58, 129 114 / 101; mixed, 500 to 4000 rows, 24 57 / 59, 28 68 / 65, 32 83 / 72, 48 92 / 103, 52 113 / 105, 64 133 / 119; 64 channels,
// 64q/8kv, 2000 rows, 32 40 / 34, 64 70 / 54.
// How many rows a cache has is on the device, and a single long one among short ones loses by this: all caches full, mixed (an eighth on), one full among caches of 8
// rows: 32 sequences of 5055 rows 131 / 111, 86 / 81, 25 / 58, 64 of them 253 / 220, 183 / 157, 37 / 58; 16q/8kv, 10111 rows, 32 241 / 214, 156 / 153, 45 / 105, 64
// 479 / 428, 331 / 302, 58 / 105.  Past that, where 128 channels of one query head alone could go, there is little to gain: 8q/8kv, 20223 rows, 32 460 / 431, 284 / 299, 85 / 202, 64
// 919 / 857, 619 / 598, 108 / 203; 64 channels, 64 of them 555 / 458, 402 / 327, 78 / 108.
// Nor is there much to take over where every wave's rows are one trip to memory: one sequence of 60 rows 7.9 / 5.1, 250 8.9 / 7.3, 380 8.6 / 9.1, 1000
// 8.6 / 15.3, twelve of 60 7.8 / 5.2, of 250 9.7 / 7.9, of 380 12.1 / 11.5.  With 128 channels and more than four heads the registers of two
// workgroups a unit do not suffice.
bool decode_takes_whole_caches(const DecodeShape &s) {
  constexpr int32_t UNITS = 256;
  if (s.dtype == WKV_F32 || (s.d == 128 && s.G > 4)) return false;
  const int32_t rows = s.B * s.Hkv;
  const bool a_round = s.capacity <= WHOLE_THREADS / 64 * 32, fills = (rows >= UNITS * 7 / 8 && rows <= UNITS) || rows >= UNITS * 13 / 8;
  return (a_round || fills) && ceil_div(s.capacity, 16) * 16 * std::max(s.G, s.d / 64) <= WHOLE_FLOATS;
}

size_t evict_layout(int32_t rows, int32_t max_moves, size_t *moves_at) {
  *moves_at = round_up((size_t)rows * sizeof(int32_t));
  return *moves_at + (size_t)rows * max_moves * sizeof(int2);
}
// (row numbers and the ends of key ranges stay below 2^31)
static wkv_status validate_cache(const wkv_decode_shape *shape, Decode *dc) {
  const wkv_status st = validate_decode(shape, dc);
  if (st != WKV_OK) return st;
  if (std::max({dc->shape.sb, dc->shape.sh, dc->shape.st}) > MAX_STRIDE) { set_error("cache strides must be at most 2^48 elements"); return WKV_ERR_INVALID_ARG; }
  if (dc->shape.capacity <= 1 << 30) return WKV_OK;
  set_error("capacity %d is not supported (at most 2^30 rows)", dc->shape.capacity);
  return WKV_ERR_UNSUPPORTED;
}

// keep + (n - keep) rows of at most `capacity`: as many moves as the smaller part.
static int32_t max_moves(int32_t capacity) { return std::max(capacity / 2, 1); }

}  // namespace wkv

using namespace wkv;

extern "C" {

wkv_status wkv_rope(const wkv_rope_shape *shape, const int32_t *positions, const void *q_in, void *q_out, const void *k_in, void *k_out,
                    void *hip_stream) {
  RopeArgs a;
  const wkv_status st = plan_rope(shape, &a);
  if (st != WKV_OK) return st;
  if (a.n_tokens == 0 || (a.q_heads == 0 && a.kv_heads == 0)) return WKV_OK;
  if (!positions) return invalid("positions is NULL");
  if (misaligned(positions, 4)) return invalid("positions must be 4-byte aligned");
  if (a.q_heads && (!q_in || !q_out)) return invalid("q_in / q_out is NULL");
  if (a.kv_heads && (!k_in || !k_out)) return invalid("k_in / k_out is NULL");
  if ((a.q_heads && (misaligned(q_in, 16) || misaligned(q_out, 16))) || (a.kv_heads && (misaligned(k_in, 16) || misaligned(k_out, 16))))
    return invalid("the tensors must be 16-byte aligned");
  a.q.in = q_in; a.q.out = q_out; a.k.in = k_in; a.k.out = k_out;
  for (const RopeTensor *t : {a.q_heads ? &a.q : nullptr, a.kv_heads ? &a.k : nullptr})
    if (t && t->in == t->out && (t->in_b != t->out_b || t->in_h != t->out_h || t->in_t != t->out_t))
      return invalid("in place, input and output strides must be the same");
  if (a.q_heads && a.kv_heads && q_out == k_out) return invalid("q_out and k_out are the same memory");
  a.positions = positions;
  return launched(launch_rope(a, (hipStream_t)hip_stream), "wkv_rope");
}

wkv_status wkv_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, int32_t original_len, double *inv_freq_out,
                                double *amplitude_out) {
  set_error("");
  if (!inv_freq_out || !amplitude_out) return invalid("inv_freq_out / amplitude_out is NULL");
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > 65536) return invalid("rotary_dim must be even, 2 .. 65536");
  if (!(theta > 1.0) || std::isinf(theta)) return invalid("theta must be finite and > 1");
  if (scaling < WKV_ROPE_PLAIN || scaling > WKV_ROPE_WAVELENGTH) { set_error("unknown scaling %d", scaling); return WKV_ERR_INVALID_ARG; }
  if (scaling != WKV_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return invalid("factor must be finite and >= 1");
  if ((scaling == WKV_ROPE_PARTS || scaling == WKV_ROPE_WAVELENGTH) && original_len < 1) return invalid("original_len must be >= 1");
  if (scaling == WKV_ROPE_BASE && rotary_dim < 4) return invalid("WKV_ROPE_BASE needs a rotary_dim of at least 4");
  const double r = rotary_dim, turn = 6.283185307179586477;
  const double base = scaling == WKV_ROPE_BASE ? theta * std::pow(factor, r / (r - 2.0)) : theta;
  // channel number (in pairs, real) that turns n times within the original context
  auto channel_of = [&](double n) { return r * std::log(original_len / (n * turn)) / (2.0 * std::log(theta)); };
  double lo = 0.0, hi = 0.0;
  if (scaling == WKV_ROPE_PARTS) {
    lo = std::max(std::floor(channel_of(32.0)), 0.0);
    hi = std::min(std::ceil(channel_of(1.0)), r - 1.0);
    if (hi <= lo) hi = lo + 0.001;
  }
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / r);
    double share = 1.0;                                  // of the unchanged frequency
    if (scaling == WKV_ROPE_LINEAR) share = 0.0;
    if (scaling == WKV_ROPE_PARTS) share = 1.0 - std::min(std::max((i - lo) / (hi - lo), 0.0), 1.0);
    if (scaling == WKV_ROPE_WAVELENGTH) share = std::min(std::max((original_len * f / turn - 1.0) / (4.0 - 1.0), 0.0), 1.0);
    inv_freq_out[i] = share == 1.0 ? f : f * share + f / factor * (1.0 - share);
  }
  *amplitude_out = scaling == WKV_ROPE_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return WKV_OK;
}

size_t wkv_attention_workspace_bytes(const wkv_attention_shape *shape) {
  AttentionPlan plan;
  return plan_attention(shape, &plan) == WKV_OK ? plan.ws_bytes : 0;
}

wkv_status wkv_prefill_attention(const wkv_attention_shape *shape, const void *q, const void *k, const void *v, void *out, float *lse_out,
                                 void *workspace, size_t workspace_bytes, void *hip_stream) {
  AttentionPlan plan;
  wkv_status st = plan_attention(shape, &plan);
  if (st != WKV_OK) return st;
  // (tensors without elements may have no address)
  bool rows = false, pairs = false;
  for (int32_t i = 0; i < plan.args.n_seqs; ++i) {
    const AttentionSeq &sq = plan.args.seq[i];
    rows |= sq.q_len > 0; pairs |= sq.q_len > 0 && sq.k_len > 0;
  }
  if ((rows && (!q || !out)) || (pairs && (!k || !v))) return invalid("q / k / v / out is NULL");
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16)) return invalid("q, k, v and out must be 16-byte aligned");
  if (plan.args.lse_rows > 0 && !lse_out) return invalid("lse_out is NULL and lse_rows is not 0");
  if (misaligned(lse_out, 4)) return invalid("lse_out must be 4-byte aligned");
  if (out && (out == q || out == k || out == v)) return invalid("out must not overlap the inputs");
  st = check_workspace(workspace, workspace_bytes, plan.ws_bytes);
  if (st != WKV_OK) return st;
  if (plan.items == 0) return WKV_OK;
  return launched(launch_attention(plan, q, k, v, out, lse_out, workspace, (hipStream_t)hip_stream), "wkv_prefill_attention");
}

size_t wkv_decode_weighted_workspace_bytes(const wkv_decode_shape *shape) {
  Decode dc;
  size_t counts_at, logits_at;
  if (validate_cache(shape, &dc) != WKV_OK) return 0;
  return decode_weighted_layout(dc.shape, dc.ws_bytes, &counts_at, &logits_at);
}

wkv_status wkv_decode_step_weighted(const wkv_decode_shape *shape, const void *q_new, const void *k_new, const void *v_new, void *k_cache,
                                    void *v_cache, int32_t *n_valid, float *weights, int32_t *tok_idx, const int32_t *position, float *out,
                                    void *workspace, size_t workspace_bytes, void *hip_stream) {
  Decode dc;
  wkv_status st = validate_cache(shape, &dc);
  if (st != WKV_OK) return st;
  if (!q_new || !k_new || !v_new || !k_cache || !v_cache || !n_valid || !weights || !out)
    return invalid("q_new / k_new / v_new / k_cache / v_cache / n_valid / weights / out is NULL");
  if ((tok_idx == nullptr) != (position == nullptr)) return invalid("tok_idx and position go together: both or neither");
  if (misaligned(q_new, 16) || misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16))
    return invalid("q_new, k_new, v_new and the caches must be 16-byte aligned");
  if (misaligned(n_valid, 4) || misaligned(weights, 4) || misaligned(tok_idx, 4) || misaligned(position, 4) || misaligned(out, 4))
    return invalid("n_valid, weights, tok_idx, position and out must be 4-byte aligned");
  size_t counts_at, logits_at;
  st = check_workspace(workspace, workspace_bytes, decode_weighted_layout(dc.shape, dc.ws_bytes, &counts_at, &logits_at));
  if (st != WKV_OK) return st;
  const DecodeWeights w = {weights, tok_idx, position, (int32_t *)((char *)workspace + counts_at), (float *)((char *)workspace + logits_at)};
  return launched(launch_decode_weighted(dc.shape, q_new, k_new, v_new, k_cache, v_cache, n_valid, w, out, (float *)workspace, (hipStream_t)hip_stream),
                  "wkv_decode_step_weighted");
}

size_t wkv_evict_workspace_bytes(const wkv_decode_shape *shape) {
  Decode dc;
  size_t moves_at;
  if (validate_cache(shape, &dc) != WKV_OK) return 0;
  return evict_layout(dc.shape.B * dc.shape.Hkv, max_moves(dc.shape.capacity), &moves_at);
}

wkv_status wkv_cache_evict(const wkv_decode_shape *shape, int32_t n_layers, void *const *k_caches, void *const *v_caches, float *weights,
                           int32_t *tok_idx, int32_t *n_valid, const int32_t *keep, int32_t recent, void *workspace, size_t workspace_bytes,
                           void *hip_stream) {
  Decode dc;
  wkv_status st = validate_cache(shape, &dc);
  if (st != WKV_OK) return st;
  if (n_layers < 1 || n_layers > WKV_MAX_LAYERS) { set_error("n_layers outside [1, %d]", WKV_MAX_LAYERS); return WKV_ERR_INVALID_ARG; }
  if (!k_caches || !v_caches || !weights || !tok_idx || !n_valid || !keep) return invalid("k_caches / v_caches / weights / tok_idx / n_valid / keep is NULL");
  if (recent < 0) return invalid("recent must be >= 0");
  if (misaligned(weights, 4) || misaligned(tok_idx, 4) || misaligned(n_valid, 4) || misaligned(keep, 4))
    return invalid("weights, tok_idx, n_valid and keep must be 4-byte aligned");
  EvictLayers layers;
  std::memset(&layers, 0, sizeof layers);
  for (int32_t l = 0; l < n_layers; ++l) {
    layers.k[l] = k_caches[l]; layers.v[l] = v_caches[l];
    if (!layers.k[l] || !layers.v[l]) { set_error("cache of layer %d is NULL", l); return WKV_ERR_INVALID_ARG; }
    if (misaligned(layers.k[l], 16) || misaligned(layers.v[l], 16)) { set_error("caches of layer %d must be 16-byte aligned", l); return WKV_ERR_INVALID_ARG; }
  }
  const DecodeShape &s = dc.shape;
  EvictArgs a;
  std::memset(&a, 0, sizeof a);
  const int64_t e = elem_bytes(s.dtype);
  a.rows = s.B * s.Hkv; a.Hkv = s.Hkv; a.capacity = s.capacity; a.recent = recent; a.row_bytes = (int32_t)(s.d * e);
  a.hkv_magic = s.kv_magic;
  a.sb = s.sb * e; a.sh = s.sh * e; a.st = s.st * e;
  a.max_moves = max_moves(s.capacity);
  size_t moves_at;
  st = check_workspace(workspace, workspace_bytes, evict_layout(a.rows, a.max_moves, &moves_at));
  if (st != WKV_OK) return st;
  return launched(launch_evict(a, layers, n_layers, weights, tok_idx, n_valid, keep, (int32_t *)workspace, (int2 *)((char *)workspace + moves_at),
                               (hipStream_t)hip_stream), "wkv_cache_evict");
}

}  // extern "C"
