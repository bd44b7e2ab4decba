// Entry points of a batch's operators: the paged 8-bit K/V cache and the log
// probabilities of logits rows.  No call allocates, synchronises or keeps
// anything between calls.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/lede.h"
#include "cache.h"

using namespace lede;

namespace {

hipStream_t S_(void* s) { return (hipStream_t)s; }
int done(hipError_t e) { return e == hipSuccess ? LEDE_OK : LEDE_E_HIP; }
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool dtype_ok(int32_t dt) { return dt == LEDE_DTYPE_F32 || dt == LEDE_DTYPE_BF16; }
int es_of(int32_t dt) { return dt == LEDE_DTYPE_BF16 ? 2 : 4; }

// Rows that the kernels read or write in 16-byte pieces.
bool rows_ok(const void* p, int64_t ld, int64_t width, int32_t dt) {
  return p && aligned(p, 16) && ld >= width && ld * es_of(dt) % 16 == 0;
}

// Row tiles and splits of an attention's grid.  The kernels are right for any
// lengths; this decides how the work spreads.
//
// Rows of a tile.  16 and 32: a block's waves take pages, so that each page is
// read once per tile, straight into registers; 64 and 128: they take rows,
// and share pages through LDS.  Measured, us (bf16 unless said otherwise; up to
// so many rows and tokens a sequence, from half of them on):
//   rows each                            16    32    64   128
//   16, 64 sequences of 8000, hd 128    153   159   209   281
//   20                                  200   163   208   277
//   40, 2 sequences of 131000           107   100    75   100
//   80, 64 of 8000                      311   246   331   285
//   96, 16 of 12000                           101   137   107
//   120, 8 of 30000                           150   158   124
//   160, 4 of 15000                            53    65    72
//   240, 2 of 130000                          210   214   166
//   256, 16 of 4000, 32 KV heads        413   266   261   221
//   500, fp32                           893   732   703
//   20, 64 of 8000, hd 64               104    87   137
//   40                                  108   123   136
//   500, 16 of 4000, 16 KV heads        158   142   138
//   1000                                320   278   243
//   200, fp32                            98         127
//   400                                 176         193
// Time of a page in a block that has its CU to itself, us (measured over 150
// pages, the fewest rows of hd 128 from memory).
double page_us(int32_t dtype, int32_t hd, int tile_rows) {
  static const double T[2][2][4] = {{{.33, .45, 1.03, 0}, {.22, .30, .79, 0}}, {{.65, .70, 1.6, 0}, {.50, .42, 1.12, 1.45}}};
  return T[hd == 128][dtype == LEDE_DTYPE_BF16][tile_rows == 16 ? 0 : tile_rows == 32 ? 1 : tile_rows == 64 ? 2 : 3];
}

struct AttnGrid { int tile_rows; bool alone, raw; int n_tiles, n_full, n_cut, n_split, min_chunk; };
AttnGrid attn_grid(int32_t dtype, int32_t n_seqs, int32_t nq, int32_t nkv, int32_t hd, int32_t max_new, int32_t max_kv) {
  AttnGrid g;
  const int64_t rows = std::max<int64_t>(1, (int64_t)max_new * (nq / nkv));
  const auto up = [](int64_t n, int64_t to) { return (n + to - 1) / to * to; };
  const int64_t groups = (int64_t)n_seqs * nkv;
  const int64_t pages = std::max<int64_t>(1, ((int64_t)max_kv + CACHE_PAGE - 1) / CACHE_PAGE);
  constexpr int64_t ROUND = 512, MOST_CUT = 8192;   // the card holds ROUND blocks at a time
  // Tiles of 128: unless much of them would be empty, or a round's blocks have
  // less than 16 pages each (8 sequences of up to 1000, 100 rows, 32 KV heads: 36
  // us, 29 in tiles of 32).
  const bool wide = up(rows, 128) * 4 <= up(rows, 32) * 5 && double(groups) * double(up(rows, 128) / 128) * double(pages) >= 16.0 * ROUND;
  if (rows <= 32) g.tile_rows = rows <= 16 ? 16 : 32;
  else if (hd == 64) g.tile_rows = rows < 512 ? 16 : 64;
  else if (rows <= 64) g.tile_rows = 64;
  else if (dtype == LEDE_DTYPE_BF16) g.tile_rows = wide ? 128 : 32;
  else g.tile_rows = rows < 256 ? 32 : 64;
  // (a task takes every n_tiles-th tile: a grid need not grow with a large max_new)
  g.n_tiles = (int)std::min((rows + g.tile_rows - 1) / g.tile_rows, 65536 / groups + 1);
  const int64_t whole = groups * g.n_tiles;
  // Short contexts of many tasks: a wave each, without a block's start, meeting
  // and end (2560 tasks of up to 128 tokens: 21 us, 28 with a block each; up to
  // 400: 45 and 43, and 18 and 20 with 640 tasks; up to 800: 93 and 81).
  g.alone = g.tile_rows == 16 && pages <= 8 && whole > ROUND;
  // Tasks of whole rounds are blocks of their own, and the rest, or all where
  // there are fewer, are cut to fill one (3 x up to 1000 rows behind up to 4100
  // tokens: 157 us, 205 uncut).  Few rows behind long contexts are cut into about
  // LONG pages in any case: lengths differ, and one long sequence must not be a
  // block's alone (100000 tokens among 63 of 1000: 81 us, 600 uncut).  64 pages
  // where the card would not be full (20 sequences of 50 to 60000 tokens: 60 us,
  // 88 with 128), else 128 (64 of up to 6000: 118 us, 125 with 64).  MOST_CUT
  // bounds the workspace and the blocks that find nothing to do (300 of 50 to
  // 60000: 955 us, 1056 with half as many).  A split's pages follow each other,
  // and so do the splits in the join: 2 sqrt(pages) of them at most (one head of
  // 130000 tokens: 26 us in 90 splits, 56 in 512).
  const int64_t LONG = whole < ROUND ? 64 : 128;
  const int64_t by_length = g.tile_rows <= 32 ? (pages + LONG - 1) / LONG : 1;
  const int64_t cut = g.alone ? 0 : by_length > 1 ? whole : whole % ROUND;
  int64_t split = cut ? std::max(whole < ROUND ? (ROUND + whole - 1) / whole : by_length > 1 ? 1 : ROUND / cut, by_length) : 1;
  split = std::min({split, std::max<int64_t>(1, MOST_CUT / std::max<int64_t>(cut, 1)), (int64_t)std::sqrt(4.0 * pages)});
  // A join costs its launch, its splits and its bytes, and short splits do not
  // earn it back: fewer (half, a quarter, ..) where a model of both says so (5 x
  // 100 rows, 16 pages: 15.6 us whole, 25 in four; 64 pages: 38 whole, 36 in two).
  const double page = page_us(dtype, hd, g.tile_rows), page_full = std::max(1.5 * page, ROUND * 128.0 * hd / 5.3e6);
  double best = INFINITY;
  for (int64_t k = split;; k = std::max<int64_t>(1, k / 2)) {
    const int64_t chunk = std::max<int64_t>(4, (pages + k - 1) / k), n = (pages + chunk - 1) / chunk, c = n > 1 ? cut : 0;
    const int64_t blocks = whole - c + c * n;
    const double steps = double(whole - c) * pages + double(c) * n * chunk;
    double us = 4 * std::max(1.0, blocks / double(ROUND)) + std::max((c < whole ? pages : chunk) * page, steps / ROUND * page_full);
    if (blocks > ROUND) us += 0.3 * (c ? chunk : pages) * page;
    if (c) us += 2 + 0.07 * n + c * n * g.tile_rows * (hd + 4) * 8 / 8e6;
    if (us < best) {
      best = us;
      g.n_cut = (int)c;
      g.n_split = c ? (int)n : 1;
      g.min_chunk = (int)chunk;
    }
    if (k == 1 || k / 2 < by_length) break;
  }
  g.n_full = (int)(whole - g.n_cut);
  g.raw = g.tile_rows == 64 && dtype == LEDE_DTYPE_BF16 && hd == 128 && g.n_full + (int64_t)g.n_cut * g.n_split > ROUND;
  return g;
}

constexpr int32_t MOST_SEQS = 65535;
bool attention_too_large(int32_t n_seqs, int32_t n_rows, int32_t nq, int32_t nkv) {
  return n_seqs > MOST_SEQS || (int64_t)n_seqs * nkv > MOST_BLOCKS / 2 || nq > 65536 || (int64_t)n_rows * (nq / nkv) >= 1ll << 30;
}
constexpr int32_t MOST_VOCAB = 1 << 20;
constexpr int32_t MOST_TOP = 32;

// Tiles of a row (its first may begin inside a 16-byte piece: up to 7
// entries before it), and how many of them a block takes: as many as leave
// the card about 1024 blocks (400 rows of 128256: 34 us, 37 with 512, 40 with
// 2048), all of them from 512 rows on (1000 rows: 60 us, 69 in two parts), and all
// of up to four (5 rows of 32000: 13.3 us in one launch; a block per tile takes
// 12.8, but a second launch and a workspace on the host).
struct ScoreGrid { int n_tiles, part_tiles, n_part; };
ScoreGrid score_grid(int32_t n_rows, int32_t V) {
  ScoreGrid g;
  g.n_tiles = (V + 7 + LP_TILE - 1) / LP_TILE;
  const int parts = g.n_tiles <= 4 || n_rows >= 512 ? 1 : std::min(g.n_tiles, std::max(1, (int)((1024 + (int64_t)n_rows - 1) / std::max(n_rows, 1))));
  g.part_tiles = std::min((g.n_tiles + parts - 1) / parts, LP_PART_TILES);
  g.n_part = (g.n_tiles + g.part_tiles - 1) / g.part_tiles;
  return g;
}

}  // namespace

extern "C" {

size_t lede_op_cache_bytes(int32_t n_pages, int32_t n_kv_heads, int32_t head_dim) {
  return check_cache(n_pages, n_kv_heads, head_dim) ? 0 : cache_bytes(n_pages, n_kv_heads, head_dim);
}

int lede_op_cache_plan(const int32_t* seq_lens, const int32_t* new_lens, const int32_t* held, int32_t n_seqs,
                       const int32_t* free_pages, int32_t n_free, const int32_t* free_head, int32_t* tables,
                       int32_t table_ld, int32_t max_rows, int32_t* kv_lens, int32_t* held_out, int32_t* row_start,
                       int64_t* slots, int32_t* status, void* stream) {
  if (!seq_lens || !new_lens || !held || !free_head || !tables || !kv_lens || !held_out || !row_start || !status)
    return LEDE_E_ARG;
  if (n_seqs < 1 || n_free < 0 || (n_free && !free_pages) || table_ld < 1 || max_rows < 0 || (max_rows && !slots))
    return LEDE_E_ARG;
  if (n_seqs > MOST_BLOCKS || max_rows > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;   // (the kernels step through both in 32 bits)
  CachePlanArgs a{};
  a.seq_lens = seq_lens; a.new_lens = new_lens; a.held = held; a.n_seqs = n_seqs;
  a.free_pages = free_pages; a.n_free = n_free; a.free_head = free_head;
  a.tables = tables; a.table_ld = table_ld; a.max_rows = max_rows;
  a.kv_lens = kv_lens; a.held_out = held_out; a.row_start = row_start; a.slots = slots; a.status = status;
  return done(launch_cache_plan(a, S_(stream)));
}

static int cache_rows(bool append, int32_t dtype, void* k, int64_t ldk, void* v, int64_t ldv, const int64_t* slots,
                      int32_t n_rows, void* cache, int32_t n_pages, int32_t n_kv, int32_t hd, void* stream) {
  if (!dtype_ok(dtype) || !cache || n_rows < 0) return LEDE_E_ARG;
  if (int rc = check_cache(n_pages, n_kv, hd)) return rc;
  if (!aligned(cache, 16)) return LEDE_E_ARG;
  if (n_rows > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;
  if (n_rows == 0) return LEDE_OK;
  const int64_t width = (int64_t)n_kv * hd;
  if (!slots || !rows_ok(k, ldk, width, dtype) || !rows_ok(v, ldv, width, dtype)) return LEDE_E_ARG;
  CacheRowsArgs a{};
  a.c = cache_view(cache, n_pages, n_kv, hd);
  a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv; a.slots = slots; a.n_rows = n_rows;
  // about 4096 blocks (the kernels say what shorter and longer windows cost)
  a.window = (int)std::min<int64_t>(CACHE_PAGE, std::max<int64_t>(1, (int64_t)n_rows * n_kv * 2 / 4096));
  return done(append ? launch_cache_append(dtype, a, S_(stream)) : launch_cache_read(dtype, a, S_(stream)));
}

int lede_op_cache_append(int32_t dtype, const void* k, int64_t ldk, const void* v, int64_t ldv, const int64_t* slots,
                         int32_t n_rows, void* cache, int32_t n_pages, int32_t n_kv_heads, int32_t head_dim,
                         void* stream) {
  return cache_rows(true, dtype, (void*)k, ldk, (void*)v, ldv, slots, n_rows, cache, n_pages, n_kv_heads, head_dim, stream);
}

int lede_op_cache_read(int32_t dtype, const void* cache, int32_t n_pages, int32_t n_kv_heads, int32_t head_dim,
                       const int64_t* slots, int32_t n_rows, void* k, int64_t ldk, void* v, int64_t ldv, void* stream) {
  return cache_rows(false, dtype, k, ldk, v, ldv, slots, n_rows, (void*)cache, n_pages, n_kv_heads, head_dim, stream);
}

size_t lede_op_cache_attention_bytes(int32_t dtype, int32_t n_seqs, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                                     int32_t head_dim, int32_t max_new, int32_t max_kv) {
  if (!dtype_ok(dtype) || n_seqs < 1 || n_rows < 0 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || max_new < 0 || max_kv < 0) return 0;
  if (check_cache(1, n_kv_heads, head_dim) || attention_too_large(n_seqs, n_rows, n_heads, n_kv_heads)) return 0;
  const AttnGrid g = attn_grid(dtype, n_seqs, n_heads, n_kv_heads, head_dim, max_new, max_kv);
  return (size_t)g.n_cut * g.n_split * g.tile_rows * (head_dim + 4) * 4;
}

int lede_op_cache_attention(int32_t dtype, const void* q, int64_t ldq, const void* cache, int32_t n_pages,
                            const int32_t* tables, int32_t table_ld, const int32_t* kv_lens, const int32_t* row_start,
                            int32_t n_seqs, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                            float scale, int32_t max_new, int32_t max_kv, void* out, int64_t ldo, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || !cache || !tables || !kv_lens || !row_start || n_seqs < 1 || n_rows < 0 || table_ld < 1)
    return LEDE_E_ARG;
  if (int rc = check_cache(n_pages, n_kv_heads, head_dim)) return rc;
  if (n_heads < 1 || n_heads % n_kv_heads || max_new < 0 || max_kv < 0 || !(std::fabs(scale) <= 1e38f)) return LEDE_E_ARG;   // (2 log2(e) scale is finite)
  if (attention_too_large(n_seqs, n_rows, n_heads, n_kv_heads)) return LEDE_E_UNSUPPORTED;
  if (!aligned(cache, 16)) return LEDE_E_ARG;
  if (n_rows == 0) return LEDE_OK;
  const int64_t width = (int64_t)n_heads * head_dim;
  if (!rows_ok(q, ldq, width, dtype) || !rows_ok(out, ldo, width, dtype)) return LEDE_E_ARG;
  const AttnGrid g = attn_grid(dtype, n_seqs, n_heads, n_kv_heads, head_dim, max_new, max_kv);
  const size_t need = lede_op_cache_attention_bytes(dtype, n_seqs, n_rows, n_heads, n_kv_heads, head_dim, max_new, max_kv);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return LEDE_E_ARG;
  CacheAttnArgs a{};
  a.c = cache_view((void*)cache, n_pages, n_kv_heads, head_dim);
  a.q = q; a.ldq = ldq; a.tables = tables; a.table_ld = table_ld; a.kv_lens = kv_lens; a.row_start = row_start;
  a.n_seqs = n_seqs; a.n_rows = n_rows; a.nq = n_heads;
  a.scale_log2x2 = (float)(std::fabs((double)scale) * 2 * 1.4426950408889634);
  a.q_sign = scale < 0 ? 0x80008000u : 0;
  a.tile_rows = g.tile_rows; a.alone = g.alone; a.raw = g.raw; a.n_tiles = g.n_tiles;
  a.n_full = g.n_full; a.n_cut = g.n_cut; a.n_split = g.n_split; a.min_chunk = g.min_chunk;
  a.part = (float*)workspace; a.out = out; a.ldo = ldo;
  return done(launch_cache_attention(dtype, a, S_(stream)));
}

size_t lede_op_logprobs_bytes(int32_t n_rows, int32_t V, int32_t n_top) {
  if (n_rows < 0 || V < 1 || V > MOST_VOCAB || n_top < 0 || n_top > MOST_TOP) return 0;
  const int parts = score_grid(n_rows, V).n_part;
  return parts == 1 ? 0 : (size_t)n_rows * parts * (16 + 8 * (size_t)n_top);
}

int lede_op_logprobs(int32_t dtype, const void* logits, int64_t ld, int32_t n_rows, int32_t V, float temperature,
                     const int32_t* tokens, int32_t n_top, float* logprobs, int32_t* ranks, float* entropy,
                     int32_t* top_ids, float* top_logprobs, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || V < 1 || n_top < 0 || n_top > V || ld < V) return LEDE_E_ARG;
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return LEDE_E_ARG;
  if (V > MOST_VOCAB || n_top > MOST_TOP) return LEDE_E_UNSUPPORTED;
  const float c = (float)(1.4426950408889634 / temperature);
  if (!std::isfinite(c)) return LEDE_E_ARG;
  if (n_rows == 0) return LEDE_OK;
  if ((logprobs || ranks) && !tokens) return LEDE_E_ARG;
  if (n_top && (!top_ids || !top_logprobs)) return LEDE_E_ARG;
  if (!logits || !aligned(logits, es_of(dtype))) return LEDE_E_ARG;
  const size_t need = lede_op_logprobs_bytes(n_rows, V, n_top);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return LEDE_E_ARG;
  LogprobsArgs a{};
  const ScoreGrid g = score_grid(n_rows, V);
  if ((int64_t)n_rows * g.n_part > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;
  a.logits = logits; a.ld = ld; a.n_rows = n_rows; a.V = V; a.n_top = n_top;
  a.n_tiles = g.n_tiles; a.part_tiles = g.part_tiles; a.n_part = g.n_part;
  a.c = c; a.tokens = tokens;
  a.logprobs = logprobs; a.ranks = ranks; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  a.part_stats = (float4*)workspace;
  a.part_keys = (uint64_t*)(a.part_stats + (size_t)n_rows * a.n_part);
  return done(launch_logprobs(dtype, a, S_(stream)));
}

}  // extern "C"
