// The paged 8-bit K/V cache of a batch of requests: its layout, and the
// kernels' arguments (cache.hip, cache_attention.hip; entry points in
// cache.cpp and pages.cpp).  Not part of the public C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lede.h"

namespace lede {

constexpr int CACHE_PAGE = 64;      // tokens of a page
constexpr int CACHE_E_MIN = -100;   // the smallest scale is 2^CACHE_E_MIN
constexpr uint32_t CACHE_NAN = 256; // scale word: the block holds a NaN code

// One layer's cache.  Codes are e4m3 (OCP); the value of a code c of a block
// (page, KV head) is c * 2^e, and the block's scale word is e + 127, plus
// CACHE_NAN while any code of it may be a NaN.  Powers of two cost e4m3 no
// precision (a code has its own exponent), they make re-scaling a block that
// grew exact except at the smallest codes, and they are applied by adding
// exponents.  Keys are rows of tokens.  Values are rows of dims: the value
// product's matrix operand is 8 tokens of one dim in consecutive bytes, so a
// lane loads its operands from memory and no transpose stands between.
struct CacheView {
  uint8_t* k;       // [page][head][64][hd]
  uint8_t* v;       // [page][head][hd][64]
  uint32_t* words;  // [page][head][2]: keys, values
  int n_pages, nkv, hd;
};
inline size_t cache_codes(int n_pages, int nkv, int hd) { return (size_t)n_pages * nkv * CACHE_PAGE * hd; }
inline size_t cache_bytes(int n_pages, int nkv, int hd) {
  return 2 * cache_codes(n_pages, nkv, hd) + (size_t)n_pages * nkv * 8;
}
inline CacheView cache_view(void* region, int n_pages, int nkv, int hd) {
  const size_t n = cache_codes(n_pages, nkv, hd);
  uint8_t* p = (uint8_t*)region;
  return {p, p + n, (uint32_t*)(p + 2 * n), n_pages, nkv, hd};
}

// A cache's shape: LEDE_OK, or why it is none.  Page and token counts stay in
// 32 bits, byte offsets are 64-bit everywhere.
inline int check_cache(int32_t n_pages, int32_t n_kv, int32_t hd) {
  if (n_pages < 1 || n_kv < 1) return LEDE_E_ARG;
  if ((hd != 64 && hd != 128) || n_kv > 1024) return LEDE_E_UNSUPPORTED;
  return LEDE_OK;
}

// Of 256 threads: a launch has fewer than 2^32 threads.
constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;

struct CachePlanArgs {
  const int32_t *seq_lens, *new_lens, *held;  // [n_seqs]
  int n_seqs;
  const int32_t* free_pages;
  int n_free;
  const int32_t* free_head;                   // [1]; may be status + 2
  int32_t* tables;
  int table_ld, max_rows;
  int32_t *kv_lens, *held_out, *row_start;    // may be seq_lens and held
  int64_t* slots;
  int32_t* status;                            // [4]: code, rows, free_head after, first failing sequence
};

struct CacheRowsArgs {   // append (rows in) and read (rows out)
  CacheView c;
  void *k, *v;
  int64_t ldk, ldv;      // elements between rows
  const int64_t* slots;
  int n_rows;
  int window;            // rows whose runs one block handles
};

struct CacheAttnArgs {
  CacheView c;
  const void* q; int64_t ldq;
  const int32_t* tables; int table_ld;
  const int32_t *kv_lens, *row_start;
  int n_seqs, n_rows, nq;
  float scale_log2x2;    // magnitude of the softmax scale, times 2 log2(e)
  uint32_t q_sign;       // 0x80008000 where it is negative: flips bf16 pairs' signs
  int tile_rows;         // rows a block: 16 or 32 (waves take pages), 64 or 128 (waves take rows)
  bool alone;            // 16 rows a wave, with all of their pages (n_cut = 0)
  bool raw;              // (64 rows, bf16, heads of 128) pages as codes in LDS
  int n_tiles;           // row tiles per (sequence, KV head) of the grid
  int n_full, n_cut, n_split, min_chunk;  // blocks of whole tasks; tasks cut into n_split blocks of at least min_chunk pages
  float* part;           // [n_cut][n_split][tile_rows][hd + 4]
  void* out; int64_t ldo;
};

// The pages' life (cache_pages.hip; entry points in pages.cpp).  The calls take what they need of these.
constexpr int CACHE_MOST_PAGES = 1 << 18;   // of a pool that is freed into or compacted: a bit a page in LDS
struct CachePagesArgs {
  const int32_t *source, *lens;               // [n_seqs]; lens may be null
  const int32_t* new_lens;                    // [n_seqs]
  int32_t *seq_lens, *held;                   // [n_seqs]
  int n_seqs;
  int32_t* tables;
  int table_ld;
  int32_t* shares;                            // [n_pages]
  int n_pages;
  int32_t* free_pages;
  int n_free;
  const int32_t* free_head;                   // [1]; may be status + 2
  int32_t* pairs;                             // [max_moves][2]: source page, destination page
  int max_moves;
  int32_t* status;
};
struct CacheCopyArgs {
  CacheView c;
  const int32_t* pairs;
  const int32_t* count;                       // [1]
  int max_moves;
};

hipError_t launch_cache_fork(const CachePagesArgs& a, hipStream_t s);
hipError_t launch_cache_own(const CachePagesArgs& a, hipStream_t s);
hipError_t launch_cache_free(const CachePagesArgs& a, hipStream_t s);
hipError_t launch_cache_compact(const CachePagesArgs& a, hipStream_t s);
hipError_t launch_cache_copy(const CacheCopyArgs& a, hipStream_t s);

hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t s);
hipError_t launch_cache_append(int dtype, const CacheRowsArgs& a, hipStream_t s);
hipError_t launch_cache_read(int dtype, const CacheRowsArgs& a, hipStream_t s);
hipError_t launch_cache_attention(int dtype, const CacheAttnArgs& a, hipStream_t s);

constexpr int LP_TILE = 8192;       // entries of a row that a block holds at a time
constexpr int LP_PART_TILES = 16;   // tiles that a block takes at most

struct LogprobsArgs {
  const void* logits;
  int64_t ld;
  int n_rows, V, n_tiles, part_tiles, n_part, n_top;   // a block takes part_tiles tiles of a row
  float c;               // log2(e) / temperature
  const int32_t* tokens;
  float *logprobs, *entropy, *top_logprobs;
  int32_t *ranks, *top_ids;
  // workspace (n_part > 1): per (row, part) {max, sum, weighted sum, rank
  // count} and the part's top keys in descending order
  float4* part_stats;    // .w holds the count's bits
  uint64_t* part_keys;   // [row][part][n_top]
};
hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s);

}  // namespace lede
