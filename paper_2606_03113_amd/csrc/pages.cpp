// Entry points of the batch cache's pages: forks, owned pages, copies, pages
// given back, compaction.  No call allocates, synchronises or keeps anything
// between calls.
#include <hip/hip_runtime.h>

#include "../../include/lede.h"
#include "cache.h"

using namespace lede;

namespace {

hipStream_t S_(void* s) { return (hipStream_t)s; }
int done(hipError_t e) { return e == hipSuccess ? LEDE_OK : LEDE_E_HIP; }

// Tables and shares that the pages' calls step through: all entries of a table
// are counted in 32 bits.
int pages_check(const int32_t* tables, int32_t table_ld, int32_t n_seqs, const int32_t* shares, int32_t n_pages, const int32_t* status) {
  if (!tables || !shares || !status || table_ld < 1 || n_seqs < 1 || n_pages < 1) return LEDE_E_ARG;
  return n_seqs > MOST_BLOCKS || (int64_t)n_seqs * table_ld > 1 << 30 ? LEDE_E_UNSUPPORTED : LEDE_OK;
}
CachePagesArgs pages_args(int32_t n_seqs, int32_t* tables, int32_t table_ld, int32_t* shares, int32_t n_pages, int32_t* status) {
  CachePagesArgs a{};
  a.n_seqs = n_seqs; a.tables = tables; a.table_ld = table_ld; a.shares = shares; a.n_pages = n_pages; a.status = status;
  return a;
}

}  // namespace

extern "C" {

int lede_op_cache_fork(const int32_t* source, const int32_t* lens, int32_t* seq_lens, int32_t* held, int32_t n_seqs,
                       int32_t* tables, int32_t table_ld, int32_t* shares, int32_t n_pages, int32_t* status, void* stream) {
  if (!source || !seq_lens || !held) return LEDE_E_ARG;
  if (int rc = pages_check(tables, table_ld, n_seqs, shares, n_pages, status)) return rc;
  CachePagesArgs a = pages_args(n_seqs, tables, table_ld, shares, n_pages, status);
  a.source = source; a.lens = lens; a.seq_lens = seq_lens; a.held = held;
  return done(launch_cache_fork(a, S_(stream)));
}

int lede_op_cache_own(const int32_t* seq_lens, const int32_t* new_lens, const int32_t* held, int32_t n_seqs,
                      const int32_t* free_pages, int32_t n_free, const int32_t* free_head, int32_t* tables, int32_t table_ld,
                      int32_t* shares, int32_t n_pages, int32_t* pairs, int32_t max_moves, int32_t* status, void* stream) {
  if (!seq_lens || !new_lens || !held || !free_head || n_free < 0 || (n_free && !free_pages) || max_moves < 0 || (max_moves && !pairs)) return LEDE_E_ARG;
  if (int rc = pages_check(tables, table_ld, n_seqs, shares, n_pages, status)) return rc;
  if (max_moves > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;
  CachePagesArgs a = pages_args(n_seqs, tables, table_ld, shares, n_pages, status);
  a.seq_lens = (int32_t*)seq_lens; a.new_lens = new_lens; a.held = (int32_t*)held;
  a.free_pages = (int32_t*)free_pages; a.n_free = n_free; a.free_head = free_head; a.pairs = pairs; a.max_moves = max_moves;
  return done(launch_cache_own(a, S_(stream)));
}

int lede_op_cache_copy(const int32_t* pairs, const int32_t* count, int32_t max_moves, void* cache, int32_t n_pages,
                       int32_t n_kv_heads, int32_t head_dim, void* stream) {
  if (!cache || max_moves < 0) return LEDE_E_ARG;
  if (int rc = check_cache(n_pages, n_kv_heads, head_dim)) return rc;
  if ((uintptr_t)cache % 16) return LEDE_E_ARG;
  if (max_moves > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;
  if (max_moves == 0) return LEDE_OK;
  if (!pairs || !count) return LEDE_E_ARG;
  CacheCopyArgs a{};
  a.c = cache_view(cache, n_pages, n_kv_heads, head_dim);
  a.pairs = pairs; a.count = count; a.max_moves = max_moves;
  return done(launch_cache_copy(a, S_(stream)));
}

int lede_op_cache_free(const int32_t* seq_lens, int32_t* held, int32_t n_seqs, int32_t* free_pages, int32_t n_free,
                       const int32_t* free_head, const int32_t* tables, int32_t table_ld, int32_t* shares, int32_t n_pages,
                       int32_t* status, void* stream) {
  if (!seq_lens || !held || !free_head || n_free < 0 || (n_free && !free_pages)) return LEDE_E_ARG;
  if (int rc = pages_check(tables, table_ld, n_seqs, shares, n_pages, status)) return rc;
  if (n_pages > CACHE_MOST_PAGES) return LEDE_E_UNSUPPORTED;
  CachePagesArgs a = pages_args(n_seqs, (int32_t*)tables, table_ld, shares, n_pages, status);
  a.seq_lens = (int32_t*)seq_lens; a.held = held; a.free_pages = free_pages; a.n_free = n_free; a.free_head = free_head;
  return done(launch_cache_free(a, S_(stream)));
}

int lede_op_cache_compact(const int32_t* held, int32_t n_seqs, int32_t* free_pages, int32_t n_free, const int32_t* free_head,
                          int32_t* tables, int32_t table_ld, int32_t* shares, int32_t n_pages, int32_t* pairs, int32_t max_moves,
                          int32_t* status, void* stream) {
  if (!held || !free_head || n_free < 0 || (n_free && !free_pages) || max_moves < 0 || (max_moves && !pairs)) return LEDE_E_ARG;
  if (int rc = pages_check(tables, table_ld, n_seqs, shares, n_pages, status)) return rc;
  if (n_pages > CACHE_MOST_PAGES || max_moves > MOST_BLOCKS) return LEDE_E_UNSUPPORTED;
  CachePagesArgs a = pages_args(n_seqs, tables, table_ld, shares, n_pages, status);
  a.held = (int32_t*)held; a.free_pages = free_pages; a.n_free = n_free; a.free_head = free_head; a.pairs = pairs; a.max_moves = max_moves;
  return done(launch_cache_compact(a, S_(stream)));
}

}  // extern "C"
