// The life of the batch cache's pages (gfx950): forks that share them, pages
// made a sequence's own before it writes, copies, pages given back, and the
// pool's compaction.
//
// shares[page] counts a page's holders besides one, so that a page that a plan
// takes from the free list needs no entry of its own: 0 for a free page and for
// one with a single holder.  The counts are whole numbers and the pages that a
// call frees or copies are listed in an order of their own, so that no order of
// the atomics shows in a result.
#include "cache.h"
#include "device.h"

#include "../../include/lede.h"

namespace lede {

constexpr int PG_THREADS = 1024, PG_WAVES = PG_THREADS / 64;

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + CACHE_PAGE - 1) / CACHE_PAGE); }

// Everything that the block's threads have written and counted is seen by all.
__device__ __forceinline__ void block_sync() {
  __threadfence();
  __syncthreads();
}

__device__ __forceinline__ int count_of(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Inclusive prefix sums over the block in thread order, and their totals.
struct Two { int x, y; };
__device__ __forceinline__ Two block_scan(Two v, Two* red, Two& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(v.x, o), y = __shfl_up(v.y, o);
    if (lane >= o) {
      v.x += x;
      v.y += y;
    }
  }
  __syncthreads();
  if (lane == 63) red[wave] = v;
  __syncthreads();
  Two base{0, 0};
  total = Two{0, 0};
#pragma unroll
  for (int w = 0; w < PG_WAVES; ++w) {
    const Two r = red[w];
    if (w < wave) {
      base.x += r.x;
      base.y += r.y;
    }
    total.x += r.x;
    total.y += r.y;
  }
  return Two{base.x + v.x, base.y + v.y};
}

// Whether a sequence's lengths fit its table row.
__device__ __forceinline__ bool lengths_ok(int seq, int held, int table_ld) {
  return seq >= 0 && held >= 0 && held <= table_ld && pages_of(seq) <= held;
}

// ---- fork -----------------------------------------------------------------------

// 0, or why sequence s cannot become the fork that it is asked to be.
__device__ __forceinline__ int fork_code(const CachePagesArgs& a, int s) {
  const int r = a.source[s];
  if (r == -1) return 0;
  if (r < 0 || r >= a.n_seqs || r == s || a.source[r] != -1) return LEDE_E_ARG;
  if (!lengths_ok(a.seq_lens[r], a.held[r], a.table_ld)) return LEDE_E_ARG;
  if (a.lens && (a.lens[s] < 0 || a.lens[s] > a.seq_lens[r])) return LEDE_E_ARG;
  return a.held[s] ? LEDE_E_STATE : 0;
}

// One block checks all sequences, then a wave takes a fork's table row.  A
// source is no fork itself, so its lengths and row stay as they are.
__global__ __launch_bounds__(PG_THREADS) void k_cache_fork(CachePagesArgs a) {
  __shared__ int bad_seq, bad_code, n_shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) {
    bad_seq = INT_MAX;
    n_shared = 0;
  }
  __syncthreads();
  for (int s = tid; s < a.n_seqs; s += PG_THREADS)
    if (fork_code(a, s)) atomicMin(&bad_seq, s);
  __syncthreads();
  if (bad_seq != INT_MAX) {
    if (tid == 0) {
      a.status[0] = fork_code(a, bad_seq);
      a.status[1] = 0;
      a.status[2] = bad_seq;
    }
    return;
  }
  int shared = 0;
  for (int s = wave; s < a.n_seqs; s += PG_WAVES) {
    const int r = a.source[s];
    if (r < 0) continue;
    const int len = a.lens ? a.lens[s] : a.seq_lens[r], n = pages_of(len);
    for (int i = lane; i < n; i += 64) {
      const int page = a.tables[(int64_t)r * a.table_ld + i];
      a.tables[(int64_t)s * a.table_ld + i] = page;
      if (page >= 0 && page < a.n_pages) atomicAdd(a.shares + page, 1);
    }
    if (lane == 0) {
      a.seq_lens[s] = len;
      a.held[s] = n;
    }
    shared += n;
  }
  if (lane == 0) atomicAdd(&n_shared, shared);
  __syncthreads();
  if (tid == 0) {
    a.status[0] = 0;
    a.status[1] = n_shared;
    a.status[2] = -1;
  }
}

// ---- own ------------------------------------------------------------------------

// The places [from, to) of a sequence's pages that its new tokens fall into
// and that it holds already; 0 or an error.
struct OwnAsk { int seq, from, to, code; };
__device__ __forceinline__ OwnAsk own_ask(const CachePagesArgs& a, int s) {
  OwnAsk r{0, 0, 0, 0};
  if (s >= a.n_seqs) return r;
  const int held = a.held[s], fresh = a.new_lens[s];
  r.seq = a.seq_lens[s];
  if (fresh < 0 || !lengths_ok(r.seq, held, a.table_ld)) {
    r.code = LEDE_E_ARG;
  } else if (fresh) {
    r.from = r.seq / CACHE_PAGE;
    r.to = min(held, pages_of((int64_t)r.seq + fresh));
  }
  return r;
}

// Every holder that writes a page leaves it (shares - 1); below zero nobody
// stays, and the first of the leaving sequences keeps it after all (INT_MIN + s
// stands for that).  The others take pages from the free list in sequence
// order, then in table order; of a page with tokens before the new ones the
// content has to follow (a pair for the copy).
__device__ __forceinline__ int32_t* own_count(const CachePagesArgs& a, int s, int place) {
  const int page = a.tables[(int64_t)s * a.table_ld + place];
  return page >= 0 && page < a.n_pages ? a.shares + page : nullptr;
}
__device__ __forceinline__ bool own_takes(const CachePagesArgs& a, int s, int place) {
  const int32_t* c = own_count(a, s, place);
  return c && count_of(c) != INT_MIN + s;
}

__global__ __launch_bounds__(PG_THREADS) void k_cache_own(CachePagesArgs a) {
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq, bad_code;
  const int tid = threadIdx.x, n = a.n_seqs, head = *a.free_head;
  const int avail = head >= 0 && head <= a.n_free ? a.n_free - head : -1;
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  for (int s = tid; s < n; s += PG_THREADS)
    if (avail < 0 || own_ask(a, s).code) atomicMin(&bad_seq, s);
  __syncthreads();
  if (bad_seq != INT_MAX) {
    if (tid == 0) {
      a.status[0] = LEDE_E_ARG;
      a.status[1] = 0;
      a.status[2] = head;
      a.status[3] = bad_seq;
    }
    for (int i = tid; i < 2 * a.max_moves; i += PG_THREADS) a.pairs[i] = -1;
    return;
  }
  for (int s = tid; s < n; s += PG_THREADS) {
    const OwnAsk q = own_ask(a, s);
    for (int i = q.from; i < q.to; ++i)
      if (int32_t* c = own_count(a, s, i)) atomicSub(c, 1);
  }
  block_sync();
  for (int s = tid; s < n; s += PG_THREADS) {
    const OwnAsk q = own_ask(a, s);
    for (int i = q.from; i < q.to; ++i)
      if (int32_t* c = own_count(a, s, i))
        if (count_of(c) < 0) atomicMin(c, INT_MIN + s);
  }
  block_sync();
  // what is taken and copied, up to the sequence that it does not suffice for
  Two done{0, 0}, total;
  for (int s0 = 0; s0 < n; s0 += PG_THREADS) {
    const int s = s0 + tid;
    const OwnAsk q = own_ask(a, s);
    Two mine{0, 0};
    for (int i = q.from; i < q.to; ++i)
      if (own_takes(a, s, i)) {
        ++mine.x;
        mine.y += i * CACHE_PAGE < q.seq;
      }
    const Two end = block_scan(mine, red, total);
    const int code = done.x + end.x > avail ? LEDE_E_KV_FULL : done.y + end.y > a.max_moves ? LEDE_E_ARG : 0;
    if (s < n && code) atomicMin(&bad_seq, s);
    __syncthreads();
    if (s == bad_seq) bad_code = code;
    done.x += total.x;
    done.y += total.y;
    __syncthreads();
    if (bad_seq != INT_MAX) break;
  }
  const bool ok = bad_seq == INT_MAX;
  if (!ok) done = Two{0, 0};
  if (ok) {
    Two at{0, 0};
    for (int s0 = 0; s0 < n; s0 += PG_THREADS) {
      const int s = s0 + tid;
      const OwnAsk q = own_ask(a, s);
      Two mine{0, 0};
      for (int i = q.from; i < q.to; ++i)
        if (own_takes(a, s, i)) {
          ++mine.x;
          mine.y += i * CACHE_PAGE < q.seq;
        }
      const Two end = block_scan(mine, red, total);
      int take = at.x + end.x - mine.x, move = at.y + end.y - mine.y;
      for (int i = q.from; i < q.to; ++i)
        if (own_takes(a, s, i)) {
          int32_t* entry = a.tables + (int64_t)s * a.table_ld + i;
          const int fresh = a.free_pages[head + take++];
          if (i * CACHE_PAGE < q.seq) {
            a.pairs[2 * move] = *entry;
            a.pairs[2 * move + 1] = fresh;
            ++move;
          }
          *entry = fresh;
          if (fresh >= 0 && fresh < a.n_pages) a.shares[fresh] = 0;
        }
      at.x += total.x;
      at.y += total.y;
    }
  }
  block_sync();
  for (int s = tid; s < n; s += PG_THREADS) {
    const OwnAsk q = own_ask(a, s);
    for (int i = q.from; i < q.to; ++i)
      if (int32_t* c = own_count(a, s, i))
        if (count_of(c) == INT_MIN + s) *c = ok ? 0 : -1;
  }
  if (!ok) {   // as it was
    block_sync();
    for (int s = tid; s < n; s += PG_THREADS) {
      const OwnAsk q = own_ask(a, s);
      for (int i = q.from; i < q.to; ++i)
        if (int32_t* c = own_count(a, s, i)) atomicAdd(c, 1);
    }
  }
  for (int i = 2 * done.y + tid; i < 2 * a.max_moves; i += PG_THREADS) a.pairs[i] = -1;
  if (tid == 0) {
    a.status[0] = ok ? 0 : bad_code;
    a.status[1] = done.y;
    a.status[2] = head + done.x;
    a.status[3] = ok ? -1 : bad_seq;
  }
}

// ---- free -----------------------------------------------------------------------

// Pages of a pool as bits in LDS.  A thread owns `per` consecutive words.
struct PageBits {
  uint32_t* bits;
  int words, per;
  __device__ __forceinline__ PageBits(uint32_t* b, int n_pages) : bits(b), words((n_pages + 31) / 32), per((words + PG_THREADS - 1) / PG_THREADS) {}
  __device__ __forceinline__ void clear() const {
    for (int w = threadIdx.x; w < words; w += PG_THREADS) bits[w] = 0;
  }
  __device__ __forceinline__ void set(int page) const { atomicOr(bits + (page >> 5), 1u << (page & 31)); }
  __device__ __forceinline__ bool has(int page) const { return bits[page >> 5] >> (page & 31) & 1; }
  __device__ __forceinline__ int first_word() const { return min((int)threadIdx.x * per, words); }
  __device__ __forceinline__ int last_word() const { return min((int)threadIdx.x * per + per, words); }
  __device__ __forceinline__ int own() const {   // bits of the thread's words
    int n = 0;
    for (int w = first_word(); w < last_word(); ++w) n += __popc(bits[w]);
    return n;
  }
  // Set bits before a page; before[t]: those before thread t's words.
  __device__ __forceinline__ int rank(const int* before, int page) const {
    const int word = page >> 5, t = word / per;
    int n = before[t];
    for (int w = t * per; w < word; ++w) n += __popc(bits[w]);
    return n + __popc(bits[word] & ((1u << (page & 31)) - 1));
  }
};

// The places [from, held) that sequence s gives back.
__device__ __forceinline__ int free_from(const CachePagesArgs& a, int s, int& held) {
  held = a.held[s];
  return min(pages_of(a.seq_lens[s]), held);
}

// A holder that leaves takes 1 from shares[page]; the one that finds 0 was the
// last, and marks the page.  The marked pages go to the list in their own
// order, which does not depend on who came last.
__global__ __launch_bounds__(PG_THREADS) void k_cache_free(CachePagesArgs a) {
  __shared__ uint32_t words[CACHE_MOST_PAGES / 32];
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_seqs, head = *a.free_head;
  const PageBits bits(words, a.n_pages);
  bits.clear();
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  for (int s = tid; s < n; s += PG_THREADS) {
    const int seq = a.seq_lens[s], held = a.held[s];
    if (seq < 0 || held < 0 || held > a.table_ld || head < 0 || head > a.n_free) atomicMin(&bad_seq, s);
  }
  __syncthreads();
  const bool valid = bad_seq == INT_MAX;
  Two total{0, 0};
  if (valid) {
    for (int s = wave; s < n; s += PG_WAVES) {
      int held;
      const int from = free_from(a, s, held);
      for (int i = from + lane; i < held; i += 64) {
        const int page = a.tables[(int64_t)s * a.table_ld + i];
        if (page >= 0 && page < a.n_pages && atomicSub(a.shares + page, 1) == 0) bits.set(page);
      }
    }
    block_sync();
    const int mine = bits.own();
    const Two end = block_scan(Two{mine, 0}, red, total);
    if (total.x <= head) {
      int at = head - total.x + end.x - mine;
      for (int w = bits.first_word(); w < bits.last_word(); ++w)
        for (uint32_t b = words[w]; b; b &= b - 1) {
          const int page = 32 * w + __ffs(b) - 1;
          a.free_pages[at++] = page;
          a.shares[page] = 0;
        }
      for (int s = tid; s < n; s += PG_THREADS) {
        int held;
        const int from = free_from(a, s, held);
        if (from < held) a.held[s] = from;
      }
    } else {   // no room before free_head: as it was
      for (int s = wave; s < n; s += PG_WAVES) {
        int held;
        const int from = free_from(a, s, held);
        for (int i = from + lane; i < held; i += 64) {
          const int page = a.tables[(int64_t)s * a.table_ld + i];
          if (page >= 0 && page < a.n_pages) atomicAdd(a.shares + page, 1);
        }
      }
    }
  }
  if (tid == 0) {
    const bool ok = valid && total.x <= head;
    a.status[0] = ok ? 0 : LEDE_E_ARG;
    a.status[1] = ok ? total.x : 0;
    a.status[2] = ok ? head - total.x : head;
    a.status[3] = valid ? -1 : bad_seq;
  }
}

// ---- compact --------------------------------------------------------------------

// With L live pages, the k-th of those from page L on (in ascending order)
// moves to the k-th hole before it: as many as there are holes, and no page is
// both read and written.
__global__ __launch_bounds__(PG_THREADS) void k_cache_compact(CachePagesArgs a) {
  __shared__ uint32_t words[CACHE_MOST_PAGES / 32];
  __shared__ int before[PG_THREADS];
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_seqs, head = *a.free_head;
  const PageBits bits(words, a.n_pages);
  bits.clear();
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  for (int s = tid; s < n; s += PG_THREADS)
    if (a.held[s] < 0 || a.held[s] > a.table_ld) atomicMin(&bad_seq, s);
  __syncthreads();
  if (bad_seq == INT_MAX)
    for (int s = wave; s < n; s += PG_WAVES) {
      const int held = a.held[s];
      for (int i = lane; i < held; i += 64) {
        const int page = a.tables[(int64_t)s * a.table_ld + i];
        if (page >= 0 && page < a.n_pages) bits.set(page);
      }
    }
  __syncthreads();
  const int mine = bits.own();
  Two total;
  const Two end = block_scan(Two{mine, 0}, red, total);
  before[tid] = end.x - mine;
  __syncthreads();
  const int live = total.x, kept = live < a.n_pages ? bits.rank(before, live) : live, moves = live - kept;
  const int new_head = a.n_free - (a.n_pages - live);
  const bool ok = bad_seq == INT_MAX && moves <= a.max_moves && new_head >= 0;
  if (ok) {
    int rank = end.x - mine;
    for (int w = bits.first_word(); w < bits.last_word(); ++w) {
      const uint32_t b = words[w];
      for (int k = 0; k < 32 && 32 * w + k < a.n_pages; ++k) {
        const int page = 32 * w + k;
        const bool set = b >> k & 1;
        if (set && page >= live) a.pairs[2 * (rank - kept)] = page;
        if (!set && page < live) a.pairs[2 * (page - rank) + 1] = page;
        rank += set;
      }
    }
    block_sync();
    for (int s = wave; s < n; s += PG_WAVES) {
      const int held = a.held[s];
      for (int i = lane; i < held; i += 64) {
        int32_t* entry = a.tables + (int64_t)s * a.table_ld + i;
        const int page = *entry;
        if (page >= live && page < a.n_pages) *entry = a.pairs[2 * (bits.rank(before, page) - kept) + 1];
      }
    }
    for (int i = tid; i < moves; i += PG_THREADS) a.shares[a.pairs[2 * i + 1]] = a.shares[a.pairs[2 * i]];
    block_sync();
    for (int p = live + tid; p < a.n_pages; p += PG_THREADS) a.shares[p] = 0;
    for (int i = new_head + tid; i < a.n_free; i += PG_THREADS) a.free_pages[i] = live + i - new_head;
  }
  for (int i = 2 * (ok ? moves : 0) + tid; i < 2 * a.max_moves; i += PG_THREADS) a.pairs[i] = -1;
  if (tid == 0) {
    a.status[0] = ok ? 0 : LEDE_E_ARG;
    a.status[1] = ok ? moves : 0;
    a.status[2] = ok ? new_head : head;
    a.status[3] = ok ? live : bad_seq == INT_MAX ? -1 : bad_seq;
  }
}

// ---- copy -----------------------------------------------------------------------

// A block copies pieces of 16 KiB (a quarter of a KV head's block and more),
// four 16-byte loads a thread in flight.  Memory-bound.
constexpr int COPY_THREADS = 256, COPY_PIECE = COPY_THREADS * 16 * 4;
__global__ __launch_bounds__(COPY_THREADS) void k_cache_copy(CacheCopyArgs a) {
  const int64_t size = (int64_t)a.c.nkv * CACHE_PAGE * a.c.hd;
  const int pieces = (int)((size + COPY_PIECE - 1) / COPY_PIECE);
  const int count = max(0, min(*a.count, a.max_moves));
  for (int64_t job = blockIdx.x; job < (int64_t)count * 2 * pieces; job += gridDim.x) {
    const int pair = (int)(job / (2 * pieces)), rest = (int)(job % (2 * pieces)), which = rest / pieces, piece = rest % pieces;
    const int src = a.pairs[2 * pair], dst = a.pairs[2 * pair + 1];
    if (src < 0 || src >= a.c.n_pages || dst < 0 || dst >= a.c.n_pages) continue;
    uint8_t* codes = which ? a.c.v : a.c.k;
    const int64_t at = (int64_t)piece * COPY_PIECE + threadIdx.x * 16;
    const uint8_t* from = codes + src * size + at;
    uint8_t* to = codes + dst * size + at;
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i * (COPY_THREADS * 16) < size) x[i] = ld16_stream(from + i * (COPY_THREADS * 16));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i * (COPY_THREADS * 16) < size) *(uint4*)(to + i * (COPY_THREADS * 16)) = x[i];
    if (rest == 0)
      for (int i = threadIdx.x; i < 2 * a.c.nkv; i += COPY_THREADS)
        a.c.words[(int64_t)dst * 2 * a.c.nkv + i] = a.c.words[(int64_t)src * 2 * a.c.nkv + i];
  }
}

hipError_t launch_cache_fork(const CachePagesArgs& a, hipStream_t s) {
  k_cache_fork<<<1, PG_THREADS, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_own(const CachePagesArgs& a, hipStream_t s) {
  k_cache_own<<<1, PG_THREADS, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_free(const CachePagesArgs& a, hipStream_t s) {
  k_cache_free<<<1, PG_THREADS, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_compact(const CachePagesArgs& a, hipStream_t s) {
  k_cache_compact<<<1, PG_THREADS, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_copy(const CacheCopyArgs& a, hipStream_t s) {
  const int64_t size = (int64_t)a.c.nkv * CACHE_PAGE * a.c.hd, pieces = (size + COPY_PIECE - 1) / COPY_PIECE;
  const int64_t jobs = (int64_t)a.max_moves * 2 * pieces;
  k_cache_copy<<<(unsigned)(jobs < 4096 ? jobs : 4096), COPY_THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lede
