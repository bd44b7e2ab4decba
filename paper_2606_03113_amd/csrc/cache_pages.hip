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

// Everything that the block's threads have written and counted is seen by all
// of them: stores and atomics are done (one CU's stores go through its own L1;
// counts are read where the atomics are made, see count_of).
__device__ __forceinline__ void block_sync() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
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

// How many of n ascending values are at most i.
__device__ __forceinline__ int at_most(const int32_t* v, int n, int i) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (v[mid] <= i) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// Table entries of PG_THREADS sequences, spread over the threads whatever the
// sequences' shares of them: thread t's sequence has count entries from place
// `from` on.  each(u, sequence, place) is called for up to FLAT entries of a
// thread, and then done() once, so that their loads can be on their way
// together (a wave a sequence, one load after the other: 12400 entries of 1001
// sequences freed by one block in 77 us against 36).
constexpr int FLAT = 4;
struct FlatEntries {
  int32_t end[PG_THREADS], from[PG_THREADS];
};
template <class Each, class Done>
__device__ __forceinline__ int flat_entries(FlatEntries& f, Two* red, int n, int from, int count, Each each, Done done) {
  Two total;
  const Two end = block_scan(Two{count, 0}, red, total);
  f.end[threadIdx.x] = end.x;
  f.from[threadIdx.x] = from;
  __syncthreads();
  n = min(n, PG_THREADS);
  for (int i0 = threadIdx.x; i0 < total.x; i0 += FLAT * PG_THREADS) {
#pragma unroll
    for (int u = 0; u < FLAT; ++u) {
      const int i = i0 + u * PG_THREADS;
      if (i >= total.x) continue;
      const int j = at_most(f.end, n, i);
      each(u, j, f.from[j] + i - (j ? f.end[j - 1] : 0));
    }
    done(i0, total.x);
  }
  __syncthreads();   // (f and red serve the next ones)
  return total.x;
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

// One block checks all sequences, then spreads the shared entries.  A source is
// no fork itself, so its lengths and row stay as they are.  Bound by the chain
// of loads (source, lengths, entry): 3 forks of 11 pages 3.5 us, 224 of up
// to 32 8.9.
__global__ __launch_bounds__(PG_THREADS) void k_cache_fork(CachePagesArgs a) {
  __shared__ FlatEntries flat;
  __shared__ Two red[PG_WAVES];
  __shared__ int32_t row[PG_THREADS];
  __shared__ int bad_seq;
  const int tid = threadIdx.x;
  if (tid == 0) bad_seq = INT_MAX;
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
  for (int s0 = 0; s0 < a.n_seqs; s0 += PG_THREADS) {
    const int s = s0 + tid, r = s < a.n_seqs ? a.source[s] : -1;
    int n = 0;
    if (r >= 0) {
      const int len = a.lens ? a.lens[s] : a.seq_lens[r];
      n = pages_of(len);
      a.seq_lens[s] = len;
      a.held[s] = n;
    }
    row[tid] = r;
    int page[FLAT];
    int32_t* to[FLAT];
    shared += flat_entries(flat, red, a.n_seqs - s0, 0, n,
        [&](int u, int j, int place) {
          page[u] = a.tables[(int64_t)row[j] * a.table_ld + place];
          to[u] = a.tables + (int64_t)(s0 + j) * a.table_ld + place;
        },
        [&](int i0, int total) {
#pragma unroll
          for (int u = 0; u < FLAT; ++u)
            if (i0 + u * PG_THREADS < total) {
              *to[u] = page[u];
              if (page[u] >= 0 && page[u] < a.n_pages) atomicAdd(a.shares + page[u], 1);
            }
        });
  }
  if (tid == 0) {
    a.status[0] = 0;
    a.status[1] = shared;
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

// A sequence's first entry that new tokens fall into, of sequences s0 ..; the
// others (long prompts over pages kept from a rollback) are read where needed.
struct OwnSeq {
  OwnAsk q;
  int page;
  bool in;   // the first entry is of the pool
};
__device__ __forceinline__ int own_page(const CachePagesArgs& a, int s, int place) { return a.tables[(int64_t)s * a.table_ld + place]; }
__device__ __forceinline__ bool in_pool(const CachePagesArgs& a, int page) { return page >= 0 && page < a.n_pages; }
__device__ __forceinline__ OwnSeq own_seq(const CachePagesArgs& a, int s) {
  OwnSeq r{own_ask(a, s), -1, false};
  if (r.q.from < r.q.to) r.page = own_page(a, s, r.q.from);
  r.in = in_pool(a, r.page);
  return r;
}
// each(place, count of its page) for a sequence's entries that are pages of the pool.
template <class Each> __device__ __forceinline__ void own_entries(const CachePagesArgs& a, int s, const OwnSeq& o, Each each) {
  if (o.in) each(o.q.from, a.shares + o.page);
  for (int i = o.q.from + 1; i < o.q.to; ++i) {
    const int page = own_page(a, s, i);
    if (in_pool(a, page)) each(i, a.shares + page);
  }
}

// Where no page that is written has another holder, as in most steps, that is
// all.  Else every holder that writes a page leaves it (shares - 1); below zero
// nobody stays, and the first of the leaving sequences keeps it after all
// (INT_MIN + s stands for that).  The others take pages from the free list in
// sequence order, then in table order; of a page with tokens before the new
// ones the content has to follow (a pair for the copy).  A chain of loads,
// atomics and their loads: 4 sequences 6.0 us, 256 7.3.
__global__ __launch_bounds__(PG_THREADS) void k_cache_own(CachePagesArgs a) {
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq, bad_code;
  const int tid = threadIdx.x, n = a.n_seqs, head = *a.free_head;
  const int avail = head >= 0 && head <= a.n_free ? a.n_free - head : -1;
  if (tid == 0) bad_seq = INT_MAX;
  const OwnSeq first = own_seq(a, tid);
  auto seq_at = [&](int s) { return s < PG_THREADS ? first : own_seq(a, s); };
  __syncthreads();
  bool shared = false;
  for (int s = tid; s < n; s += PG_THREADS) {
    const OwnSeq o = seq_at(s);
    if (avail < 0 || o.q.code) atomicMin(&bad_seq, s);
    own_entries(a, s, o, [&](int, const int32_t* c) { shared |= *c != 0; });
  }
  shared = __syncthreads_or(shared);
  Two done{0, 0}, total;
  bool ok = bad_seq == INT_MAX;
  if (!ok) bad_code = LEDE_E_ARG;
  if (ok && shared) {
    for (int s = tid; s < n; s += PG_THREADS) own_entries(a, s, seq_at(s), [&](int, int32_t* c) { atomicSub(c, 1); });
    block_sync();
    for (int s = tid; s < n; s += PG_THREADS)
      own_entries(a, s, seq_at(s), [&](int, int32_t* c) {
        if (count_of(c) < 0) atomicMin(c, INT_MIN + s);
      });
    block_sync();
    // what is taken (x) and copied (y), up to the sequence that it does not suffice for
    auto ask = [&](int s, const OwnSeq& o) {
      Two mine{0, 0};
      if (s < n)
        own_entries(a, s, o, [&](int i, const int32_t* c) {
          if (count_of(c) == INT_MIN + s) return;
          ++mine.x;
          mine.y += i < pages_of(o.q.seq);
        });
      return mine;
    };
    Two mine{0, 0}, end{0, 0};
    for (int s0 = 0; s0 < n; s0 += PG_THREADS) {
      const int s = s0 + tid;
      mine = ask(s, seq_at(s));
      end = block_scan(mine, red, total);
      const int code = done.x + end.x > avail ? LEDE_E_KV_FULL : done.y + end.y > a.max_moves ? LEDE_E_ARG : 0;
      if (s < n && code) atomicMin(&bad_seq, s);
      __syncthreads();
      if (s == bad_seq) bad_code = code;
      done.x += total.x;
      done.y += total.y;
      __syncthreads();
      if (bad_seq != INT_MAX) break;
    }
    ok = bad_seq == INT_MAX;
    if (!ok) done = Two{0, 0};
    Two at{0, 0};
    for (int s0 = 0; ok && s0 < n; s0 += PG_THREADS) {
      const int s = s0 + tid;
      const OwnSeq o = seq_at(s);
      if (n > PG_THREADS) {   // (one round: the sums above serve)
        mine = ask(s, o);
        end = block_scan(mine, red, total);
      }
      int take = at.x + end.x - mine.x, move = at.y + end.y - mine.y;
      // (no more than was counted, also where a page is held and listed as free)
      const int last = at.x + end.x, last_move = at.y + end.y;
      if (mine.x)
        own_entries(a, s, o, [&](int i, int32_t* c) {
          if (take == last || count_of(c) == INT_MIN + s) return;
          const int fresh = a.free_pages[head + take++];
          if (i < pages_of(o.q.seq) && move < last_move) {
            a.pairs[2 * move] = (int)(c - a.shares);
            a.pairs[2 * move + 1] = fresh;
            ++move;
          }
          a.tables[(int64_t)s * a.table_ld + i] = fresh;
          if (in_pool(a, fresh)) a.shares[fresh] = 0;
        });
      at.x += total.x;
      at.y += total.y;
    }
    block_sync();
    // (entries that were replaced lead to pages whose count is 0, but for the
    // first, whose page is the old one still: it is not this sequence's to keep)
    for (int s = tid; s < n; s += PG_THREADS)
      own_entries(a, s, seq_at(s), [&](int, int32_t* c) {
        if (count_of(c) == INT_MIN + s) *c = ok ? 0 : -1;
      });
    if (!ok) {   // as it was
      block_sync();
      for (int s = tid; s < n; s += PG_THREADS) own_entries(a, s, seq_at(s), [&](int, int32_t* c) { atomicAdd(c, 1); });
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

// Table entries up to which one block does it all.
constexpr int64_t FREE_ALONE = 8192;

// The first sequence that cannot give pages back, INT_MAX: none.  All threads.
__device__ __forceinline__ int free_bad(const CachePagesArgs& a, int head, int* bad_seq) {
  if (threadIdx.x == 0) *bad_seq = INT_MAX;
  __syncthreads();
  for (int s = threadIdx.x; s < a.n_seqs; s += blockDim.x) {
    const int seq = a.seq_lens[s], held = a.held[s];
    if (seq < 0 || held < 0 || held > a.table_ld || head < 0 || head > a.n_free) atomicMin(bad_seq, s);
  }
  __syncthreads();
  return *bad_seq;
}
// What sequence s gives back: places [from, held).
__device__ __forceinline__ int free_from(const CachePagesArgs& a, int s, int& held) {
  held = s < a.n_seqs ? a.held[s] : 0;
  return s < a.n_seqs ? min(pages_of(a.seq_lens[s]), held) : 0;
}
// A holder leaves page, whose count was x: true for the last.  Without other
// holders, the usual case, that is a load; else each leaving one takes 1 and
// the atomic says who found 0 after all.
__device__ __forceinline__ bool leaves(const CachePagesArgs& a, int page, int x) { return x == 0 || atomicSub(a.shares + page, 1) == 0; }

// Many entries: a wave a sequence, over the card.  Pages without a holder are
// marked with -1.  (Each block checks all sequences, so there are few blocks.)
constexpr int LEAVE_BLOCKS = 512;
__global__ __launch_bounds__(256) void k_cache_leave(CachePagesArgs a) {
  __shared__ int bad_seq;
  if (free_bad(a, *a.free_head, &bad_seq) != INT_MAX) return;
  for (int s = blockIdx.x * 4 + (threadIdx.x >> 6); s < a.n_seqs; s += gridDim.x * 4) {
    int held;
    const int from = free_from(a, s, held);
    for (int i = from + (threadIdx.x & 63); i < held; i += 64) {
      const int page = a.tables[(int64_t)s * a.table_ld + i];
      if (in_pool(a, page) && leaves(a, page, count_of(a.shares + page)))
        __hip_atomic_store(a.shares + page, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

// The pages without a holder go to the list in ascending order, which does not
// depend on who came last.  MARKED: k_cache_leave has found them.  Bound by
// chains of loads: 71 entries of 64 sequences 6.4 us in one launch,
// 12400 of 1001 17 in two (in one 36).
template <bool MARKED>
__global__ __launch_bounds__(PG_THREADS) void k_cache_free(CachePagesArgs a) {
  __shared__ uint32_t words[CACHE_MOST_PAGES / 32];
  __shared__ int before[PG_THREADS];
  __shared__ FlatEntries flat;
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq;
  const int tid = threadIdx.x, n = a.n_seqs, head = *a.free_head;
  const PageBits bits(words, a.n_pages);
  if (!MARKED) bits.clear();
  const bool valid = free_bad(a, head, &bad_seq) == INT_MAX;
  // each(page) of the pool's pages that the sequences give back
  auto entries = [&](auto load, auto each) {
    for (int s0 = 0; s0 < n; s0 += PG_THREADS) {
      int page[FLAT], x[FLAT], held;
      const int from = free_from(a, s0 + tid, held);
      flat_entries(flat, red, n - s0, from, held - from,
          [&](int u, int j, int place) { page[u] = a.tables[(int64_t)(s0 + j) * a.table_ld + place]; },
          [&](int i0, int total) {
#pragma unroll
            for (int u = 0; u < FLAT; ++u) {
              if (i0 + u * PG_THREADS >= total || !in_pool(a, page[u])) page[u] = -1;
              x[u] = page[u] >= 0 ? load(page[u]) : 0;
            }
#pragma unroll
            for (int u = 0; u < FLAT; ++u)
              if (page[u] >= 0) each(page[u], x[u]);
          });
    }
  };
  Two total{0, 0};
  if (valid) {
    if (MARKED) {
#pragma unroll 4
      for (int p0 = 0; p0 < a.n_pages; p0 += PG_THREADS) {
        const uint64_t b = __ballot(p0 + tid < a.n_pages && a.shares[p0 + tid] == -1);
        if ((tid & 31) == 0 && p0 + tid < a.n_pages) words[(p0 + tid) >> 5] = (uint32_t)(tid & 32 ? b >> 32 : b);
      }
      __syncthreads();
    } else {
      entries([&](int page) { return count_of(a.shares + page); },
              [&](int page, int x) {
                if (leaves(a, page, x)) bits.set(page);
              });
      block_sync();
    }
    const int mine = bits.own();
    const Two end = block_scan(Two{mine, 0}, red, total);
    before[tid] = end.x - mine;
    __syncthreads();
    const bool room = total.x <= head;
    const int at = head - total.x;
    for (int page = tid; page < a.n_pages; page += PG_THREADS) {
      if (!bits.has(page)) continue;
      if (room) a.free_pages[at + bits.rank(before, page)] = page;
      a.shares[page] = room ? 0 : -1;
    }
    if (room) {
      for (int s = tid; s < n; s += PG_THREADS) {
        int held;
        const int from = free_from(a, s, held);
        if (from < held) a.held[s] = from;
      }
    } else {   // as it was: every leaving holder once more
      block_sync();
      entries([](int) { return 0; }, [&](int page, int) { atomicAdd(a.shares + page, 1); });
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
// both read and written.  Bound by the chains of loads: 3500 entries of 150
// sequences in a pool of 5000 14.1 us, 120 of 9 6.8.
__global__ __launch_bounds__(PG_THREADS) void k_cache_compact(CachePagesArgs a) {
  __shared__ uint32_t words[CACHE_MOST_PAGES / 32];
  __shared__ int before[PG_THREADS];
  __shared__ FlatEntries flat;
  __shared__ Two red[PG_WAVES];
  __shared__ int bad_seq;
  const int tid = threadIdx.x, n = a.n_seqs, head = *a.free_head;
  const PageBits bits(words, a.n_pages);
  bits.clear();
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  for (int s = tid; s < n; s += PG_THREADS)
    if (a.held[s] < 0 || a.held[s] > a.table_ld) atomicMin(&bad_seq, s);
  __syncthreads();
  // each(entry, page) of the held entries that are pages of the pool
  auto entries = [&](auto each) {
    for (int s0 = 0; s0 < n; s0 += PG_THREADS) {
      int32_t* entry[FLAT];
      int page[FLAT];
      flat_entries(flat, red, n - s0, 0, s0 + tid < n ? a.held[s0 + tid] : 0,
          [&](int u, int j, int place) {
            entry[u] = a.tables + (int64_t)(s0 + j) * a.table_ld + place;
            page[u] = *entry[u];
          },
          [&](int i0, int total) {
#pragma unroll
            for (int u = 0; u < FLAT; ++u)
              if (i0 + u * PG_THREADS < total && in_pool(a, page[u])) each(entry[u], page[u]);
          });
    }
  };
  if (bad_seq == INT_MAX) entries([&](int32_t*, int page) { bits.set(page); });
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
    for (int page = tid; moves && page < a.n_pages; page += PG_THREADS) {
      const bool set = bits.has(page);
      if (set == (page < live)) continue;   // neither moves nor is a hole
      const int rank = bits.rank(before, page);
      a.pairs[set ? 2 * (rank - kept) : 2 * (page - rank) + 1] = page;
    }
    block_sync();
    if (moves)
      entries([&](int32_t* entry, int page) {
        if (page >= live) *entry = a.pairs[2 * (bits.rank(before, page) - kept) + 1];
      });
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
  if ((int64_t)a.n_seqs * a.table_ld <= FREE_ALONE) {
    k_cache_free<false><<<1, PG_THREADS, 0, s>>>(a);
  } else {
    k_cache_leave<<<min((a.n_seqs + 3) / 4, LEAVE_BLOCKS), 256, 0, s>>>(a);
    k_cache_free<true><<<1, PG_THREADS, 0, s>>>(a);
  }
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
