// Pages, slots, appends and read-back of the paged 8-bit K/V cache (gfx950).
#include "cache.h"
#include "device.h"

#include "../../include/lede.h"

namespace lede {

// ---- page tables and the slot map ---------------------------------------------

constexpr int PLAN_THREADS = 1024;

// Inclusive prefix sums of two values over the block, in thread order, and
// their totals.
struct Pair { int64_t x, y; };
__device__ __forceinline__ Pair block_scan(Pair v, Pair* red, Pair& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t x = __shfl_up(v.x, o), y = __shfl_up(v.y, o);
    if (lane >= o) {
      v.x += x;
      v.y += y;
    }
  }
  __syncthreads();
  if (lane == 63) red[wave] = v;
  __syncthreads();
  Pair base{0, 0};
  total = Pair{0, 0};
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 64; ++w) {
    const Pair r = red[w];
    if (w < wave) {
      base.x += r.x;
      base.y += r.y;
    }
    total.x += r.x;
    total.y += r.y;
  }
  return Pair{base.x + v.x, base.y + v.y};
}

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + CACHE_PAGE - 1) / CACHE_PAGE); }

// What a sequence asks for, and the error that its lengths alone make (0: none).
struct PlanAsk { int seq, fresh, held, need, code; };
__device__ __forceinline__ PlanAsk plan_ask(const CachePlanArgs& a, int s) {
  PlanAsk r{0, 0, 0, 0, 0};
  if (s >= a.n_seqs) return r;
  r.seq = a.seq_lens[s];
  r.fresh = a.new_lens[s];
  r.held = a.held[s];
  if (r.seq < 0 || r.fresh < 0 || r.held < 0 || r.held > a.table_ld || pages_of(r.seq) > r.held) r.code = LEDE_E_ARG;
  else if ((int64_t)r.seq + r.fresh > INT32_MAX || pages_of((int64_t)r.seq + r.fresh) > a.table_ld) r.code = LEDE_E_CTX_OVERFLOW;
  else r.need = max(0, pages_of((int64_t)r.seq + r.fresh) - r.held);
  if (r.code) r.fresh = 0;
  return r;
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

// One block: prefix sums of the rows and of the pages to take, in sequence
// order, PLAN_THREADS sequences at a time; a first pass finds the first
// sequence that fails, a second writes (one chunk: the first's sums serve).
// The taken pages' table entries, and with SLOTS the rows' slots, are spread
// over the threads whatever the sequences' sizes.  Latency-bound: two rounds of
// loads, a scan and the stores; 64 sequences of one row each 5 us.
template <bool SLOTS>
__global__ __launch_bounds__(PLAN_THREADS) void k_cache_plan(CachePlanArgs a) {
  __shared__ Pair red[PLAN_THREADS / 64];
  __shared__ int bad_seq, bad_code;
  __shared__ int32_t row_end[PLAN_THREADS], page_end[PLAN_THREADS], seq_len[PLAN_THREADS], held[PLAN_THREADS];
  const int tid = threadIdx.x;
  const int head = *a.free_head;
  const int64_t avail = head >= 0 && head <= a.n_free ? a.n_free - head : -1;
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  PlanAsk q;
  Pair end, total, done{0, 0};   // rows, pages
  for (int s0 = 0; s0 < a.n_seqs; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    q = plan_ask(a, s);
    end = block_scan(Pair{q.fresh, q.need}, red, total);
    const int code = q.code                          ? q.code
                     : avail < 0                     ? LEDE_E_ARG
                     : done.y + end.y > avail        ? LEDE_E_KV_FULL
                     : done.x + end.x > a.max_rows   ? LEDE_E_ARG
                                                     : 0;
    if (s < a.n_seqs && code) atomicMin(&bad_seq, s);
    __syncthreads();
    if (s == bad_seq) bad_code = code;
    done.x += total.x;
    done.y += total.y;
    __syncthreads();
    if (bad_seq != INT_MAX) break;
  }
  const bool ok = bad_seq == INT_MAX;
  if (!ok) done = Pair{0, 0};
  if (tid == 0) {
    a.row_start[0] = 0;
    a.status[0] = ok ? 0 : bad_code;
    a.status[1] = (int)done.x;
    a.status[2] = head + (int)done.y;
    a.status[3] = ok ? -1 : bad_seq;
  }
  int rows = 0, taken = 0;   // (they fit: the first pass held them to max_rows and n_free)
  for (int s0 = 0; s0 < a.n_seqs; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    if (ok && a.n_seqs > PLAN_THREADS) {
      q = plan_ask(a, s);
      end = block_scan(Pair{q.fresh, q.need}, red, total);
    }
    if (s < a.n_seqs) {
      if (ok) {
        row_end[tid] = (int)end.x;
        page_end[tid] = (int)end.y;
        seq_len[tid] = q.seq;
        held[tid] = q.held;
      }
      a.kv_lens[s] = ok ? q.seq + q.fresh : a.seq_lens[s];
      a.held_out[s] = ok ? q.held + q.need : a.held[s];
      a.row_start[s + 1] = ok ? rows + (int)end.x : 0;
    }
    if (!ok) continue;
    __syncthreads();
    const int n = min(PLAN_THREADS, a.n_seqs - s0);
    for (int i = tid; i < (int)total.y; i += PLAN_THREADS) {
      const int j = at_most(page_end, n, i), from = j ? page_end[j - 1] : 0;
      a.tables[(int64_t)(s0 + j) * a.table_ld + held[j] + i - from] = a.free_pages[head + taken + i];
    }
    if (SLOTS) {
      for (int r = tid; r < (int)total.x; r += PLAN_THREADS) {
        const int j = at_most(row_end, n, r), pos = seq_len[j] + r - (j ? row_end[j - 1] : 0);
        const int i = pos / CACHE_PAGE - held[j];   // taken in this call: its entry may not be written yet
        const int64_t page = i < 0 ? a.tables[(int64_t)(s0 + j) * a.table_ld + pos / CACHE_PAGE]
                                   : a.free_pages[head + taken + (j ? page_end[j - 1] : 0) + i];
        a.slots[rows + r] = page * CACHE_PAGE + pos % CACHE_PAGE;
      }
    }
    rows += (int)total.x;
    taken += (int)total.y;
    __syncthreads();
  }
  if (SLOTS)
    for (int r = rows + tid; r < a.max_rows; r += PLAN_THREADS) a.slots[r] = -1;
}

// The slot of every row, by many blocks: the row's sequence from row_start.
__global__ __launch_bounds__(256) void k_cache_slots(CachePlanArgs a) {
  const int rows = a.status[1];
  for (int r = blockIdx.x * 256 + threadIdx.x; r < a.max_rows; r += gridDim.x * 256) {
    int64_t slot = -1;
    if (r < rows) {
      const int s = at_most(a.row_start + 1, a.n_seqs, r);
      const int pos = a.kv_lens[s] - a.row_start[s + 1] + r;
      slot = (int64_t)a.tables[(int64_t)s * a.table_ld + pos / CACHE_PAGE] * CACHE_PAGE + pos % CACHE_PAGE;
    }
    a.slots[r] = slot;
  }
}

// Few rows: one launch (64 rows: 6.3 us, 7.4 in two); many: a second spreads them
// over the card (8000 rows: 10 us, 13 in one; 255500: 13 and 228).
hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t s) {
  if (a.max_rows <= 4 * PLAN_THREADS) {
    k_cache_plan<true><<<1, PLAN_THREADS, 0, s>>>(a);
  } else {
    k_cache_plan<false><<<1, PLAN_THREADS, 0, s>>>(a);
    k_cache_slots<<<(int)min((a.max_rows + 255ll) / 256, 2048ll), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

// ---- append ---------------------------------------------------------------------

// The smallest e >= CACHE_E_MIN with amax <= 448 * 2^e (amax finite): 448 is
// 1.75 * 2^8, so the mantissa against 1.75 decides.
__device__ __forceinline__ int block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFF) > 0x600000);
  return max(e, CACHE_E_MIN);   // (subnormal amax: far below the smallest scale)
}

// x 2^e, rounded once.
__device__ __forceinline__ float scale_by(float x, int e) { return ldexpf(x, e); }

__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// x 2^-e as a code; what is not finite becomes a NaN code.
__device__ __forceinline__ float to_scale(float x, int e) {
  return fabsf(x) < INFINITY ? scale_by(x, -e) : __builtin_nanf("");
}
template <int I> __device__ __forceinline__ float decode1(uint32_t w) { return __builtin_amdgcn_cvt_f32_fp8((int)w, I); }

// Eight consecutive elements of a row, as they came (half the registers of
// their values, for bf16).
template <int DT> struct Eight {
  uint4 u[DT ? 1 : 2];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (DT ? 1 : 2); ++i) u[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    u[0] = ld16((const uint8_t*)p + i * Elem<DT>::ES_);
    if (DT == 0) u[DT ? 0 : 1] = ld16((const uint8_t*)p + i * Elem<DT>::ES_ + 16);
  }
  // The largest magnitude's fp32 bits: from 0x7F800000 on, one is not finite.
  __device__ __forceinline__ uint32_t most(uint32_t m) const {
    if (DT == 1) {
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      auto low = [](uint32_t x) { return __builtin_bit_cast(u16x2, x & 0x7FFF7FFFu); };
      const u16x2 x = __builtin_elementwise_max(__builtin_elementwise_max(low(u[0].x), low(u[0].y)), __builtin_elementwise_max(low(u[0].z), low(u[0].w)));
      return max(m, (uint32_t)max(x[0], x[1]) << 16);
    }
#pragma unroll
    for (int i = 0; i < (DT ? 1 : 2); ++i) m = max(max(max(m, u[i].x & 0x7FFFFFFF), u[i].y & 0x7FFFFFFF), max(u[i].z & 0x7FFFFFFF, u[i].w & 0x7FFFFFFF));
    return m;
  }
  __device__ __forceinline__ float operator[](int e) const {   // (e is a constant of an unrolled loop)
    const uint4 q = DT ? u[0] : u[DT ? 0 : e / 4];
    const int w = DT ? e / 2 : e % 4;
    const uint32_t x = w == 0 ? q.x : w == 1 ? q.y : w == 2 ? q.z : q.w;
    return DT == 0 ? __uint_as_float(x) : e & 1 ? bf16hi(x) : bf16lo(x);
  }
};

// Four codes re-scaled by 2^d (d <= 0), rounded to the nearest code.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, int d) {
  return encode4(scale_by(decode1<0>(w), d), scale_by(decode1<1>(w), d), scale_by(decode1<2>(w), d), scale_by(decode1<3>(w), d));
}

// A block of 2 HD threads works on a page's (KV head, keys or values) block:
// a thread has the four tokens 4 g .. 4 g + 3 and eight dims 8 c .. 8 c + 7.
// Keys: neighbouring threads have neighbouring dims (a token's codes are
// contiguous); values: neighbouring token groups (a dim's codes are), and four
// tokens' codes of a dim are one dword, so that nothing is transposed.
template <int HD> struct BlockPart {
  int c, g;
  __device__ __forceinline__ explicit BlockPart(bool values) {
    const int tid = threadIdx.x;
    c = values ? tid / 16 : tid % (HD / 8);
    g = values ? tid % 16 : tid / (HD / 8);
  }
};

// Rows whose slots lie in one page and follow each other in a call: a run.
// ASCENDING: with rising places, too (a place then has one row).  A wave's
// view from row w0 on: lane i has the slots of rows w0 + i and of the one
// before it.
template <bool ASCENDING> struct Rows {
  const CacheRowsArgs& a;
  int64_t n_slots, at, prev;
  __device__ __forceinline__ Rows(const CacheRowsArgs& a_, int w0) : a(a_), n_slots((int64_t)a_.c.n_pages * CACHE_PAGE) { load(w0); }
  __device__ __forceinline__ void load(int w0) {
    const int r = w0 + (threadIdx.x & 63);
    at = r < a.n_rows ? a.slots[r] : -1;
    prev = r < a.n_rows && r > 0 ? a.slots[r - 1] : -1;
  }
  __device__ __forceinline__ bool valid(int64_t s) const { return s >= 0 && s < n_slots; }
  __device__ __forceinline__ bool joins() const {
    return valid(prev) && valid(at) && prev / CACHE_PAGE == at / CACHE_PAGE && !(ASCENDING && at <= prev);
  }
  // Which of the first n rows begin a run.
  __device__ __forceinline__ uint64_t leaders(int n) const { return __ballot((int)(threadIdx.x & 63) < n && valid(at) && !joins()); }
  // The run at w0: its length (at most 64), its page, lane i its row i's place (-1 behind it).
  __device__ __forceinline__ int run(int64_t& page, int& place) const {
    const int lane = threadIdx.x & 63;
    const uint64_t out = ~__ballot(lane == 0 || joins());
    const int n = out ? __ffsll((unsigned long long)out) - 1 : 64;
    place = lane < n ? (int)(at % CACHE_PAGE) : -1;
    page = __shfl(at, 0) / CACHE_PAGE;
    return n;
  }
};

// The run's row of every place of the page (-1: none), by the first wave.
__device__ __forceinline__ void place_rows(int8_t* row_of, int n, int place) {
  if (threadIdx.x < 64) row_of[threadIdx.x] = -1;
  __syncthreads();
  if (threadIdx.x < n && threadIdx.x < 64) row_of[place] = (int8_t)threadIdx.x;
  __syncthreads();
}

// The block's maximum.
template <int NW> __device__ __forceinline__ uint32_t block_most(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) v = max(v, red[i]);
  return v;
}

// The rows of a call that lie in one page are a run of consecutive rows; a
// block handles the runs that begin in its window of rows, for one KV head
// and for keys or values.  A run that holds the page's first token starts the
// block's scale anew; any other run keeps the old scale, or, where its rows
// need a larger one, re-scales the page's other codes.  A prompt's rows (6406
// of 32 heads of 128, bf16: 157 MB) are memory-bound, 33 us, 4.8 TB/s; a step's
// single rows wait for three dependent loads, 5.2 us.  The window is short
// where blocks are few and a run's search would be repeated (48 rows: 5 us
// with one row, 44 with 16), long where rows fill pages (the prompt: 32 us with
// 64 rows, 207 with one).
template <int DT, int HD>
__global__ __launch_bounds__(2 * HD) void k_cache_append(CacheRowsArgs a) {
  constexpr int NW = 2 * HD / 64;
  __shared__ uint32_t red[NW];
  __shared__ __align__(4) int8_t row_of[CACHE_PAGE];
  const int head = blockIdx.y, which = blockIdx.z;
  const void* src = which ? a.v : a.k;
  const int64_t ld = which ? a.ldv : a.ldk;
  const BlockPart<HD> my(which);
  const int w0 = blockIdx.x * a.window;
  Rows<false> rows(a, w0);
  for (uint64_t left = rows.leaders(a.window); left; left &= left - 1) {
    const int r0 = w0 + __ffsll((unsigned long long)left) - 1;
    if (r0 > w0) rows.load(r0);
    int64_t page;
    int place;
    const int n = rows.run(page, place);
    const int64_t block = page * a.c.nkv + head;
    const bool fresh = __ballot(place == 0) != 0;
    uint32_t* word = a.c.words + block * 2 + which;
    const uint32_t old = *word;
    place_rows(row_of, n, place);
    // this thread's pieces of the rows, their largest finite magnitude
    Eight<DT> x[4];
    uint32_t in = 0;   // which of the four tokens the run has
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int r = row_of[4 * my.g + p];
      x[p].zero();
      if (r >= 0) {
        in |= 1u << p;
        x[p].load(src, (r0 + r) * ld + head * HD + my.c * 8);
      }
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) most = x[p].most(most);
    most = block_most<NW>(most, red);
    const bool bad = most >= 0x7F800000u;
    if (__builtin_expect(bad, 0)) {   // of the finite ones
      most = 0;
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t m = __float_as_uint(x[p][e]) & 0x7FFFFFFF;
          most = m < 0x7F800000u ? max(most, m) : most;
        }
      most = block_most<NW>(most, red);
    }
    const float amax = __uint_as_float(most);
    const int e_old = max((int)(old & 255) - 127, CACHE_E_MIN), e_new = block_exponent(amax);
    const int e = fresh ? e_new : max(e_old, e_new);
    const bool grew = !fresh && e > e_old;
    uint8_t* codes = (which ? a.c.v : a.c.k) + block * (size_t)(CACHE_PAGE * HD);
    if (in || grew) {
      if (!which) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          uint2* at = (uint2*)(codes + (4 * my.g + p) * HD + my.c * 8);
          if (in >> p & 1) {
            *at = make_uint2(encode4(to_scale(x[p][0], e), to_scale(x[p][1], e), to_scale(x[p][2], e), to_scale(x[p][3], e)),
                             encode4(to_scale(x[p][4], e), to_scale(x[p][5], e), to_scale(x[p][6], e), to_scale(x[p][7], e)));
          } else if (grew) {
            const uint2 c = *at;
            *at = make_uint2(rescale4(c.x, e_old - e), rescale4(c.y, e_old - e));
          }
        }
      } else {
        uint32_t had[8], keep = 0;   // bytes of the tokens that the run does not have
#pragma unroll
        for (int p = 0; p < 4; ++p) keep |= in >> p & 1 ? 0u : 0xFFu << (8 * p);
        uint32_t* at = (uint32_t*)(codes + my.c * 8 * CACHE_PAGE) + my.g;
        if (grew && keep)
#pragma unroll
          for (int d = 0; d < 8; ++d) had[d] = at[d * (CACHE_PAGE / 4)];
        uint32_t w[8];
#pragma unroll
        for (int d = 0; d < 8; ++d) w[d] = encode4(to_scale(x[0][d], e), to_scale(x[1][d], e), to_scale(x[2][d], e), to_scale(x[3][d], e));
        if (grew && keep)
#pragma unroll
          for (int d = 0; d < 8; ++d) w[d] = (w[d] & ~keep) | (rescale4(had[d], e_old - e) & keep);
        if (grew || !keep) {
#pragma unroll
          for (int d = 0; d < 8; ++d) at[d * (CACHE_PAGE / 4)] = w[d];
        } else {
#pragma unroll
          for (int p = 0; p < 4; ++p)
            if (in >> p & 1)
#pragma unroll
              for (int d = 0; d < 8; ++d) ((uint8_t*)(at + d * (CACHE_PAGE / 4)))[p] = (uint8_t)(w[d] >> (8 * p));
        }
      }
    }
    if (threadIdx.x == 0) *word = (uint32_t)(e + 127) | (bad || (!fresh && (old & CACHE_NAN)) ? CACHE_NAN : 0);
    __syncthreads();
  }
}

// ---- read-back ----------------------------------------------------------------------

// Byte I of a dword as the value of its code times 2^e.
template <int I> __device__ __forceinline__ float value_of(uint32_t w, int e) { return scale_by(decode1<I>(w), e); }

// A thread's four tokens and eight dims of a page's block, to their rows (r: the
// run's row of each token, -1 none).
template <int DT, int HD, bool VALUES>
__device__ __forceinline__ void read_part(const uint8_t* codes, const BlockPart<HD>& my, const int (&r)[4], int e, uint8_t* dst, int64_t pitch) {
  float x[4][8];
  if (VALUES) {
    uint32_t w[8];
#pragma unroll
    for (int d = 0; d < 8; ++d) w[d] = *((const uint32_t*)(codes + (my.c * 8 + d) * CACHE_PAGE) + my.g);
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      x[0][d] = value_of<0>(w[d], e);
      x[1][d] = value_of<1>(w[d], e);
      x[2][d] = value_of<2>(w[d], e);
      x[3][d] = value_of<3>(w[d], e);
    }
  } else {
    uint2 w[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) w[p] = *(const uint2*)(codes + (4 * my.g + p) * HD + my.c * 8);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      x[p][0] = value_of<0>(w[p].x, e); x[p][1] = value_of<1>(w[p].x, e); x[p][2] = value_of<2>(w[p].x, e); x[p][3] = value_of<3>(w[p].x, e);
      x[p][4] = value_of<0>(w[p].y, e); x[p][5] = value_of<1>(w[p].y, e); x[p][6] = value_of<2>(w[p].y, e); x[p][7] = value_of<3>(w[p].y, e);
    }
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    if (r[p] < 0) continue;
    uint8_t* at = dst + r[p] * pitch + my.c * 8 * Elem<DT>::ES_;
    if (DT == 1) {
      *(uint4*)at = make_uint4(f32_to_bf16x2(x[p][0], x[p][1]), f32_to_bf16x2(x[p][2], x[p][3]), f32_to_bf16x2(x[p][4], x[p][5]),
                               f32_to_bf16x2(x[p][6], x[p][7]));
    } else {
      *(float4*)at = make_float4(x[p][0], x[p][1], x[p][2], x[p][3]);
      *(float4*)(at + 16) = make_float4(x[p][4], x[p][5], x[p][6], x[p][7]);
    }
  }
}

// Runs as those of an append (of rising places), values the other way: 27 us
// for the prompt, 141 with one row a window.
template <int DT, int HD>
__global__ __launch_bounds__(2 * HD) void k_cache_read(CacheRowsArgs a) {
  __shared__ __align__(4) int8_t row_of[CACHE_PAGE];
  const int head = blockIdx.y, which = blockIdx.z;
  const int64_t ld = which ? a.ldv : a.ldk;
  const BlockPart<HD> my(which);
  const int w0 = blockIdx.x * a.window;
  Rows<true> rows(a, w0);
  for (uint64_t left = rows.leaders(a.window); left; left &= left - 1) {
    const int r0 = w0 + __ffsll((unsigned long long)left) - 1;
    if (r0 > w0) rows.load(r0);
    int64_t page;
    int place;
    const int n = rows.run(page, place);
    const int64_t block = page * a.c.nkv + head;
    const int e = (int)(a.c.words[block * 2 + which] & 255) - 127;
    place_rows(row_of, n, place);
    int r[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) r[p] = row_of[4 * my.g + p];
    if (max(max(r[0], r[1]), max(r[2], r[3])) >= 0) {
      const uint8_t* codes = (which ? a.c.v : a.c.k) + block * (size_t)(CACHE_PAGE * HD);
      uint8_t* dst = (uint8_t*)(which ? a.v : a.k) + (r0 * ld + head * HD) * Elem<DT>::ES_;
      if (which) read_part<DT, HD, true>(codes, my, r, e, dst, ld * Elem<DT>::ES_);
      else read_part<DT, HD, false>(codes, my, r, e, dst, ld * Elem<DT>::ES_);
    }
    __syncthreads();
  }
}

template <int DT, bool APPEND>
static hipError_t rows_hd(const CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid((a.n_rows + a.window - 1) / a.window, a.c.nkv, 2);
  if (APPEND) {
    if (a.c.hd == 128) k_cache_append<DT, 128><<<grid, 256, 0, s>>>(a);
    else k_cache_append<DT, 64><<<grid, 128, 0, s>>>(a);
  } else {
    if (a.c.hd == 128) k_cache_read<DT, 128><<<grid, 256, 0, s>>>(a);
    else k_cache_read<DT, 64><<<grid, 128, 0, s>>>(a);
  }
  return hipGetLastError();
}
hipError_t launch_cache_append(int dtype, const CacheRowsArgs& a, hipStream_t s) {
  return dtype ? rows_hd<1, true>(a, s) : rows_hd<0, true>(a, s);
}
hipError_t launch_cache_read(int dtype, const CacheRowsArgs& a, hipStream_t s) {
  return dtype ? rows_hd<1, false>(a, s) : rows_hd<0, false>(a, s);
}

}  // namespace lede
