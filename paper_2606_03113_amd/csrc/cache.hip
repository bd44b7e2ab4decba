// Pages, slots, appends and read-back of the paged 8-bit K/V cache (gfx950).
#include "cache.h"
#include "device.h"

#include "../../include/lede.h"

namespace lede {

// ---- page tables and the slot map ---------------------------------------------

constexpr int PLAN_THREADS = 1024;

// Inclusive prefix sum over the block, in thread order; `total` to everyone.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* red, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();
  if (lane == 63) red[wave] = v;
  __syncthreads();
  int64_t base = 0, all = 0;
  for (int w = 0; w < PLAN_THREADS / 64; ++w) {
    if (w < wave) base += red[w];
    all += red[w];
  }
  total = all;
  return base + v;
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
  else if (pages_of((int64_t)r.seq + r.fresh) > a.table_ld) r.code = LEDE_E_CTX_OVERFLOW;
  else r.need = max(0, pages_of((int64_t)r.seq + r.fresh) - r.held);
  if (r.code) r.fresh = 0;
  return r;
}

__device__ __forceinline__ int64_t plan_slot(const CachePlanArgs& a, int s, int pos) {
  const int64_t page = a.tables[(int64_t)s * a.table_ld + pos / CACHE_PAGE];
  return page * CACHE_PAGE + pos % CACHE_PAGE;
}

// One block: prefix sums of the rows and of the pages to take, in sequence
// order; a first pass finds the first sequence that fails, a second writes.
// Latency-bound: three loads, two scans and the stores.
__global__ __launch_bounds__(PLAN_THREADS) void k_cache_plan(CachePlanArgs a) {
  __shared__ int64_t red[PLAN_THREADS / 64];
  __shared__ int bad_seq, bad_code;
  const int tid = threadIdx.x;
  const int head = *a.free_head;
  const int64_t avail = head >= 0 && head <= a.n_free ? a.n_free - head : -1;
  if (tid == 0) bad_seq = INT_MAX;
  __syncthreads();
  int64_t rows = 0, taken = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    const PlanAsk q = plan_ask(a, s);
    int64_t t_rows, t_taken;
    const int64_t r_end = rows + block_scan(q.fresh, red, t_rows);
    const int64_t p_end = taken + block_scan(q.need, red, t_taken);
    const int code = q.code              ? q.code
                     : avail < 0         ? LEDE_E_ARG
                     : p_end > avail     ? LEDE_E_KV_FULL
                     : r_end > a.max_rows ? LEDE_E_ARG
                                         : 0;
    if (s < a.n_seqs && code) atomicMin(&bad_seq, s);
    __syncthreads();
    if (s == bad_seq) bad_code = code;
    rows += t_rows;
    taken += t_taken;
    __syncthreads();
    if (bad_seq != INT_MAX) break;
  }
  const bool ok = bad_seq == INT_MAX;
  rows = taken = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    const PlanAsk q = plan_ask(a, s);
    int64_t t_rows = 0, t_taken = 0, r_end = 0, p_end = 0;
    if (ok) {
      r_end = rows + block_scan(q.fresh, red, t_rows);
      p_end = taken + block_scan(q.need, red, t_taken);
    }
    if (s < a.n_seqs) {
      if (ok)
        for (int j = 0; j < q.need; ++j) a.tables[(int64_t)s * a.table_ld + q.held + j] = a.free_pages[head + p_end - q.need + j];
      a.kv_lens[s] = ok ? q.seq + q.fresh : a.seq_lens[s];
      a.held_out[s] = ok ? q.held + q.need : a.held[s];
      a.row_start[s + 1] = (int)r_end;
    }
    rows += t_rows;
    taken += t_taken;
  }
  if (tid == 0) {
    a.row_start[0] = 0;
    a.status[0] = ok ? 0 : bad_code;
    a.status[1] = (int)rows;
    a.status[2] = head + (int)taken;
    a.status[3] = ok ? -1 : bad_seq;
  }
}

// The slot of every row: the row's sequence by binary search of row_start.
__global__ __launch_bounds__(256) void k_cache_slots(CachePlanArgs a) {
  const int rows = a.status[1];
  for (int r = blockIdx.x * 256 + threadIdx.x; r < a.max_rows; r += gridDim.x * 256) {
    int64_t slot = -1;
    if (r < rows) {
      int lo = 0, hi = a.n_seqs;   // row_start[lo] <= r < row_start[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.row_start[mid] <= r) lo = mid; else hi = mid;
      }
      const int n = a.row_start[lo + 1] - a.row_start[lo];
      slot = plan_slot(a, lo, a.kv_lens[lo] - n + (r - a.row_start[lo]));
    }
    a.slots[r] = slot;
  }
}

hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t s) {
  k_cache_plan<<<1, PLAN_THREADS, 0, s>>>(a);
  if (a.max_rows > 0) k_cache_slots<<<(int)min((a.max_rows + 255ll) / 256, 2048ll), 256, 0, s>>>(a);
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

// 2^e for e in [-252, 254], as a product of two normal factors.
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

// Eight consecutive elements of a row.
template <int DT> __device__ __forceinline__ void row8(const void* p, int64_t i, float* o) {
  if (DT == 1) {
    const uint4 u = ld16((const uint16_t*)p + i);
    o[0] = bf16lo(u.x); o[1] = bf16hi(u.x); o[2] = bf16lo(u.y); o[3] = bf16hi(u.y);
    o[4] = bf16lo(u.z); o[5] = bf16hi(u.z); o[6] = bf16lo(u.w); o[7] = bf16hi(u.w);
  } else {
    const float4 a = *(const float4*)((const float*)p + i), b = *(const float4*)((const float*)p + i + 4);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w; o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
  }
}

// Sixteen codes re-scaled by 2^d (d <= 0), rounded to the nearest code.
__device__ __forceinline__ uint4 rescale16(uint4 c, int d) {
  uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = encode4(scale_by(decode1<0>(w[i]), d), scale_by(decode1<1>(w[i]), d), scale_by(decode1<2>(w[i]), d),
                   scale_by(decode1<3>(w[i]), d));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The rows of a call that lie in one page are a run of consecutive rows; a
// block handles the runs that begin in its window of rows, for one KV head
// and for keys or values.  A run that holds the page's first token starts the
// block's scale anew; any other run keeps the old scale, or, where its rows
// need a larger one, re-scales the page's codes first.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_cache_append(CacheRowsArgs a) {
  constexpr int TPR = HD / 8, RPP = 256 / TPR, NP = CACHE_PAGE / RPP;  // threads per row, rows per pass, passes
  __shared__ float red[4];
  __shared__ int red_bad[4];
  __shared__ __align__(16) uint8_t stage[CACHE_PAGE][HD + 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = blockIdx.y, which = blockIdx.z;
  const void* src = which ? a.v : a.k;
  const int64_t ld = which ? a.ldv : a.ldk;
  const int64_t n_slots = (int64_t)a.c.n_pages * CACHE_PAGE;
  const int w0 = blockIdx.x * a.window;
  for (int r0 = w0; r0 < min(w0 + a.window, a.n_rows); ++r0) {
    const int64_t first = a.slots[r0];
    if (first < 0 || first >= n_slots) continue;
    const int64_t page = first / CACHE_PAGE;
    if (r0 > 0) {
      const int64_t prev = a.slots[r0 - 1];
      if (prev >= 0 && prev < n_slots && prev / CACHE_PAGE == page) continue;  // inside a run
    }
    // lane i holds the place of the run's row i
    const int64_t mine = r0 + lane < a.n_rows ? a.slots[r0 + lane] : -1;
    const bool in = mine >= 0 && mine < n_slots && mine / CACHE_PAGE == page;
    const uint64_t mask = __ballot(in);
    const int n = ~mask ? __ffsll((unsigned long long)~mask) - 1 : 64;
    const int off = lane < n ? (int)(mine % CACHE_PAGE) : -1;
    const bool fresh = __ballot(off == 0) != 0;
    uint32_t* word = a.c.words + (page * a.c.nkv + head) * 2 + which;
    const uint32_t old = *word;
    // this thread's pieces of the rows, their largest finite magnitude
    const int part = tid % TPR;
    float x[NP][8];
    float amax = 0.f;
    bool bad = false;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int r = p * RPP + tid / TPR;
      if (r < n) {
        row8<DT>(src, (r0 + r) * ld + head * HD + part * 8, x[p]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = fabsf(x[p][e]);
          if (m < INFINITY) amax = fmaxf(amax, m); else bad = true;
        }
      }
    }
    amax = wave_max(amax);
    bad = __ballot(bad) != 0;
    __syncthreads();
    if (lane == 0) {
      red[wave] = amax;
      red_bad[wave] = bad;
    }
    __syncthreads();
    amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    bad = red_bad[0] | red_bad[1] | red_bad[2] | red_bad[3];
    const int e_old = max((int)(old & 255) - 127, CACHE_E_MIN), e_new = block_exponent(amax);
    const int e = fresh ? e_new : max(e_old, e_new);
    uint8_t* codes = (which ? a.c.v : a.c.k) + (page * a.c.nkv + head) * (size_t)(CACHE_PAGE * HD);
    if (!fresh && e > e_old) {
#pragma unroll
      for (int i = tid * 16; i < CACHE_PAGE * HD; i += 256 * 16) *(uint4*)(codes + i) = rescale16(ld16(codes + i), e_old - e);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int r = p * RPP + tid / TPR;
      const int o = __shfl(off, r & 63);
      if (r < n) {
        const uint2 c = make_uint2(encode4(to_scale(x[p][0], e), to_scale(x[p][1], e), to_scale(x[p][2], e), to_scale(x[p][3], e)),
                                   encode4(to_scale(x[p][4], e), to_scale(x[p][5], e), to_scale(x[p][6], e), to_scale(x[p][7], e)));
        *(uint2*)&stage[o][part * 8] = c;
      }
    }
    __syncthreads();  // (the re-scaled codes are written, too)
    uint64_t have = 0;   // tokens of the page that the run holds
    for (int i = 0; i < n; ++i) have |= 1ull << __shfl(off, i);
    if (!which) {
      for (int i = tid; i < CACHE_PAGE * HD / 16; i += 256) {
        const int t = i / (HD / 16), d = i % (HD / 16) * 16;
        if (have >> t & 1) *(uint4*)(codes + t * HD + d) = *(const uint4*)&stage[t][d];
      }
    } else {
      for (int i = tid; i < CACHE_PAGE * HD / 16; i += 256) {
        const int d = i / 4, t0 = i % 4 * 16;
        const uint32_t h = (uint32_t)(have >> t0) & 0xFFFF;
        if (h == 0xFFFF) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = stage[t0 + 4 * j][d] | stage[t0 + 4 * j + 1][d] << 8 | stage[t0 + 4 * j + 2][d] << 16 | (uint32_t)stage[t0 + 4 * j + 3][d] << 24;
          *(uint4*)(codes + d * CACHE_PAGE + t0) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (h) {
          for (int j = 0; j < 16; ++j)
            if (h >> j & 1) codes[d * CACHE_PAGE + t0 + j] = stage[t0 + j][d];
        }
      }
    }
    if (tid == 0) *word = (uint32_t)(e + 127) | (bad || (!fresh && (old & CACHE_NAN)) ? CACHE_NAN : 0);
    __syncthreads();
  }
}

// ---- read-back ----------------------------------------------------------------------

template <int DT, int HD>
__global__ __launch_bounds__(256) void k_cache_read(CacheRowsArgs a) {
  constexpr int TPR = HD / 8;
  const int head = blockIdx.y;
  const int r = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, part = threadIdx.x % TPR;
  if (r >= a.n_rows) return;
  const int64_t slot = a.slots[r];
  if (slot < 0 || slot >= (int64_t)a.c.n_pages * CACHE_PAGE) return;
  const int64_t block = slot / CACHE_PAGE * a.c.nkv + head;
  const int t = (int)(slot % CACHE_PAGE);
  const uint2 words = *(const uint2*)(a.c.words + block * 2);
  const int ek = (int)(words.x & 255) - 127, ev = (int)(words.y & 255) - 127;
  const uint2 kc = *(const uint2*)(a.c.k + block * (size_t)(CACHE_PAGE * HD) + t * HD + part * 8);
  const uint8_t* vp = a.c.v + block * (size_t)(CACHE_PAGE * HD) + part * 8 * CACHE_PAGE + t;
  uint32_t vc[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    vc[i] = vp[(4 * i) * CACHE_PAGE] | vp[(4 * i + 1) * CACHE_PAGE] << 8 | vp[(4 * i + 2) * CACHE_PAGE] << 16 |
            (uint32_t)vp[(4 * i + 3) * CACHE_PAGE] << 24;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint32_t lo = which ? vc[0] : kc.x, hi = which ? vc[1] : kc.y;
    const int e = which ? ev : ek;
    const float4 x = make_float4(scale_by(decode1<0>(lo), e), scale_by(decode1<1>(lo), e), scale_by(decode1<2>(lo), e), scale_by(decode1<3>(lo), e));
    const float4 y = make_float4(scale_by(decode1<0>(hi), e), scale_by(decode1<1>(hi), e), scale_by(decode1<2>(hi), e), scale_by(decode1<3>(hi), e));
    uint8_t* dst = (uint8_t*)(which ? a.v : a.k) + (r * (which ? a.ldv : a.ldk) + head * HD) * Elem<DT>::ES_;
    store4<DT>(dst, part * 8, x);
    store4<DT>(dst, part * 8 + 4, y);
  }
}

template <int DT>
static hipError_t append_hd(const CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid((a.n_rows + a.window - 1) / a.window, a.c.nkv, 2);
  if (a.c.hd == 128) k_cache_append<DT, 128><<<grid, 256, 0, s>>>(a);
  else k_cache_append<DT, 64><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_append(int dtype, const CacheRowsArgs& a, hipStream_t s) {
  return dtype ? append_hd<1>(a, s) : append_hd<0>(a, s);
}

template <int DT>
static hipError_t read_hd(const CacheRowsArgs& a, hipStream_t s) {
  const int rpb = 256 / (a.c.hd / 8);
  const dim3 grid((a.n_rows + rpb - 1) / rpb, a.c.nkv);
  if (a.c.hd == 128) k_cache_read<DT, 128><<<grid, 256, 0, s>>>(a);
  else k_cache_read<DT, 64><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_read(int dtype, const CacheRowsArgs& a, hipStream_t s) {
  return dtype ? read_hd<1>(a, s) : read_hd<0>(a, s);
}

}  // namespace lede
