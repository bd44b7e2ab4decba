// Log probabilities of given tokens, their ranks, the entropy and the most
// likely tokens of logits rows (gfx950).
#include "cache.h"
#include "device.h"

namespace lede {

// For a row z, its maximum m and a temperature T, with x_v = (z_v - m) c and c = log2(e) / T:
//   S = sum 2^x_v,  W = sum 2^x_v x_v,  log p_v = x_v ln 2 - ln S,  H = ln S - ln 2 W / S.
// (The difference comes before the product: m c would overflow in a row of a type's lowest values.)
//
// One pass over memory.  A block walks its part of a row in tiles that it
// holds in registers, the next one's loads in flight and no barrier before
// its end: each thread keeps a running maximum and sums of its own entries,
// and writes down the largest of each tile's.  These maxima lead to the top
// tokens: the n_top-th largest over groups of threads is a lower bound that
// few threads' tiles reach, and only those are read again.  Memory-bound for
// many rows: 2048 rows of 128256 in bf16 101 us without top tokens, 112 with 20
// (5.2 and 4.7 TB/s); a running list of the top ones took 162.
constexpr int LP_THREADS = 256, LP_PER = 32;
static_assert(LP_THREADS * LP_PER == LP_TILE, "a tile is LP_PER entries per thread");
constexpr float LP_FAR = 65536.f;   // |max c| from which the difference comes before the product everywhere
constexpr int LP_MAX_TOP = 32;
constexpr int LP_LIST = 512;     // candidates
constexpr int LP_SETS = 128;     // (tile, thread) pairs that are read again
static_assert(LP_LIST >= LP_MAX_TOP + LP_THREADS, "the best and one entry of each thread");

// Order of a value and its index: larger values first, a NaN before them all,
// -0 and +0 alike, then lower indices.
__device__ __forceinline__ uint64_t row_key(float z, int idx) {
  z = z == z ? z + 0.f : __builtin_nanf("");
  return argmax_key(z, idx);
}

// The largest float below z; NaN below -infinity.
__device__ __forceinline__ float below(float z) {
  if (z == 0.f) return -__uint_as_float(1);
  const uint32_t u = __float_as_uint(z);
  return __uint_as_float(u & 0x80000000u ? u + 1 : u - 1);
}

// The entries of a 16-byte piece.
template <int DT> __device__ __forceinline__ void unpack(uint4 r, float* z) {
  constexpr int E = 16 / Elem<DT>::ES_;
  const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int e = 0; e < E; ++e) z[e] = DT == 0 ? __uint_as_float(u[e & 3]) : e & 1 ? bf16hi(u[e / 2 & 3]) : bf16lo(u[e / 2 & 3]);
}

struct RowSums { float m, s, w; };
// (s, w) of entries with maximum a.m at the common maximum m.
__device__ __forceinline__ void rebase(RowSums& a, float m, float c) {
  const float d = fmaxf((a.m - m) * c, -1e4f), f = __builtin_amdgcn_exp2f(d);   // (no entry yet: f = 0)
  a.w = f * fmaf(a.s, d, a.w);
  a.s *= f;
  a.m = m;
}

// The row's numbers from its sums and its rank count (one thread).
// Returns ln S.
template <int DT>
__device__ __forceinline__ double finish_row(const LogprobsArgs& a, int row, RowSums t, int larger) {
  const double ln2 = 0.6931471805599453, ls = log((double)t.s);
  const float none = __builtin_nanf("");
  if (a.tokens) {
    const int tok = a.tokens[row];
    const bool given = tok >= 0 && tok < a.V;
    const uint8_t* zr = (const uint8_t*)a.logits + (int64_t)row * a.ld * Elem<DT>::ES_;
    if (a.logprobs) a.logprobs[row] = given ? (float)(((double)Elem<DT>::load(zr, tok) - t.m) * a.c * ln2 - ls) : none;
    if (a.ranks) a.ranks[row] = given ? larger : -1;
  }
  if (a.entropy) a.entropy[row] = (float)(ls - ln2 * ((double)t.w / t.s));
  return ls;
}
__device__ __forceinline__ void finish_top(const LogprobsArgs& a, int row, int place, uint64_t key, float m, double ls) {
  const int64_t at = (int64_t)row * a.n_top + place;
  a.top_ids[at] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
  a.top_logprobs[at] = (float)(((double)key_logit(key) - m) * a.c * 0.6931471805599453 - ls);
}

// How many of n keys in descending order are above k.
__device__ __forceinline__ int larger_keys(const uint64_t* keys, int n, uint64_t k) {
  int lo = 0, hi = n;   // entries [0, lo) are
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (keys[mid] > k) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// The best `top` of n keys, sorted, into dst; all threads of the block.
__device__ __forceinline__ void cut_list(const uint64_t* src, int n, uint64_t* dst, int top) {
  for (int i = threadIdx.x; i < n; i += LP_THREADS) {
    const uint64_t k = src[i];
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) before += src[j] > k;
    if (before < top) dst[before] = k;
  }
  __syncthreads();
}

template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs(LogprobsArgs a) {
  constexpr int ES = Elem<DT>::ES_, E = 16 / ES, NC = LP_PER / E;  // elements of a 16-byte piece, pieces per thread
  __shared__ float red[3][4];
  __shared__ int redi[4];
  __shared__ float tile_max[LP_PART_TILES][LP_THREADS];
  __shared__ uint64_t list[2][LP_LIST];
  __shared__ uint32_t group_max[64], bound;
  __shared__ uint16_t sets[LP_SETS];
  __shared__ int n_sets, n_found;
  __shared__ double row_ls;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / a.n_part, part = blockIdx.x % a.n_part;
  const int t_begin = part * a.part_tiles, t_end = min(t_begin + a.part_tiles, a.n_tiles);
  const uint8_t* zr = (const uint8_t*)a.logits + (int64_t)row * a.ld * ES;
  // pieces lie on 16-byte boundaries of memory: the row's first may begin before it
  const int lead = (int)((uintptr_t)zr & 15) / ES;
  const int V = a.V, top = a.n_top;
  const float c = a.c;
  const int tok = a.tokens ? a.tokens[row] : -1;
  const bool given = tok >= 0 && tok < V;
  const float zt = given ? Elem<DT>::load(zr, tok) : 0.f;
  // entries before the token count from zt on, those behind it above zt; a
  // NaN counts before everything (comparisons are written so that it does),
  // and only NaNs before a NaN token
  const bool nan_tok = !(zt == zt);
  const float thr_before = nan_tok ? INFINITY : below(zt);
  if (tid == 0) n_sets = n_found = 0;
  // entry e of piece i is the row's entry base + i * PITCH + e, with the
  // tile's and thread's own base: constants against one register
  constexpr int PITCH = LP_THREADS * E;
  auto base_of = [&](int t) { return t * LP_TILE + tid * E - lead; };
  uint4 raw[NC];
  auto load = [&](int t) {
    const int v0 = t * LP_TILE - lead, base = base_of(t);
    if (v0 >= 0 && v0 + LP_TILE <= V) {
      const uint8_t* p = zr + (int64_t)base * ES;
#pragma unroll
      for (int i = 0; i < NC; ++i) raw[i] = ld16_stream(p + i * (PITCH * ES));
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int p = base + i * PITCH;
        if (p >= 0 && p + E <= V) {
          raw[i] = ld16_stream(zr + (int64_t)p * ES);
        } else {
          float z[E];
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = p + e >= 0 && p + e < V ? Elem<DT>::load(zr, p + e) : -INFINITY;
          if (DT == 1) raw[i] = make_uint4(f32_to_bf16x2(z[0], z[1]), f32_to_bf16x2(z[2], z[3]), f32_to_bf16x2(z[E - 4], z[E - 3]), f32_to_bf16x2(z[E - 2], z[E - 1]));
          else raw[i] = make_uint4(__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3]));
        }
      }
    }
  };
  RowSums r{-INFINITY, 0.f, 0.f};
  int larger = 0, before_wave = 0;   // entries before the token: of this thread, of this wave
  float most = -INFINITY;   // of this thread's entries; a NaN if there is one
  load(t_begin);
  for (int t = t_begin; t < t_end; ++t) {
    float z[NC][E];
    const int base = base_of(t), lo = -base, hi = V - base, own = tok - base;   // places against i * PITCH + e
#pragma unroll
    for (int i = 0; i < NC; ++i) unpack<DT>(raw[i], z[i]);
    if (t + 1 < t_end) load(t + 1);
    float tm = z[0][0];
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) tm = __builtin_elementwise_maximum(tm, z[i][e]);
    most = __builtin_elementwise_maximum(most, tm);
    if (top) tile_max[t - t_begin][tid] = tm;
    if (tm > r.m) rebase(r, tm, c);
    const float shift = r.m == -INFINITY ? 0.f : r.m, sc = shift * c;
    const int v0 = t * LP_TILE - lead;
    if (v0 >= 0 && v0 + LP_TILE <= V && (tok < v0 || tok >= v0 + LP_TILE) && __ballot(fabsf(sc) < LP_FAR) == ~0ull) {
      // a whole tile before or behind the token: one bound for all, counted
      // on the scalar unit.  x = z c - sc, one operation; sc's rounding,
      // the same for all of them, is put right at the end of the tile: it is
      // at most 2^-9, and 2^off = 1 + g + g^2 / 2 to 2^-31, g = off ln 2
      const float thr = v0 < tok ? thr_before : zt;
      float s = 0.f, w = 0.f;
      int n = 0;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = fmaf(z[i][e], c, -sc), p = __builtin_amdgcn_exp2f(x);
          s += p;
          w = fmaf(p, fmaxf(x, -1e4f), w);   // (x = -infinity: p = 0)
          n += __popcll(__ballot(!(z[i][e] <= thr)));
        }
        __builtin_amdgcn_sched_barrier(0);   // (pieces one after the other: all at once take twice the registers)
      }
      const float off = -fmaf(shift, c, -sc);   // the true x is off larger
      const float g1 = off * 0.6931472f, g = fmaf(0.5f * g1, g1, g1);
      w = fmaf(off, s, w);
      r.s += fmaf(s, g, s);
      r.w += fmaf(w, g, w);
      if (!(nan_tok && v0 > tok)) before_wave += n;
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int o = i * PITCH;
        const float thr = o < own ? thr_before : zt;
        int n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = (z[i][e] - shift) * c, p = __builtin_amdgcn_exp2f(x);
          r.s += p;
          r.w = fmaf(p, fmaxf(x, -1e4f), r.w);
          n += !(z[i][e] <= thr);
        }
        if ((o <= own && own < o + E) || o < lo || o + E > hi) {   // the token's own piece, the row's ends
          n = 0;
          const uint64_t kt = row_key(zt, tok);
#pragma unroll 1
          for (int v = max(base + o, 0); v < min(base + o + E, V); ++v) n += row_key(Elem<DT>::load(zr, v), v) > kt;
        } else if (nan_tok && o > own) {
          n = 0;
        }
        larger += n;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // the block's sums at the block's maximum
  float m = wave_max(r.m);
  if (lane == 0) red[0][wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const bool none = r.m == -INFINITY && r.s == r.s;
  rebase(r, m, c);
  if (none) r.s = r.w = 0.f;
  const float ws = wave_sum(r.s), ww = wave_sum(r.w);
#pragma unroll
  for (int o = 32; o; o >>= 1) larger += __shfl_xor(larger, o);
  if (lane == 0) {
    red[1][wave] = ws;
    red[2][wave] = ww;
    redi[wave] = larger + before_wave;
  }
  __syncthreads();
  const RowSums all{m, red[1][0] + red[1][1] + red[1][2] + red[1][3], red[2][0] + red[2][1] + red[2][2] + red[2][3]};
  const int count = redi[0] + redi[1] + redi[2] + redi[3];
  int cur = 0, n_list = 0;
  if (top) {
    // the top-th largest of 64 groups' maxima, bit by bit from above
    auto order = [](float z) { return (uint32_t)(row_key(z, 0) >> 32); };
    uint32_t u = order(most);
    u = max(u, (uint32_t)__shfl_xor((int)u, 1));
    u = max(u, (uint32_t)__shfl_xor((int)u, 2));
    if ((tid & 3) == 0) group_max[tid >> 2] = u;
    __syncthreads();
    if (wave == 0) {
      const uint32_t g = group_max[lane];
      uint32_t b = 0;
      for (uint32_t bit = 1u << 31; bit; bit >>= 1)
        if (__popcll(__ballot(g >= (b | bit))) >= top) b |= bit;
      if (lane == 0) bound = b;
    }
    __syncthreads();
    const uint32_t least_u = bound;
    const int nt = t_end - t_begin;
    for (int t = 0; t < nt; ++t)
      if (order(tile_max[t][tid]) >= least_u && base_of(t_begin + t) < V) {
        const int at = atomicAdd(&n_sets, 1);
        if (at < LP_SETS) sets[at] = (uint16_t)(t << 8 | tid);
      }
    __syncthreads();
    const int ns = n_sets;
    auto read = [&](int t, int thread, int j) -> uint64_t {   // the key of a thread's entry j, 0 outside the row
      const int v = (t_begin + t) * LP_TILE + thread * E - lead + j / E * PITCH + j % E;
      return v >= 0 && v < V ? row_key(Elem<DT>::load(zr, v), v) : 0;
    };
    for (int i = tid >> 5; ns <= LP_SETS && i < ns; i += LP_THREADS / 32) {
      const uint64_t k = read(sets[i] >> 8, sets[i] & 255, tid & 31);
      if (k && (uint32_t)(k >> 32) >= least_u) {
        const int at = atomicAdd(&n_found, 1);
        if (at < LP_LIST) list[0][at] = k;
      }
    }
    __syncthreads();
    n_list = n_found;
    if (ns <= LP_SETS && n_list <= LP_LIST) {
      cut_list(list[0], n_list, list[1], top);
      cur = 1;
      n_list = min(n_list, top);
    } else {
      // many entries as large as the bound (a row of equal logits, one whose
      // mask leaves a few): tile by tile, one entry of each thread a round.
      // Once the list is full, a tile that holds nothing larger than its
      // last key cannot add to it: equal ones behind it come later.
      n_list = 0;
      uint64_t least = 0;
      for (int t = 0; t < nt; ++t) {
        if (!__syncthreads_or(!least || !(tile_max[t][tid] <= key_logit(least)))) continue;
        for (int j = 0; j < LP_PER; ++j) {
          if (tid == 0) n_found = 0;
          __syncthreads();
          const uint64_t k = read(t, tid, j);
          if (k && k >= least) list[cur][n_list + atomicAdd(&n_found, 1)] = k;
          __syncthreads();
          const int n = n_list + n_found;
          if (n == n_list) {
            __syncthreads();   // (all have read n_found)
            continue;
          }
          cut_list(list[cur], n, list[cur ^ 1], top);
          cur ^= 1;
          n_list = min(n, top);
          if (n_list == top) least = list[cur][top - 1];
        }
      }
    }
  }
  if (a.n_part > 1) {
    const int64_t at = (int64_t)row * a.n_part + part;
    if (tid == 0) a.part_stats[at] = make_float4(all.m, all.s, all.w, __int_as_float(count));
    if (tid < top) a.part_keys[at * top + tid] = tid < n_list ? list[cur][tid] : 0;
    return;
  }
  if (tid == 0) row_ls = finish_row<DT>(a, row, all, count);
  __syncthreads();
  if (tid < top) finish_top(a, row, tid, list[cur][tid], m, row_ls);
}

// One block per row: the parts' sums at their common maximum, the ranks, and
// the top keys: those of the parts' sorted lists that reach a bound, each
// placed by how many of them are larger.  A chain of LDS reads, so few of them:
// 5 rows of 128256, 20 top, 15 us with the parts' kernel, 28 with every key
// sought in every list (a row of 2^20, 32 top: 25 and 713).
template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_join(LogprobsArgs a) {
  extern __shared__ uint64_t keys[];
  __shared__ float row_m;
  __shared__ double row_ls;
  __shared__ uint64_t bound, found[LP_LIST];
  __shared__ int n_found;
  const int tid = threadIdx.x, row = blockIdx.x, top = a.n_top;
  const int n = a.n_part * top;
  if (tid == 0) {
    bound = 0;
    n_found = 0;
  }
  const uint64_t* src = a.part_keys + (int64_t)row * n;
  for (int i = tid; i < n; i += LP_THREADS) keys[i] = src[i];
  if (tid < 64) {
    const float4* p = a.part_stats + (int64_t)row * a.n_part;
    float m = -INFINITY;
    for (int i = tid; i < a.n_part; i += 64) m = fmaxf(m, p[i].x);
    m = wave_max(m);
    float s = 0.f, w = 0.f;
    int larger = 0;
    for (int i = tid; i < a.n_part; i += 64) {
      const float4 q = p[i];
      larger += __float_as_int(q.w);
      RowSums r{q.x, q.y, q.z};
      const bool none = r.m == -INFINITY && r.s == r.s;
      rebase(r, m, a.c);
      if (!none) {
        s += r.s;
        w += r.w;
      }
    }
    s = wave_sum(s);
    w = wave_sum(w);
#pragma unroll
    for (int o = 32; o; o >>= 1) larger += __shfl_xor(larger, o);
    if (tid == 0) {
      row_m = m;
      row_ls = finish_row<DT>(a, row, {m, s, w}, larger);
    }
  }
  __syncthreads();
  if (!top) return;
  // a bound that at least top keys reach: with i entries of each of c parts
  // the c-th largest of the i-th ones (i c >= top), or a part's last one
  const int i0 = (top + a.n_part - 1) / a.n_part, c0 = (top + i0 - 1) / i0;
  for (int p = tid; p < a.n_part; p += LP_THREADS) {
    const uint64_t k = keys[p * top + i0 - 1];
    int before = 0;
#pragma unroll 8
    for (int h = 0; h < a.n_part; ++h) before += keys[h * top + i0 - 1] > k;
    const uint64_t last = keys[p * top + top - 1];
    atomicMax((unsigned long long*)&bound, (unsigned long long)(k && before == c0 - 1 ? max(k, last) : last));
  }
  __syncthreads();
  const uint64_t least = bound;
  for (int i = tid; i < n; i += LP_THREADS)
    if (keys[i] && keys[i] >= least) {
      const int at = atomicAdd(&n_found, 1);
      if (at < LP_LIST) found[at] = keys[i];
    }
  __syncthreads();
  const float m = row_m;
  const double ls = row_ls;
  const bool fits = n_found <= LP_LIST;
  for (int i = tid; i < (fits ? n_found : n); i += LP_THREADS) {
    const uint64_t k = fits ? found[i] : keys[i];
    int before = 0;
    if (!k) continue;
    if (fits) {
#pragma unroll 8
      for (int j = 0; j < n_found; ++j) before += found[j] > k;
    } else {   // many as large: by the parts' sorted lists
      for (int h = 0; h < a.n_part && before < top; ++h) before += larger_keys(keys + h * top, top, k);
    }
    if (before < top) finish_top(a, row, before, k, m, ls);
  }
}

template <int DT>
static hipError_t logprobs_dt(const LogprobsArgs& a, hipStream_t s) {
  k_logprobs<DT><<<(unsigned)((int64_t)a.n_rows * a.n_part), LP_THREADS, 0, s>>>(a);
  if (a.n_part > 1) k_logprobs_join<DT><<<a.n_rows, LP_THREADS, (size_t)a.n_part * a.n_top * 8, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s) {
  return dtype ? logprobs_dt<1>(a, s) : logprobs_dt<0>(a, s);
}

}  // namespace lede
