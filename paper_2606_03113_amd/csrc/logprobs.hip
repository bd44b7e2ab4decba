// Log probabilities of given tokens, their ranks, the entropy and the most
// likely tokens of logits rows (gfx950).
#include "cache.h"
#include "device.h"

namespace lede {

// For a row z, its maximum m and a temperature T, with x_v = (z_v - m) c and c = log2(e) / T:
//   S = sum 2^x_v,  W = sum 2^x_v x_v,  log p_v = x_v ln 2 - ln S,  H = ln S - ln 2 W / S.
// (The difference comes before the product: m c would overflow in a row of a type's lowest values.)
// One pass: a block keeps a segment of a row in registers, so that the
// maximum, the sums, the count of larger entries and the search for the top
// tokens all see one load of it.  A second kernel joins a row's segments.
constexpr int LP_THREADS = 256, LP_PER = 32, LP_SEG = LP_THREADS * LP_PER;
constexpr int LP_GROUP = 4;                    // threads whose largest entry is one of the 64 that bound the top ones
constexpr int LP_MAX_TOP = 32;
constexpr int LP_CAND = LP_MAX_TOP * LP_GROUP * LP_PER;

// Order of a value and its index: larger values first, a NaN before them all,
// -0 and +0 alike, then lower indices.
__device__ __forceinline__ uint64_t row_key(float z, int idx) {
  z = z == z ? z + 0.f : __builtin_nanf("");
  return argmax_key(z, idx);
}

template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs(LogprobsArgs a) {
  constexpr int ES = Elem<DT>::ES_, E = 16 / ES, NC = LP_PER / E;  // elements of a 16-byte piece, pieces per thread
  __shared__ float red[4], red2[4];
  __shared__ int redi[4];
  __shared__ uint64_t cand[LP_CAND];
  __shared__ uint64_t bound;
  __shared__ int n_cand;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / a.n_seg, seg = blockIdx.x % a.n_seg;
  const uint8_t* zr = (const uint8_t*)a.logits + (int64_t)row * a.ld * ES;
  // pieces lie on 16-byte boundaries of memory: the row's first may begin before it
  const int lead = (int)((uintptr_t)zr & 15) / ES;
  const int V = a.V;
  const int tok = a.tokens ? a.tokens[row] : -1;
  const bool given = tok >= 0 && tok < V;
  const float zt = given ? Elem<DT>::load(zr, tok) : 0.f;
  if (tid == 0) n_cand = 0;
  float z[NC][E];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int v0 = seg * LP_SEG + (i * LP_THREADS + tid) * E - lead;
    if (v0 >= 0 && v0 + E <= V) {
      const uint4 u = ld16_stream(zr + (int64_t)v0 * ES);
      if (DT == 1) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < E; ++e) z[i][e] = e & 1 ? bf16hi(w[e / 2]) : bf16lo(w[e / 2]);
      } else {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < E; ++e) z[i][e] = __uint_as_float(w[e & 3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) z[i][e] = v0 + e >= 0 && v0 + e < V ? Elem<DT>::load(zr, v0 + e) : -INFINITY;
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) mx = fmaxf(mx, z[i][e]);
  float bm = wave_max(mx);
  if (lane == 0) red[wave] = bm;
  __syncthreads();
  bm = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float shift = bm == -INFINITY ? 0.f : bm;
  float s = 0.f, w = 0.f;
  int larger = 0;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int v0 = seg * LP_SEG + (i * LP_THREADS + tid) * E - lead;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float x = (z[i][e] - shift) * a.c;
      const float p = __builtin_amdgcn_exp2f(x);
      s += p;
      w = fmaf(p, fmaxf(x, -1e4f), w);   // (x = -infinity: p = 0)
      larger += z[i][e] > zt || (z[i][e] == zt && v0 + e < tok && v0 + e >= 0);
    }
  }
  // a NaN (or an infinite) entry shows in the sum: then orders go by whole keys
  const bool odd = __syncthreads_or(!(s == s) || !(zt == zt));
  if (odd) {
    larger = 0;
    const uint64_t kt = row_key(zt, tok);
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = seg * LP_SEG + (i * LP_THREADS + tid) * E - lead + e;
        larger += v >= 0 && v < V && row_key(z[i][e], v) > kt;
      }
  }
  const float ws = wave_sum(s), ww = wave_sum(w);
  int wl = larger;
#pragma unroll
  for (int o = 32; o; o >>= 1) wl += __shfl_xor(wl, o);
  __syncthreads();
  if (lane == 0) {
    red[wave] = ws;
    red2[wave] = ww;
    redi[wave] = wl;
  }
  __syncthreads();
  if (tid == 0) {
    const int n = redi[0] + redi[1] + redi[2] + redi[3];
    a.seg_stats[(int64_t)row * a.n_seg + seg] =
        make_float4(bm, red[0] + red[1] + red[2] + red[3], red2[0] + red2[1] + red2[2] + red2[3], __int_as_float(n));
  }
  const int top = a.n_top;
  if (!top) return;
  // the largest key of each thread, then of each group of threads; the
  // top-th largest of the 64 groups' bounds the top ones from below, and at
  // most top groups hold entries that reach it
  uint64_t key = 0;
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = seg * LP_SEG + (i * LP_THREADS + tid) * E - lead + e;
      if ((odd || z[i][e] == mx) && v >= 0 && v < V) {
        const uint64_t k = row_key(z[i][e], v);
        key = k > key ? k : key;
      }
    }
#pragma unroll
  for (int o = 1; o < LP_GROUP; o <<= 1) {
    const uint64_t k = __shfl_xor((unsigned long long)key, o);
    key = k > key ? k : key;
  }
  if (tid % LP_GROUP == 0) cand[tid / LP_GROUP] = key;
  __syncthreads();
  if (wave == 0) {
    const uint64_t mine = cand[lane];
    int before = 0;
    for (int i = 0; i < 64; ++i) {
      const uint64_t k = cand[i];
      before += k > mine || (k == mine && i < lane);   // (equal keys: empty groups only)
    }
    if (before == top - 1) bound = mine;
  }
  __syncthreads();
  const uint64_t least = bound;
  const float lz = least ? key_logit(least) : -INFINITY;
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (!(z[i][e] < lz)) {
        const int v = seg * LP_SEG + (i * LP_THREADS + tid) * E - lead + e;
        if (v >= 0 && v < V) {
          const uint64_t k = row_key(z[i][e], v);
          if (k >= least) cand[atomicAdd(&n_cand, 1)] = k;
        }
      }
  __syncthreads();
  const int n = n_cand;
  uint64_t* out = a.seg_keys + ((int64_t)row * a.n_seg + seg) * top;
  for (int i = tid; i < n; i += LP_THREADS) {
    const uint64_t k = cand[i];
    int before = 0;
    for (int j = 0; j < n; ++j) before += cand[j] > k;
    if (before < top) out[before] = k;
  }
  for (int i = n + tid; i < top; i += LP_THREADS) out[i] = 0;
}

// One block per row: the segments' sums at their common shift, the ranks, and
// the top keys, each placed by how many larger ones the segments' sorted
// lists hold.
template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_join(LogprobsArgs a) {
  constexpr int ES = Elem<DT>::ES_;
  extern __shared__ uint64_t keys[];
  __shared__ __align__(16) float st[4];
  const int tid = threadIdx.x, row = blockIdx.x, top = a.n_top;
  const int n = a.n_seg * top;
  const uint64_t* src = a.seg_keys + (int64_t)row * n;
  for (int i = tid; i < n; i += LP_THREADS) keys[i] = src[i];
  if (tid < 64) {
    const float4* p = a.seg_stats + (int64_t)row * a.n_seg;
    float c = -INFINITY;
    for (int i = tid; i < a.n_seg; i += 64) c = fmaxf(c, p[i].x);
    c = wave_max(c);
    const float base = c == -INFINITY ? 0.f : c;
    float s = 0.f, w = 0.f;
    int larger = 0;
    for (int i = tid; i < a.n_seg; i += 64) {
      const float4 q = p[i];
      larger += __float_as_int(q.w);
      if (q.x == -INFINITY && q.y == q.y) continue;
      const float d = (q.x - base) * a.c, f = __builtin_amdgcn_exp2f(d);
      s = fmaf(q.y, f, s);
      w = fmaf(f, q.z + q.y * fmaxf(d, -1e4f), w);
    }
    s = wave_sum(s);
    w = wave_sum(w);
#pragma unroll
    for (int o = 32; o; o >>= 1) larger += __shfl_xor(larger, o);
    if (tid == 0) {
      const double ln2 = 0.6931471805599453, ls = log((double)s);
      const float none = __builtin_nanf("");
      st[0] = base;
      const uint8_t* zr = (const uint8_t*)a.logits + (int64_t)row * a.ld * ES;
      if (a.tokens) {
        const int tok = a.tokens[row];
        const bool given = tok >= 0 && tok < a.V;
        if (a.logprobs) a.logprobs[row] = given ? (float)(((double)Elem<DT>::load(zr, tok) - base) * a.c * ln2 - ls) : none;
        if (a.ranks) a.ranks[row] = given ? larger : -1;
      }
      if (a.entropy) a.entropy[row] = (float)(ls - ln2 * ((double)w / s));
      *(double*)(st + 2) = ls;
    }
  }
  __syncthreads();
  const float base = st[0];
  const double ls = *(const double*)(st + 2);
  for (int i = tid; i < n; i += LP_THREADS) {
    const uint64_t k = keys[i];
    const int g = i / top;
    int before = i % top;
    if (!k) continue;
    for (int h = 0; h < a.n_seg && before < top; ++h) {
      if (h == g) continue;
      int lo = 0, hi = top;   // entries [0, lo) are larger
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (keys[h * top + mid] > k) lo = mid + 1; else hi = mid;
      }
      before += lo;
    }
    if (before < top) {
      const int64_t at = (int64_t)row * top + before;
      a.top_ids[at] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
      a.top_logprobs[at] = (float)(((double)key_logit(k) - base) * a.c * 0.6931471805599453 - ls);
    }
  }
}

template <int DT>
static hipError_t logprobs_dt(const LogprobsArgs& a, hipStream_t s) {
  k_logprobs<DT><<<(unsigned)((int64_t)a.n_rows * a.n_seg), LP_THREADS, 0, s>>>(a);
  k_logprobs_join<DT><<<a.n_rows, LP_THREADS, (size_t)a.n_seg * a.n_top * 8, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s) {
  return dtype ? logprobs_dt<1>(a, s) : logprobs_dt<0>(a, s);
}

}  // namespace lede
