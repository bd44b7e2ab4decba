// Attention over the paged 8-bit K/V cache (gfx950), for ragged batches.
#include "cache.h"
#include "device.h"

namespace lede {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// For query row i of a sequence with n rows and L cached tokens (its own
// included), p = L - n + i the row's position and t <= p:
//   s_t = scale q . k_t,  m = max s_t,  o = sum exp(s_t - m) v_t / sum exp(s_t - m).
// A row at a negative position sees nothing: o = 0.
//
// Codes become matrix operands in registers: e4m3 is exact in bf16 and fp16,
// and a block's power-of-two scale multiplies the page's scores (keys) and
// its value product (values), so no precision is lost there.  q is exact in
// one bf16 operand (bf16 queries) or in three (fp32 queries).  The weights
// enter the value product in fp16: 11 bits for bf16 outputs, whose own half
// step is 8 times larger, and as a high and a low part of 22 bits together
// for fp32.  They are computed as 2^P_UP exp(s - m), which cancels in the
// quotient and keeps weights down to 2^-14-P_UP in fp16's normal range.
constexpr int P_UP = 12;

// Token of a page that row `r` of its score tile `t` (16 tokens x 16 queries)
// holds.  A lane then has, of its query, the scores of 16 consecutive tokens
// (16 lg + 4 t + i from rows 4 lg + i), which is the value product's operand.
__device__ __forceinline__ int tile_token(int t, int r) { return (r >> 2) * 16 + 4 * t + (r & 3); }

// Eight codes as a bf16 or fp16 matrix operand.
__device__ __forceinline__ uint4 codes_bf16(uint2 c) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.f, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.f, true)));
}
__device__ __forceinline__ uint4 codes_f16(uint2 c) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, 1.f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, 1.f, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, 1.f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, 1.f, true)));
}
__device__ __forceinline__ f32x4 mfma_f16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

// Bytes [0, n) of a dword kept (n <= 0: none, n >= 4: all).
__device__ __forceinline__ uint32_t keep_bytes(uint32_t x, int n) {
  return n <= 0 ? 0u : n >= 4 ? x : x & (0xFFFFFFFFu >> (32 - 8 * n));
}
// 0x80 in every byte whose code is a NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7F7F7F7F) + 0x01010101) & 0x80808080; }
// fp16 ones where the bits of nan_bytes are set: a matrix operand of eight tokens.
__device__ __forceinline__ uint4 ones_f16(uint2 m) {
  auto two = [](uint32_t x, int i) {
    return ((x >> (8 * i + 7) & 1) ? 0x3C00u : 0u) | ((x >> (8 * i + 15) & 1) ? 0x3C000000u : 0u);
  };
  return make_uint4(two(m.x, 0), two(m.x, 2), two(m.y, 0), two(m.y, 2));
}

// The pages of a sequence that one split takes: chunks of at least min_chunk
// pages, as many pages for each split where there are more.
__device__ __forceinline__ int split_chunk(const CacheAttnArgs& a, int pages) {
  return max(a.min_chunk, (pages + a.n_split - 1) / a.n_split);
}

// A sequence's rows and cached length, held to the call's own bounds.
struct AttnSeq { int row0, n, len; };
__device__ __forceinline__ AttnSeq attn_seq(const CacheAttnArgs& a, int s) {
  const int r0 = min(max(a.row_start[s], 0), a.n_rows), r1 = min(max(a.row_start[s + 1], r0), a.n_rows);
  const int64_t cap = (int64_t)a.table_ld * CACHE_PAGE;
  return {r0, r1 - r0, (int)min((int64_t)max(a.kv_lens[s], 0), cap)};
}

// Up to 16 query rows ((row, query head of the group) pairs of one sequence
// and KV head) against one split of the sequence's pages.  The four waves
// take the pages in turn, each with a running maximum, sum and output of its
// own, all in registers: a page's keys and values are loaded straight into
// operand order, the scores' result layout is the weights' operand layout,
// and the next page's keys and values are requested as soon as this one's
// are used.  The waves meet in LDS once, at the end.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_cache_attn(CacheAttnArgs a) {
  constexpr int KH = HD / 64;          // 16-byte pieces of a key that a lane loads
  constexpr int ND = HD / 16;          // 16-dim output tiles
  constexpr int NQ = DT ? 1 : 3;       // bf16 parts of q
  constexpr int NP = DT ? 1 : 2;       // fp16 parts of the weights
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __align__(16) float so[4][16][HD + 4];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
  int bid = blockIdx.x;
  const int split = bid % a.n_split;
  bid /= a.n_split;
  const int kvh = bid % a.c.nkv;
  bid /= a.c.nkv;
  const int s = bid / a.n_tiles;
  const AttnSeq q = attn_seq(a, s);
  const int G = a.nq / a.c.nkv;
  const int64_t R = (int64_t)q.n * G;
  const int pages_all = (q.len + CACHE_PAGE - 1) / CACHE_PAGE;
  const int chunk = split_chunk(a, pages_all);
  const bool direct = pages_all <= chunk;
  const int32_t* table = a.tables + (int64_t)s * a.table_ld;
  const uint8_t* kc = a.c.k + (size_t)kvh * (CACHE_PAGE * HD);
  const uint8_t* vc = a.c.v + (size_t)kvh * (CACHE_PAGE * HD);
  const size_t page_bytes = (size_t)a.c.nkv * (CACHE_PAGE * HD);
  for (int64_t r0 = (int64_t)(bid % a.n_tiles) * 16; r0 < R; r0 += (int64_t)a.n_tiles * 16) {
    const int nr = (int)min((int64_t)16, R - r0);
    const int64_t rr = r0 + min(lr, nr - 1);   // rows past nr repeat the last one
    const int m_row = (int)(rr / G), head = kvh * G + (int)(rr % G);
    const int row_pos = q.len - q.n + m_row;
    const int pos_lo = q.len - q.n + (int)(r0 / G), pos_hi = q.len - q.n + (int)((r0 + nr - 1) / G);
    const int pages = pos_hi < 0 ? 0 : pos_hi / CACHE_PAGE + 1;   // that some row of the tile sees
    const int j_end = min(pages, (split + 1) * chunk);
    if (split * chunk >= pages && !(direct && split == 0)) continue;
    // this lane's query: dims 64 h + 16 lg + 8 half .. + 7 as operand (h, half)
    uint4 qf[NQ][KH][2];
    {
      const int64_t at = (int64_t)(q.row0 + m_row) * a.ldq + head * HD;
#pragma unroll
      for (int h = 0; h < KH; ++h)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int64_t i = at + 64 * h + 16 * lg + 8 * half;
          if (DT == 1) {
            qf[0][h][half] = ld16((const uint16_t*)a.q + i);
          } else {
            float x[8];
            *(float4*)x = *(const float4*)((const float*)a.q + i);
            *(float4*)(x + 4) = *(const float4*)((const float*)a.q + i + 4);
#pragma unroll
            for (int p = 0; p < NQ; ++p) {
              uint32_t u[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                u[e] = f32_to_bf16x2(x[2 * e], x[2 * e + 1]);
                x[2 * e] -= bf16lo(u[e]);
                x[2 * e + 1] -= bf16hi(u[e]);
              }
              qf[p][h][half] = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
        }
    }
    float mx = -INFINITY, sum = 0.f;
    f32x4 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint4 kf[4][KH], vf[ND];
    uint2 words = make_uint2(0, 0);
    int page = -1;
    auto find = [&](int j) {
      page = table[j];
      const int p = page >= 0 && page < a.c.n_pages ? page : 0;
      return p;
    };
    auto load_k = [&](int p) {
      const uint8_t* base = kc + p * page_bytes + 16 * lg;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < KH; ++h) kf[t][h] = ld16(base + tile_token(t, lr) * HD + 64 * h);
    };
    auto load_v = [&](int p) {
      const uint8_t* base = vc + p * page_bytes + lr * CACHE_PAGE + 16 * lg;
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = ld16(base + d * 16 * CACHE_PAGE);
    };
    int j = split * chunk + w;
    if (j < j_end) {
      const int p = find(j);
      load_k(p);
      load_v(p);
      words = *(const uint2*)(a.c.words + ((size_t)p * a.c.nkv + kvh) * 2);
    }
    for (; j < j_end; j += 4) {
      const bool known = page >= 0 && page < a.c.n_pages;
      const uint2 wd = words;
      const int t0 = j * CACHE_PAGE;
      const float ks = ldexpf(a.scale_log2, (int)(wd.x & 255) - 127);
      // scores: token t0 + 16 lg + 4 t + i of this lane's query
      float sv[16];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < KH; ++h) {
          const uint4 k0 = codes_bf16(make_uint2(kf[t][h].x, kf[t][h].y)), k1 = codes_bf16(make_uint2(kf[t][h].z, kf[t][h].w));
#pragma unroll
          for (int p = 0; p < NQ; ++p) {
            acc = mfma_tile<1>(k0, qf[p][h][0], acc);
            acc = mfma_tile<1>(k1, qf[p][h][1], acc);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sv[4 * t + i] = acc[i] * ks;
      }
      int next = 0;
      const bool more = j + 4 < j_end;
      if (more) {
        next = find(j + 4);
        load_k(next);
        words = *(const uint2*)(a.c.words + ((size_t)next * a.c.nkv + kvh) * 2);
      }
      if (!known || t0 + CACHE_PAGE - 1 > pos_lo) {
        // a table entry outside the pool: rows that see the page become NaN
#pragma unroll
        for (int i = 0; i < 16; ++i) sv[i] = t0 + 16 * lg + i > row_pos ? -INFINITY : known ? sv[i] : __builtin_nanf("");
        // value codes past the sequence's end are whatever the page held before
        const int nv = known ? q.len - t0 - 16 * lg : 0;
        if (nv < 16)
#pragma unroll
          for (int d = 0; d < ND; ++d)
            vf[d] = make_uint4(keep_bytes(vf[d].x, nv), keep_bytes(vf[d].y, nv - 4), keep_bytes(vf[d].z, nv - 8), keep_bytes(vf[d].w, nv - 12));
      }
      float pm = sv[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) pm = fmaxf(pm, sv[i]);
      pm = fmaxf(pm, __shfl_xor(pm, 16));
      pm = fmaxf(pm, __shfl_xor(pm, 32));
      const float nm = fmaxf(mx, pm);
      const float base = nm == -INFINITY ? 0.f : nm;   // nothing seen yet: weights 0
      const float alpha = __builtin_amdgcn_exp2f(mx - base);
      mx = nm;
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = __builtin_amdgcn_exp2f(sv[i] - base + P_UP);
      float ps = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) ps += sv[i];
      sum = fmaf(sum, alpha, ps);
      uint4 pf[NP][2];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float& x0 = sv[8 * half + 2 * e];
            float& x1 = sv[8 * half + 2 * e + 1];
            u[e] = pack_f16(x0, x1);
            if (p + 1 < NP) {
              const f16x2 r = __builtin_bit_cast(f16x2, u[e]);
              x0 -= (float)r[0];
              x1 -= (float)r[1];
            }
          }
          pf[p][half] = make_uint4(u[0], u[1], u[2], u[3]);
        }
      const float vs = ldexpf(1.f, (int)(wd.y & 255) - 127);
      if (__builtin_expect((wd.y & CACHE_NAN) != 0, 0)) {
        // NaN codes reach the rows that see their tokens, and no others: a
        // product of indicators finds those rows, and the codes become zero
        uint4 seen[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int t = t0 + 16 * lg + 8 * half;
          uint2 mk = make_uint2(0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (t + e <= row_pos) mk.x |= 0x80u << (8 * e);
            if (t + 4 + e <= row_pos) mk.y |= 0x80u << (8 * e);
          }
          seen[half] = ones_f16(mk);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          uint32_t c[4] = {vf[d].x, vf[d].y, vf[d].z, vf[d].w}, nb[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            nb[e] = nan_bytes(c[e]);
            c[e] &= ~((nb[e] >> 7) * 0xFFu);
          }
          f32x4 hit = {0.f, 0.f, 0.f, 0.f};
          hit = mfma_f16(ones_f16(make_uint2(nb[0], nb[1])), seen[0], hit);
          hit = mfma_f16(ones_f16(make_uint2(nb[2], nb[3])), seen[1], hit);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (hit[i] > 0.f) o[d][i] = __builtin_nanf("");
          vf[d] = make_uint4(c[0], c[1], c[2], c[3]);
        }
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const uint4 v0 = codes_f16(make_uint2(vf[d].x, vf[d].y)), v1 = codes_f16(make_uint2(vf[d].z, vf[d].w));
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          acc = mfma_f16(v0, pf[p][0], acc);
          acc = mfma_f16(v1, pf[p][1], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][i] = fmaf(acc[i], vs, o[d][i] * alpha);
      }
      if (more) load_v(next);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lg == 0) {
      sm[w][lr] = mx;
      sl[w][lr] = sum;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f32x4*)&so[w][lr][16 * d + 4 * lg] = o[d];
    __syncthreads();
    // the waves' states joined, four dims of a row per thread
    for (int i = threadIdx.x; i < nr * (HD / 4); i += 256) {
      const int r = i / (HD / 4), d = i % (HD / 4) * 4;
      const float m4 = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
      const float base = m4 == -INFINITY ? 0.f : m4;
      float lsum = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float f = __builtin_amdgcn_exp2f(sm[u][r] - base);
        lsum = fmaf(sl[u][r], f, lsum);
        const f32x4 x = *(const f32x4*)&so[u][r][d];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(x[e], f, acc[e]);
      }
      const int64_t ri = r0 + r;
      const int64_t row = q.row0 + ri / G;
      const int hd = kvh * G + (int)(ri % G);
      if (direct) {
        // a row that sees nothing is 0; one whose scores are all -infinity has no softmax
        const float inv = q.len - q.n + ri / G < 0 ? 0.f : 1.f / lsum;
        store4<DT>((uint8_t*)a.out + (row * a.ldo + hd * HD) * Elem<DT>::ES_, d,
                   make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv));
      } else {
        float* p = a.part + ((row * a.nq + hd) * a.n_split + split) * (HD + 2);
        *(float2*)(p + d) = make_float2(acc[0], acc[1]);
        *(float2*)(p + d + 2) = make_float2(acc[2], acc[3]);
        if (d == 0) *(float2*)(p + HD) = make_float2(m4, lsum);
      }
    }
    __syncthreads();
  }
}

// The splits of a (row, query head) joined in order: a wave each, lanes over
// the dims, sixteen splits requested at a time.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_cache_attn_join(CacheAttnArgs a) {
  constexpr int DL = HD / 64;
  const int l = threadIdx.x & 63;
  const int s = blockIdx.y;
  const AttnSeq q = attn_seq(a, s);
  const int pages_all = (q.len + CACHE_PAGE - 1) / CACHE_PAGE;
  const int chunk = split_chunk(a, pages_all);
  if (pages_all <= chunk) return;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < (int64_t)q.n * a.nq; i += (int64_t)gridDim.x * 4) {
    const int64_t row = q.row0 + i / a.nq;
    const int head = (int)(i % a.nq);
    const int pos = q.len - q.n + (int)(i / a.nq);
    const int n = pos < 0 ? 0 : pos / CACHE_PAGE / chunk + 1;
    const float* p = a.part + (row * a.nq + head) * a.n_split * (HD + 2);
    float mx = -INFINITY, sum = 0.f, acc[DL];
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[d] = 0.f;
    constexpr int B = 16;
    for (int j0 = 0; j0 < n; j0 += B) {
      float pm[B], pl[B], pa[B][DL];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const float* x = p + min(j0 + u, n - 1) * (HD + 2);
        const float2 ml = *(const float2*)(x + HD);
        pm[u] = j0 + u < n ? ml.x : -INFINITY;
        pl[u] = ml.y;
#pragma unroll
        for (int d = 0; d < DL; ++d) pa[u][d] = x[l * DL + d];
      }
      float nm = mx;
#pragma unroll
      for (int u = 0; u < B; ++u) nm = fmaxf(nm, pm[u]);
      const float base = nm == -INFINITY ? 0.f : nm;
      const float f0 = __builtin_amdgcn_exp2f(mx - base);
      sum *= f0;
#pragma unroll
      for (int d = 0; d < DL; ++d) acc[d] *= f0;
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const float f = __builtin_amdgcn_exp2f(pm[u] - base);
        const bool live = j0 + u < n;
        sum = live ? fmaf(pl[u], f, sum) : sum;
#pragma unroll
        for (int d = 0; d < DL; ++d) acc[d] = live ? fmaf(pa[u][d], f, acc[d]) : acc[d];
      }
      mx = nm;
    }
    const float inv = n == 0 ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < DL; ++d) Elem<DT>::store(a.out, row * a.ldo + head * HD + l * DL + d, acc[d] * inv);
  }
}

template <int DT, int HD>
static hipError_t attention_hd(const CacheAttnArgs& a, hipStream_t s) {
  k_cache_attn<DT, HD><<<(unsigned)((int64_t)a.n_seqs * a.n_tiles * a.c.nkv * a.n_split), 256, 0, s>>>(a);
  if (a.n_split > 1) {
    const int64_t per_seq = ((int64_t)a.n_rows * a.nq / a.n_seqs + 3) / 4;
    k_cache_attn_join<DT, HD><<<dim3((unsigned)(per_seq < 1 ? 1 : per_seq > 4096 ? 4096 : per_seq), a.n_seqs), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
hipError_t launch_cache_attention(int dtype, const CacheAttnArgs& a, hipStream_t s) {
  if (dtype) return a.c.hd == 128 ? attention_hd<1, 128>(a, s) : attention_hd<1, 64>(a, s);
  return a.c.hd == 128 ? attention_hd<0, 128>(a, s) : attention_hd<0, 64>(a, s);
}

}  // namespace lede
