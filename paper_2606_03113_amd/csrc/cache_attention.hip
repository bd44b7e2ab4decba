// Attention over the paged 8-bit K/V cache (gfx950), for ragged batches.
#include "cache.h"
#include "device.h"

namespace lede {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// For query row i of a sequence with n rows and L cached tokens (its own
// included), p = L - n + i the row's position and t <= p:
//   o = sum w_t v_t / sum w_t,  w_t = exp(scale q . k_t).
// A row at a negative position sees nothing: o = 0.
//
// Codes become matrix operands in registers: e4m3 is exact in bf16 and fp16.
// q is exact in one bf16 operand (bf16 queries) or in three (fp32 queries).
// With E_k and E_v a page's scale exponents and c_t, d_t its codes, the kernels
// form the exponent of a whole term of the sum,
//   x_t = scale log2(e) q . (2^E_k c_t) + E_v - B,  o = sum 2^x_t d_t / sum 2^(x_t - E_v),
// so that the value product's accumulators take any mix of scales, its
// weights 2^x are as precise as the term's share of the result asks, and both
// scales cost nothing (one an operand of the codes' conversion, one of the add
// of a fused step).
// B is a whole number (its rounding cancels), P_UP below the largest x so
// far, and follows it only when some x passes P_LIM: until then neither the
// accumulators nor the maximum across lanes are touched.  The weights enter
// the product in fp16: 11 bits for bf16 outputs, whose own half step is 8
// times larger, and a high and a low part, 22 bits, for fp32.  Below 2^-14
// they lose bits, below 2^-25 they vanish: 2^-33 (bf16) or 2^-38 (fp32) of
// the largest term, from a million tokens together less than the rounding of
// the output.
// A page of small values (E_v = -100 if all are zero) has small terms, but its
// full part in the sum of 2^(x - E_v), and the result's dims in which the
// large pages hold zeros.  Where E_v is more than EV_NEAR below the largest so
// far, its weights are 2^lift as large, and so is o while they are added
// (2^O_LIFT at most: o is below 2^15 448 times the number of tokens); where
// that does not reach, its part of the sum is formed in fp32 apart.  Nearer
// pages' weights go in as they are, and lose less than 2^-28 of the largest
// weight each.  (A chunk of 3 x 1000 rows behind 4100 tokens: 157 us, 187 with
// values 2^12 larger in each first page.)  The sum is kept in fp32 at
// 2^-SUM_DOWN, and where B moves or sums of different B meet, it takes the
// factor in two halves: E_v goes from -100 to 120, so sums from 2^-122 to 2^105
// a token of the largest weight.
constexpr int P_LIM = 15, SUM_DOWN = 10, EV_NEAR = 4, O_LIFT = 64;
constexpr float B_NONE = -__FLT_MAX__;   // B of a row that has seen nothing: any finite score moves it, or has the weight 1
// From scores of 2^22 on, where fp32 has no room for B's whole part, the
// multiply and the add are rounded one by one, so that the largest score
// itself comes out as it went into B.
constexpr float B_FAR = 4194304.f;

// The square root of 2^d: a sum that is re-based takes it twice, since it may
// be as large as 2^d is small (B follows the values' scales, 2^-100 to 2^120).
__device__ __forceinline__ float half_step(float d) { return __builtin_amdgcn_exp2f(0.5f * d); }

// Token of a page that row `r` of its score tile `t` (16 tokens x 16 queries)
// holds.  A lane then has, of its query, the scores of 16 consecutive tokens
// (16 lg + 4 t + i from rows 4 lg + i), which is the value product's operand.
__device__ __forceinline__ int tile_token(int t, int r) { return (r >> 2) * 16 + 4 * t + (r & 3); }

// Half the scale of a page's keys, from its scale word: codes times it are the
// keys' halves, which bf16 holds for every scale (448 2^120 is above its
// largest number), so that a product overflows where half the score does.
__device__ __forceinline__ float key_scale(uint32_t word) { return __uint_as_float((max(word & 255, 127u + CACHE_E_MIN) - 1) << 23); }

// Eight codes times a power of two as a bf16 matrix operand, and as they are
// as an fp16 one.
__device__ __forceinline__ uint4 codes_bf16(uint2 c, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, scale, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, scale, true)));
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
// fp16 ones at an operand's NaNs, and the operand with zeros there.
__device__ __forceinline__ uint4 nan_ones(uint4 v) {
  auto one = [](uint32_t u) { return ((u & 0x7FFFu) > 0x7C00u ? 0x3C00u : 0u) | ((u >> 16 & 0x7FFFu) > 0x7C00u ? 0x3C000000u : 0u); };
  return make_uint4(one(v.x), one(v.y), one(v.z), one(v.w));
}
__device__ __forceinline__ uint4 nan_zeros(uint4 v) {
  auto zero = [](uint32_t u) { return u & (((u & 0x7FFFu) > 0x7C00u ? 0u : 0xFFFFu) | ((u >> 16 & 0x7FFFu) > 0x7C00u ? 0u : 0xFFFF0000u)); };
  return make_uint4(zero(v.x), zero(v.y), zero(v.z), zero(v.w));
}
// Four codes, and eight, zero where they are NaNs.
__device__ __forceinline__ uint32_t nan_codes_zero(uint32_t x) { return x & ~((((x & 0x7F7F7F7F) + 0x01010101) >> 7 & 0x01010101) * 0xFFu); }
__device__ __forceinline__ uint2 nan_zeros(uint2 c) { return make_uint2(nan_codes_zero(c.x), nan_codes_zero(c.y)); }
// fp16 ones at the first n of an operand's eight tokens.
__device__ __forceinline__ uint4 first_ones(int n) {
  auto two = [n](int i) { return (i < n ? 0x3C00u : 0u) | (i + 1 < n ? 0x3C000000u : 0u); };
  return make_uint4(two(0), two(2), two(4), two(6));
}

// A block's work: a tile of a sequence's (row, query head of the group) pairs
// for one KV head, and a split of its pages.  The first n_full tasks are
// blocks of their own; the others, which would leave the card partly idle in
// a last round, are n_split blocks each.  Of a sequence, tiles with more pages
// come first.
struct Task { int s, kvh, tile, split, n_split, slot; };
__device__ __forceinline__ Task attn_task(const CacheAttnArgs& a, int i) {   // task i, whole
  Task t{0, 0, 0, 0, 1, i - a.n_full};
  t.kvh = i % a.c.nkv;
  i /= a.c.nkv;
  t.tile = a.n_tiles - 1 - i % a.n_tiles;
  t.s = i / a.n_tiles;
  return t;
}
// Blocks of cut tasks: as many tasks as a sequence has together, one split
// after the other.  One long context among short ones is then under way from
// the start (30000 tokens among 63 of 1000: 67 us, and 99 with the first splits
// of all sequences before the others), and blocks that run together read
// neighbouring heads of the same pages (40 heads, 58590 tokens, fp32: 131 us,
// and 139 with a task's splits together).
__device__ __forceinline__ Task attn_block(const CacheAttnArgs& a, int bid) {
  const int x = bid - a.n_full;
  if (x < 0) return attn_task(a, bid);
  const int per = a.n_tiles * a.c.nkv, g = x / (per * a.n_split), n = min(per, a.n_cut - g * per), y = x - g * per * a.n_split;
  Task t = attn_task(a, a.n_full + g * per + y % n);
  t.split = y / n;
  t.n_split = a.n_split;
  return t;
}
// Pages of one split where a tile's rows see `pages`; all of them: no split.
__device__ __forceinline__ int split_chunk(const CacheAttnArgs& a, int n_split, int pages) {
  return n_split == 1 ? pages : max(a.min_chunk, (pages + n_split - 1) / n_split);
}
// A split's partial results of a tile's row: HD sums, then B and the weights' sum.
template <int HD>
__device__ __forceinline__ float* part_of(const CacheAttnArgs& a, int slot, int split, int r) {
  return a.part + (((int64_t)slot * a.n_split + split) * a.tile_rows + r) * (HD + 4);
}

// A sequence's rows and cached length, held to the call's own bounds.
struct AttnSeq { int row0, n, len; };
__device__ __forceinline__ AttnSeq attn_seq(const CacheAttnArgs& a, int s) {
  const int r0 = min(max(a.row_start[s], 0), a.n_rows), r1 = min(max(a.row_start[s + 1], r0), a.n_rows);
  const int64_t cap = (int64_t)a.table_ld * CACHE_PAGE;
  return {r0, r1 - r0, (int)min((int64_t)max(a.kv_lens[s], 0), cap)};
}

// NT tiles of 16 query rows ((row, query head of the group) pairs of one
// sequence and KV head), as a wave holds them.  A lane has the query lr = lane
// % 16 of each tile, and of its outputs the dims 16 d + 4 lg .. + 3, lg = lane
// / 16: both products' results lie so.  QL: the queries' operands are in LDS,
// for waves that share their rows.
template <int DT, int HD, int NT, bool QL = false>
struct Tiles {
  static constexpr int KH = HD / 64;      // 16-byte pieces of a key that a lane loads
  static constexpr int ND = HD / 16;      // 16-dim output tiles
  static constexpr int NQ = DT ? 1 : 3;   // bf16 parts of q
  static constexpr int NP = DT ? 1 : 2;   // fp16 parts of the weights
  static constexpr int P_UP = DT ? 8 : 13;
  static constexpr bool PIPE = !QL;       // operands come from LDS: a step's taken while the one before is multiplied
  uint4 qf[QL ? 1 : NT][NQ][KH][2];
  const uint4 (*ql)[NQ][KH][2][64];   // [NT]
  f32x4 o[NT][ND];
  float sum[NT], base[NT];
  int ev_most;                        // the largest value exponent of the pages so far
  int lift[NT];                       // o is at 2^lift
  bool lifted;                        // the last page was a small one (otherwise all lifts are 0)
  int pos[QL ? 1 : NT];
  const int (*pl)[16];                // [NT]: positions, beside the queries

  // Tile n of rows r0 .. of the R (row, head) pairs; tiles past R repeat the last.
  __device__ __forceinline__ static int row_at(int r0, int n, int R) { return min(r0 + 16 * n + (int)(threadIdx.x & 15), R - 1); }

  // Dims 64 h + 16 lg + 8 half .. + 7 of a tile's queries are the operand (h, half).
  __device__ __forceinline__ static void load_q(const CacheAttnArgs& a, const AttnSeq& q, int kvh, int G, int rr, uint4 (&f)[NQ][KH][2]) {
    const int lg = (threadIdx.x & 63) >> 4, m = rr / G, head = kvh * G + (rr - m * G);
    const int64_t at = (int64_t)(q.row0 + m) * a.ldq + head * HD;
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int64_t i = at + 64 * h + 16 * lg + 8 * half;
        if (DT == 1) {
          const uint4 u = ld16((const uint16_t*)a.q + i);
          f[0][h][half] = make_uint4(u.x ^ a.q_sign, u.y ^ a.q_sign, u.z ^ a.q_sign, u.w ^ a.q_sign);
        } else {
          float x[8];
          *(float4*)x = *(const float4*)((const float*)a.q + i);
          *(float4*)(x + 4) = *(const float4*)((const float*)a.q + i + 4);
#pragma unroll
          for (int p = 0; p < NQ; ++p) {
            uint32_t u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // (cut off, 8 bits a part: rounded, a number above bf16's largest would become infinite)
              u[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302);
              x[2 * e] -= bf16lo(u[e]);
              x[2 * e + 1] -= bf16hi(u[e]);
            }
            f[p][h][half] = make_uint4(u[0] ^ a.q_sign, u[1] ^ a.q_sign, u[2] ^ a.q_sign, u[3] ^ a.q_sign);
          }
        }
      }
  }

  __device__ __forceinline__ void init(const CacheAttnArgs& a, const AttnSeq& q, int kvh, int G, int r0, int R) {
    ev_most = INT_MIN / 2;
    lifted = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int rr = row_at(r0, n, R);
      if (!QL) pos[QL ? 0 : n] = q.len - q.n + rr / G;
      sum[n] = 0.f;
      lift[n] = 0;
      base[n] = B_NONE;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (!QL) load_q(a, q, kvh, G, rr, qf[QL ? 0 : n]);
    }
  }
  __device__ __forceinline__ int position(int n) const { return QL ? pl[n][threadIdx.x & 15] : pos[QL ? 0 : n]; }
  __device__ __forceinline__ uint4 query(int n, int p, int h, int half) const {
    return QL ? ql[n][p][h][half][threadIdx.x & 63] : qf[QL ? 0 : n][p][h][half];
  }

  // The value sums of tile n at 2^to, and all at 1.
  __device__ __forceinline__ void lift_sums(int n, int to) {
    const float f = ldexpf(1.f, to - lift[n]);
    lift[n] = to;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][d][i] *= f;
  }
  __device__ __forceinline__ void settle() {
    if (lifted)
#pragma unroll
      for (int n = 0; n < NT; ++n) lift_sums(n, 0);
  }

  // One page: tokens t0 .. t0 + 63; this lane's key operand (t, h, half), times
  // key_scale, and value operand (d, half) from kf and vf.  wv: its values'
  // scale word.
  // pos_lo: the lowest position of the tiles' rows.  after_keys() once the
  // keys are used.
  template <class KF, class VF, class AK>
  __device__ __forceinline__ void page(const CacheAttnArgs& a, int t0, int pos_lo, bool known, uint32_t wv, KF kf, VF vf,
                                       AK after_keys) {
    const int lg = (threadIdx.x & 63) >> 4;
    const int ev = max((int)(wv & 255) - 127, CACHE_E_MIN);   // (a word of a block never written is 0)
    const int gap = ev_most - ev;
    const bool small = gap > EV_NEAR, rare = small || lifted;
    const float lim = rare ? -INFINITY : P_LIM;
    const int unit = gap > O_LIFT ? -1000 : -ev - SUM_DOWN;   // (of the weights' sum; O_LIFT above: not taken)
    ev_most = max(ev_most, ev);
    // lane: token t0 + 16 lg + 4 t + i of its query.  Two key tiles at a time:
    // products on one accumulator wait for each other
    f32x4 x[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t) x[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint4 cur[2];
    if (PIPE) {
      cur[0] = kf(0, 0, 0);
      cur[1] = kf(1, 0, 0);
    }
    __builtin_amdgcn_s_setprio(1);   // a wave in its products goes first; the SIMD's other has its exponentials (3%)
#pragma unroll
    for (int i = 0; i < 4 * KH; ++i) {
      const int t = i / (2 * KH) * 2, h = i / 2 % KH, half = i & 1;
      uint4 nxt[2];
      if (!PIPE) {
        cur[0] = kf(t, h, half);
        cur[1] = kf(t + 1, h, half);
      } else if (i + 1 < 4 * KH) {
        const int t1 = (i + 1) / (2 * KH) * 2, h1 = (i + 1) / 2 % KH;
        nxt[0] = kf(t1, h1, (i + 1) & 1);
        nxt[1] = kf(t1 + 1, h1, (i + 1) & 1);
      } else {
        nxt[0] = vf(0, 0);
        nxt[1] = vf(1, 0);
      }
#pragma unroll
      for (int p = 0; p < NQ; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 qo = query(n, p, h, half);
#pragma unroll
          for (int u = 0; u < 2; ++u) x[n][t + u] = mfma_tile<1>(cur[u], qo, x[n][t + u]);
        }
      if (PIPE) {
        cur[0] = nxt[0];
        cur[1] = nxt[1];
      }
      if (NT > 1) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    after_keys();
    const bool edge = !known || t0 + CACHE_PAGE - 1 > pos_lo;
    uint4 pf[NT][NP][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float up = (float)(ev + P_UP) - base[n];
      const bool far = __ballot(fabsf(up) > B_FAR) != 0;
      float m = -INFINITY, kx = a.scale_log2x2;   // x = kx x' + up
      if (edge || far) {
        // a table entry outside the pool: rows that see the page become NaN
        kx = 1.f;
        const int last = position(n);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[n][t][i] = t0 + 16 * lg + 4 * t + i > last ? -INFINITY : known ? x[n][t][i] * a.scale_log2x2 : __builtin_nanf("");
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, x[n][t][i]);
      m *= kx;   // (the scale is not negative: q takes its sign)
      float off = up;
      if (__ballot(m + up >= lim)) {
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        if (!rare || __ballot(m + up > P_LIM)) {
          // the row's new B, the same in its four lanes
          const float b = !(m + up > P_LIM) ? base[n] : fabsf(m) < B_FAR ? ceilf(m + ev) : m + (float)(ev + P_UP);
          const float h = half_step(base[n] - b), f = h * h;
          base[n] = b;
          off = (float)(ev + P_UP) - b;
          sum[n] = sum[n] * h * h;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][d][i] *= f;
          if (__ballot(fabsf(off) > B_FAR)) {   // a step of such scores may be more than P_LIM
            const float most = P_LIM - off;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float y = x[n][t][i] * kx;
                x[n][t][i] = y > most ? most : y;
              }
            kx = 1.f;
          }
        }
        if (rare) {
          // a small page's weights as if its values were the largest, 2^more
          // times as large, where the row's limit leaves room
          int next = 0;
          if (small) {
            const float more = fminf((float)gap, fmaxf(P_LIM - ceilf(m + off), 0.f));
            next = min((int)more, O_LIFT);
            if (__ballot(fabsf(off) > B_FAR)) {   // (no room for a few powers of two more)
#pragma unroll
              for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][t][i] = fmaf(x[n][t][i], kx, off);
              kx = 1.f;
              off = 0.f;
            }
            if (gap > O_LIFT) {   // the weights are not 2^more larger, but the sum's
              float own = 0.f;
#pragma unroll
              for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) own += __builtin_amdgcn_exp2f(fmaf(x[n][t][i], kx, off + more));
              sum[n] += ldexpf(own, -ev - SUM_DOWN - (int)more);
            }
            off += (float)next;
          }
          if (__ballot(next != lift[n])) lift_sums(n, next);
        }
      }
      float ps = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[n][t][i] = __builtin_amdgcn_exp2f(fmaf(x[n][t][i], kx, off));
          if (DT == 0) ps += x[n][t][i];
        }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = 2 * half + e / 2, i = 2 * (e & 1);
            u[e] = pack_f16(x[n][t][i], x[n][t][i + 1]);
            // (the weights as the product takes them, two an operation)
            if (DT == 1) ps = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, u[e]), f16x2{(_Float16)1.f, (_Float16)1.f}, ps, false);
            if (p + 1 < NP) {
              const f16x2 r = __builtin_bit_cast(f16x2, u[e]);
              x[n][t][i] -= (float)r[0];
              x[n][t][i + 1] -= (float)r[1];
            }
          }
          pf[n][p][half] = make_uint4(u[0], u[1], u[2], u[3]);
        }
      sum[n] += ldexpf(ps, unit - lift[n]);
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int d = i / 2 * 2, half = i & 1;
      uint4 nxt[2];
      if (!PIPE) {
        cur[0] = vf(d, half);
        cur[1] = vf(d + 1, half);
      } else if (i + 1 < ND) {
        nxt[0] = vf((i + 1) / 2 * 2, (i + 1) & 1);
        nxt[1] = vf((i + 1) / 2 * 2 + 1, (i + 1) & 1);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int u = 0; u < 2; ++u) o[n][d + u] = mfma_f16(cur[u], pf[n][p][half], o[n][d + u]);
      if (PIPE && i + 1 < ND) {
        cur[0] = nxt[0];
        cur[1] = nxt[1];
      }
      if (NT > 1) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    lifted = small;
  }

  // A page with NaN values: they reach the rows that see their tokens, and no
  // others.  A product of indicators finds those rows; page() then takes the
  // values with zeros in their place.
  template <class VF>
  __device__ __forceinline__ void mark_nans(int t0, VF vf) {
    const int lg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const uint4 n0 = nan_ones(vf(d, 0)), n1 = nan_ones(vf(d, 1));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int seen = position(n) - (t0 + 16 * lg) + 1;
        f32x4 hit = {0.f, 0.f, 0.f, 0.f};
        hit = mfma_f16(n0, first_ones(seen), hit);
        hit = mfma_f16(n1, first_ones(seen - 8), hit);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][d][i] = hit[i] > 0.f ? __builtin_nanf("") : o[n][d][i];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Value codes of tokens from nv on are whatever the page held before: zero.
__device__ __forceinline__ uint4 keep_tokens(uint4 v, int nv) {
  return make_uint4(keep_bytes(v.x, nv), keep_bytes(v.y, nv - 4), keep_bytes(v.z, nv - 8), keep_bytes(v.w, nv - 12));
}

// The next pages of a walk: 64 at a time, page and scale words in the lanes.
// An entry outside the pool reads page 0 (and is known to).
struct Walk {
  int id = -1;
  uint2 words = {0, 0};
  // lane i: logical page j + stride * i, of those below j_end
  __device__ __forceinline__ void load(const CacheAttnArgs& a, const int32_t* table, int kvh, int j, int stride, int j_end) {
    const int64_t at = j + (int64_t)stride * (threadIdx.x & 63);
    id = at < j_end ? table[at] : -1;
    const int p = id >= 0 && id < a.c.n_pages ? id : 0;
    words = *(const uint2*)(a.c.words + ((size_t)p * a.c.nkv + kvh) * 2);
  }
};

// A result's four dims d .. d + 3: of an output row, or of a split's partial.
template <int DT, int HD>
__device__ __forceinline__ void put4(const CacheAttnArgs& a, const AttnSeq& q, int kvh, int G, int ri, int d, float* part, f32x4 acc,
                                     float base, float sum) {
  if (!part) {
    const int m = ri / G, head = kvh * G + (ri - m * G);
    const int64_t row = q.row0 + m;
    // a row that sees nothing is 0; one whose scores are all -infinity has no softmax
    const float inv = q.len - q.n + m < 0 ? 0.f : ldexpf(1.f / sum, -SUM_DOWN);
    store4<DT>((uint8_t*)a.out + (row * a.ldo + head * HD) * Elem<DT>::ES_, d, make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv));
  } else {
    *(f32x4*)(part + d) = acc;
    if (d == 0) *(float2*)(part + HD) = make_float2(base, sum);
  }
}

// Few rows, 16 NT a tile: one split of a sequence's pages, which the block's four
// waves take in turn for all of its rows, each with sums of its own.  Keys and
// values go from memory straight into the operands' registers (no LDS, no
// barrier), the next page's requested as soon as this one's are used; of two
// tiles the queries are in LDS, to leave them room.  The waves meet in LDS
// once, at the end.  ALONE: each wave has a task of its own, and nothing to do
// with the others.  Memory-bound: 64 sequences of up to 6000 tokens (8 KV
// heads of 128, 609 MB) 115-120 us, 5.1-5.3 TB/s, as fast as a kernel that only
// reads; with 32 rows each (up to 8000 tokens, 819 MB) 164 us, 5.0 TB/s.  A second
// page ahead in registers would not fit: the compiler spills 256 of them, and
// the step takes 384 us.
template <int DT, int HD, int NT, bool ALONE>
__global__ __launch_bounds__(256, 2) void k_cache_attn(CacheAttnArgs a) {
  static_assert(!ALONE || NT == 1, "queries in LDS are the block's");
  constexpr int STEP = ALONE ? 1 : 4;   // a wave takes every STEP-th page
  typedef Tiles<DT, HD, NT, (NT > 1)> T;
  constexpr int KH = T::KH, ND = T::ND;
  __shared__ uint4 ql[NT > 1 ? NT : 1][T::NQ][KH][2][NT > 1 ? 64 : 1];
  __shared__ int pl[NT][16];
  __shared__ float sm[STEP][16], sl[STEP][16];
  __shared__ __align__(16) float so[STEP][16][HD + 4];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
  if (ALONE && (int)blockIdx.x * 4 + w >= a.n_full) return;
  const Task task = attn_block(a, ALONE ? blockIdx.x * 4 + w : blockIdx.x);
  const int s = task.s, kvh = task.kvh;
  const AttnSeq q = attn_seq(a, s);
  const int G = a.nq / a.c.nkv;
  const int R = q.n * G;
  const int32_t* table = a.tables + (int64_t)s * a.table_ld;
  const uint8_t* kc = a.c.k + (size_t)kvh * (CACHE_PAGE * HD);
  const uint8_t* vc = a.c.v + (size_t)kvh * (CACHE_PAGE * HD);
  const size_t page_bytes = (size_t)a.c.nkv * (CACHE_PAGE * HD);
  // (rows behind the expected ones: every n_tiles-th tile more, whole)
  int n_split = task.n_split;
  for (int r0 = task.tile * (16 * NT); r0 < R; r0 += a.n_tiles * (16 * NT), n_split = 1) {
    const int nr = min(16 * NT, R - r0);
    const int pos_lo = q.len - q.n + r0 / G, pos_hi = q.len - q.n + (r0 + nr - 1) / G;
    const int pages = pos_hi < 0 ? 0 : pos_hi / CACHE_PAGE + 1;   // that some row of the tiles sees
    const int chunk = split_chunk(a, n_split, pages), j0 = task.split * chunk, j_end = min(pages, j0 + chunk);
    const bool direct = chunk >= pages;
    if (direct ? task.split > 0 : j0 >= pages) continue;
    int j = ALONE ? j0 : j0 + w;
    Walk walk;
    walk.load(a, table, kvh, j, STEP, j_end);
    T tiles;
    tiles.init(a, q, kvh, G, r0, R);
    if constexpr (NT > 1) {
      if (w < NT) {
        uint4 f[T::NQ][KH][2];
        T::load_q(a, q, kvh, G, T::row_at(r0, w, R), f);
#pragma unroll
        for (int p = 0; p < T::NQ; ++p)
#pragma unroll
          for (int h = 0; h < KH; ++h)
#pragma unroll
            for (int half = 0; half < 2; ++half) ql[w][p][h][half][l] = f[p][h][half];
        if (l < 16) pl[w][l] = q.len - q.n + T::row_at(r0, w, R) / G;
      }
      tiles.ql = ql;
      tiles.pl = pl;
      __syncthreads();
    }
    uint4 kf[4][KH], vf[ND];
    int id = 0;   // of the page in the registers
    auto page_at = [&](int i) {
      const int p = __builtin_amdgcn_readlane(walk.id, i);
      return p;
    };
    auto load_k = [&](int p) {
      const uint8_t* base = kc + (p >= 0 && p < a.c.n_pages ? p : 0) * page_bytes + 16 * lg;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < KH; ++h) kf[t][h] = ld16(base + tile_token(t, lr) * HD + 64 * h);
    };
    auto load_v = [&](int p) {
      const uint8_t* base = vc + (p >= 0 && p < a.c.n_pages ? p : 0) * page_bytes + lr * CACHE_PAGE + 16 * lg;
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = ld16(base + d * 16 * CACHE_PAGE);
    };
    if (j < j_end) {
      id = page_at(0);
      load_k(id);
      load_v(id);
    }
    for (int i = 0; j < j_end; j += STEP) {
      const bool known = id >= 0 && id < a.c.n_pages;
      const uint32_t wk = __builtin_amdgcn_readlane(walk.words.x, i), wv = __builtin_amdgcn_readlane(walk.words.y, i);
      const int t0 = j * CACHE_PAGE;
      const bool more = j + STEP < j_end;
      if (++i == 64) {
        i = 0;
        if (more) walk.load(a, table, kvh, j + STEP, STEP, j_end);
      }
      const int next = page_at(i);
      const int nv = known ? q.len - t0 : 0;
      if (nv < CACHE_PAGE)
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[d] = keep_tokens(vf[d], nv - 16 * lg);
      const auto value = [&](int d, int half) { return codes_f16(half ? make_uint2(vf[d].z, vf[d].w) : make_uint2(vf[d].x, vf[d].y)); };
      if (__builtin_expect((wv & CACHE_NAN) != 0, 0)) {
        tiles.mark_nans(t0, value);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          vf[d] = make_uint4(nan_codes_zero(vf[d].x), nan_codes_zero(vf[d].y), nan_codes_zero(vf[d].z), nan_codes_zero(vf[d].w));
      }
      const float ks = key_scale(wk);
      tiles.page(a, t0, pos_lo, known, wv,
                 [&](int t, int h, int half) { return codes_bf16(half ? make_uint2(kf[t][h].z, kf[t][h].w) : make_uint2(kf[t][h].x, kf[t][h].y), ks); },
                 value, [&] { if (more) load_k(next); });
      if (more) load_v(next);
      id = next;
    }
    tiles.settle();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (16 * n >= nr) break;
      float sum = tiles.sum[n];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (ALONE) {
        if (lr < nr)
#pragma unroll
          for (int d = 0; d < ND; ++d) put4<DT, HD>(a, q, kvh, G, r0 + lr, 16 * d + 4 * lg, nullptr, tiles.o[n][d], tiles.base[n], sum);
        continue;
      }
      if (lg == 0) {
        sm[w][lr] = tiles.base[n];
        sl[w][lr] = sum;
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) *(f32x4*)&so[w][lr][16 * d + 4 * lg] = tiles.o[n][d];
      __syncthreads();
      // the waves' states joined, four dims of a row per thread
      for (int i = threadIdx.x; i < min(16, nr - 16 * n) * (HD / 4); i += 256) {
        const int r = i / (HD / 4), d = i % (HD / 4) * 4;
        const float b = fmaxf(fmaxf(sm[0][r], sm[1 % STEP][r]), fmaxf(sm[2 % STEP][r], sm[3 % STEP][r]));
        float lsum = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
          const float h = half_step(sm[u][r] - b), f = h * h;
          lsum = fmaf(sl[u][r] * h, h, lsum);
          const f32x4 x = *(const f32x4*)&so[u][r][d];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = fmaf(x[e], f, acc[e]);
        }
        put4<DT, HD>(a, q, kvh, G, r0 + 16 * n + r, d, direct ? nullptr : part_of<HD>(a, task.slot, task.split, 16 * n + r), acc, b, lsum);
      }
      __syncthreads();
    }
  }
}

// What a staged piece holds, codes (uint2) or their operand (uint4), from
// codes, and its operand.  ks: the keys' scale.
template <bool B, class X, class Y> struct Pick { typedef X type; };
template <class X, class Y> struct Pick<false, X, Y> { typedef Y type; };
template <class T, bool KEYS> __device__ __forceinline__ T hold(uint2 c, float ks = 1.f) {
  if constexpr (sizeof(T) == 8) return c;
  else return KEYS ? codes_bf16(c, ks) : codes_f16(c);
}
template <bool KEYS> __device__ __forceinline__ uint4 operand(uint4 x, float = 1.f) { return x; }
template <bool KEYS> __device__ __forceinline__ uint4 operand(uint2 c, float ks = 1.f) { return KEYS ? codes_bf16(c, ks) : codes_f16(c); }

// Many rows: four waves with 16 NT rows each walk the same pages.  A page comes
// into LDS once per block, as 16-bit operands in the order in which the lanes
// take them (16 bytes per lane, a contiguous KiB per operand: no bank
// conflict either way), so that each wave converts a quarter of the codes;
// two pages' room, so one barrier a page.  Bound by the matrix units (41% of
// the SIMDs' clocks) and the vector instructions beside them (51%; both at once
// 7%): 995 TFLOP/s over whole rounds of 128-row tiles (bf16, heads of 128),
// against 1269 of a large library product; with the codes themselves in LDS,
// converted by every wave, 890.  RAW: codes all the same, for 64 bf16 rows and
// heads of 128 behind long contexts, bound by memory: half the LDS makes room
// for a third block, where there is one (30 sequences of up to 20000 tokens:
// 239 us, 271 with operands; 2 of up to 131000, one round of blocks: 77 and 75).
template <int DT, int HD, int NT, bool RAW>
__global__ __launch_bounds__(256, 2) void k_cache_attn_rows(CacheAttnArgs a) {
  typedef Tiles<DT, HD, NT> T;
  constexpr int KH = T::KH, ND = T::ND, VW = ND / 4;
  typedef typename Pick<RAW, uint2, uint4>::type Held;
  __shared__ Held sk[2][8 * KH][64], sv[2][2 * ND][64];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
  const Task task = attn_block(a, blockIdx.x);
  const int s = task.s, kvh = task.kvh;
  const AttnSeq q = attn_seq(a, s);
  const int G = a.nq / a.c.nkv;
  const int R = q.n * G;
  const int32_t* table = a.tables + (int64_t)s * a.table_ld;
  const uint8_t* kc = a.c.k + (size_t)kvh * (CACHE_PAGE * HD);
  const uint8_t* vc = a.c.v + (size_t)kvh * (CACHE_PAGE * HD);
  const size_t page_bytes = (size_t)a.c.nkv * (CACHE_PAGE * HD);
  constexpr int ROWS = 64 * NT;
  int n_split = task.n_split;
  for (int b0 = task.tile * ROWS; b0 < R; b0 += a.n_tiles * ROWS, n_split = 1) {
    const int pos_top = q.len - q.n + (min(b0 + ROWS, R) - 1) / G;
    const int pages = pos_top < 0 ? 0 : pos_top / CACHE_PAGE + 1;   // that some row of the block sees
    const int chunk = split_chunk(a, n_split, pages), j0 = task.split * chunk, j_end = min(pages, j0 + chunk);
    const bool direct = chunk >= pages;
    if (direct ? task.split > 0 : j0 >= pages) continue;
    const int r0 = b0 + w * (16 * NT), nr = min(16 * NT, R - r0);   // of this wave; none or less: it only loads
    const int pos_lo = q.len - q.n + min(r0, R - 1) / G;
    Walk walk;
    T tiles;
    tiles.init(a, q, kvh, G, r0, R);
    uint4 kr[KH], vr[VW];   // this wave's part of the next page: key tile w, value tiles VW w ..
    auto load = [&](int id) {
      const size_t at = (id >= 0 && id < a.c.n_pages ? id : 0) * page_bytes;
      const uint8_t* kb = kc + at + tile_token(w, lr) * HD + 16 * lg;
      const uint8_t* vb = vc + at + (w * VW * 16 + lr) * CACHE_PAGE + 16 * lg;
#pragma unroll
      for (int h = 0; h < KH; ++h) kr[h] = ld16(kb + 64 * h);
#pragma unroll
      for (int d = 0; d < VW; ++d) vr[d] = ld16(vb + d * 16 * CACHE_PAGE);
    };
    auto stage = [&](int buf, int id, int j, uint32_t wk) {
      const float ks = key_scale(wk);
      const int nv = id >= 0 && id < a.c.n_pages ? q.len - j * CACHE_PAGE : 0;
      if (nv < CACHE_PAGE)
#pragma unroll
        for (int d = 0; d < VW; ++d) vr[d] = keep_tokens(vr[d], nv - 16 * lg);
#pragma unroll
      for (int h = 0; h < KH; ++h) {
        sk[buf][2 * (w * KH + h)][l] = hold<Held, true>(make_uint2(kr[h].x, kr[h].y), ks);
        sk[buf][2 * (w * KH + h) + 1][l] = hold<Held, true>(make_uint2(kr[h].z, kr[h].w), ks);
      }
#pragma unroll
      for (int d = 0; d < VW; ++d) {
        sv[buf][2 * (w * VW + d)][l] = hold<Held, false>(make_uint2(vr[d].x, vr[d].y));
        sv[buf][2 * (w * VW + d) + 1][l] = hold<Held, false>(make_uint2(vr[d].z, vr[d].w));
      }
    };
    int id = 0;
    uint32_t wk = 0;   // of the page in LDS, as id
    if (j0 < j_end) {
      walk.load(a, table, kvh, j0, 1, j_end);
      id = __builtin_amdgcn_readlane(walk.id, 0);
      wk = __builtin_amdgcn_readlane(walk.words.x, 0);
      load(id);
      stage(0, id, j0, wk);
    }
    __syncthreads();
    for (int j = j0, i = 0, buf = 0; j < j_end; ++j, buf ^= 1) {
      const bool known = id >= 0 && id < a.c.n_pages;
      const uint32_t wv = __builtin_amdgcn_readlane(walk.words.y, i);
      const float ks = key_scale(wk);   // (of codes in LDS)
      const bool more = j + 1 < j_end;
      if (++i == 64) {
        i = 0;
        if (more) walk.load(a, table, kvh, j + 1, 1, j_end);
      }
      id = __builtin_amdgcn_readlane(walk.id, i);
      wk = __builtin_amdgcn_readlane(walk.words.x, i);
      if (more) load(id);
      if (__builtin_expect((wv & CACHE_NAN) != 0, 0)) {   // (the same for the whole block)
        tiles.mark_nans(j * CACHE_PAGE, [&](int d, int half) { return operand<false>(sv[buf][2 * d + half][l]); });
        __syncthreads();
#pragma unroll
        for (int d = 0; d < 2 * VW; ++d) sv[buf][2 * w * VW + d][l] = nan_zeros(sv[buf][2 * w * VW + d][l]);
        __syncthreads();
      }
      // (a wave whose rows end before the page, or that has none, computes masked scores: a branch
      // around the page costs every page a copy of the accumulators)
      tiles.page(a, j * CACHE_PAGE, pos_lo, known, wv, [&](int t, int h, int half) { return operand<true>(sk[buf][2 * (t * KH + h) + half][l], ks); },
                 [&](int d, int half) { return operand<false>(sv[buf][2 * d + half][l]); }, [] {});
      if (more) stage(buf ^ 1, id, j + 1, wk);
      __syncthreads();
    }
    tiles.settle();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float sum = tiles.sum[n];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (16 * n + lr < nr) {
        float* part = direct ? nullptr : part_of<HD>(a, task.slot, task.split, w * (16 * NT) + 16 * n + lr);
#pragma unroll
        for (int d = 0; d < ND; ++d) put4<DT, HD>(a, q, kvh, G, r0 + 16 * n + lr, 16 * d + 4 * lg, part, tiles.o[n][d], tiles.base[n], sum);
      }
    }
  }
}

// The splits of a row of a cut task joined in order: HD / 4 lanes a row, four
// dims each, B splits requested at a time (fp32 chunk of 5 x 77 rows: 6 us, and
// 9 with one dim a lane).
template <int DT, int HD, int B>
__global__ __launch_bounds__(256) void k_cache_attn_join(CacheAttnArgs a) {
  constexpr int LANES = HD / 4, ROWS = 256 / LANES;
  const int d = threadIdx.x % LANES * 4;
  const int G = a.nq / a.c.nkv;
  for (int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; i < (int64_t)a.n_cut * a.tile_rows; i += (int64_t)gridDim.x * ROWS) {
    const int slot = (int)(i / a.tile_rows), r = (int)(i % a.tile_rows);
    const Task t = attn_task(a, a.n_full + slot);
    const AttnSeq q = attn_seq(a, t.s);
    const int r0 = t.tile * a.tile_rows, ri = r0 + r, R = q.n * G;
    if (ri >= R) continue;
    const int pos_top = q.len - q.n + (min(r0 + a.tile_rows, R) - 1) / G;
    const int pages = pos_top < 0 ? 0 : pos_top / CACHE_PAGE + 1, chunk = split_chunk(a, a.n_split, pages);
    if (chunk >= pages) continue;
    const int pos = q.len - q.n + ri / G;
    const int n = pos < 0 ? 0 : pos / CACHE_PAGE / chunk + 1;
    const float* p = part_of<HD>(a, slot, 0, r);
    const int64_t pitch = (int64_t)a.tile_rows * (HD + 4);
    float b = B_NONE, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < n; j0 += B) {
      float2 bs[B];
      f32x4 pa[B];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const float* x = p + min(j0 + u, n - 1) * pitch;
        bs[u] = *(const float2*)(x + HD);
        pa[u] = *(const f32x4*)(x + d);
      }
      float nb = b, low = INFINITY;
#pragma unroll
      for (int u = 0; u < B; ++u) {
        nb = fmaxf(nb, j0 + u < n ? bs[u].x : B_NONE);
        low = fminf(low, j0 + u < n ? bs[u].x : INFINITY);
      }
      const float h0 = half_step(b - nb), f0 = h0 * h0;
      sum = sum * h0 * h0;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= f0;
      const float before = sum;
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const bool live = j0 + u < n;
        const float f = __builtin_amdgcn_exp2f(bs[u].x - nb);
        sum = live ? fmaf(bs[u].y, f, sum) : sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = live ? fmaf(pa[u][e], f, acc[e]) : acc[e];
      }
      if (__ballot(low - nb < -120.f)) {   // 2^(low - nb) is no number, its part of the sum may be one
        sum = before;
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const float h = half_step(bs[u].x - nb);
          sum = j0 + u < n ? fmaf(bs[u].y * h, h, sum) : sum;
        }
      }
      b = nb;
    }
    put4<DT, HD>(a, q, t.kvh, G, ri, d, nullptr, acc, b, sum);
  }
}

template <int DT, int HD>
static hipError_t attention_hd(const CacheAttnArgs& a, hipStream_t s) {
  const unsigned blocks = (unsigned)(a.n_full + a.n_cut * a.n_split);
  if (a.alone) k_cache_attn<DT, HD, 1, true><<<(blocks + 3) / 4, 256, 0, s>>>(a);
  else if (a.tile_rows == 16) k_cache_attn<DT, HD, 1, false><<<blocks, 256, 0, s>>>(a);
  else if (a.tile_rows == 32) k_cache_attn<DT, HD, 2, false><<<blocks, 256, 0, s>>>(a);
  else if (a.tile_rows == 64 && !a.raw) k_cache_attn_rows<DT, HD, 1, false><<<blocks, 256, 0, s>>>(a);
  else if constexpr (DT == 1 && HD == 128) {
    if (a.raw) k_cache_attn_rows<DT, HD, 1, true><<<blocks, 256, 0, s>>>(a);
    else k_cache_attn_rows<DT, HD, 2, false><<<blocks, 256, 0, s>>>(a);
  }
  if (a.n_cut > 0) {
    const int64_t rows = (int64_t)a.n_cut * a.tile_rows;
    const int64_t need = rows * (HD / 4) / 256;
    const unsigned grid = (unsigned)(need < 16384 ? need : 16384);
    if (a.n_split <= 2) k_cache_attn_join<DT, HD, 2><<<grid, 256, 0, s>>>(a);
    else if (a.n_split <= 4) k_cache_attn_join<DT, HD, 4><<<grid, 256, 0, s>>>(a);
    else k_cache_attn_join<DT, HD, 16><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
hipError_t launch_cache_attention(int dtype, const CacheAttnArgs& a, hipStream_t s) {
  if (dtype) return a.c.hd == 128 ? attention_hd<1, 128>(a, s) : attention_hd<1, 64>(a, s);
  return a.c.hd == 128 ? attention_hd<0, 128>(a, s) : attention_hd<0, 64>(a, s);
}

}  // namespace lede
