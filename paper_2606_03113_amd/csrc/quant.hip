// Matrices of 4-bit weights with group scales: rounding to them, their packed
// layout, and products of rows with them (gfx950).
#include "device.h"
#include "products.h"

#include <type_traits>

namespace lede {

// ---- weights to codes -----------------------------------------------------------

// The nearest e2m1 magnitude of x >= 0 over a scale, ties to the even code.  The
// midpoints times a bf16 scale are exact in fp32 (at most 3 and 8 bits), so no
// quotient is rounded on the way.
__device__ __forceinline__ uint32_t nearest_e2m1(float x, float s) {
  return (x > 0.25f * s) + (x >= 0.75f * s) + (x > 1.25f * s) + (x >= 1.75f * s) + (x > 2.5f * s) + (x >= 3.5f * s) + (x > 5.f * s);
}

// A lane has eight columns of a row, the lanes of a group meet its largest
// magnitude by shuffles.  Done once for a matrix: 28672 x 4096 in 208 us from fp32
// (2.5 TB/s), 193 from bf16 (1.6), bound by loads of an element and stores of a byte.
template <int DT>
__global__ __launch_bounds__(256) void k_quantize(QuantizeArgs a) {
  const int groups = (a.K + a.group - 1) / a.group, lanes = a.group / 8;   // lanes of a group: 4, 8, 16
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;    // group of the matrix
  const int part = threadIdx.x % lanes;
  const bool in = at < (int64_t)a.N * groups;
  const int row = in ? (int)(at / groups) : 0, g = in ? (int)(at % groups) : 0;
  const int k0 = g * a.group + part * 8;
  float x[8], m = 0.f;
  bool finite = true;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = in && k0 + e < a.K ? Elem<DT>::load((const uint8_t*)a.w + row * a.ldw * Elem<DT>::ES_, k0 + e) : 0.f;
    finite = finite && fabsf(x[e]) < INFINITY;
    m = fmaxf(m, fabsf(x[e]));
  }
  int bad = !finite;
  for (int o = 1; o < lanes; o <<= 1) {
    m = fmaxf(m, __shfl_xor(m, o));
    bad |= __shfl_xor(bad, o);
  }
  if (!in) return;
  const uint16_t word = bad ? 0x7FC0 : f32_to_bf16(m / 6.f);
  const float s = bf16_to_f32(word);
  const int64_t pitch = (a.K + 1) / 2;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    if (k0 + 2 * b >= a.K) break;
    uint32_t c = 0;
    if (!bad && s > 0.f) {
      c = nearest_e2m1(fabsf(x[2 * b]), s) | (__float_as_uint(x[2 * b]) >> 31) << 3;
      c |= (nearest_e2m1(fabsf(x[2 * b + 1]), s) | (__float_as_uint(x[2 * b + 1]) >> 31) << 3) << 4;
    }
    a.codes[row * pitch + k0 / 2 + b] = (uint8_t)c;
  }
  if (part == 0) a.scales[at] = word;
}

template <int DT>
static hipError_t quantize_dt(const QuantizeArgs& a, hipStream_t s) {
  const int64_t threads = (int64_t)a.N * ((a.K + a.group - 1) / a.group) * (a.group / 8);
  k_quantize<DT><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s) { return dtype ? quantize_dt<1>(a, s) : quantize_dt<0>(a, s); }

// A wave packs a tile: a lane its 16 bytes of codes and some of its scales.  Done once
// for a matrix: 28672 x 4096 in 117 us (1.1 TB/s), bound by loads of a byte.
__global__ __launch_bounds__(64) void k_quant_pack(QuantPackArgs a, int tiles) {
  const int lane = threadIdx.x, g = blockIdx.x / tiles, t = blockIdx.x % tiles;
  const int row = g * 16 + (lane & 15);
  const int64_t pitch = (a.K + 1) / 2;
  uint32_t w[4] = {0, 0, 0, 0};
  if (row < a.N) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int k = t * QT_K + 32 * j + 8 * (lane >> 4) + 2 * b;
        if (k >= a.K) continue;
        const uint32_t c = a.codes[row * pitch + k / 2];
        w[j] |= (k + 1 < a.K ? c : c & 15) << (8 * b);
      }
  }
  *(uint4*)(a.dst_codes + (int64_t)blockIdx.x * 1024 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  const int per = QT_K / a.group, groups = (a.K + a.group - 1) / a.group;
  if (lane < 16 * per) {
    const int r = g * 16 + lane / per, c = t * per + lane % per;
    a.dst_scales[(int64_t)blockIdx.x * 16 * per + lane] = r < a.N && c < groups ? a.scales[(int64_t)r * groups + c] : 0;
  }
}
hipError_t launch_quant_pack(const QuantPackArgs& a, hipStream_t s) {
  const int tiles = q_tiles(a.K);
  k_quant_pack<<<(unsigned)((int64_t)q_groups(a.N) * tiles), 64, 0, s>>>(a, tiles);
  return hipGetLastError();
}

// ---- y = x W^T --------------------------------------------------------------------

// y[m][n] = sum over groups g of s[n][g] sum over k in g of x[m][k] c[n][k]: the
// inner sums are matrix products of bf16 numbers, exact in both operands (a
// code has two bits, an fp32 x is three bf16 numbers), summed in fp32 and
// scaled there.  Codes enter as c 2^-10, which the conversion gives for
// nothing: a group's sum is then no larger than its largest x, and overflows
// only where the result does.
constexpr float Q_DOWN = 0x1p-10f, Q_UP = 0x1p10f;

template <int I> __device__ __forceinline__ bf16x8 codes8(uint4 w) {
  const uint32_t c = I == 0 ? w.x : I == 1 ? w.y : I == 2 ? w.z : w.w;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, Q_DOWN, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, Q_DOWN, 1);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, Q_DOWN, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, Q_DOWN, 3);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

__device__ uint4 q_zeros[2];   // what is read in place of columns past the last

// Eight elements of a row of x as they came, and as matrix operands: one, or
// (fp32) three that sum to them exactly, cut off rather than rounded so that
// the first cannot overflow.  What is not finite is in the first part alone.
template <int DT> struct X8 {
  uint4 u[DT ? 1 : 2];
  __device__ __forceinline__ void zero() { u[0] = u[DT ? 0 : 1] = make_uint4(0, 0, 0, 0); }
  // VEC: rows in 16-byte pieces, K a multiple of 8
  template <bool VEC> __device__ __forceinline__ void load(const uint8_t* row, int k, int K) {
    if (VEC) {
      const uint8_t* p = k < K ? row + (int64_t)k * Elem<DT>::ES_ : (const uint8_t*)q_zeros;
      u[0] = ld16(p);
      if (DT == 0) u[DT ? 0 : 1] = ld16(p + 16);
      return;
    }
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      e[i] = k + i >= K ? 0 : DT ? ((const uint16_t*)row)[k + i] : ((const uint32_t*)row)[k + i];
    if (DT == 1) {
      u[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    } else {
      u[0] = make_uint4(e[0], e[1], e[2], e[3]);
      u[DT ? 0 : 1] = make_uint4(e[4], e[5], e[6], e[7]);
    }
  }
  static constexpr int PARTS = DT ? 1 : 3;
  __device__ __forceinline__ void parts(bf16x8 (&p)[PARTS]) const {
    if (DT == 1) {
      p[0] = __builtin_bit_cast(bf16x8, u[0]);
      return;
    }
    const uint4 hi = u[DT ? 0 : 1];
    const uint32_t e[8] = {u[0].x, u[0].y, u[0].z, u[0].w, hi.x, hi.y, hi.z, hi.w};
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t q[3];
      split3(e[i], q);
#pragma unroll
      for (int j = 0; j < 3; ++j) w[j][i / 2] = i & 1 ? w[j][i / 2] | (q[j] & 0xFFFF0000u) : q[j] >> 16;
    }
#pragma unroll
    for (int j = 0; j < PARTS; ++j) p[j] = __builtin_bit_cast(bf16x8, make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]));
  }
  static __device__ __forceinline__ void split3(uint32_t bits, uint32_t (&q)[3]) {
    const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
    q[0] = finite ? bits : bits | ((bits & 0x7FFFFFu) ? 0x400000u : 0u);   // (a NaN stays one without its low bits)
    const float rest = __uint_as_float(bits) - __uint_as_float(bits & 0xFFFF0000u);
    q[1] = finite ? __float_as_uint(rest) : 0u;
    q[2] = finite ? __float_as_uint(rest - __uint_as_float(q[1] & 0xFFFF0000u)) : 0u;
  }
};

__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// What a tile of W takes besides its codes: the scales of a lane's row.
template <int GROUP> struct Scales {
  static constexpr int PER = QT_K / GROUP;
  typedef typename std::conditional<PER == 4, uint2, typename std::conditional<PER == 2, uint32_t, uint16_t>::type>::type T;
  static __device__ __forceinline__ float get(const T& s, int p) { return __uint_as_float((uint32_t)((const uint16_t*)&s)[p] << 16); }
};

// acc[n][mt] += the products of TN tiles of 16 rows of W (codes w, scales s) with
// 16 MT rows of x, whose operands x(j, mt, part) gives for columns 32 j .. + 31.
// Results of lane l: W row l & 15, x rows 4 (l >> 4) + i, of which MR can be rows
// at all.  The next group's operands are read, and its products started,
// before a group is scaled.
template <int GROUP, int TN, int MT, int MR, int PARTS, class X>
__device__ __forceinline__ void tile_products(const uint4 (&w)[TN], const typename Scales<GROUP>::T (&s)[TN], f32x4 (&acc)[TN][MT], X x) {
  constexpr int PER = Scales<GROUP>::PER, J = 4 / PER, UNITS = PER * TN;
  f32x4 c[2][MT];
  bf16x8 xf[2][J][MT][PARTS];
  auto read = [&](int p) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int q = 0; q < PARTS; ++q) xf[p & 1][j][m][q] = x(p * J + j, m, q);
  };
  auto scale = [&](int u) {
    const int p = u / TN, n = u % TN;
    const float f = Scales<GROUP>::get(s[n], p);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < MR; ++i) acc[n][m][i] = fmaf(f, c[u & 1][m][i], acc[n][m][i]);
  };
  read(0);
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int p = u / TN, n = u % TN;
    if (n == 0 && p + 1 < PER) read(p + 1);
#pragma unroll
    for (int m = 0; m < MT; ++m) c[u & 1][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int jj = p * J + j;
      const bf16x8 b = jj == 0 ? codes8<0>(w[n]) : jj == 1 ? codes8<1>(w[n]) : jj == 2 ? codes8<2>(w[n]) : codes8<3>(w[n]);
#pragma unroll
      for (int q = PARTS - 1; q >= 0; --q)   // (the smallest part first)
#pragma unroll
        for (int m = 0; m < MT; ++m) c[u & 1][m] = mfma_bf16(xf[p & 1][j][m][q], b, c[u & 1][m]);
    }
    if (u) scale(u - 1);
  }
  scale(UNITS - 1);
}

__device__ __forceinline__ void store_y(const QuantLinearArgs& a, int m, int n, float v) {
  if (m >= a.M || n >= a.N) return;
  v *= Q_UP;
  if (a.y_dtype) Elem<1>::store(a.y, m * a.ldy + n, v);
  else Elem<0>::store(a.y, m * a.ldy + n, v);
}

// Few rows, all of x in LDS: a block has 16 rows of W; its waves take the tiles
// of K in turn, straight from memory into registers, D tiles ahead, and meet in
// LDS once.  The first tiles are on their way while x is brought to LDS as
// matrix operands ([part][row][column], rows 16 bytes apart besides).
template <int DT, int GROUP, bool VEC, int MR, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_quant_thin(QuantLinearArgs a) {
  constexpr int PARTS = X8<DT>::PARTS;
  typedef typename Scales<GROUP>::T S;
  __shared__ float part[WAVES][MR][64];
  extern __shared__ __align__(16) uint8_t xs[];
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, T = a.tiles;
  const uint8_t* wp = a.codes + (int64_t)g * T * 1024 + lane * 16;
  const S* sp = (const S*)a.scales + (int64_t)g * T * 16 + lr;
  uint4 w[D][1];
  S sc[D][1];
  auto load = [&](int u, int t) {
    w[u][0] = ld16_stream(wp + (int64_t)t * 1024);
    sc[u][0] = sp[t * 16];
  };
#pragma unroll
  for (int u = 0; u < D; ++u)
    if (wave + WAVES * u < T) load(u, wave + WAVES * u);
  const int pitch = T * QT_K * 2 + 16, plane = a.M * pitch, chunks = T * (QT_K / 8);
  for (int i = threadIdx.x; i < a.M * chunks; i += WAVES * 64) {
    const int m = i / chunks, k = (i - m * chunks) * 8;
    X8<DT> x;
    x.template load<VEC>((const uint8_t*)a.x + m * a.ldx * Elem<DT>::ES_, k, a.K);
    bf16x8 p[PARTS];
    x.parts(p);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) *(uint4*)(xs + q * plane + m * pitch + k * 2) = __builtin_bit_cast(uint4, p[q]);
  }
  __syncthreads();
  const uint8_t* xl = xs + min(lr, a.M - 1) * pitch + lg * 16;   // (rows past the last: the last)
  f32x4 acc[1][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}};
  for (int t0 = wave; t0 < T; t0 += WAVES * D) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      const int t = t0 + WAVES * u;
      if (t < T) {
        tile_products<GROUP, 1, 1, MR, PARTS>(w[u], sc[u], acc, [&](int j, int, int q) {
          return __builtin_bit_cast(bf16x8, lds_ld16(xl + q * plane + (t * QT_K + 32 * j) * 2));
        });
        if (t + WAVES * D < T) load(u, t + WAVES * D);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MR; ++i) part[wave][i][lane] = acc[0][0][i];
  __syncthreads();
  const int i = threadIdx.x >> 6;   // thread (i, lane) sums one result
  if (i >= MR) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < WAVES; ++q) v += part[q][i][lane];
  store_y(a, 4 * lg + i, g * 16 + lr, v);
}

// More rows: a block has 16 MT rows of x and WN x TN row groups of W.  WK tiles
// of K are a step: waves take them and the row groups; x's part of a step is in
// LDS for all waves, the next one's on its way in registers (where it becomes
// matrix operands), W's tiles straight in registers D steps ahead.
template <int DT, int GROUP, bool VEC, int MT, int TN, int WN, int WK, int D>
__global__ __launch_bounds__(WN * WK * 64) void k_quant_wide(QuantLinearArgs a) {
  constexpr int PARTS = X8<DT>::PARTS, THREADS = WN * WK * 64, ROWS = 16 * MT;
  constexpr int CH = ROWS * WK * 16, PER = CH / THREADS;              // 8-column chunks of x a step, of a thread
  constexpr int STAGE = PARTS * CH * 16;
  static_assert(CH % THREADS == 0, "");
  typedef typename Scales<GROUP>::T S;
  extern __shared__ __align__(16) uint8_t smem[];   // [2][part][tile of K][row][16 chunks, permuted by the row]
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wk = wave / WN, T = a.tiles;
  const int g0 = (blockIdx.x * WN + wn) * TN, m0 = blockIdx.y * ROWS;
  const uint8_t* wp[TN];
  const S* sp[TN];
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    const int64_t g = min(g0 + n, a.n_groups - 1);
    wp[n] = a.codes + g * T * 1024 + lane * 16;
    sp[n] = (const S*)a.scales + g * T * 16 + lr;
  }
  uint4 w[D][TN];
  S sc[D][TN];
  auto load_w = [&](int u, int t) {
    t = min(t, T - 1);
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      w[u][n] = ld16(wp[n] + (int64_t)t * 1024);
      sc[u][n] = sp[n][t * 16];
    }
  };
  X8<DT> x[D][PER];
  const uint8_t* xp[PER];
  int xk[PER];   // the column of a thread's chunk in a step
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = threadIdx.x + i * THREADS, row = c / (WK * 16);
    xk[i] = c % (WK * 16) * 8;
    xp[i] = (const uint8_t*)a.x + min(m0 + row, a.M - 1) * a.ldx * Elem<DT>::ES_;
  }
  auto load_x = [&](int u, int s) {
#pragma unroll
    for (int i = 0; i < PER; ++i) x[u][i].template load<VEC>(xp[i], s * WK * QT_K + xk[i], a.K);
  };
  auto store_x = [&](int u, int s) {
    uint8_t* stage = smem + (s & 1) * STAGE;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = threadIdx.x + i * THREADS, row = c / (WK * 16), kc = c % (WK * 16);
      bf16x8 p[PARTS];
      x[u][i].parts(p);
#pragma unroll
      for (int q = 0; q < PARTS; ++q)
        *(uint4*)(stage + (((q * WK + kc / 16) * ROWS + row) * 16 + ((kc ^ row) & 15)) * 16) = __builtin_bit_cast(uint4, p[q]);
    }
  };
  f32x4 acc[TN][MT];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (T + WK - 1) / WK;
  // Loads return in order: those of x wait for W's that were asked for before
  // them, so both are asked for equally far ahead; and no branch stands around
  // them (past the end they read the last tile and zeros), or the wait at the
  // place where its ways meet would be for all of them.
#pragma unroll
  for (int u = 0; u < D; ++u) {
    load_x(u, u);
    load_w(u, u * WK + wk);
  }
  for (int s0 = 0; s0 < steps; s0 += D) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      const int s = s0 + u, t = s * WK + wk;
      store_x(u, s);
      load_x(u, s + D);
      __syncthreads();
      if (t < T) {
        const uint8_t* xt = smem + (s & 1) * STAGE + wk * ROWS * 256;
        tile_products<GROUP, TN, MT, 4, PARTS>(w[u], sc[u], acc, [&](int j, int m, int q) {
          return __builtin_bit_cast(bf16x8, lds_ld16(xt + (q * WK * ROWS + 16 * m + lr) * 256 + (((4 * j + lg) ^ lr) << 4)));
        });
      }
      load_w(u, t + D * WK);
    }
  }
  if (WK == 1) {
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) store_y(a, m0 + 16 * m + 4 * lg + i, (g0 + n) * 16 + lr, acc[n][m][i]);
    return;
  }
  // the waves that share row groups meet: [wk][wn][n][m][lane]
  __syncthreads();
  float4* part = (float4*)smem;
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      part[(((wk * WN + wn) * TN + n) * MT + m) * 64 + lane] = make_float4(acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3]);
  __syncthreads();
  for (int o = wave; o < WN * TN * MT; o += WN * WK) {
    float4 v = part[o * 64 + lane];
#pragma unroll
    for (int q = 1; q < WK; ++q) {
      const float4 p = part[(q * WN * TN * MT + o) * 64 + lane];
      v = make_float4(v.x + p.x, v.y + p.y, v.z + p.z, v.w + p.w);
    }
    const int m = m0 + 16 * (o % MT) + 4 * lg, n = (blockIdx.x * WN * TN + o / MT) * 16 + lr;
    store_y(a, m, n, v.x);
    store_y(a, m + 1, n, v.y);
    store_y(a, m + 2, n, v.z);
    store_y(a, m + 3, n, v.w);
  }
}

constexpr size_t THIN_LDS = 64 * 1024;
static size_t thin_lds(int dtype, const QuantLinearArgs& a) { return (size_t)(dtype ? 1 : 3) * a.M * (a.tiles * QT_K * 2 + 16); }

template <int DT, int GROUP, bool VEC, int MR, int D, int WAVES>
static hipError_t launch_thin(const QuantLinearArgs& a, hipStream_t s) {
  const size_t lds = thin_lds(DT, a);
  const void* f = (const void*)k_quant_thin<DT, GROUP, VEC, MR, D, WAVES>;
  if (lds + WAVES * MR * 256 > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  void* args[] = {(void*)&a};
  return hipLaunchKernel(f, dim3(a.n_groups), dim3(WAVES * 64), args, lds, s);
}
template <int DT, int GROUP, bool VEC, int MT, int TN, int WN, int WK, int D>
static hipError_t launch_wide(const QuantLinearArgs& a, hipStream_t s) {
  constexpr size_t stage = (size_t)X8<DT>::PARTS * 16 * MT * WK * 256, meet = WK == 1 ? 0 : (size_t)WK * WN * TN * MT * 1024;
  constexpr size_t lds = 2 * stage > meet ? 2 * stage : meet;
  static_assert(lds <= 160 * 1024, "");
  const void* f = (const void*)k_quant_wide<DT, GROUP, VEC, MT, TN, WN, WK, D>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  void* args[] = {(void*)&a};
  return hipLaunchKernel(f, dim3((a.n_groups + WN * TN - 1) / (WN * TN), (a.M + 16 * MT - 1) / (16 * MT)), dim3(WN * WK * 64), args, lds, s);
}

// Which kernel, by sizes alone (us; all matrices 4096 wide but where another K is
// given, bf16 with groups of 64, fp32 likewise; weights from memory):
//  - x in LDS (k_quant_thin) where its rows take at most 64 KiB; of large
//    matrices for up to two rows (28672 outputs: 2 rows 14.1, 15.4 in
//    k_quant_wide; 4 rows 16.9, 13.8), for fp32 always (2 rows 23, 32).
//    16 waves share a K of few row groups (4096 outputs of 11008, one row: 6.7,
//    8.4 with 8), 8 of many (28672: 12.2, 15.1 with 16);
//  - k_quant_wide's blocks cover 32 or 64 rows of W by 16 of x, or 128 by 32 or
//    64.  The smaller ones while they are about a block a CU, the larger ones
//    read x and W less often:
//      outputs x rows       32 x 16  64 x 16  128 x 32  128 x 64
//      4096 x 16                6.3      7.3       12        20
//      5120 x 16                7.4      8.2
//      4096 x 64                9.3      7.3       13        20
//      28672 x 16                22       17       20        27
//      10000 x 40, K 5000        22       17       17        26
//      16384 x 64                32       23       17        23
//      22016 x 64                40       31       30        24
//      28672 x 256              206      145      105        90
//    fp32 (three parts of x, so less of it in LDS)  32 x 16  64 x 16  128 x 32
//      4096 x 32                                        15       16        34
//      4096 x 64                                        28       18        35
//      12288 x 24                                       40       31        36
//      12288 x 64                                       79       51        38
constexpr int MANY_GROUPS = 512;   // 8192 outputs
template <int DT, int GROUP, bool VEC>
static hipError_t linear_vec(const QuantLinearArgs& a, hipStream_t s) {
  const bool many = a.n_groups >= MANY_GROUPS;
  if (thin_lds(DT, a) <= THIN_LDS && a.M <= (DT && many ? 2 : 16)) {
    if (a.M == 1) return many ? launch_thin<DT, GROUP, VEC, 1, 4, 8>(a, s) : launch_thin<DT, GROUP, VEC, 1, 2, 16>(a, s);
    return many ? launch_thin<DT, GROUP, VEC, 4, 4, 8>(a, s) : launch_thin<DT, GROUP, VEC, 4, 2, 16>(a, s);
  }
  const int64_t m = (a.M + 15) / 16, b32 = (a.n_groups + 1) / 2 * m, b64 = (a.n_groups + 3) / 4 * m, b128 = (a.n_groups + 7) / 8 * ((m + 1) / 2);
  if constexpr (DT == 1) {
    if (b32 <= 256) return launch_wide<1, GROUP, VEC, 1, 2, 1, 8, 2>(a, s);
    if (m == 1 || b64 <= 512) return launch_wide<1, GROUP, VEC, 1, 2, 2, 4, 2>(a, s);
    if constexpr (VEC)   // (element by element it does not fit the registers)
      if (b128 <= 256) return launch_wide<1, GROUP, VEC, 2, 2, 4, 4, 2>(a, s);
    return launch_wide<1, GROUP, VEC, 4, 2, 4, 2, 2>(a, s);
  } else {
    if (b32 <= 256) return launch_wide<0, GROUP, VEC, 1, 1, 2, 4, 2>(a, s);
    if (m == 1 || b64 <= 512) return launch_wide<0, GROUP, VEC, 1, 2, 2, 4, 2>(a, s);
    return launch_wide<0, GROUP, VEC, 2, 2, 4, 2, 2>(a, s);
  }
}
// Rows of x that cannot be read in 16-byte pieces go element by element.
template <int DT, int GROUP>
static hipError_t linear_group(const QuantLinearArgs& a, hipStream_t s) {
  return a.vec ? linear_vec<DT, GROUP, true>(a, s) : linear_vec<DT, GROUP, false>(a, s);
}
template <int DT>
static hipError_t linear_dt(const QuantLinearArgs& a, hipStream_t s) {
  return a.group == 32 ? linear_group<DT, 32>(a, s) : a.group == 64 ? linear_group<DT, 64>(a, s) : linear_group<DT, 128>(a, s);
}
hipError_t launch_quant_linear(int dtype, const QuantLinearArgs& a, hipStream_t s) { return dtype ? linear_dt<1>(a, s) : linear_dt<0>(a, s); }

}  // namespace lede
