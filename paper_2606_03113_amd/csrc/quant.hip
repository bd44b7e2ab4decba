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
// magnitude by shuffles.  Memory-bound, and done once.
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

// A wave packs a tile: a lane its 16 bytes of codes and some of its scales.
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

// Eight elements of a row of x as they came, and as matrix operands: one, or
// (fp32) three that sum to them exactly, cut off rather than rounded so that
// the first cannot overflow.  What is not finite is in the first part alone.
template <int DT> struct X8 {
  uint4 u[DT ? 1 : 2];
  __device__ __forceinline__ void load(const uint8_t* row, int k, int K, bool vec) {
    if (vec && k + 8 <= K) {
      u[0] = ld16(row + (int64_t)k * Elem<DT>::ES_);
      if (DT == 0) u[DT ? 0 : 1] = ld16(row + (int64_t)k * Elem<DT>::ES_ + 16);
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

// Few rows: a block has 16 rows of W and 16 of x; its eight waves take the
// tiles of K in turn, straight from memory into the operands' registers, D
// tiles ahead, and meet in LDS once.  Lane l has x row l & 15 (rows past the
// last: the last) and the results of W row l & 15 for x rows 4 (l >> 4) + i.
// MR: how many of these i can be rows at all.
constexpr int QL_WAVES = 8;
template <int DT, int GROUP, int MR, int D>
__global__ __launch_bounds__(QL_WAVES * 64) void k_quant_thin(QuantLinearArgs a) {
  constexpr int PER = QT_K / GROUP, PARTS = X8<DT>::PARTS;
  typedef typename std::conditional<PER == 4, uint2, typename std::conditional<PER == 2, uint32_t, uint16_t>::type>::type Scales;
  __shared__ float part[QL_WAVES][MR][64];
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, m0 = blockIdx.y * 16, T = a.tiles;
  const uint8_t* wp = a.codes + (int64_t)g * T * 1024 + lane * 16;
  const Scales* sp = (const Scales*)a.scales + (int64_t)g * T * 16 + lr;
  const uint8_t* xr = (const uint8_t*)a.x + min(m0 + lr, a.M - 1) * a.ldx * Elem<DT>::ES_;
  uint4 w[D];
  Scales sc[D];
  X8<DT> x[D][4];
  auto load = [&](int u, int t) {   // (a step past the end reads the last tile again)
    t = min(t, T - 1);
    w[u] = ld16_stream(wp + (int64_t)t * 1024);
    sc[u] = sp[t * 16];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[u][j].load(xr, t * QT_K + 32 * j + 8 * lg, a.K, a.vec);
  };
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  auto step = [&](int u) {
    f32x4 c[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) c[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x8 b = j == 0 ? codes8<0>(w[u]) : j == 1 ? codes8<1>(w[u]) : j == 2 ? codes8<2>(w[u]) : codes8<3>(w[u]);
      bf16x8 p[PARTS];
      x[u][j].parts(p);
#pragma unroll
      for (int q = PARTS - 1; q >= 0; --q) c[j * PER / 4] = mfma_bf16(p[q], b, c[j * PER / 4]);   // (the smallest part first)
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const uint32_t word = ((const uint16_t*)&sc[u])[p];
      const float s = __uint_as_float(word << 16);
#pragma unroll
      for (int i = 0; i < MR; ++i) acc[i] = fmaf(s, c[p][i], acc[i]);
    }
  };
#pragma unroll
  for (int u = 0; u < D; ++u) load(u, wave + QL_WAVES * u);
  for (int t = wave; t < T; t += QL_WAVES * D) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      if (t + QL_WAVES * u < T) step(u);
      if (t + QL_WAVES * (u + D) < T) load(u, t + QL_WAVES * (u + D));
    }
  }
#pragma unroll
  for (int i = 0; i < MR; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  // thread (i, lane) sums one result
  const int i = threadIdx.x >> 6, m = m0 + 4 * lg + i, n = g * 16 + lr;
  if (i >= MR || m >= a.M || n >= a.N) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < QL_WAVES; ++q) v += part[q][i][lane];
  v *= Q_UP;
  if (a.y_dtype) Elem<1>::store(a.y, m * a.ldy + n, v);
  else Elem<0>::store(a.y, m * a.ldy + n, v);
}

template <int DT, int GROUP>
static hipError_t linear_group(const QuantLinearArgs& a, hipStream_t s) {
  const dim3 grid(a.n_groups, (a.M + 15) / 16);
  if (a.M == 1) k_quant_thin<DT, GROUP, 1, 4><<<grid, QL_WAVES * 64, 0, s>>>(a);
  else k_quant_thin<DT, GROUP, 4, 2><<<grid, QL_WAVES * 64, 0, s>>>(a);
  return hipGetLastError();
}
template <int DT>
static hipError_t linear_dt(const QuantLinearArgs& a, hipStream_t s) {
  return a.group == 32 ? linear_group<DT, 32>(a, s) : a.group == 64 ? linear_group<DT, 64>(a, s) : linear_group<DT, 128>(a, s);
}
hipError_t launch_quant_linear(int dtype, const QuantLinearArgs& a, hipStream_t s) { return dtype ? linear_dt<1>(a, s) : linear_dt<0>(a, s); }

}  // namespace lede
