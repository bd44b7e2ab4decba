// The vocabulary head's loss and its gradient without the logits (gfx950).
//
// For rows h_m, the head's rows w_v and targets t_m:
//   z_mv = h_m . w_v,  lse_m = log sum_v exp z_mv,  loss_m = lse_m - z_m,t
//   dz_mv = g_m (exp(z_mv - lse_m) - [v = t_m]),  dh = dz W,  dW = dz^T h
// Three products of 2 M V K operations, and the logits' once more in the
// backward pass, so that M V logits are never held (16384 rows of 128256 8.4 GB).
// That is memory for time: 2048 fp32 rows of 32000 are written and read in about
// 0.1 ms, their product of 4096 takes 0.4; and of few rows it reads the head a second
// time, where the logits would be little beside it (21 fp32 rows of 118860 x 5120:
// 478 us of 1.85 ms).  The forward pass keeps a maximum and a sum for each row and tile
// of the vocabulary; the backward pass holds dz for a piece of the vocabulary
// at a time.  Compute-bound for many rows, bound by the head's bytes for few.
#include "device.h"
#include "loss.h"

#include <algorithm>
#include <type_traits>

namespace lede {

// Four 16-bit entries of a column: of the 16 lanes of a group, lane i gives the
// address of entries 4 (i & 3) .. + 3 of row i >> 2 (of four rows) and gets
// column i's four.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t lds8;
__device__ __forceinline__ uint2 lds_column4(const lds8* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}
__device__ __forceinline__ bf16x8 lds_row8(const lds8* p) { return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) u32x4*)p); }

// An operand's tile in LDS: T rows (of the product's output) by 64 entries of
// the contraction, in one of two layouts, as it lies in memory:
//   rows  [T][64]: 128 bytes a row, 16-byte chunk c of row r at c ^ (r & 7)
//   columns  [64][T]: 2 T bytes an entry k of the contraction, its 32-byte unit u
//            at u ^ f(k), f such that the 16 entries k that a wave reads of a
//            unit at once (4 of each group of 8) lie in different banks
// Copies go from memory to LDS directly, 1 KiB a wave instruction in lane order;
// the permutation is in the lanes' source addresses.
constexpr int HD_K = 64;
constexpr uint32_t BUFFER_RANGE = 0xFFFFFFF0u;   // (a tile's rows span less than 2^31 bytes)
template <bool COLUMNS, int T, int NW> struct Operand {
  static constexpr int BYTES = T * HD_K * 2, PER = T / (8 * NW);   // copies of a wave
  static constexpr int CH = T / 8, RPI = 512 / T;                  // (columns) chunks of a row, rows of a copy
  const uint8_t* base;   // of the next step's copies: the same in all lanes
  uint32_t off[PER];
  int64_t step;

  // f(k) of a lane that reads entries 8 lg + 4 j + (lr >> 2); k & 3 and (k >> 3) & 3 stand for these bits.
  static __device__ __forceinline__ int perm(int k) {
    return T == 256 ? (k & 3) | (k >> 3 & 3) << 2 : T == 128 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1;
  }
  // The first entry of the contraction that copy i of a lane reads, in its step.
  static __device__ __forceinline__ int entry(int i, int wave) {
    const int lane = threadIdx.x & 63;
    return COLUMNS ? (wave * PER + i) * RPI + lane / CH : 8 * ((lane & 7) ^ (lane >> 3));
  }
  // From row r0 of n (clamped: what lies past the end is computed and not
  // kept; columns are read eight at a time), entry c0 of the contraction.
  __device__ __forceinline__ void begin(const uint8_t* p, int64_t ld, int r0, int n, int c0, int wave) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (!COLUMNS) {
        off[i] = ((uint32_t)min((wave * PER + i) * 8 + (lane >> 3), n - 1 - r0) * (uint32_t)ld + entry(i, wave)) * 2;
      } else {
        const int k = entry(i, wave), c = (lane % CH) ^ (perm(k) << 1);
        off[i] = ((uint32_t)k * (uint32_t)ld + min(8 * c, ((n + 7) & ~7) - 8 - r0)) * 2;
      }
    }
    base = p + (COLUMNS ? (int64_t)c0 * ld + r0 : (int64_t)r0 * ld + c0) * 2;
    step = COLUMNS ? HD_K * ld * 2 : HD_K * 2;
  }
  // The next step's copies; `left` entries of the contraction are left: what
  // lies behind them is out of the buffer's range and read as zeros.  (Buffer
  // loads: behind global ones, which are flat instructions, the compiler waits
  // for all LDS reads on their way instead of the oldest.)
  __device__ __forceinline__ void copy(lds8* tile, int left, int wave) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)BUFFER_RANGE, 0x00020000);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t o = left < HD_K && entry(i, wave) >= left ? BUFFER_RANGE : off[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(tile + (wave * PER + i) * 1024), 16, (int)o, 0, 0, 0);
    }
    base += step;
  }
  // The matrix operand of rows r0 .. r0 + 15, entries 32 h .. + 31.
  static __device__ __forceinline__ bf16x8 read(const lds8* tile, int r0, int h) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    if (!COLUMNS) {
      const int r = r0 + lr;
      return lds_row8(tile + r * 128 + (((4 * h + lg) ^ (r & 7)) << 4));
    }
    const int k = 32 * h + 8 * lg + (lr >> 2);
    const lds8* p = tile + k * (2 * T) + (((r0 >> 4) ^ perm(8 * lg + (lr >> 2))) << 5) + ((lr & 3) << 3);
    const uint2 a = lds_column4(p), b = lds_column4(p + 4 * 2 * T);
    return __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y));
  }
};

// This wave's LDS accesses, then all: loads on their way to registers are not waited for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_barrier() {   // this wave's copies but the last N, and its LDS reads; then all
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Two tiles' four entries of a lane (i = 4 lg ..), rounded: neighbouring lanes
// exchange them, so that each has eight in a row, from place i on of the two
// tiles' 32 (dW of 8 rows over 128256 x 5120 366 us, with stores of 8 bytes a
// lane 455).
__device__ __forceinline__ uint4 eight(const float (&d0)[4], const float (&d1)[4], int& i) {
  const int lg = (threadIdx.x & 63) >> 4;
  const bool odd = lg & 1;
  const uint32_t a0 = f32_to_bf16x2(d0[0], d0[1]), a1 = f32_to_bf16x2(d0[2], d0[3]), b0 = f32_to_bf16x2(d1[0], d1[1]), b1 = f32_to_bf16x2(d1[2], d1[3]);
  const uint32_t r0 = __shfl_xor((int)(odd ? a0 : b0), 16), r1 = __shfl_xor((int)(odd ? a1 : b1), 16);
  i = 16 * (lg & 1) + 4 * (lg & 2);
  return odd ? make_uint4(r0, r1, b0, b1) : make_uint4(a0, a1, r0, r1);
}

// The copies of the two operands, step after step.
template <class OA, class OB> struct Copies {
  OA oa;
  OB ob;
  int left, wave, done = 0;   // entries of the contraction that are left
  __device__ __forceinline__ void next(lds8* tile) {
    oa.copy(tile, left, wave);
    ob.copy(tile + OA::BYTES, left, wave);
    left -= HD_K;
    ++done;
  }
};

// The products of row x of a wave's tiles.
template <int NI, int NJ> __device__ __forceinline__ void multiply_row(int x, const bf16x8 (&fa)[NI], const bf16x8 (&fb)[NJ], f32x4 (&acc)[NI][NJ]) {
#pragma unroll
  for (int y = 0; y < NJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[x], fb[y], acc[x][y], 0, 0, 0);
}

// What stands between two barriers: the copies of a later step to the place `to`
// that the barrier has set free, all reads of the step in `cur`, which has arrived,
// and products.  The operands of half a step are read while the other half is
// multiplied: those of A into the registers that its products have just left,
// those of B into a second set; the second half's last products are made behind the
// next barrier, under its first reads (all steps but the FIRST begin with those of the
// step before).  cur and to are two places of the ring, so that within this
// function, where no barrier is, neither's accesses touch the other: told so, the
// compiler reads columns without waiting for copies on their way.  The barriers
// stand in the caller, where nothing is said of the pointers, and order all of it.
template <class OA, class OB, bool ORDER, bool FIRST, bool COPY, int EARLY, int NI, int NJ, class Copies_>
__device__ __forceinline__ void head_step(const lds8* __restrict__ cur, lds8* __restrict__ to, Copies_& copies, int wi, int wj, bf16x8 (&fa)[NI],
                                          bf16x8 (&fb)[2][NJ], f32x4 (&acc)[NI][NJ]) {
  auto keep_order = []() {
    if (ORDER) __builtin_amdgcn_sched_barrier(0);
  };
  auto read_a = [&](int h, int x) { fa[x] = OA::read(cur, (wi * NI + x) * 16, h); };
  auto read_b = [&](int h) {
#pragma unroll
    for (int y = 0; y < NJ; ++y) fb[h][y] = OB::read(cur + OA::BYTES, (wj * NJ + y) * 16, h);
  };
  if (COPY) copies.next(to);
  read_b(0);
#pragma unroll
  for (int x = 0; x < EARLY; ++x) read_a(0, x);
#pragma unroll
  for (int x = EARLY; x < NI; ++x) {
    if (!FIRST) multiply_row(x, fa, fb[1], acc);
    read_a(0, x);
    keep_order();
  }
  __builtin_amdgcn_sched_barrier(0);   // (dh's columns, of 2048 rows of 32000 x 4096: 452 us without it, 402 with)
#pragma unroll
  for (int x = 0; x < NI; ++x) {
    multiply_row(x, fa, fb[0], acc);
    if (x == 0) {   // (not before it: the count of reads on their way ends at 15)
      keep_order();
      read_b(1);
    }
    read_a(1, x);
    keep_order();   // (left alone, reads stand right before what waits for them)
  }
#pragma unroll
  for (int x = 0; x < EARLY; ++x) {
    multiply_row(x, fa, fb[1], acc);
    keep_order();
  }
}

// A block's place: blocks b, b + 8, .. run on one XCD, which takes an eighth of
// the tiles: one part of the contraction after the other, bands of four tiles
// of i with all tiles of j, so that what runs at a time is about square and
// shares its operands in the XCD's L2.  Of short contractions, bound by what
// they write, whole rows of the result instead (dW of 35 rows over 128256 x 5120
// 321 us, 357 in bands; for so few there is k_head_outer now).
struct HeadPlace { int part, it, jt; };
__device__ __forceinline__ bool head_place(const HeadArgs& a, HeadPlace& p) {
  const int per_part = a.i_tiles * a.j_tiles, per_xcd = (per_part * a.split + 7) / 8;
  const int at = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (at >= per_part * a.split) return false;
  p.part = at / per_part;
  const int rest = at - p.part * per_part, band = rest / (a.band * a.j_tiles);
  const int in_band = rest - band * a.band * a.j_tiles, rows = min(a.band, a.i_tiles - a.band * band);
  p.it = a.band * band + in_band % rows;
  p.jt = in_band / rows;
  return true;
}

// Whether row r, whose target is t, takes no part in a gradient.
__device__ __forceinline__ bool left_out(int t, const float* weights, int64_t r, int V) { return t < 0 || t >= V || (weights && weights[r] == 0.f); }

// What becomes of a block's tile of sums.  Lane (lr, lg) of a wave holds, of each
// of its 16 x 16 tiles, i = 4 lg + 0..3 of j = lr.
template <int DT, int EPI, int TI, int TJ, int WI, int WJ, int NI, int NJ>
__device__ __forceinline__ void head_finish(const HeadArgs& a, f32x4 (&acc)[NI][NJ], uint8_t* smem, const HeadPlace& place, int wi, int wj) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int it = place.it, i0 = it * TI, j0 = place.jt * TJ, part = place.part;
  if (EPI == HEAD_SUMS) {
    // of each row the maximum and the sum of exponentials of the tile's entries
    float2* red = (float2*)smem;   // [TJ][WI]
    copies_barrier<0>();
#pragma unroll
    for (int y = 0; y < NJ; ++y) {
      const int jl = (wj * NJ + y) * 16 + lr, j = j0 + jl;
      const int t = j < a.n_j ? a.targets[j] - a.v0 : -1;
      float m = -INFINITY;
      bool nan = false;
#pragma unroll
      for (int x = 0; x < NI; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + (wi * NI + x) * 16 + 4 * lg + e;
          if (i >= a.n_i) acc[x][y][e] = -INFINITY;
          const float z = acc[x][y][e];
          nan |= !(z == z);
          m = fmaxf(m, z);
          if (i == t && t < a.n_i) a.target_z[j] = z;
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      float sum = 0.f;
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int x = 0; x < NI; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __expf(acc[x][y][e] - base);
      if (nan) sum = __builtin_nanf("");
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (lg == 0) red[jl * WI + wi] = make_float2(m, sum);
    }
    __syncthreads();
    for (int jl = threadIdx.x; jl < TJ; jl += WI * WJ * 64) {
      if (j0 + jl >= a.n_j) break;
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < WI; ++w) m = fmaxf(m, red[jl * WI + w].x);
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int w = 0; w < WI; ++w) sum += red[jl * WI + w].y * __expf(red[jl * WI + w].x - base);
      a.sums[(int64_t)(j0 + jl) * a.ld_sums + it] = make_float2(m, sum);
    }
  } else if (EPI == HEAD_DZ) {
#pragma unroll
    for (int y = 0; y < NJ; ++y) {
      const int j = j0 + (wj * NJ + y) * 16 + lr, jc = min(j, a.n_j - 1);
      const int t = a.targets[jc];
      const float g = a.weights ? a.weights[jc] : 1.f, lse = a.lse[jc];
      const bool out = t < 0 || t >= a.V || g == 0.f;
      auto dz = [&](int x, float (&d)[4]) {
        const int i = i0 + (wi * NI + x) * 16 + 4 * lg, at = t - a.v0 - i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float q = acc[x][y][e] - lse;
          // (fp32's parts make NaN of a logit of -infinity; with a finite lse there is no other that is not finite)
          if (DT == 0 && !(q == q) && fabsf(lse) < INFINITY) q = -INFINITY;
          d[e] = DT ? __expf(q) : expf(q);
          if (e == at) d[e] = expm1f(q);   // (p - 1 keeps its bits where p is near 1)
          d[e] = out || i + e >= a.n_i ? 0.f : d[e] * g;
          if (DT && e == at && j < a.n_j) a.rest[j] = d[e] - Elem<1>::round(d[e]);
        }
      };
      if constexpr (DT == 0) {
#pragma unroll
        for (int x = 0; x < NI; ++x) {
          float d[4];
          dz(x, d);
          const int i = i0 + (wi * NI + x) * 16 + 4 * lg;
          if (j < a.n_j && i < a.ldz) *(float4*)((float*)a.dz + (int64_t)j * a.ldz + i) = make_float4(d[0], d[1], d[2], d[3]);
        }
      } else {
#pragma unroll
        for (int x = 0; x < NI; x += 2) {
          float d[2][4];
          dz(x, d[0]);
          dz(x + 1, d[1]);
          int i;
          const uint4 u = eight(d[0], d[1], i);
          i += i0 + (wi * NI + x) * 16;
          if (j < a.n_j && i < a.ldz) *(uint4*)(a.dz + ((int64_t)j * a.ldz + i) * 2) = u;
        }
      }
    }
  } else {
    // sums of a part of the contraction (HEAD_PART, added to what is there in
    // later pieces), or the result
#pragma unroll
    for (int y = 0; y < NJ; ++y) {
      const int j = j0 + (wj * NJ + y) * 16 + lr;
      if (EPI == HEAD_OUT && DT) {
#pragma unroll
        for (int x = 0; x < NI; x += 2) {
          int i;
          const f32x4 v = acc[x][y], w = acc[x + 1][y];
          const float d0[4] = {v[0], v[1], v[2], v[3]}, d1[4] = {w[0], w[1], w[2], w[3]};
          const uint4 u = eight(d0, d1, i);
          i += i0 + (wi * NI + x) * 16;
          if (j < a.n_j && i < a.n_i) *(uint4*)((uint8_t*)a.out + ((int64_t)j * a.ldo + i) * 2) = u;
        }
        continue;
      }
      if (j >= a.n_j) continue;
#pragma unroll
      for (int x = 0; x < NI; ++x) {
        const int i = i0 + (wi * NI + x) * 16 + 4 * lg;
        if (i >= a.n_i) continue;
        float4 v = make_float4(acc[x][y][0], acc[x][y][1], acc[x][y][2], acc[x][y][3]);
        if (EPI == HEAD_PART) {
          float4* to = (float4*)(a.part + ((int64_t)part * a.n_j + j) * a.n_i + i);
          if (a.add) {
            const float4 o = *to;
            v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
          }
          *to = v;
        } else {
          *(float4*)((uint8_t*)a.out + ((int64_t)j * a.ldo + i) * 4) = v;
        }
      }
    }
  }
}

// dW's part of what rounding took from the targets' dz (rest): rest[m] h_m for row
// t_m of dW, whose largest dz this is.  The block lists the rows whose target lies
// in its tile, in ascending order, and multiplies 64 of them at a time: their rows
// of hidden are gathered into A's place in the ring, and an operand of rest in a
// row's target's place and zeros elsewhere is made in registers (rest in bf16: 2^-16
// of dz are left).  2048 rows of 32000 x 4096: the error of dW against 64 bits 2.4e-3
// -> 1.7e-3, bf16's own, for about 30 us of 476; chains of loads at a block's end, of
// which targets loaded before the product began save nothing.
template <int TI, int TJ, int WI, int WJ, int NI, int NJ>
__device__ __forceinline__ void head_rest(const HeadArgs& a, f32x4 (&acc)[NI][NJ], uint8_t* smem, int i0, int j0, int wi, int wj) {
  constexpr int NW = WI * WJ, THREADS = NW * 64;
  typedef Operand<true, TI, NW> OA;
  static_assert(4 * THREADS * 4 <= TJ * HD_K * 2, "the list has B's place in the ring");
  __shared__ int found[NW];
  __shared__ int2 taken[HD_K];   // (place in the tile, rest) of a batch's rows
  int* const list = (int*)(smem + OA::BYTES);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t first = a.v0 + j0, cols = min(TJ, a.n_j - j0);
  for (int r0 = 0; r0 < a.C; r0 += 4 * THREADS) {
    const int r = r0 + 4 * tid;
    bool in[4];
    int at = 0, total = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      in[u] = r + u < a.C && (uint32_t)a.targets[r + u] - first < cols;   // (rows left out for their weight are zeros in A)
      const uint64_t b = __ballot(in[u]);
      at += __popcll(b & ((1ull << lane) - 1));
      total += __popcll(b);
    }
    __syncthreads();   // (the ring, and the last rows' list, have been read)
    if (lane == 0) found[wave] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int n = found[w];
      at += w < wave ? n : 0;
      total += n;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (in[u]) list[at++] = r + u;
    for (int b0 = 0; b0 < total; b0 += HD_K) {
      __syncthreads();   // (the list is there; the last batch has been read)
      const int n = min(HD_K, total - b0);
      if (tid < HD_K) {
        const int m = list[b0 + min(tid, n - 1)];
        taken[tid] = tid < n ? make_int2((int)((uint32_t)a.targets[m] - first), f32_to_bf16(a.rest[m])) : make_int2(-1, 0);
      }
#pragma unroll
      for (int i = 0; i < OA::PER; ++i) {
        const int k = OA::entry(i, wave), c = (lane % OA::CH) ^ (OA::perm(k) << 1);
        const int64_t row = list[b0 + min(k, n - 1)];
        uint4 x = ld16(a.A + (row * a.lda + i0 + min(8 * c, ((a.n_i + 7) & ~7) - 8 - i0)) * 2);
        if (k >= n) x = make_uint4(0, 0, 0, 0);
        *(uint4*)(smem + (wave * OA::PER + i) * 1024 + lane * 16) = x;
      }
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (32 * h >= n) break;
        int2 q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = taken[32 * h + 8 * lg + e];
        bf16x8 fb[NJ];
#pragma unroll
        for (int y = 0; y < NJ; ++y) {
          u32x4 w;
          const int j = (wj * NJ + y) * 16 + lr;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = (q[2 * e].x == j ? (uint32_t)q[2 * e].y : 0u) | (q[2 * e + 1].x == j ? (uint32_t)q[2 * e + 1].y << 16 : 0u);
          fb[y] = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int x = 0; x < NI; ++x) {
          const bf16x8 fa = OA::read((const lds8*)smem, (wi * NI + x) * 16, h);
#pragma unroll
          for (int y = 0; y < NJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, fb[y], acc[x][y], 0, 0, 0);
        }
      }
    }
  }
}

// out[j][i] = sum_c A[i][c] B[j][c] of bf16 operands, TI x TJ of them a block, WI x
// WJ waves.  A ring of S steps of the contraction in LDS: one is multiplied while
// the next ones are on their way; one barrier a step.  2048 rows of 32000 x 4096:
// 406 to 476 us a product, 1130 to 1320 TFLOP/s (a library product of 8192^3 1450 here).
template <bool CA, bool CB, int TI, int TJ, int WI, int WJ, int S, int EPI>
__global__ __launch_bounds__(WI * WJ * 64) void k_head(HeadArgs a) {
  constexpr int NW = WI * WJ, NI = TI / WI / 16, NJ = TJ / WJ / 16;
  typedef Operand<CA, TI, NW> OA;
  typedef Operand<CB, TJ, NW> OB;
  constexpr int PER = OA::PER + OB::PER, STAGE = OA::BYTES + OB::BYTES;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave % WI, wj = wave / WI;
  HeadPlace place;
  if (!head_place(a, place)) return;
  const int i0 = place.it * TI, j0 = place.jt * TJ;
  const int c_begin = place.part * a.chunk, c_end = min(c_begin + a.chunk, a.C);

  f32x4 acc[NI][NJ];
#pragma unroll
  for (int x = 0; x < NI; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int total = (c_end - c_begin + HD_K - 1) / HD_K;
  if (total > 0) {
    lds8* ring = (lds8*)smem;
    Copies<OA, OB> copies;
    copies.left = c_end - c_begin;
    copies.wave = wave;
    copies.oa.begin(a.A, a.lda, i0, a.n_i, c_begin, wave);
    copies.ob.begin(a.B, a.ldb, j0, a.n_j, c_begin, wave);
    for (int i = 0; i < S && i < total; ++i) copies.next(ring + i * STAGE);
    if (total >= S) copies_barrier<(S - 1) * PER>();
    else copies_barrier<0>();
    constexpr int EARLY = NI > 2 ? 2 : 1;   // rows of tiles of a step's second half before the barrier
    bf16x8 fa[NI], fb[2][NJ];
    head_step<OA, OB, !CA, true, false, EARLY>(ring, ring, copies, wi, wj, fa, fb, acc);
    int slot = 0;
    auto after = [&](int x) { return x + 1 == S ? 0 : x + 1; };
    for (int s = S; s < total; ++s) {   // (step s is copied to where step s - S was)
      lds8* left = ring + slot * STAGE;
      slot = after(slot);
      copies_barrier<(S - 2) * PER>();
      head_step<OA, OB, !CA, false, true, EARLY>(ring + slot * STAGE, left, copies, wi, wj, fa, fb, acc);
    }
#pragma unroll 1
    for (int s = 1; s < min(S, total); ++s) {
      slot = after(slot);
      copies_barrier<0>();
      head_step<OA, OB, !CA, false, false, EARLY>(ring + slot * STAGE, ring, copies, wi, wj, fa, fb, acc);
    }
#pragma unroll
    for (int x = EARLY; x < NI; ++x) multiply_row(x, fa, fb[1], acc);
  }

  if constexpr (EPI == HEAD_OUT) head_rest<TI, TJ, WI, WJ>(a, acc, smem, i0, j0, wi, wj);
  head_finish<1, EPI, TI, TJ, WI, WJ>(a, acc, smem, place, wi, wj);
}

// ---- fp32 ---------------------------------------------------------------------------

// The same for fp32 operands: each is three bf16 numbers that sum to it (cut off
// rather than rounded, so that the first cannot overflow), and of the nine
// products of parts the six down to 2^-14 of the whole are made, the smallest
// first (the others are below 2^-21, 2^-21 and 2^-28 of it): a sixth of bf16's
// rate, where the fp32 matrix instructions have a sixteenth.  Operands are split on their way to LDS, 5.5 operations an entry,
// so that they are read once a tile (in planes of parts, split before: 47 rows of
// 32000 x 5120 4.8 ms against 0.9, 1024 rows 7.0 against 6.7, 2048 rows alike).
// A step is KS entries of the contraction, loaded into registers AHEAD steps
// before; two barriers a step, and other blocks on the CU meanwhile.  What is
// not finite becomes NaN in the second part, and so do the logits it meets, which
// are formed again (head_join_again).
__device__ float4 head_zeros[2];   // what is read in place of entries past the contraction's end
constexpr int PRODUCTS = 6;
__device__ __forceinline__ void split8(const float (&v)[8], u32x4 (&w)[3]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t b[3][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      b[0][h] = __float_as_uint(v[e + h]);
      const float rest = v[e + h] - __uint_as_float(b[0][h] & 0xFFFF0000u);
      b[1][h] = __float_as_uint(rest);
      b[2][h] = __float_as_uint(rest - __uint_as_float(b[1][h] & 0xFFFF0000u));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][e / 2] = __builtin_amdgcn_perm(b[p][1], b[p][0], 0x07060302);
  }
}
// acc += the products of the parts of NI and NJ operands.
template <int NI, int NJ>
__device__ __forceinline__ void split_products(const bf16x8 (&fa)[3][NI], const bf16x8 (&fb)[3][NJ], f32x4 (&acc)[NI][NJ]) {
#pragma unroll
  for (int p = 0; p < PRODUCTS; ++p) {
    constexpr int PA[PRODUCTS] = {2, 0, 1, 1, 0, 0}, PB[PRODUCTS] = {0, 2, 1, 0, 1, 0};
#pragma unroll
    for (int x = 0; x < NI; ++x)
#pragma unroll
      for (int y = 0; y < NJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[PA[p]][x], fb[PB[p]][y], acc[x][y], 0, 0, 0);
  }
}
template <bool COLUMNS, int T, int KS, int AHEAD> struct Split {
  static constexpr int PLANE = T * KS * 2, CHUNKS = T * KS / 8, PER = (CHUNKS + 255) / 256;   // chunks of eight entries; of a thread
  const float* src[PER];
  int64_t step;
  float4 x[AHEAD][PER][2];
  static __device__ __forceinline__ int chunk(int i) { return (threadIdx.x + 256 * i) % CHUNKS; }
  static __device__ __forceinline__ int entry(int i) {   // of the contraction, in a step: a chunk's first
    const int q = chunk(i);
    return COLUMNS ? q / (T / 8) : q % (KS / 8) * 8;
  }
  __device__ __forceinline__ void begin(const float* p, int64_t ld, int r0, int n, int c0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int q = chunk(i);
      src[i] = COLUMNS ? p + (int64_t)(c0 + entry(i)) * ld + min(r0 + q % (T / 8) * 8, ((n + 7) & ~7) - 8)
                       : p + (int64_t)min(r0 + q / (KS / 8), n - 1) * ld + c0 + entry(i);
    }
    step = COLUMNS ? KS * ld : KS;
  }
  __device__ __forceinline__ void load(int u, int left) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float4* p = entry(i) < left ? (const float4*)src[i] : head_zeros;
      x[u][i][0] = p[0];
      x[u][i][1] = p[1];
      src[i] += step;
    }
  }
  // The layouts of Operand; rows of 32 entries: 64 bytes, chunk c of row r at c ^ (r >> 1 & 3).
  __device__ __forceinline__ void store(int u, lds8* planes) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int q = chunk(i);
      if (CHUNKS < 256 && threadIdx.x >= CHUNKS) return;
      int at;
      if (COLUMNS) {
        const int k = q / (T / 8), c = q % (T / 8);
        at = k * (2 * T) + ((c ^ (Operand<true, T, 4>::perm(k) << 1)) << 4);
      } else {
        const int r = q / (KS / 8), c = q % (KS / 8);
        at = r * (2 * KS) + ((c ^ (KS == 64 ? r & 7 : r >> 1 & 3)) << 4);
      }
      const float v[8] = {x[u][i][0].x, x[u][i][0].y, x[u][i][0].z, x[u][i][0].w, x[u][i][1].x, x[u][i][1].y, x[u][i][1].z, x[u][i][1].w};
      u32x4 w[3];
      split8(v, w);
#pragma unroll
      for (int p = 0; p < 3; ++p)
        *(__attribute__((address_space(3))) u32x4*)(planes + p * PLANE + at) = w[p];
    }
  }
  static __device__ __forceinline__ bf16x8 read(const lds8* plane, int r0, int h) {
    if (COLUMNS || KS == 64) return Operand<COLUMNS, T, 4>::read(plane, r0, h);
    const int lane = threadIdx.x & 63, r = r0 + (lane & 15);
    return lds_row8(plane + r * 64 + (((lane >> 4) ^ (r >> 1 & 3)) << 4));
  }
};

template <bool CA, bool CB, int TI, int TJ, int WI, int WJ, int KS, int AHEAD, int EPI>
__global__ __launch_bounds__(256) void k_head_fp32(HeadArgs a) {
  constexpr int NI = TI / WI / 16, NJ = TJ / WJ / 16;
  typedef Split<CA, TI, KS, AHEAD> SA;
  typedef Split<CB, TJ, KS, AHEAD> SB;
  extern __shared__ __align__(16) uint8_t smem[];   // 3 (SA::PLANE + SB::PLANE)
  static_assert(TJ * WI * 8 <= 3 * (SA::PLANE + SB::PLANE), "the sums of the waves");
  lds8 *la = (lds8*)smem, *lb = la + 3 * SA::PLANE;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave % WI, wj = wave / WI;
  HeadPlace place;
  if (!head_place(a, place)) return;
  const int i0 = place.it * TI, j0 = place.jt * TJ;
  const int c_begin = place.part * a.chunk, c_end = min(c_begin + a.chunk, a.C);
  f32x4 acc[NI][NJ];
#pragma unroll
  for (int x = 0; x < NI; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  SA sa;
  SB sb;
  if (c_begin < c_end) {
    sa.begin((const float*)a.A, a.lda, i0, a.n_i, c_begin);
    sb.begin((const float*)a.B, a.ldb, j0, a.n_j, c_begin);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      sa.load(u, c_end - c_begin - u * KS);
      sb.load(u, c_end - c_begin - u * KS);
    }
  }
  for (int c0 = c_begin; c0 < c_end; c0 += AHEAD * KS) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int left = c_end - c0 - u * KS;   // (behind the last step: zeros)
      lds_barrier();
      sa.store(u, la);
      sb.store(u, lb);
      sa.load(u, left - AHEAD * KS);
      sb.load(u, left - AHEAD * KS);
      lds_barrier();
      if (left <= 0) continue;
#pragma unroll
      for (int h = 0; h < KS / 32; ++h) {
        bf16x8 fa[3][NI], fb[3][NJ];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
#pragma unroll
          for (int x = 0; x < NI; ++x) fa[p][x] = SA::read(la + p * SA::PLANE, (wi * NI + x) * 16, h);
#pragma unroll
          for (int y = 0; y < NJ; ++y) fb[p][y] = SB::read(lb + p * SB::PLANE, (wj * NJ + y) * 16, h);
        }
        split_products<NI, NJ>(fa, fb, acc);
      }
    }
  }
  head_finish<0, EPI, TI, TJ, WI, WJ>(a, acc, smem, place, wi, wj);
}

// Few fp32 rows over a large head, which is read once and bounds it: no two waves
// share entries of it, so they go straight into registers, two steps ahead; the
// rows' parts are in LDS, one step's written while the other's are read.
// Columns: a lane has four neighbouring ones of eight entries of the contraction,
// one for each of the four tiles, whose row r is column 4 r + x.  21 rows of 118860
// x 5120 524 us a pass (4.6 TB/s; 656 in k_head_fp32), dh's 403 (559).
template <bool CA, int NI, int TJ, int EPI>
__global__ __launch_bounds__(256, 2) void k_head_thin(HeadArgs a) {
  constexpr int KS = CA ? 32 : 64, NJ = TJ / 16, TI = 64 * NI, H = KS / 32, N4 = H * 8;   // 16-byte loads of a step
  typedef Split<false, TJ, KS, 2> SB;
  extern __shared__ __align__(16) uint8_t smem[];   // 6 SB::PLANE
  lds8* lb = (lds8*)smem;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  HeadPlace place;
  if (!head_place(a, place)) return;
  const int i0 = place.it * TI, j0 = place.jt * TJ;
  const int c_begin = place.part * a.chunk, c_end = min(c_begin + a.chunk, a.C);
  f32x4 acc[NI][NJ];
#pragma unroll
  for (int x = 0; x < NI; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (c_begin < c_end) {
    SB sb;
    sb.begin((const float*)a.B, a.ldb, j0, a.n_j, c_begin);
    const float *src[CA ? 1 : NI], *A = (const float*)a.A;
    if (CA) {
      src[0] = A + (int64_t)(c_begin + 8 * lg) * a.lda + min(i0 + wave * 64 + 4 * lr, a.n_i - 4);
    } else {
#pragma unroll
      for (int x = 0; x < NI; ++x) src[x] = A + (int64_t)min(i0 + (wave * NI + x) * 16 + lr, a.n_i - 1) * a.lda + c_begin + 8 * lg;
    }
    float4 v[2][N4];
    auto load = [&](int u, int left) {
#pragma unroll
      for (int n = 0; n < N4; ++n) {
        const int h = CA ? 0 : n / (2 * NI), x = CA ? 0 : n / 2 % NI;   // columns: entry n of the lane's eight
        const float* p = CA ? src[0] + (int64_t)n * a.lda : src[x] + 32 * h + 4 * (n & 1);
        v[u][n] = *(const float4*)((CA ? 8 * lg + n : 32 * h + 8 * lg) < left ? p : (const float*)head_zeros);
      }
      if (CA) src[0] += KS * a.lda;
      else
#pragma unroll
        for (int x = 0; x < NI; ++x) src[x] += KS;
    };
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sb.load(u, c_end - c_begin - u * KS);
      load(u, c_end - c_begin - u * KS);
    }
    for (int c0 = c_begin; c0 < c_end; c0 += 2 * KS) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int left = c_end - c0 - u * KS;   // (behind the last step: zeros)
        lds8* planes = lb + u * 3 * SB::PLANE;
        sb.store(u, planes);
        sb.load(u, left - 2 * KS);
        lds_barrier();
        u32x4 w[H][NI][3];
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int x = 0; x < NI; ++x) {
            float e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float4 q = CA ? v[u][k] : v[u][(h * NI + x) * 2 + k / 4];
              const int at = CA ? x : k % 4;
              e[k] = at == 0 ? q.x : at == 1 ? q.y : at == 2 ? q.z : q.w;
            }
            split8(e, w[h][x]);
          }
        load(u, left - 2 * KS);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          bf16x8 fa[3][NI], fb[3][NJ];
#pragma unroll
          for (int p = 0; p < 3; ++p) {
#pragma unroll
            for (int x = 0; x < NI; ++x) fa[p][x] = __builtin_bit_cast(bf16x8, w[h][x][p]);
#pragma unroll
            for (int y = 0; y < NJ; ++y) fb[p][y] = SB::read(planes + p * SB::PLANE, y * 16, h);
          }
          split_products<NI, NJ>(fa, fb, acc);
        }
      }
    }
  }
  if (EPI != HEAD_PART) {
    head_finish<0, EPI, TI, TJ, 4, 1>(a, acc, smem, place, wave, 0);
    return;
  }
#pragma unroll
  for (int y = 0; y < NJ; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + 16 * y + lr, i = i0 + wave * 64 + 4 * (4 * lg + e);
      if (j >= a.n_j || i >= a.n_i) continue;
      float4* to = (float4*)(a.part + ((int64_t)place.part * a.n_j + j) * a.n_i + i);
      float4 s = make_float4(acc[0][y][e], acc[CA ? 1 : 0][y][e], acc[CA ? 2 : 0][y][e], acc[CA ? 3 : 0][y][e]);
      if (a.add) {
        const float4 o = *to;
        s = make_float4(o.x + s.x, o.y + s.y, o.z + s.z, o.w + s.w);
      }
      *to = s;
    }
}

// dW of few rows, bound by its stores: a wave keeps its 64 columns of all rows of
// hidden (zeros for those that are left out) as operands (the contraction is 32 H
// rows) and walks over the vocabulary, 64 entries at a time, the next ones' dz on its way.  Neighbouring
// columns are of four tiles, so that a lane stores four of them and 16 lanes a row's
// 64; blocks beside each other take the entries in turn, so that the card writes
// one stretch of dW at a time.  21 fp32 rows over 118860 x 5120 434 us (5.6 TB/s;
// in k_head_fp32 600), 2 bf16 rows over 128256 x 5120 229 (5.7; in k_head 289), 35
// of them 299 (321).
template <int DT, int H>
__global__ __launch_bounds__(256, 2) void k_head_outer(HeadArgs a) {
  constexpr int PARTS = DT ? 1 : 3, ES = DT ? 2 : 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int i0 = (blockIdx.x * 4 + wave) * 64;
  if (i0 >= a.n_i) return;
  // Four neighbours' eight entries of the contraction, as they lie in memory and as four tiles' operands.
  typedef typename std::conditional<DT == 1, uint2, float4>::type Four;
  auto load = [&](Four (&v)[H * 8], const uint8_t* p, int64_t ld, int at) {
#pragma unroll
    for (int n = 0; n < H * 8; ++n) {
      const int c = (n / 8) * 32 + 8 * lg + n % 8;
      v[n] = *(const Four*)(c < a.C ? p + (c * ld + at) * ES : (const uint8_t*)head_zeros);
    }
  };
  auto operands = [&](const Four (&v)[H * 8], bf16x8 (&f)[H][4][PARTS]) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (DT == 1) {
          u32x4 w;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint2 p = v[h * 8 + 2 * k], q = v[h * 8 + 2 * k + 1];
            w[k] = __builtin_amdgcn_perm(x < 2 ? q.x : q.y, x < 2 ? p.x : p.y, x & 1 ? 0x07060302 : 0x05040100);
          }
          f[h][x][0] = __builtin_bit_cast(bf16x8, w);
        } else {
          float e[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float4 q = v[h * 8 + k];
            e[k] = x == 0 ? q.x : x == 1 ? q.y : x == 2 ? q.z : q.w;
          }
          u32x4 w[3];
          split8(e, w);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) f[h][x][p] = __builtin_bit_cast(bf16x8, w[p]);
        }
      }
  };
  Four v[H * 8];
  bf16x8 fh[H][4][PARTS];
  const int k = i0 + 4 * lr;
  load(v, a.A, a.lda, min(k, a.n_i - 4));
  const uint64_t kept = __ballot(lane < a.C && !left_out(a.targets[lane], a.weights, lane, a.V));
#pragma unroll
  for (int n = 0; n < H * 8; ++n)
    if (!(kept >> ((n / 8) * 32 + 8 * lg + n % 8) & 1)) v[n] = Four{};
  operands(v, fh);
  // Lane c: row c's target in the piece, and what rounding took from its dz (-1: nothing).
  int place = -1, rest = 0;
  if (DT == 1 && (kept >> lane & 1)) {
    const int t = a.targets[lane] - a.v0;
    if (t >= 0 && t < a.n_j && a.rest[lane] != 0.f) {
      place = t;
      rest = f32_to_bf16(a.rest[lane]);
    }
  }
  const int most = ((a.n_j + 3) & ~3) - 4;
  auto load_dz = [&](int j0) { load(v, a.B, a.ldb, min(j0 + 4 * lr, most)); };
  load_dz(blockIdx.y * 64);
  for (int j0 = blockIdx.y * 64; j0 < a.n_j; j0 += gridDim.y * 64) {
    bf16x8 fz[H][4][PARTS];
    operands(v, fz);
    load_dz(j0 + gridDim.y * 64);
    f32x4 acc[4][4];   // [y][x]: entry 4 (4 lg + e) + y of the vocabulary, column 4 lr + x
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[y][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int p = 0; p < (DT ? 1 : PRODUCTS); ++p) {
        constexpr int PA[PRODUCTS] = {2, 0, 1, 1, 0, 0}, PB[PRODUCTS] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            acc[y][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fz[h][y][DT ? 0 : PB[p]], fh[h][x][DT ? 0 : PA[p]], acc[y][x], 0, 0, 0);
      }
    if (DT == 1 && __ballot(place >= j0 && place < j0 + 64)) {   // (as in head_rest)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        int t[8], r[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          t[n] = __shfl(place, 32 * h + 8 * lg + n) - j0 - 4 * lr;
          r[n] = __shfl(rest, 32 * h + 8 * lg + n);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          u32x4 w;
#pragma unroll
          for (int n = 0; n < 4; ++n) w[n] = (t[2 * n] == y ? (uint32_t)r[2 * n] : 0u) | (t[2 * n + 1] == y ? (uint32_t)r[2 * n + 1] << 16 : 0u);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            acc[y][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), fh[h][x][0], acc[y][x], 0, 0, 0);
        }
      }
    }
    if (k >= a.n_i) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int j = j0 + 4 * (4 * lg + e) + y;
        if (j < a.n_j) store4<DT>((uint8_t*)a.out + (int64_t)j * a.ldo * ES, k, make_float4(acc[y][0][e], acc[y][1][e], acc[y][2][e], acc[y][3][e]));
      }
  }
}

// ---- rows before and after ----------------------------------------------------------

// Rows of hidden for dW, zeros in place of those that are left out: what they hold
// (a padded place may hold anything) must not reach dW as 0 x NaN.
__global__ __launch_bounds__(256) void k_head_copy(HeadCopyArgs a) {   // rows of `chunks` 16-byte pieces
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= a.n * a.chunks) return;
  const int64_t r = at / a.chunks, c = at % a.chunks;
  const int t = a.targets[r];
  const bool out = left_out(t, a.weights, r, a.V);
  *(uint4*)(a.dst + at * 16) = out ? make_uint4(0, 0, 0, 0) : ld16((const uint8_t*)a.src + r * a.pitch + c * 16);
}

// A row's maximum m and sum s of fp32 logits of which some tiles' are NaN: these are
// formed again, in 64 bits and without parts, so that an infinite entry of the head
// does what it does to a product (a vocabulary masked by logits of -infinity keeps
// its others), and so is the target's logit zt among them.  A row of hidden with an
// entry that is not finite has no sum, whatever the head is.  A wave's loads are of 64
// rows of the head: 1024 rows of 32000 x 5120, whose last 40 entries are masked,
// 1.65 -> 2.0 ms, the last 2000 8.0 (a row of the head at a time over the lanes 15).
__device__ __forceinline__ void head_join_again(const HeadJoinArgs& a, int j, const float2* p, float& m, float& s, float& zt) {
  const int lane = threadIdx.x & 63;
  const float* h = a.hidden + j * a.ldh;
  bool finite = true;
  for (int k = lane; k < a.K; k += 64) finite = finite && fabsf(h[k]) < INFINITY;
  if (__ballot(!finite)) return;
  m = -INFINITY;
  s = 0.f;
  auto add = [&](float z, float n) {   // n e^z
    const float most = fmaxf(m, z), base = most == -INFINITY ? 0.f : most;
    s = s * __expf(m - base) + n * __expf(z - base);
    m = most;
  };
  for (int t0 = 0; t0 < a.tiles; t0 += 64) {
    const float2 q = t0 + lane < a.tiles ? p[t0 + lane] : make_float2(-INFINITY, 0.f);
    const bool nan = !(q.y == q.y);
    if (!nan) add(q.x, q.y);
    for (uint64_t left = __ballot(nan); left; left &= left - 1) {
      const int first = (t0 + __ffsll((unsigned long long)left) - 1) * a.tile, end = min(first + a.tile, a.V);
      for (int v0 = first; v0 < end; v0 += 64) {
        const int v = v0 + lane;
        double z = 0.0;
        if (v < end) {
          const float* w = a.head + v * a.ldw;
#pragma unroll 8
          for (int k = 0; k < a.K; k += 4) {
            const float4 x = *(const float4*)(h + k), y = *(const float4*)(w + k);
            z = fma((double)x.x, (double)y.x, fma((double)x.y, (double)y.y, fma((double)x.z, (double)y.z, fma((double)x.w, (double)y.w, z))));
          }
          add((float)z, z == z ? 1.f : (float)z);
        }
        const uint64_t target = __ballot(v < end && v == a.targets[j]);
        if (target) zt = __shfl((float)z, __ffsll((unsigned long long)target) - 1);
      }
    }
  }
  const float most = wave_max(m);
  s = wave_sum(s * __expf(m - (most == -INFINITY ? 0.f : most)));
  m = most;
}

// A wave joins a row's tiles.
__global__ __launch_bounds__(256) void k_head_join(HeadJoinArgs a) {
  const int lane = threadIdx.x & 63, j = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (j >= a.n) return;
  const float2* p = a.sums + (int64_t)j * a.tiles;
  float m = -INFINITY;
  for (int i = lane; i < a.tiles; i += 64) m = fmaxf(m, p[i].x);
  m = wave_max(m);
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f;
  for (int i = lane; i < a.tiles; i += 64) s += p[i].y * __expf(p[i].x - base);
  s = wave_sum(s);
  const int t = a.targets[j];
  const bool in = t >= 0 && t < a.V;
  float zt = in ? a.target_z[j] : 0.f;
  if (a.hidden && !(s == s)) head_join_again(a, j, p, m, s, zt);
  if (lane) return;
  const double lse = m == -INFINITY ? (double)__builtin_nanf("") : (double)m + log((double)s);
  if (a.loss) a.loss[j] = in ? (float)(lse - (double)zt) : 0.f;
  a.lse[j] = (float)lse;
}

// The parts of dh, summed in a fixed order (`lanes` lanes take parts in turn and
// meet by shuffles) and rounded.  A row's largest dz is usually its target's,
// and what bf16 rounded away of it is an error along that whole row of W: here
// it is put back (the error of dh falls from 2.4e-3 to 1.7e-3, bf16's own).
template <int DT>
__global__ __launch_bounds__(256) void k_head_out(HeadOutArgs a, int lanes) {
  const int64_t per = a.K / 4, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;
  const int lane = threadIdx.x % lanes;
  const bool in = at < a.n * per;
  const int64_t r = in ? at / per : 0;
  const int k = in ? (int)(at % per) * 4 : 0;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = lane; s < a.split; s += lanes) {
    const float4 o = *(const float4*)(a.part + ((int64_t)s * a.n + r) * a.K + k);
    v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
  }
  for (int o = 1; o < lanes; o <<= 1) v = make_float4(v.x + __shfl_xor(v.x, o), v.y + __shfl_xor(v.y, o), v.z + __shfl_xor(v.z, o), v.w + __shfl_xor(v.w, o));
  if (!in || lane) return;
  const int t = a.targets[r];
  if (left_out(t, a.weights, r, a.V)) {
    v = make_float4(0.f, 0.f, 0.f, 0.f);   // (the sums are NaN where the head is not finite)
  } else if (DT == 1) {
    const float rest = a.rest[r];
    const uint2 w = *(const uint2*)((const uint16_t*)a.head + t * a.ldw + k);
    if (rest != 0.f)
      v = make_float4(fmaf(rest, bf16lo(w.x), v.x), fmaf(rest, bf16hi(w.x), v.y), fmaf(rest, bf16lo(w.y), v.z), fmaf(rest, bf16hi(w.y), v.w));
  }
  store4<DT>((uint8_t*)a.out + r * a.ldo * Elem<DT>::ES_, k, v);
}

// ---- launchers ----------------------------------------------------------------------

static hipError_t launch_blocks(const void* f, HeadArgs& a, int ti, int tj, int threads, int lds, hipStream_t s) {
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  a.i_tiles = (a.n_i + ti - 1) / ti;
  a.j_tiles = (a.n_j + tj - 1) / tj;
  a.band = a.C <= 512 && a.split == 1 ? a.i_tiles : 4;
  const dim3 grid((unsigned)(((int64_t)a.i_tiles * a.j_tiles * a.split + 7) / 8 * 8));
  void* args[] = {(void*)&a};
  return hipLaunchKernel(f, grid, dim3(threads), args, lds, s);
}
template <bool CA, bool CB, int TI, int TJ, int WI, int WJ, int S, int EPI>
static hipError_t launch_bf16(HeadArgs a, hipStream_t s) {
  // (no more of the ring than there are steps: short contractions leave room for a second block)
  const int steps = (std::min(a.chunk, a.C) + HD_K - 1) / HD_K;
  return launch_blocks((const void*)k_head<CA, CB, TI, TJ, WI, WJ, S, EPI>, a, TI, TJ, WI * WJ * 64, std::max(1, std::min(S, steps)) * (TI + TJ) * HD_K * 2, s);
}
template <bool CA, bool CB, int TI, int TJ, int WI, int WJ, int KS, int AHEAD, int EPI>
static hipError_t launch_fp32(HeadArgs a, hipStream_t s) {
  return launch_blocks((const void*)k_head_fp32<CA, CB, TI, TJ, WI, WJ, KS, AHEAD, EPI>, a, TI, TJ, 256, 3 * (TI + TJ) * KS * 2, s);
}
template <bool CA, int NI, int TJ, int EPI>
static hipError_t launch_thin(HeadArgs a, hipStream_t s) {
  return launch_blocks((const void*)k_head_thin<CA, NI, TJ, EPI>, a, 64 * NI, TJ, 256, 6 * TJ * (CA ? 32 : 64) * 2, s);
}
template <bool CA, bool CB, int EPI>
static hipError_t launch_tile(int dtype, const HeadArgs& a, HeadTile tile, hipStream_t s) {
  if (dtype) {
    if (tile.i == 128) return launch_bf16<CA, CB, 128, 64, 4, 1, 6, EPI>(a, s);
    if (tile.j == 64) return launch_bf16<CA, CB, 256, 64, 8, 1, 3, EPI>(a, s);
    if (tile.j == 128) return launch_bf16<CA, CB, 256, 128, 4, 2, 3, EPI>(a, s);
    return launch_bf16<CA, CB, 256, 256, 2, 4, 2, EPI>(a, s);
  }
  if constexpr (EPI != HEAD_OUT) {
    if (tile.thin) {
      constexpr int NI = CA ? 4 : 2;
      if constexpr (!CA) {
        if (tile.i == 64 && tile.j == 16) return launch_thin<CA, 1, 16, EPI>(a, s);
        if (tile.i == 64 && tile.j == 32) return launch_thin<CA, 1, 32, EPI>(a, s);
        if (tile.i == 64) return launch_thin<CA, 1, 64, EPI>(a, s);
      }
      if (tile.j == 16) return launch_thin<CA, NI, 16, EPI>(a, s);
      if (tile.j == 32) return launch_thin<CA, NI, 32, EPI>(a, s);
      return launch_thin<CA, NI, 64, EPI>(a, s);
    }
  }
  if constexpr (CA)   // (few rows with the head's: thin)
    if (tile.i == 64 && tile.j == 64) return launch_fp32<CA, CB, 64, 64, 2, 2, 64, 1, EPI>(a, s);
  if (tile.i == 64) return launch_fp32<CA, CB, 64, 128, 2, 2, 32, 2, EPI>(a, s);
  return launch_fp32<CA, CB, 128, 128, 2, 2, 32, 2, EPI>(a, s);
}
hipError_t launch_head(int dtype, int epi, const HeadArgs& a, HeadTile tile, hipStream_t s) {
  if (epi == HEAD_SUMS) return launch_tile<false, false, HEAD_SUMS>(dtype, a, tile, s);
  if (epi == HEAD_DZ) return launch_tile<false, false, HEAD_DZ>(dtype, a, tile, s);
  if (epi == HEAD_PART) return launch_tile<true, false, HEAD_PART>(dtype, a, tile, s);
  return launch_tile<true, true, HEAD_OUT>(dtype, a, tile, s);
}

// Blocks for two rounds of two a CU (one round: 458 us for 442, the same case).
hipError_t launch_head_outer(int dtype, const HeadArgs& a, hipStream_t s) {
  const int x = (a.n_i + 255) / 256, y = std::max(1, std::min((a.n_j + 63) / 64, 1024 / x));
  const dim3 grid(x, y);
  if (dtype && a.C > 32) k_head_outer<1, 2><<<grid, 256, 0, s>>>(a);
  else if (dtype) k_head_outer<1, 1><<<grid, 256, 0, s>>>(a);
  else k_head_outer<0, 1><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_head_copy(const HeadCopyArgs& a, hipStream_t s) {
  k_head_copy<<<(unsigned)((a.n * a.chunks + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_head_join(const HeadJoinArgs& a, hipStream_t s) {
  k_head_join<<<(a.n + 3) / 4, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_head_out(int dtype, const HeadOutArgs& a, hipStream_t s) {
  const int lanes = a.split <= 4 ? 1 : a.split <= 32 ? 8 : 16;
  const unsigned blocks = (unsigned)((a.n * (a.K / 4) * lanes + 255) / 256);
  if (dtype) k_head_out<1><<<blocks, 256, 0, s>>>(a, lanes);
  else k_head_out<0><<<blocks, 256, 0, s>>>(a, lanes);
  return hipGetLastError();
}

}  // namespace lede
