// Products of a batch's rows with matrices of 4-bit weights (quant.hip), and
// their arguments (entry points in products.cpp).  Not part of the public C
// ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lede {

// A matrix W [N][K] of e2m1 codes (OCP; the card's own 4-bit type: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6 and their negatives) with a bf16 scale for each `group`
// columns of a row.  Packed: tiles of 16 rows x 128 columns.  A tile's codes
// are 64 lanes x 16 bytes: dword j of lane l holds row l & 15, columns
// 32 j + 8 (l >> 4) .. + 7, first column in the low four bits -- the operand
// layout of four 16x16x32 matrix instructions, so a tile is one coalesced 1 KiB
// wave load.  Its scales are [row][128 / group].  Codes come first
// ([row group][tile][1024]), then the scales; rows are padded to 16 and
// columns to 128 with zeros.
constexpr int QT_K = 128;
inline int q_groups(int N) { return (N + 15) / 16; }
inline int q_tiles(int K) { return (K + QT_K - 1) / QT_K; }
inline size_t q_code_bytes(int N, int K) { return (size_t)q_groups(N) * q_tiles(K) * 1024; }
inline size_t q_bytes(int N, int K, int group) { return q_code_bytes(N, K) + (size_t)q_groups(N) * q_tiles(K) * 16 * (QT_K / group) * 2; }

struct QuantizeArgs {
  const void* w;
  int64_t ldw;
  int N, K, group;
  uint8_t* codes;     // [N][ceil(K / 2)], the lower column in the low four bits
  uint16_t* scales;   // [N][ceil(K / group)]
};
struct QuantPackArgs {
  const uint8_t* codes;
  const uint16_t* scales;
  int N, K, group;
  uint8_t* dst_codes;
  uint16_t* dst_scales;
};
struct QuantLinearArgs {
  const uint8_t* codes;
  const uint16_t* scales;
  int N, K, group, n_groups, tiles;
  const void* x; int64_t ldx;
  int M;
  bool vec;           // x can be read in pieces of eight columns, 16-byte aligned
  int y_dtype;
  void* y; int64_t ldy;
};
hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s);
hipError_t launch_quant_pack(const QuantPackArgs& a, hipStream_t s);
hipError_t launch_quant_linear(int dtype, const QuantLinearArgs& a, hipStream_t s);

}  // namespace lede
