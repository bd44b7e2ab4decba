// The vocabulary head's loss and its gradient (loss.hip; entry points in
// products.cpp): the kernels' arguments.  Not part of the public C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lede {

// What a product's tile becomes.
enum HeadEpi : int {
  HEAD_SUMS = 0,   // i = v, j = m: each row's maximum and sum of exponentials over the tile, and the target's logit
  HEAD_DZ = 1,     // i = v, j = m: dz, in the operands' type
  HEAD_PART = 2,   // i = k, j = m: fp32 sums of a part of the contraction over v
  HEAD_OUT = 3,    // i = k, j = v: dW (of few rows: launch_head_outer)
};

// A block's tile of a product: bf16 256 x 64, 128 or 256, or 128 x 64; fp32 64 x
// 64, 64 x 128 or 128 x 128, or thin: 64 or 128 x 16, 32 or 64, of columns 256 x
// those.
struct HeadTile { int i, j; bool thin = false; };   // thin: few fp32 rows over a large head

constexpr int HEAD_OUTER_F32 = 32, HEAD_OUTER_BF16 = 64;   // rows of launch_head_outer, at most
struct HeadArgs {
  const uint8_t *A, *B;
  int64_t lda, ldb;                // elements
  int n_i, n_j, C;                 // rows of A and B, length of the contraction
  int chunk;                       // entries of the contraction that a block takes
  int i_tiles, j_tiles, split;     // of the grid
  int band;                        // tiles of i that are taken with all of j
  const int32_t* targets; const float *weights, *lse;
  int V, v0;                       // the vocabulary, the piece's first entry
  float2* sums; int ld_sums;   // HEAD_SUMS: [row][tile of the vocabulary]
  float* target_z;
  uint8_t* dz; int ldz;            // HEAD_DZ: [row][ldz], zeros past the piece
  float* rest;                     // (bf16) [row]: what rounding took from the target's dz
  float* part; bool add;           // HEAD_PART: [split][row][K]
  void* out; int64_t ldo;          // HEAD_OUT
};
struct HeadCopyArgs {
  const void* src; int64_t pitch;  // bytes between rows
  int64_t n; int chunks;           // of 16 bytes, in a row
  uint8_t* dst;
  const int32_t* targets; const float* weights; int V;
};
struct HeadJoinArgs {
  const float2* sums; const float* target_z;
  int n, tiles, tile, V;           // (tile: entries of the vocabulary)
  const int32_t* targets;
  float *loss, *lse;
  const float *hidden, *head;      // (fp32; else null)
  int64_t ldh, ldw;
  int K;
};
struct HeadOutArgs {
  const float* part;
  int split; int64_t n; int K;
  const int32_t* targets; const float* weights; int V;
  const float* rest; const void* head; int64_t ldw;   // (bf16)
  void* out; int64_t ldo;
};
hipError_t launch_head(int dtype, int epi, const HeadArgs& a, HeadTile tile, hipStream_t s);
hipError_t launch_head_outer(int dtype, const HeadArgs& a, hipStream_t s);   // dW; of few rows
hipError_t launch_head_copy(const HeadCopyArgs& a, hipStream_t s);
hipError_t launch_head_join(const HeadJoinArgs& a, hipStream_t s);
hipError_t launch_head_out(int dtype, const HeadOutArgs& a, hipStream_t s);

}  // namespace lede
