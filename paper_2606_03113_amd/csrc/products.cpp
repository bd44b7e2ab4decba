// Entry points of the products of a batch's rows with 4-bit weights, and of the
// vocabulary head's loss with its gradient.  No call allocates, synchronises
// or keeps anything between calls.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "../../include/lede.h"
#include "loss.h"
#include "products.h"

using namespace lede;

namespace {

hipStream_t S_(void* s) { return (hipStream_t)s; }
int done(hipError_t e) { return e == hipSuccess ? LEDE_OK : LEDE_E_HIP; }
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool dtype_ok(int32_t dt) { return dt == LEDE_DTYPE_F32 || dt == LEDE_DTYPE_BF16; }
int es_of(int32_t dt) { return dt == LEDE_DTYPE_BF16 ? 2 : 4; }

// A 4-bit matrix's shape: LEDE_OK, or why it is none.  Tiles (16 rows x 128
// columns) are numbered in 31 bits, rows and columns are below 2^24.
constexpr int32_t MOST_SIDE = (1 << 24) - 1;
int check_quant(int32_t N, int32_t K, int32_t group) {
  if (N < 1 || K < 1) return LEDE_E_ARG;
  if (group != 32 && group != 64 && group != 128) return LEDE_E_UNSUPPORTED;
  if (N > MOST_SIDE || K > MOST_SIDE || (int64_t)q_groups(N) * q_tiles(K) > (1 << 23)) return LEDE_E_UNSUPPORTED;
  return LEDE_OK;
}

// ---- the vocabulary head's loss ----

constexpr int32_t MOST_ROWS = 1 << 18, MOST_VOCAB = 1 << 20, MOST_WIDTH = 1 << 15;
constexpr int32_t LAUNCH_ROWS = 1 << 17;   // with MOST_VOCAB, of whose tiles a launch has fewer than 2^32 threads
int check_head(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  if (!dtype_ok(dtype) || M < 0 || V < 1 || K < 1) return LEDE_E_ARG;
  return K % 8 || M > MOST_ROWS || V > MOST_VOCAB || K > MOST_WIDTH ? LEDE_E_UNSUPPORTED : LEDE_OK;
}
// Row strides: a tile's rows are addressed with 32 bits.
bool stride_ok(int64_t ld) { return ld < 1 << 22; }
// Rows that the kernels read or write in 16-byte pieces.  The stride of a single
// one has nothing to meet but to hold it, and becomes `width`.
bool rows_ok(const void* p, int64_t& ld, int64_t rows, int64_t width, int32_t dt) {
  if (!p || !aligned(p, 16) || ld < width) return false;
  if (rows == 1) ld = width;
  return ld * es_of(dt) % 16 == 0;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// The tile of a product's blocks, n_i x n_j outputs: wide ones read each operand
// less often; where they would be few, small ones of which more are on the card
// and more steps on their way (fp32, 32 rows of 1024 x 256 with the
// gradient in tiles of 64 43 us, of 128 58; bf16, 2 rows of 32000 82, in tiles of
// 256 161).
// Fp32 rows with the head's: thin ones where rows or blocks are few (200 rows of
// 1024 x 512 8 us, 22 with 64 x 128); of 64 head rows where there are few of 128
// (47 rows of 32000 x 5120 222 and 233, 21 of 118860 x 5120 566 and 542), and as
// narrow as lets each block have a CU (60 rows of 1024 x 2048 20, 42 with 64).
HeadTile thin_tile(int i, int64_t n_j) { return {i, n_j <= 16 ? 16 : n_j <= 32 ? 32 : 64, true}; }
HeadTile head_tile(int32_t dtype, int64_t n_i, int64_t n_j, bool head_rows) {
  const auto blocks = [&](int i, int j) { return (n_i + i - 1) / i * ((n_j + j - 1) / j); };
  if (dtype == LEDE_DTYPE_F32) {
    if (head_rows && (n_j <= 64 || blocks(64, 128) < 128)) {
      if (blocks(128, 64) >= 512) return thin_tile(128, n_j);
      return thin_tile(64, blocks(64, 16) <= 256 ? 16 : blocks(64, 32) <= 256 ? std::min<int64_t>(n_j, 32) : n_j);
    }
    const int j = n_j <= 64 ? 64 : 128;
    return {j == 64 || blocks(128, j) < 128 ? 64 : 128, j};
  }
  const int j = n_j <= 64 ? 64 : n_j <= 128 ? 128 : 256;
  return blocks(256, j) < 64 ? HeadTile{128, 64} : HeadTile{256, j};
}

// Entries of the vocabulary at a time: dz of a piece takes at most DZ_BYTES (or
// it is one tile wide).  A multiple of 256, so that tiles of the pieces are
// tiles of the whole.
constexpr int64_t DZ_BYTES = 128 << 20;
int piece_size(int32_t dtype, int32_t M, int32_t V) {
  int64_t most = DZ_BYTES / std::max<int64_t>((int64_t)M * es_of(dtype), 1);
  if (most >= V) return V;
  most = std::max<int64_t>(256, most / 256 * 256);
  const int64_t n = (V + most - 1) / most, each = (V + n - 1) / n;
  return (int)((each + 255) / 256 * 256);
}

// Bytes of the workspaces' parts, in their order.
struct LossPlan {
  int tiles;
  HeadTile tile;
  size_t sums, target, total;
  LossPlan(int32_t dtype, int32_t M, int32_t V) {
    tile = head_tile(dtype, V, M, true);
    tiles = (V + tile.i - 1) / tile.i;
    sums = up256((size_t)M * tiles * 8);
    target = up256((size_t)M * 4);
    total = sums + target;
  }
};
struct GradPlan {
  int piece, ldz, split, chunk;
  HeadTile tile_z, tile_h, tile_w;   // of dz, dh and dW
  size_t h, dz, rest, part, total;
  GradPlan(int32_t dtype, int32_t M, int32_t V, int32_t K) {
    const bool f32 = dtype == LEDE_DTYPE_F32;
    piece = piece_size(dtype, M, V);
    const int n = std::min(piece, V);
    ldz = (n + 7) & ~7;
    tile_z = head_tile(dtype, n, M, true);
    tile_w = head_tile(dtype, K, n, false);
    // dh has few tiles: its contraction over the vocabulary is split so that
    // about a block is there for each CU (fp32, of whose blocks a CU holds
    // several: three or four)
    const auto parts = [&](HeadTile t, int64_t most) {
      const int64_t blocks = (int64_t)((K + t.i - 1) / t.i) * std::max(1, (M + t.j - 1) / t.j);
      const int64_t want = std::max<int64_t>(1, std::min<int64_t>(most / blocks, ldz / 256));
      return std::pair<int64_t, int64_t>{want, blocks * want};
    };
    tile_h = f32 ? thin_tile(256, M) : HeadTile{256, M <= 64 ? 64 : M <= 128 ? 128 : 256};
    auto p = parts(tile_h, f32 ? 768 : 256);
    if (f32 && (M > 64 || p.second < 128)) {
      tile_h = {M <= 64 ? 64 : 128, M <= 64 ? 64 : 128};
      p = parts(tile_h, 1024);
      if (p.second < 128) tile_h.i = 64;
    }
    if (!f32 && p.second < 64) tile_h = {128, 64};
    const int64_t want = p.first;
    chunk = (int)((ldz + want - 1) / want + 63) & ~63;
    split = (ldz + chunk - 1) / chunk;
    h = up256((size_t)M * K * es_of(dtype));
    dz = up256((size_t)M * ldz * es_of(dtype));
    rest = up256((size_t)M * 4);
    part = up256((size_t)split * M * K * 4);
    total = h + dz + rest + part;
  }
};

}  // namespace

extern "C" {

size_t lede_op_head_loss_bytes(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  return check_head(dtype, M, V, K) ? 0 : LossPlan(dtype, M, V).total;
}
size_t lede_op_head_loss_grad_bytes(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  return check_head(dtype, M, V, K) ? 0 : GradPlan(dtype, M, V, K).total;
}

int lede_op_head_loss(int32_t dtype, const void* hidden, int64_t ldh, int32_t M, const void* head, int64_t ldw, int32_t V,
                      int32_t K, const int32_t* targets, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                      void* stream) {
  if (int rc = check_head(dtype, M, V, K)) return rc;
  if (M == 0) return LEDE_OK;
  if (!targets || !lse || !rows_ok(hidden, ldh, M, K, dtype) || !rows_ok(head, ldw, V, K, dtype)) return LEDE_E_ARG;
  if (!stride_ok(ldh) || !stride_ok(ldw)) return LEDE_E_UNSUPPORTED;
  const LossPlan p(dtype, M, V);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total) return LEDE_E_ARG;
  hipStream_t s = S_(stream);
  HeadArgs a{};
  float2* const sums = (float2*)workspace;
  float* const target_z = (float*)((uint8_t*)workspace + p.sums);
  a.ld_sums = p.tiles;
  a.A = (const uint8_t*)head; a.lda = ldw; a.n_i = V;
  a.ldb = ldh;
  a.C = a.chunk = K; a.split = 1;
  a.V = V;
  for (int m0 = 0; m0 < M; m0 += LAUNCH_ROWS) {
    a.B = (const uint8_t*)hidden + m0 * ldh * es_of(dtype); a.n_j = std::min(LAUNCH_ROWS, M - m0);
    a.sums = sums + (int64_t)m0 * p.tiles; a.target_z = target_z + m0; a.targets = targets + m0;
    if (hipError_t e = launch_head(dtype, HEAD_SUMS, a, p.tile, s)) return done(e);
  }
  HeadJoinArgs j{};
  j.sums = sums; j.target_z = target_z; j.n = M; j.tiles = p.tiles; j.tile = p.tile.i; j.V = V; j.targets = targets; j.loss = loss; j.lse = lse;
  if (dtype == LEDE_DTYPE_F32) {
    j.hidden = (const float*)hidden; j.ldh = ldh; j.head = (const float*)head; j.ldw = ldw; j.K = K;
  }
  return done(launch_head_join(j, s));
}

int lede_op_head_loss_grad(int32_t dtype, const void* hidden, int64_t ldh, int32_t M, const void* head, int64_t ldw, int32_t V,
                           int32_t K, const int32_t* targets, const float* lse, const float* weights, void* d_hidden, int64_t ld_dh,
                           void* d_head, int64_t ld_dw, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_head(dtype, M, V, K)) return rc;
  if (!d_head && (!d_hidden || M == 0)) return LEDE_OK;
  if (d_head && !rows_ok(d_head, ld_dw, V, K, dtype)) return LEDE_E_ARG;
  if (M && (!targets || !lse || !rows_ok(hidden, ldh, M, K, dtype) || !rows_ok(head, ldw, V, K, dtype))) return LEDE_E_ARG;
  if (M && d_hidden && !rows_ok(d_hidden, ld_dh, M, K, dtype)) return LEDE_E_ARG;
  if (M && (!stride_ok(ldw) || !stride_ok(ldh))) return LEDE_E_UNSUPPORTED;
  const GradPlan p(dtype, M, V, K);
  if (p.total && (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total)) return LEDE_E_ARG;
  hipStream_t s = S_(stream);
  uint8_t *wh = (uint8_t*)workspace, *wz = wh + p.h, *wr = wz + p.dz, *wp = wr + p.rest;
  const bool outer = M <= (dtype == LEDE_DTYPE_F32 ? HEAD_OUTER_F32 : HEAD_OUTER_BF16);
  if (d_head && !outer) {
    HeadCopyArgs c{};
    c.src = hidden; c.pitch = ldh * es_of(dtype); c.n = M; c.chunks = K * es_of(dtype) / 16; c.dst = wh;
    c.targets = targets; c.weights = weights; c.V = V;
    if (hipError_t e = launch_head_copy(c, s)) return done(e);
  }
  for (int v0 = 0; v0 < V; v0 += p.piece) {
    const int n = std::min(p.piece, V - v0);
    const uint8_t* w = (const uint8_t*)head + v0 * ldw * es_of(dtype);
    HeadArgs a{};
    a.V = V; a.v0 = v0; a.split = 1;
    if (M) {
      HeadArgs z = a;
      z.A = w; z.lda = ldw; z.n_i = n;
      z.B = (const uint8_t*)hidden; z.ldb = ldh; z.n_j = M;
      z.C = z.chunk = K;
      z.targets = targets; z.weights = weights; z.lse = lse;
      z.dz = wz; z.ldz = p.ldz; z.rest = (float*)wr;
      if (hipError_t e = launch_head(dtype, HEAD_DZ, z, p.tile_z, s)) return done(e);
    }
    if (M && d_hidden) {
      HeadArgs h = a;
      h.A = w; h.lda = ldw; h.n_i = K;
      h.B = wz; h.ldb = p.ldz; h.n_j = M;
      h.C = n; h.chunk = p.chunk; h.split = p.split;
      h.part = (float*)wp; h.add = v0 > 0;
      if (hipError_t e = launch_head(dtype, HEAD_PART, h, p.tile_h, s)) return done(e);
    }
    if (d_head) {
      HeadArgs d = a;
      d.A = wh; d.lda = K; d.n_i = K;
      d.B = wz; d.ldb = p.ldz; d.n_j = n;
      d.C = d.chunk = M;
      d.out = (uint8_t*)d_head + v0 * ld_dw * es_of(dtype); d.ldo = ld_dw;
      d.targets = targets; d.weights = weights; d.rest = (float*)wr;
      if (outer) {
        d.A = (const uint8_t*)hidden; d.lda = ldh;
      }
      if (hipError_t e = outer ? launch_head_outer(dtype, d, s) : launch_head(dtype, HEAD_OUT, d, p.tile_w, s)) return done(e);
    }
  }
  if (M && d_hidden) {
    HeadOutArgs o{};
    o.part = (const float*)wp; o.split = p.split; o.n = M; o.K = K; o.out = d_hidden; o.ldo = ld_dh;
    o.targets = targets; o.weights = weights; o.rest = (const float*)wr; o.V = V; o.head = head; o.ldw = ldw;
    return done(launch_head_out(dtype, o, s));
  }
  return LEDE_OK;
}

size_t lede_op_quant_bytes(int32_t N, int32_t K, int32_t group) { return check_quant(N, K, group) ? 0 : q_bytes(N, K, group); }

int lede_op_quantize(int32_t dtype, const void* w, int64_t ldw, int32_t N, int32_t K, int32_t group, uint8_t* codes,
                     uint16_t* scales, void* stream) {
  if (!dtype_ok(dtype) || !w || !codes || !scales) return LEDE_E_ARG;
  if (int rc = check_quant(N, K, group)) return rc;
  if (ldw < K || !aligned(w, es_of(dtype)) || !aligned(scales, 2)) return LEDE_E_ARG;
  QuantizeArgs a{};
  a.w = w; a.ldw = ldw; a.N = N; a.K = K; a.group = group; a.codes = codes; a.scales = scales;
  return done(launch_quantize(dtype, a, S_(stream)));
}

int lede_op_quant_pack(const uint8_t* codes, const uint16_t* scales, int32_t N, int32_t K, int32_t group, void* packed, void* stream) {
  if (!codes || !scales || !packed) return LEDE_E_ARG;
  if (int rc = check_quant(N, K, group)) return rc;
  if (!aligned(packed, 16) || !aligned(scales, 2)) return LEDE_E_ARG;
  QuantPackArgs a{};
  a.codes = codes; a.scales = scales; a.N = N; a.K = K; a.group = group;
  a.dst_codes = (uint8_t*)packed;
  a.dst_scales = (uint16_t*)(a.dst_codes + q_code_bytes(N, K));
  return done(launch_quant_pack(a, S_(stream)));
}

int lede_op_quant_linear(int32_t dtype, const void* packed, int32_t N, int32_t K, int32_t group, const void* x, int64_t ldx,
                         int32_t M, int32_t y_dtype, void* y, int64_t ldy, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(y_dtype) || !packed || M < 0) return LEDE_E_ARG;
  if (int rc = check_quant(N, K, group)) return rc;
  if (!aligned(packed, 16)) return LEDE_E_ARG;
  if (M >= 1 << 20 || (int64_t)N * M > 1ll << 34) return LEDE_E_UNSUPPORTED;   // (a launch has fewer than 2^32 threads)
  if (M == 0) return LEDE_OK;
  if (!x || !y || ldx < K || ldy < N || !aligned(x, es_of(dtype)) || !aligned(y, es_of(y_dtype))) return LEDE_E_ARG;
  QuantLinearArgs a{};
  a.codes = (const uint8_t*)packed;
  a.scales = (const uint16_t*)(a.codes + q_code_bytes(N, K));
  a.N = N; a.K = K; a.group = group; a.n_groups = q_groups(N); a.tiles = q_tiles(K);
  a.x = x; a.ldx = ldx; a.M = M;
  a.vec = K % 8 == 0 && aligned(x, 16) && (M == 1 || ldx * es_of(dtype) % 16 == 0);
  a.y_dtype = y_dtype; a.y = y; a.ldy = ldy;
  return done(launch_quant_linear(dtype, a, S_(stream)));
}

}  // extern "C"
