// Entry points of the products of a batch's rows with 4-bit weights, and of the
// vocabulary head's loss with its gradient.  No call allocates, synchronises
// or keeps anything between calls.
#include <hip/hip_runtime.h>

#include <algorithm>

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
int check_head(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  if (!dtype_ok(dtype) || M < 0 || V < 1 || K < 1) return LEDE_E_ARG;
  return K % 8 || M > MOST_ROWS || V > MOST_VOCAB || K > MOST_WIDTH ? LEDE_E_UNSUPPORTED : LEDE_OK;
}
// Row strides: a tile's rows are addressed with 32 bits.
bool stride_ok(int64_t ld) { return ld < 1 << 22; }
// Rows that the kernels read or write in 16-byte pieces.
bool rows_ok(const void* p, int64_t ld, int64_t width, int32_t dt) {
  return p && aligned(p, 16) && ld >= width && ld * es_of(dt) % 16 == 0;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// fp32 rows up to which the operands are split on their way to LDS (us, with the
// gradient, 32000 x 5120: FEW_TABLE).
constexpr int32_t FEW_ROWS = 128;
HeadMode head_mode(int32_t dtype, int32_t M) { return dtype == LEDE_DTYPE_BF16 ? HEAD_BF16 : M <= FEW_ROWS ? HEAD_FP32 : HEAD_PARTS; }

// The tile of a product's blocks, n_i x n_j outputs: wide ones read each operand
// less often; where they would be few, small ones of which more are on the card
// and more steps on their way.
HeadTile head_tile(HeadMode mode, int64_t n_i, int64_t n_j) {
  if (mode == HEAD_FP32) return {128, n_j <= 64 ? 64 : 128};
  const int j = n_j <= 64 ? 64 : n_j <= 128 ? 128 : 256;
  if ((n_i + 255) / 256 * ((n_j + j - 1) / j) < 64) return {128, 64};
  return {256, j};
}
int64_t head_blocks(HeadTile t, int64_t n_i, int64_t n_j) { return (n_i + t.i - 1) / t.i * ((n_j + t.j - 1) / t.j); }

// Entries of the vocabulary at a time: dz of a piece takes at most DZ_BYTES, the
// parts of its rows of an fp32 head at most W_BYTES (or it is one tile wide);
// pieces must be wide enough to fill the card (500 rows over 32000 x 2048 in
// three pieces 2.7 ms, in one PIECE_ONE).  A multiple of 256, so that tiles of
// the pieces are tiles of the whole.
constexpr int64_t DZ_BYTES = 128 << 20, W_BYTES = 1 << 30;
int piece_size(HeadMode mode, int32_t M, int32_t V, int32_t K, bool grad) {
  int64_t most = V;
  if (grad) most = std::min(most, DZ_BYTES / std::max<int64_t>((int64_t)M * (mode == HEAD_BF16 ? 2 : mode == HEAD_PARTS ? 6 : 4), 1));
  if (mode == HEAD_PARTS) most = std::min(most, W_BYTES / ((int64_t)K * 6));
  if (most >= V) return V;
  most = std::max<int64_t>(256, most / 256 * 256);
  const int64_t n = (V + most - 1) / most, each = (V + n - 1) / n;
  return (int)((each + 255) / 256 * 256);
}

// Bytes of the workspaces' parts, in their order.
struct LossPlan {
  HeadMode mode;
  int tiles, piece;
  HeadTile tile;
  int64_t plane_h, plane_w;
  size_t sums, target, h, w, total;
  LossPlan(int32_t dtype, int32_t M, int32_t V, int32_t K) {
    mode = head_mode(dtype, M);
    piece = piece_size(mode, M, V, K, false);
    tile = head_tile(mode, piece, M);
    tiles = (V + tile.i - 1) / tile.i;
    plane_h = (int64_t)M * K * 2;
    plane_w = (int64_t)std::min(piece, V) * K * 2;
    sums = up256((size_t)M * tiles * 8);
    target = up256((size_t)M * 4);
    h = mode == HEAD_PARTS ? up256(3 * plane_h) : 0;
    w = mode == HEAD_PARTS ? up256(3 * plane_w) : 0;
    total = sums + target + h + w;
  }
};
struct GradPlan {
  HeadMode mode;
  int piece, ldz, split, chunk;
  HeadTile tile_z, tile_h, tile_w;   // of dz, dh and dW
  int64_t plane_h, plane_w, plane_dz;
  size_t h, w, dz, rest, part, total;
  GradPlan(int32_t dtype, int32_t M, int32_t V, int32_t K) {
    mode = head_mode(dtype, M);
    piece = piece_size(mode, M, V, K, true);
    const int n = std::min(piece, V);
    ldz = (n + 7) & ~7;
    tile_z = head_tile(mode, n, M);
    tile_w = head_tile(mode, K, n);
    // dh has few tiles: its contraction over the vocabulary is split so that
    // about a block is there for each CU (of k_head_few's, four)
    tile_h = mode == HEAD_FP32 ? head_tile(mode, K, M) : HeadTile{256, M <= 64 ? 64 : M <= 128 ? 128 : 256};
    const int64_t blocks = std::max<int64_t>(1, head_blocks(tile_h, K, M));
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>((mode == HEAD_FP32 ? 1024 : 256) / blocks, ldz / 256));
    if (mode != HEAD_FP32 && blocks * want < 64) tile_h = {128, 64};
    chunk = (int)((ldz + want - 1) / want + 63) & ~63;
    split = (ldz + chunk - 1) / chunk;
    plane_h = (int64_t)M * K * 2;
    plane_w = (int64_t)n * K * 2;
    plane_dz = (int64_t)M * ldz * 2;
    h = up256((mode == HEAD_BF16 ? 1 : mode == HEAD_PARTS ? 3 : 2) * plane_h);
    w = mode == HEAD_PARTS ? up256(3 * plane_w) : 0;
    dz = up256((mode == HEAD_BF16 ? 1 : mode == HEAD_PARTS ? 3 : 2) * plane_dz);
    rest = up256((size_t)M * 4);
    part = up256((size_t)split * M * K * 4);
    total = h + w + dz + rest + part;
  }
};

}  // namespace

extern "C" {

size_t lede_op_head_loss_bytes(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  return check_head(dtype, M, V, K) ? 0 : LossPlan(dtype, M, V, K).total;
}
size_t lede_op_head_loss_grad_bytes(int32_t dtype, int32_t M, int32_t V, int32_t K) {
  return check_head(dtype, M, V, K) ? 0 : GradPlan(dtype, M, V, K).total;
}

int lede_op_head_loss(int32_t dtype, const void* hidden, int64_t ldh, int32_t M, const void* head, int64_t ldw, int32_t V,
                      int32_t K, const int32_t* targets, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                      void* stream) {
  if (int rc = check_head(dtype, M, V, K)) return rc;
  if (M == 0) return LEDE_OK;
  if (!targets || !lse || !rows_ok(hidden, ldh, K, dtype) || !rows_ok(head, ldw, K, dtype)) return LEDE_E_ARG;
  if (!stride_ok(ldh) || !stride_ok(ldw)) return LEDE_E_UNSUPPORTED;
  const LossPlan p(dtype, M, V, K);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total) return LEDE_E_ARG;
  hipStream_t s = S_(stream);
  uint8_t* ws = (uint8_t*)workspace;
  HeadArgs a{};
  a.sums = (float2*)ws; a.ld_sums = p.tiles;
  a.target_z = (float*)(ws + p.sums);
  uint8_t *wh = ws + p.sums + p.target, *ww = wh + p.h;
  a.mode = p.mode;
  a.n_j = M; a.C = a.chunk = K;
  a.targets = targets; a.V = V;
  if (p.mode != HEAD_PARTS) {
    a.A = (const uint8_t*)head; a.lda = ldw; a.B = (const uint8_t*)hidden; a.ldb = ldh; a.n_i = V;
    if (hipError_t e = launch_head(HEAD_SUMS, a, 1, p.tile, s)) return done(e);
  } else {
    HeadCopyArgs c{};
    c.src = hidden; c.ld = ldh; c.n = M; c.K = K; c.dst = wh; c.plane = p.plane_h;
    if (hipError_t e = launch_head_copy(p.mode, c, s)) return done(e);
    a.A = ww; a.lda = K; a.plane_a = p.plane_w; a.B = wh; a.ldb = K; a.plane_b = p.plane_h;
    for (int v0 = 0; v0 < V; v0 += p.piece) {
      a.v0 = v0; a.n_i = std::min(p.piece, V - v0); a.tile0 = v0 / p.tile.i;
      c.src = (const float*)head + v0 * ldw; c.ld = ldw; c.n = a.n_i; c.dst = ww; c.plane = p.plane_w;
      if (hipError_t e = launch_head_copy(p.mode, c, s)) return done(e);
      if (hipError_t e = launch_head(HEAD_SUMS, a, 1, p.tile, s)) return done(e);
    }
  }
  HeadJoinArgs j{};
  j.sums = a.sums; j.target_z = a.target_z; j.n = M; j.tiles = p.tiles; j.V = V; j.targets = targets; j.loss = loss; j.lse = lse;
  return done(launch_head_join(j, s));
}

int lede_op_head_loss_grad(int32_t dtype, const void* hidden, int64_t ldh, int32_t M, const void* head, int64_t ldw, int32_t V,
                           int32_t K, const int32_t* targets, const float* lse, const float* weights, void* d_hidden, int64_t ld_dh,
                           void* d_head, int64_t ld_dw, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_head(dtype, M, V, K)) return rc;
  if (!d_head && (!d_hidden || M == 0)) return LEDE_OK;
  if (d_head && !rows_ok(d_head, ld_dw, K, dtype)) return LEDE_E_ARG;
  if (M && (!targets || !lse || !rows_ok(hidden, ldh, K, dtype) || !rows_ok(head, ldw, K, dtype))) return LEDE_E_ARG;
  if (M && d_hidden && !rows_ok(d_hidden, ld_dh, K, dtype)) return LEDE_E_ARG;
  if (M && !stride_ok(ldw)) return LEDE_E_UNSUPPORTED;
  const GradPlan p(dtype, M, V, K);
  if (p.total && (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total)) return LEDE_E_ARG;
  hipStream_t s = S_(stream);
  uint8_t *wh = (uint8_t*)workspace, *ww = wh + p.h, *wz = ww + p.w, *wr = wz + p.dz, *wp = wr + p.rest;
  if (M) {
    HeadCopyArgs c{};
    c.src = hidden; c.ld = ldh; c.n = M; c.K = K; c.dst = wh; c.plane = p.plane_h;
    c.targets = targets; c.weights = weights; c.V = V;
    if (hipError_t e = launch_head_copy(p.mode, c, s)) return done(e);
  }
  for (int v0 = 0; v0 < V; v0 += p.piece) {
    const int n = std::min(p.piece, V - v0);
    const uint8_t* w = (const uint8_t*)head + v0 * ldw * es_of(dtype);
    int64_t lw = ldw;
    if (M && p.mode == HEAD_PARTS) {
      HeadCopyArgs c{};
      c.src = w; c.ld = ldw; c.n = n; c.K = K; c.dst = ww; c.plane = p.plane_w;
      if (hipError_t e = launch_head_copy(p.mode, c, s)) return done(e);
      w = ww;
      lw = K;
    }
    HeadArgs a{};
    a.mode = p.mode;
    a.V = V; a.v0 = v0;
    if (M) {
      HeadArgs z = a;
      z.A = w; z.lda = lw; z.plane_a = p.plane_w; z.n_i = n;
      z.B = wh; z.ldb = K; z.plane_b = p.plane_h; z.n_j = M;
      z.C = z.chunk = K;
      z.targets = targets; z.weights = weights; z.lse = lse;
      z.dz = wz; z.plane_dz = p.plane_dz; z.ldz = p.ldz; z.rest = (float*)wr;
      if (hipError_t e = launch_head(HEAD_DZ, z, 1, p.tile_z, s)) return done(e);
    }
    if (M && d_hidden) {
      HeadArgs h = a;
      h.A = w; h.lda = lw; h.plane_a = p.plane_w; h.n_i = K;
      h.B = wz; h.ldb = p.ldz; h.plane_b = p.plane_dz; h.n_j = M;
      h.C = n; h.chunk = p.chunk;
      h.part = (float*)wp; h.add = v0 > 0;
      if (hipError_t e = launch_head(HEAD_PART, h, p.split, p.tile_h, s)) return done(e);
    }
    if (d_head) {
      HeadArgs d = a;
      d.A = wh; d.lda = K; d.plane_a = p.plane_h; d.n_i = K;
      d.B = wz; d.ldb = p.ldz; d.plane_b = p.plane_dz; d.n_j = n;
      d.C = d.chunk = M;
      d.out = (uint8_t*)d_head + v0 * ld_dw * es_of(dtype); d.ldo = ld_dw;
      if (hipError_t e = launch_head(HEAD_OUT, d, 1, p.tile_w, s)) return done(e);
    }
  }
  if (M && d_hidden) {
    HeadOutArgs o{};
    o.part = (const float*)wp; o.split = p.split; o.n = M; o.K = K; o.out = d_hidden; o.ldo = ld_dh;
    o.targets = targets; o.rest = (const float*)wr; o.V = V; o.head = head; o.ldw = ldw;
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
