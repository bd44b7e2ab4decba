// Entry points of the products of a batch's rows with 4-bit weights.  No call
// allocates, synchronises or keeps anything between calls.
#include <hip/hip_runtime.h>

#include "../../include/lede.h"
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
  if (N > MOST_SIDE || K > MOST_SIDE || (int64_t)q_groups(N) * q_tiles(K) > (1 << 24)) return LEDE_E_UNSUPPORTED;
  return LEDE_OK;
}

}  // namespace

extern "C" {

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
  if (M > 65535 * 16) return LEDE_E_UNSUPPORTED;
  if (M == 0) return LEDE_OK;
  if (!x || !y || ldx < K || ldy < N || !aligned(x, es_of(dtype)) || !aligned(y, es_of(y_dtype))) return LEDE_E_ARG;
  QuantLinearArgs a{};
  a.codes = (const uint8_t*)packed;
  a.scales = (const uint16_t*)(a.codes + q_code_bytes(N, K));
  a.N = N; a.K = K; a.group = group; a.n_groups = q_groups(N); a.tiles = q_tiles(K);
  a.x = x; a.ldx = ldx; a.M = M;
  a.vec = aligned(x, 16) && (M == 1 || ldx * es_of(dtype) % 16 == 0);
  a.y_dtype = y_dtype; a.y = y; a.ldy = ldy;
  return done(launch_quant_linear(dtype, a, S_(stream)));
}

}  // extern "C"
