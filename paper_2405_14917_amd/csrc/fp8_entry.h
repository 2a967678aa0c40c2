// Checks and workspace that the entry points of the 8-bit layers share.
#pragma once

#include "fp8_device.h"

namespace slimfp8 {

constexpr int FL_MAX = 1 << 23;            // rows and leading dimensions: offsets inside a tile of 256 rows fit 32 bits

inline bool is_16(slim_dtype d) { return d == SLIM_F16 || d == SLIM_BF16; }

inline size_t activation_bytes(int64_t rows, int64_t contraction) {
  return slim_ws_round((size_t)rows * quantized_ld(contraction)) + slim_ws_round((size_t)rows * scales_ld(contraction));
}
inline bool carve(slim_ctx* ctx, int64_t rows, int64_t contraction, uint8_t*& q, uint8_t*& s) {
  q = static_cast<uint8_t*>(slim_ws_alloc(ctx, (size_t)rows * quantized_ld(contraction)));
  s = static_cast<uint8_t*>(slim_ws_alloc(ctx, (size_t)rows * scales_ld(contraction)));
  return q && s;
}

inline slim_status check_stored(slim_ctx* ctx, const char* fn, const char* what, const uint8_t* q, int64_t ldq, const uint8_t* s, int64_t lds,
                         int rows, int cols) {
  SLIM_REQUIRE(ctx, q && s, "%s: null %s", fn, what);
  SLIM_REQUIRE(ctx, rows > 0 && cols > 0 && rows <= FL_MAX && cols <= FL_MAX, "%s: %s is %d x %d", fn, what, rows, cols);
  SLIM_REQUIRE(ctx, slim_aligned16(q) && ((uintptr_t)s & 3u) == 0, "%s: %s has to be 16-byte aligned, its scales 4-byte", fn, what);
  SLIM_REQUIRE(ctx, ldq >= padded(cols) && ldq % BLOCK == 0 && ldq <= FL_MAX, "%s: rows of %s are whole blocks of 128 (ld = %lld)", fn, what,
               (long long)ldq);
  SLIM_REQUIRE(ctx, lds >= slim_cdiv(cols, BLOCK) && lds % 4 == 0 && lds <= FL_MAX, "%s: rows of the scales of %s are whole words (ld = %lld)", fn, what,
               (long long)lds);
  return SLIM_OK;
}

}  // namespace slimfp8
