// Entry points of the 8-bit linear layer.  Forward: few tokens or little work in one launch (fp8_few.hip), more as a launch that quantises the
// activations into the workspace and one that multiplies (fp8_gemm.hip).  Backward: one launch quantises the gradient of the
// outputs in both directions (blocks of outputs for dX, blocks of tokens for dW) and the activations along the tokens, one multiplies:
//   Y  (t x n) : A = W  (n rows),            B = Q(X)    (t rows),  contraction over m
//   dX (t x m) : A = Wt (m rows),            B = Q(dY)   (t rows),  contraction over n
//   dW (n x m) : A = Qt(X) (m rows),         B = Qt(dY)  (n rows),  contraction over t
// With an epilogue the same kernels add bias and residual and apply the activation before the outputs are stored (where a product is cut along
// its contraction, the kernel that adds the parts does), and the activations may come in 8 bits; in its backward pass the launch that quantises the
// gradient of the outputs first multiplies it by the activation's derivative, and leaves the sums of 128 rows for the bias
// (11008 x 4096, 4096 tokens, gelu, both gradients in 16 bits and the bias: 404 to 418 us, of them that launch 76, the sums' 6, the products 324, 2.28 PFLOP/s; dW in fp32 544).
#include "fp8_entry.h"

namespace {

using namespace slimfp8;

Product forward_product(int n, int m, int t, slim_dtype y_dtype) {
  Product p = {};
  p.a.rows = n;
  p.a.shift = 7;
  p.b.rows = t;
  p.c_dtype = y_dtype;
  p.nk = slim_cdiv(m, BLOCK);
  return p;
}
// products of the backward pass: of the gradients that are asked for
int backward_products(int n, int m, int t, bool dx, bool dw, slim_dtype dw_dtype, Product (&p)[2]) {
  int count = 0;
  if (dx) {
    p[count] = Product{};
    p[count].a.rows = m;
    p[count].a.shift = 7;
    p[count].b.rows = t;
    p[count++].nk = slim_cdiv(n, BLOCK);
  }
  if (dw) {
    p[count] = Product{};
    p[count].a.rows = m;
    p[count].b.rows = n;
    p[count].c_dtype = dw_dtype;
    p[count++].nk = slim_cdiv(t, BLOCK);
  }
  return count;
}
size_t forward_need(int n, int m, int t, slim_dtype y_dtype, int ncu) {
  if (takes_few_tokens(n, m, t, ncu)) return 0;
  const Product p = forward_product(n, m, t, y_dtype);
  return activation_bytes(t, m) + gemm_workspace(&p, 1, ncu);
}
size_t backward_need(int n, int m, int t, bool dx, bool dw, slim_dtype dw_dtype, int ncu) {
  if (t <= 0) return 0;
  Product p[2];
  const int count = backward_products(n, m, t, dx, dw, dw_dtype, p);
  return (dx ? activation_bytes(t, n) : 0) + (dw ? activation_bytes(n, t) + activation_bytes(m, t) : 0) + gemm_workspace(p, count, ncu);
}

// dX and dW (either may be null) from the quantised gradient of the outputs and activations
slim_status gradient_products(slim_ctx* ctx, const char* name, const Activations (&a)[2], int t, const uint8_t* qt, int64_t ldqt, const uint8_t* st,
                              int64_t ldst, int n, int m, void* dX, slim_dtype x_dtype, int64_t lddx, void* dW, slim_dtype dw_dtype, int64_t lddw) {
  Product p[2];
  const int count = backward_products(n, m, t, dX != nullptr, dW != nullptr, dw_dtype, p);
  if (dX) {
    p[0].a = Operand{qt, st, ldqt, ldst, m, 7};
    p[0].b = Operand{a[0].rows_q, a[0].rows_s, quantized_ld(n), scales_ld(n), t, 0};
    p[0].c = dX;
    p[0].ldc = lddx;
    p[0].c_dtype = x_dtype;
  }
  if (dW) {
    Product& w = p[count - 1];
    w.a = Operand{a[1].cols_q, a[1].cols_s, quantized_ld(t), scales_ld(t), m, 0};
    w.b = Operand{a[0].cols_q, a[0].cols_s, quantized_ld(t), scales_ld(t), n, 0};
    w.c = dW;
    w.ldc = lddw;
  }
  return gemm(ctx, name, p, count);
}

}  // namespace

extern "C" {

size_t slim_fp8_linear_workspace(int n, int m, int t, slim_dtype y_dtype, int num_cus) {
  if (n <= 0 || m <= 0 || t <= 0) return 0;
  return forward_need(n, m, t, y_dtype, num_cus > 0 ? num_cus : 256);
}

size_t slim_fp8_linear_backward_workspace(int n, int m, int t, int dx, int dw, slim_dtype dw_dtype, int num_cus) {
  if (n <= 0 || m <= 0 || t <= 0) return 0;
  return backward_need(n, m, t, dx != 0, dw != 0, dw_dtype, num_cus > 0 ? num_cus : 256);
}

slim_status slim_fp8_linear(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const uint8_t* q, int64_t ldq,
                            const uint8_t* s, int64_t lds, int n, int m, void* Y, slim_dtype y_dtype, int64_t ldy) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_fp8_linear";
  if (const slim_status st = check_stored(ctx, fn, "W", q, ldq, s, lds, n, m); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, t >= 0 && t <= FL_MAX, "%s: t = %d", fn, t);
  if (!is_16(x_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: X is F16 or BF16", fn);
  if (!is_16(y_dtype) && y_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: Y is F16, BF16 or F32", fn);
  if (t == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, X && Y && ldx >= m && ldy >= n, "%s: null pointer, or rows shorter than the layer (ldx = %lld, ldy = %lld)", fn,
               (long long)ldx, (long long)ldy);
  const Operand w = {q, s, ldq, lds, n, 7};
  if (takes_few_tokens(n, m, t, ctx->num_cus)) return few_tokens(ctx, X, x_dtype, t, ldx, Operand{}, w, m, nullptr, Y, y_dtype, ldy);
  if (const slim_status st = slim_ws_reserve(ctx, forward_need(n, m, t, y_dtype, ctx->num_cus)); st != SLIM_OK) return st;
  Activations a = {X, ldx, t, m, nullptr, nullptr, nullptr, nullptr};
  if (!carve(ctx, t, m, a.rows_q, a.rows_s)) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
  if (const slim_status st = quantize(ctx, "fp8_quantize_x", x_dtype, &a, 1); st != SLIM_OK) return st;
  Product p = forward_product(n, m, t, y_dtype);
  p.a = w;
  p.b = Operand{a.rows_q, a.rows_s, quantized_ld(m), scales_ld(m), t, 0};
  p.c = Y;
  p.ldc = ldy;
  return gemm(ctx, "fp8_linear", &p, 1);
}

slim_status slim_fp8_linear_backward(slim_ctx* ctx, const void* dY, const void* X, slim_dtype x_dtype, int t, int64_t lddy, int64_t ldx,
                                     const uint8_t* qt, int64_t ldqt, const uint8_t* st, int64_t ldst, int n, int m, void* dX, int64_t lddx,
                                     void* dW, slim_dtype dw_dtype, int64_t lddw) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_fp8_linear_backward";
  SLIM_REQUIRE(ctx, n > 0 && m > 0 && n <= FL_MAX && m <= FL_MAX && t >= 0 && t <= FL_MAX, "%s: n = %d, m = %d, t = %d", fn, n, m, t);
  SLIM_REQUIRE(ctx, dX || dW, "%s: neither dX nor dW", fn);
  if (dX)
    if (const slim_status e = check_stored(ctx, fn, "Wt", qt, ldqt, st, ldst, m, n); e != SLIM_OK) return e;
  if (!is_16(x_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: dY, X and dX are F16 or BF16", fn);
  if (dW && !is_16(dw_dtype) && dw_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: dW is F16, BF16 or F32", fn);
  SLIM_REQUIRE(ctx, t == 0 || (dY && lddy >= n && (!dX || lddx >= m)), "%s: null dY, or rows shorter than the layer", fn);
  SLIM_REQUIRE(ctx, !dW || (lddw >= m && (t == 0 || (X && ldx >= m))), "%s: null X, or rows shorter than the layer", fn);
  if (t == 0) dX = nullptr;                       // (no rows; dW is zero, the product over no blocks)
  if (!dX && !dW) return SLIM_OK;
  if (const slim_status e = slim_ws_reserve(ctx, backward_need(n, m, t, dX != nullptr, dW != nullptr, dw_dtype, ctx->num_cus)); e != SLIM_OK) return e;
  Activations a[2] = {{dY, lddy, t, n, nullptr, nullptr, nullptr, nullptr}, {X, ldx, t, m, nullptr, nullptr, nullptr, nullptr}};
  if (t > 0) {
    bool ok = true;
    if (dX) ok = carve(ctx, t, n, a[0].rows_q, a[0].rows_s);
    if (dW) ok = ok && carve(ctx, n, t, a[0].cols_q, a[0].cols_s) && carve(ctx, m, t, a[1].cols_q, a[1].cols_s);
    if (!ok) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
    if (const slim_status e = quantize(ctx, "fp8_quantize_grad", x_dtype, a, dW ? 2 : 1); e != SLIM_OK) return e;
  }
  return gradient_products(ctx, "fp8_linear_grad", a, t, qt, ldqt, st, ldst, n, m, dX, x_dtype, lddx, dW, dw_dtype, lddw);
}

size_t slim_fp8_linear_act_workspace(int n, int m, int t, int x_8bit, slim_dtype y_dtype, int num_cus) {
  if (n <= 0 || m <= 0 || t <= 0) return 0;
  const int ncu = num_cus > 0 ? num_cus : 256;
  if (!x_8bit) return forward_need(n, m, t, y_dtype, ncu);
  const Product p = forward_product(n, m, t, y_dtype);
  return takes_few_tokens(n, m, t, ncu) ? 0 : gemm_workspace(&p, 1, ncu);
}

slim_status slim_fp8_linear_act(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const uint8_t* xq, int64_t ldxq,
                                const uint8_t* xs, int64_t ldxs, const uint8_t* q, int64_t ldq, const uint8_t* s, int64_t lds, int n, int m,
                                const slim_epilogue* epilogue, void* Y, slim_dtype y_dtype, int64_t ldy) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_fp8_linear_act";
  if (const slim_status st = check_stored(ctx, fn, "W", q, ldq, s, lds, n, m); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, t >= 0 && t <= FL_MAX, "%s: t = %d", fn, t);
  SLIM_REQUIRE(ctx, !X || (!xq && !xs), "%s: X in 16 bits and in 8", fn);
  const bool x8 = xq || xs;
  if (!x8 && !is_16(x_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: X is F16 or BF16, or in 8 bits", fn);
  if (!is_16(y_dtype) && y_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: Y is F16, BF16 or F32", fn);
  Epilogue e = {};
  if (epilogue) {
    e = Epilogue{epilogue->bias, epilogue->R, epilogue->Z, epilogue->ldr, epilogue->ldz, (int)epilogue->bias_dtype, epilogue->act, (int)y_dtype};
    SLIM_REQUIRE(ctx, e.act >= SLIM_ACT_NONE && e.act <= SLIM_ACT_SILU, "%s: act = %d", fn, e.act);
    if (e.bias && e.bias_dtype != (int)y_dtype && e.bias_dtype != SLIM_F32)
      return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: the bias is of Y's type or F32", fn);
  }
  if (t == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, (X || x8) && Y && (!X || ldx >= m) && ldy >= n, "%s: null pointer, or rows shorter than the layer (ldx = %lld, ldy = %lld)", fn,
               (long long)ldx, (long long)ldy);
  SLIM_REQUIRE(ctx, (!e.R || e.ldr >= n) && (!e.Z || e.ldz >= n), "%s: rows of R or Z shorter than the layer (ldr = %lld, ldz = %lld)", fn,
               (long long)e.ldr, (long long)e.ldz);
  if (x8)
    if (const slim_status st = check_stored(ctx, fn, "the 8-bit X", xq, ldxq, xs, ldxs, t, m); st != SLIM_OK) return st;
  const Operand w = {q, s, ldq, lds, n, 7};
  Operand x = {xq, xs, ldxq, ldxs, t, 0};
  if (takes_few_tokens(n, m, t, ctx->num_cus)) return few_tokens(ctx, X, x_dtype, t, ldx, x, w, m, &e, Y, y_dtype, ldy);
  if (const slim_status st = slim_ws_reserve(ctx, slim_fp8_linear_act_workspace(n, m, t, x8, y_dtype, ctx->num_cus)); st != SLIM_OK) return st;
  if (!x8) {
    Activations a = {X, ldx, t, m, nullptr, nullptr, nullptr, nullptr};
    if (!carve(ctx, t, m, a.rows_q, a.rows_s)) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
    if (const slim_status st = quantize(ctx, "fp8_quantize_x", x_dtype, &a, 1); st != SLIM_OK) return st;
    x = Operand{a.rows_q, a.rows_s, quantized_ld(m), scales_ld(m), t, 0};
  }
  Product p = forward_product(n, m, t, y_dtype);
  p.a = w;
  p.b = x;
  p.c = Y;
  p.ldc = ldy;
  p.e = &e;
  return gemm(ctx, "fp8_linear_act", &p, 1);
}

size_t slim_fp8_linear_act_backward_workspace(int n, int m, int t, int dx, int dw, slim_dtype dw_dtype, int db, int num_cus) {
  if (n <= 0 || m <= 0 || t <= 0) return 0;
  return backward_need(n, m, t, dx != 0, dw != 0, dw_dtype, num_cus > 0 ? num_cus : 256) + (db ? slim_ws_round(sizeof(float) * (size_t)slim_cdiv(t, BLOCK) * n) : 0);
}

slim_status slim_fp8_linear_act_backward(slim_ctx* ctx, const void* dY, const void* Z, int act, const void* X, slim_dtype x_dtype, int t,
                                         int64_t lddy, int64_t ldz, int64_t ldx, const uint8_t* qt, int64_t ldqt, const uint8_t* st, int64_t ldst,
                                         int n, int m, void* dX, int64_t lddx, void* dW, slim_dtype dw_dtype, int64_t lddw, void* db,
                                         slim_dtype db_dtype) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_fp8_linear_act_backward";
  SLIM_REQUIRE(ctx, act >= SLIM_ACT_NONE && act <= SLIM_ACT_SILU, "%s: act = %d", fn, act);
  if (act == SLIM_ACT_NONE && !db)           // nothing in front of the products
    return slim_fp8_linear_backward(ctx, dY, X, x_dtype, t, lddy, ldx, qt, ldqt, st, ldst, n, m, dX, lddx, dW, dw_dtype, lddw);
  SLIM_REQUIRE(ctx, n > 0 && m > 0 && n <= FL_MAX && m <= FL_MAX && t >= 0 && t <= FL_MAX, "%s: n = %d, m = %d, t = %d", fn, n, m, t);
  SLIM_REQUIRE(ctx, dX || dW || db, "%s: no gradient is wanted", fn);
  if (dX)
    if (const slim_status e = check_stored(ctx, fn, "Wt", qt, ldqt, st, ldst, m, n); e != SLIM_OK) return e;
  if (!is_16(x_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: dY, Z, X and dX are F16 or BF16", fn);
  if (dW && !is_16(dw_dtype) && dw_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: dW is F16, BF16 or F32", fn);
  if (db && !is_16(db_dtype) && db_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: db is F16, BF16 or F32", fn);
  SLIM_REQUIRE(ctx, t == 0 || (dY && lddy >= n && (act == SLIM_ACT_NONE || (Z && ldz >= n)) && (!dX || lddx >= m)),
               "%s: null dY or Z, or rows shorter than the layer", fn);
  SLIM_REQUIRE(ctx, !dW || (lddw >= m && (t == 0 || (X && ldx >= m))), "%s: null X, or rows shorter than the layer", fn);
  if (t == 0) dX = nullptr;                       // (no rows; dW and db are zero)
  const size_t need = slim_fp8_linear_act_backward_workspace(n, m, t, dX != nullptr, dW != nullptr, dw_dtype, db != nullptr, ctx->num_cus);
  if (const slim_status e = slim_ws_reserve(ctx, need); e != SLIM_OK) return e;
  Activations a[2] = {{dY, lddy, t, n, nullptr, nullptr, nullptr, nullptr}, {X, ldx, dW ? t : 0, m, nullptr, nullptr, nullptr, nullptr}};
  float* sums = nullptr;
  if (t > 0) {
    bool ok = true;
    if (dX) ok = carve(ctx, t, n, a[0].rows_q, a[0].rows_s);
    if (dW) ok = ok && carve(ctx, n, t, a[0].cols_q, a[0].cols_s) && carve(ctx, m, t, a[1].cols_q, a[1].cols_s);
    if (db) ok = ok && (sums = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)slim_cdiv(t, BLOCK) * n)));
    if (!ok) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
    const ActGradient g = {act == SLIM_ACT_NONE ? nullptr : Z, ldz, act, sums};
    if (const slim_status e = quantize_gradient(ctx, "fp8_quantize_act", x_dtype, a, g); e != SLIM_OK) return e;
  }
  if (db)
    if (const slim_status e = join_columns(ctx, "fp8_bias_grad", sums, t > 0 ? slim_cdiv(t, BLOCK) : 0, n, db, db_dtype); e != SLIM_OK) return e;
  if (!dX && !dW) return SLIM_OK;
  return gradient_products(ctx, "fp8_linear_act_grad", a, t, qt, ldqt, st, ldst, n, m, dX, x_dtype, lddx, dW, dw_dtype, lddw);
}

}  // extern "C"
