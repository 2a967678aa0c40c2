// Layer norm and its form without the mean (RMS norm): outputs, and the gradients of inputs, weight and bias.
//
//   mu = mean x (0 without the mean), r = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) r, y = xh w + b
//   g = dy w:   dx = r (g - mean g - xh mean(g xh))   (no mean g without the mean);   dw = sum over rows of dy xh,  db = sum of dy
//
// Bound by memory: x is read and y written, dy and x are read and dx written, once each.  A row lives in the registers of a group of
// wavefronts as it came (16-byte pieces of its own type), so that the deviations are taken from the mean itself and not from the
// difference of two sums; means and deviations in fp32.  A workgroup goes through rows blockIdx, blockIdx + gridDim, ... with w and b kept in
// registers, and sums its share of dw and db there: column sums of its rows, which a second kernel adds over the workgroups in a fixed
// order.  Rows that the registers of 16 wavefronts do not hold are read again instead.
//
// 16384 x 4096 bf16 without the mean: forward 43 us (6.3 TB/s), backward 68 (5.9: a part of the inputs is still in the cache behind the
// L2), the second kernel 5.
#include "norm_device.h"

namespace {

using namespace slimnorm;

// W wavefronts per row, P pieces per lane; W == 1: four rows per workgroup.  Outputs are stored past the caches: the inputs then stay there for
// the backward pass, which reads them again (16384 x 4096 bf16: backward 82 -> 67 us; a kernel that reads the outputs next is as fast).
template <typename T, typename TW, int W, int P>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void norm_forward(NormArgs a) {
  constexpr int E = Piece<T>::E, LANES = 64 * W, RPW = W == 1 ? 4 : 1;
  __shared__ float red[2][W][1];
  const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * RPW + (W == 1 ? threadIdx.x >> 6 : 0), step = (int64_t)gridDim.x * RPW;
  const float inv_n = 1.f / (float)a.cols;
  int slot = 0;
  Piece<T> x[P];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      x[i].load(static_cast<const T*>(a.X) + row * a.ldx + c, a.cols - c);
    }
  };
  // w and b are kept where the registers hold them: read again for every row they made it 57 us in place of 43 (16384 x 4096 bf16 without
  // the mean)
  constexpr int Q = E / Piece<TW>::E;
  constexpr bool KEEP = W < 16 || P * E <= 16;
  Piece<TW> wk[KEEP ? P : 1][Q], bk[KEEP ? P : 1][Q];
  auto affine = [&](Piece<TW> (&w)[Q], Piece<TW> (&b)[Q], int c) {
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const int at = c + k * Piece<TW>::E;
      w[k].load(static_cast<const TW*>(a.w) + at, a.cols - at);
      if (a.b) b[k].load(static_cast<const TW*>(a.b) + at, a.cols - at);
    }
  };
  if (row0 < a.rows) fetch(row0);
  if constexpr (KEEP)
#pragma unroll
    for (int i = 0; i < P; ++i) affine(wk[i], bk[i], (i * LANES + lane) * E);
  for (int64_t row = row0; row < a.rows; row += step) {
    float s[1] = {0.f};
    float mean = 0.f;
    if (!a.rms) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] += x[i].get(e);
      row_sums<W, 1>(s, red, slot);
      mean = s[0] * inv_n;
      s[0] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int left = a.cols - (i * LANES + lane) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = e < left ? x[i].get(e) - mean : 0.f;
        s[0] = fmaf(d, d, s[0]);
      }
    }
    row_sums<W, 1>(s, red, slot);
    const float r = 1.f / sqrtf(fmaf(s[0], inv_n, a.eps));
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      if (c >= a.cols) break;
      float y[E];
      if constexpr (!KEEP) affine(wk[0], bk[0], c);
      const auto& w = wk[KEEP ? i : 0];
      const auto& b = bk[KEEP ? i : 0];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        constexpr int F = Piece<TW>::E;
        const float xh = (x[i].get(e) - mean) * r;
        y[e] = a.b ? fmaf(xh, w[e / F].get(e % F), b[e / F].get(e % F)) : xh * w[e / F].get(e % F);
      }
      Piece<T> o;
      o.set(y);
      o.store(static_cast<T*>(a.Y) + row * a.ldy + c, a.cols - c);
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = r;
    }
    if (row + step < a.rows) fetch(row + step);
  }
}

// Rows that no group of wavefronts holds: passes over them by single elements, the column sums by a kernel of their own (the backward pass of
// 4000 x 12288 fp32 258 us, 2.3 TB/s).
template <typename T, typename TW>
__global__ __launch_bounds__(1024) void norm_forward_long(NormArgs a) {
  __shared__ float red[2][16][1];
  int slot = 0;
  const float inv_n = 1.f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t x0 = row * a.ldx;
    float s[1] = {0.f};
    float mean = 0.f;
    if (!a.rms) {
      for (int c = threadIdx.x; c < a.cols; c += 1024) s[0] += value<T>(a.X, x0 + c);
      row_sums<16, 1>(s, red, slot);
      mean = s[0] * inv_n;
      s[0] = 0.f;
    }
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float d = value<T>(a.X, x0 + c) - mean;
      s[0] = fmaf(d, d, s[0]);
    }
    row_sums<16, 1>(s, red, slot);
    const float r = 1.f / sqrtf(fmaf(s[0], inv_n, a.eps));
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float xh = (value<T>(a.X, x0 + c) - mean) * r, w = value<TW>(a.w, c);
      put<T>(a.Y, row * a.ldy + c, a.b ? fmaf(xh, w, value<TW>(a.b, c)) : xh * w);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = r;
    }
  }
}
template <typename T, typename TW>
slim_status forward(slim_ctx* ctx, const NormArgs& a) {
  constexpr int E = Piece<T>::E;
  const int pieces = slim_cdiv(a.cols, E);
  const int64_t many = (int64_t)8 * ctx->num_cus;
  const char* name = "norm_forward";
  auto grid = [&](int64_t groups, int per_cu) { return dim3((unsigned)std::min<int64_t>(groups, (int64_t)per_cu * ctx->num_cus)); };
  const bool few = a.rows < many;              // rows that do not fill the chip: more lanes per row
  if (pieces <= 64) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 1, 1>), grid((a.rows + 3) / 4, 8), dim3(256), 0, a);
  else if (pieces <= 256 && (few || pieces > 128)) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 4, 1>), grid(a.rows, 8), dim3(256), 0, a);
  else if (pieces <= 128) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 1, 2>), grid((a.rows + 3) / 4, 8), dim3(256), 0, a);
  else if (pieces <= 512) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 4, 2>), grid(a.rows, 8), dim3(256), 0, a);
  else if (pieces <= 1024) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 4, 4>), grid(a.rows, 8), dim3(256), 0, a);
  else if (pieces <= 2048) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 16, 2>), grid(a.rows, 2), dim3(1024), 0, a);
  else if (pieces <= 4096) SLIM_LAUNCH(ctx, name, (norm_forward<T, TW, 16, 4>), grid(a.rows, 2), dim3(1024), 0, a);
  else SLIM_LAUNCH(ctx, name, (norm_forward_long<T, TW>), grid(a.rows, 2), dim3(1024), 0, a);
  return SLIM_OK;
}

}  // namespace

extern "C" {

size_t slim_layer_norm_backward_workspace(int64_t rows, int cols, slim_dtype x_dtype, int bias, int num_cus) {
  if (rows <= 0 || cols <= 0) return 0;
  const int ncu = num_cus > 0 ? num_cus : 256;
  const size_t one = slim_ws_round(sizeof(float) * (size_t)std::max(parts_of(rows, cols, x_dtype, ncu, false), parts_of(rows, cols, x_dtype, ncu, true)) * cols);
  return bias ? 2 * one : one;
}

slim_status slim_layer_norm(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int64_t rows, int cols, int64_t ldx, const void* w, const void* b,
                            slim_dtype w_dtype, double eps, int rms, void* Y, int64_t ldy, float* mean, float* rstd) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_layer_norm";
  if (const slim_status st = check(ctx, fn, x_dtype, w_dtype, rows, cols); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, w, "%s: null weight", fn);
  SLIM_REQUIRE(ctx, eps >= 0.0, "%s: eps = %g", fn, eps);
  if (rows == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, X && Y && ldx >= cols && ldy >= cols, "%s: null pointer, or rows shorter than cols (ldx = %lld, ldy = %lld)", fn,
               (long long)ldx, (long long)ldy);
  NormArgs a = {};
  a.X = X;
  a.w = w;
  a.b = b;
  a.Y = Y;
  a.ldx = ldx;
  a.ldy = ldy;
  a.mean = rms ? nullptr : mean;
  a.rstd = rstd;
  a.rows = rows;
  a.cols = cols;
  a.eps = (float)eps;
  a.rms = rms != 0;
  return by_type(x_dtype, w_dtype, [&](auto x, auto wt) { return forward<decltype(x), decltype(wt)>(ctx, a); });
}

slim_status slim_layer_norm_backward(slim_ctx* ctx, const void* dY, const void* X, slim_dtype x_dtype, int64_t rows, int cols, int64_t lddy,
                                     int64_t ldx, const void* w, slim_dtype w_dtype, const float* mean, const float* rstd, void* dX,
                                     int64_t lddx, void* dw, void* db) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_layer_norm_backward";
  if (const slim_status st = check(ctx, fn, x_dtype, w_dtype, rows, cols); st != SLIM_OK) return st;
  NormArgs a = {};
  int parts = 0;
  if (const slim_status st = backward_args(ctx, fn, a, dY, X, x_dtype, rows, cols, lddy, ldx, w, mean, rstd, dX, lddx, dw, db, parts); st != SLIM_OK)
    return st;
  if (rows > 0)
    return by_type(x_dtype, w_dtype, [&](auto x, auto wt) { return backward<decltype(x), decltype(wt)>(ctx, a, dw, db, parts); });
  // no rows: the sums are zero
  return by_type(x_dtype, w_dtype, [&](auto, auto wt) {
    SLIM_LAUNCH(ctx, "norm_join", norm_join<decltype(wt)>, dim3(slim_cdiv(cols, 32), db ? 2 : 1), dim3(1024), 0, a.pw, a.pb, 0, cols, dw, db);
    return SLIM_OK;
  });
}

}  // extern "C"
