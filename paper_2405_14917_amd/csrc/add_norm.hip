// The norm of the residual stream: h = x + r, rounded to their type, goes back to the stream and through the norm, whose output leaves in its own
// type, in the 8-bit form that the linear layers multiply (e4m3 numbers with a scale for 128 channels, of the rounded output: the same numbers that
// slim_fp8_linear makes of it), or in both.  Backward: dX = dR = dH + the norm's gradient at h (norm_device.h).
//
// Bound by memory: x and r are read, h and the output written, once each.  As in norm.hip a row lives in the registers of a group of
// wavefronts; a block of 128 channels is 16 (16-bit types) or 32 lanes one after another, so that its largest magnitude takes a few moves
// inside the wavefront, on packed 16-bit patterns where the type has 16 bits.
//
// 16384 x 4096 bf16 without the mean, the output in both forms: forward 107 us (5.6 TB/s), backward 108 to 111 (4.9 TB/s), the second kernel 5.
#include "fp8_device.h"
#include "norm_device.h"

namespace {

using namespace slimnorm;
using slimfp8::BLOCK;

// Sums over the W wavefronts of a row, of the lanes' sums in fp64: what is off in a row's factor is off in all of its numbers, and moves those next
// to a border of the 8-bit form to its other side (fp32 outputs are 4.6e-8 to 5.1e-8 off, with these sums in fp32 6.0e-8 to 6.6e-8; one rounding is
// 2.5e-8; with deviations and outputs in fp64 as well 16384 x 4096 took 102 us in place of 87)
template <int W>
__device__ __forceinline__ double row_sum(double v, double (*red)[W], int& slot) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) v += red[slot][i];
    slot ^= 1;
  }
  return v;
}
// 1 / sqrt(v): the hardware's estimate of some 26 bits and two of Newton's steps
__device__ __forceinline__ double inverse_root(double v) {
  const double r0 = __builtin_amdgcn_rsq(v);
  double r = r0 * fma(-0.5 * v * r0, r0, 1.5);
  r = r * fma(-0.5 * v * r, r, 1.5);
  return v > 0.0 && v < __longlong_as_double(0x7ff0000000000000ll) ? r : r0;
}

// h of one piece: the sum, rounded (pairs of elements stay packed)
template <typename T>
__device__ __forceinline__ void add(Piece<T>& x, const Piece<T>& r) {
  constexpr int E = Piece<T>::E;
  float h[E];
#pragma unroll
  for (int e = 0; e < E; ++e) h[e] = x.get(e) + r.get(e);
  x.set(h);
}

// The 8-bit form of a piece at column c (zeros behind the last column).  All lanes of a wavefront are here.
template <typename T>
__device__ __forceinline__ void store_e4m3(const NormArgs& a, int64_t row, int c, const Piece<T>& y) {
  unsigned b;
  const bool in = c < (a.cols + BLOCK - 1) / BLOCK * BLOCK;
  uint8_t* q = a.q + row * a.ldq + c;
  if constexpr (sizeof(T) == 2) {
    b = slimfp8::block_scale<T>(y.v);
    const float sc = __uint_as_float(b << 23);
    const uint2 v = make_uint2(slimfp8::to_e4m3<T>(y.v[0], y.v[1], sc), slimfp8::to_e4m3<T>(y.v[2], y.v[3], sc));
    if (in) *reinterpret_cast<uint2*>(q) = v;
  } else {
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned u = y.v[e] & 0x7fffffffu;
      top = max(top, u < 0x7f800000u ? u : 0u);
    }
    top = max(top, (unsigned)dpp_b32<DPP_XOR1>((int)top));
    top = max(top, (unsigned)dpp_b32<DPP_XOR2>((int)top));
    top = max(top, (unsigned)dpp_b32<DPP_HALF_MIRROR>((int)top));
    top = max(top, (unsigned)dpp_b32<DPP_MIRROR>((int)top));
    const auto both = __builtin_amdgcn_permlane16_swap(top, top, false, false);        // the two rows of 16 lanes of a block
    b = slimfp8::scale_byte(max(both[0], both[1]));
    const float inv = __uint_as_float((254u - b) << 23);      // 1 / s, a power of two of the normal range (b is 1 .. 247)
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = (y.v[e] & 0x7fffffffu) < 0x7f800000u ? __uint_as_float(y.v[e]) * inv : __uint_as_float(0x7fc00000u);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    if (in) *reinterpret_cast<int*>(q) = w;
  }
  if (in && c % BLOCK == 0) a.s[row * a.lds + c / BLOCK] = (uint8_t)b;
}

// W wavefronts per row, P pieces per lane; W == 1: four rows per workgroup
template <typename T, typename TW, int W, int P>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void add_norm_forward(NormArgs a) {
  constexpr int E = Piece<T>::E, LANES = 64 * W, RPW = W == 1 ? 4 : 1;
  __shared__ double red[2][W];
  const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * RPW + (W == 1 ? threadIdx.x >> 6 : 0), step = (int64_t)gridDim.x * RPW;
  const double inv_n = 1.0 / (double)a.cols;
  int slot = 0;
  Piece<T> x[P], r[P];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      x[i].load(static_cast<const T*>(a.X) + row * a.ldx + c, a.cols - c);
      if (a.R) r[i].load(static_cast<const T*>(a.R) + row * a.ldr + c, a.cols - c);
    }
  };
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
    float s = 0.f, mean = 0.f;
    if (a.R)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int c = (i * LANES + lane) * E;
        add(x[i], r[i]);
        if (a.H && c < a.cols) x[i].store(static_cast<T*>(a.H) + row * a.ldh + c, a.cols - c);
      }
    if (!a.rms) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) s += x[i].get(e);
      mean = (float)(row_sum<W>((double)s, red, slot) * inv_n);
      s = 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int left = a.cols - (i * LANES + lane) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = e < left ? x[i].get(e) - mean : 0.f;
        s = fmaf(d, d, s);
      }
    }
    const float rs = (float)inverse_root(fma(row_sum<W>((double)s, red, slot), inv_n, (double)a.eps));
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      float y[E];
      if constexpr (!KEEP) affine(wk[0], bk[0], c);
      const auto& w = wk[KEEP ? i : 0];
      const auto& b = bk[KEEP ? i : 0];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        constexpr int F = Piece<TW>::E;
        const float xh = (x[i].get(e) - mean) * rs;
        y[e] = a.b ? fmaf(xh, w[e / F].get(e % F), b[e / F].get(e % F)) : xh * w[e / F].get(e % F);
        if (e >= a.cols - c) y[e] = 0.f;
      }
      Piece<T> o;
      o.set(y);
      if (a.Y && c < a.cols) o.store(static_cast<T*>(a.Y) + row * a.ldy + c, a.cols - c);
      if (a.q) store_e4m3(a, row, c, o);
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rs;
    }
    if (row + step < a.rows) fetch(row + step);
  }
}

// Rows that the registers of 16 wavefronts do not hold: the pieces are fetched again for every pass, a piece by the same lane each time (so that H
// and Y may take the place of X or R).
template <typename T, typename TW>
__global__ __launch_bounds__(1024) void add_norm_forward_long(NormArgs a) {
  constexpr int E = Piece<T>::E;
  __shared__ double red[2][16];
  int slot = 0;
  const double inv_n = 1.0 / (double)a.cols;
  const int padded = (a.cols + BLOCK - 1) / BLOCK * BLOCK, lane0 = threadIdx.x * E;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    auto sum = [&](int c) {                   // h, from where it still is
      Piece<T> x, r;
      x.load(static_cast<const T*>(a.X) + row * a.ldx + c, a.cols - c);
      if (a.R) {
        r.load(static_cast<const T*>(a.R) + row * a.ldr + c, a.cols - c);
        add(x, r);
      }
      return x;
    };
    auto again = [&](int c) {
      if (!a.H || !a.R) return sum(c);
      Piece<T> h;
      h.load(static_cast<const T*>(a.H) + row * a.ldh + c, a.cols - c);
      return h;
    };
    float s = 0.f;
    for (int c = lane0; c < a.cols; c += 1024 * E) {
      const Piece<T> h = sum(c);
      if (a.H && a.R) h.store(static_cast<T*>(a.H) + row * a.ldh + c, a.cols - c);
      if (!a.rms)
#pragma unroll
        for (int e = 0; e < E; ++e) s += h.get(e);
    }
    float mean = 0.f;
    if (!a.rms) {
      mean = (float)(row_sum<16>((double)s, red, slot) * inv_n);
      s = 0.f;
    }
    for (int c = lane0; c < a.cols; c += 1024 * E) {
      const Piece<T> h = again(c);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = e < a.cols - c ? h.get(e) - mean : 0.f;
        s = fmaf(d, d, s);
      }
    }
    const float rs = (float)inverse_root(fma(row_sum<16>((double)s, red, slot), inv_n, (double)a.eps));
    for (int c = lane0; c - lane0 < padded; c += 1024 * E) {       // (whole wavefronts, for the blocks' maxima)
      const Piece<T> h = again(c);
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y[e] = 0.f;
        if (e < a.cols - c) {
          const float xh = (h.get(e) - mean) * rs, w = value<TW>(a.w, c + e);
          y[e] = a.b ? fmaf(xh, w, value<TW>(a.b, c + e)) : xh * w;
        }
      }
      Piece<T> o;
      o.set(y);
      if (a.Y && c < a.cols) o.store(static_cast<T*>(a.Y) + row * a.ldy + c, a.cols - c);
      if (a.q) store_e4m3(a, row, c, o);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rs;
    }
  }
}

// Workgroups a CU (forward passes, bf16, weight and bias fp32): one piece a lane six (12000 x 1504 27.6 -> 25.8 us, 16384 x 512 13.9 -> 12.7), four pieces
// four (9000 x 8192 115 -> 108, 2100 x 8192 32.5 -> 27.9; fp32 9000 x 4096 112 and 114), between them eight (16384 x 4000 98, with six 102, with five 112).
template <typename T, typename TW>
slim_status forward(slim_ctx* ctx, const NormArgs& a) {
  constexpr int E = Piece<T>::E;
  const int pieces = slim_cdiv(a.cols, E);
  const int64_t many = (int64_t)8 * ctx->num_cus;
  const char* name = "add_norm_forward";
  auto grid = [&](int64_t groups, int per_cu) { return dim3((unsigned)std::min<int64_t>(groups, (int64_t)per_cu * ctx->num_cus)); };
  const bool few = a.rows < many;              // rows that do not fill the chip: more lanes per row
  if (pieces <= 64) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 1, 1>), grid((a.rows + 3) / 4, 6), dim3(256), 0, a);
  else if (pieces <= 256 && (few || pieces > 128)) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 4, 1>), grid(a.rows, 6), dim3(256), 0, a);
  else if (pieces <= 128) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 1, 2>), grid((a.rows + 3) / 4, 8), dim3(256), 0, a);
  else if (pieces <= 512) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 4, 2>), grid(a.rows, 8), dim3(256), 0, a);
  else if (pieces <= 1024) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 4, 4>), grid(a.rows, 4), dim3(256), 0, a);
  else if (pieces <= 2048) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 16, 2>), grid(a.rows, 2), dim3(1024), 0, a);
  else if (pieces <= 4096) SLIM_LAUNCH(ctx, name, (add_norm_forward<T, TW, 16, 4>), grid(a.rows, 2), dim3(1024), 0, a);
  else SLIM_LAUNCH(ctx, name, (add_norm_forward_long<T, TW>), grid(a.rows, 2), dim3(1024), 0, a);
  return SLIM_OK;
}

// (columns are counted in 32 bits, several thousand beyond the last)
slim_status check_columns(slim_ctx* ctx, const char* fn, int cols) {
  return cols <= 1 << 30 ? SLIM_OK : slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: rows of %d numbers are too long", fn, cols);
}

}  // namespace

extern "C" {

slim_status slim_add_norm(slim_ctx* ctx, const void* X, const void* R, slim_dtype x_dtype, int64_t rows, int cols, int64_t ldx, int64_t ldr,
                          const void* w, const void* b, slim_dtype w_dtype, double eps, int rms, void* H, int64_t ldh, void* Y, int64_t ldy,
                          uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, float* mean, float* rstd) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_add_norm";
  if (const slim_status st = check(ctx, fn, x_dtype, w_dtype, rows, cols); st != SLIM_OK) return st;
  if (const slim_status st = check_columns(ctx, fn, cols); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, w, "%s: null weight", fn);
  SLIM_REQUIRE(ctx, eps >= 0.0, "%s: eps = %g", fn, eps);
  SLIM_REQUIRE(ctx, !q == !s && (Y || q || rows == 0), "%s: neither Y nor its 8-bit form, or half of that", fn);
  if (rows == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, X && ldx >= cols && (!R || ldr >= cols) && (!R || !H || ldh >= cols) && (!Y || ldy >= cols),
               "%s: null pointer, or rows shorter than cols (ldx = %lld, ldr = %lld, ldh = %lld, ldy = %lld)", fn, (long long)ldx, (long long)ldr,
               (long long)ldh, (long long)ldy);
  SLIM_REQUIRE(ctx, !q || (slim_aligned16(q) && ldq >= slimfp8::padded(cols) && ldq % BLOCK == 0),
               "%s: q has to be 16-byte aligned, its rows whole blocks of 128 (ldq = %lld)", fn, (long long)ldq);
  SLIM_REQUIRE(ctx, !s || (((uintptr_t)s & 3u) == 0 && lds >= slim_cdiv(cols, BLOCK) && lds % 4 == 0),
               "%s: s has to be 4-byte aligned, its rows whole words (lds = %lld)", fn, (long long)lds);
  NormArgs a = {};
  a.X = X;
  a.R = R;
  a.w = w;
  a.b = b;
  a.H = R ? H : nullptr;                     // (without R the sum is X)
  a.Y = Y;
  a.q = q;
  a.s = s;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldh = ldh;
  a.ldy = ldy;
  a.ldq = ldq;
  a.lds = lds;
  a.mean = rms ? nullptr : mean;
  a.rstd = rstd;
  a.rows = rows;
  a.cols = cols;
  a.eps = (float)eps;
  a.rms = rms != 0;
  return by_type(x_dtype, w_dtype, [&](auto x, auto wt) { return forward<decltype(x), decltype(wt)>(ctx, a); });
}

slim_status slim_add_norm_backward(slim_ctx* ctx, const void* dY, const void* dH, const void* H, slim_dtype x_dtype, int64_t rows, int cols,
                                   int64_t lddy, int64_t lddh, int64_t ldh, const void* w, slim_dtype w_dtype, const float* mean,
                                   const float* rstd, void* dX, int64_t lddx, void* dw, void* db) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_add_norm_backward";
  if (const slim_status st = check_columns(ctx, fn, cols); st != SLIM_OK) return st;
  if (!dH || rows == 0)
    return slim_layer_norm_backward(ctx, dY, H, x_dtype, rows, cols, lddy, ldh, w, w_dtype, mean, rstd, dX, lddx, dw, db);
  NormArgs a = {};
  a.dH = dH;
  a.lddh = lddh;
  if (const slim_status st = check(ctx, fn, x_dtype, w_dtype, rows, cols); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, lddh >= cols, "%s: rows of dH shorter than cols", fn);
  int parts = 0;
  if (const slim_status st = backward_args(ctx, fn, a, dY, H, x_dtype, rows, cols, lddy, ldh, w, mean, rstd, dX, lddx, dw, db, parts); st != SLIM_OK)
    return st;
  return by_type(x_dtype, w_dtype, [&](auto x, auto wt) { return backward<decltype(x), decltype(wt), true>(ctx, a, dw, db, parts); });
}

}  // extern "C"
