// Shared by the norms (norm.hip) and the norms of the residual stream (add_norm.hip): rows in pieces, sums over their wavefronts, and the
// backward pass.
#pragma once

#include "piece_device.h"
#include "slim_internal.h"

namespace slimnorm {
namespace {

using namespace slimdev;

struct NormArgs {
  const void *X, *dY, *w, *b;
  void *Y, *dX;
  int64_t ldx, lddy, ldy, lddx;
  // the residual stream (add_norm.hip): what is added to X and where the sum goes (may be null), the e4m3 form of Y (may be null), and the gradient
  // that reaches the sum past the norm
  const void *R, *dH;
  void* H;
  uint8_t *q, *s;
  int64_t ldr, ldh, ldq, lds, lddh;
  float *mean, *rstd;                    // written by the forward pass (may be null), read by the backward pass
  float *pw, *pb;                        // partial column sums: gridDim x cols
  void *dw, *db;                         // of one workgroup for all rows: the sums themselves
  int64_t rows;
  int cols;
  float eps;
  int rms;
};

// Sums over the W wavefronts of a row (of several rows of W each, with a `red` for each; the barrier is all of theirs).  `slot` alternates
// between calls, so that one barrier per call is enough.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[W][N], int& slot) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum_f32(v[k]);
  if constexpr (W > 1) {
    const int wave = (threadIdx.x >> 6) % W;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) red[slot][wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) s += red[slot][i][k];
      v[k] = s;
    }
    slot ^= 1;
  }
}

// W wavefronts per row, P pieces per lane, G rows at a time; the G shares of dw and db are added in LDS (cols floats each, in turn).
// ADD: dX takes dH too.
template <typename T, typename TW, int W, int P, int G, bool ADD>
__global__ __launch_bounds__(64 * W * G) void norm_backward(NormArgs a) {
  constexpr int E = Piece<T>::E, LANES = 64 * W;
  __shared__ float red[G][2][W][2];
  extern __shared__ float share[];
  const int group = G == 1 ? 0 : threadIdx.x / LANES, lane = G == 1 ? threadIdx.x : threadIdx.x % LANES;
  const float inv_n = 1.f / (float)a.cols;
  int slot = 0;
  float w[P][E], dw[P][E], db[P][E];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = (i * LANES + lane) * E;
#pragma unroll
    for (int k = 0; k < E; k += Piece<TW>::E) {
      Piece<TW> t;
      t.load(static_cast<const TW*>(a.w) + min(c + k, a.cols - 1), a.cols - c - k);
#pragma unroll
      for (int e = 0; e < Piece<TW>::E; ++e) w[i][k + e] = t.get(e);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) dw[i][e] = db[i][e] = 0.f;
  }
  Piece<T> x[P], dy[P], dh[ADD ? P : 1];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      x[i].load(static_cast<const T*>(a.X) + row * a.ldx + c, a.cols - c);
      dy[i].load(static_cast<const T*>(a.dY) + row * a.lddy + c, a.cols - c);
      if constexpr (ADD) dh[i].load(static_cast<const T*>(a.dH) + row * a.lddh + c, a.cols - c);
    }
  };
  // (a group without a row in the last round goes through it with what it has, and keeps nothing of it)
  const int64_t first = (int64_t)blockIdx.x * G + group, step = (int64_t)gridDim.x * G;
  fetch(min(first, a.rows - 1));
  for (int64_t row0 = (int64_t)blockIdx.x * G; row0 < a.rows; row0 += step) {
    const int64_t row = row0 + group;
    const bool live = G == 1 || row < a.rows;
    const int64_t at = live ? row : a.rows - 1;
    const float mean = a.mean ? a.mean[at] : 0.f, r = a.rstd[at];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = live ? dy[i].get(e) : 0.f, xh = (x[i].get(e) - mean) * r, g = d * w[i][e];     // (behind the last column d is 0)
        s[0] += g;
        s[1] = fmaf(g, xh, s[1]);
        if (live) dw[i][e] = fmaf(d, xh, dw[i][e]);
        db[i][e] += d;
      }
    row_sums<W, 2>(s, red[group], slot);
    const float mg = a.rms ? 0.f : s[0] * inv_n, mgx = s[1] * inv_n;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      if (c >= a.cols || !live) break;
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = (x[i].get(e) - mean) * r;
        o[e] = r * (fmaf(dy[i].get(e), w[i][e], -mg) - xh * mgx);
        if constexpr (ADD) o[e] += dh[i].get(e);
      }
      Piece<T> p;
      p.set(o);
      p.store(static_cast<T*>(a.dX) + row * a.lddx + c, a.cols - c);
    }
    if (row0 + step < a.rows) fetch(min(row + step, a.rows - 1));
  }
  auto columns = [&](auto use) {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (i * LANES + lane) * E + e;
        if (c < a.cols) use(c, dw[i][e], db[i][e]);
      }
  };
#pragma unroll
  for (int g = 1; g < G; ++g) {
    if (g > 1) __syncthreads();
    if (group == g) columns([&](int c, float& p, float& q) {
      share[c] = p;
      if (a.pb || a.db) share[a.cols + c] = q;
    });
    __syncthreads();
    if (group == 0) columns([&](int c, float& p, float& q) {
      p += share[c];
      if (a.pb || a.db) q += share[a.cols + c];
    });
  }
  if (group != 0) return;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = (i * LANES + lane) * E, left = a.cols - c;
    if (left <= 0) break;
    if (a.dw) {
      put_run<TW, E>(a.dw, c, left, dw[i]);
      if (a.db) put_run<TW, E>(a.db, c, left, db[i]);
    } else {
      put_run<float, E>(a.pw + (int64_t)blockIdx.x * a.cols, c, left, dw[i]);
      if (a.pb) put_run<float, E>(a.pb + (int64_t)blockIdx.x * a.cols, c, left, db[i]);
    }
  }
}

// Rows that no group of wavefronts holds (norm.hip)
template <typename T, typename TW, bool ADD>
__global__ __launch_bounds__(1024) void norm_backward_long(NormArgs a) {
  __shared__ float red[2][16][2];
  int slot = 0;
  const float inv_n = 1.f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.mean ? a.mean[row] : 0.f, r = a.rstd[row];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float g = value<T>(a.dY, row * a.lddy + c) * value<TW>(a.w, c), xh = (value<T>(a.X, row * a.ldx + c) - mean) * r;
      s[0] += g;
      s[1] = fmaf(g, xh, s[1]);
    }
    row_sums<16, 2>(s, red, slot);
    const float mg = a.rms ? 0.f : s[0] * inv_n, mgx = s[1] * inv_n;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float g = value<T>(a.dY, row * a.lddy + c) * value<TW>(a.w, c), xh = (value<T>(a.X, row * a.ldx + c) - mean) * r;
      float o = r * (g - mg - xh * mgx);
      if constexpr (ADD) o += value<T>(a.dH, row * a.lddh + c);
      put<T>(a.dX, row * a.lddx + c, o);
    }
  }
}
template <typename T>
__global__ __launch_bounds__(256) void norm_columns(NormArgs a, int64_t per) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float dw = 0.f, db = 0.f;
  for (int64_t row = r0; row < r1; ++row) {
    const float d = value<T>(a.dY, row * a.lddy + c);
    dw = fmaf(d, (value<T>(a.X, row * a.ldx + c) - (a.mean ? a.mean[row] : 0.f)) * a.rstd[row], dw);
    db += d;
  }
  a.pw[(int64_t)blockIdx.y * a.cols + c] = dw;
  if (a.pb) a.pb[(int64_t)blockIdx.y * a.cols + c] = db;
}

// dw, db: the sums of the workgroups' shares; 32 columns x 32 ranges of workgroups, a range's rows eight at a time so that their loads are
// under way together.  Eight by a tree in fp32, the rest in fp64: hundreds one after another in fp32 were 2.3e-7 off at 3001 x 1501.
template <typename TW>
__global__ __launch_bounds__(1024) void norm_join(const float* __restrict__ pw, const float* __restrict__ pb, int parts, int cols,
                                                  void* dw, void* db) {
  __shared__ double red[32][33];
  const int x = threadIdx.x & 31, c = blockIdx.x * 32 + x, k = threadIdx.x >> 5;
  const float* p = (blockIdx.y ? pb : pw) + min(c, cols - 1);
  const int per = (parts + 31) / 32, i0 = k * per, i1 = min(parts, i0 + per);
  double s = 0.0;
  for (int i = i0; i < i1; i += 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j < i1 ? p[(int64_t)(i + j) * cols] : 0.f;
    s += (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
  }
  red[k][x] = s;
  __syncthreads();
  if (k == 0 && c < cols) {
    double t[4] = {};
#pragma unroll
    for (int i = 1; i < 32; ++i) t[i & 3] += red[i][x];
    s += (t[0] + t[1]) + (t[2] + t[3]);
    put<TW>(blockIdx.y ? db : dw, c, (float)s);
  }
}

// Wavefronts per row, pieces per lane, rows at a time, and workgroups per CU of the backward pass: as many wavefronts as hide the loads, and no
// more partial sums than that takes.  With the forward pass: 16384 x 4096 bf16, one row at a time, three workgroups per CU 128 us, two 135,
// two rows at a time 142 (too few registers); 3001 x 1501 fp32 the other way, 28.5 (four) and 26.0; 30000 x 640 bf16 one wavefront per row 52,
// four 68.
// With a gradient that joins dX (`add`) two workgroups per CU: 16384 x 4096 bf16 one row at a time, forward and backward, two 216, three 220.
// Up to four rounds of rows: one workgroup, which needs no second kernel (52 x 64: 24 -> 20 us with the forward pass, most of it the host's).
struct Shape {
  int w, p, g, per_cu;
};
Shape shape_of(int64_t rows, int cols, int e, bool add) {
  const int pieces = slim_cdiv(cols, e);
  if (pieces <= 64) return rows <= 64 ? Shape{1, 1, 16, 0} : Shape{1, 1, 4, 4};
  if (pieces <= 128) return rows <= 32 ? Shape{1, 2, 8, 0} : Shape{1, 2, 4, 3};
  if (pieces <= 256) return rows <= 16 ? Shape{4, 1, 4, 0} : Shape{4, 1, 2, 2};
  if (add && pieces > 256 && pieces <= 512 && rows > 8 && e == 8) return {4, 2, 1, 2};
  if (pieces <= 512) return rows <= 8 ? Shape{4, 2, 2, 0} : e == 8 ? Shape{4, 2, 1, 3} : Shape{4, 2, 2, 2};
  if (pieces <= 1024) return {8, 2, 1, rows <= 4 ? 0 : 2};
  if (pieces <= 2048) return {16, 2, 1, rows <= 4 ? 0 : 1};
  return {0, 0, 1, 2};
}
// workgroups, and with them partial sums, of the backward pass; 0: one for all rows, without partial sums
int parts_of(int64_t rows, int cols, slim_dtype d, int ncu, bool add) {
  const Shape s = shape_of(rows, cols, d == SLIM_F32 ? 4 : 8, add);
  return (int)std::min<int64_t>((rows + s.g - 1) / s.g, (int64_t)s.per_cu * ncu);
}

template <typename T, typename TW, bool ADD = false>
slim_status backward(slim_ctx* ctx, const NormArgs& a, void* dw, void* db, int parts) {
  const Shape s = shape_of(a.rows, a.cols, Piece<T>::E, ADD);
  const char* name = "norm_backward";
  const dim3 grid(std::max(1, parts)), block(64 * s.w * s.g);
  const size_t smem = s.g > 1 ? sizeof(float) * (db ? 2 : 1) * (size_t)a.cols : 0;
  switch (s.w * 1000 + s.p * 100 + s.g) {
    case 1104: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 1, 4, ADD>), grid, block, smem, a); break;
    case 1116: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 1, 16, ADD>), grid, block, smem, a); break;
    case 1204: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 2, 4, ADD>), grid, block, smem, a); break;
    case 1208: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 2, 8, ADD>), grid, block, smem, a); break;
    case 4102: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 1, 2, ADD>), grid, block, smem, a); break;
    case 4104: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 1, 4, ADD>), grid, block, smem, a); break;
    case 4201:
      if constexpr (Piece<T>::E == 8) SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 2, 1, ADD>), grid, block, smem, a);
      break;
    case 4202: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 2, 2, ADD>), grid, block, smem, a); break;
    case 8201: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 8, 2, 1, ADD>), grid, block, smem, a); break;
    case 16201: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 16, 2, 1, ADD>), grid, block, smem, a); break;
    default:
      // (the columns first: dX may take the place of dY or X, which both kernels read)
      SLIM_LAUNCH(ctx, "norm_columns", norm_columns<T>, dim3(slim_cdiv(a.cols, 256), parts), dim3(256), 0, a, (a.rows + parts - 1) / parts);
      SLIM_LAUNCH(ctx, name, (norm_backward_long<T, TW, ADD>), grid, dim3(1024), 0, a);
  }
  if (parts == 0) return SLIM_OK;
  SLIM_LAUNCH(ctx, "norm_join", norm_join<TW>, dim3(slim_cdiv(a.cols, 32), db ? 2 : 1), dim3(1024), 0, a.pw, a.pb, parts, a.cols, dw, db);
  return SLIM_OK;
}

bool is_float(slim_dtype d) { return d == SLIM_F16 || d == SLIM_BF16 || d == SLIM_F32; }

template <typename F>
slim_status by_type(slim_dtype x, slim_dtype w, F f) {
  if (x == SLIM_F32) return f(float(), float());
  if (x == SLIM_F16) return w == SLIM_F32 ? f(__half(), float()) : f(__half(), __half());
  return w == SLIM_F32 ? f(__hip_bfloat16(), float()) : f(__hip_bfloat16(), __hip_bfloat16());
}

slim_status check(slim_ctx* ctx, const char* fn, slim_dtype x, slim_dtype w, int64_t rows, int cols) {
  if (!is_float(x)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: X is F16, BF16 or F32", fn);
  if (w != x && w != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: weight and bias are of the type of X or F32", fn);
  SLIM_REQUIRE(ctx, rows >= 0 && cols > 0, "%s: rows = %lld, cols = %d", fn, (long long)rows, cols);
  return SLIM_OK;
}

// The backward pass's checks, arguments and workspace; parts: workgroups that leave partial column sums
slim_status backward_args(slim_ctx* ctx, const char* fn, NormArgs& a, const void* dY, const void* X, slim_dtype x_dtype, int64_t rows, int cols,
                          int64_t lddy, int64_t ldx, const void* w, const float* mean, const float* rstd, void* dX, int64_t lddx, void* dw,
                          void* db, int& parts) {
  SLIM_REQUIRE(ctx, w && dw, "%s: null weight or dw", fn);
  SLIM_REQUIRE(ctx, rows == 0 || (dY && X && dX && rstd && lddy >= cols && ldx >= cols && lddx >= cols),
               "%s: null pointer, or rows shorter than cols", fn);
  parts = rows ? parts_of(rows, cols, x_dtype, ctx->num_cus, a.dH != nullptr) : 0;
  if (const slim_status st = slim_ws_reserve(ctx, slim_layer_norm_backward_workspace(rows, cols, x_dtype, db != nullptr, ctx->num_cus)); st != SLIM_OK)
    return st;
  a.X = X;
  a.dY = dY;
  a.w = w;
  a.dX = dX;
  a.ldx = ldx;
  a.lddy = lddy;
  a.lddx = lddx;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.rows = rows;
  a.cols = cols;
  a.rms = mean == nullptr;
  if (parts > 0) {
    a.pw = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)parts * cols));
    a.pb = db ? static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)parts * cols)) : nullptr;
    if (!a.pw || (db && !a.pb)) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
  } else if (rows > 0) {
    a.dw = dw;
    a.db = db;
  }
  return SLIM_OK;
}

}  // namespace
}  // namespace slimnorm
