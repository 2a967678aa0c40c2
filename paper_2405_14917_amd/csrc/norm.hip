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
#include "slim_device.h"
#include "slim_internal.h"

namespace {

using namespace slimdev;

struct NormArgs {
  const void *X, *dY, *w, *b;
  void *Y, *dX;
  int64_t ldx, lddy, ldy, lddx;
  float *mean, *rstd;                    // written by the forward pass (may be null), read by the backward pass
  float *pw, *pb;                        // partial column sums: gridDim x cols
  void *dw, *db;                         // of one workgroup for all rows: the sums themselves
  int64_t rows;
  int cols;
  float eps;
  int rms;
};

template <typename T>
struct Elem;
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float widen(unsigned short v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ unsigned short narrow(float v) { return __builtin_bit_cast(unsigned short, (_Float16)v); }
};
template <>
struct Elem<__hip_bfloat16> {
  static __device__ __forceinline__ float widen(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
  static __device__ __forceinline__ unsigned short narrow(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
};

// A piece: 16 bytes of a row (4 or 8 elements)
template <typename T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  unsigned v[4];
  // from p on, of which `left` elements exist (the others are zero); p is aligned to its type only
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= E) {
      __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = 0u;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < left) v[i] = reinterpret_cast<const unsigned*>(p)[i];
      } else {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) v[i / 2] |= (unsigned)q[i] << (16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return Elem<T>::widen((unsigned short)(v[i / 2] >> (16 * (i & 1))));
  }
  __device__ __forceinline__ void set(const float (&f)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
      else v[i] = (unsigned)Elem<T>::narrow(f[2 * i]) | (unsigned)Elem<T>::narrow(f[2 * i + 1]) << 16;
    }
  }
  __device__ __forceinline__ void store(T* p, int left) const {
    if (left >= E) {
      store16_once(p, v);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) reinterpret_cast<unsigned*>(p)[i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(v[i / 2] >> (16 * (i & 1)));
    }
  }
};

template <typename T>
__device__ __forceinline__ float value(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 4) return static_cast<const float*>(p)[i];
  else return Elem<T>::widen(static_cast<const unsigned short*>(p)[i]);
}
template <typename T>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
  if constexpr (sizeof(T) == 4) static_cast<float*>(p)[i] = v;
  else static_cast<unsigned short*>(p)[i] = Elem<T>::narrow(v);
}

// E values one after another, of which `left` are wanted (as single stores, a lane's E apart, 16384 columns took 15 us)
template <typename T, int E>
__device__ __forceinline__ void put_run(void* p, int c, int left, const float (&f)[E]) {
  if (left >= E) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(static_cast<float*>(p) + c, f, sizeof(f));
    } else {
      unsigned short h[E];
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = Elem<T>::narrow(f[e]);
      __builtin_memcpy(static_cast<unsigned short*>(p) + c, h, sizeof(h));
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < left) put<T>(p, c + e, f[e]);
  }
}

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

// W wavefronts per row, P pieces per lane, G rows at a time; the G shares of dw and db are added in LDS (cols floats each, in turn)
template <typename T, typename TW, int W, int P, int G>
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
  Piece<T> x[P], dy[P];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = (i * LANES + lane) * E;
      x[i].load(static_cast<const T*>(a.X) + row * a.ldx + c, a.cols - c);
      dy[i].load(static_cast<const T*>(a.dY) + row * a.lddy + c, a.cols - c);
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
      put<T>(a.dX, row * a.lddx + c, r * (g - mg - xh * mgx));
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
// Up to four rounds of rows: one workgroup, which needs no second kernel (52 x 64: 24 -> 20 us with the forward pass, most of it the host's).
struct Shape {
  int w, p, g, per_cu;
};
Shape shape_of(int64_t rows, int cols, int e) {
  const int pieces = slim_cdiv(cols, e);
  if (pieces <= 64) return rows <= 64 ? Shape{1, 1, 16, 0} : Shape{1, 1, 4, 4};
  if (pieces <= 128) return rows <= 32 ? Shape{1, 2, 8, 0} : Shape{1, 2, 4, 3};
  if (pieces <= 256) return rows <= 16 ? Shape{4, 1, 4, 0} : Shape{4, 1, 2, 2};
  if (pieces <= 512) return rows <= 8 ? Shape{4, 2, 2, 0} : e == 8 ? Shape{4, 2, 1, 3} : Shape{4, 2, 2, 2};
  if (pieces <= 1024) return {8, 2, 1, rows <= 4 ? 0 : 2};
  if (pieces <= 2048) return {16, 2, 1, rows <= 4 ? 0 : 1};
  return {0, 0, 1, 2};
}
// workgroups, and with them partial sums, of the backward pass; 0: one for all rows, without partial sums
int parts_of(int64_t rows, int cols, slim_dtype d, int ncu) {
  const Shape s = shape_of(rows, cols, d == SLIM_F32 ? 4 : 8);
  return (int)std::min<int64_t>((rows + s.g - 1) / s.g, (int64_t)s.per_cu * ncu);
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

template <typename T, typename TW>
slim_status backward(slim_ctx* ctx, const NormArgs& a, void* dw, void* db, int parts) {
  const Shape s = shape_of(a.rows, a.cols, Piece<T>::E);
  const char* name = "norm_backward";
  const dim3 grid(std::max(1, parts)), block(64 * s.w * s.g);
  const size_t smem = s.g > 1 ? sizeof(float) * (db ? 2 : 1) * (size_t)a.cols : 0;
  switch (s.w * 1000 + s.p * 100 + s.g) {
    case 1104: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 1, 4>), grid, block, smem, a); break;
    case 1116: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 1, 16>), grid, block, smem, a); break;
    case 1204: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 2, 4>), grid, block, smem, a); break;
    case 1208: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 1, 2, 8>), grid, block, smem, a); break;
    case 4102: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 1, 2>), grid, block, smem, a); break;
    case 4104: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 1, 4>), grid, block, smem, a); break;
    case 4201:
      if constexpr (Piece<T>::E == 8) SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 2, 1>), grid, block, smem, a);
      break;
    case 4202: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 4, 2, 2>), grid, block, smem, a); break;
    case 8201: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 8, 2, 1>), grid, block, smem, a); break;
    case 16201: SLIM_LAUNCH(ctx, name, (norm_backward<T, TW, 16, 2, 1>), grid, block, smem, a); break;
    default:
      // (the columns first: dX may take the place of dY or X, which both kernels read)
      SLIM_LAUNCH(ctx, "norm_columns", norm_columns<T>, dim3(slim_cdiv(a.cols, 256), parts), dim3(256), 0, a, (a.rows + parts - 1) / parts);
      SLIM_LAUNCH(ctx, name, (norm_backward_long<T, TW>), grid, dim3(1024), 0, a);
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

}  // namespace

extern "C" {

size_t slim_layer_norm_backward_workspace(int64_t rows, int cols, slim_dtype x_dtype, int bias, int num_cus) {
  if (rows <= 0 || cols <= 0) return 0;
  const size_t one = slim_ws_round(sizeof(float) * (size_t)parts_of(rows, cols, x_dtype, num_cus > 0 ? num_cus : 256) * cols);
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
  SLIM_REQUIRE(ctx, w && dw, "%s: null weight or dw", fn);
  SLIM_REQUIRE(ctx, rows == 0 || (dY && X && dX && rstd && lddy >= cols && ldx >= cols && lddx >= cols),
               "%s: null pointer, or rows shorter than cols", fn);
  const int parts = rows ? parts_of(rows, cols, x_dtype, ctx->num_cus) : 0;
  if (const slim_status st = slim_ws_reserve(ctx, slim_layer_norm_backward_workspace(rows, cols, x_dtype, db != nullptr, ctx->num_cus)); st != SLIM_OK)
    return st;
  NormArgs a = {};
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
  if (rows > 0) {
    if (parts > 0) {
      a.pw = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)parts * cols));
      a.pb = db ? static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)parts * cols)) : nullptr;
      if (!a.pw || (db && !a.pb)) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
    } else {
      a.dw = dw;
      a.db = db;
    }
    return by_type(x_dtype, w_dtype, [&](auto x, auto wt) { return backward<decltype(x), decltype(wt)>(ctx, a, dw, db, parts); });
  }
  // no rows: the sums are zero
  return by_type(x_dtype, w_dtype, [&](auto, auto wt) {
    SLIM_LAUNCH(ctx, "norm_join", norm_join<decltype(wt)>, dim3(slim_cdiv(cols, 32), db ? 2 : 1), dim3(1024), 0, a.pw, a.pb, 0, cols, dw, db);
    return SLIM_OK;
  });
}

}  // extern "C"
