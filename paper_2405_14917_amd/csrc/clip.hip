// The norm of many tensors together, and their scaling to a limit: n = sqrt(sum of all squares), g <- g min(1, limit / n).
//
// Bound by memory: everything is read twice, since the factor depends on all of it, and written once.  The tensors are one row of chunks of
// 16 KiB; a launch takes up to 60 tensors (their addresses are its arguments, so that a captured call needs no table in memory).  First kernel:
// a workgroup takes chunks blockIdx, blockIdx + gridDim, ... and leaves one sum of squares, in fp64: no square of an fp32 or bf16 number leaves its
// range, and 10^9 of them added one after another in fp32 would lose their digits.  Second kernel: every workgroup adds these sums, in their
// order, and scales its chunks, the last ones first: the end of what the first kernel read is still in the cache behind the L2.
#include <memory>

#include "piece_device.h"
#include "slim_internal.h"

namespace {

using namespace slimnorm;

// Three workgroups a CU, four pieces a lane: what is under way together is enough, and more of it costs the memory its pages (two matrices' layers of
// 4096 x 11008 and the like, 810 MB: 414 us; two workgroups a CU 424, four 421, eight 448; eight pieces and two workgroups 424).
constexpr int CL_TENSORS = 60, CL_THREADS = 256, CL_PIECES = 4, CL_BYTES = 16 * CL_THREADS * CL_PIECES, CL_PER_CU = 3;

struct ClipTensor {
  const void* in;
  void* out;
  int64_t n, cols, ldi, ldo;             // elements; ldi == ldo == 0: one after another
  int64_t first;                         // chunks in front of it
  int dtype;
};
struct ClipArgs {
  ClipTensor t[CL_TENSORS];
  int count;
  int64_t chunks;
};
static_assert(sizeof(ClipArgs) <= 4096 - 64, "the arguments of a launch");

// The tensor of a chunk (the same in every lane): `first` is what lane l holds of tensor l.  (A search by halves is a chain of loads of the arguments.)
__device__ __forceinline__ int64_t first_of_lane(const ClipArgs& a) {
  const int lane = threadIdx.x & 63;
  return lane < a.count ? a.t[lane].first : INT64_MAX;
}
__device__ __forceinline__ int tensor_of(int64_t first, int64_t chunk) {
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= chunk)) - 1);
}
static_assert(CL_TENSORS <= 64, "a lane for every tensor");

template <typename T, typename F>
__device__ __forceinline__ void each_element(const ClipTensor& t, int64_t e0, F use) {
  for (int i = threadIdx.x; i < CL_BYTES / (int)sizeof(T); i += CL_THREADS) {
    const int64_t e = e0 + i;
    if (e >= t.n) break;
    const int64_t row = e / t.cols, col = e - row * t.cols;
    use(row * t.ldi + col, row * t.ldo + col);
  }
}

template <typename T>
__device__ __forceinline__ double squares(const ClipTensor& t, int64_t chunk) {
  constexpr int E = Piece<T>::E;
  const int64_t e0 = chunk * (CL_BYTES / (int64_t)sizeof(T));
  double s = 0.0;
  if (t.ldi == 0) {
    Piece<T> p[CL_PIECES];
    const T* in = static_cast<const T*>(t.in) + e0;
    const int64_t left = t.n - e0;
#pragma unroll
    for (int i = 0; i < CL_PIECES; ++i) {
      const int c = (i * CL_THREADS + threadIdx.x) * E;
      p[i].load(in + c, (int)min((int64_t)E, left - c));
    }
#pragma unroll
    for (int i = 0; i < CL_PIECES; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double v = (double)p[i].get(e);
        s = fma(v, v, s);
      }
  } else {
    each_element<T>(t, e0, [&](int64_t i, int64_t) {
      const double v = (double)value<T>(t.in, i);
      s = fma(v, v, s);
    });
  }
  return s;
}

// A factor below 1 in two fp32 parts and, where fp32 has no room for it (gradients of 1e38 and a limit of 1e-6, say), an exponent: a product is rounded once
// to fp32.  (In fp64 204 MB in fp16 took 158 us in place of 97, 810 MB in bf16 439 in place of 410.)
struct Factor {
  float hi, lo;
  int exponent;
  __device__ explicit Factor(double f) {
    exponent = 0;
    if (f < 0x1p-64) f = frexp(f, &exponent);
    hi = (float)f;
    lo = (float)(f - (double)hi);
  }
  __device__ __forceinline__ float times(float v) const { return ldexpf(fmaf(v, hi, v * lo), exponent); }
};

template <typename T>
__device__ __forceinline__ void scale(const ClipTensor& t, int64_t chunk, const Factor& factor, bool copy) {
  constexpr int E = Piece<T>::E;
  const int64_t e0 = chunk * (CL_BYTES / (int64_t)sizeof(T));
  if (t.ldi == 0) {
    Piece<T> p[CL_PIECES];
    const T* in = static_cast<const T*>(t.in) + e0;
    T* out = static_cast<T*>(t.out) + e0;
    const int64_t left = t.n - e0;
#pragma unroll
    for (int i = 0; i < CL_PIECES; ++i) {
      const int c = (i * CL_THREADS + threadIdx.x) * E;
      p[i].load(in + c, (int)min((int64_t)E, left - c));
    }
#pragma unroll
    for (int i = 0; i < CL_PIECES; ++i) {
      const int c = (i * CL_THREADS + threadIdx.x) * E;
      if (!copy) {
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = factor.times(p[i].get(e));
        p[i].set(f);
      }
      p[i].store(out + c, (int)min((int64_t)E, left - c));
    }
  } else {
    each_element<T>(t, e0, [&](int64_t i, int64_t o) {
      if (copy) static_cast<T*>(t.out)[o] = static_cast<const T*>(t.in)[i];
      else put<T>(t.out, o, factor.times(value<T>(t.in, i)));
    });
  }
}

__global__ __launch_bounds__(CL_THREADS) void clip_squares(ClipArgs a, double* __restrict__ sums) {
  __shared__ double red[CL_THREADS / 64];
  const int64_t first = first_of_lane(a);
  double s = 0.0;
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const ClipTensor& t = a.t[tensor_of(first, chunk)];
    const int64_t c = chunk - t.first;
    s += t.dtype == SLIM_F32 ? squares<float>(t, c) : t.dtype == SLIM_F16 ? squares<__half>(t, c) : squares<__hip_bfloat16>(t, c);
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(CL_THREADS) void clip_scale(ClipArgs a, const double* __restrict__ sums, int parts, double limit, float* norm) {
  __shared__ double red[CL_THREADS / 64];
  const int64_t first = first_of_lane(a);
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += CL_THREADS) s += sums[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  const double n = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  // a norm that is no finite fp32 number leaves everything as it is: the caller sees it and drops the step
  const bool copy = !(n > limit) || !((float)n < __builtin_inff());
  const Factor factor(copy ? 1.0 : limit / n);
  for (int64_t k = blockIdx.x; k < a.chunks; k += gridDim.x) {
    const int64_t chunk = a.chunks - 1 - k;
    const ClipTensor& t = a.t[tensor_of(first, chunk)];
    if (copy && t.in == t.out) continue;
    const int64_t c = chunk - t.first;
    if (t.dtype == SLIM_F32) scale<float>(t, c, factor, copy);
    else if (t.dtype == SLIM_F16) scale<__half>(t, c, factor, copy);
    else scale<__hip_bfloat16>(t, c, factor, copy);
  }
}

int64_t elements(const slim_tensor& t) { return t.rows * t.cols; }
int64_t chunks_of(const slim_tensor& t) {
  const int64_t per = CL_BYTES / (t.dtype == SLIM_F32 ? 4 : 2);
  return (elements(t) + per - 1) / per;
}

slim_status check(slim_ctx* ctx, const char* fn, const slim_tensor* t, int count) {
  SLIM_REQUIRE(ctx, count >= 0 && (t || count == 0), "%s: null list of %d tensors", fn, count);
  for (int i = 0; i < count; ++i) {
    SLIM_REQUIRE(ctx, t[i].rows >= 0 && t[i].cols >= 0, "%s: tensor %d is %lld x %lld", fn, i, (long long)t[i].rows, (long long)t[i].cols);
    SLIM_REQUIRE(ctx, t[i].cols == 0 || t[i].rows <= (INT64_MAX >> 8) / t[i].cols, "%s: tensor %d is %lld x %lld", fn, i, (long long)t[i].rows,
                 (long long)t[i].cols);
    if (elements(t[i]) == 0) continue;
    SLIM_REQUIRE(ctx, t[i].data && (t[i].rows == 1 || (t[i].ld >= t[i].cols && t[i].ld <= (INT64_MAX >> 8) / t[i].rows)),
                 "%s: null tensor %d, or rows that overlap (ld = %lld)", fn, i, (long long)t[i].ld);
    if (t[i].dtype != SLIM_F16 && t[i].dtype != SLIM_BF16 && t[i].dtype != SLIM_F32)
      return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: tensor %d is not F16, BF16 or F32", fn, i);
  }
  return SLIM_OK;
}

// A tensor's bytes: rows of `width`, `step` apart (no less)
struct Span {
  uintptr_t begin, end, step, width;
  int64_t rows;
  int index;
  bool written;
};
Span span_of(const slim_tensor& t, int index, bool written) {
  const uintptr_t size = t.dtype == SLIM_F32 ? 4 : 2, begin = reinterpret_cast<uintptr_t>(t.data);
  const bool dense = t.rows == 1 || t.ld == t.cols;
  const uintptr_t width = (uintptr_t)(dense ? elements(t) : t.cols) * size, step = dense ? width : (uintptr_t)t.ld * size;
  const int64_t rows = dense ? 1 : t.rows;
  return {begin, begin + (uintptr_t)(rows - 1) * step + width, step, width, rows, index, written};
}
// whether any row of b meets one of a, which begins no later: of a's rows that begin before the end of a row of b the last one reaches farthest.  With
// one step b's first row tells; else the rows of the one with fewer are gone through.
bool meet(const Span& a, const Span& b) {
  auto row_meets = [](const Span& s, uintptr_t from, uintptr_t to) {
    if (to <= s.begin) return false;
    const uintptr_t k = std::min<uintptr_t>((uintptr_t)s.rows - 1, (to - 1 - s.begin) / s.step);
    return s.begin + k * s.step + s.width > from;
  };
  if (b.begin >= a.end) return false;
  if (a.step == b.step) return row_meets(a, b.begin, b.begin + b.width);
  const Span &few = a.rows < b.rows ? a : b, &many = a.rows < b.rows ? b : a;
  for (int64_t i = 0; i < few.rows; ++i)
    if (row_meets(many, few.begin + (uintptr_t)i * few.step, few.begin + (uintptr_t)i * few.step + few.width)) return true;
  return false;
}
// Workgroups read and write in no order: an output is its own input, or in memory that nothing else here lies in.
slim_status check_outputs(slim_ctx* ctx, const char* fn, const slim_tensor* in, const slim_tensor* out, int count) {
  const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[2 * (size_t)count + 1]);
  if (!spans) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: host memory", fn);
  Span* end = spans.get();
  for (int i = 0; i < count; ++i) {
    if (elements(out[i]) == 0) continue;
    *end++ = span_of(out[i], i, true);
    if (in != out && !(in[i].data == out[i].data && (in[i].rows == 1 || in[i].ld == out[i].ld))) *end++ = span_of(in[i], i, false);
  }
  std::sort(spans.get(), end, [](const Span& a, const Span& b) { return a.begin < b.begin; });
  for (const Span* a = spans.get(); a != end; ++a)
    for (const Span* b = a + 1; b != end && b->begin < a->end; ++b)
      if ((a->written || b->written) && meet(*a, *b)) {
        const Span &w = a->written ? *a : *b, &o = &w == a ? *b : *a;
        SLIM_REQUIRE(ctx, false, o.written ? "%s: outputs %d and %d overlap" : "%s: output %d overlaps input %d", fn, w.index, o.index);
      }
  return SLIM_OK;
}

int grid_of(int64_t chunks, int ncu) { return (int)std::max<int64_t>(1, std::min<int64_t>(chunks, (int64_t)CL_PER_CU * ncu)); }
size_t need(int count, int ncu) { return slim_ws_round(sizeof(double) * (size_t)std::max(1, slim_cdiv(count, CL_TENSORS)) * CL_PER_CU * ncu); }

// the tensors from `at` on as arguments of one launch; returns the first one that did not fit
int fill(ClipArgs& a, const slim_tensor* in, const slim_tensor* out, int at, int count) {
  a.count = 0;
  a.chunks = 0;
  for (; at < count && a.count < CL_TENSORS; ++at) {
    if (elements(in[at]) == 0) continue;
    const slim_tensor &t = in[at], &o = out ? out[at] : in[at];
    ClipTensor& c = a.t[a.count++];
    c.in = t.data;
    c.out = o.data;
    c.n = elements(t);
    c.cols = t.cols;
    const bool dense = t.rows == 1 || (t.ld == t.cols && o.ld == o.cols);
    c.ldi = dense ? 0 : t.ld;
    c.ldo = dense ? 0 : o.ld;
    c.first = a.chunks;
    c.dtype = (int)t.dtype;
    a.chunks += chunks_of(t);
  }
  return at;
}

slim_status norm_and_scale(slim_ctx* ctx, const char* fn, const slim_tensor* in, const slim_tensor* out, int count, double limit, float* norm) {
  if (const slim_status st = slim_ws_reserve(ctx, need(count, ctx->num_cus)); st != SLIM_OK) return st;
  double* sums = static_cast<double*>(slim_ws_alloc(ctx, need(count, ctx->num_cus)));
  if (!sums) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
  ClipArgs a;
  int parts = 0;
  for (int at = 0; at < count;) {
    at = fill(a, in, out, at, count);
    if (a.count == 0) break;
    const int grid = grid_of(a.chunks, ctx->num_cus);
    SLIM_LAUNCH(ctx, "clip_squares", clip_squares, dim3(grid), dim3(CL_THREADS), 0, a, sums + parts);
    parts += grid;
  }
  if (!out) {
    a.count = 0;
    a.chunks = 0;
    SLIM_LAUNCH(ctx, "clip_scale", clip_scale, dim3(1), dim3(CL_THREADS), 0, a, sums, parts, limit, norm);
    return SLIM_OK;
  }
  for (int at = 0; at < count || norm;) {
    if (at > 0 || count > CL_TENSORS || parts == 0) at = fill(a, in, out, at, count);
    else at = count;                          // (one launch: the arguments are there)
    SLIM_LAUNCH(ctx, "clip_scale", clip_scale, dim3(grid_of(a.chunks, ctx->num_cus)), dim3(CL_THREADS), 0, a, sums, parts, limit, norm);
    norm = nullptr;
  }
  return SLIM_OK;
}

}  // namespace

extern "C" {

size_t slim_grad_norm_workspace(int count, int num_cus) { return count < 0 ? 0 : need(count, num_cus > 0 ? num_cus : 256); }

slim_status slim_grad_norm(slim_ctx* ctx, const slim_tensor* tensors, int count, float* norm) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_grad_norm";
  if (const slim_status st = check(ctx, fn, tensors, count); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, norm, "%s: null norm", fn);
  return norm_and_scale(ctx, fn, tensors, nullptr, count, 0.0, norm);
}

slim_status slim_clip_gradients(slim_ctx* ctx, const slim_tensor* tensors, const slim_tensor* out, int count, double limit, float* norm) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_clip_gradients";
  if (const slim_status st = check(ctx, fn, tensors, count); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, norm, "%s: null norm", fn);
  SLIM_REQUIRE(ctx, limit >= 0.0, "%s: limit = %g", fn, limit);
  if (!out) out = tensors;
  if (const slim_status st = check(ctx, fn, out, count); st != SLIM_OK) return st;
  for (int i = 0; i < count; ++i)
    SLIM_REQUIRE(ctx, out[i].rows == tensors[i].rows && out[i].cols == tensors[i].cols && out[i].dtype == tensors[i].dtype,
                 "%s: output %d is of another shape or type", fn, i);
  if (const slim_status st = check_outputs(ctx, fn, tensors, out, count); st != SLIM_OK) return st;
  return norm_and_scale(ctx, fn, tensors, out, count, limit, norm);
}

}  // extern "C"
