// Distillation from a teacher's top logits: the divergence of a row and the gradient of the student's logits.
//
//   p = softmax of the row's teacher logits / tau over its slots, or, where the teacher's log-sum-exp is given, exp(t / tau - lse) and the
//   rest 1 - sum p as one more class (none below 2^-20);  q = softmax(S / tau);  loss = sum p ln(p / q), the rest included
//   dS = dloss / tau (q - p) in a slot, dloss / tau (q - rest q / q_rest) elsewhere (q without a rest);  rows of no p: zero
//
// Bound by memory: a row of logits is read once and its gradient written once.  One workgroup per row, which keeps it in registers as it
// came: maximum, sum of exponentials, then the gradient, without a second read.  Rows that do not fit are read twice, the first time with a
// running maximum and sum.  Outside the slots the gradient is one factor times the exponential; the slots are written over it
// afterwards.  The sum outside the slots (with a rest) leaves them out by a bit per class in LDS: taking them from the whole sum would
// cancel where they hold nearly all of it.  Sums over the vocabulary in fp32 (a lane's few, then a tree), exponentials of differences from
// the maximum; whatever has one value per slot or row in fp64: the loss is a small difference of large terms.
#include "slim_device.h"
#include "slim_internal.h"

namespace {

using namespace slimdev;

constexpr int DL_MAX_K = 2048, DL_MAX_V = 1 << 19;
constexpr float LOG2E = 1.44269504088896340736f;

struct DistillArgs {
  const void* S;
  const void* index;
  const void* teacher;
  const float *lse, *dloss;
  float* loss;
  void* dS;
  int64_t lds, ldk, ldds;
  int V, K;
  int index64, t_dtype;
  double tau;
};

template <typename T>
__device__ __forceinline__ float widen(unsigned short v);
template <>
__device__ __forceinline__ float widen<__half>(unsigned short v) { return (float)__builtin_bit_cast(_Float16, v); }
template <>
__device__ __forceinline__ float widen<__hip_bfloat16>(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
template <typename T>
__device__ __forceinline__ unsigned short narrow(float v) {
  if constexpr (__is_same(T, __half)) return __builtin_bit_cast(unsigned short, (_Float16)v);
  else return __builtin_bit_cast(unsigned short, (__bf16)v);
}
template <typename T>
__device__ __forceinline__ float value(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 4) return static_cast<const float*>(p)[i];
  else return widen<T>(static_cast<const unsigned short*>(p)[i]);
}
template <typename T>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
  if constexpr (sizeof(T) == 4) static_cast<float*>(p)[i] = v;
  else static_cast<unsigned short*>(p)[i] = narrow<T>(v);
}

// 16 bytes of a row; elements behind the row's end read as minus infinity, whose exponential is zero
template <typename T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  unsigned v[4];
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= E) {
      __builtin_memcpy(v, p, 16);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = i < left ? reinterpret_cast<const unsigned*>(p)[i] : 0xff800000u;
    } else {
      constexpr unsigned NONE = __is_same(T, __half) ? 0xfc00u : 0xff80u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        v[i] = (2 * i < left ? q[2 * i] : NONE) | (2 * i + 1 < left ? q[2 * i + 1] : NONE) << 16;
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return widen<T>((unsigned short)(v[i / 2] >> (16 * (i & 1))));
  }
  // The widened values are not kept from one use to the next: they would take twice the registers.
  __device__ __forceinline__ void narrow_again() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
#endif
  }
  __device__ __forceinline__ float top() const {
    float m = get(0);
#pragma unroll
    for (int i = 1; i < E; ++i) m = fmaxf(m, get(i));
    return m;
  }
};
template <typename T>
__device__ __forceinline__ void store_piece(T* p, int left, const float (&f)[16 / sizeof(T)]) {
  constexpr int E = 16 / sizeof(T);
  unsigned v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
    else v[i] = (unsigned)narrow<T>(f[2 * i]) | (unsigned)narrow<T>(f[2 * i + 1]) << 16;
  }
  if (left >= E) {
    __builtin_memcpy(p, v, 16);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) reinterpret_cast<unsigned*>(p)[i] = v[i];
        else reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(v[i / 2] >> (16 * (i & 1)));
      }
  }
}

__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s, WAVE));
  return v;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s, WAVE);
  return v;
}

// P pieces of the row per thread in registers; P = 0: the row is read twice
template <typename T, int THREADS, int P, bool REST, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill(DistillArgs a) {
  constexpr int E = Piece<T>::E, W = THREADS / 64;
  extern __shared__ __align__(16) char smem_dl[];
  double* sp = reinterpret_cast<double*>(smem_dl);                 // p of a slot (without a rest: before its division by the sum)
  double* se = sp + a.K;                                           // exp(z - top) of a slot
  int* si = reinterpret_cast<int*>(se + a.K);                      // its class, or -1
  unsigned* bits = reinterpret_cast<unsigned*>(si + a.K);          // REST: a bit per class
  __shared__ float red_m[W], red_t[W], red_e[W];
  __shared__ double red_d[W][3];
  __shared__ float share[2];
  __shared__ double rows_[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const T* S = static_cast<const T*>(a.S) + row * a.lds;
  const double itau = 1.0 / a.tau;
  const float c = (float)(1.44269504088896340736 * itau);

  Piece<T> x[P > 0 ? P : 1];
  if constexpr (P > 0) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * THREADS + tid) * E;
      x[i].load(S + at, a.V - at);
    }
  }
  if constexpr (REST)
    for (int i = tid; i < (a.V + 31) / 32; i += THREADS) bits[i] = 0u;
  // slots
  float t_top = -INFINITY;
  for (int k = tid; k < a.K; k += THREADS) {
    const int64_t at = row * a.ldk + k;
    const int64_t cls = a.index64 ? static_cast<const int64_t*>(a.index)[at] : (int64_t)static_cast<const int*>(a.index)[at];
    const bool used = cls >= 0 && cls < a.V;
    si[k] = used ? (int)cls : -1;
    if (used) {
      const float t = a.t_dtype == SLIM_F32 ? value<float>(a.teacher, at) : a.t_dtype == SLIM_F16 ? value<__half>(a.teacher, at)
                                                                                                  : value<__hip_bfloat16>(a.teacher, at);
      sp[k] = (double)t;
      se[k] = (double)value<T>(S, cls);
      t_top = fmaxf(t_top, t);
    }
  }
  // maximum (P = 0: with the sum relative to it)
  float m = -INFINITY, e = 0.f;
  if constexpr (P > 0) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      m = fmaxf(m, x[i].top());
      x[i].narrow_again();
    }
  }
  if constexpr (REST) {
    __syncthreads();
    for (int k = tid; k < a.K; k += THREADS)
      if (si[k] >= 0) atomicOr(&bits[si[k] >> 5], 1u << (si[k] & 31));
    __syncthreads();
  }
  auto sum_piece = [&](const Piece<T>& p, int at, float top) {
    float s = 0.f;
    int mask = 0;
    if constexpr (REST) mask = at < a.V ? (int)reinterpret_cast<const uint8_t*>(bits)[at >> 3] >> (at & 7 & ~(E - 1)) : 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float v = __builtin_amdgcn_exp2f((p.get(i) - top) * c);
      if constexpr (REST) v = __uint_as_float(__float_as_uint(v) & ~(unsigned)((mask << (31 - i)) >> 31));
      s += v;
    }
    return s;
  };
  if constexpr (P == 0) {
    for (int at = tid * E; at < a.V; at += THREADS * E) {
      Piece<T> p;
      p.load(S + at, a.V - at);
      const float mp = p.top();
      if (mp > m) {
        e *= __builtin_amdgcn_exp2f((m - mp) * c);
        m = mp;
      }
      e += m > -INFINITY ? sum_piece(p, at, m) : (mp != mp ? mp : 0.f);
    }
  }
  const float own_m = m;
  m = wave_max_f32(m);
  t_top = wave_max_f32(t_top);
  if (lane == 0) {
    red_m[wave] = m;
    red_t[wave] = t_top;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) {
    m = fmaxf(m, red_m[i]);
    t_top = fmaxf(t_top, red_t[i]);
  }
  const float top = m;
  if constexpr (P > 0) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      e += sum_piece(x[i], (i * THREADS + tid) * E, top);
      x[i].narrow_again();
    }
  } else {
    e = own_m > -INFINITY ? e * __builtin_amdgcn_exp2f((own_m - top) * c) : e;
  }
  // slots: A = sum p (t - z), B = sum p, C = sum exp(z - top); logits over tau
  double d[3] = {0.0, 0.0, 0.0};
  const double t0 = REST ? (double)a.lse[row] : (t_top > -INFINITY ? (double)t_top * itau : 0.0), z0 = (double)top * itau;
  for (int k = tid; k < a.K; k += THREADS) {
    double p = 0.0, ez = 0.0;
    if (si[k] >= 0) {
      const double t = sp[k] * itau, z = se[k] * itau;
      p = exp(t - t0);
      ez = exp(z - z0);
      if (p != 0.0) d[0] += p * (t - z);
      d[1] += p;
      d[2] += ez;
    }
    sp[k] = p;
    se[k] = ez;
  }
  e = wave_sum_f32(e);
#pragma unroll
  for (int i = 0; i < 3; ++i) d[i] = wave_sum(d[i]);
  if (lane == 0) {
    red_e[wave] = e;
#pragma unroll
    for (int i = 0; i < 3; ++i) red_d[wave][i] = d[i];
  }
  __syncthreads();
  if (tid == 0) {
    double es = 0.0, A = 0.0, B = 0.0, C = 0.0;
    for (int i = 0; i < W; ++i) {
      es += (double)red_e[i];
      A += red_d[i][0];
      B += red_d[i][1];
      C += red_d[i][2];
    }
    const double total = REST ? es + C : es;
    double rest = 0.0;
    if (REST) {
      rest = 1.0 - B;
      if (rest < 0x1p-20) rest = 0.0;
    }
    const bool live = !(B + rest <= 0.0);
    const double g = GRAD && live ? (double)a.dloss[row] * itau : 0.0;
    const double other = rest > 0.0 && es > 0.0 ? 1.0 - rest * total / es : 1.0;
    if (GRAD) {
      share[0] = (float)(g * other / total);
      share[1] = live ? 1.f : 0.f;
      rows_[0] = g / total;
      rows_[1] = REST ? g : g / B;
    }
    const double lq = z0 + log(total);
    double l = REST ? A + B * (lq - t0) : A / B + lq - (t0 + log(B));
    if (rest > 0.0) l += rest * (log(rest) - log(es / total));
    a.loss[row] = live ? (float)l : 0.f;
  }
  if constexpr (GRAD) {
    __syncthreads();
    T* dS = static_cast<T*>(a.dS) + row * a.ldds;
    const float f = share[0];
    const bool live = share[1] != 0.f;
    auto write = [&](const Piece<T>& p, int at) {
      float o[E];
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] = live ? __builtin_amdgcn_exp2f((p.get(i) - top) * c) * f : 0.f;
      store_piece<T>(dS + at, a.V - at, o);
    };
    if constexpr (P > 0) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int at = (i * THREADS + tid) * E;
        if (at < a.V) write(x[i], at);
      }
    } else {
      for (int at = tid * E; at < a.V; at += THREADS * E) {
        Piece<T> p;
        p.load(S + at, a.V - at);
        write(p, at);
      }
    }
    __syncthreads();
    if (live)
      for (int k = tid; k < a.K; k += THREADS)
        if (si[k] >= 0) put<T>(dS, si[k], (float)(se[k] * rows_[0] - sp[k] * rows_[1]));
  }
}

template <typename T, int THREADS, int P, bool REST, bool GRAD>
slim_status launch(slim_ctx* ctx, const DistillArgs& a, int64_t rows) {
  const size_t smem = (size_t)a.K * 20 + (REST ? (size_t)(a.V + 31) / 32 * 4 : 0);
  const char* name = GRAD ? "distill_grad" : "distill_loss";
  if (smem > 48 * 1024)
    SLIM_HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(&distill<T, THREADS, P, REST, GRAD>),
                                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  SLIM_LAUNCH(ctx, name, (distill<T, THREADS, P, REST, GRAD>), dim3((unsigned)rows), dim3(THREADS), smem, a);
  return SLIM_OK;
}

template <typename T, bool REST, bool GRAD>
slim_status by_size(slim_ctx* ctx, const DistillArgs& a, int64_t rows) {
  const int pieces = slim_cdiv(a.V, Piece<T>::E);
  if (pieces <= 1024) return launch<T, 256, 4, REST, GRAD>(ctx, a, rows);
  if (pieces <= 4096) return launch<T, 512, 8, REST, GRAD>(ctx, a, rows);
  if (pieces <= 16384) return launch<T, 1024, 16, REST, GRAD>(ctx, a, rows);
  return launch<T, 1024, 0, REST, GRAD>(ctx, a, rows);
}

template <typename T>
slim_status by_form(slim_ctx* ctx, const DistillArgs& a, int64_t rows, bool grad) {
  if (a.lse) return grad ? by_size<T, true, true>(ctx, a, rows) : by_size<T, true, false>(ctx, a, rows);
  return grad ? by_size<T, false, true>(ctx, a, rows) : by_size<T, false, false>(ctx, a, rows);
}

slim_status run(slim_ctx* ctx, const char* fn, DistillArgs a, slim_dtype s_dtype, int64_t rows, slim_dtype t_dtype, bool grad) {
  auto is_float = [](slim_dtype d) { return d == SLIM_F16 || d == SLIM_BF16 || d == SLIM_F32; };
  if (!is_float(s_dtype) || !is_float(t_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: logits are F16, BF16 or F32", fn);
  SLIM_REQUIRE(ctx, rows >= 0 && rows < (1ll << 31) && a.V > 0 && a.K >= 0, "%s: rows = %lld, V = %d, K = %d", fn, (long long)rows, a.V, a.K);
  if (a.V > DL_MAX_V || a.K > DL_MAX_K)
    return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: up to %d classes and %d slots a row, got %d and %d", fn, DL_MAX_V, DL_MAX_K, a.V, a.K);
  SLIM_REQUIRE(ctx, a.tau > 0.0 && a.tau <= 1e30, "%s: tau = %g", fn, a.tau);
  if (rows == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, a.S && a.loss && (a.K == 0 || (a.index && a.teacher)), "%s: null pointer", fn);
  SLIM_REQUIRE(ctx, a.lds >= a.V && a.ldk >= a.K, "%s: rows shorter than V or K", fn);
  SLIM_REQUIRE(ctx, !grad || (a.dS && a.dloss && a.ldds >= a.V), "%s: null pointer, or rows shorter than V", fn);
  a.t_dtype = (int)t_dtype;
  if (s_dtype == SLIM_F32) return by_form<float>(ctx, a, rows, grad);
  return s_dtype == SLIM_F16 ? by_form<__half>(ctx, a, rows, grad) : by_form<__hip_bfloat16>(ctx, a, rows, grad);
}

}  // namespace

extern "C" {

slim_status slim_distill_loss(slim_ctx* ctx, const void* S, slim_dtype s_dtype, int64_t rows, int V, int64_t lds, const void* index,
                              int index64, const void* teacher, slim_dtype t_dtype, int K, int64_t ldk, const float* lse, double tau,
                              float* loss) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  DistillArgs a = {S, index, teacher, lse, nullptr, loss, nullptr, lds, ldk, 0, V, K, index64 != 0, 0, tau};
  return run(ctx, "slim_distill_loss", a, s_dtype, rows, t_dtype, false);
}

slim_status slim_distill_loss_grad(slim_ctx* ctx, const void* S, slim_dtype s_dtype, int64_t rows, int V, int64_t lds, const void* index,
                                   int index64, const void* teacher, slim_dtype t_dtype, int K, int64_t ldk, const float* lse, double tau,
                                   const float* dloss, float* loss, void* dS, int64_t ldds) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  DistillArgs a = {S, index, teacher, lse, dloss, loss, dS, lds, ldk, ldds, V, K, index64 != 0, 0, tau};
  return run(ctx, "slim_distill_loss_grad", a, s_dtype, rows, t_dtype, true);
}

}  // extern "C"
