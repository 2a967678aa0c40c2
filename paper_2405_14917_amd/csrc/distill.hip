// Distillation from a teacher's top logits: the divergence of a row and the gradient of the student's logits.
//
//   p = softmax of the row's teacher logits / tau over its slots, or, where the teacher's log-sum-exp is given, exp(t / tau - lse) and the
//   rest 1 - sum p as one more class (none below 2^-20);  q = softmax(S / tau);  loss = sum p ln(p / q), the rest included
//   dS = dloss / tau (q - p) in a slot, dloss / tau (q - rest q / q_rest) elsewhere (q without a rest);  rows of no p: zero
//
// Bound by memory: a row of logits is read once and its gradient written once.  One workgroup per row, which keeps it in registers as it
// came: maximum, sum of exponentials, then the gradient, without a second read.  Rows that do not fit are
// cut into chunks of a workgroup each: one kernel leaves every chunk's maximum and sum, a second one joins them and writes the
// gradient, its own read of the logits mostly from the cache behind the L2.  Outside the slots the gradient is one factor times the
// exponential; the slots are written over it afterwards.  With a rest, the classes outside the slots have a maximum and a sum of their own
// (the slots are dropped from the row in registers by a bit per class in LDS): taken from the whole sum they would cancel where the slots
// hold nearly all of it, and relative to the slots' maximum their exponentials would vanish where it leads them by more than fp32's range.
// So the gradient there is r (q_rest - rest), r their softmax among themselves.  Sums over the vocabulary in fp32 (a lane's few,
// then a tree; chunks in fp64), exponentials of the difference from the maximum, 2^((x - top) log2(e) / tau): a common shift of a row's logits
// changes nothing, and a row of nothing but the type's lowest value is one of zeros.  Whatever has one value per slot or row in fp64, differences
// too: the loss is a small difference of large terms.
#include "slim_device.h"
#include "slim_internal.h"

namespace {

using namespace slimdev;

constexpr int DL_MAX_K = 2048;
constexpr double LOG2E = 1.44269504088896340736;

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
  double itau;                       // 1 / tau
  float c;                           // log2(e) / tau
  // rows in chunks: `chunks` of them, their maxima and sums (rows x chunks), and the slots' sums (5 per row)
  int chunks;
  float2* part;
  double* slots;
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

// 16 bytes of a row
template <typename T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  unsigned v[4];
  static constexpr unsigned NONE = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __half) ? 0xfc00fc00u : 0xff80ff80u;      // minus infinity
  __device__ __forceinline__ void none() {                           // logits whose exponential is zero
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = NONE;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return widen<T>((unsigned short)(v[i / 2] >> (16 * (i & 1))));
  }
  __device__ __forceinline__ void set(const float (&f)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
      else v[i] = (unsigned)narrow<T>(f[2 * i]) | (unsigned)narrow<T>(f[2 * i + 1]) << 16;
    }
  }
  __device__ __forceinline__ void drop(unsigned m) {                 // the elements whose bit is set become minus infinity
    auto all = [&](int e) { return (unsigned)((int)(m << (31 - e)) >> 31); };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned to = 0;
      if constexpr (sizeof(T) == 4) to = all(i);
      else to = (all(2 * i) & 0xffffu) | (all(2 * i + 1) & 0xffff0000u);
      v[i] = (v[i] & ~to) | (NONE & to);
    }
  }
  // The widened values are not kept from one use to the next: they would take twice the registers.
  __device__ __forceinline__ void narrow_again() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
#endif
  }
};

// Exponentials relative to the maximum `top`, times 2^LIFT: the instruction counts results below 2^-126 as zero, which lifted are below
// 2^-150 of the largest, the least fp32 number; 2^30 classes of 2^LIFT are no overflow.
constexpr int LIFT = 24;
constexpr double UNLIFT = 1.0 / (1 << LIFT);

// How they are taken: 2^(v c - off), c = log2(e) / tau, off = top c - LIFT rounded to fp32, is one instruction for the argument; k makes up for
// that rounding, so that only c's own remains, of v - top.  (From v - top itself: 2048 x 12000 fp16 30.2 us in place of 28.3.)  Where top c is
// so large that the rounding is no small number, the row itself is shifted to a maximum of 0 (Range::shift).
struct Scale {
  float c, top, off, k;
  bool near;
  // (a maximum of minus infinity, of nothing or of excluded classes alone, is a base of 0, against which they stay zero)
  __device__ __forceinline__ Scale(float c_, float top_) : c(c_), top(top_ > -INFINITY ? top_ : 0.f) {
    const double exact = fma((double)top, (double)c, -(double)LIFT);
    off = (float)exact;
    near = fabsf(off) <= 0x1p22f;
    k = near ? __builtin_amdgcn_exp2f((float)((double)off - exact)) : 1.f;
    if (!near) off = -(float)LIFT;
  }
  __device__ __forceinline__ float exp_of(float v) const { return __builtin_amdgcn_exp2f(fmaf(v, c, -off)); }
};

// A range of a row in the registers of a workgroup: P pieces per thread, and the elements behind the last whole piece, one per thread.
template <typename T, int THREADS, int P>
struct Range {
  static constexpr int E = Piece<T>::E;
  Piece<T> x[P];
  float last;
  int pieces, rest, tid;
  __device__ __forceinline__ void load(const T* S, int n, int t) {
    tid = t;
    pieces = n / E;
    rest = n % E;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (i * THREADS + tid < pieces) __builtin_memcpy(x[i].v, S + (i * THREADS + tid) * E, 16);
      else x[i].none();
    }
    last = tid < rest ? value<T>(S, (int64_t)pieces * E + tid) : -INFINITY;
  }
  __device__ __forceinline__ float top() {
    float m = last;
#pragma unroll
    for (int i = 0; i < P; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, x[i].get(e));
      x[i].narrow_again();
    }
    return m;
  }
  // the classes whose bit is set become minus infinity
  __device__ __forceinline__ void drop(const uint8_t* bits) {
    if (tid < rest && (bits[(pieces * E + tid) >> 3] >> ((pieces * E + tid) & 7) & 1)) last = -INFINITY;
    constexpr int PER = 32 / E;                                      // pieces whose bits fill a word
    unsigned mask[(P + PER - 1) / PER] = {}, any = 0;                // (all read before the first is looked at)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = min(i * THREADS + tid, max(pieces - 1, 0)) * E;
      const unsigned m = ((unsigned)bits[at >> 3] >> (at & 7)) & ((1u << E) - 1);
      mask[i / PER] |= m << (i % PER * E);
    }
#pragma unroll
    for (unsigned m : mask) any |= m;
    if (!any) return;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (const unsigned m = mask[i / PER] >> (i % PER * E) & ((1u << E) - 1)) x[i].drop(m);
  }
  // Logits so far from zero that top c exceeds 2^22 become their difference from `top`.  In the type of the logits: where the difference
  // counts (150 / 2^22 of top and less) it is exact in fp32 and zero in 16 bits.
  __device__ __forceinline__ void shift(const Scale& to) {
    if (__builtin_expect(to.near, 1)) return;
    last -= to.top;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = x[i].get(e) - to.top;
      x[i].set(o);
    }
  }
  // sum of the exponentials, lifted
  __device__ __forceinline__ float sum(const Scale& to) {
    float s = to.exp_of(last);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float p = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) p += to.exp_of(x[i].get(e));
      s += p;
      x[i].narrow_again();
    }
    return s * to.k;
  }
  // f times the exponentials, f for lifted ones
  __device__ __forceinline__ void write(T* dS, const Scale& to, float f) {
    f *= to.k;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (i * THREADS + tid < pieces) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = to.exp_of(x[i].get(e)) * f;
        Piece<T> p;
        p.set(o);
        store16_once(dS + (i * THREADS + tid) * E, p.v);
      }
    if (tid < rest) put<T>(dS, (int64_t)pieces * E + tid, to.exp_of(last) * f);
  }
  __device__ __forceinline__ void write_zero(T* dS) {
    Piece<T> p = {};
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (i * THREADS + tid < pieces) __builtin_memcpy(dS + (i * THREADS + tid) * E, p.v, 16);
    if (tid < rest) put<T>(dS, (int64_t)pieces * E + tid, 0.f);
  }
};

// class of a slot, -1 for an empty one
__device__ __forceinline__ int class_of(const DistillArgs& a, int64_t at) {
  const int64_t c = a.index64 ? static_cast<const int64_t*>(a.index)[at] : (int64_t)static_cast<const int*>(a.index)[at];
  return c >= 0 && c < a.V ? (int)c : -1;
}
__device__ __forceinline__ float teacher_of(const DistillArgs& a, int64_t at) {
  return a.t_dtype == SLIM_F32 ? value<float>(a.teacher, at) : a.t_dtype == SLIM_F16 ? value<__half>(a.teacher, at) : value<__hip_bfloat16>(a.teacher, at);
}

// What a row's slots and sums make of it.  Slots, whose logits z are relative to a base zs: A = sum p (t - z), B = sum p (without a
// rest before its division by itself), C = sum exp(z) (with a rest); es: the sum of the exponentials of the classes outside the slots (without
// a rest: of all) relative to their maximum, gap: that less zs.  All logits over tau.
struct Row {
  double rest, es, total, A, B, gap, q_rest, slot;               // slot: q of a slot over its exp(z)
  bool live;
  __device__ __forceinline__ Row(double A_, double B_, double C, double es_, double gap_, bool with_rest)
      : rest(with_rest ? 1.0 - B_ : 0.0), es(es_), total(es_), A(A_), B(B_), gap(gap_), q_rest(1.0), slot(1.0 / es_) {
    if (rest < 0x1p-20) rest = 0.0;
    live = !(B + rest <= 0.0);
    if (with_rest) {
      const double e = exp(-fabs(gap)), out = gap > 0.0 ? 1.0 : e, in = gap > 0.0 ? e : 1.0;
      total = es * out + C * in;                                  // relative to the larger of the two maxima
      q_rest = es * out / total;
      slot = in / total;
    }
  }
  // the gradient outside the slots over the lifted exponential; 0 where the slots leave no class with a probability, NaN where there is none at all
  __device__ __forceinline__ float factor(double g) const {
    return es == 0.0 ? (total == 0.0 ? NAN : 0.f) : (float)(g * UNLIFT * (q_rest - rest) / es);
  }
  __device__ __forceinline__ float loss(bool with_rest) const {
    const double lt = with_rest ? fmax(gap, 0.0) + log(total) : log(es) + gap;      // of the sum over all classes, less zs
    double l = with_rest ? A + B * lt : A / B + lt - log(B);
    if (rest > 0.0) l += rest * (log(rest) - (log(es) + gap - lt));
    return live ? (float)l : 0.f;
  }
};

// sums of N values over a workgroup of W wavefronts, in every thread
template <int W, int N>
__device__ __forceinline__ void group_sums(double (&d)[N], double (*red)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) d[i] = wave_sum(d[i]);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[threadIdx.x >> 6][i] = d[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    d[i] = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) d[i] += red[w][i];
  }
}
template <int W>
__device__ __forceinline__ float group_max(float m, float* red) {
  m = wave_max_f32(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) m = fmaxf(m, red[w]);
  return m;
}

// ---- a row per workgroup --------------------------------------------------------------------------------------
template <typename T, int THREADS, int P, bool REST, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill(DistillArgs a) {
  constexpr int W = THREADS / 64;
  extern __shared__ __align__(16) char smem_dl[];
  double* sp = reinterpret_cast<double*>(smem_dl);                 // p of a slot
  double* se = sp + a.K;                                           // exp(z) of a slot, relative to zs
  int* si = reinterpret_cast<int*>(se + a.K);                      // its class, or -1
  unsigned* bits = reinterpret_cast<unsigned*>(si + a.K);          // REST: a bit per class
  __shared__ float red_m[W], red_t[W];
  __shared__ double red_d[W][4];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* S = static_cast<const T*>(a.S) + row * a.lds;
  const double itau = a.itau;

  Range<T, THREADS, P> x;
  x.load(S, a.V, tid);
  if constexpr (REST) {
    for (int i = tid; i < (a.V + 31) / 32; i += THREADS) bits[i] = 0u;
    __syncthreads();
  }
  float high = -INFINITY;                                          // of the slots: the student's logits, without a rest the teacher's
  for (int k = tid; k < a.K; k += THREADS) {
    const int cls = class_of(a, row * a.ldk + k);
    si[k] = cls;
    if (cls >= 0) {
      const float t = teacher_of(a, row * a.ldk + k), z = value<T>(S, cls);
      sp[k] = (double)t;
      se[k] = (double)z;
      high = fmaxf(high, REST ? z : t);
      if constexpr (REST) atomicOr(&bits[cls >> 5], 1u << (cls & 31));
    }
  }
  high = group_max<W>(high, red_t);                                // (its barrier: the bits are set)
  if constexpr (REST) x.drop(reinterpret_cast<const uint8_t*>(bits));
  const Scale to(a.c, group_max<W>(x.top(), red_m));
  x.shift(to);
  double d[4] = {0.0, 0.0, 0.0, (double)x.sum(to) * UNLIFT};
  // (teacher: t / tau less its maximum, or less its log-sum-exp)
  const double t0 = REST || high == -INFINITY ? 0.0 : (double)high, tl = REST ? (double)a.lse[row] : 0.0, zs = REST && high > -INFINITY ? (double)high : (double)to.top;
  for (int k = tid; k < a.K; k += THREADS) {
    double p = 0.0, ez = 0.0;
    if (si[k] >= 0) {
      const double t = (sp[k] - t0) * itau - tl, z = (se[k] - zs) * itau;
      p = exp(t);
      ez = exp(z);
      if (p != 0.0) d[0] += p * (t - z);
      d[1] += p;
      d[2] += ez;
    }
    sp[k] = p;
    se[k] = ez;
  }
  group_sums<W, 4>(d, red_d);
  if (!GRAD && tid < THREADS - 64) return;
  const Row r(d[0], d[1], d[2], d[3], ((double)to.top - zs) * itau, REST);
  if constexpr (GRAD) {
    T* dS = static_cast<T*>(a.dS) + row * a.ldds;
    const double g = (double)a.dloss[row] * itau;
    if (r.live) {
      x.write(dS, to, r.factor(g));
      __syncthreads();
      const double ge = g * r.slot, gp = REST ? g : g / r.B;
      for (int k = tid; k < a.K; k += THREADS)
        if (si[k] >= 0) put<T>(dS, si[k], (float)(se[k] * ge - sp[k] * gp));
    } else {
      x.write_zero(dS);
    }
  }
  if (tid == THREADS - 64) a.loss[row] = r.loss(REST);                // (the last wavefront, whose share of the row is the smallest)
}

// ---- a chunk per workgroup --------------------------------------------------------------------------------------
constexpr int CH_THREADS = 256, CH_P = 4;
template <typename T>
constexpr int CHUNK = CH_THREADS * CH_P * Piece<T>::E;            // elements

// first kernel: a chunk's maximum and sum; the workgroup of the first chunk also the slots' sums
template <typename T, bool REST>
__global__ __launch_bounds__(CH_THREADS) void distill_chunks(DistillArgs a) {
  constexpr int W = CH_THREADS / 64;
  __shared__ unsigned bits[CHUNK<T> / 32];
  __shared__ float red_m[W], red_t[W], red_z[W];
  __shared__ double red_d[W][3], red_e[W][1];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x / a.chunks;
  const int chunk = (int)(blockIdx.x % a.chunks), c0 = chunk * CHUNK<T>, n = min(CHUNK<T>, a.V - c0);
  const T* S = static_cast<const T*>(a.S) + row * a.lds;
  const double itau = a.itau;
  Range<T, CH_THREADS, CH_P> x;
  x.load(S + c0, n, tid);
  if constexpr (REST) {
    for (int i = tid; i < CHUNK<T> / 32; i += CH_THREADS) bits[i] = 0u;
    __syncthreads();
    for (int k = tid; k < a.K; k += CH_THREADS) {
      const int cls = class_of(a, row * a.ldk + k) - c0;
      if (cls >= 0 && cls < n) atomicOr(&bits[cls >> 5], 1u << (cls & 31));
    }
  }
  if constexpr (REST) {
    __syncthreads();
    x.drop(reinterpret_cast<const uint8_t*>(bits));
  }
  const float top = group_max<W>(x.top(), red_m);
  const Scale to(a.c, top);
  x.shift(to);
  double e[1] = {(double)x.sum(to) * UNLIFT};
  group_sums<W, 1>(e, red_e);
  if (tid == 0) a.part[row * a.chunks + chunk] = make_float2(top, (float)e[0]);
  if (chunk != 0) return;
  float t_top = -INFINITY, z_top = -INFINITY;
  for (int k = tid; k < a.K; k += CH_THREADS) {
    const int cls = class_of(a, row * a.ldk + k);
    if (cls >= 0) {
      t_top = fmaxf(t_top, teacher_of(a, row * a.ldk + k));
      z_top = fmaxf(z_top, value<T>(S, cls));
    }
  }
  t_top = group_max<W>(t_top, red_t);
  z_top = group_max<W>(z_top, red_z);
  const double t0 = REST || t_top == -INFINITY ? 0.0 : (double)t_top, tl = REST ? (double)a.lse[row] : 0.0,
               zs = z_top > -INFINITY ? (double)z_top : 0.0;
  double d[3] = {0.0, 0.0, 0.0};
  for (int k = tid; k < a.K; k += CH_THREADS) {
    const int cls = class_of(a, row * a.ldk + k);
    if (cls >= 0) {
      const double t = ((double)teacher_of(a, row * a.ldk + k) - t0) * itau - tl, z = ((double)value<T>(S, cls) - zs) * itau, p = exp(t);
      if (p != 0.0) d[0] += p * (t - z);
      d[1] += p;
      if constexpr (REST) d[2] += exp(z);
    }
  }
  group_sums<W, 3>(d, red_d);
  if (tid == 0) {
    double* s = a.slots + row * 5;
    s[0] = d[0];
    s[1] = d[1];
    s[2] = d[2];
    s[3] = (double)z_top;
    s[4] = t0;
  }
}

// second kernel: the row from its chunks, the gradient of a chunk; the workgroup of the first chunk also the loss.  Without the gradient one
// wavefront per row.
template <typename T, bool REST, bool GRAD>
__global__ __launch_bounds__(GRAD ? CH_THREADS : 64) void distill_join(DistillArgs a) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int per_row = GRAD ? a.chunks : 1;
  const int64_t row = blockIdx.x / per_row;
  const int chunk = (int)(blockIdx.x % per_row), c0 = chunk * CHUNK<T>, n = min(CHUNK<T>, a.V - c0);
  const T* S = static_cast<const T*>(a.S) + row * a.lds;
  const double itau = a.itau;
  Range<T, CH_THREADS, CH_P> x;
  if constexpr (GRAD) x.load(S + c0, n, tid);
  const float2* part = a.part + row * a.chunks;
  float top = -INFINITY;
  for (int i = lane; i < a.chunks; i += 64) top = fmaxf(top, part[i].x);
  const Scale to(a.c, wave_max_f32(top));
  double es = 0.0;
  for (int i = lane; i < a.chunks; i += 64) {
    const float2 v = part[i];
    // (that of a chunk without a maximum is 0 or NaN)
    es += v.x == -INFINITY ? (double)v.y : (double)v.y * exp(((double)v.x - (double)to.top) * itau);
  }
  es = wave_sum(es);
  const double* s = a.slots + row * 5;
  const double zs = s[3] > -INFINITY ? s[3] : (double)to.top, t0 = s[4], tl = REST ? (double)a.lse[row] : 0.0;
  const Row r(s[0], s[1], s[2], es, ((double)to.top - zs) * itau, REST);
  if constexpr (GRAD) {
    T* dS = static_cast<T*>(a.dS) + row * a.ldds;
    const double g = (double)a.dloss[row] * itau;
    if (r.live) {
      // the gradients of the slots of this chunk, before their logits are written over (dS may be S)
      extern __shared__ __align__(16) char smem_dl[];
      float* sv = reinterpret_cast<float*>(smem_dl);
      int* si = reinterpret_cast<int*>(sv + a.K);
      const double ge = g * r.slot, gp = REST ? g : g / r.B, zb = REST ? zs : (double)to.top;
      for (int k = tid; k < a.K; k += CH_THREADS) {
        const int cls = class_of(a, row * a.ldk + k), at = cls - c0;
        si[k] = cls >= 0 && at >= 0 && at < n ? at : -1;
        if (si[k] >= 0)
          sv[k] = (float)(exp(((double)value<T>(S, cls) - zb) * itau) * ge - exp(((double)teacher_of(a, row * a.ldk + k) - t0) * itau - tl) * gp);
      }
      __syncthreads();
      x.shift(to);
      x.write(dS + c0, to, r.factor(g));
      __syncthreads();
      for (int k = tid; k < a.K; k += CH_THREADS)
        if (si[k] >= 0) put<T>(dS, c0 + si[k], sv[k]);
    } else {
      x.write_zero(dS + c0);
    }
  }
  if (chunk == 0 && tid == 0) a.loss[row] = r.loss(REST);
}

template <typename T, int THREADS, int P, bool REST, bool GRAD>
slim_status launch(slim_ctx* ctx, const DistillArgs& a, int64_t rows) {
  const size_t smem = (size_t)a.K * 20 + (REST ? (size_t)(a.V + 31) / 32 * 4 : 0);
  SLIM_LAUNCH(ctx, GRAD ? "distill_grad" : "distill_loss", (distill<T, THREADS, P, REST, GRAD>), dim3((unsigned)rows), dim3(THREADS), smem, a);
  return SLIM_OK;
}

// Rows as chunks: where a row does not fit a workgroup's registers (301 x 50257 fp32: 38 us; with 16 pieces in each of 1024 threads, one row
// per CU, 88).
constexpr int DL_ROW_PIECES = 4096;
int chunks_of(int V, slim_dtype d) {
  const int e = d == SLIM_F32 ? 4 : 8, chunk = CH_THREADS * CH_P * e;
  return slim_cdiv(V, e) <= DL_ROW_PIECES ? 0 : slim_cdiv(V, chunk);
}
size_t part_bytes(int64_t rows, int chunks) { return slim_ws_round(sizeof(float2) * (size_t)rows * chunks); }
size_t slot_bytes(int64_t rows) { return slim_ws_round(sizeof(double) * 5 * (size_t)rows); }
size_t need(int64_t rows, int V, slim_dtype d) {
  const int chunks = chunks_of(V, d);
  return chunks ? part_bytes(rows, chunks) + slot_bytes(rows) : 0;
}

// Threads of a row in one workgroup.  Eight pieces per thread up to 2048 pieces: of 4000 x 3000 bf16 one wavefront a row takes 19.9 us, four
// 24.9; 2048 x 12000 with four 26.6 us, with eight 38.0.  Beyond, many rows: four wavefronts of 16 pieces (2048 x 32000 bf16 with 64 slots
// 61.6 us against 65.3 with eight of 8, with 256 slots 68.1 and 70.7; 1600 x 32000 50.9 and 54.6), but fewer rows, a last round of which
// leaves CUs idle, and many slots, a thread's share of which is twice as long: eight of 8 (400 x 32000 16.0 us against 17.1, 1200 x 32000
// 35.3 and 36.3; between them 600 rows 22.3 and 20.6; 2048 x 32000 with 1024 slots 91.5 and 93.9, 3000 130.9 and 141.8).
int threads_of(int pieces, int64_t rows, int K, bool grad, int ncu) {
  if (pieces <= 512) return 64;
  if (pieces <= 1024) return 128;
  return pieces <= 2048 || (grad && rows > 6 * ncu && K <= 512) ? 256 : 512;
}

template <typename T, bool REST, bool GRAD>
slim_status by_size(slim_ctx* ctx, DistillArgs a, int64_t rows) {
  constexpr int E = Piece<T>::E;
  const int pieces = a.V / E;
  a.chunks = chunks_of(a.V, sizeof(T) == 4 ? SLIM_F32 : SLIM_BF16);
  if (a.chunks) {
    a.part = static_cast<float2*>(slim_ws_alloc(ctx, part_bytes(rows, a.chunks)));
    a.slots = static_cast<double*>(slim_ws_alloc(ctx, slot_bytes(rows)));
    if (!a.part || !a.slots) return slim_fail(ctx, SLIM_ERR_ALLOC, "slim_distill_loss: workspace");
    SLIM_LAUNCH(ctx, "distill_chunks", (distill_chunks<T, REST>), dim3((unsigned)(rows * a.chunks)), dim3(CH_THREADS), 0, a);
    SLIM_LAUNCH(ctx, GRAD ? "distill_join_grad" : "distill_join_loss", (distill_join<T, REST, GRAD>), dim3((unsigned)(GRAD ? rows * a.chunks : rows)),
                dim3(GRAD ? CH_THREADS : 64), GRAD ? (size_t)a.K * 8 : 0, a);
    return SLIM_OK;
  }
  switch (threads_of(pieces, rows, a.K, GRAD, ctx->num_cus)) {
    case 64: return launch<T, 64, 8, REST, GRAD>(ctx, a, rows);
    case 128: return launch<T, 128, 8, REST, GRAD>(ctx, a, rows);
    case 512: return launch<T, 512, 8, REST, GRAD>(ctx, a, rows);
  }
  if constexpr (GRAD)
    if (pieces > 2048) return launch<T, 256, 16, REST, GRAD>(ctx, a, rows);
  return launch<T, 256, 8, REST, GRAD>(ctx, a, rows);
}

template <typename T>
slim_status by_form(slim_ctx* ctx, const DistillArgs& a, int64_t rows, bool grad) {
  if (a.lse) return grad ? by_size<T, true, true>(ctx, a, rows) : by_size<T, true, false>(ctx, a, rows);
  return grad ? by_size<T, false, true>(ctx, a, rows) : by_size<T, false, false>(ctx, a, rows);
}

slim_status run(slim_ctx* ctx, const char* fn, DistillArgs a, slim_dtype s_dtype, int64_t rows, slim_dtype t_dtype, double tau, bool grad) {
  auto is_float = [](slim_dtype d) { return d == SLIM_F16 || d == SLIM_BF16 || d == SLIM_F32; };
  if (!is_float(s_dtype) || !is_float(t_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: logits are F16, BF16 or F32", fn);
  SLIM_REQUIRE(ctx, rows >= 0 && a.V > 0 && a.V < (1 << 30) && a.K >= 0, "%s: rows = %lld, V = %d, K = %d", fn, (long long)rows, a.V, a.K);
  if (a.K > DL_MAX_K) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: up to %d slots a row, got %d", fn, DL_MAX_K, a.K);
  // (a launch has fewer than 2^32 threads)
  const int chunks = chunks_of(a.V, s_dtype), threads = threads_of(a.V / (s_dtype == SLIM_F32 ? 4 : 8), rows, a.K, grad, ctx->num_cus);
  if (rows >= (1ll << 31) || rows * (chunks ? (int64_t)chunks * CH_THREADS : threads) >= (1ll << 32))
    return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: %lld rows of %d classes are too many for one call", fn, (long long)rows, a.V);
  SLIM_REQUIRE(ctx, tau > 0.0 && tau <= 1e30, "%s: tau = %g", fn, tau);
  if (rows == 0) return SLIM_OK;
  SLIM_REQUIRE(ctx, a.S && a.loss && (a.K == 0 || (a.index && a.teacher)), "%s: null pointer", fn);
  SLIM_REQUIRE(ctx, a.lds >= a.V && a.ldk >= a.K, "%s: rows shorter than V or K", fn);
  SLIM_REQUIRE(ctx, !grad || (a.dS && a.dloss && a.ldds >= a.V), "%s: null pointer, or rows shorter than V", fn);
  if (const size_t bytes = need(rows, a.V, s_dtype))
    if (const slim_status st = slim_ws_reserve(ctx, bytes); st != SLIM_OK) return st;
  a.t_dtype = (int)t_dtype;
  a.itau = 1.0 / tau;
  a.c = (float)std::min(LOG2E * a.itau, 3e38);
  if (s_dtype == SLIM_F32) return by_form<float>(ctx, a, rows, grad);
  return s_dtype == SLIM_F16 ? by_form<__half>(ctx, a, rows, grad) : by_form<__hip_bfloat16>(ctx, a, rows, grad);
}

}  // namespace

extern "C" {

size_t slim_distill_workspace(int64_t rows, int V, slim_dtype s_dtype) { return rows > 0 && V > 0 ? need(rows, V, s_dtype) : 0; }

slim_status slim_distill_loss(slim_ctx* ctx, const void* S, slim_dtype s_dtype, int64_t rows, int V, int64_t lds, const void* index,
                              int index64, const void* teacher, slim_dtype t_dtype, int K, int64_t ldk, const float* lse, double tau,
                              float* loss) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  DistillArgs a = {S, index, teacher, lse, nullptr, loss, nullptr, lds, ldk, 0, V, K, index64 != 0, 0, 0.0, 0.f, 0, nullptr, nullptr};
  return run(ctx, "slim_distill_loss", a, s_dtype, rows, t_dtype, tau, false);
}

slim_status slim_distill_loss_grad(slim_ctx* ctx, const void* S, slim_dtype s_dtype, int64_t rows, int V, int64_t lds, const void* index,
                                   int index64, const void* teacher, slim_dtype t_dtype, int K, int64_t ldk, const float* lse, double tau,
                                   const float* dloss, float* loss, void* dS, int64_t ldds) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  DistillArgs a = {S, index, teacher, lse, dloss, loss, dS, lds, ldk, ldds, V, K, index64 != 0, 0, 0.0, 0.f, 0, nullptr, nullptr};
  return run(ctx, "slim_distill_loss_grad", a, s_dtype, rows, t_dtype, tau, true);
}

}  // extern "C"
