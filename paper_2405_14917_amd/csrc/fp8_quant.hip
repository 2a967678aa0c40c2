// Activations and weights of the 8-bit linear layer to e4m3 in blocks of 128 (fp8_device.h: the quantiser).
//
// Bound by memory: one pass over the inputs.  A row's block of 128 is 16 lanes of 8 elements, whose largest magnitude is found on
// packed 16-bit patterns (they order like the values) by moves inside a row of 16 lanes; what is not finite shows as a pattern at or
// above infinity's, and only then is the search done again without it.  The transposed form (blocks of 128 tokens, for the gradient of
// the weights) takes a tile of 128 x 128 through LDS once, in bytes; the gradient of the outputs needs both forms and is read once for
// them.
#include "act_device.h"
#include "fp8_device.h"

namespace {

using namespace slimfp8;

constexpr int RQ_THREADS = 256, RQ_UNITS = 2;     // units of 512 elements a wavefront holds at a time

// Rows: a wavefront takes units of 512 elements (four blocks) of one row.
template <typename T>
__global__ __launch_bounds__(RQ_THREADS) void fp8_rows(const T* __restrict__ X, int64_t ldx, int rows, int cols, int units,
                                                       uint8_t* __restrict__ q, uint8_t* __restrict__ s, int64_t ldq, int64_t lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t u0 = ((int64_t)blockIdx.x * (RQ_THREADS / 64) + wave) * RQ_UNITS, total = (int64_t)rows * units;
  unsigned v[RQ_UNITS][4];
#pragma unroll
  for (int i = 0; i < RQ_UNITS; ++i) {
    const int64_t u = min(u0 + i, total - 1);
    const int r = (int)(u / units), c = (int)(u % units) * 512 + lane * 8;
    fetch8(X + (int64_t)r * ldx + c, cols - c, cols, v[i]);
  }
#pragma unroll
  for (int i = 0; i < RQ_UNITS; ++i) {
    const int64_t u = u0 + i;
    if (u >= total) break;
    const int r = (int)(u / units), c = (int)(u % units) * 512 + lane * 8;
    row_end_shift<8>(v[i], cols < 8 ? 8 : cols - c);
    const unsigned b = block_scale<T>(v[i]);
    const float sc = __uint_as_float(b << 23);
    if (c < (cols + BLOCK - 1) / BLOCK * BLOCK) {
      *reinterpret_cast<uint2*>(q + (int64_t)r * ldq + c) = make_uint2(to_e4m3<T>(v[i][0], v[i][1], sc), to_e4m3<T>(v[i][2], v[i][3], sc));
      if ((lane & 15) == 0) s[(int64_t)r * lds + c / BLOCK] = (uint8_t)b;
    }
  }
}

struct TileArgs {
  Activations a[2];
  int tiles[2], tiles_c[2];        // tiles of 128 x 128, and along the columns
  ActGradient g;                   // (ACT: of the first matrix)
};

// Tiles of 128 x 128: thread t holds rows 8 (t / 16) .. + 7 of columns 8 (t % 16) .. + 7.  ACT: the first matrix is the gradient behind an
// activation; it is formed in fp32 and rounded in its place, and its columns' sums are taken before the rounding.
template <typename T, bool ACT>
__global__ __launch_bounds__(256) void fp8_tiles(TileArgs ta) {
  __shared__ __align__(16) unsigned colmax[4][64];         // per wavefront, pairs of columns
  __shared__ __align__(16) float colsum[ACT ? 4 : 1][BLOCK];
  __shared__ __align__(16) uint8_t tile[BLOCK * BLOCK];    // [column][row], units of 8 bytes at unit ^ (column / 8)
  const int p = (int)blockIdx.x >= ta.tiles[0];
  const Activations& a = ta.a[p];
  const int id = (int)blockIdx.x - (p ? ta.tiles[0] : 0), tr = id / ta.tiles_c[p], tc = id % ta.tiles_c[p];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 15, rg = tid >> 4;
  const int r0 = tr * BLOCK + rg * 8, c0 = tc * BLOCK + cg * 8;
  unsigned v[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fetch8(static_cast<const T*>(a.X) + (int64_t)min(r0 + i, a.rows - 1) * a.ldx + c0, a.cols - c0, a.cols, v[i]);
  }
  unsigned z[ACT ? 8 : 1][4] = {};
  if constexpr (ACT)
    if (p == 0 && ta.g.Z)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        fetch8(static_cast<const T*>(ta.g.Z) + (int64_t)min(r0 + i, a.rows - 1) * ta.g.ldz + c0, a.cols - c0, a.cols, z[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    row_end_shift<8>(v[i], a.cols < 8 ? 8 : a.cols - c0);
    if (r0 + i >= a.rows) v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0u;
  }
  if constexpr (ACT)
    if (p == 0) {
      float cs[8] = {};
      slimact::with_act(ta.g.act, [&](auto act) {
        constexpr int A = decltype(act)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (A != SLIM_ACT_NONE) row_end_shift<8>(z[i], a.cols < 8 ? 8 : a.cols - c0);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float d[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              d[h] = __uint_as_float(Half16<T>::float_bits((v[i][j] >> (16 * h)) & 0xffffu));
              if constexpr (A != SLIM_ACT_NONE) {
                const float f = slimact::slope(__uint_as_float(Half16<T>::float_bits((z[i][j] >> (16 * h)) & 0xffffu)), A);
                d[h] = r0 + i < a.rows ? d[h] * f : 0.f;               // (behind the last row: the last one's, which need not be finite)
              }
              cs[2 * j + h] += d[h];
            }
            if constexpr (A != SLIM_ACT_NONE) v[i][j] = (unsigned)to_16(d[0], Half16<T>::INF == 0x7f80u) | (unsigned)to_16(d[1], Half16<T>::INF == 0x7f80u) << 16;
          }
        }
      });
      if (ta.g.sums) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          cs[e] += __shfl_xor(cs[e], 16, 64);
          cs[e] += __shfl_xor(cs[e], 32, 64);
        }
        if (lane < 16) {
          *reinterpret_cast<float4*>(&colsum[wave][cg * 8]) = make_float4(cs[0], cs[1], cs[2], cs[3]);
          *reinterpret_cast<float4*>(&colsum[wave][cg * 8 + 4]) = make_float4(cs[4], cs[5], cs[6], cs[7]);
        }
        __syncthreads();
        if (tid < BLOCK && tc * BLOCK + tid < a.cols)
          ta.g.sums[(int64_t)tr * a.cols + tc * BLOCK + tid] = (colsum[0][tid] + colsum[1][tid]) + (colsum[2][tid] + colsum[3][tid]);
      }
    }
  // Largest magnitudes.  Rows: of the lane's eight numbers, two rows to a word, then over the 16 lanes of a row; columns: of the lane's
  // eight rows, the four groups of 16 lanes, the four wavefronts.
  unsigned rm[4], m[4];
  auto maxima = [&](auto magnitude) {
    unsigned r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned u = magnitude(v[i][j]);
        r[i] = j ? max_u16x2(r[i], u) : u;
        m[j] = i ? max_u16x2(m[j], u) : u;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      rm[i] = row_max_x2(max_u16x2(__builtin_amdgcn_perm(r[2 * i + 1], r[2 * i], 0x05040100u), __builtin_amdgcn_perm(r[2 * i + 1], r[2 * i], 0x07060302u)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto a32 = __builtin_amdgcn_permlane32_swap(m[j], m[j], false, false);
      const unsigned h = max_u16x2(a32[0], a32[1]);
      const auto a16 = __builtin_amdgcn_permlane16_swap(h, h, false, false);
      m[j] = max_u16x2(a16[0], a16[1]);
    }
    if (lane < 16) *reinterpret_cast<uint4*>(&colmax[wave][cg * 4]) = make_uint4(m[0], m[1], m[2], m[3]);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint4 o = *reinterpret_cast<const uint4*>(&colmax[w][cg * 4]);
      m[0] = w ? max_u16x2(m[0], o.x) : o.x;
      m[1] = w ? max_u16x2(m[1], o.y) : o.y;
      m[2] = w ? max_u16x2(m[2], o.z) : o.z;
      m[3] = w ? max_u16x2(m[3], o.w) : o.w;
    }
  };
  maxima([](unsigned u) { return u & 0x7fff7fffu; });
  // (every wavefront sees the maxima of all columns: the branch is the workgroup's)
  const unsigned top = larger_half(max_u16x2(max_u16x2(m[0], m[1]), max_u16x2(m[2], m[3])));
  if (__builtin_expect(__any(top >= Half16<T>::INF), 0)) {
    __syncthreads();
    maxima([](unsigned u) { return finite_x2<T>(u); });
  }
  if (a.rows_q) {
    const int64_t ldq = quantized_ld(a.cols), lds = (int64_t)((a.cols + BLOCK - 1) / BLOCK + 3) / 4 * 4;
    uint8_t* q = a.rows_q + (int64_t)r0 * ldq + c0;
    uint8_t* s = a.rows_s + (int64_t)r0 * lds + tc;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned b = scale_byte(Half16<T>::float_bits((i & 1) ? rm[i / 2] >> 16 : rm[i / 2] & 0xffffu));
      const float sc = __uint_as_float(b << 23);
      if (r0 + i < a.rows) {
        *reinterpret_cast<uint2*>(q) = make_uint2(to_e4m3<T>(v[i][0], v[i][1], sc), to_e4m3<T>(v[i][2], v[i][3], sc));
        if (cg == 0) *s = (uint8_t)b;
      }
      q += ldq;
      s += lds;
    }
  }
  if (!a.cols_q) return;
  const int64_t lds = (int64_t)((a.rows + BLOCK - 1) / BLOCK + 3) / 4 * 4;
  uint8_t* const tile0 = tile + cg * 8 * BLOCK + ((rg ^ cg) * 8);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned b = scale_byte(Half16<T>::float_bits(h ? m[j] >> 16 : m[j] & 0xffffu));
      const float sc = __uint_as_float(b << 23);
      unsigned pr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_perm(v[2 * i + 1][j], v[2 * i][j], h ? 0x07060302u : 0x05040100u);
      const int c = cg * 8 + 2 * j + h;
      *reinterpret_cast<uint2*>(tile0 + (2 * j + h) * BLOCK) = make_uint2(to_e4m3<T>(pr[0], pr[1], sc), to_e4m3<T>(pr[2], pr[3], sc));
      if (rg == 0 && tc * BLOCK + c < a.cols) a.cols_s[(int64_t)(tc * BLOCK + c) * lds + tr] = (uint8_t)b;
    }
  }
  __syncthreads();
  const int64_t ldq = quantized_ld(a.rows);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 32 + (tid >> 3), u = tid & 7, x = c >> 3;      // 16 bytes: units 2 u and 2 u + 1
    uint4 w = *reinterpret_cast<const uint4*>(tile + c * BLOCK + ((2 * u) ^ (x & 14)) * 8);
    if (x & 1) w = make_uint4(w.z, w.w, w.x, w.y);
    if (tc * BLOCK + c < a.cols) *reinterpret_cast<uint4*>(a.cols_q + (int64_t)(tc * BLOCK + c) * ldq + tr * BLOCK + u * 16) = w;
  }
}

// out = the columns' sums of `parts` rows: 32 columns x 32 ranges of rows, in fp64
__global__ __launch_bounds__(1024) void fp8_join_columns(const float* __restrict__ sums, int parts, int cols, void* out, int dtype) {
  __shared__ double red[32][33];
  const int x = threadIdx.x & 31, c = blockIdx.x * 32 + x, k = threadIdx.x >> 5;
  double s = 0.0;
  for (int i = k; i < parts; i += 32) s += (double)sums[(int64_t)i * cols + min(c, cols - 1)];
  red[k][x] = s;
  __syncthreads();
  if (k == 0 && c < cols) {
    for (int i = 1; i < 32; ++i) s += red[i][x];
    to_any(out, dtype, c, (float)s);
  }
}

struct WeightArgs {
  const void* W;
  int64_t ldw, ldq, lds, ldqt, ldst;
  int n, m;
  uint8_t *q, *s, *qt, *st;
};
template <typename T>
__device__ __forceinline__ float as_float(T v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __uint_as_float(Half16<T>::float_bits(__builtin_bit_cast(unsigned short, v)));
}

// Weights: blocks of 128 x 128, one workgroup each; a block's transpose has the same scale, so both forms hold the same numbers.
template <typename T>
__global__ __launch_bounds__(256) void fp8_weights(WeightArgs a) {
  __shared__ unsigned wmax[4];
  __shared__ uint8_t tile[BLOCK * (BLOCK + 4)];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r0 = blockIdx.y * BLOCK, c0 = blockIdx.x * BLOCK, c = (tid & 31) * 4;
  float v[16][4];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = i * 8 + (tid >> 5);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[i][j] = 0.f;
      if (r0 + r < a.n && c0 + c + j < a.m) v[i][j] = as_float(static_cast<const T*>(a.W)[(int64_t)(r0 + r) * a.ldw + c0 + c + j]);
      const unsigned u = __float_as_uint(v[i][j]) & 0x7fffffffu;
      if (u < 0x7f800000u) top = max(top, u);
      else v[i][j] = __uint_as_float(0x7fc00000u);
    }
  }
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, x, 64));
  if (lane == 0) wmax[wave] = top;
  __syncthreads();
  top = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));
  const unsigned b = scale_byte(top);
  const float inv = __uint_as_float((254u - b) << 23);      // 1 / s, a power of two of the normal range (b is 1 .. 247)
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = i * 8 + (tid >> 5);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][0] * inv, v[i][1] * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][2] * inv, v[i][3] * inv, w, true);
    if (r0 + r < a.n) *reinterpret_cast<int*>(a.q + (int64_t)(r0 + r) * a.ldq + c0 + c) = w;
#pragma unroll
    for (int j = 0; j < 4; ++j) tile[(c + j) * (BLOCK + 4) + r] = (uint8_t)(w >> (8 * j));
  }
  if (tid == 0) a.s[(int64_t)blockIdx.y * a.lds + blockIdx.x] = (uint8_t)b;
  if (!a.qt) return;
  if (tid == 0) a.st[(int64_t)blockIdx.x * a.ldst + blockIdx.y] = (uint8_t)b;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int cc = i * 8 + (tid >> 5);
    if (c0 + cc < a.m)
      *reinterpret_cast<int*>(a.qt + (int64_t)(c0 + cc) * a.ldqt + r0 + c) = *reinterpret_cast<const int*>(tile + cc * (BLOCK + 4) + c);
  }
}

}  // namespace

namespace slimfp8 {

slim_status quantize(slim_ctx* ctx, const char* name, slim_dtype x_dtype, const Activations* a, int count) {
  if (count == 1 && !a->cols_q) {
    const int units = slim_cdiv(a->cols, 512);
    const int64_t waves = ((int64_t)a->rows * units + RQ_UNITS - 1) / RQ_UNITS;
    if (waves > (1ll << 26) - 4)                                // (a launch has fewer than 2^32 threads)
      return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: %d rows of %d channels are too many for one call", name, a->rows, a->cols);
    const dim3 grid(slim_cdiv(waves, RQ_THREADS / 64));
    if (x_dtype == SLIM_F16)
      SLIM_LAUNCH(ctx, name, fp8_rows<__half>, grid, dim3(RQ_THREADS), 0, static_cast<const __half*>(a->X), a->ldx, a->rows, a->cols, units,
                  a->rows_q, a->rows_s, quantized_ld(a->cols), scales_ld(a->cols));
    else
      SLIM_LAUNCH(ctx, name, fp8_rows<__hip_bfloat16>, grid, dim3(RQ_THREADS), 0, static_cast<const __hip_bfloat16*>(a->X), a->ldx, a->rows,
                  a->cols, units, a->rows_q, a->rows_s, quantized_ld(a->cols), scales_ld(a->cols));
    return SLIM_OK;
  }
  TileArgs ta = {};
  int tiles = 0;
  for (int i = 0; i < count; ++i) {
    ta.a[i] = a[i];
    ta.tiles_c[i] = slim_cdiv(a[i].cols, BLOCK);
    ta.tiles[i] = ta.tiles_c[i] * slim_cdiv(a[i].rows, BLOCK);
    tiles += ta.tiles[i];
  }
  if (x_dtype == SLIM_F16)
    SLIM_LAUNCH(ctx, name, (fp8_tiles<__half, false>), dim3(tiles), dim3(256), 0, ta);
  else
    SLIM_LAUNCH(ctx, name, (fp8_tiles<__hip_bfloat16, false>), dim3(tiles), dim3(256), 0, ta);
  return SLIM_OK;
}

slim_status quantize_gradient(slim_ctx* ctx, const char* name, slim_dtype x_dtype, const Activations (&a)[2], const ActGradient& g) {
  TileArgs ta = {};
  ta.g = g;
  int tiles = 0;
  for (int i = 0; i < 2; ++i) {
    ta.a[i] = a[i];
    ta.tiles_c[i] = slim_cdiv(a[i].cols, BLOCK);
    ta.tiles[i] = ta.tiles_c[i] * slim_cdiv(a[i].rows, BLOCK);
    tiles += ta.tiles[i];
  }
  if (x_dtype == SLIM_F16)
    SLIM_LAUNCH(ctx, name, (fp8_tiles<__half, true>), dim3(tiles), dim3(256), 0, ta);
  else
    SLIM_LAUNCH(ctx, name, (fp8_tiles<__hip_bfloat16, true>), dim3(tiles), dim3(256), 0, ta);
  return SLIM_OK;
}

slim_status join_columns(slim_ctx* ctx, const char* name, const float* sums, int parts, int cols, void* out, slim_dtype dtype) {
  SLIM_LAUNCH(ctx, name, fp8_join_columns, dim3(slim_cdiv(cols, 32)), dim3(1024), 0, sums, parts, cols, out, (int)dtype);
  return SLIM_OK;
}

}  // namespace slimfp8

extern "C" slim_status slim_fp8_quantize_weights(slim_ctx* ctx, const void* W, slim_dtype w_dtype, int n, int m, int64_t ldw, uint8_t* q,
                                                 int64_t ldq, uint8_t* s, int64_t lds, uint8_t* qt, int64_t ldqt, uint8_t* st,
                                                 int64_t ldst) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  SLIM_REQUIRE(ctx, W && q && s && (!qt == !st), "slim_fp8_quantize_weights: null pointer");
  SLIM_REQUIRE(ctx, n > 0 && m > 0 && ldw >= m, "slim_fp8_quantize_weights: n = %d, m = %d, ldw = %lld", n, m, (long long)ldw);
  if (w_dtype != SLIM_F16 && w_dtype != SLIM_BF16 && w_dtype != SLIM_F32)
    return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "slim_fp8_quantize_weights: W is F16, BF16 or F32");
  SLIM_REQUIRE(ctx, ldq >= padded(m) && ldq % BLOCK == 0 && lds >= slim_cdiv(m, BLOCK) && lds % 4 == 0,
               "slim_fp8_quantize_weights: rows of q are whole blocks of 128 (ldq = %lld), rows of s whole words (lds = %lld)", (long long)ldq,
               (long long)lds);
  SLIM_REQUIRE(ctx, !qt || (ldqt >= padded(n) && ldqt % BLOCK == 0 && ldst >= slim_cdiv(n, BLOCK) && ldst % 4 == 0),
               "slim_fp8_quantize_weights: rows of qt are whole blocks of 128 (ldqt = %lld), rows of st whole words (ldst = %lld)",
               (long long)ldqt, (long long)ldst);
  SLIM_REQUIRE(ctx, slim_aligned16(q) && (!qt || slim_aligned16(qt)) && ((uintptr_t)s & 3u) == 0 && ((uintptr_t)st & 3u) == 0,
               "slim_fp8_quantize_weights: q and qt are 16-byte aligned, s and st 4-byte");
  const int nb = slim_cdiv(n, BLOCK), mb = slim_cdiv(m, BLOCK);
  if (nb > 65535) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "slim_fp8_quantize_weights: at most 65535 blocks of rows, n = %d", n);
  const WeightArgs a = {W, ldw, ldq, lds, ldqt, ldst, n, m, q, s, qt, st};
  const dim3 grid(mb, nb);
  if (w_dtype == SLIM_F16)
    SLIM_LAUNCH(ctx, "fp8_weights", fp8_weights<__half>, grid, dim3(256), 0, a);
  else if (w_dtype == SLIM_BF16)
    SLIM_LAUNCH(ctx, "fp8_weights", fp8_weights<__hip_bfloat16>, grid, dim3(256), 0, a);
  else
    SLIM_LAUNCH(ctx, "fp8_weights", fp8_weights<float>, grid, dim3(256), 0, a);
  return SLIM_OK;
}
