// Shared by the kernels of the 8-bit linear layer: the quantiser of blocks of 128 and the scaled matrix product.
//
// Quantiser: a = largest finite |x| of a block, s = the smallest power of two >= 2^-126 with a <= 448 s, stored are the e4m3 numbers
// nearest to x / s (ties to even) and the byte log2(s) + 127.  448 = 1.75 * 2^8, so the byte is the exponent field of a, less 8, plus
// one if a's mantissa is above 1.75: one addition carries it.  That byte is what the matrix cores take as the scale of 32 elements of
// an operand (v_mfma_scale_*_f8f6f4), so the scales cost the product nothing and the sums run over the whole contraction in fp32.
#pragma once

#include "slim_device.h"
#include "slim_internal.h"

namespace slimfp8 {

using namespace slimdev;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v2s __attribute__((ext_vector_type(2)));
typedef unsigned short v2u __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr int BLOCK = 128;

inline int64_t padded(int64_t m) { return (m + BLOCK - 1) / BLOCK * BLOCK; }
// Rows of quantised activations are an odd number of blocks apart: a tile's rows at a multiple of 4 KiB share few of the L2's channels
// (8192 x 28672, 4096 tokens: 789 us; 28544 channels: 754).
__host__ __device__ inline int64_t quantized_ld(int64_t m) { return ((m + BLOCK - 1) / BLOCK | 1) * BLOCK; }
inline int64_t scales_ld(int64_t m) { return (slim_cdiv(m, BLOCK) + 3) / 4 * 4; }

// 16-bit types: the pattern of infinity, and the float that a pattern stands for
template <typename T>
struct Half16;
template <>
struct Half16<__half> {
  static constexpr unsigned INF = 0x7c00u;
  static __device__ __forceinline__ unsigned float_bits(unsigned h) {
    return __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)h));
  }
};
template <>
struct Half16<__hip_bfloat16> {
  static constexpr unsigned INF = 0x7f80u;
  static __device__ __forceinline__ unsigned float_bits(unsigned h) { return h << 16; }
};

// the stored scale of a block whose largest finite magnitude has these float bits
__device__ __forceinline__ unsigned scale_byte(unsigned a) { return (unsigned)max((int)((a + 0x1fffffu) >> 23) - 8, 1); }

__device__ __forceinline__ unsigned max_u16x2(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(v2u, a), __builtin_bit_cast(v2u, b)));
}
// the magnitudes of two 16-bit values, zero for what is not finite
template <typename T>
__device__ __forceinline__ unsigned finite_x2(unsigned v) {
  const unsigned lo = v & 0x7fffu, hi = (v >> 16) & 0x7fffu;
  return (lo < Half16<T>::INF ? lo : 0u) | (hi < Half16<T>::INF ? hi << 16 : 0u);
}
// largest magnitudes (the even and the odd places) of N pairs
template <int N>
__device__ __forceinline__ unsigned amax_x2(const unsigned (&v)[N]) {
  unsigned m = v[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < N; ++i) m = max_u16x2(m, v[i] & 0x7fff7fffu);
  return m;
}
template <typename T, int N>
__device__ __forceinline__ unsigned amax_finite_x2(const unsigned (&v)[N]) {
  unsigned m = finite_x2<T>(v[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) m = max_u16x2(m, finite_x2<T>(v[i]));
  return m;
}
__device__ __forceinline__ unsigned larger_half(unsigned m) { return max(m & 0xffffu, m >> 16); }

// four values (two pairs) over 2^(byte - 127) as e4m3 numbers; what is not finite becomes NaN
template <typename T>
__device__ __forceinline__ unsigned to_e4m3(unsigned a, unsigned b, float scale) {
  v2s r = {0, 0};
  if constexpr (sizeof(T) == 2 && Half16<T>::INF == 0x7f80u) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, b), scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(v2h, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(v2h, b), scale, true);
  }
  return __builtin_bit_cast(unsigned, r);
}

// Eight stored numbers times their scale as bf16, which holds them exactly (four significant bits, the exponents of fp32; what is below
// 2^-126 may count as zero): the operand of the products whose sums keep 24 bits.  The matrix cores' own e4m3 products are summed in
// groups of eight in which only about 13 bits below the largest product are kept (measured: of 2^16 - 2^16 + 2^k they lose 2^2 and less;
// the bf16 ones 2^-9 and less): 1.5e-5 to 7e-5 of a result's norm, which is below the 2.1e-4 and 1.7e-3 of rounding it to fp16 and bf16, but far
// above the rounding to fp32, and no smaller in an element whose products cancel.
__device__ __forceinline__ v8bf dequantized(int lo, int hi, float scale) {
  const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true),
             c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// byte J of a word of scales as a float
template <int J>
__device__ __forceinline__ float scale_of(int word) { return __uint_as_float((((unsigned)word >> (8 * J)) & 255u) << 23); }

// eight 16-bit values from p on, of which `left` exist (the others read as zero); p may have any alignment of its type
template <typename T>
__device__ __forceinline__ void load8(const T* p, int left, unsigned (&v)[4]) {
  if (left >= 8) {
    __builtin_memcpy(v, p, 16);
  } else {
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned lo = 2 * i < left ? q[2 * i] : 0u, hi = 2 * i + 1 < left ? q[2 * i + 1] : 0u;
      v[i] = lo | hi << 16;
    }
  }
}

// The same, row_end_shift<8> pending (which with fewer than 8 columns has nothing to do).
template <typename T>
__device__ __forceinline__ void fetch8(const T* p, int left, int cols, unsigned (&v)[4]) {
  if (cols >= 8) __builtin_memcpy(v, row_end_address<8>(p, left), 16);
  else load8(p, left, v);
}

// ---- what fp8_gemm.hip offers the entry points ---------------------------------------------------------------
// rows x K e4m3 numbers (whole blocks of K, ld bytes apart), and a scale for every block: that of row r is in row r >> shift
struct Operand {
  const uint8_t* q;
  const uint8_t* s;
  int64_t ld, lds;
  int rows, shift;
};
// C[b][a] = sum over nk blocks of A[a] . B[b]
struct Product {
  Operand a, b;
  void* c;
  int64_t ldc;
  slim_dtype c_dtype;
  int nk;
};
// bytes of workspace of a set of products, enough too for those of fewer rows and shorter contractions; 256-byte multiples
size_t gemm_workspace(const Product* p, int count, int num_cus);
slim_status gemm(slim_ctx* ctx, const char* name, const Product* p, int count);

// ---- and fp8_quant.hip: activations to e4m3 -------------------------------------------------------------------
// X (rows x cols, 16 bits).  `rows_q`: in blocks along the rows (rows of quantized_ld(cols)); `cols_q`: transposed, in blocks of 128 rows
// (rows of quantized_ld(rows)); either may be null, not both.  Their scales have rows of scales_ld(cols) and scales_ld(rows) bytes.
struct Activations {
  const void* X;
  int64_t ldx;
  int rows, cols;
  uint8_t *rows_q, *rows_s, *cols_q, *cols_s;
};
slim_status quantize(slim_ctx* ctx, const char* name, slim_dtype x_dtype, const Activations* a, int count);

// ---- and fp8_few.hip: few tokens, or little work, in one launch -----------------------------------------------------
bool takes_few_tokens(int n, int m, int t, int ncu);
slim_status few_tokens(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& w, int m, void* Y,
                       slim_dtype y_dtype, int64_t ldy);

// value to one of the output types, rounded to nearest even
__device__ __forceinline__ unsigned short to_16(float v, bool bf16) {
  if (bf16) return __builtin_bit_cast(unsigned short, (__bf16)v);
  return __builtin_bit_cast(unsigned short, (_Float16)v);
}

}  // namespace slimfp8
