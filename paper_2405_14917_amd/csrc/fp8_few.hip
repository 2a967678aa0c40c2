// The 8-bit linear layer for the few tokens of a decoding step (up to 16), in one launch: Y = Q(X) W^T.
//
// Bound by reading the weights once.  A workgroup takes 16 RT output rows; its wavefronts share the blocks of channels, four blocks
// (512 channels, one word of four scales) at a time, so that a wavefront has 8 KiB per 16 rows in flight; their sums are joined in LDS
// in a fixed order.  The rows of W are the first operand of v_mfma_f32_16x16x32_bf16, the tokens the second, both as the exact products of number and scale (the
// matrix cores are idle here, so that the sums may as well keep 24 bits for every type of output): a lane holds one token's channels 16 c .. + 15 and 64 + 16 c .. + 15 of a block (c = lane / 16; the contraction may run in any order), so
// that a load of the weights covers 64 consecutive bytes of 16 rows.  The activations are quantised in registers by every wavefront for the blocks
// that it multiplies: no second launch, and nothing is written.  Their loads come first, so that they are converted while the weights are
// still on their way.
#include "fp8_device.h"

namespace {

using namespace slimfp8;

struct FewArgs {
  const void* X;
  const uint8_t* q;
  const uint8_t* s;
  void* Y;
  int64_t ldx, ldq, lds, ldy;
  int t, n, m, mb;                  // mb: blocks of channels
  int y_dtype;
};

template <typename T, int RT>
__global__ __launch_bounds__(512) void fp8_few(FewArgs a) {
  constexpr int ROWS = 16 * RT, LD = ROWS + 4;                 // floats per token of a wavefront's sums
  extern __shared__ __align__(16) float part[];                // [wavefront][token][row]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), nw = blockDim.x >> 6;
  const int l16 = lane & 15, c = lane >> 4;
  const int row0 = blockIdx.x * ROWS;
  const bool live = l16 < a.t;
  const T* xrow = static_cast<const T*>(a.X) + (int64_t)min(l16, a.t - 1) * a.ldx + c * 16;
  const uint8_t* wrow[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) wrow[r] = a.q + (int64_t)min(row0 + r * 16 + l16, a.n - 1) * a.ldq + c * 16;
  const uint8_t* srow = a.s + (int64_t)(row0 / BLOCK) * a.lds;  // (ROWS divides 128)
  v4f acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = v4f{0.f, 0.f, 0.f, 0.f};

  const int steps = (a.mb + 3) / 4;
  for (int st = wave; st < steps; st += nw) {
    unsigned x[4][2][8];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int ch = (st * 4 + j) * BLOCK + h * 64;          // (behind the last channel everything reads as zero)
        unsigned (&v)[8] = x[j][h];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0u;
        if (live) {
          load8(xrow + ch, a.m - ch - c * 16, *reinterpret_cast<unsigned(*)[4]>(&v[0]));
          load8(xrow + ch + 8, a.m - ch - c * 16 - 8, *reinterpret_cast<unsigned(*)[4]>(&v[4]));
        }
      }
    uint4 w[4][RT][2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h)                            // (a block behind the last: the last one again, times zeros)
          w[j][r][h] = *reinterpret_cast<const uint4*>(wrow[r] + (int64_t)min(st * 4 + j, a.mb - 1) * BLOCK + h * 64);
    int ws = *reinterpret_cast<const int*>(srow + st * 4);
    if (st * 4 + 4 > a.mb) ws &= (1 << (8 * (a.mb - st * 4))) - 1;      // (what pads a row of scales may be anything, a NaN's code too)
    auto block = [&](auto index) {
      constexpr int J = decltype(index)::value;
      unsigned (&v)[16] = *reinterpret_cast<unsigned(*)[16]>(&x[J][0][0]);
      unsigned mx = amax_x2(v);
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
      unsigned top = larger_half(mx);
      if (__builtin_expect(__any(top >= Half16<T>::INF), 0)) {
        mx = amax_finite_x2<T>(v);
        mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
        mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
        top = larger_half(mx);
      }
      const float sx = __uint_as_float(scale_byte(Half16<T>::float_bits(top)) << 23), sw = scale_of<J>(ws);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const v8bf xb = dequantized((int)to_e4m3<T>(v[4 * i], v[4 * i + 1], sx), (int)to_e4m3<T>(v[4 * i + 2], v[4 * i + 3], sx), sx);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const uint4 wv = w[J][r][i >> 1];
          acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequantized((int)((i & 1) ? wv.z : wv.x), (int)((i & 1) ? wv.w : wv.y), sw), xb, acc[r], 0, 0, 0);
        }
      }
    };
    block(std::integral_constant<int, 0>());
    block(std::integral_constant<int, 1>());
    block(std::integral_constant<int, 2>());
    block(std::integral_constant<int, 3>());
  }
  // a lane holds rows 4 c .. + 3 of its token
#pragma unroll
  for (int r = 0; r < RT; ++r) *reinterpret_cast<v4f*>(part + (wave * 16 + l16) * LD + r * 16 + c * 4) = acc[r];
  __syncthreads();
  const int last = min(ROWS, a.n - row0);
  for (int e = threadIdx.x; e < a.t * ROWS; e += blockDim.x) {
    const int tok = e / ROWS, r = e % ROWS;
    float sum = 0.f;
    for (int i = 0; i < nw; ++i) sum += part[(i * 16 + tok) * LD + r];
    if (r < last) {
      const int64_t at = (int64_t)tok * a.ldy + row0 + r;
      if (a.y_dtype == SLIM_F32) static_cast<float*>(a.Y)[at] = sum;
      else static_cast<unsigned short*>(a.Y)[at] = to_16(sum, a.y_dtype == SLIM_BF16);
    }
  }
}

template <typename T>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  // Wavefronts: one per 512 channels, eight at most.
  const int steps = (a.mb + 3) / 4;
  const int nw = std::min(8, steps);
  const bool wide = slim_cdiv(a.n, 32) >= 2 * ctx->num_cus;
  const int rows = wide ? 32 : 16;
  const dim3 grid(slim_cdiv(a.n, rows)), block(64 * nw);
  const size_t shmem = sizeof(float) * (size_t)nw * 16 * (rows + 4);
  if (wide)
    SLIM_LAUNCH(ctx, "fp8_linear_few", (fp8_few<T, 2>), grid, block, shmem, a);
  else
    SLIM_LAUNCH(ctx, "fp8_linear_few", (fp8_few<T, 1>), grid, block, shmem, a);
  return SLIM_OK;
}

}  // namespace

namespace slimfp8 {

slim_status few_tokens(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& w, int m, void* Y,
                       slim_dtype y_dtype, int64_t ldy) {
  const FewArgs a = {X, w.q, w.s, Y, ldx, w.ld, w.lds, ldy, t, w.rows, m, slim_cdiv(m, BLOCK), (int)y_dtype};
  return x_dtype == SLIM_F16 ? launch<__half>(ctx, a) : launch<__hip_bfloat16>(ctx, a);
}

}  // namespace slimfp8
