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
__global__ __launch_bounds__(RT == 1 ? 1024 : 512) void fp8_few(FewArgs a) {
  constexpr int ROWS = 16 * RT, LD = ROWS + 4;                 // floats per token of a wavefront's sums
  extern __shared__ __align__(16) float part[];                // [wavefront][token][row]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), nw = blockDim.x >> 6;
  const int l16 = lane & 15, c = lane >> 4;
  const int row0 = blockIdx.x * ROWS;
  // (tokens that do not exist are the last one again: their columns of the product are not stored)
  const T* xrow = static_cast<const T*>(a.X) + (int64_t)min(l16, a.t - 1) * a.ldx + c * 16;
  const uint8_t* wrow[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) wrow[r] = a.q + (int64_t)min(row0 + r * 16 + l16, a.n - 1) * a.ldq + c * 16;
  const uint8_t* srow = a.s + (int64_t)(row0 / BLOCK) * a.lds;  // (ROWS divides 128)
  v4f acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = v4f{0.f, 0.f, 0.f, 0.f};

  const int steps = (a.mb + 3) / 4;
  unsigned x[4][16];
  uint4 w[4][RT][2];
  int ws;
  auto load_x = [&](int j, int st) {
    const int ch = (st * 4 + j) * BLOCK;
    if (ch + BLOCK <= a.m) {
#pragma unroll
      for (int h = 0; h < 4; ++h) __builtin_memcpy(&x[j][4 * h], xrow + ch + (h >> 1) * 64 + (h & 1) * 8, 16);
    } else {                                                    // (behind the last channel everything reads as zero)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int at = ch + (h >> 1) * 64 + (h & 1) * 8;
        fetch8(xrow + at, a.m - at - c * 16, a.m, *reinterpret_cast<unsigned(*)[4]>(&x[j][4 * h]));
      }
    }
  };
  auto end_x = [&](int j, int st) {
    const int ch = (st * 4 + j) * BLOCK;
    if (ch + BLOCK > a.m && a.m >= 8)
#pragma unroll
      for (int h = 0; h < 4; ++h) row_end_shift<8>(*reinterpret_cast<unsigned(*)[4]>(&x[j][4 * h]), a.m - ch - (h >> 1) * 64 - (h & 1) * 8 - c * 16);
  };
  auto load_w = [&](int j, int st) {
    const int64_t at = (int64_t)min(st * 4 + j, a.mb - 1) * BLOCK;   // (a block behind the last: the last one again, times zeros)
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[j][r][h] = *reinterpret_cast<const uint4*>(wrow[r] + at + h * 64);
  };
  auto load_s = [&](int st) {
    int v = *reinterpret_cast<const int*>(srow + st * 4);
    if (st * 4 + 4 > a.mb) v &= (1 << (8 * (a.mb - st * 4))) - 1;      // (what pads a row of scales may be anything, a NaN's code too)
    return v;
  };
  auto block = [&](auto index, int st) {
    constexpr int J = decltype(index)::value;
    end_x(J, st);
    unsigned mx = amax_x2(x[J]);
    mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
    mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
    unsigned top = larger_half(mx);
    if (__builtin_expect(__any(top >= Half16<T>::INF), 0)) {
      mx = amax_finite_x2<T>(x[J]);
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
      top = larger_half(mx);
    }
    const float sx = __uint_as_float(scale_byte(Half16<T>::float_bits(top)) << 23), sw = scale_of<J>(ws);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const v8bf xb = dequantized((int)to_e4m3<T>(x[J][4 * i], x[J][4 * i + 1], sx), (int)to_e4m3<T>(x[J][4 * i + 2], x[J][4 * i + 3], sx), sx);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint4 wv = w[J][r][i >> 1];
        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequantized((int)((i & 1) ? wv.z : wv.x), (int)((i & 1) ? wv.w : wv.y), sw), xb, acc[r], 0, 0, 0);
      }
    }
  };
  if (wave < steps) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      load_x(j, wave);
      load_w(j, wave);
    }
    ws = load_s(wave);
  }
  for (int st = wave; st < steps; st += nw) {
    const int next = st + nw;
    const int ws_next = next < steps ? load_s(next) : 0;
    auto refill = [&](int j) {                                  // a block that is used up makes room for the one four on
      if (next < steps) {
        load_x(j, next);
        load_w(j, next);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    block(std::integral_constant<int, 0>(), st);
    refill(0);
    block(std::integral_constant<int, 1>(), st);
    refill(1);
    block(std::integral_constant<int, 2>(), st);
    refill(2);
    block(std::integral_constant<int, 3>(), st);
    refill(3);
    ws = ws_next;
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

template <typename T, int RT>
slim_status launch(slim_ctx* ctx, const FewArgs& a, int nw) {
  constexpr int ROWS = 16 * RT;
  SLIM_LAUNCH(ctx, "fp8_linear_few", (fp8_few<T, RT>), dim3(slim_cdiv(a.n, ROWS)), dim3(64 * nw), sizeof(float) * (size_t)nw * 16 * (ROWS + 4), a);
  return SLIM_OK;
}

template <typename T>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  const int steps = (a.mb + 3) / 4, ncu = ctx->num_cus;
  const int rt = slim_cdiv(a.n, 64) * 5 >= ncu * 3 ? 4 : slim_cdiv(a.n, 32) * 5 >= ncu * 3 ? 2 : 1;
  const int nw = std::max(1, std::min(steps, std::max(2, std::min(rt == 1 ? 16 : 8, 8 * ncu / slim_cdiv(a.n, 16 * rt)))));
  return rt == 4 ? launch<T, 4>(ctx, a, nw) : rt == 2 ? launch<T, 2>(ctx, a, nw) : launch<T, 1>(ctx, a, nw);
}

}  // namespace

namespace slimfp8 {

slim_status few_tokens(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& w, int m, void* Y,
                       slim_dtype y_dtype, int64_t ldy) {
  const FewArgs a = {X, w.q, w.s, Y, ldx, w.ld, w.lds, ldy, t, w.rows, m, slim_cdiv(m, BLOCK), (int)y_dtype};
  return x_dtype == SLIM_F16 ? launch<__half>(ctx, a) : launch<__hip_bfloat16>(ctx, a);
}

}  // namespace slimfp8
