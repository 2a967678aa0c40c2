// The 8-bit linear layer for the few tokens of a decoding step (16 to a workgroup), and for small layers, in one launch: Y = Q(X) W^T.
//
// Bound by reading the weights once.  A workgroup takes 16 RT output rows; its eight wavefronts share the blocks of channels and
// their sums are joined in LDS in a fixed order.  The rows of W are the first operand of v_mfma_f32_16x16x32_bf16, the tokens the second,
// both as the exact products of number and scale (the matrix cores are idle here, so that the sums may as well keep 24 bits for every
// type of output): a lane holds one token's channels 16 c .. + 15 and 64 + 16 c .. + 15 of a block (c = lane / 16; the contraction may run in
// any order), so that a load of the weights covers 64 consecutive bytes of 16 rows.  The activations are quantised in registers by every
// wavefront for the blocks that it multiplies: no second launch, and nothing is written.  A block's loads come before its predecessor's
// products end and after its registers are free: with eight wavefronts on a CU deeper rings of registers gained nothing (46.6 and 44.4 us).
//
// 28672 x 8192: 44 us for 16 tokens, 43 for one (5.4 and 5.5 TB/s; a kernel that only reads reaches 6.3 to 7.0).
#include "fp8_device.h"

namespace {

using namespace slimfp8;

constexpr int FEW_WAVES = 8, FEW_RT = 7;

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
__global__ __launch_bounds__(64 * FEW_WAVES) void fp8_few(FewArgs a) {
  constexpr int ROWS = 16 * RT, LD = ROWS + 4;                 // floats per token of a wavefront's sums
  extern __shared__ __align__(16) float part[];                // [wavefront][token][row]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), nw = blockDim.x >> 6;
  const int l16 = lane & 15, c = lane >> 4;
  const int row0 = blockIdx.x * ROWS, tok0 = blockIdx.y * 16, tn = min(16, a.t - tok0);
  // (tokens that do not exist are the last one again: their columns of the product are not stored)
  const T* xrow = static_cast<const T*>(a.X) + (int64_t)min(tok0 + l16, a.t - 1) * a.ldx + c * 16;
  const uint8_t* wrow[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) wrow[r] = a.q + (int64_t)min(row0 + r * 16 + l16, a.n - 1) * a.ldq + c * 16;
  // the workgroup's rows lie in one or two blocks of 128: the first `cut` sixteens in the first
  const int cut = (BLOCK - row0 % BLOCK) / 16;
  const uint8_t* srow[2] = {a.s + (int64_t)(row0 / BLOCK) * a.lds, a.s + (int64_t)min(row0 / BLOCK + 1, (a.n - 1) / BLOCK) * a.lds};
  v4f acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = v4f{0.f, 0.f, 0.f, 0.f};

  const int per = (a.mb + nw - 1) / nw, first = wave * per, end = min(a.mb, first + per);
  unsigned x[16];
  uint4 w[RT][2];
  auto load = [&](int kb) {
    const int ch = kb * BLOCK;
    if (ch + BLOCK <= a.m) {
#pragma unroll
      for (int h = 0; h < 4; ++h) __builtin_memcpy(&x[4 * h], xrow + ch + (h >> 1) * 64 + (h & 1) * 8, 16);
    } else {                                                    // (behind the last channel everything reads as zero)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int at = ch + (h >> 1) * 64 + (h & 1) * 8;
        fetch8(xrow + at, a.m - at - c * 16, a.m, *reinterpret_cast<unsigned(*)[4]>(&x[4 * h]));
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[r][h] = *reinterpret_cast<const uint4*>(wrow[r] + ch + h * 64);
  };
  auto block = [&](int kb) {
    const int ch = kb * BLOCK;
    if (ch + BLOCK > a.m && a.m >= 8)
#pragma unroll
      for (int h = 0; h < 4; ++h) row_end_shift<8>(*reinterpret_cast<unsigned(*)[4]>(&x[4 * h]), a.m - ch - (h >> 1) * 64 - (h & 1) * 8 - c * 16);
    float sw[2];
#pragma unroll
    for (int i = 0; i < (128 % (16 * RT) ? 2 : 1); ++i)
      sw[i] = __uint_as_float(((*reinterpret_cast<const unsigned*>(srow[i] + (kb & ~3)) >> (8 * (kb & 3))) & 255u) << 23);
    unsigned mx = amax_x2(x);
    mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
    mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
    unsigned top = larger_half(mx);
    if (__builtin_expect(__any(top >= Half16<T>::INF), 0)) {
      mx = amax_finite_x2<T>(x);
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 16, 64));
      mx = max_u16x2(mx, (unsigned)__shfl_xor((int)mx, 32, 64));
      top = larger_half(mx);
    }
    const float sx = __uint_as_float(scale_byte(Half16<T>::float_bits(top)) << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const v8bf xb = dequantized((int)to_e4m3<T>(x[4 * i], x[4 * i + 1], sx), (int)to_e4m3<T>(x[4 * i + 2], x[4 * i + 3], sx), sx);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint4 wv = w[r][i >> 1];
        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequantized((int)((i & 1) ? wv.z : wv.x), (int)((i & 1) ? wv.w : wv.y), 128 % (16 * RT) && r >= cut ? sw[1] : sw[0]), xb, acc[r], 0, 0, 0);
      }
    }
  };
  if (first < end) load(first);
  for (int k = first; k < end; ++k) {
    block(k);
    if (k + 1 < end) load(k + 1);
  }
  // a lane holds rows 4 c .. + 3 of its token
#pragma unroll
  for (int r = 0; r < RT; ++r) *reinterpret_cast<v4f*>(part + (wave * 16 + l16) * LD + r * 16 + c * 4) = acc[r];
  __syncthreads();
  const int last = min(ROWS, a.n - row0);
  for (int e = threadIdx.x; e < tn * ROWS; e += blockDim.x) {
    const int tok = e / ROWS, r = e % ROWS;
    float sum = 0.f;
    for (int i = 0; i < nw; ++i) sum += part[(i * 16 + tok) * LD + r];
    if (r < last) {
      const int64_t at = (int64_t)(tok0 + tok) * a.ldy + row0 + r;
      if (a.y_dtype == SLIM_F32) static_cast<float*>(a.Y)[at] = sum;
      else static_cast<unsigned short*>(a.Y)[at] = to_16(sum, a.y_dtype == SLIM_BF16);
    }
  }
}

template <typename T, int RT>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  constexpr int ROWS = 16 * RT;
  const int nw = std::min(FEW_WAVES, a.mb);
  SLIM_LAUNCH(ctx, "fp8_linear_few", (fp8_few<T, RT>), dim3(slim_cdiv(a.n, ROWS), slim_cdiv(a.t, 16)), dim3(64 * nw), sizeof(float) * (size_t)nw * 16 * (ROWS + 4), a);
  return SLIM_OK;
}

// Tiles of 16 x 16 outputs that the busiest CU gets with `rt` sixteens of rows per workgroup
int64_t busiest(int n, int t, int ncu, int rt) { return ((int64_t)slim_cdiv(n, 16 * rt) * slim_cdiv(t, 16) + ncu - 1) / ncu * rt; }
int64_t least_busiest(int n, int t, int ncu) {
  int64_t least = busiest(n, t, ncu, 1);
  for (int r = 2; r <= FEW_RT; ++r) least = std::min(least, busiest(n, t, ncu, r));
  return least;
}
// Sixteens of rows per workgroup: what the busiest CU gets is to be as small as it can (within 8 %), then as many as possible, since
// every workgroup quantises the activations anew.  28672 x 8192, 16 tokens: seven (256 workgroups) 44 us, four (448) 53; 11008 x 4096: three
// (230) 11.8, four 13.5; 32000 x 4096: four 30, eight (250, and one wavefront's registers fewer) 33.
int sixteens(int n, int t, int ncu) {
  const int64_t least = least_busiest(n, t, ncu);
  int rt = 1;
  for (int r = 2; r <= FEW_RT; ++r)
    if (busiest(n, t, ncu, r) * 100 <= least * 108) rt = r;
  return rt;
}

template <typename T>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  switch (sixteens(a.n, a.t, ctx->num_cus)) {
    case 1: return launch<T, 1>(ctx, a);
    case 2: return launch<T, 2>(ctx, a);
    case 3: return launch<T, 3>(ctx, a);
    case 4: return launch<T, 4>(ctx, a);
    case 5: return launch<T, 5>(ctx, a);
    case 6: return launch<T, 6>(ctx, a);
    default: return launch<T, FEW_RT>(ctx, a);
  }
}

}  // namespace

namespace slimfp8 {

// Up to 16 tokens; more while the busiest CU has no more than 64 blocks of 16 x 16 x 128 to multiply, where the two launches of the other
// way cost more than the work.  Of 37 shapes with 1 to 28 blocks a wavefront in a row, host's share included: up to 64 blocks one launch is the
// faster by 1 to 6 us (384 x 384, 3000 tokens, 54 blocks: 9.3 and 11.8; 4096 x 4096, 32 tokens, 64: 10.1 and 15.0; 512 x 8192, 128 tokens,
// 64, the deepest: 13.5 and 14.5; the other way only 2048 x 128, 2000 tokens, 63: 12.5 and 11.7); from 66 to 126 either one is (1000 x 3000, 200
// tokens, 96: 10.8 and 15.1; 700 x 700, 1000 tokens, 66: 14.3 and 11.5; 2048 x 256, 2000 tokens, 126: 17.4 and 11.7); from 128 on two are, but
// for one shape.
bool takes_few_tokens(int n, int m, int t, int ncu) {
  return t <= 16 || (t <= 65535 * 16 && least_busiest(n, t, ncu) * slim_cdiv(m, BLOCK) <= 64);
}

slim_status few_tokens(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& w, int m, void* Y,
                       slim_dtype y_dtype, int64_t ldy) {
  const FewArgs a = {X, w.q, w.s, Y, ldx, w.ld, w.lds, ldy, t, w.rows, m, slim_cdiv(m, BLOCK), (int)y_dtype};
  return x_dtype == SLIM_F16 ? launch<__half>(ctx, a) : launch<__hip_bfloat16>(ctx, a);
}

}  // namespace slimfp8
