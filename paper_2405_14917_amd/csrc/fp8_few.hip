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
#include "act_device.h"
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
  const uint8_t *xq, *xs;           // the activations' 8-bit form (T = uint8_t)
  int64_t ldxq, ldxs;
  Epilogue e;                       // (FINISH)
  Softmax sm;                       // (SOFTMAX)
};
enum { PLAIN, FINISH, SOFTMAX };    // what becomes of the sums: stored, stored through the epilogue, or what the softmax needs of them

// T = uint8_t: the activations come in 8 bits (rows of whole blocks).
template <typename T, int RT, int MODE>
__global__ __launch_bounds__(64 * FEW_WAVES) void fp8_few(FewArgs a) {
  constexpr int ROWS = 16 * RT, LD = ROWS + 4;                 // floats per token of a wavefront's sums
  constexpr bool Q8 = sizeof(T) == 1;
  extern __shared__ __align__(16) float part[];                // [wavefront][token][row]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), nw = blockDim.x >> 6;
  const int l16 = lane & 15, c = lane >> 4;
  const int row0 = blockIdx.x * ROWS, tok0 = blockIdx.y * 16, tn = min(16, a.t - tok0);
  // (tokens that do not exist are the last one again: their columns of the product are not stored)
  const T* xrow = Q8 ? (const T*)(a.xq + (int64_t)min(tok0 + l16, a.t - 1) * a.ldxq + c * 16)
                     : static_cast<const T*>(a.X) + (int64_t)min(tok0 + l16, a.t - 1) * a.ldx + c * 16;
  const uint8_t* xsrow = Q8 ? a.xs + (int64_t)min(tok0 + l16, a.t - 1) * a.ldxs : nullptr;
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
  unsigned x[Q8 ? 8 : 16];
  uint4 w[RT][2];
  auto load = [&](int kb) {
    const int ch = kb * BLOCK;
    if constexpr (Q8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) __builtin_memcpy(&x[4 * h], xrow + ch + h * 64, 16);
    } else if (ch + BLOCK <= a.m) {
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
    if (!Q8 && ch + BLOCK > a.m && a.m >= 8)
#pragma unroll
      for (int h = 0; h < (Q8 ? 0 : 4); ++h) row_end_shift<8>(*reinterpret_cast<unsigned(*)[4]>(&x[4 * h]), a.m - ch - (h >> 1) * 64 - (h & 1) * 8 - c * 16);
    float sw[2];
#pragma unroll
    for (int i = 0; i < (128 % (16 * RT) ? 2 : 1); ++i)
      sw[i] = __uint_as_float(((*reinterpret_cast<const unsigned*>(srow[i] + (kb & ~3)) >> (8 * (kb & 3))) & 255u) << 23);
    float sx;
    if constexpr (Q8) {
      sx = __uint_as_float((unsigned)xsrow[kb] << 23);
    } else {
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
      sx = __uint_as_float(scale_byte(Half16<T>::float_bits(top)) << 23);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v8bf xb;
      if constexpr (Q8) xb = dequantized((int)x[2 * i], (int)x[2 * i + 1], sx);
      else xb = dequantized((int)to_e4m3<T>(x[4 * i], x[4 * i + 1], sx), (int)to_e4m3<T>(x[4 * i + 2], x[4 * i + 3], sx), sx);
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
  const int last = min(ROWS, a.n - row0);
  // element e of the tile's: row e % ROWS of token e / ROWS
  auto sum_of = [&](int e) {
    const float* p = part + (e / ROWS) * LD + e % ROWS;
    float sum = 0.f;
    for (int i = 0; i < nw; ++i) sum += p[i * 16 * LD];
    return sum;
  };
  if constexpr (MODE == FINISH) {
    // Bias and residual of a thread's elements are fetched before the wavefronts' sums are waited for, and there is one branch for the activation
    // (1000 x 1504, 301 tokens, 8-bit activations, gelu, kept sums: 9.5 -> 9.1 us).
    constexpr int EACH = (16 * ROWS + 64 * FEW_WAVES - 1) / (64 * FEW_WAVES);      // elements of a thread, with all the wavefronts
    for (int e0 = threadIdx.x, first = 1; first || e0 - (int)threadIdx.x < tn * ROWS; e0 += EACH * blockDim.x, first = 0) {
      float v[EACH], b[EACH], res[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int e = e0 + i * blockDim.x, tok = e / ROWS, r = e % ROWS;
        const bool there = tok < tn && r < last;
        b[i] = there && a.e.bias ? from_any(a.e.bias, a.e.bias_dtype, row0 + r) : 0.f;
        res[i] = there && a.e.R ? from_any(a.e.R, a.e.r_dtype, (int64_t)(tok0 + tok) * a.e.ldr + row0 + r) : 0.f;
      }
      if (first) __syncthreads();
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int e = e0 + i * blockDim.x, tok = e / ROWS, r = e % ROWS;
        v[i] = tok < tn ? sum_of(e) + b[i] : 0.f;
        if (a.e.Z && tok < tn && r < last) to_any(a.e.Z, a.y_dtype, (int64_t)(tok0 + tok) * a.e.ldz + row0 + r, v[i]);
      }
      slimact::activate(v, a.e.act);
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int e = e0 + i * blockDim.x, tok = e / ROWS, r = e % ROWS;
        if (tok < tn && r < last) to_any(a.Y, a.y_dtype, (int64_t)(tok0 + tok) * a.ldy + row0 + r, a.e.R ? v[i] + res[i] : v[i]);
      }
    }
    return;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < tn * ROWS; e += blockDim.x) {
    const int tok = e / ROWS, r = e % ROWS;
    const float sum = sum_of(e);
    if constexpr (MODE == SOFTMAX) {
      part[tok * LD + r] = r < last ? sum : -__builtin_inff();      // (the first wavefront's sum, which nobody else reads)
      if (row0 + r < a.sm.keep && r < last) static_cast<float*>(a.Y)[(int64_t)(tok0 + tok) * a.ldy + row0 + r] = sum;
    } else if (r < last) to_any(a.Y, a.y_dtype, (int64_t)(tok0 + tok) * a.ldy + row0 + r, sum);
  }
  if constexpr (MODE == SOFTMAX) {
    __syncthreads();
    for (int tok = wave; tok < tn; tok += nw) {
      const float* z = part + tok * LD;
      const int64_t row = tok0 + tok, at = label_at(a.sm.labels, a.sm.labels64, row) - row0;
      // (the label's own logit counts in neither the maximum nor the sum)
      const float z0 = lane < ROWS && lane != at ? z[lane] : -__builtin_inff(), z1 = lane + 64 < ROWS && lane + 64 != at ? z[lane + 64] : -__builtin_inff();
      const float top = wave_max_f32(fmaxf(z0, z1)), from = top == -__builtin_inff() ? 0.f : top;
      const float sum = wave_sum_f32(__builtin_amdgcn_exp2f((z0 - from) * slimact::LOG2E_HI) + __builtin_amdgcn_exp2f((z1 - from) * slimact::LOG2E_HI));
      if (lane == 0) {
        a.sm.part[row * a.sm.parts + blockIdx.x] = make_float2(top, sum);
        if (at >= 0 && at < last) a.sm.z[row] = z[at];
      }
    }
  }
}

template <typename T, int MODE, int RT>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  constexpr int ROWS = 16 * RT;
  const int nw = std::min(FEW_WAVES, a.mb);
  SLIM_LAUNCH(ctx, "fp8_linear_few", (fp8_few<T, RT, MODE>), dim3(slim_cdiv(a.n, ROWS), slim_cdiv(a.t, 16)), dim3(64 * nw), sizeof(float) * (size_t)nw * 16 * (ROWS + 4), a);
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

template <typename T, int MODE>
slim_status launch(slim_ctx* ctx, const FewArgs& a) {
  switch (sixteens(a.n, a.t, ctx->num_cus)) {
    case 1: return launch<T, MODE, 1>(ctx, a);
    case 2: return launch<T, MODE, 2>(ctx, a);
    case 3: return launch<T, MODE, 3>(ctx, a);
    case 4: return launch<T, MODE, 4>(ctx, a);
    case 5: return launch<T, MODE, 5>(ctx, a);
    case 6: return launch<T, MODE, 6>(ctx, a);
    default: return launch<T, MODE, FEW_RT>(ctx, a);
  }
}

}  // namespace

namespace slimfp8 {

// Up to 16 tokens; more while the busiest CU has no more than 64 blocks of 16 x 16 x 128 to multiply, where the two launches of the other
// way cost more than the work.  Of 37 shapes with 1 to 28 blocks a wavefront in a row, host's share included: up to 64 blocks one launch is the
// faster by 1 to 6 us (384 x 384, 3000 tokens, 54 blocks: 9.3 and 11.8; 4096 x 4096, 32 tokens, 64: 10.1 and 15.0; 512 x 8192, 128 tokens,
// 64, the deepest: 13.5 and 14.5; the other way only 2048 x 128, 2000 tokens, 63: 12.5 and 11.7); from 66 to 126 either one is (1000 x 3000, 200
// tokens, 96: 10.8 and 15.1; 700 x 700, 1000 tokens, 66: 14.3 and 11.5; 2048 x 256, 2000 tokens, 126: 17.4 and 11.7); from 128 on two are, but
// for one shape.  Activations in 8 bits, whose other way is one launch too unless the product is cut, with gelu and kept sums: of 54 shapes up to 64 blocks one is at
// most 1.3 % slower and 26 % faster (1000 x 1504, 301 tokens, 60 blocks: 11.6 and 11.7; 4096 x 4096, 32 tokens: 11.3 and 14.3) but for 636 x 153, 1952 tokens, 40:
// 13.9 and 12.0; from 84 on either one (1000 x 1504, 600 tokens, 120: 12.6 and 11.7).  The head's loss: up to 16 tokens 10 to 59 % faster (32000 x 4096: 23.3 to 28.8
// and 29.8 to 31.6), above them up to 64 blocks up to 51 %, but 19464 x 199, 76 tokens, 48 16.0 and 14.4 and 4169 x 770, 116, 63 17.3 and 13.7.  With its gradients, whose
// activations are quantised anyway: up to 16 tokens 1 to 19 % faster, above them between 13 % faster (728 x 2316, 197 tokens, 57: 34 and 39) and 12 % slower
// (4169 x 770, 116: 52 and 45).
bool takes_few_tokens(int n, int m, int t, int ncu) {
  return t <= 16 || (t <= 65535 * 16 && least_busiest(n, t, ncu) * slim_cdiv(m, BLOCK) <= 64);
}

slim_status few_tokens(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& xq, const Operand& w, int m,
                       const Epilogue* e, void* Y, slim_dtype y_dtype, int64_t ldy) {
  FewArgs a = {X, w.q, w.s, Y, ldx, w.ld, w.lds, ldy, t, w.rows, m, slim_cdiv(m, BLOCK), (int)y_dtype, xq.q, xq.s, xq.ld, xq.lds, {}, {}};
  if (e) a.e = *e;
  if (!X) return launch<uint8_t, FINISH>(ctx, a);
  if (e) return x_dtype == SLIM_F16 ? launch<__half, FINISH>(ctx, a) : launch<__hip_bfloat16, FINISH>(ctx, a);
  return x_dtype == SLIM_F16 ? launch<__half, PLAIN>(ctx, a) : launch<__hip_bfloat16, PLAIN>(ctx, a);
}

int softmax_parts_few(int n, int t, int ncu) { return slim_cdiv(n, 16 * sixteens(n, t, ncu)); }

slim_status softmax_few(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& w, int m, const Softmax& sm, float* kept, int64_t ldk) {
  FewArgs a = {X, w.q, w.s, kept, ldx, w.ld, w.lds, ldk, t, w.rows, m, slim_cdiv(m, BLOCK), (int)SLIM_F32, nullptr, nullptr, 0, 0, {}, sm};
  return x_dtype == SLIM_F16 ? launch<__half, SOFTMAX>(ctx, a) : launch<__hip_bfloat16, SOFTMAX>(ctx, a);
}

}  // namespace slimfp8
