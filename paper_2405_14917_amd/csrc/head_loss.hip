// The cross entropy of labels in the softmax of an 8-bit head's outputs (the logits), and its gradients:
//
//   z = Q(x) W^T,  loss = ln sum exp z - z[label];   dz = dloss (softmax z - [label]),  dx = Q(dz) W,  dW = Qt(dz)^T Qt(x)
//
// One product over the whole vocabulary leaves, of every tile, the maximum and the sum of exponentials of its classes for each token, its label's apart
// (fp8_gemm.hip, fp8_few.hip); `head_join` puts a token's tiles together in fp64.  dz at the label is -dloss times the others' share of the sum: as a difference
// of the probability and one it is off by 6 % at 1 - p = 1e-6 and by a third at 1e-7.  The loss alone needs no more: no logit is in memory.  The gradients need the logits a
// second time, once the sums are known.  Up to 64 Mi of them wait in memory in fp32, and `head_gradient` turns them into dz in e4m3, in blocks of 128
// classes and of 128 tokens; of the classes behind those the product is made again, and its end does the same.  It goes a piece of the vocabulary
// at a time, so that the 8-bit forms stay small, and the two products of the backward pass follow each piece in one launch; dx is
// summed over the pieces in fp32.  Both products of logits keep 24 bits (the bf16 matrix cores): a difference of large logits is a probability's exponent.
//
// Bound by the matrix cores.  32000 x 4096, 2048 tokens, bf16, both gradients: 1075 to 1097 us, of them the logits 437 to 450 (1.2 PFLOP/s; without
// storing them 394 to 405), dz 79 (5.0 TB/s; made again 466), dx and dw 537 (2.00).  One token, the loss alone: 23.5 to 27 us, the weights' read
// (5.7 TB/s), and 4 for `head_join`.
#include "act_device.h"
#include "fp8_entry.h"

namespace {

using namespace slimfp8;

// One wavefront per token.  Pairs in a fixed order, eight a lane under way at a time with the sum carried along to the new maximum (one token and
// 2000 pairs: the loss took 2 us more with two passes of one load after another); stat may be null.
__global__ __launch_bounds__(256) void head_join(const float2* __restrict__ part, int parts, const float* __restrict__ z, const void* labels, int labels64,
                                                 const float* __restrict__ dloss, int t, int V, float* __restrict__ loss, TokenStat* __restrict__ stat) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= t) return;
  const float2* p = part + row * parts;
  const int64_t label = label_at(labels, labels64, row);
  const bool live = label >= 0 && label < V;
  const float at_label = live ? z[row] : 0.f;
  auto e = [](float x) { return slimact::exp_of(fmaxf(x, -126.f)); };
  constexpr int DEEP = 8;                          // pairs of a lane that are fetched together
  float own = -__builtin_inff();
  double sum = 0.0;
  for (int i0 = lane; i0 < parts; i0 += 64 * DEEP) {
    float2 v[DEEP];
    float most = own;
#pragma unroll
    for (int d = 0; d < DEEP; ++d) v[d] = i0 + 64 * d < parts ? p[i0 + 64 * d] : make_float2(-__builtin_inff(), 0.f);
#pragma unroll
    for (int d = 0; d < DEEP; ++d) most = fmaxf(most, v[d].x);
    sum *= (double)e(own - most);
#pragma unroll
    for (int d = 0; d < DEEP; ++d) sum += (double)(v[d].y * e(v[d].x - most));
    own = most;
  }
  const float most = wave_max_f32(own);
  sum = wave_sum(sum * (double)e(own - most));
  if (lane == 0) {
    const float zl = live ? at_label : most, top = fmaxf(most, zl);
    const double lead = (double)zl - (double)most, less = exp(-fabs(lead));      // (one of the two is 1; without a label: most, and no term of its own)
    const double others = lead > 0.0 ? sum * less : sum, all = others + (!live ? 0.0 : lead > 0.0 ? 1.0 : less);
    loss[row] = live ? (float)((double)top - (double)zl + (lead > 0.0 ? log1p(others) : log(all))) : 0.f;
    if (stat) {
      const float g = live ? dloss[row] : 0.f, fine = g - g == 0.f ? g : __builtin_nanf("");      // (an infinite one is NaN in 8 bits in any case)
      stat[row] = TokenStat{top, (float)(-(double)fine * (others / all)), (float)((double)fine / all), live ? (int)label : -1};
    }
  }
}

struct GradientArgs {
  const float* z;                  // t x classes logits of this piece
  SoftmaxGradient g;
  int64_t ldz;
  int t, classes, tiles_c;
};

__device__ __forceinline__ unsigned four_e4m3(float a, float b, float c, float d, float inv) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

// Kept logits to dz in e4m3, as the end of the product does it (fp8_gemm.hip: quantize_gradient): tiles of 128 tokens x 128 classes, a thread holds
// tokens 8 (tid / 16) .. + 7 of classes 8 (tid % 16) .. + 7; the transposed form goes through LDS in bytes.  Bound by memory.
__global__ __launch_bounds__(256) void head_gradient(GradientArgs a) {
  __shared__ __align__(16) unsigned colmax[4][BLOCK];
  __shared__ __align__(16) uint8_t tile[BLOCK * BLOCK];    // [class][token], units of 8 bytes at unit ^ (class / 8 % 16)
  const int tr = blockIdx.x / a.tiles_c, tc = blockIdx.x % a.tiles_c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 15, rg = tid >> 4;
  const int r0 = tr * BLOCK + rg * 8, c0 = tc * BLOCK + cg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // (rows of kept logits have whole blocks of 128 classes: those behind the last class are not looked at)
    const float* p = a.z + (int64_t)min(r0 + i, a.t - 1) * a.ldz + c0;
    *reinterpret_cast<float4*>(&v[i][0]) = *reinterpret_cast<const float4*>(p);
    *reinterpret_cast<float4*>(&v[i][4]) = *reinterpret_cast<const float4*>(p + 4);
  }
  unsigned rm[8], m[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const TokenStat s = a.g.stat[min(r0 + i, a.t - 1)];
    const bool live = r0 + i < a.t && s.label >= 0;
    const int at = s.label - a.g.first - c0;
    rm[i] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float d = __builtin_amdgcn_exp2f((v[i][j] - s.top) * slimact::LOG2E_HI) * s.scaled;
      if (at == j) d = s.own;
      v[i][j] = live && c0 + j < a.classes ? d : 0.f;
      unsigned u = __float_as_uint(v[i][j]) & 0x7fffffffu;           // (patterns order like the values)
      u = u < 0x7f800000u ? u : 0u;
      rm[i] = max(rm[i], u);
      m[j] = max(m[j], u);
    }
  }
  if (a.g.rows_q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned u = rm[i];                                            // of the 16 lanes of a row
      u = max(u, (unsigned)dpp_b32<DPP_XOR1>((int)u));
      u = max(u, (unsigned)dpp_b32<DPP_XOR2>((int)u));
      u = max(u, (unsigned)dpp_b32<DPP_HALF_MIRROR>((int)u));
      u = max(u, (unsigned)dpp_b32<DPP_MIRROR>((int)u));
      const unsigned b = scale_byte(u);
      const float inv = __uint_as_float((254u - b) << 23);
      if (r0 + i < a.t) {
        const int64_t row = r0 + i;
        *reinterpret_cast<uint2*>(a.g.rows_q + row * a.g.ldrq + c0) =
            make_uint2(four_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], inv), four_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], inv));
        if (cg == 0) a.g.rows_s[row * a.g.ldrs + tc] = (uint8_t)b;
      }
    }
  }
  if (!a.g.cols_q) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const auto a32 = __builtin_amdgcn_permlane32_swap(m[j], m[j], false, false);
    const unsigned h = max(a32[0], a32[1]);
    const auto a16 = __builtin_amdgcn_permlane16_swap(h, h, false, false);
    m[j] = max(a16[0], a16[1]);
  }
  if (lane < 16) {
    *reinterpret_cast<uint4*>(&colmax[wave][cg * 8]) = make_uint4(m[0], m[1], m[2], m[3]);
    *reinterpret_cast<uint4*>(&colmax[wave][cg * 8 + 4]) = make_uint4(m[4], m[5], m[6], m[7]);
  }
  __syncthreads();
  uint8_t* const tile0 = tile + cg * 8 * BLOCK + ((rg ^ cg) * 8);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = cg * 8 + j;
    const unsigned b = scale_byte(max(max(colmax[0][c], colmax[1][c]), max(colmax[2][c], colmax[3][c])));
    const float inv = __uint_as_float((254u - b) << 23);
    *reinterpret_cast<uint2*>(tile0 + j * BLOCK) =
        make_uint2(four_e4m3(v[0][j], v[1][j], v[2][j], v[3][j], inv), four_e4m3(v[4][j], v[5][j], v[6][j], v[7][j], inv));
    if (rg == 0 && tc * BLOCK + c < a.classes) a.g.cols_s[(int64_t)(tc * BLOCK + c) * a.g.ldcs + tr] = (uint8_t)b;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 32 + (tid >> 3), u = tid & 7, x = c >> 3;      // 16 bytes: units 2 u and 2 u + 1
    uint4 w = *reinterpret_cast<const uint4*>(tile + c * BLOCK + ((2 * u) ^ (x & 14)) * 8);
    if (x & 1) w = make_uint4(w.z, w.w, w.x, w.y);
    if (tc * BLOCK + c < a.classes) *reinterpret_cast<uint4*>(a.g.cols_q + (int64_t)(tc * BLOCK + c) * a.g.ldcq + tr * BLOCK + u * 16) = w;
  }
}

// Pieces: as many classes as make 64 Mi logits (in e4m3, twice, 128 MB of workspace), 1024 at least; whole words of four scales.  The first one's
// are kept (256 MB, in fp32).  Measured: 32000 x 4096 with 2048 tokens, 62.5 Mi logits: none kept 1436 us, 16, 32 and 64 Mi in pieces of 16 Mi 1391,
// 1313 and 1143, in pieces of 32 and 64 Mi 1085 and 1068 (fewer rounds that end unevenly, dx once through memory); pieces of 16, 32 and 64 Mi behind 64 Mi kept:
// 131072 x 1024, 2000 tokens 2298, 2218 and 1883, 100000 x 300, 8000 tokens 3942, 3973 and 2997.  With fewer logits than that, without and with keeping
// them: 50257 x 1501, 301 tokens 274 and 242, 32000 x 4096, 16 tokens 209 and 182, 1000 x 300, 100 tokens 34 and 29.  More would cost
// memory that grows with the batch, which is what this operator is there to spare.
constexpr int64_t HL_LOGITS = 1 << 26;
constexpr int HL_LEAST = 1024, HL_STEP = 4 * BLOCK;
int piece_of(int V, int t) {
  const int64_t c = std::max<int64_t>(HL_LEAST, HL_LOGITS / std::max(1, t) / HL_STEP * HL_STEP);
  return (int)std::min<int64_t>(c, (V + HL_STEP - 1) / HL_STEP * HL_STEP);
}

int kept_of(int V, int t) { return (int64_t)piece_of(V, t) * t <= HL_LOGITS ? piece_of(V, t) : 0; }     // (1024 classes may be more)
constexpr int HL_APART = 32;                       // numbers between the rows of kept logits (at a multiple of 4 KiB they share few of the L2's channels)

Product logits_product(int V, int m, int t, const Softmax* sm) {
  Product p = {};
  p.a.rows = V;
  p.a.shift = 7;
  p.b.rows = t;
  p.c_dtype = SLIM_F32;
  p.nk = slim_cdiv(m, BLOCK);
  p.sm = sm;
  return p;
}

// Bytes of the pairs of all tokens, no fewer than for any smaller number of them: 16 classes a workgroup for up to 16 tokens, or while all the
// workgroups are few (takes_few_tokens), else tiles of 64 classes at least
size_t pair_bytes(int V, int t, int ncu) {
  const int64_t few = std::min((int64_t)t * slim_cdiv(V, 16), std::max((int64_t)16 * slim_cdiv(V, 16), (int64_t)70 * 16 * ncu));
  return slim_ws_round(sizeof(float2) * (size_t)std::max(few, (int64_t)t * slim_cdiv(V, 64)));
}
size_t sums_need(int V, int t, int ncu) { return pair_bytes(V, t, ncu) + slim_ws_round(sizeof(float) * (size_t)t); }
size_t loss_need(int V, int m, int t, int ncu) { return sums_need(V, t, ncu) + activation_bytes(t, m); }
// What the pieces need lies where the tokens' pairs were.  In the pieces' terms: t times a piece is no more than `logits`, which grows with t, and a
// piece no more than the vocabulary.
size_t grad_need(int V, int m, int t, bool dx, bool dw, slim_dtype dw_dtype, int ncu) {
  if (t <= 0) return 0;
  const int64_t Vp = (int64_t)(V + HL_STEP - 1) / HL_STEP * HL_STEP;
  const int64_t logits = std::min(t * Vp, std::max(HL_LOGITS, (int64_t)HL_LEAST * t));
  size_t stay = activation_bytes(t, m) + slim_ws_round(sizeof(TokenStat) * (size_t)t) +
                slim_ws_round(sizeof(float) * (size_t)(std::min(t * Vp, HL_LOGITS) + HL_APART * (int64_t)t));
  size_t bytes = 0;
  size_t parts = 0;                               // of the products that are cut, one after another
  Product p = {};
  if (dx) {
    bytes += slim_ws_round((size_t)(logits + 2 * BLOCK * (int64_t)t)) + slim_ws_round((size_t)(logits / BLOCK + 4 * (int64_t)t)) +
             slim_ws_round(sizeof(float) * (size_t)t * ((m + 3) / 4 * 4));
    p.a.rows = m;
    p.b.rows = t;
    p.nk = (int)(Vp / BLOCK);
    parts += gemm_workspace(&p, 1, ncu);
  }
  if (dw) {
    stay += activation_bytes(m, t);
    bytes += slim_ws_round((size_t)(logits + 2 * BLOCK * Vp)) + slim_ws_round((size_t)(logits / BLOCK + 8 * Vp));
    p.a.rows = m;
    p.b.rows = (int)Vp;
    p.nk = slim_cdiv(t, BLOCK);
    parts += gemm_workspace(&p, 1, ncu);
  }
  return stay + std::max(sums_need(V, t, ncu), bytes + parts);
}

slim_status check_head(slim_ctx* ctx, const char* fn, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const uint8_t* q, int64_t ldq, const uint8_t* s,
                       int64_t lds, int V, int m, const void* labels, const float* loss) {
  if (const slim_status st = check_stored(ctx, fn, "W", q, ldq, s, lds, V, m); st != SLIM_OK) return st;
  SLIM_REQUIRE(ctx, t >= 0 && t <= FL_MAX, "%s: t = %d", fn, t);
  if (!is_16(x_dtype)) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: X is F16 or BF16", fn);
  SLIM_REQUIRE(ctx, t == 0 || (X && labels && loss && ldx >= m), "%s: null pointer, or rows shorter than the layer (ldx = %lld)", fn, (long long)ldx);
  if ((int64_t)slim_cdiv(V, 64) * slim_cdiv(t, 64) >= 1 << 24)   // (a launch has fewer than 2^32 threads)
    return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: %d tokens are too many for one call with %d classes", fn, t, V);
  return SLIM_OK;
}

// Losses and, with `stat`, the tokens' sums; x: the quantised activations (not looked at where a few tokens are multiplied in one launch).  The
// logits of the first `keep` classes go to `kept`.
slim_status losses(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const Operand& x, const Operand& w, int m, const void* labels,
                   int labels64, const float* dloss, float* loss, TokenStat* stat, float* kept, int64_t ldk, int keep) {
  const int V = w.rows, ncu = ctx->num_cus;
  const bool few = takes_few_tokens(V, m, t, ncu);
  Softmax sm = {nullptr, nullptr, labels, labels64, 0, keep};
  Product p = logits_product(V, m, t, &sm);
  p.a = w;
  p.b = x;
  p.c = kept;
  p.ldc = ldk;
  sm.parts = few ? softmax_parts_few(V, t, ncu) : softmax_parts(p, ncu);
  sm.part = static_cast<float2*>(slim_ws_alloc(ctx, sizeof(float2) * (size_t)sm.parts * t));
  sm.z = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)t));
  if (!sm.part || !sm.z) return slim_fail(ctx, SLIM_ERR_ALLOC, "head_loss: workspace");
  if (const slim_status st = few ? softmax_few(ctx, X, x_dtype, t, ldx, w, m, sm, kept, ldk) : gemm(ctx, "head_logits", &p, 1); st != SLIM_OK) return st;
  SLIM_LAUNCH(ctx, "head_join", head_join, dim3(slim_cdiv(t, 4)), dim3(256), 0, sm.part, sm.parts, sm.z, labels, labels64, dloss, t, V, loss, stat);
  return SLIM_OK;
}

}  // namespace

extern "C" {

size_t slim_head_loss_workspace(int V, int m, int t, int num_cus) {
  if (V <= 0 || m <= 0 || t <= 0) return 0;
  return loss_need(V, m, t, num_cus > 0 ? num_cus : 256);
}
size_t slim_head_loss_grad_workspace(int V, int m, int t, int dx, int dw, slim_dtype dw_dtype, int num_cus) {
  if (V <= 0 || m <= 0 || t <= 0) return 0;
  return grad_need(V, m, t, dx != 0, dw != 0, dw_dtype, num_cus > 0 ? num_cus : 256);
}

slim_status slim_head_loss(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const uint8_t* q, int64_t ldq, const uint8_t* s,
                           int64_t lds, int V, int m, const void* labels, int labels64, float* loss) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_head_loss";
  if (const slim_status st = check_head(ctx, fn, X, x_dtype, t, ldx, q, ldq, s, lds, V, m, labels, loss); st != SLIM_OK) return st;
  if (t == 0) return SLIM_OK;
  if (const slim_status st = slim_ws_reserve(ctx, loss_need(V, m, t, ctx->num_cus)); st != SLIM_OK) return st;
  Activations a = {X, ldx, t, m, nullptr, nullptr, nullptr, nullptr};
  if (!takes_few_tokens(V, m, t, ctx->num_cus)) {
    if (!carve(ctx, t, m, a.rows_q, a.rows_s)) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
    if (const slim_status st = quantize(ctx, "fp8_quantize_x", x_dtype, &a, 1); st != SLIM_OK) return st;
  }
  const Operand x = {a.rows_q, a.rows_s, quantized_ld(m), scales_ld(m), t, 0};
  return losses(ctx, X, x_dtype, t, ldx, x, Operand{q, s, ldq, lds, V, 7}, m, labels, labels64, nullptr, loss, nullptr, nullptr, 0, 0);
}

slim_status slim_head_loss_grad(slim_ctx* ctx, const void* X, slim_dtype x_dtype, int t, int64_t ldx, const uint8_t* q, int64_t ldq, const uint8_t* s,
                                int64_t lds, const uint8_t* qt, int64_t ldqt, const uint8_t* st, int64_t ldst, int V, int m, const void* labels,
                                int labels64, const float* dloss, float* loss, void* dX, int64_t lddx, void* dW, slim_dtype dw_dtype, int64_t lddw) {
  if (!ctx) return SLIM_ERR_INVALID_ARG;
  const char* fn = "slim_head_loss_grad";
  if (const slim_status e = check_head(ctx, fn, X, x_dtype, t, ldx, q, ldq, s, lds, V, m, labels, loss); e != SLIM_OK) return e;
  SLIM_REQUIRE(ctx, dX || dW, "%s: neither dX nor dW", fn);
  if (dX)
    if (const slim_status e = check_stored(ctx, fn, "Wt", qt, ldqt, st, ldst, m, V); e != SLIM_OK) return e;
  if (dW && !is_16(dw_dtype) && dw_dtype != SLIM_F32) return slim_fail(ctx, SLIM_ERR_UNSUPPORTED, "%s: dW is F16, BF16 or F32", fn);
  SLIM_REQUIRE(ctx, (t == 0 || (dloss && (!dX || lddx >= m))) && (!dW || lddw >= m), "%s: null dloss, or rows shorter than the layer", fn);
  const int ncu = ctx->num_cus;
  if (const slim_status e = slim_ws_reserve(ctx, grad_need(V, m, t, dX != nullptr, dW != nullptr, dw_dtype, ncu)); e != SLIM_OK) return e;
  if (t == 0) {                                   // (no rows; dW is zero, the product over no blocks)
    if (!dW) return SLIM_OK;
    Product p = {};
    p.a.rows = m;
    p.b.rows = V;
    p.c = dW;
    p.ldc = lddw;
    p.c_dtype = dw_dtype;
    return gemm(ctx, "head_dw", &p, 1);
  }
  Activations a = {X, ldx, t, m, nullptr, nullptr, nullptr, nullptr};
  bool ok = carve(ctx, t, m, a.rows_q, a.rows_s);
  if (dW) ok = ok && carve(ctx, m, t, a.cols_q, a.cols_s);
  TokenStat* const stat = static_cast<TokenStat*>(slim_ws_alloc(ctx, sizeof(TokenStat) * (size_t)t));
  const int keep = kept_of(V, t);
  const int64_t ldk = keep + HL_APART;
  float* const kept = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)t * ldk));
  if (!ok || !stat || !kept) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
  if (const slim_status e = quantize(ctx, "fp8_quantize_x", x_dtype, &a, 1); e != SLIM_OK) return e;
  const Operand x = {a.rows_q, a.rows_s, quantized_ld(m), scales_ld(m), t, 0}, xt = {a.cols_q, a.cols_s, quantized_ld(t), scales_ld(t), m, 0};
  const Operand w = {q, s, ldq, lds, V, 7};
  const size_t stay = ctx->ws_off;
  if (const slim_status e = losses(ctx, X, x_dtype, t, ldx, x, w, m, labels, labels64, dloss, loss, stat, kept, ldk, keep); e != SLIM_OK) return e;
  ctx->ws_off = stay;
  const int piece = piece_of(V, t);
  const int64_t ldacc = (m + 3) / 4 * 4;
  SoftmaxGradient g = {};
  g.stat = stat;
  float* acc = nullptr;
  if (dX) {
    g.ldrq = quantized_ld(piece);
    g.ldrs = scales_ld(piece);
    ok = ok && carve(ctx, t, piece, g.rows_q, g.rows_s);
    if (piece < V) ok = ok && (acc = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)t * ldacc)));
  }
  if (dW) {
    g.ldcq = quantized_ld(t);
    g.ldcs = scales_ld(t);
    ok = ok && carve(ctx, piece, t, g.cols_q, g.cols_s);
  }
  if (!ok) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", fn);
  const size_t mark = ctx->ws_off;
  for (int v0 = 0; v0 < V; v0 += piece) {
    const int n = std::min(piece, V - v0);
    g.first = v0;
    if (v0 < keep) {
      const GradientArgs ga = {kept + v0, g, ldk, t, n, slim_cdiv(n, BLOCK)};
      SLIM_LAUNCH(ctx, "head_gradient_kept", head_gradient, dim3(ga.tiles_c * slim_cdiv(t, BLOCK)), dim3(256), 0, ga);
    } else {
      Product p = logits_product(n, m, t, nullptr);
      p.a = Operand{q + v0 * ldq, s + v0 / BLOCK * lds, ldq, lds, n, 7};
      p.b = x;
      p.sg = &g;
      if (const slim_status e = gemm(ctx, "head_gradient", &p, 1); e != SLIM_OK) return e;
    }
    Product both[2] = {};                         // dX's share, and the piece's rows of dW
    int count = 0;
    Epilogue sum = {};
    if (dX) {
      Product& d = both[count++];
      d.a = Operand{qt + v0, st + v0 / BLOCK, ldqt, ldst, m, 7};
      d.b = Operand{g.rows_q, g.rows_s, g.ldrq, g.ldrs, t, 0};
      d.nk = slim_cdiv(n, BLOCK);
      d.coarse = true;
      const bool last = v0 + n == V;
      d.c = last ? dX : acc;
      d.ldc = last ? lddx : ldacc;
      d.c_dtype = last ? x_dtype : SLIM_F32;
      sum.R = acc;
      sum.ldr = ldacc;
      sum.r_dtype = SLIM_F32;
      if (v0 > 0) d.e = &sum;
    }
    if (dW) {
      Product& d = both[count++];
      d.a = xt;
      d.b = Operand{g.cols_q, g.cols_s, g.ldcq, g.ldcs, n, 0};
      d.nk = slim_cdiv(t, BLOCK);
      d.c = static_cast<char*>(dW) + (int64_t)v0 * lddw * (dw_dtype == SLIM_F32 ? 4 : 2);
      d.ldc = lddw;
      d.c_dtype = dw_dtype;
    }
    ctx->ws_off = mark;                           // (the parts of products that are cut are done with once these are enqueued)
    if (const slim_status e = gemm(ctx, "head_dx_dw", both, count); e != SLIM_OK) return e;
  }
  return SLIM_OK;
}

}  // extern "C"
