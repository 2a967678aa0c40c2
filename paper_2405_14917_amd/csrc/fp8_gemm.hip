// The scaled matrix product of the 8-bit linear layer: C[b][a] = sum over blocks of 128 of 2^(ea + eb - 254) A[a] . B[b], both operands
// rows of e4m3 numbers along the contraction; forward A = weights, B = activations; gradients: fp8_linear.hip.
//
//  * 16-bit C: v_mfma_scale_f32_32x32x64_f8f6f4 takes the scales themselves (one byte per row and 32 of the contraction, here the same for
//    128), so the fp32 sums stay in its registers from the first block to the last: no rescaling between blocks.  fp32 C: the numbers
//    times their scales as bf16 (fp8_device.h: dequantized), converted in registers beside the products of v_mfma_f32_32x32x16_bf16.
//  * Workgroup tile TA x TB, contraction 128 bytes a step, from memory to LDS directly, four loads to a word of M0 (the instruction's
//    offset counts on both sides).  A row of a stage is 8 chunks of 16 bytes, chunk c at place c ^ (row / 2 % 8): 16 lanes that read one
//    chunk of 16 rows hit sixteen different groups of four banks.  The scales of four steps (a word per row) come the same way.
//  * Four wavefronts; the large tile is 128 x 128 of each, 256 accumulation registers, one wavefront per SIMD: 64 bytes of LDS per
//    clock of matrix work in place of 96 with eight.  The operands of half a step are read beside the products of the half before, also
//    across steps: the one barrier of a step is in its middle, behind it the step's stage is free for the loads of the step STAGES on.
//  * The rows of A are the rows of an MFMA tile, so a lane ends up with 4 consecutive outputs of one row of C at a time; the tile goes through
//    LDS, wavefront by wavefront, and leaves in rows.
//  * What becomes of a tile's sums (MODE): they are stored; bias, residual and activation first (FINISH, the residuals fetched many at a
//    time: 4096 x 11008 with 2048 tokens, on one card, 110 us, one round of loads after another 120); of a tile of logits the maximum and the sum of exponentials
//    of every token, with or without the logits themselves (SOFTMAX); or the logits' gradients, quantised in both directions for the products behind them (GRADIENT).
//  * Several products share a launch (the two gradients, where their outputs are of one kind).  A product whose tiles do not fill the chip
//    is cut along the contraction; the parts go to the workspace in fp32 and are added in a fixed order by a second kernel.
//
// What bounds it: the operands' way from L2 to LDS.  8192 x 28672 with 4096 tokens: 790 us (2430 TFLOP/s); without the loads the same
// loop takes 517 us, with loads that all hit in the L2 661; the fp32 form 1415 us for as many products (1360 TFLOP/s, the bf16 matrix
// cores at the clock the power allows).
#include <atomic>

#include "act_device.h"
#include "fp8_device.h"

namespace {

using namespace slimfp8;

constexpr int FG_BAND = 4;                 // tiles of A per band of the tile order

struct ProductArgs {
  Operand a, b;
  void* c;
  int64_t ldc;
  int c_dtype, nk;
  int tiles_a, tiles_b, splits, per;       // per: steps of a part (a multiple of 4)
  int64_t part;                            // elements from one part to the next
};
struct GemmArgs {
  ProductArgs p[2];
  int first;                               // workgroups of the first product
  Epilogue e;                              // (FINISH)
  Softmax sm;                              // (SOFTMAX)
  SoftmaxGradient sg;                      // (GRADIENT)
};
// what becomes of the sums: stored, stored through the epilogue, what the softmax needs of them, or the quantised gradient of its logarithm
enum { PLAIN, FINISH, SOFTMAX, GRADIENT };

// Direct loads, if step `k` is below `n` (the branch is in here so that the code around it stays one block for the scheduler).
// load_lds16x4: four times 16 bytes per lane, to 4 KiB of LDS one after another, from gbase + off[i]; the instruction's offset counts
// on both sides, so that off[i] is 1024 i less than what it means.
__device__ __forceinline__ void load_lds16x4(unsigned lds_addr, const unsigned* off, const uint8_t* gbase, int k, int n) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_cmp_ge_i32 %6, %7\n\ts_cbranch_scc1 1f\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
               "global_load_lds_dwordx4 %2, %5 offset:%8\n\tglobal_load_lds_dwordx4 %3, %5 offset:%9\n\tglobal_load_lds_dwordx4 %4, %5 offset:%10\n1:"
               : : "s"(lds_addr), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(gbase), "s"(k), "s"(n), "n"(1 << 10), "n"(2 << 10), "n"(3 << 10)
               : "m0", "scc");
#else
  (void)lds_addr, (void)off, (void)gbase, (void)k, (void)n;
#endif
}
__device__ __forceinline__ void load_lds4(unsigned lds_addr, unsigned voff, const uint8_t* gbase, int k, int n) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_cmp_ge_i32 %3, %4\n\ts_cbranch_scc1 1f\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n1:"
               : : "s"(lds_addr), "v"(voff), "s"(gbase), "s"(k), "s"(n) : "m0", "scc");
#else
  (void)lds_addr, (void)voff, (void)gbase, (void)k, (void)n;
#endif
}
// waits until at most N of the wavefront's loads are outstanding (none, if k is above n), and for its reads of LDS
template <int N>
__device__ __forceinline__ void wait_loads(int k, int n) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  else asm volatile("s_cmp_le_i32 %0, %1\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(0)\n1:\n\ts_waitcnt vmcnt(%2) lgkmcnt(0)" ::"s"(k), "s"(n), "n"(N) : "memory", "scc");
#else
  (void)k, (void)n;
#endif
}

// an address that is the same in every lane, in scalar registers
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t u = (uint64_t)p;
  return (const uint8_t*)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u) |
                          (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(u >> 32)) << 32);
}

template <int TA_, int TB_, int WA_, int WB_, int STAGES_>
struct Tile {
  static constexpr int TA = TA_, TB = TB_, WA = WA_, WB = WB_, STAGES = STAGES_;
  static constexpr int WAVES = WA * WB, THREADS = 64 * WAVES, MA = TA / WA / 32, MB = TB / WB / 32;
  static constexpr int STAGE = (TA + TB) * BLOCK;              // bytes of operands per step
  static constexpr int LOADS = STAGE / 1024 / WAVES, GROUPS = LOADS / 4;   // direct loads of a wavefront per step, four at a time
  static constexpr int SLOADS = ((TA + TB) / 64 + WAVES - 1) / WAVES;      // and of scales per four steps
  static constexpr int SCALES = 256 * WAVES * SLOADS;          // bytes of scales per four steps (a word per row)
  static constexpr int OUT_LD = MA * 32 + 4;                   // floats per row of C in the epilogue
  static constexpr int OUT = WAVES * 32 * OUT_LD * 4;
  static constexpr int LDS = STAGES * STAGE + 2 * SCALES > OUT ? STAGES * STAGE + 2 * SCALES : OUT;
};

// four values of a row of C from column `col` on, of which `left` exist
__device__ __forceinline__ void store4(void* row, int dtype, int col, int left, const float4& v) {
  if (dtype == SLIM_F32) {
    float* p = static_cast<float*>(row) + col;
    if (left >= 4) {
      __builtin_memcpy(p, &v, 16);
    } else {
      if (left > 0) p[0] = v.x;
      if (left > 1) p[1] = v.y;
      if (left > 2) p[2] = v.z;
    }
  } else {
    const bool bf = dtype == SLIM_BF16;
    const unsigned short h[4] = {to_16(v.x, bf), to_16(v.y, bf), to_16(v.z, bf), to_16(v.w, bf)};
    unsigned short* p = static_cast<unsigned short*>(row) + col;
    if (left >= 4) {
      __builtin_memcpy(p, h, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) p[i] = h[i];
    }
  }
}

// Four values of a row from column `col` on as they lie there, of which `left` exist (the others are zero), and as floats
struct alignas(16) Quad {
  unsigned v[4];
};
__device__ __forceinline__ Quad load_quad(const void* row, int dtype, int col, int left) {
  Quad r = {{0u, 0u, 0u, 0u}};
  if (dtype == SLIM_F32) {
    const unsigned* p = static_cast<const unsigned*>(row) + col;
    if (left >= 4) {
      __builtin_memcpy(r.v, p, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) r.v[i] = p[i];
    }
  } else {
    const unsigned short* p = static_cast<const unsigned short*>(row) + col;
    if (left >= 4) {
      __builtin_memcpy(r.v, p, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) r.v[i / 2] |= (unsigned)p[i] << (16 * (i & 1));
    }
  }
  return r;
}
__device__ __forceinline__ float4 widen(const Quad& r, int dtype) {
  if (dtype == SLIM_F32) return make_float4(__uint_as_float(r.v[0]), __uint_as_float(r.v[1]), __uint_as_float(r.v[2]), __uint_as_float(r.v[3]));
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned h = (r.v[i / 2] >> (16 * (i & 1))) & 0xffffu;
    f[i] = __uint_as_float(dtype == SLIM_BF16 ? Half16<__hip_bfloat16>::float_bits(h) : Half16<__half>::float_bits(h));
  }
  return make_float4(f[0], f[1], f[2], f[3]);
}

// f of 0 .. N - 1 as constants (a loop whose body is too long to be unrolled would keep the accumulators in memory)
template <int I, int N, typename F>
__device__ __forceinline__ void static_for(const F& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>());
    static_for<I + 1, N>(f);
  }
}

// The residuals of N quads, quad i in row `row + i step` from column `col` on (rows behind the last one: what is there is not used)
template <int N>
__device__ __forceinline__ void load_residuals(const Epilogue& e, int row, int step, int rows, int col, int left, Quad (&r)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (row + i * step < rows) r[i] = load_quad(static_cast<const char*>(e.R) + (row + i * step) * e.ldr * (int64_t)(e.r_dtype == SLIM_F32 ? 4 : 2), e.r_dtype, col, left);
}
// These quads' sums through the epilogue (Z and C are stored here)
template <int N>
__device__ __forceinline__ void finish(const Epilogue& e, char* c, int64_t ldc, int dtype, int row, int step, int rows, int col, int left, float (&v)[4 * N],
                                       const Quad (&r)[N]) {
  const int64_t size = dtype == SLIM_F32 ? 4 : 2;
  if (e.bias) {
    const float4 b = widen(load_quad(e.bias, e.bias_dtype, col, left), e.bias_dtype);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[4 * i] += b.x;
      v[4 * i + 1] += b.y;
      v[4 * i + 2] += b.z;
      v[4 * i + 3] += b.w;
    }
  }
  if (e.Z)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (row + i * step < rows)
        store4(static_cast<char*>(e.Z) + (row + i * step) * e.ldz * size, dtype, col, left, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
  slimact::activate(v, e.act);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (row + i * step < rows) {
      float4 y = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      if (e.R) {
        const float4 s = widen(r[i], e.r_dtype);
        y = make_float4(y.x + s.x, y.y + s.y, y.z + s.z, y.w + s.w);
      }
      store4(c + (row + i * step) * ldc * size, dtype, col, left, y);
    }
}

// The operands of half a step (64 of the contraction) in registers: 32 bytes per lane and 32 rows
template <typename T>
struct Half {
  uint4 a[T::MA][2], b[T::MB][2];
};
// what a lane knows of its operands' places: chunk c of its rows of A and B (LDS bytes inside a stage)
struct Places {
  int a[4], b[4];
};

__device__ __forceinline__ v8i joined(const uint4 (&v)[2]) {
  return v8i{(int)v[0].x, (int)v[0].y, (int)v[0].z, (int)v[0].w, (int)v[1].x, (int)v[1].y, (int)v[1].z, (int)v[1].w};
}

// read r of 2 (MA + MB) of half KK of the stage at `st`, in the order in which the products need them: the first rows of A, B, the other rows
template <typename T, int KK>
__device__ __forceinline__ void read_operand(Half<T>& f, const char* st, const Places& at, int r) {
  const int o = r >> 1, c = r & 1;
  if (o >= 1 && o <= T::MB) {
    f.b[o - 1][c] = *reinterpret_cast<const uint4*>(st + at.b[KK * 2 + c] + (o - 1) * 32 * BLOCK);
  } else {
    const int i = o == 0 ? 0 : o - T::MB;
    f.a[i][c] = *reinterpret_cast<const uint4*>(st + at.a[KK * 2 + c] + i * 32 * BLOCK);
  }
}
// the share of n things that belongs beside product m of M, all of them beside the first half of the products
template <int M>
__device__ __forceinline__ constexpr int share_from(int m, int n) { return m * 2 >= M ? n : m * 2 * n / M; }

// The sums of a tile as logits: dz in their place, then its two 8-bit forms.  A lane holds, of 32 tokens l32 of each j, the classes 32 i + 8 (q / 4) + 4 h + q % 4:
// a token's block of 128 classes is in two lanes (and two wavefronts, where a wavefront's part is 64 wide), a class's block of 128 tokens in
// the 32 lanes of a half (and two wavefronts).  What is not finite fills a token's whole row (`scaled` and `own` are not), so that one flag a
// token is enough.  Exponentials with log2(e) in one part: exp(-x) is off by x 7.5e-8 of itself, where e4m3's half step is 2^-4.  Both forms leave through a part of LDS of the wavefront's own, in rows of the block.
template <typename T>
__device__ __forceinline__ void quantize_gradient(v16f (&acc)[T::MA][T::MB], const SoftmaxGradient& sg, const ProductArgs& p, char* smem, int a0, int b0, int wa,
                                                  int wb, int wave, int lane) {
  constexpr int MA = T::MA, MB = T::MB, PA = 32 * MA, PB = 32 * MB, LD = 16;      // LD: bytes between the rows of a part
  static_assert(BLOCK % PA == 0 && BLOCK % PB == 0 && T::TA % BLOCK == 0 && T::TB % BLOCK == 0, "a tile is made of whole blocks");
  const int l32 = lane & 31, h = lane >> 5;
  const int first = a0 + wa * PA + h * 4, tok0 = b0 + wb * PB;
  unsigned* const row_max = reinterpret_cast<unsigned*>(smem);                    // [part of A][token], [part of B][class]
  unsigned* const col_max = row_max + T::WA * T::TB;
  constexpr int PART = PA > PB ? PA * (PB + LD) : PB * (PA + LD);
  uint8_t* const scale = reinterpret_cast<uint8_t*>(col_max + T::WB * T::TA) + wave * PA;
  char* const part = smem + 4 * (T::WA * T::TB + T::WB * T::TA) + T::WAVES * PA + wave * PART;
  static_assert(PA % 16 == 0 && 4 * (T::WA * T::TB + T::WB * T::TA) + T::WAVES * (PA + PART) <= T::LDS, "the stages' place is enough");
  TokenStat st[MB];
#pragma unroll
  for (int j = 0; j < MB; ++j) st[j] = sg.stat[min(tok0 + j * 32 + l32, p.b.rows - 1)];
  unsigned rmax[MB], fine[MB];                       // fine: all ones where the token's gradients are finite
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const bool live = tok0 + j * 32 + l32 < p.b.rows && st[j].label >= 0;
#pragma unroll
    for (int i = 0; i < MA; ++i)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = __builtin_amdgcn_exp2f((acc[i][j][q] - st[j].top) * slimact::LOG2E_HI) * st[j].scaled;
    const int label = st[j].label - sg.first - first, at = live && label >= 0 && label < PA ? label : -1;
    if (__any(at >= 0)) {
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q)
          if (at == i * 32 + 8 * (q / 4) + q % 4) acc[i][j][q] = fmaf(acc[i][j][q], 0.f, st[j].own);      // (`own`; as a move it spilled 68 registers)
    }
    if (__any(!live)) {
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] = live ? acc[i][j][q] : 0.f;
    }
    if (a0 + T::TA > p.a.rows) {                     // (the last tile: classes that do not exist)
      int left = p.a.rows - first;
#if defined(__HIP_DEVICE_COMPILE__)
      asm volatile("" : "+v"(left));                 // (or 64 results of comparisons are kept from one j for the next, and spilled)
#endif
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q)
          if (i * 32 + 8 * (q / 4) + q % 4 >= left) acc[i][j][q] = 0.f;
    }
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < MA; ++i)
#pragma unroll
      for (int q = 0; q < 16; ++q) m = max(m, __float_as_uint(acc[i][j][q]) & 0x7fffffffu);
    m = max(m, (unsigned)__shfl_xor((int)m, 32, 64));
    fine[j] = m < 0x7f800000u ? ~0u : 0u;            // (patterns order like the values, NaN above infinity)
    rmax[j] = m & fine[j];
    if (PA < BLOCK && h == 0) row_max[wa * T::TB + wb * PB + j * 32 + l32] = rmax[j];
  }
  unsigned cmax[MA][16];
  if (sg.cols_q) {
#pragma unroll
    for (int i = 0; i < MA; ++i)
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < MB; ++j) m = max(m, __float_as_uint(acc[i][j][q]) & 0x7fffffffu & fine[j]);
        m = max(m, (unsigned)dpp_b32<DPP_XOR1>((int)m));
        m = max(m, (unsigned)dpp_b32<DPP_XOR2>((int)m));
        m = max(m, (unsigned)dpp_b32<DPP_HALF_MIRROR>((int)m));
        m = max(m, (unsigned)dpp_b32<DPP_MIRROR>((int)m));
        const auto both = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        cmax[i][q] = max(both[0], both[1]);
        if (PB < BLOCK && l32 == 0) col_max[wb * T::TA + wa * PA + h * 4 + i * 32 + 8 * (q / 4) + q % 4] = cmax[i][q];
      }
  }
  if constexpr (PA < BLOCK || PB < BLOCK) __syncthreads();
  // the other wavefront's half of a block
  auto joined = [&](unsigned own, const unsigned* shared, int w, int width, int at) { return max(own, shared[(w ^ 1) * width + at]); };
  if (sg.rows_q) {
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      const int in_b = wb * PB + j * 32 + l32;
      const unsigned b = scale_byte(PA < BLOCK ? joined(rmax[j], row_max, wa, T::TB, in_b) : rmax[j]);
      const float inv = __uint_as_float((254u - b) << 23);
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(acc[i][j][4 * q] * inv, acc[i][j][4 * q + 1] * inv, 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(acc[i][j][4 * q + 2] * inv, acc[i][j][4 * q + 3] * inv, w, true);
          *reinterpret_cast<int*>(part + (j * 32 + l32) * (PA + LD) + i * 32 + q * 8 + h * 4) = w;
        }
      if (h == 0 && b0 + in_b < p.b.rows && first < p.a.rows && (PA == BLOCK || wa % 2 == 0)) sg.rows_s[(int64_t)(b0 + in_b) * sg.ldrs + first / BLOCK] = (uint8_t)b;
    }
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = PA / 16;                   // of a row
    if ((a0 + wa * PA) / BLOCK * BLOCK < p.a.rows)   // (a block that exists: its end behind the last class is zeros)
#pragma unroll
      for (int r = 0; r < PB; r += 64 / LANES) {
        const int row = r + lane / LANES, c = lane % LANES * 16;
        const uint4 v = *reinterpret_cast<const uint4*>(part + row * (PA + LD) + c);
        if (tok0 + row < p.b.rows) *reinterpret_cast<uint4*>(sg.rows_q + (int64_t)(tok0 + row) * sg.ldrq + a0 + wa * PA + c) = v;
      }
  }
  if (sg.cols_q) {
    // four lanes' words (four classes of a token each) become four words of a class: bytes change places with the lane beside, then pairs of bytes with
    // the lane two on
    __builtin_amdgcn_wave_barrier();
    const unsigned sel1 = lane & 1 ? 0x03070105u : 0x06020400u, sel2 = lane & 2 ? 0x03020706u : 0x05040100u;
#pragma unroll
    for (int i = 0; i < MA; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float inv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int in_a = wa * PA + h * 4 + i * 32 + 8 * q + k;
          const unsigned b = scale_byte(PB < BLOCK ? joined(cmax[i][4 * q + k], col_max, wb, T::TA, in_a) : cmax[i][4 * q + k]);
          inv[k] = __uint_as_float((254u - b) << 23);
          if (l32 == 0) scale[h * 4 + i * 32 + 8 * q + k] = (uint8_t)b;
        }
#pragma unroll
        for (int j = 0; j < MB; ++j) {
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(acc[i][j][4 * q] * inv[0], acc[i][j][4 * q + 1] * inv[1], 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(acc[i][j][4 * q + 2] * inv[2], acc[i][j][4 * q + 3] * inv[3], w, true);
          w = (int)__builtin_amdgcn_perm((unsigned)dpp_b32<DPP_XOR1>(w), (unsigned)w, sel1);
          w = (int)__builtin_amdgcn_perm((unsigned)dpp_b32<DPP_XOR2>(w), (unsigned)w, sel2);
          *reinterpret_cast<int*>(part + (i * 32 + 8 * q + h * 4 + (lane & 3)) * (PB + LD) + j * 32 + (l32 & ~3)) = w;
        }
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = PB / 16;
    for (int c = lane; c < PA; c += 64)
      if (a0 + wa * PA + c < p.a.rows && tok0 < p.b.rows && (PB == BLOCK || wb % 2 == 0))
        sg.cols_s[(int64_t)(a0 + wa * PA + c) * sg.ldcs + tok0 / BLOCK] = scale[c];
    if (tok0 / BLOCK * BLOCK < p.b.rows)
#pragma unroll
      for (int r = 0; r < PA; r += 64 / LANES) {
        const int row = r + lane / LANES, c = lane % LANES * 16, cls = a0 + wa * PA + row;
        const uint4 v = *reinterpret_cast<const uint4*>(part + row * (PB + LD) + c);
        if (cls < p.a.rows) *reinterpret_cast<uint4*>(sg.cols_q + (int64_t)cls * sg.ldcq + tok0 + c) = v;
      }
  }
}

// EXACT: products of the numbers in bf16 (fp32 outputs).  MODE other than PLAIN: of the first product, which is not cut; SOFTMAX and GRADIENT have
// no second one.
template <typename T, bool EXACT, int MODE>
__global__ __launch_bounds__(T::THREADS, T::MA * T::MB >= 8 ? 1 : 2) void fp8_gemm(GemmArgs ga) {
  constexpr int MA = T::MA, MB = T::MB, M = MA * MB, READS = 2 * (MA + MB), S = T::STAGES;
  extern __shared__ __align__(16) char smem_fg[];
  const bool second = (int)blockIdx.x >= ga.first;
  const ProductArgs& p = ga.p[second];
  const int bid = (int)blockIdx.x - (second ? ga.first : 0);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Order: workgroups with one residue mod 8 run on one XCD and take a run of consecutive tiles; bands of FG_BAND tiles of A, B slowest
  // inside a band, so that what an XCD works on at one time shares its operands in its L2.
  const int tiles = p.tiles_a * p.tiles_b, total = tiles * p.splits, each = total / 8, rest8 = total % 8, c8 = bid % 8;
  const int id0 = c8 * each + min(c8, rest8) + bid / 8, split = id0 / tiles, id = id0 - split * tiles;
  const int full = p.tiles_b * FG_BAND, band = id / full, inband = id - band * full, bw = min(FG_BAND, p.tiles_a - band * FG_BAND);
  const int a0 = (band * FG_BAND + inband % bw) * T::TA, b0 = (inband / bw) * T::TB;
  const int k0 = split * p.per, nk = __builtin_amdgcn_readfirstlane(min(p.per, p.nk - k0));
  const int wa = wave % T::WA, wb = wave / T::WA;

  // A direct load fills 1 KiB of a stage: 8 rows; the lane fetches the chunk that belongs at its place.  Four of a wavefront are 32 rows
  // one after another, of A or of B.  Rows behind the last one are the last one again (their sums are not stored).
  constexpr unsigned LOWER = 4096;          // what the bases are lowered by so that no offset is negative
  unsigned off[T::LOADS];
#pragma unroll
  for (int i = 0; i < T::LOADS; ++i) {
    const int r = ((i / 4) * T::WAVES + wave) * 32 + (i % 4) * 8 + (lane >> 3), ch = (lane & 7) ^ ((r >> 1) & 7);
    off[i] = LOWER - (i % 4) * 1024u + ch * 16u +
             (r < T::TA ? (unsigned)((int64_t)min(r, p.a.rows - 1 - a0) * p.a.ld) : (unsigned)((int64_t)min(r - T::TA, p.b.rows - 1 - b0) * p.b.ld));
  }
  const uint8_t* abase = uniform(p.a.q + (int64_t)a0 * p.a.ld + (int64_t)k0 * BLOCK - LOWER);
  const uint8_t* bbase = uniform(p.b.q + (int64_t)b0 * p.b.ld + (int64_t)k0 * BLOCK - LOWER);
  // scales: one load is the words of 64 rows (rows behind those of the tile: the last ones again, not used)
  unsigned soff[T::SLOADS];
  const uint8_t* sbase[T::SLOADS];
#pragma unroll
  for (int i = 0; i < T::SLOADS; ++i) {
    const int r = min((i * T::WAVES + wave) * 64, T::TA + T::TB - 64);
    const bool in_b = r >= T::TA;
    const Operand& o = in_b ? p.b : p.a;
    const int r0 = in_b ? b0 : a0, row = min(r0 + r - (in_b ? T::TA : 0) + lane, o.rows - 1);
    soff[i] = (unsigned)((int64_t)((row >> o.shift) - (r0 >> o.shift)) * o.lds);
    sbase[i] = uniform(o.s + (int64_t)(r0 >> o.shift) * o.lds + k0);
  }
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)((__attribute__((address_space(3))) char*)smem_fg));
  unsigned slot = 0;                        // of the next step to be loaded: LDS bytes of its stage
  int loading = 0;                          // and its number
  auto load_operands = [&](int g) {         // group g of this wavefront's loads
    const int r0 = (g * T::WAVES + wave) * 32;
    load_lds16x4(lds0 + slot + (unsigned)r0 * BLOCK, off + 4 * g, r0 < T::TA ? abase : bbase, loading, nk);
  };
  auto load_scales = [&]() {                // (first, so that they are not behind the operands of their step; one step in four)
#pragma unroll
    for (int i = 0; i < T::SLOADS; ++i)
      load_lds4(lds0 + (unsigned)(S * T::STAGE) + (unsigned)((loading >> 2) & 1) * T::SCALES + (unsigned)(i * T::WAVES + wave) * 256u, soff[i],
                sbase[i] + loading, loading + ((loading & 3) << 20), nk);
  };
  auto loaded = [&]() {
    abase += BLOCK;
    bbase += BLOCK;
    slot = slot == (unsigned)((S - 1) * T::STAGE) ? 0u : slot + (unsigned)T::STAGE;
    ++loading;
  };

  v16f acc[MA][MB];
#pragma unroll
  for (int i = 0; i < MA; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  const int l32 = lane & 31, h = lane >> 5, sw = (l32 >> 1) & 7;
  const int ra = wa * MA * 32 + l32, rb = T::TA + wb * MB * 32 + l32;
  Places at;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int place = (((c >> 1) * 4 + h * 2 + (c & 1)) ^ sw) * 16;
    at.a[c] = ra * BLOCK + place;
    at.b[c] = rb * BLOCK + place;
  }
  int sa[MA], sb[MB];                       // scales of this step
  auto read_scales = [&](int (&a)[MA], int (&b)[MB], int k) {
    const uint8_t* sc = reinterpret_cast<const uint8_t*>(smem_fg) + S * T::STAGE + ((k >> 2) & 1) * T::SCALES + (k & 3);
#pragma unroll
    for (int i = 0; i < MA; ++i) a[i] = sc[(ra + i * 32) * 4];
#pragma unroll
    for (int j = 0; j < MB; ++j) b[j] = sc[(rb + j * 32) * 4];
  };
  // Half a step: its products, and between them what `between(m)` has to do
  auto half = [&](const Half<T>& g, auto between) {
    if constexpr (EXACT) {
      v8bf ba[2][MA], bb[2][MB];
      auto convert = [&](int q, int r) {    // operand r of MA + MB, eighth q of its chunk pair
        if (r < MA) ba[q & 1][r] = dequantized((int)((q & 1) ? g.a[r][q >> 1].z : g.a[r][q >> 1].x), (int)((q & 1) ? g.a[r][q >> 1].w : g.a[r][q >> 1].y), __uint_as_float((unsigned)sa[r] << 23));
        else bb[q & 1][r - MA] = dequantized((int)((q & 1) ? g.b[r - MA][q >> 1].z : g.b[r - MA][q >> 1].x), (int)((q & 1) ? g.b[r - MA][q >> 1].w : g.b[r - MA][q >> 1].y), __uint_as_float((unsigned)sb[r - MA] << 23));
      };
#pragma unroll
      for (int r = 0; r < MA + MB; ++r) convert(0, r);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int m = 0; m < M; ++m) {
          acc[m / MB][m % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ba[q & 1][m / MB], bb[q & 1][m % MB], acc[m / MB][m % MB], 0, 0, 0);
          if (q < 3)
#pragma unroll
            for (int r = m * (MA + MB) / M; r < (m + 1) * (MA + MB) / M; ++r) convert(q + 1, r);
          if ((q * M + m) % 4 == 0) between((q * M + m) / 4);
          __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        acc[m / MB][m % MB] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(joined(g.a[m / MB]), joined(g.b[m % MB]), acc[m / MB][m % MB], 0, 0, 0,
                                                                             sa[m / MB], 0, sb[m % MB]);
        between(m);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  if (nk > 0) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      load_scales();
#pragma unroll
      for (int g = 0; g < T::GROUPS; ++g) load_operands(g);
      loaded();
    }
    // Loads complete in order: with those of S - 1 steps outstanding, the first one's have landed.
    wait_loads<(S - 1) * T::LOADS>(S, nk);
    __syncthreads();
    read_scales(sa, sb, 0);
  }
  const char* stage = smem_fg;
  int na[MA], nb[MB];                       // scales of the next step
  auto pass_scales = [&]() {
#pragma unroll
    for (int i = 0; i < MA; ++i) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < MB; ++j) sb[j] = nb[j];
  };
  if constexpr (M == 1) {
    // One product per half: too few to read anything beside.  The whole next step is read beside this one's two.
    Half<T> w[2][2];
#pragma unroll
    for (int r = 0; r < READS; ++r) {
      read_operand<T, 0>(w[0][0], stage, at, r);
      read_operand<T, 1>(w[0][1], stage, at, r);
    }
    auto step = [&](auto parity, int k) {
      constexpr int P = decltype(parity)::value;
      wait_loads<(S - 2) * T::LOADS>(k + S, nk);
      __syncthreads();                      // everybody's loads of the next step; everybody has read this one's stage
      stage = stage == smem_fg + (S - 1) * T::STAGE ? smem_fg : stage + T::STAGE;
      read_scales(na, nb, k + 1);
#pragma unroll
      for (int r = 0; r < READS; ++r) {
        read_operand<T, 0>(w[P ^ 1][0], stage, at, r);
        read_operand<T, 1>(w[P ^ 1][1], stage, at, r);
      }
      load_scales();
#pragma unroll
      for (int g = 0; g < T::GROUPS; ++g) load_operands(g);
      loaded();
      __builtin_amdgcn_sched_barrier(0);
      half(w[P][0], [](int) {});
      half(w[P][1], [](int) {});
      pass_scales();
    };
#pragma unroll 1
    for (int k = 0; k < nk; k += 2) {
      step(std::integral_constant<int, 0>(), k);
      if (k + 1 < nk) step(std::integral_constant<int, 1>(), k + 1);
    }
  } else {
    Half<T> f[2];
#pragma unroll
    for (int r = 0; r < READS; ++r) read_operand<T, 0>(f[0], stage, at, r);
#pragma unroll 1
    for (int k = 0; k < nk; ++k) {
      // First half: the second half's operands are read.  Then the step's stage is free, and the step S on is loaded into it beside the
      // second half, which reads the next step's first operands (behind the last step: what lies there, unused).
      half(f[0], [&](int m) {
#pragma unroll
        for (int r = share_from<M>(m, READS); r < share_from<M>(m + 1, READS); ++r) read_operand<T, 1>(f[1], stage, at, r);
      });
      wait_loads<(S - 2) * T::LOADS>(k + S, nk);
      __syncthreads();                      // everybody's loads of the next step; everybody has read this one's stage
      stage = stage == smem_fg + (S - 1) * T::STAGE ? smem_fg : stage + T::STAGE;
      load_scales();
      read_scales(na, nb, k + 1);
      half(f[1], [&](int m) {
#pragma unroll
        for (int r = share_from<M>(m, READS); r < share_from<M>(m + 1, READS); ++r) read_operand<T, 0>(f[0], stage, at, r);
#pragma unroll
        for (int g = m * T::GROUPS / M; g < (m + 1) * T::GROUPS / M; ++g) load_operands(g);
      });
      loaded();
      pass_scales();
    }
  }

  // A lane holds column b = lane % 32 of an MFMA tile and rows 8 (q / 4) + 4 h + q % 4.
  __syncthreads();
  if constexpr (MODE == SOFTMAX) {
    // So the rows of A that a lane holds of a row of B are joined in its registers, then with the lane 32 on and with the other wavefronts.
    float2* const share = reinterpret_cast<float2*>(smem_fg);        // [part of A][row of B]
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      const int first = a0 + wa * MA * 32 + h * 4, in_b = (wb * MB + j) * 32 + l32, row = b0 + in_b;
      if (a0 + T::TA > p.a.rows) {                                   // (the last tile: classes that do not exist)
        int left = p.a.rows - first;
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(left));                               // (or 64 results of comparisons are kept from one j for the next, and spilled)
#endif
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (i * 32 + 8 * (q / 4) + q % 4 >= left) acc[i][j][q] = -__builtin_inff();
      }
      // the label's logit goes its own way, and counts in neither the maximum nor the sum: -inf in its place (NaN if it is not finite), also among
      // the kept ones, where nobody looks at it
      const int64_t label = row < p.b.rows ? label_at(ga.sm.labels, ga.sm.labels64, row) : -1;
      int at = label >= first && label < min(p.a.rows, first + MA * 32) ? (int)(label - first) : -1;
      if (__any(at >= 0)) {
        float z = 0.f;
        bool mine = false;                                           // (the other half of the lanes holds four classes in eight)
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (at == i * 32 + 8 * (q / 4) + q % 4) {
              z = acc[i][j][q];
              mine = true;
            }
        if (mine) ga.sm.z[row] = z;
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(at));                                 // (compared again: kept, or in one loop, 81 registers are spilled)
#endif
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (at == i * 32 + 8 * (q / 4) + q % 4) acc[i][j][q] = fmaf(acc[i][j][q], 0.f, -__builtin_inff());
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) top = fmaxf(top, acc[i][j][q]);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float from = top == -__builtin_inff() ? 0.f : top;       // (classes behind the last one, or the label, alone)
      float sum = 0.f;                                               // (log2(e) in one part: exp(-x) is off by x 7.5e-8 of itself, 2.8e-8 of the sum at most)
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) sum += __builtin_amdgcn_exp2f((acc[i][j][q] - from) * slimact::LOG2E_HI);
      sum += __shfl_xor(sum, 32, 64);
      if (h == 0) share[wa * T::TB + in_b] = make_float2(top, sum);
      __builtin_amdgcn_sched_barrier(0);                             // (one j at a time in the registers)
    }
    __syncthreads();
    for (int r = tid; r < T::TB && b0 + r < p.b.rows; r += T::THREADS) {
      float2 s = share[r];
#pragma unroll
      for (int w = 1; w < T::WA; ++w) {
        const float2 o = share[w * T::TB + r];
        const float top = fmaxf(s.x, o.x), from = top == -__builtin_inff() ? 0.f : top;
        s = make_float2(top, s.y * __builtin_amdgcn_exp2f((s.x - from) * slimact::LOG2E_HI) + o.y * __builtin_amdgcn_exp2f((o.x - from) * slimact::LOG2E_HI));
      }
      ga.sm.part[(int64_t)(b0 + r) * ga.sm.parts + a0 / T::TA] = s;
    }
    if (a0 >= ga.sm.keep) return;
    __syncthreads();
  }
  if constexpr (MODE == GRADIENT) {
    quantize_gradient<T>(acc, ga.sg, p, smem_fg, a0, b0, wa, wb, wave, lane);
    return;
  }
  // 32 rows of C at a time through a part of LDS of the wavefront's own.
  float* out = reinterpret_cast<float*>(smem_fg) + wave * 32 * T::OUT_LD;
  constexpr int QUADS = T::MA * 8, RPI = 64 / QUADS;           // lanes per row of C, rows per instruction
  static_assert(QUADS <= 64, "a row of a wavefront's part is read by one instruction");
  char* cbase = static_cast<char*>(p.c) + (int64_t)split * p.part * 4;
  const int esize = p.c_dtype == SLIM_F32 ? 4 : 2;
  if (MODE == FINISH && !second) {
    // N quads of a lane at a time.  Residuals are fetched many at a time and ahead of their use, not one round of loads after another: where N is all
    // of a j, those of every j first (4096 x 11008, 2048 tokens, 16-bit activations: 120 -> 110 us), else those of the j to come, which wait in a
    // part of LDS, since a loop of several rounds cannot count through registers (8192 x 4096, 4096 tokens: 223 -> 168).
    constexpr int N = RPI >= 4 ? 32 / RPI : 4, ALL = 32 / RPI;
    constexpr bool AHEAD = N * RPI == 32 && MB <= 2;
    static_assert(AHEAD || T::OUT + T::THREADS * ALL * 16 <= T::LDS, "the stages' place is enough");
    uint4* const waiting = reinterpret_cast<uint4*>(smem_fg + T::OUT) + tid;      // quad i of this lane at i T::THREADS
    const int col = (lane % QUADS) * 4, ca = a0 + wa * T::MA * 32 + col, row0 = b0 + wb * T::MB * 32 + lane / QUADS;
    const bool some = ca < p.a.rows;
    Quad ahead[AHEAD ? MB : 1][ALL];
    if (some && ga.e.R)
#pragma unroll
      for (int j = 0; j < (AHEAD ? MB : 1); ++j) load_residuals<ALL>(ga.e, row0 + j * 32, RPI, p.b.rows, ca, p.a.rows - ca, ahead[j]);
    static_for<0, MB>([&](auto block) __attribute__((always_inline)) {
      constexpr int j = decltype(block)::value;
#pragma unroll
      for (int i = 0; i < T::MA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(out + l32 * T::OUT_LD + i * 32 + q * 8 + h * 4) =
              make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
      if (!AHEAD && some && ga.e.R) {
#pragma unroll
        for (int i = 0; i < ALL; ++i) waiting[i * T::THREADS] = *reinterpret_cast<const uint4*>(ahead[0][i].v);
        if (j + 1 < MB) load_residuals<ALL>(ga.e, row0 + (j + 1) * 32, RPI, p.b.rows, ca, p.a.rows - ca, ahead[0]);
      }
#pragma unroll 1
      for (int r = 0; r < 32; r += N * RPI) {
        const int row = row0 + j * 32 + r;
        float v[4 * N];
        Quad res[N] = {};
        if (AHEAD) {
#pragma unroll
          for (int i = 0; i < N; ++i) res[i] = ahead[AHEAD ? j : 0][i];
        } else if (some && ga.e.R) {
#pragma unroll
          for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(res[i].v) = waiting[(r / RPI + i) * T::THREADS];
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
          *reinterpret_cast<float4*>(&v[4 * i]) = *reinterpret_cast<const float4*>(out + (r + lane / QUADS + i * RPI) * T::OUT_LD + col);
        if (some) finish<N>(ga.e, cbase, p.ldc, p.c_dtype, row, RPI, p.b.rows, ca, p.a.rows - ca, v, res);
      }
    });
    return;
  }
#pragma unroll
  for (int j = 0; j < T::MB; ++j) {
#pragma unroll
    for (int i = 0; i < T::MA; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(out + l32 * T::OUT_LD + i * 32 + q * 8 + h * 4) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
#pragma unroll
    for (int r = 0; r < 32; r += RPI) {
      const int rr = r + lane / QUADS, col = (lane % QUADS) * 4;
      const float4 v = *reinterpret_cast<const float4*>(out + rr * T::OUT_LD + col);
      const int row = b0 + (wb * T::MB + j) * 32 + rr, ca = a0 + wa * T::MA * 32 + col;
      if (row < p.b.rows) store4(cbase + (int64_t)row * p.ldc * esize, p.c_dtype, ca, p.a.rows - ca, v);
    }
  }
}

// C = the sum of a product's parts, in their order
template <bool FINISH_>
__global__ __launch_bounds__(256) void fp8_join(ProductArgs p, const float* __restrict__ parts, int64_t ldp, void* c, int64_t ldc, int dtype, Epilogue e) {
  const int quads = (p.a.rows + 3) / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)quads * p.b.rows) return;
  const int row = (int)(id / quads), col = (int)(id % quads) * 4;
  const float* src = parts + (int64_t)row * ldp + col;
  float4 s = *reinterpret_cast<const float4*>(src);
  for (int i = 1; i < p.splits; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(src + i * p.part);
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  if constexpr (FINISH_) {
    float v[4] = {s.x, s.y, s.z, s.w};
    Quad r[1] = {};
    if (e.R) load_residuals<1>(e, row, 1, p.b.rows, col, p.a.rows - col, r);
    return finish<1>(e, static_cast<char*>(c), ldc, dtype, row, 1, p.b.rows, col, p.a.rows - col, v, r);
  }
  store4(static_cast<char*>(c) + (int64_t)row * ldc * (dtype == SLIM_F32 ? 4 : 2), dtype, col, p.a.rows - col, s);
}

enum { TILE_LARGE, TILE_MEDIUM, TILE_SMALL };
typedef Tile<256, 256, 2, 2, 2> Large;
typedef Tile<128, 128, 2, 2, 2> Medium;
typedef Tile<64, 64, 2, 2, 4> Small;

struct Plan {
  int splits[2];
  int64_t ldp[2];
};
constexpr int TILE_A[] = {Large::TA, Medium::TA, Small::TA}, TILE_B[] = {Large::TB, Medium::TB, Small::TB};

bool exact(const Product& p) { return p.sm || p.sg || (p.c_dtype == SLIM_F32 && !p.coarse); }
int tiles_of(const Product& p, int tile) { return slim_cdiv(p.a.rows, TILE_A[tile]) * slim_cdiv(p.b.rows, TILE_B[tile]); }

// Parts along the contraction, where `tiles` do not fill the chip; eight steps a part at least.  (A softmax needs the whole sums.)
int parts_of(const Product& p, int tile, int ncu) {
  if (p.sm || p.sg) return 1;
  const int nk = p.nk;
  const int s = std::max(1, std::min(ncu / std::max(1, tiles_of(p, tile)), nk / 8));
  const int per = slim_cdiv(slim_cdiv(std::max(1, nk), s), 4) * 4;
  return std::max(1, slim_cdiv(nk, per));
}

// A product's tile: by what a round of workgroups costs, and a step of them.  Measured (us, 16-bit and fp32 C): a round of large tiles 15 +
// 1.44 (2.6) a step, of two medium ones per CU 5.4 + 0.82 (1.42), of two small ones 2.7 + 0.34 (0.56), a medium one alone on its CU 0.6 of
// that a step; 6 for the launch.  So 15872 x 128, 6139 tokens, takes medium tiles (81; large ones 110, small ones 147), as does 14666 x 2048, 2078 tokens,
// whose 522 large ones are three rounds (78 and 102), 2048 x 2048, 1024 tokens, small ones (17; medium ones 26), and 8192 x 28672, 4096
// tokens, large ones (790; medium ones above 900).  The bytes of the operands are in the measured step, not a term of their own.
// With residuals or kept sums a round of large tiles costs 3 more than one of medium ones, whose epilogues run beside another workgroup's products: 8192 x
// 4096, 4096 tokens, residual 168 and 164, with gelu and kept sums too 225 and 202; 8192 x 28672 792 and 985.
double tile_time(const Product& p, int tile, int parts = 1, bool alone = false) {
  static const double round[] = {15.0, 5.4, 2.7}, step[2][3] = {{1.44, 0.82, 0.34}, {2.6, 1.42, 0.56}};
  const double epilogue = tile == TILE_LARGE && p.e && (p.e->R || p.e->Z) ? 3.0 : 0.0;
  return round[tile] + epilogue + step[exact(p)][tile] * (alone ? 0.6 : 1.0) * slim_cdiv(p.nk, parts);
}
double tile_cost(const Product& p, int tile, int ncu) {
  const int tiles = tiles_of(p, tile), s = parts_of(p, tile, ncu), at_once = tile == TILE_LARGE ? ncu : 2 * ncu;
  const double join = s > 1 ? 4.0 + 8.0 * s * p.a.rows * (double)p.b.rows / 4.85e6 : 0.0;
  return 6.0 + slim_cdiv((int64_t)tiles * s, at_once) * tile_time(p, tile, s, tile == TILE_MEDIUM && tiles * s <= ncu) + join;
}
int tile_of(const Product& p, int ncu) {
  int best = p.sg ? TILE_MEDIUM : TILE_SMALL;                       // (a gradient's tile holds whole blocks of 128)
  for (int t : {TILE_MEDIUM, TILE_LARGE})
    if (tile_cost(p, t, ncu) < tile_cost(p, best, ncu)) best = t;
  return best;
}

// Two products' tiles in one launch on `slots` places, none of them cut, the first one's first: a CU that is done with a tile takes the next.  `sum`: if no
// CU waited at the end.
double joint_cost(const Product* p, int tile, int slots, double& sum) {
  const int count = tiles_of(p[0], tile), more = count % slots;
  const double t0 = tile_time(p[0], tile), t1 = tile_time(p[1], tile);
  sum = (count * t0 + tiles_of(p[1], tile) * t1) / slots;
  double least = count / slots * t0, most = least + t0, end = more ? most : least;      // slots - more of them are done with the first, and more
  for (int left = tiles_of(p[1], tile); left > 0;) {
    const bool early = !more || least <= most;
    double& done = early ? least : most;
    left -= early ? slots - more : more;
    done += t1;
    end = std::max(end, done);
  }
  return end;
}
int places(int tile, int ncu) { return tile == TILE_LARGE ? ncu : 2 * ncu; }
// The mean of the costs with all places and with a sixteenth fewer: tiles that fill their rounds to the last place need another round as soon as some take
// longer (5504 x 3584, 1792 tokens: 77 by the costs in large tiles and 76 in medium ones, 118 us and 96).
double safe_cost(const Product* p, int tile, int ncu) {
  double sum;
  return (joint_cost(p, tile, places(tile, ncu), sum) + joint_cost(p, tile, places(tile, ncu) * 15 / 16, sum)) / 2;
}
// Whether two products share a launch, and its tile (own: each one's alone): not where they differ in their kind or tile (a gradient of long contraction and
// few tiles beside one of many).
// Two whose tiles differ, or are medium, take large ones together where they fill each other's last rounds.  Of 281 pairs of 16-bit gradients (n x m, t tokens)
// that would by the costs alone: two launches -> one (111 of 122 by this rule) 7.4 % less on average (25053 x 2798, 3193: 607 -> 503 us; at most 1.8 % more; the
// other 11 3.2 % less on average, but up to 4.4 % more), medium -> large (46 of 159) 5.6 % (16384 x 4096, 2048: 334 -> 304; at most 2.6 % more, 3522 x 1434, 3351;
// the others 1.2 % less on average, but up to 22 % more).  Large ones move half the operands' bytes, which the costs leave out: hence the margins.
bool in_one_launch(const Product (&p)[2], const int (&own)[2], int ncu, int& tile) {
  tile = own[0];
  const int other = own[1];
  if (exact(p[0]) != exact(p[1])) return false;
  if ((tile == TILE_LARGE && other == TILE_LARGE) || tile == TILE_SMALL || other == TILE_SMALL || parts_of(p[0], tile, ncu) > 1 || parts_of(p[1], other, ncu) > 1)
    return tile == other;
  double sum, of_medium;
  const double large = joint_cost(p, TILE_LARGE, ncu, sum), safe = safe_cost(p, TILE_LARGE, ncu);
  if (tile != other) {
    const double apart = tile_cost(p[0], tile, ncu) + tile_cost(p[1], other, ncu);
    if (6.0 + large >= apart || 6.0 + safe > 1.03 * apart) return false;
    tile = TILE_LARGE;
  } else {
    (void)joint_cost(p, tile, places(tile, ncu), of_medium);
    if (safe <= 1.02 * safe_cost(p, tile, ncu) && sum <= 1.04 * of_medium) tile = TILE_LARGE;
  }
  return true;
}

// Each product's parts as if it were alone: beside another one of many tiles, few of long contraction would be what the launch waits for
// (gradients of 14666 x 2078, 88 tokens: 17 tiles of 115 steps took 82 us beside 1955 of one).
Plan make_plan(const Product* p, int count, int tile, const int* own, int ncu) {
  Plan pl = {};
  for (int i = 0; i < count; ++i) {
    pl.splits[i] = tile == own[i] ? parts_of(p[i], tile, ncu) : 1;
    pl.ldp[i] = (p[i].a.rows + 3) / 4 * 4;
  }
  return pl;
}

// Bytes that a product's parts take at most, and those of one of fewer rows or a shorter contraction: with more than one part the tiles times
// the parts are no more than the CUs (so the parts hold no more than a large tile for each), and the parts no more than an eighth of the
// steps.  What the parts of the very product take is no bound for fewer tokens: they vanish once the tiles fill the chip (32000 x 4096: 34 MB
// at 768 tokens, none at 769).
size_t parts_bytes(const Product& p, int ncu) {
  const int64_t most = std::min(ncu, p.nk / 8), ldp = (p.a.rows + 3) / 4 * 4;
  return most < 2 ? 0 : slim_ws_round(sizeof(float) * (size_t)std::min((int64_t)ncu * Large::TA * Large::TB, most * ldp * p.b.rows));
}

template <typename T, bool EXACT, int MODE>
slim_status launch(slim_ctx* ctx, const char* name, const GemmArgs& ga, int grid) {
  // (an attribute of the function on the device, asked for once: it costs a call as much as a third of the launch)
  static std::atomic<uint64_t> allowed{0};
  const uint64_t bit = ctx->device < 64 ? 1ull << ctx->device : 0;
  if (T::LDS > 64 * 1024 && !(allowed.load(std::memory_order_relaxed) & bit)) {
    SLIM_HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_gemm<T, EXACT, MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
    allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  SLIM_LAUNCH(ctx, name, (fp8_gemm<T, EXACT, MODE>), dim3(grid), dim3(T::THREADS), T::LDS, ga);
  return SLIM_OK;
}
template <bool EXACT, int MODE>
slim_status launch(slim_ctx* ctx, const char* name, int tile, const GemmArgs& ga, int grid) {
  return tile == TILE_LARGE    ? launch<Large, EXACT, MODE>(ctx, name, ga, grid)
         : tile == TILE_MEDIUM ? launch<Medium, EXACT, MODE>(ctx, name, ga, grid)
                               : launch<Small, EXACT, MODE>(ctx, name, ga, grid);
}
slim_status launch(slim_ctx* ctx, const char* name, int tile, const GemmArgs& ga, int grid, bool exact, int mode) {
  if (mode == GRADIENT) return tile == TILE_LARGE ? launch<Large, true, GRADIENT>(ctx, name, ga, grid) : launch<Medium, true, GRADIENT>(ctx, name, ga, grid);
  if (mode == SOFTMAX) return launch<true, SOFTMAX>(ctx, name, tile, ga, grid);
  if (mode == FINISH) return exact ? launch<true, FINISH>(ctx, name, tile, ga, grid) : launch<false, FINISH>(ctx, name, tile, ga, grid);
  return exact ? launch<true, PLAIN>(ctx, name, tile, ga, grid) : launch<false, PLAIN>(ctx, name, tile, ga, grid);
}

slim_status multiply(slim_ctx* ctx, const char* name, const Product* p, int count, int tile, const int* own) {
  const Plan pl = make_plan(p, count, tile, own, ctx->num_cus);
  GemmArgs ga = {};
  float* parts[2] = {};
  int grid = 0;
  for (int i = 0; i < count; ++i) {
    ProductArgs& q = ga.p[i];
    q.a = p[i].a;
    q.b = p[i].b;
    q.nk = p[i].nk;
    q.splits = pl.splits[i];
    q.per = slim_cdiv(slim_cdiv(std::max(1, q.nk), q.splits), 4) * 4;
    q.tiles_a = slim_cdiv(q.a.rows, TILE_A[tile]);
    q.tiles_b = slim_cdiv(q.b.rows, TILE_B[tile]);
    q.c = p[i].c;
    q.ldc = p[i].ldc;
    q.c_dtype = p[i].c_dtype;
    if (q.splits > 1) {
      q.part = pl.ldp[i] * q.b.rows;
      parts[i] = static_cast<float*>(slim_ws_alloc(ctx, sizeof(float) * (size_t)q.splits * q.part));
      if (!parts[i]) return slim_fail(ctx, SLIM_ERR_ALLOC, "%s: workspace", name);
      q.c = parts[i];
      q.ldc = pl.ldp[i];
      q.c_dtype = SLIM_F32;
    }
    if (i == 0) ga.first = q.tiles_a * q.tiles_b * q.splits;
    grid += q.tiles_a * q.tiles_b * q.splits;
  }
  const Epilogue* const e = p[0].e;          // (where the product is cut, the parts' sum goes through it)
  if (e) ga.e = *e;
  if (p[0].sm) ga.sm = *p[0].sm;
  if (p[0].sg) ga.sg = *p[0].sg;
  const slim_status st = launch(ctx, name, tile, ga, grid, exact(p[0]), p[0].sg ? GRADIENT : p[0].sm ? SOFTMAX : e && !parts[0] ? FINISH : PLAIN);
  if (st != SLIM_OK) return st;
  for (int i = 0; i < count; ++i)
    if (parts[i]) {
      const int64_t quads = (int64_t)slim_cdiv(p[i].a.rows, 4) * p[i].b.rows;
      const dim3 g(slim_cdiv(quads, 256));
      if (e && i == 0) SLIM_LAUNCH(ctx, "fp8_join", fp8_join<true>, g, dim3(256), 0, ga.p[i], parts[i], pl.ldp[i], p[i].c, p[i].ldc, (int)p[i].c_dtype, ga.e);
      else SLIM_LAUNCH(ctx, "fp8_join", fp8_join<false>, g, dim3(256), 0, ga.p[i], parts[i], pl.ldp[i], p[i].c, p[i].ldc, (int)p[i].c_dtype, ga.e);
    }
  return SLIM_OK;
}

}  // namespace

namespace slimfp8 {

int softmax_parts(const Product& p, int num_cus) { return slim_cdiv(p.a.rows, TILE_A[tile_of(p, num_cus)]); }

size_t gemm_workspace(const Product* p, int count, int num_cus) {
  size_t bytes = 0;
  for (int i = 0; i < count; ++i) bytes += parts_bytes(p[i], num_cus);
  return bytes;
}

slim_status gemm(slim_ctx* ctx, const char* name, const Product* p, int count) {
  if (count == 1) {
    const int tile = tile_of(*p, ctx->num_cus);
    return multiply(ctx, name, p, 1, tile, &tile);
  }
  // Tiles of the longer contraction first: those of the shorter one fill what they leave (525 x 3810, 7784 tokens: 81 -> 64 us, 2560 x 2048, 6000: 88 -> 72).
  // Small tiles only where it is twice as long: of 205 pairs those 123 take 3.0 % less on average (three 2 to 3.5 % more), the others 0.9 %, but some 4 % more.
  const bool swap = p[1].nk > p[0].nk && !p[0].e;
  const Product in_order[2] = {p[swap], p[!swap]};
  const int own[2] = {tile_of(in_order[0], ctx->num_cus), tile_of(in_order[1], ctx->num_cus)}, given[2] = {own[swap], own[!swap]};
  int tile;
  if (!in_one_launch(in_order, own, ctx->num_cus, tile)) {
    if (const slim_status st = multiply(ctx, name, p, 1, given[0], given); st != SLIM_OK) return st;
    return multiply(ctx, name, p + 1, 1, given[1], given + 1);
  }
  if (tile == TILE_SMALL && in_order[0].nk < 2 * in_order[1].nk) return multiply(ctx, name, p, 2, tile, given);
  return multiply(ctx, name, in_order, 2, tile, own);
}

}  // namespace slimfp8
