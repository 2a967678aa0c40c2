// The scaled matrix product of the 8-bit linear layer: C[b][a] = sum over blocks of 128 of 2^(ea + eb - 254) A[a] . B[b], both operands
// rows of e4m3 numbers along the contraction; forward A = weights, B = activations; gradients: fp8_linear.hip.
//
//  * v_mfma_scale_f32_32x32x64_f8f6f4 takes the scales themselves (one byte per row and 32 of the contraction, here the same for 128),
//    so the fp32 sums stay in its registers from the first block to the last: no rescaling between blocks.
//  * Workgroup tile TA x TB, contraction 128 bytes a step, from memory to LDS directly, two stages; one wait and one barrier a step.
//    A row of a stage is 8 chunks of 16 bytes, chunk c at place c ^ (row / 2 % 8): 16 lanes that read one chunk of 16 rows hit sixteen
//    different groups of four banks.  The scales of four steps (a word per row) come the same way.
//  * The rows of A are the rows of an MFMA tile, so a lane ends up with 4 consecutive outputs of one row of C at a time; the tile goes through
//    LDS, wavefront by wavefront, and leaves in rows.
//  * Several products share a launch (the two gradients).  A product whose tiles do not fill the chip is cut along the contraction; the
//    parts go to the workspace in fp32 and are added in a fixed order by a second kernel.
#include "fp8_device.h"

namespace {

using namespace slimfp8;

constexpr int FG_BAND = 8;                 // tiles of A per band of the tile order

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
};

__device__ __forceinline__ void load_lds16(unsigned lds_addr, unsigned voff, const uint8_t* gbase) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_addr), "v"(voff), "s"(gbase) : "m0");
#else
  (void)lds_addr, (void)voff, (void)gbase;
#endif
}
__device__ __forceinline__ void load_lds4(unsigned lds_addr, unsigned voff, const uint8_t* gbase) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_addr), "v"(voff), "s"(gbase) : "m0");
#else
  (void)lds_addr, (void)voff, (void)gbase;
#endif
}

// an address that is the same in every lane, in scalar registers
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t u = (uint64_t)p;
  return (const uint8_t*)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u) |
                          (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(u >> 32)) << 32);
}

template <int TA_, int TB_, int WA_, int WB_>
struct Tile {
  static constexpr int TA = TA_, TB = TB_, WA = WA_, WB = WB_;
  static constexpr int WAVES = WA * WB, THREADS = 64 * WAVES, MA = TA / WA / 32, MB = TB / WB / 32;
  static constexpr int STAGE = (TA + TB) * BLOCK, SCALES = (TA + TB) * 4;
  static constexpr int LOADS = STAGE / 1024 / WAVES;           // direct loads of a wavefront per step
  static constexpr int OUT_LD = MA * 32 + 4;                   // floats per row of C in the epilogue
  static constexpr int OUT = WAVES * 32 * OUT_LD * 4;
  static constexpr int LDS = 2 * STAGE + 2 * SCALES > OUT ? 2 * STAGE + 2 * SCALES : OUT;
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

// EXACT: products of the numbers in bf16 (fp32 outputs)
template <typename T, bool EXACT>
__global__ __launch_bounds__(T::THREADS) void fp8_gemm(GemmArgs ga) {
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
  const int k0 = split * p.per, nk = min(p.per, p.nk - k0);
  const int wa = wave % T::WA, wb = wave / T::WA;

  // A direct load fills 1 KiB of a stage: 8 rows; the lane fetches the chunk that belongs at its place.  Rows behind the last one
  // are the last one again (their sums are not stored).
  unsigned off[T::LOADS];
#pragma unroll
  for (int i = 0; i < T::LOADS; ++i) {
    const int r = (wave * T::LOADS + i) * 8 + (lane >> 3), ch = (lane & 7) ^ ((r >> 1) & 7);
    off[i] = r < T::TA ? (unsigned)((int64_t)min(r, p.a.rows - 1 - a0) * p.a.ld) + ch * 16u
                       : (unsigned)((int64_t)min(r - T::TA, p.b.rows - 1 - b0) * p.b.ld) + ch * 16u;
  }
  const uint8_t* abase = uniform(p.a.q + (int64_t)a0 * p.a.ld + (int64_t)k0 * BLOCK);
  const uint8_t* bbase = uniform(p.b.q + (int64_t)b0 * p.b.ld + (int64_t)k0 * BLOCK);
  // scales: one load is the words of 64 rows
  const bool scale_wave = wave < (T::TA + T::TB) / 64, scale_b = wave >= T::TA / 64;
  unsigned soff = 0;
  const uint8_t* sbase = nullptr;
  if (scale_wave) {
    const Operand& o = scale_b ? p.b : p.a;
    const int r0 = scale_b ? b0 : a0, r = (scale_b ? wave - T::TA / 64 : wave) * 64 + lane;
    soff = (unsigned)((int64_t)((min(r0 + r, o.rows - 1) >> o.shift) - (r0 >> o.shift)) * o.lds);
    sbase = uniform(o.s + (int64_t)(r0 >> o.shift) * o.lds + k0);
  }
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)((__attribute__((address_space(3))) char*)smem_fg));
  auto issue = [&](int k) {
    const unsigned st = lds0 + (unsigned)(k & 1) * T::STAGE + (unsigned)wave * T::LOADS * 1024u;
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
      const bool in_a = (wave * T::LOADS + i) * 8 < T::TA;
      load_lds16(st + i * 1024u, off[i], in_a ? abase : bbase);
    }
    abase += BLOCK;
    bbase += BLOCK;
    if ((k & 3) == 0 && scale_wave) {
      load_lds4(lds0 + 2u * T::STAGE + (unsigned)((k >> 2) & 1) * T::SCALES + (unsigned)wave * 256u, soff, sbase);
      sbase += 4;
    }
  };

  v16f acc[T::MA][T::MB];
#pragma unroll
  for (int i = 0; i < T::MA; ++i)
#pragma unroll
    for (int j = 0; j < T::MB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  const int l32 = lane & 31, h = lane >> 5, sw = (l32 >> 1) & 7;
  const int ra = wa * T::MA * 32 + l32, rb = T::TA + wb * T::MB * 32 + l32;
  int sa[T::MA], sb[T::MB];
  auto fragment = [&](const char* row, int kk) {
    const uint4 lo = *reinterpret_cast<const uint4*>(row + (((kk * 4 + h * 2) ^ sw) * 16));
    const uint4 hi = *reinterpret_cast<const uint4*>(row + (((kk * 4 + h * 2 + 1) ^ sw) * 16));
    return v8i{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
  };
  if (nk > 0) issue(0);
  auto step = [&](auto index, int k) {
    constexpr int J = decltype(index)::value;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                       // everybody's loads of this step; everybody is done with the step before
    if (k + 1 < nk) issue(k + 1);
    const char* st = smem_fg + (J & 1) * T::STAGE;
    if (J == 0) {
      const int* sc = reinterpret_cast<const int*>(smem_fg + 2 * T::STAGE + ((k >> 2) & 1) * T::SCALES);
#pragma unroll
      for (int i = 0; i < T::MA; ++i) sa[i] = sc[ra + i * 32];
#pragma unroll
      for (int j = 0; j < T::MB; ++j) sb[j] = sc[rb + j * 32];
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      v8i fa[T::MA], fb[T::MB];
#pragma unroll
      for (int j = 0; j < T::MB; ++j) fb[j] = fragment(st + (rb + j * 32) * BLOCK, kk);
#pragma unroll
      for (int i = 0; i < T::MA; ++i) fa[i] = fragment(st + (ra + i * 32) * BLOCK, kk);
      if constexpr (EXACT) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v8bf ba[T::MA], bb[T::MB];
#pragma unroll
          for (int j = 0; j < T::MB; ++j) bb[j] = dequantized(fb[j][2 * q], fb[j][2 * q + 1], scale_of<J>(sb[j]));
#pragma unroll
          for (int i = 0; i < T::MA; ++i) ba[i] = dequantized(fa[i][2 * q], fa[i][2 * q + 1], scale_of<J>(sa[i]));
#pragma unroll
          for (int i = 0; i < T::MA; ++i)
#pragma unroll
            for (int j = 0; j < T::MB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ba[i], bb[j], acc[i][j], 0, 0, 0);
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < T::MA; ++i)
#pragma unroll
        for (int j = 0; j < T::MB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[i], fb[j], acc[i][j], 0, 0, J, sa[i], J, sb[j]);
    }
  };
  for (int k = 0; k < nk; k += 4) {
    step(std::integral_constant<int, 0>(), k);
    if (k + 1 < nk) step(std::integral_constant<int, 1>(), k + 1);
    if (k + 2 < nk) step(std::integral_constant<int, 2>(), k + 2);
    if (k + 3 < nk) step(std::integral_constant<int, 3>(), k + 3);
  }

  // A lane holds column b = lane % 32 of an MFMA tile and rows 8 (q / 4) + 4 h + q % 4.  32 rows of C at a time through a
  // part of LDS of the wavefront's own.
  __syncthreads();
  float* out = reinterpret_cast<float*>(smem_fg) + wave * 32 * T::OUT_LD;
  constexpr int QUADS = T::MA * 8, RPI = 64 / QUADS;           // lanes per row of C, rows per instruction
  static_assert(QUADS <= 64, "a row of a wavefront's part is read by one instruction");
  char* cbase = static_cast<char*>(p.c) + (int64_t)split * p.part * 4;
  const int esize = p.c_dtype == SLIM_F32 ? 4 : 2;
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
__global__ __launch_bounds__(256) void fp8_join(ProductArgs p, const float* __restrict__ parts, int64_t ldp, void* c, int64_t ldc, int dtype) {
  const int quads = (p.a.rows + 3) / 4;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= (int64_t)quads * p.b.rows) return;
  const int row = (int)(e / quads), col = (int)(e % quads) * 4;
  const float* src = parts + (int64_t)row * ldp + col;
  float4 s = *reinterpret_cast<const float4*>(src);
  for (int i = 1; i < p.splits; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(src + i * p.part);
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  store4(static_cast<char*>(c) + (int64_t)row * ldc * (dtype == SLIM_F32 ? 4 : 2), dtype, col, p.a.rows - col, s);
}

enum { TILE_LARGE, TILE_MEDIUM, TILE_SMALL };
typedef Tile<256, 256, 2, 4> Large;
typedef Tile<128, 128, 2, 2> Medium;
typedef Tile<64, 64, 2, 2> Small;

struct Plan {
  int tile, splits[2];
  int64_t ldp[2];
  size_t bytes;
};

template <typename T>
int tiles_of(const Product& p) { return slim_cdiv(p.a.rows, T::TA) * slim_cdiv(p.b.rows, T::TB); }

// The tile: the largest of which there are enough to fill the chip; parts: where even the smallest do not.
Plan make_plan(const Product* p, int count, int ncu) {
  Plan pl = {};
  int large = 0, medium = 0, small = 0;
  for (int i = 0; i < count; ++i) {
    large += tiles_of<Large>(p[i]);
    medium += tiles_of<Medium>(p[i]);
    small += tiles_of<Small>(p[i]);
  }
  pl.tile = large >= ncu ? TILE_LARGE : medium >= ncu / 2 ? TILE_MEDIUM : TILE_SMALL;
  const int tiles = pl.tile == TILE_LARGE ? large : pl.tile == TILE_MEDIUM ? medium : small;
  for (int i = 0; i < count; ++i) {
    int s = std::max(1, std::min(ncu / std::max(1, tiles), p[i].nk / 8));
    const int per = slim_cdiv(slim_cdiv(std::max(1, p[i].nk), s), 4) * 4;
    s = std::max(1, slim_cdiv(p[i].nk, per));
    pl.splits[i] = s;
    pl.ldp[i] = (p[i].a.rows + 3) / 4 * 4;
    if (s > 1) pl.bytes += slim_ws_round(sizeof(float) * (size_t)s * pl.ldp[i] * p[i].b.rows);
  }
  return pl;
}

template <typename T, bool EXACT>
slim_status launch(slim_ctx* ctx, const char* name, const GemmArgs& ga, int grid) {
  if (T::LDS > 64 * 1024)
    SLIM_HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_gemm<T, EXACT>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
  SLIM_LAUNCH(ctx, name, (fp8_gemm<T, EXACT>), dim3(grid), dim3(T::THREADS), T::LDS, ga);
  return SLIM_OK;
}
template <bool EXACT>
slim_status launch(slim_ctx* ctx, const char* name, int tile, const GemmArgs& ga, int grid) {
  return tile == TILE_LARGE ? launch<Large, EXACT>(ctx, name, ga, grid)
         : tile == TILE_MEDIUM ? launch<Medium, EXACT>(ctx, name, ga, grid) : launch<Small, EXACT>(ctx, name, ga, grid);
}

// products of one launch: all, or one where they differ in their kind
int in_one_launch(const Product* p, int count) { return count == 2 && (p[0].c_dtype == SLIM_F32) != (p[1].c_dtype == SLIM_F32) ? 1 : count; }

slim_status multiply(slim_ctx* ctx, const char* name, const Product* p, int count) {
  const Plan pl = make_plan(p, count, ctx->num_cus);
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
    const int ta = pl.tile == TILE_LARGE ? Large::TA : pl.tile == TILE_MEDIUM ? Medium::TA : Small::TA;
    const int tb = pl.tile == TILE_LARGE ? Large::TB : pl.tile == TILE_MEDIUM ? Medium::TB : Small::TB;
    q.tiles_a = slim_cdiv(q.a.rows, ta);
    q.tiles_b = slim_cdiv(q.b.rows, tb);
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
  const slim_status st = p[0].c_dtype == SLIM_F32 ? launch<true>(ctx, name, pl.tile, ga, grid) : launch<false>(ctx, name, pl.tile, ga, grid);
  if (st != SLIM_OK) return st;
  for (int i = 0; i < count; ++i)
    if (parts[i]) {
      const int64_t quads = (int64_t)slim_cdiv(p[i].a.rows, 4) * p[i].b.rows;
      SLIM_LAUNCH(ctx, "fp8_join", fp8_join, dim3(slim_cdiv(quads, 256)), dim3(256), 0, ga.p[i], parts[i], pl.ldp[i], p[i].c, p[i].ldc,
                  (int)p[i].c_dtype);
    }
  return SLIM_OK;
}

}  // namespace

namespace slimfp8 {

size_t gemm_workspace(const Product* p, int count, int num_cus) {
  size_t bytes = 0;
  for (int i = 0, c = in_one_launch(p, count); i < count; i += c) bytes += make_plan(p + i, c, num_cus).bytes;
  return bytes;
}

slim_status gemm(slim_ctx* ctx, const char* name, const Product* p, int count) {
  for (int i = 0, c = in_one_launch(p, count); i < count; i += c)
    if (const slim_status st = multiply(ctx, name, p + i, c); st != SLIM_OK) return st;
  return SLIM_OK;
}

}  // namespace slimfp8
