// Products of block-scaled matrices, and the forward pass of the gated block.  gfx950 only.
//   out[p][q] = alpha sum_r x[p][r] z[q][r],   x = code * 2^e of its block of 128 along r, z likewise
//   H = act(X Wg^T) (X Wu^T)
// One stage of the contraction is 128 values, one block of every row.  Two pipelines, as for per-tensor scales:
//   exact (default)   a code becomes the bfloat16 number code * 2^e, which is exact, by one conversion for two codes that takes the
//                     scale along; v_mfma_f32_16x16x32_bf16: exact products, binary32 sums
//   fp8               v_mfma_scale_f32_16x16x128_f8f6f4: codes and scales as they are, one instruction a stage; it aligns the eight
//                     products of a group to 14 bits before adding them
// Tiles: operand rows of a stage go from global memory straight into LDS (buffer_load ... lds), 128 bytes a row, 16-byte chunk c of
// row r at chunk c ^ (r / 2 % 8); the scales beside them, four bytes (four stages) a row.  The product is taken transposed inside a wave
// (Z rows as the first MFMA operand): a lane ends with four neighbouring q of one p.
// 8192^3: exact 760 to 780 us (1.41 to 1.45 PFLOP/s), fp8 446 to 491 (2.2 to 2.5), by the card.  Bound by the matrix pipeline, of which 256 x 256
// tiles leave a third idle in the exact form: LDS reads and conversions share a wave's issue with its MFMAs, and the eight waves meet once a stage
// (without any loads 678 us; four waves of 128 x 128 each spill and are slower; raised wave priorities change nothing).  Smaller tiles fill no unit:
// 1009 x 2048 x 5632 on 512 fp8 tiles of 64 x 64, 24 to 26 us, has the matrix pipeline busy in 16 % of the launch's cycles, vector issue and LDS
// reads in 20 % each; its waves, two a SIMD, live 20 us, 1100 cycles a stage (loads, barrier, LDS reads, MFMAs in a row), in which a CU gets 72 GB/s.
// Few rows (P <= 16): waves read the rows of Z from global memory into registers, once, and split the contraction between them.
#include "srq_block_plan.hpp"
#include "srq_blocks.hpp"
#include "srq_mma.hpp"

namespace srq {
namespace {

using mma::lds_void;
using mma::v4f;
using mma::v4i;
using mma::v8bf;
using mma::v8i;
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

constexpr uint32_t OOB = 0x80000000u;  // beyond any piece of an operand: loads as zero

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

// 64 lanes x 16 (or 4) bytes from `rsrc` at byte offset `voff` (out of range reads as zero) to LDS address `lds_addr` + lane * 16 (4).
// Inline so that the compiler does not wait for it: the kernel counts.
__device__ __forceinline__ void lds_dma16(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}
__device__ __forceinline__ void lds_dma4(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}

// ---- pipelines: 32 codes a lane and operand row, both rows' scale bytes ------------------------------------------------------
template <int KIND>
__device__ __forceinline__ v8bf widen8(int w0, int w1, float scale) {
  v2bf p[4];
  if constexpr (KIND == SRQ_E5M2) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)w0, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)w0, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)w1, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)w1, scale, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w0, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w0, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w1, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w1, scale, true);
  }
  return v8bf{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// One stage of a wave: TM x TN tiles of 16 x 16, sums in acc.  x: the lane's row of the wave's first tile of X in LDS; z_of(j): of tile j
// of Z.  Lane l has row l % 16 of a tile and of its codes chunks l / 16 and l / 16 + 4, at c0 and c1.  sx, sz: the rows' scale bytes (low byte).
// LDS reads run two steps ahead and are spread between the MFMAs, as is the widening of the next step's operand.
constexpr int BK = 128;
template <int KX, int KZ, int TM, int TN, class Z, class Issue>
__device__ __forceinline__ void multiply_stage_f8(v4f (&acc)[TM][TN], const uint8_t* x, Z z_of, uint32_t c0, uint32_t c1,
                                                  const uint32_t (&sx)[TM], const uint32_t (&sz)[TN], Issue issue) {
  constexpr int FX = KX == SRQ_E5M2 ? 1 : 0, FZ = KZ == SRQ_E5M2 ? 1 : 0, AHEAD = TM < 3 ? TM : 3;
  auto frag = [&](const uint8_t* row) {
    const v4i a = *reinterpret_cast<const v4i*>(row + c0), b = *reinterpret_cast<const v4i*>(row + c1);
    return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  };
  v8i zf[TN], xf[AHEAD];
  xf[0] = frag(x);
#pragma unroll
  for (int j = 0; j < TN; ++j) zf[j] = frag(z_of(j));
#pragma unroll
  for (int i = 1; i < AHEAD; ++i) xf[i] = frag(x + i * 16 * BK);
  __builtin_amdgcn_sched_barrier(0);
  issue();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(zf[j], xf[i % AHEAD], acc[i][j], FZ, FX, 0, (int)sz[j], 0, (int)sx[i]);
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < TM) xf[i % AHEAD] = frag(x + (i + AHEAD) * 16 * BK);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The products of a stage's last step wait until the next stage's first reads are under way: after the barrier between them the matrix
// pipeline would have nothing to do until those have come.  What they need is kept here; zeros before a tile's first stage.
template <int TM, int TN>
struct ExactCarry {
  v8bf x[2][2], z[TN][2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[1][h] = v8bf{};
#pragma unroll
      for (int j = 0; j < TN; ++j) z[j][h] = v8bf{};
    }
  }
  __device__ __forceinline__ void multiply(v4f (&acc)[TM][TN]) const {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[TM - 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z[j][0], x[1][0], acc[TM - 1][j], 0, 0, 0);
      acc[TM - 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z[j][1], x[1][1], acc[TM - 1][j], 0, 0, 0);
    }
  }
};

template <int KX, int KZ, int TM, int TN, class Z, class Issue>
__device__ __forceinline__ void multiply_stage_exact(v4f (&acc)[TM][TN], ExactCarry<TM, TN>& last, const uint8_t* x, Z z_of, uint32_t c0, uint32_t c1,
                                                     const uint32_t (&sx)[TM], const uint32_t (&sz)[TN], Issue issue) {
  constexpr int STEPS = 2 * TM;  // half a row's codes of one tile of X
  v4i xr[3], zr[TN];
  auto& xe = last.x;
  auto& ze = last.z;
  auto read_x = [&](int n) { return *reinterpret_cast<const v4i*>(x + (n % TM) * 16 * BK + (n < TM ? c0 : c1)); };
  xr[0] = read_x(0);
#pragma unroll
  for (int j = 0; j < TN; ++j) zr[j] = *reinterpret_cast<const v4i*>(z_of(j) + c0);
  xr[1] = read_x(1);
  __builtin_amdgcn_sched_barrier(0);
  last.multiply(acc);
  __builtin_amdgcn_sched_barrier(0);
  issue();
  __builtin_amdgcn_sched_barrier(0);
  float fx[TM], fz[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) fx[i] = __uint_as_float((sx[i] & 255u) << 23);
#pragma unroll
  for (int j = 0; j < TN; ++j) fz[j] = __uint_as_float((sz[j] & 255u) << 23);
  auto widen_x = [&](int n) {
    const v4i& r = xr[n % 3];
    xe[n & 1][0] = widen8<KX>(r[0], r[1], fx[n % TM]);
    xe[n & 1][1] = widen8<KX>(r[2], r[3], fx[n % TM]);
  };
  auto widen_z = [&](int j) {
    ze[j][0] = widen8<KZ>(zr[j][0], zr[j][1], fz[j]);
    ze[j][1] = widen8<KZ>(zr[j][2], zr[j][3], fz[j]);
  };
  widen_x(0);
  widen_z(0);
#pragma unroll
  for (int n = 0; n < STEPS - 1; ++n) {
    const int i = n % TM;
    const bool first = n == 0, turn = n == TM - 1;
    if (n + 2 < STEPS) xr[(n + 2) % 3] = read_x(n + 2);
    if (n == (TM > 1 ? 1 : 0) && TM > 1) {
#pragma unroll
      for (int j = 0; j < TN; ++j) zr[j] = *reinterpret_cast<const v4i*>(z_of(j) + c1);
    }
    widen_x(n + 1);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ze[j][0], xe[n & 1][0], acc[i][j], 0, 0, 0);
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ze[j][1], xe[n & 1][1], acc[i][j], 0, 0, 0);
      if (first && j + 1 < TN) widen_z(j + 1);
      if (turn) {
        if constexpr (TM == 1) zr[j] = *reinterpret_cast<const v4i*>(z_of(j) + c1);
        widen_z(j);
      }
    }
    // (the reads first: left to itself the compiler puts them right before their use, a step later)
    __builtin_amdgcn_sched_group_barrier(0x100, 1 + TN, 0);
#pragma unroll
    for (int m = 0; m < 2 * TN; ++m) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (first || turn) __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
      else __builtin_amdgcn_sched_group_barrier(0x002, (8 + 2 * TN - 1) / (2 * TN), 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ---- tiles ------------------------------------------------------------------------------------------------------------------
struct TileParams {
  BlockOperand X, Z;
  uint32_t P, Q, R;          // R: up to the end of the last 16 codes
  uint32_t tiles_p, tiles_q;
  // XCD x has tiles [x chunk, (x + 1) chunk); of them the first `whole` are one item of work each, the others `nsplit`, over
  // stages_per_split stages of the contraction each, whose sums go to `partial`, a tile of BM x BN for every slice of every such tile
  uint32_t chunk, whole, nsplit, stages_per_split;
  float* partial;
  void* out;
  float alpha;
  int out_bf16, accumulate;
  // the gated block
  uint32_t F;
  uint8_t *h_scales, *gu, *gu_scales;
  int h_codes;
  Rounding rnd_h, rnd_gu;
};

// Place of tile n in the output: bands of eight tile rows, column by column.
__device__ __forceinline__ void tile_at(const TileParams& g, uint32_t tile, uint32_t& tp, uint32_t& tq) {
  constexpr uint32_t GROUP = 8;
  const uint32_t band = tile / (GROUP * g.tiles_q), in_band = tile - band * GROUP * g.tiles_q;
  const uint32_t band_rows = min(GROUP, g.tiles_p - band * GROUP);
  tp = band * GROUP + in_band % band_rows;
  tq = in_band / band_rows;
}

__device__ __forceinline__ void store_results(const TileParams& g, uint32_t p, uint32_t q, v4f v, bool vec) {
  const size_t at = (size_t)p * g.Q + q;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __fmul_rn(v[e], g.alpha);
  if (g.out_bf16) {
    typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
    __bf16* const o = static_cast<__bf16*>(g.out) + at;
    if (vec) *reinterpret_cast<v4bf*>(o) = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    else
      for (int e = 0; e < 4 && q + e < g.Q; ++e) o[e] = (__bf16)v[e];
  } else {
    float* const o = static_cast<float*>(g.out) + at;
    if (vec) {
      if (g.accumulate) v += *reinterpret_cast<const v4f*>(o);
      __builtin_nontemporal_store(v, reinterpret_cast<v4f*>(o));
    } else {
      for (int e = 0; e < 4 && q + e < g.Q; ++e) o[e] = g.accumulate ? v[e] + o[e] : v[e];
    }
  }
}

// One row's sums of a block of 128 hidden columns to H and the checkpoint.  Sixteen neighbouring lanes hold the row, eight columns each
// (a of G, u of U), so that a block's largest is theirs, a lane's values are one group of thresholds and its codes eight bytes.
// The row: r of the tile that begins at (p0, f0), which are the wave's; places within the tile are products of 24 bits and take 32.
template <int GATED>
__device__ __forceinline__ void gated_row(const TileParams& g, const float (&a)[8], const float (&u)[8], uint32_t p0, uint32_t r, uint32_t f0) {
  const uint32_t cg = threadIdx.x & 15u, rf = __umul24(r, g.F) + 8 * cg, rk = __umul24(r, 2 * g.F) + 8 * cg;
  const uint32_t nb = g.F / SBLOCK, hp = (nb + 3) / 4 * 4, kp = (2 * nb + 3) / 4 * 4;
  const size_t tile_h = (size_t)p0 * g.F + f0, tile_k = (size_t)p0 * 2 * g.F + f0;
  float h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float act, slope;
    activate<GATED == 2 ? SRQ_ACT_GELU : SRQ_ACT_SILU>(a[e], act, slope);
    h[e] = act * u[e];
  }
  auto put = [&](const float (&v)[8], uint8_t* codes, uint8_t* scale, const Rounding& rnd, size_t first) {
    const Extent x = extent_of(v);
    const uint32_t byte = scale_byte<SRQ_E4M3>(max16(most_finite(v, x)));
    uint32_t w[4];
    if (rnd.sr) {
      thresholds<true>(rnd, first_block(rnd.counter_offset, rnd.counter_dev) + first / 8, w);
      *reinterpret_cast<u32x2*>(codes) = codes_of_octet<SRQ_E4M3, true>(v, x, byte, w);
    } else {
      thresholds<false>(rnd, 0, w);
      *reinterpret_cast<u32x2*>(codes) = codes_of_octet<SRQ_E4M3, false>(v, x, byte, w);
    }
    if (cg == 0) *scale = (uint8_t)byte;
  };
  if (g.h_codes) {
    put(h, static_cast<uint8_t*>(g.out) + tile_h + rf, g.h_scales + ((size_t)p0 * hp + f0 / SBLOCK) + __umul24(r, hp), g.rnd_h, tile_h + rf);
  } else {
    typedef __bf16 v8b __attribute__((ext_vector_type(8)));
    v8b b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (__bf16)h[e];
    *reinterpret_cast<v8b*>(static_cast<__bf16*>(g.out) + tile_h + rf) = b;
  }
  if (g.gu) {
    uint8_t* const codes = g.gu + tile_k;
    uint8_t* const scale = g.gu_scales + ((size_t)p0 * kp + f0 / SBLOCK);
    const uint32_t rs = __umul24(r, kp);
    put(a, codes + rk, scale + rs, g.rnd_gu, tile_k + rk);
    put(u, codes + g.F + rk, scale + nb + rs, g.rnd_gu, tile_k + g.F + rk);
  }
}

// A workgroup walks a list of tiles: the loads of the next tile's first stages are under way while it finishes one.  With two
// stages the ring has one in flight; it has landed by the time the results go out (every wave looks before it stores), so that the first
// wait of the next tile does not stand behind the stores.
// GATED: BN = 256 rows of Z are 128 of Wg and the 128 of Wu that go with them; a wave has the same columns of both, so that the activation and the
// product are on sums that never leave the chip.  16384 x 2048 x 5632 SiLU, H and checkpoint in E4M3: 635 to 650 us (1.16 to 1.19 PFLOP/s), without the
// checkpoint 575, H in bfloat16 by the fp8 pipeline 348; the finish of the tiles, vector work, is 150 of the first.  113 rows of the same, GELU, on 176
// tiles of 32 x 256: 19.5 us; vector work (widening, the finish) fills 37 % of the issue slots of the CUs that have a tile, the matrix pipeline
// 13 %, and a CU, with one workgroup and two stages ahead, gets 31 GB/s.
struct Item {
  uint32_t p0, q0, kt, kt1;  // first row and column, stages of the contraction [kt, kt1)
  float* partial;            // null: the whole contraction
  bool valid;
};

constexpr int max_of(int a, int b) { return a > b ? a : b; }
template <int BM, int BN, int STAGES>
constexpr int tile_lds() { return STAGES * ((BM + BN) * BK + (max_of(BM, 64) + BN) * 4) + 1024; }

template <int KX, int KZ, bool F8, int BM, int BN, int WGM, int WGN, int STAGES, int GATED>
__global__ __launch_bounds__(WGM* WGN * 64) void block_tile_kernel(TileParams g) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  constexpr int NW = WGM * WGN;
  constexpr int WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 16, TN = WTN / 16;
  constexpr int SXROWS = max_of(BM, 64), CODES = (BM + BN) * BK, STAGE = CODES + (SXROWS + BN) * 4;
  // loads a wave and stage: of 8 rows of X, of 8 rows of Z, of 64 rows' scales; what is not there reads as zeros into a spare kilobyte,
  // so that every wave has the same number in flight
  constexpr int XB = BM / 8, ZB = BN / 8, SXB = SXROWS / 64, SB = SXB + BN / 64;
  constexpr int XL = (XB + NW - 1) / NW, ZL = ZB / NW, SLW = (SB + NW - 1) / NW, LOADS = XL + ZL + SLW;
  static_assert(ZL * NW == ZB && (ZL == 1 || ZL % 2 == 0) && (XL == 1 || (XL % 2 == 0 && XL * NW == XB)), "whole loads");
  static_assert(!GATED || (BN == 256 && TN % 2 == 0), "128 columns of G and the same of U");
  const uint32_t tid = threadIdx.x, lane = tid & 63u;
  const uint32_t wave = uniform(tid >> 6);
  const uint32_t wp = wave / WGN, wq = wave % WGN;
  const uint32_t lds_base = (uint32_t)(size_t)(lds_void*)lds;

  // XCD x (workgroup ids = x mod 8) has a contiguous range of the tiles, which its workgroups walk side by side
  const uint32_t ntiles = g.tiles_p * g.tiles_q, stages = (g.R + BK - 1) / BK;
  const uint32_t xcd = blockIdx.x & 7u, slots = gridDim.x >> 3, first_tile = xcd * g.chunk;
  const uint32_t mine = first_tile < ntiles ? min(ntiles - first_tile, g.chunk) : 0u;
  const uint32_t rest = g.chunk - g.whole;  // (tiles of an XCD in slices; the last XCDs may have fewer)
  uint32_t next_work = blockIdx.x >> 3;
  auto next_item = [&]() {
    Item it = {0, 0, 0, 0, nullptr, false};
    uint32_t tile = 0;
    while (true) {
      const uint32_t w = next_work;
      next_work += slots;
      if (w < g.whole) {
        if (w >= mine) continue;
        tile = w;
        it.kt1 = stages;
      } else {
        const uint32_t slice = rest ? (w - g.whole) / rest : g.nsplit;
        if (slice >= g.nsplit) return it;
        tile = w - slice * rest;
        if (tile >= mine) continue;
        it.kt = slice * g.stages_per_split;
        it.kt1 = min(stages, it.kt + g.stages_per_split);
        it.partial = g.partial + (((size_t)xcd * rest + tile - g.whole) * g.nsplit + slice) * (BM * BN);
      }
      break;
    }
    uint32_t tp, tq;
    tile_at(g, first_tile + tile, tp, tq);
    it.p0 = tp * BM;
    it.q0 = tq * (GATED ? BN / 2 : BN);
    it.valid = true;
    return it;
  };

  // Loads.  A buffer begins at the tile's first row and ends with its last, so that offsets are small whatever the operand's size.  The
  // rows of Z that a wave loads are all of Wg or all of Wu, the scales those of 64 rows of X or of either.
  constexpr uint32_t ZN = GATED ? BN / 2 : BN;  // rows of Z from one place
  static_assert(!GATED || (ZN % (ZL * 8) == 0 && ZN % 64 == 0), "");
  const uint32_t zrows = GATED ? g.F : g.Q;
  const uint32_t xpitch = (uint32_t)g.X.pitch, zpitch = (uint32_t)g.Z.pitch;
  const bool up = GATED && wave * ZL * 8 >= ZN;
  const uint8_t *xbase = nullptr, *zbase = nullptr, *sbase[SLW];
  uint32_t xbytes = 0, zbytes = 0, sbytes[SLW], sstep[SLW];
  auto rows_left = [](uint32_t first, uint32_t rows, uint32_t most) { return first < rows ? min(rows - first, most) : 0u; };
  auto load_from = [&](const Item& it) {
    const uint32_t xn = rows_left(it.p0, g.P, BM), zn = rows_left(it.q0, zrows, ZN);
    xbase = g.X.codes + it.p0 * g.X.pitch;
    xbytes = XL * NW > XB && wave >= XB ? 0u : xn * xpitch;
    zbase = g.Z.codes + (it.q0 + (up ? (size_t)g.F : 0)) * g.Z.pitch;
    zbytes = zn * zpitch;
#pragma unroll
    for (int i = 0; i < SLW; ++i) {
      const uint32_t n = wave + i * NW, r0 = n < SXB ? n * 64 : (n - SXB) * 64;
      const bool is_x = n < SXB, u = GATED && !is_x && r0 >= ZN;
      const uint32_t first = r0 - (u ? ZN : 0u), rows = n >= SB ? 0u : is_x ? xn : zn;
      const uint8_t* const scales = is_x ? g.X.scales : g.Z.scales;
      sstep[i] = is_x ? (uint32_t)g.X.spitch : (uint32_t)g.Z.spitch;
      const uint8_t* const at = scales + ((is_x ? it.p0 : it.q0 + (u ? (size_t)g.F : 0)) + first) * sstep[i];
      // (uniform, which the compiler does not see of a choice between two)
      sbase[i] = reinterpret_cast<const uint8_t*>((size_t)uniform((uint32_t)((size_t)at >> 32)) << 32 | (size_t)uniform((uint32_t)(size_t)at));
      sbytes[i] = uniform((first < rows ? rows - first : 0u) * sstep[i]);
    }
  };
  auto rsrc = [](const uint8_t* base, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)bytes, 0x00020000); };
  // chunk of a row that lane l fetches for the LDS place l of an instruction's 1 KiB (8 rows): rows of even and odd blocks of 8
  const uint32_t lrow = lane >> 3, lchunk0 = ((lane & 7u) ^ (lane >> 4)) * 16, lchunk1 = lchunk0 ^ 64u;
  const uint32_t xoff = lrow * xpitch, zoff = lrow * zpitch;
  constexpr uint32_t SPARE = STAGES * STAGE;
  auto issue = [&](uint32_t kt, uint32_t buf) {
    const uint32_t base = lds_base + buf * STAGE, k = kt * BK;
    const uint32_t left = g.R - k;  // codes from here on
    const uint32_t dead0 = lchunk0 < left ? 0u : OOB, dead1 = lchunk1 < left ? 0u : OOB;
    const auto xr = rsrc(xbase, xbytes), zr = rsrc(zbase, zbytes);
    const uint32_t x0 = (xoff + lchunk0) | dead0, x1 = (xoff + lchunk1) | dead1, z0 = (zoff + lchunk0) | dead0, z1 = (zoff + lchunk1) | dead1;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const uint32_t blk = wave * XL + i, odd = XL == 1 ? (blk & 1u) : (uint32_t)(i & 1);
      const bool spare = XL * NW > XB && blk >= XB;
      lds_dma16(xr, spare ? lds_base + SPARE : base + blk * 1024, (odd ? x1 : x0) + (blk * 8 * xpitch + k));
    }
#pragma unroll
    for (int i = 0; i < ZL; ++i) {
      const uint32_t blk = wave * ZL + i, odd = ZL == 1 ? (blk & 1u) : (uint32_t)(i & 1);
      lds_dma16(zr, base + BM * BK + blk * 1024, (odd ? z1 : z0) + ((blk * 8 - (up ? ZN : 0u)) * zpitch + k));
    }
#pragma unroll
    for (int i = 0; i < SLW; ++i) {
      const uint32_t n = wave + i * NW;
      const bool spare = SLW * NW > SB && n >= SB;
      lds_dma4(rsrc(sbase[i], sbytes[i]), spare ? lds_base + SPARE : base + CODES + n * 256, lane * sstep[i] + (kt & ~3u));
    }
  };

  // operand reads: lane (row = lane % 16, group = lane / 16) has chunks group and group + 4 of its row (which of them is the same for both operands).
  // LDS serves a read of 16 bytes a lane in sets of sixteen lanes: 0-3, 12-15 and 20-27, then 4-11, 16-19 and 28-31, so two groups' rows have to fall on
  // different banks (with chunks 2 group and 2 group + 1 every read took four cycles more).
  const uint32_t r16 = lane & 15u, grp = lane >> 4, sw = (lane >> 1) & 7u;
  const uint32_t c0 = (grp ^ sw) << 4, c1 = c0 ^ 64u;
  const uint32_t xrow = wp * WTM + r16;
  auto zrow = [&](int j) {  // LDS row of the wave's tile j of Z
    return GATED ? (j < TN / 2 ? 0u : (uint32_t)ZN) + wq * (WTN / 2) + (uint32_t)(j % (TN / 2)) * 16 + r16 : wq * WTN + (uint32_t)j * 16 + r16;
  };
  v4f acc[TM][TN];
  ExactCarry<TM, TN> last;
  auto compute = [&](uint32_t kt, uint32_t buf, auto issue) {
    const uint8_t* const x = lds + buf * STAGE;
    const uint8_t* const z = x + BM * BK;
    const uint32_t* const sc = reinterpret_cast<const uint32_t*>(x + CODES);
    const uint32_t shift = (kt & 3u) * 8;
    uint32_t sx[TM], sz[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) sx[i] = sc[xrow + i * 16] >> shift;
#pragma unroll
    for (int j = 0; j < TN; ++j) sz[j] = sc[SXROWS + zrow(j)] >> shift;
    const auto z_of = [&](int j) { return z + zrow(j) * BK; };
    if constexpr (F8) multiply_stage_f8<KX, KZ>(acc, x + xrow * BK, z_of, c0, c1, sx, sz, issue);
    else multiply_stage_exact<KX, KZ>(acc, last, x + xrow * BK, z_of, c0, c1, sx, sz, issue);
  };

  Item cur = next_item(), ahead = cur, nxt = cur;  // multiplied; loaded; the one after that (ahead may be on it)
  if (!cur.valid) return;
  nxt = next_item();
  uint32_t ahead_kt = ahead.kt, issued = 0, gs = 0;  // stages issued and multiplied so far, over all tiles
  auto issue_next = [&]() {
    if (ahead_kt >= ahead.kt1) {
      if (!nxt.valid || nxt.p0 == ~0u) return;
      ahead = nxt;
      ahead_kt = ahead.kt;
      load_from(ahead);
      nxt.p0 = ~0u;  // taken
      if (ahead_kt >= ahead.kt1) return;  // (a contraction over nothing)
    }
    issue(ahead_kt++, issued % STAGES);
    ++issued;
  };
  load_from(ahead);
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue_next();
  bool landed = false;
  while (true) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    if constexpr (!F8) last.clear();
    for (uint32_t kt = cur.kt; kt < cur.kt1; ++kt) {
      // stage gs has landed; up to STAGES - 2 later ones may be in flight
      if (STAGES > 2 && issued - gs == STAGES - 1) {
        wait_vmcnt<(STAGES - 2) * LOADS>();
      } else if (!landed) {
        wait_vmcnt<0>();
      }
      landed = false;
      __syncthreads();  // ... for every wave, and every wave has left the stage before
      compute(kt, gs % STAGES, issue_next);
      ++gs;
    }
    if constexpr (!F8) last.multiply(acc);
    if constexpr (STAGES == 2) {
      wait_vmcnt<0>();  // the next tile's first stage
      landed = true;
    }
    const uint32_t lo = opaque(lane);
    if (cur.partial) {
      // MFMA result register r of lane l: q = 4 (l / 16) + r, p = l % 16
      float* const o = cur.partial + (wp * WTM + (lo & 15u)) * BN + wq * (GATED ? WTN / 2 : WTN) + 4 * (lo >> 4);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if (cur.p0 + wp * WTM + i * 16 + (lo & 15u) >= g.P) continue;
          const uint32_t col = GATED ? (j < TN / 2 ? 0u : SBLOCK) + (j % (TN / 2)) * 16 : j * 16;
          *reinterpret_cast<v4f*>(o + i * 16 * BN + col) = acc[i][j];
        }
    } else if constexpr (!GATED) {
      const bool q_vec = (g.Q & 3u) == 0;
      const uint32_t pr = cur.p0 + wp * WTM + (lo & 15u), qr = cur.q0 + wq * WTN + 4 * (lo >> 4);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const uint32_t p = pr + i * 16, q = qr + j * 16;
          if (p < g.P && q < g.Q) store_results(g, p, q, acc[i][j], q_vec);
        }
    } else {
      // The sums go to LDS as they are, into the buffer of the last stage, some rows at a time, a row of G's and U's 128 columns each
      // (and a gap, so that sixteen rows written at one column fall on different banks), and come back a row at a time.
      constexpr int PITCH = 2 * SBLOCK + 4;
      constexpr int FIT = STAGE / (PITCH * 4) / (WGM * 16), IH = FIT >= 4 && TM >= 4 ? 4 : FIT >= 2 && TM >= 2 ? 2 : 1;  // tiles of a wave at a time
      static_assert(FIT >= 1 && TM % IH == 0, "");
      float* const sums = reinterpret_cast<float*>(lds + (gs + STAGES - 1) % STAGES * STAGE);
#pragma unroll
      for (int part = 0; part < TM / IH; ++part) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < IH; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const uint32_t col = (j < TN / 2 ? 0u : SBLOCK) + wq * (WTN / 2) + (j % (TN / 2)) * 16 + 4 * (lo >> 4);
            *reinterpret_cast<v4f*>(sums + ((wp * IH + i) * 16 + (lo & 15u)) * PITCH + col) = acc[part * IH + i][j];
          }
        __syncthreads();
#pragma unroll 1
        for (uint32_t r = tid / 16; r < WGM * IH * 16; r += NW * 4) {
          const uint32_t row = r / (IH * 16) * WTM + part * IH * 16 + r % (IH * 16);
          if (cur.p0 + row >= g.P) continue;
          const float* const at = sums + r * PITCH + 8 * (tid & 15u);
          const v4f a0 = *reinterpret_cast<const v4f*>(at), a1 = *reinterpret_cast<const v4f*>(at + 4);
          const v4f u0 = *reinterpret_cast<const v4f*>(at + SBLOCK), u1 = *reinterpret_cast<const v4f*>(at + SBLOCK + 4);
          gated_row<GATED>(g, {a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]}, {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]},
                           cur.p0, row, cur.q0);
        }
      }
    }
    // on to the tile whose loads are under way
    if (nxt.valid && nxt.p0 == ~0u) {
      cur = ahead;
      nxt = next_item();
    } else if (nxt.valid) {  // (not begun: a tile without stages)
      cur = nxt;
      ahead = nxt;
      ahead_kt = ahead.kt;
      load_from(ahead);
      nxt = next_item();
    } else {
      break;
    }
  }
}

// The tiles in slices: their sums in order, and on to what a whole tile's sums become.  A workgroup has 8 rows of a tile (product: a quad of
// columns a thread) or 16 (gated: sixteen lanes a row).
template <int BM, int BN, int GATED>
__global__ __launch_bounds__(256) void block_slices_kernel(TileParams g) {
  constexpr uint32_t ROWS = GATED ? 16 : 1024 / BN, PIECES = BM / ROWS;
  const uint32_t n = blockIdx.x / PIECES, piece = blockIdx.x % PIECES, rest = g.chunk - g.whole;
  const uint32_t tile = n / rest * g.chunk + g.whole + n % rest;
  if (tile >= g.tiles_p * g.tiles_q) return;
  uint32_t tp, tq;
  tile_at(g, tile, tp, tq);
  const uint32_t r = piece * ROWS + (GATED ? threadIdx.x / 16 : threadIdx.x / (BN / 4)), p = tp * BM + r;
  if (p >= g.P) return;
  const float* const at = g.partial + (size_t)n * g.nsplit * (BM * BN) + r * BN + (GATED ? 8 * (threadIdx.x & 15u) : 4 * (threadIdx.x % (BN / 4)));
  if constexpr (GATED) {
    v4f v[4] = {};
#pragma unroll 4
    for (uint32_t s = 0; s < g.nsplit; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += *reinterpret_cast<const v4f*>(at + s * (BM * BN) + (k >> 1) * SBLOCK + (k & 1) * 4);
    gated_row<GATED>(g, {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]},
                     {v[2][0], v[2][1], v[2][2], v[2][3], v[3][0], v[3][1], v[3][2], v[3][3]}, tp * BM, r, tq * (BN / 2));
  } else {
    const uint32_t q = tq * BN + 4 * (threadIdx.x % (BN / 4));
    if (q >= g.Q) return;
    v4f v = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t s = 0; s < g.nsplit; ++s) v += *reinterpret_cast<const v4f*>(at + s * (BM * BN));
    store_results(g, p, q, v, (g.Q & 3u) == 0);
  }
}

// ---- few rows -----------------------------------------------------------------------------------------------------------------
// Up to FEW rows of X: the rows of Z are what takes time, and each is read once, straight into registers: a wave has sixteen rows, whose
// lanes read a stage of 128 bytes of each in two loads of 64, AHEAD stages under way, and X's beside them (which sixteen codes a lane has is
// the same for both).  Of a workgroup's eight waves `share` (1 << log_share) split a contraction between them and add their sums through LDS
// in order; the launch gives a wave AHEAD stages where eight of them reach that far, so that all loads are one latency (beyond 4096 values: two and more).
// SUMS: the gated block, whose sums go to `partial` as the tiles of block_slices_kernel<FEW, 256>, which finishes them.
// Bound by the launch and latencies in a row: one row, 2048 x 128 takes 4.0 us, 2048 x 5632 (128 workgroups, five or six stages a wave) 7.7 (as tiles in slices 12, in two launches; X in
// LDS first 7.9; the fp8 pipeline instead of the widening, or sixteen waves a workgroup, no faster).
constexpr uint32_t FEW = FEW_ROWS, FEW_WAVES = 8;

template <int KX, int KZ, bool SUMS>
__global__ __launch_bounds__(FEW_WAVES * 64) void block_few_kernel(TileParams g, uint32_t log_share, uint32_t first) {
  __shared__ v4f sums[FEW_WAVES * 64];
  constexpr uint32_t AHEAD = 4;
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uniform(tid >> 6), r16 = lane & 15u, grp = lane >> 4;
  const uint32_t stages = (g.R + BK - 1) / BK, share = 1u << log_share, part = wave & (share - 1);
  const uint32_t q0 = ((first + blockIdx.x) * FEW_WAVES + wave) >> log_share << 4, zn = q0 < g.Q ? min(g.Q - q0, 16u) : 0u;  // this wave's rows of Z
  auto rows = [](const uint8_t* base, size_t pitch, size_t first, uint32_t n) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base) + first * pitch, 0, (int)(n * (uint32_t)pitch), 0x00020000);
  };
  const auto zr = rows(g.Z.codes, g.Z.pitch, q0, zn), zsr = rows(g.Z.scales, g.Z.spitch, q0, zn);
  const auto xr = rows(g.X.codes, g.X.pitch, 0, g.P), xsr = rows(g.X.scales, g.X.spitch, 0, g.P);
  const uint32_t xrow = min(r16, g.P - 1);  // (columns of the MFMA beyond the rows repeat the last; their results go nowhere)
  const uint32_t zoff = r16 * (uint32_t)g.Z.pitch + grp * 16, xoff = xrow * (uint32_t)g.X.pitch + grp * 16;
  const uint32_t zsoff = r16 * (uint32_t)g.Z.spitch, xsoff = xrow * (uint32_t)g.X.spitch;
  const uint32_t begin = (part * stages) >> log_share, end = ((part + 1) * stages) >> log_share;
  v4i z[AHEAD][2], x[AHEAD][2];
  uint32_t zs[AHEAD], xs[AHEAD];
  auto fetch = [&](uint32_t i, uint32_t s) {  // (behind the last stage zeros)
    const uint32_t k = s * BK, left = s < end ? g.R - k : 0u;
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      const uint32_t dead = grp * 16 + h * 64 < left ? 0u : OOB;
      z[i][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(zr, (zoff + k + h * 64) | dead, 0, KEPT));
      x[i][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(xr, (xoff + k + h * 64) | dead, 0, KEPT));
    }
    zs[i] = __builtin_amdgcn_raw_buffer_load_b8(zsr, left ? zsoff + s : OOB, 0, KEPT);
    xs[i] = __builtin_amdgcn_raw_buffer_load_b8(xsr, left ? xsoff + s : OOB, 0, KEPT);
  };
#pragma unroll
  for (uint32_t i = 0; i < AHEAD; ++i) fetch(i, begin + i);
  v4f acc[2] = {};
  for (uint32_t s = begin; s < end; s += AHEAD) {
#pragma unroll
    for (uint32_t i = 0; i < AHEAD; ++i) {
      const float fz = __uint_as_float(zs[i] << 23), fx = __uint_as_float(xs[i] << 23);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<KZ>(z[i][h][2 * e], z[i][h][2 * e + 1], fz),
                                                           widen8<KX>(x[i][h][2 * e], x[i][h][2 * e + 1], fx), acc[e], 0, 0, 0);
      fetch(i, s + AHEAD + i);
    }
  }
  acc[0] += acc[1];
  // MFMA result register r of lane l: q = 4 (l / 16) + r, p = l % 16
  if (share > 1) {
    sums[tid] = acc[0];
    __syncthreads();
    if (part == 0)
      for (uint32_t w = 1; w < share; ++w) acc[0] += sums[tid + w * 64];
  }
  const uint32_t q = q0 + 4 * grp;
  if (part != 0 || r16 >= g.P || q >= g.Q) return;
  if constexpr (SUMS) {
    const uint32_t f = q < g.F ? q : q - g.F;
    *reinterpret_cast<v4f*>(g.partial + (f / SBLOCK * FEW + r16) * (2 * SBLOCK) + (q < g.F ? 0u : SBLOCK) + f % SBLOCK) = acc[0];
  } else {
    store_results(g, r16, q, acc[0], (g.Q & 3u) == 0);
  }
}

template <int KX, int KZ, bool SUMS>
hipError_t launch_few(const TileParams& g, hipStream_t stream) {
  const uint32_t stages = (g.R + BK - 1) / BK, tiles = (g.Q + 15) / 16;
  uint32_t log_share = 0;
  while (log_share < 3 && stages > 4u << log_share) ++log_share;
  in_launches(((tiles << log_share) + FEW_WAVES - 1) / FEW_WAVES,
              [&](uint32_t first, unsigned wgs) { block_few_kernel<KX, KZ, SUMS><<<wgs, FEW_WAVES * 64, 0, stream>>>(g, log_share, first); });
  return hipGetLastError();
}

template <int KX, int KZ, bool F8, int BM, int BN, int WGM, int WGN, int STAGES, int GATED>
hipError_t launch_tiles(TileParams g, const BlockCut& c, int per_cu, hipStream_t stream) {
  constexpr int LDS = tile_lds<BM, BN, STAGES>();
  static_assert(LDS <= 160 * 1024, "LDS of a CU");
  const auto kernel = block_tile_kernel<KX, KZ, F8, BM, BN, WGM, WGN, STAGES, GATED>;
  static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (once != hipSuccess) return once;
  g.tiles_p = (g.P + BM - 1) / BM;
  g.tiles_q = GATED ? g.F / (BN / 2) : (g.Q + BN - 1) / BN;
  g.chunk = c.chunk;
  g.whole = c.whole;
  g.nsplit = c.nsplit;
  g.stages_per_split = c.per_split;
  const uint32_t rest = c.chunk - c.whole, items = c.whole + rest * c.nsplit;  // of an XCD
  kernel<<<8 * std::min(items, 32u * per_cu), WGM * WGN * 64, LDS, stream>>>(g);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (rest) {
    constexpr uint32_t PIECES = BM / (GATED ? 16 : 1024 / BN);
    block_slices_kernel<BM, BN, GATED><<<8 * rest * PIECES, 256, 0, stream>>>(g);
  }
  return hipGetLastError();
}

}  // namespace

size_t block_product_workspace(size_t P, size_t Q, size_t R, int f8) { return P > FEW && Q ? product_cut(P, Q, R, f8).partial_bytes : 0; }
size_t gated_forward_workspace(size_t M, size_t F, size_t K, int f8) { return M > FEW ? gated_cut(M, F, K, f8).partial_bytes : M ? 2 * F * FEW * sizeof(float) : 0; }

hipError_t launch_block_product(const BlockProduct& p, hipStream_t stream) {
  TileParams g = {};
  g.X = p.X; g.Z = p.Z;
  g.P = (uint32_t)p.P; g.Q = (uint32_t)p.Q; g.R = (uint32_t)((p.R + 15) / 16 * 16);
  g.out = p.out; g.partial = p.partial; g.alpha = p.alpha; g.out_bf16 = p.out_bf16; g.accumulate = p.accumulate;
  const BlockCut c = p.P > FEW ? product_cut(p.P, p.Q, p.R, p.f8) : BlockCut{};
  const auto as = [&](auto kx, auto kz, auto f8) {
    if (p.P <= FEW) return launch_few<kx.value, kz.value, false>(g, stream);
    switch (c.form) {
      case 0: return launch_tiles<kx.value, kz.value, f8.value, 256, 256, 2, 4, 2, 0>(g, c, 1, stream);
      case 1: return launch_tiles<kx.value, kz.value, f8.value, 128, 128, 2, 2, 2, 0>(g, c, 2, stream);
      case 2: return launch_tiles<kx.value, kz.value, f8.value, 64, 128, 2, 2, 3, 0>(g, c, 2, stream);
      default: return launch_tiles<kx.value, kz.value, f8.value, 64, 64, 2, 2, 4, 0>(g, c, 2, stream);
    }
  };
  using std::integral_constant;
  constexpr integral_constant<int, SRQ_E4M3> e4;
  constexpr integral_constant<int, SRQ_E5M2> e5;
  const auto pipe = [&](auto kx, auto kz) { return p.f8 ? as(kx, kz, std::true_type{}) : as(kx, kz, std::false_type{}); };
  if (p.kindX == SRQ_E5M2) return p.kindZ == SRQ_E5M2 ? pipe(e5, e5) : pipe(e5, e4);
  return p.kindZ == SRQ_E5M2 ? pipe(e4, e5) : pipe(e4, e4);
}

hipError_t launch_gated_forward(const GatedForward& a, hipStream_t stream) {
  TileParams g = {};
  g.X = a.X; g.Z = a.W;
  g.P = a.M; g.Q = 2 * a.F; g.F = a.F; g.R = a.K;
  g.partial = a.partial;
  g.out = a.h; g.h_scales = a.h_scales; g.h_codes = a.h_scales != nullptr;
  g.gu = a.gu; g.gu_scales = a.gu_scales;
  g.rnd_h = a.rnd_h; g.rnd_gu = a.rnd_gu;
  const BlockCut c = a.M > FEW ? gated_cut(a.M, a.F, a.K, a.f8) : BlockCut{};
  const auto as = [&](auto f8, auto act) -> hipError_t {
    constexpr int E = SRQ_E4M3;
    if (a.M <= FEW) {
      if (hipError_t e = launch_few<E, E, true>(g, stream); e != hipSuccess) return e;
      g.tiles_p = 1;
      g.tiles_q = a.F / SBLOCK;
      g.chunk = (g.tiles_q + 7) / 8;
      g.nsplit = 1;
      block_slices_kernel<FEW, 256, act.value><<<8 * g.chunk, 256, 0, stream>>>(g);
      return hipGetLastError();
    }
    switch (c.form) {
      case 0: return launch_tiles<E, E, f8.value, 256, 256, 2, 4, 2, act.value>(g, c, 1, stream);
      case 1: return launch_tiles<E, E, f8.value, 128, 256, 2, 4, 2, act.value>(g, c, 1, stream);
      case 2: return launch_tiles<E, E, false, 64, 256, 2, 4, 3, act.value>(g, c, 1, stream);
      default: return launch_tiles<E, E, false, 32, 256, 2, 4, 3, act.value>(g, c, 1, stream);
    }
  };
  using std::integral_constant;
  const auto act = [&](auto f8) { return a.act == SRQ_ACT_SILU ? as(f8, integral_constant<int, 1>{}) : as(f8, integral_constant<int, 2>{}); };
  return a.f8 ? act(std::true_type{}) : act(std::false_type{});
}

}  // namespace srq
