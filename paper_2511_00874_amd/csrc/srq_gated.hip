// Backward pass of the gated block's activation and product, from the 8-bit checkpoint of G and U:
//   H = act(G) U:   dU = dH act(G),   dG = dH U act'(G)
// as codes along the rows and turned, G's gradient beside U's: operands of the input and weight gradients.  Memory-bound: dH and the
// checkpoint are read once, four bytes written for each of their values; the gradients themselves are never in memory.
#include "srq_blocks.hpp"

namespace srq {
namespace {

// A workgroup makes one of the two gradients of a tile; the one that makes the other is eight ids on, on the same XCD, and finds dH
// and the checkpoint in its L2.  With both in one workgroup a thread holds 204 to 220 registers, two waves a SIMD; one after the other there, with
// the next tile's loads ahead, it needs more than the 128 that four waves have, and spills (485 us).
// 16384 x 5632 SiLU, bfloat16 to E5M2: 248 us, 3.0 TB/s of what has to be moved; GELU 274.  Vector work (75 instructions for a pair of gradients, of
// them decoding and activation twice) fills 79 % of the issue slots and, rounding to nearest, 67 %, at 245 us: a sixth fewer instructions hardly
// shorten it, so that what bounds it is as much the loads' latency between a workgroup's barriers.
template <int DTYPE, int ACT, int KIND, bool SR>
__global__ __launch_bounds__(TILE_THREADS) void gated_backward_kernel(GatedBackward g, uint32_t tiles_f, uint32_t tiles) {
  __shared__ TileLds lds;
  const uint32_t tile = blockIdx.x >> 4 << 3 | (blockIdx.x & 7u);
  const bool of_u = blockIdx.x & 8u;
  if (tile >= tiles) return;
  tile_begin(lds);
  const uint32_t row0 = tile / tiles_f * SBLOCK, f0 = tile % tiles_f * SBLOCK;
  const uint32_t cg = threadIdx.x & 15u, rg = threadIdx.x >> 4, f = f0 + 8 * cg;
  const uint32_t nb = g.F / SBLOCK, ld = 2 * g.F, spitch = (uint32_t)g.out.spitch;  // (the checkpoint has the gradients' shape)
  const auto dh_rows = rows_buffer(g.dh, (size_t)g.F * (DTYPE == SRQ_F32 ? 4 : 2), row0, g.out.rows, SBLOCK);
  const auto gu_rows = rows_buffer(g.gu, ld, row0, g.out.rows, SBLOCK);
  const auto scale_rows = rows_buffer(g.gu_scales, spitch, row0, g.out.rows, SBLOCK);
  Octet<DTYPE> dh[TILE_ROWS];
  CodeOctet<SRQ_E4M3> gc[TILE_ROWS], uc[TILE_ROWS];
  float gs[TILE_ROWS], us[TILE_ROWS];
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i) {
    const uint32_t row = TILE_ROWS * rg + i;
    dh[i].template fetch<KEPT>(dh_rows, row * g.F + f);
    gc[i].template fetch<KEPT>(gu_rows, row * ld + f);
    gs[i] = scale_value(__builtin_amdgcn_raw_buffer_load_b8(scale_rows, row * spitch + f0 / SBLOCK, 0, KEPT));
    if (!of_u) {
      uc[i].template fetch<KEPT>(gu_rows, row * ld + g.F + f);
      us[i] = scale_value(__builtin_amdgcn_raw_buffer_load_b8(scale_rows, row * spitch + nb + f0 / SBLOCK, 0, KEPT));
    }
  }
  float v[TILE_ROWS][8];
  const auto each = [&](auto gradient) {
#pragma unroll
    for (int i = 0; i < TILE_ROWS; ++i) {
      float a[8], d[8];
      gc[i].get(a, gs[i]);
      dh[i].get(d);
      gradient(a, d, i);
    }
  };
  if (of_u) {
    each([&](const float (&a)[8], const float (&d)[8], int i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float act, slope;
        activate<ACT>(a[j], act, slope);
        v[i][j] = d[j] * act;
      }
    });
  } else {
    each([&](const float (&a)[8], const float (&d)[8], int i) {
      float b[8];
      uc[i].get(b, us[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float act, slope;
        activate<ACT>(a[j], act, slope);
        v[i][j] = d[j] * b[j] * slope;
      }
    });
  }
  const uint32_t col0 = f0 + (of_u ? g.F : 0u);
  tile_to_codes<KIND, SR, true>(v, g.out, lds, row0, col0, (size_t)row0 * ld + col0, ld, g.rnd,
                                SR ? first_block(g.rnd.counter_offset, g.rnd.counter_dev) : 0);
}

template <int DTYPE, int ACT>
void go(const GatedBackward& g, hipStream_t stream) {
  const uint32_t tiles_f = g.F / SBLOCK, tiles = (g.out.rows + SBLOCK - 1) / SBLOCK * tiles_f;
  const auto run = [&](auto kernel) { kernel<<<(tiles + 7) / 8 * 16, TILE_THREADS, 0, stream>>>(g, tiles_f, tiles); };
  if (g.kind == SRQ_E5M2) run(g.rnd.sr ? gated_backward_kernel<DTYPE, ACT, SRQ_E5M2, true> : gated_backward_kernel<DTYPE, ACT, SRQ_E5M2, false>);
  else run(g.rnd.sr ? gated_backward_kernel<DTYPE, ACT, SRQ_E4M3, true> : gated_backward_kernel<DTYPE, ACT, SRQ_E4M3, false>);
}

}  // namespace

hipError_t launch_gated_backward(const GatedBackward& g, hipStream_t stream) {
  if (g.dtype == SRQ_F32) {
    if (g.act == SRQ_ACT_SILU) go<SRQ_F32, SRQ_ACT_SILU>(g, stream);
    else go<SRQ_F32, SRQ_ACT_GELU>(g, stream);
  } else {
    if (g.act == SRQ_ACT_SILU) go<SRQ_BF16, SRQ_ACT_SILU>(g, stream);
    else go<SRQ_BF16, SRQ_ACT_GELU>(g, stream);
  }
  return hipGetLastError();
}

}  // namespace srq
