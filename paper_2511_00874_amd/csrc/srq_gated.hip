// Backward pass of the gated block's activation and product, from the 8-bit checkpoint of G and U:
//   H = act(G) U:   dU = dH act(G),   dG = dH U act'(G)
// as codes along the rows and turned, G's gradient beside U's: operands of the input and weight gradients.  Memory-bound: dH and the
// checkpoint are read once, four bytes written for each of their values; the gradients themselves are never in memory.
#include "srq_blocks.hpp"

namespace srq {
namespace {

template <int DTYPE, int ACT, int KIND>
__global__ __launch_bounds__(256) void gated_backward_kernel(GatedBackward g, uint32_t tiles_f) {
  __shared__ TileLds lds;
  const uint32_t row0 = blockIdx.x / tiles_f * SBLOCK, f0 = blockIdx.x % tiles_f * SBLOCK;
  const uint32_t cg = threadIdx.x & 15u, rg = threadIdx.x >> 4, f = f0 + 8 * cg;
  const uint32_t nb = g.F / SBLOCK;
  const size_t gpitch = 2 * (size_t)g.F, spitch = g.out.spitch;  // (the checkpoint has the gradients' shape)
  Octet<DTYPE> dh[8];
  CodeOctet<SRQ_E4M3> gc[8], uc[8];
  float gs[8], us[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t row = row0 + 8 * rg + i;
    dh[i].zero();
    gc[i].zero();
    uc[i].zero();
    gs[i] = us[i] = 0.0f;
    if (row < g.out.rows) {
      dh[i].load(g.dh, (size_t)row * g.F + f);
      gc[i].load(g.gu, row * gpitch + f);
      uc[i].load(g.gu, row * gpitch + g.F + f);
      gs[i] = scale_value(g.gu_scales[row * spitch + f0 / SBLOCK]);
      us[i] = scale_value(g.gu_scales[row * spitch + nb + f0 / SBLOCK]);
    }
  }
  const uint64_t counter = first_block(g.rnd.counter_offset, g.rnd.counter_dev);
  float v[8][8];
#pragma unroll 1
  for (uint32_t half = 0; half < 2; ++half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a[8], b[8], d[8];
      gc[i].get(a, gs[i]);
      uc[i].get(b, us[i]);
      dh[i].get(d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float act, slope;
        activate<ACT>(a[j], act, slope);
        v[i][j] = half ? d[j] * act : d[j] * b[j] * slope;
      }
    }
    const uint32_t col0 = f0 + half * g.F;
    tile_to_codes<KIND, true, true>(v, g.out, lds, row0, col0, (size_t)row0 * gpitch + col0, gpitch, g.rnd, counter);
    __syncthreads();
  }
}

template <int DTYPE, int ACT>
void go(const GatedBackward& g, hipStream_t stream) {
  const uint32_t tiles_f = g.F / SBLOCK;
  const unsigned tiles = (unsigned)(((size_t)g.out.rows + SBLOCK - 1) / SBLOCK * tiles_f);
  if (g.kind == SRQ_E5M2) gated_backward_kernel<DTYPE, ACT, SRQ_E5M2><<<tiles, 256, 0, stream>>>(g, tiles_f);
  else gated_backward_kernel<DTYPE, ACT, SRQ_E4M3><<<tiles, 256, 0, stream>>>(g, tiles_f);
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
