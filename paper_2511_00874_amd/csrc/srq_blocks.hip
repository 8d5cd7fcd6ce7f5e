// Block-scaled codes of a tensor (an operand, or an activation checkpoint): along its rows, turned, or both from one pass;
// a checkpoint turned for the product that contracts over its rows; codes back to values.
// Memory-bound: a value is read once, and one byte a layout written.
#include "srq_blocks.hpp"

namespace srq {
namespace {

// Along the rows alone: sixteen neighbouring lanes hold one block, eight values each.  16384 x 2048 bfloat16 to E5M2: 20.3 us (5.0 TB/s), rounded
// stochastically 25.3.
template <int SRC, int KIND, bool SR>
__global__ __launch_bounds__(256) void block_rows_kernel(BlockQuantize q) {
  const uint32_t cols = q.out.cols, blocks = (cols + SBLOCK - 1) / SBLOCK;
  const size_t total = (size_t)q.out.rows * blocks;
  const uint64_t counter = SR ? first_block(q.rnd.counter_offset, q.rnd.counter_dev) : 0;
  const uint32_t cg = threadIdx.x & 15u;
  for (size_t n = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4); n < total; n += (size_t)gridDim.x * 16) {
    const size_t row = n / blocks;
    const uint32_t b = (uint32_t)(n - row * blocks), col = b * SBLOCK + 8 * cg;
    const bool live = col < cols;
    Octet<SRC> o;
    o.zero();
    if (live) o.load(q.x, row * q.x_pitch + col);
    float v[8];
    o.get(v);
    const Extent e = extent_of(v);
    const uint32_t byte = scale_byte<KIND>(max16(most_finite(v, e)));
    uint32_t r[4];
    thresholds<SR>(q.rnd, counter + (row * cols + col) / 8, r);
    const u32x2 c = codes_of_octet<KIND, SR>(v, e, byte, r);
    if (live) __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(q.out.codes + row * q.out.pitch + col));
    if (cg == 0) q.out.scales[row * q.out.spitch + b] = (uint8_t)byte;
  }
}

// Turned, or both: tiles of 128 x 128, a block in either direction, so that one read serves both layouts and either scale is known in the tile.
// 16384 x 2048 bfloat16 to E5M2 in both layouts 30 us (4.5 TB/s), stochastically 32; a checkpoint of 12289 x 5632 turned 38.4 (3.6 TB/s): there
// vector work fills 71 % of the issue slots (finding the columns' largest and shifting on the codes themselves, decoding only groups with zeros or
// subnormal numbers: 43, nearly every wave has such a group).
template <int SRC, int KIND, bool SR, bool ROWS>
__global__ __launch_bounds__(TILE_THREADS) void block_tiles_kernel(BlockQuantize q, uint32_t tiles_c, uint32_t first) {
  __shared__ TileLds lds;
  tile_begin(lds);
  const uint32_t tile = first + blockIdx.x, row0 = tile / tiles_c * SBLOCK, col0 = tile % tiles_c * SBLOCK;
  const uint32_t cg = threadIdx.x & 15u, rg = threadIdx.x >> 4, col = col0 + 8 * cg;
  constexpr size_t ES = SRC == BSRC_F32 ? 4 : SRC == BSRC_BF16 ? 2 : 1;
  const auto buffer = rows_buffer(q.x, q.x_pitch * ES, row0, q.out.rows, SBLOCK);
  Octet<SRC> o[TILE_ROWS];
  float scale[TILE_ROWS];
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i)
    o[i].template fetch<STREAMED>(buffer, col < q.out.cols ? (TILE_ROWS * rg + i) * (uint32_t)q.x_pitch + col : OUT / ES);
  if constexpr (SRC >= BSRC_E4M3) {
    const auto scales = rows_buffer(q.x_scales, q.x_spitch, row0, q.out.rows, SBLOCK);
#pragma unroll
    for (int i = 0; i < TILE_ROWS; ++i)
      scale[i] = scale_value(__builtin_amdgcn_raw_buffer_load_b8(scales, (TILE_ROWS * rg + i) * (uint32_t)q.x_spitch + col0 / SBLOCK, 0, KEPT));
  }
  float v[TILE_ROWS][8];
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i) {
    if constexpr (SRC >= BSRC_E4M3) o[i].get(v[i], scale[i]);
    else o[i].get(v[i]);
  }
  tile_to_codes<KIND, SR, ROWS>(v, q.out, lds, row0, col0, (size_t)row0 * q.out.cols + col0, q.out.cols, q.rnd,
                                SR ? first_block(q.rnd.counter_offset, q.rnd.counter_dev) : 0);
}

template <int SRC, int KIND, bool SR>
void launch_quantize_as(const BlockQuantize& q, hipStream_t stream) {
  const size_t blocks = (q.out.cols + SBLOCK - 1) / SBLOCK;
  const size_t tiles = ((size_t)q.out.rows + SBLOCK - 1) / SBLOCK * blocks;
  if (!q.out.codes_t) {
    if constexpr (SRC < BSRC_E4M3) {  // (a checkpoint is only turned)
      const size_t wgs = std::min<size_t>(((size_t)q.out.rows * blocks + 15) / 16, 1u << 20);
      block_rows_kernel<SRC, KIND, SR><<<(unsigned)wgs, 256, 0, stream>>>(q);
    }
    return;
  }
  const auto run = [&](auto kernel) {
    in_launches(tiles, [&](uint32_t first, unsigned wgs) { kernel<<<wgs, TILE_THREADS, 0, stream>>>(q, (uint32_t)blocks, first); });
  };
  if (!q.out.codes) run(block_tiles_kernel<SRC, KIND, SR, false>);
  else if constexpr (SRC < BSRC_E4M3) run(block_tiles_kernel<SRC, KIND, SR, true>);
}

template <int KIND, bool SR>
void launch_quantize_kind(const BlockQuantize& q, hipStream_t stream) {
  switch (q.src) {
    case BSRC_F32: launch_quantize_as<BSRC_F32, KIND, SR>(q, stream); break;
    case BSRC_BF16: launch_quantize_as<BSRC_BF16, KIND, SR>(q, stream); break;
    case BSRC_E4M3: launch_quantize_as<BSRC_E4M3, KIND, SR>(q, stream); break;
    default: launch_quantize_as<BSRC_E5M2, KIND, SR>(q, stream); break;
  }
}

// Codes times scale: exact in both types where the result is a normal number of the type.  16384 x 2048 to bfloat16 18.9 us (5.4 TB/s), to binary32 33
// (5.1).
template <int KIND, int DTYPE>
__global__ __launch_bounds__(256) void block_restore_kernel(void* x, const uint8_t* codes, const uint8_t* scales, size_t rows,
                                                            uint32_t cols, size_t pitch, size_t spitch) {
  const uint32_t groups = cols / 8;
  for (size_t n = (size_t)blockIdx.x * 256 + threadIdx.x; n < rows * groups; n += (size_t)gridDim.x * 256) {
    const size_t row = n / groups;
    const uint32_t col = (uint32_t)(n - row * groups) * 8;
    CodeOctet<KIND> o;
    o.load(codes, row * pitch + col);
    float v[8];
    o.get(v, scale_value(scales[row * spitch + col / SBLOCK]));
    if constexpr (DTYPE == SRQ_F32) {
      f32x4* const at = reinterpret_cast<f32x4*>(static_cast<float*>(x) + row * cols + col);
      __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, at);
      __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, at + 1);
    } else {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
      __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(x) + row * cols + col));
    }
  }
}

}  // namespace

hipError_t launch_block_quantize(const BlockQuantize& q, hipStream_t stream) {
  if (q.kind == SRQ_E5M2) q.rnd.sr ? launch_quantize_kind<SRQ_E5M2, true>(q, stream) : launch_quantize_kind<SRQ_E5M2, false>(q, stream);
  else q.rnd.sr ? launch_quantize_kind<SRQ_E4M3, true>(q, stream) : launch_quantize_kind<SRQ_E4M3, false>(q, stream);
  return hipGetLastError();
}

hipError_t launch_block_restore(void* x, int dtype, const uint8_t* codes, size_t pitch, const uint8_t* scales, size_t rows, size_t cols,
                                int kind, hipStream_t stream) {
  const size_t wgs = std::min<size_t>((rows * (cols / 8) + 255) / 256, 1u << 20);
  const size_t spitch = scale_pitch(cols);
  const auto go = [&](auto kernel) { kernel<<<(unsigned)wgs, 256, 0, stream>>>(x, codes, scales, rows, (uint32_t)cols, pitch, spitch); };
  if (kind == SRQ_E5M2) {
    if (dtype == SRQ_F32) go(block_restore_kernel<SRQ_E5M2, SRQ_F32>);
    else go(block_restore_kernel<SRQ_E5M2, SRQ_BF16>);
  } else {
    if (dtype == SRQ_F32) go(block_restore_kernel<SRQ_E4M3, SRQ_F32>);
    else go(block_restore_kernel<SRQ_E4M3, SRQ_BF16>);
  }
  return hipGetLastError();
}

}  // namespace srq
