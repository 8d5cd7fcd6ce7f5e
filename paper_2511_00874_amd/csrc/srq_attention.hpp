// What the attention kernels share: which rows belong together, tiles of rows in LDS, and the products' operands.  gfx950 only.
//
// All products are bf16 matrix instructions of 32 x 32 x 16 with binary32 sums.  Of C = A B a lane holds column lane % 32 and sixteen rows, r-th
// row 8 (r / 4) + 4 (lane / 32) + r % 4; of A and B it holds one row / column, lane % 32, and eight places of the contraction.  Every kernel
// computes the scores so that what a softmax or its gradient belongs to (a query in the forward pass and for dq, a key for dk and dv) is a
// column: its statistics are one register a lane.  The scores' registers 8 s .. 8 s + 7, rounded to bfloat16, are then the B operand of the second
// product as they are, if A holds in place 4 a + b of lane group g the tile's row 16 s + 8 a + 4 g + b: any order of a contraction will do.
// Tiles lie in LDS as they lie in memory, row by row; operands that run along the rows are read 16 bytes a lane, those that run across them by
// the transposing read (a group of sixteen lanes reads four rows of sixteen values, and lane i gets column i).
#pragma once
#include "srq_decoder.hpp"
#include "srq_mma.hpp"

namespace srq {
namespace attn {

using mma::lds_void;
using mma::v16f;
using mma::v4i;
using mma::v8bf;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr uint32_t OOB = 0x80000000u;  // beyond any tile: loads as zero
#define SRQ_INF __builtin_inff()

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---- which rows -----------------------------------------------------------------------------------------------------------------
struct Span {
  uint32_t first, rows;
};
__device__ __forceinline__ uint32_t within(int v, uint32_t rows) { return v < 0 ? 0u : min((uint32_t)v, rows); }
// Rows of sequence b.
__device__ __forceinline__ Span span_of(const int32_t* offsets, uint32_t rows, uint32_t sequences, uint32_t b) {
  if (!offsets) {
    const uint32_t per = rows / sequences;
    return {b * per, per};
  }
  const uint32_t from = uniform(within(offsets[b], rows)), to = uniform(within(offsets[b + 1], rows));
  return {from, to > from ? to - from : 0u};
}
__device__ __forceinline__ Span keys_of(const AttentionShape& s, uint32_t b) {
  Span k = span_of(s.offsets_k, s.rows_k, s.sequences, b);
  if (s.lengths_k) k.rows = min(k.rows, uniform(within(s.lengths_k[b], s.rows_k)));
  return k;
}
// Sequence b's tiles of bm rows have the slots floor(first row / BM) + b and on: these begins ascend by at least as many as the sequence has tiles,
// so a slot is found by search, without the lengths on the host; a few slots have no tile.
inline __host__ __device__ uint32_t slots_of(const int32_t* offsets, uint32_t rows, uint32_t sequences, uint32_t bm) {
  return offsets ? rows / bm + sequences : sequences * ((rows / sequences + bm - 1) / bm);
}
struct Tile {
  uint32_t sequence, first, rows, row;  // the sequence, its rows, the tile's first of them
  bool valid;
};
__device__ __forceinline__ Tile tile_of(const int32_t* offsets, uint32_t rows, uint32_t sequences, uint32_t bm, uint32_t slot) {
  Tile t;
  uint32_t index;
  if (!offsets) {
    t.sequence = slot % sequences;  // (equal ones: all their first tiles, all second ones ..)
    index = slot / sequences;
  } else {
    // how many sequences begin at or before the slot: 64 places of the list at a time
    const uint32_t lane = threadIdx.x & 63u;
    const auto at = [&](uint32_t b) { return within(offsets[b], rows) / bm + b <= slot; };
    uint32_t lo = 0, hi = sequences;
    while (hi - lo > 64) {
      const uint32_t step = (hi - lo + 63) / 64, b = lo + (lane + 1) * step - 1;
      const uint32_t n = (uint32_t)__popcll(__ballot(b < hi && at(min(b, hi - 1))));
      hi = min(hi, lo + (n + 1) * step - 1);
      lo = min(hi, lo + n * step);
    }
    const uint32_t n = lo + (uint32_t)__popcll(__ballot(lo + lane < hi && at(min(lo + lane, sequences - 1))));
    t.sequence = uniform(n ? n - 1 : 0u);
    index = n ? slot - t.sequence : ~0u;
  }
  const Span s = span_of(offsets, rows, sequences, t.sequence);
  t.first = s.first;
  t.rows = s.rows;
  if (offsets) index = index == ~0u || index < s.first / bm ? ~0u : uniform(index - s.first / bm);
  t.valid = index < (s.rows + bm - 1) / bm;
  t.row = t.valid ? index * bm : 0u;
  return t;
}

// Workgroup of a launch to head and slot.  Workgroups are dealt to the eight XCDs in turn, and heads share nothing but, in groups, their keys: so each
// XCD, or as many as make whole heads, gets heads of its own, neighbours.  Of those come all in one slot, then all in the next, so that what is heavy is begun
// first (with one head after the other, 8 x 1024 rows of 12 heads gave a CU three heavy tiles or three light ones).
struct Place {
  uint32_t head, slot;
  bool valid;
};
inline __host__ __device__ uint32_t groups_of(uint32_t heads) { return heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1; }
__device__ __forceinline__ Place place_of(uint32_t heads, uint32_t slots) {
  const uint32_t groups = groups_of(heads), each = heads / groups, xcd = blockIdx.x & 7u, i = (blockIdx.x >> 3) * (8 / groups) + xcd / groups;
  return {xcd % groups * each + i % each, i / each, i < slots * each};
}
inline uint32_t workgroups_of(uint32_t heads, uint32_t slots) {
  const uint32_t groups = groups_of(heads), r = 8 / groups;
  return (slots * (heads / groups) + r - 1) / r * 8;
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------------------------------
// Rows of DP values, chunk c (16 bytes) of row r at chunk c ^ swizzle(r).  A 16-byte read is served sixteen lanes at a time, whose rows are sixteen
// different ones mod 16: all 64 banks.  A transposing read is served in halves of the wave, four neighbouring rows of 64 bytes each: rows differ in the
// chunk's upper bits, so these too are all 64 banks.
template <int DP>
struct Rows {
  static constexpr uint32_t PITCH = DP * 2, CHUNKS = DP / 8, PER_LOAD = 1024 / PITCH;  // bytes, chunks of a row; rows of a wave's load of 1 KiB
  static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
    if constexpr (DP == 128) return ((r & 3u) << 2) | ((r >> 2) & 3u);
    else return (((r >> 1) & 1u) << 2) | ((r >> 2) & 3u);
  }
};

// Waits as builtins, which the compiler counts by, between barriers to its moving of memory accesses: it does not see the loads to LDS.  (Registers loaded in
// front of a loop have to be waited for there, by one of these with 0: else their first use waits, in every turn, for all that is under way.)
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
  asm volatile("" : : : "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (0x7 << 4) | (3 << 14));
  asm volatile("" : : : "memory");
}
// All that this wave loads and reads is there, then all waves'.
__device__ __forceinline__ void landed_everywhere() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0x7 << 4);
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}
__device__ __forceinline__ void lds_dma16(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_void*)p; }

// The rows of one head of a sequence, to be fetched to LDS in tiles; rows behind the last, and values behind the head's, are zeros.
struct RowSource {
  const uint8_t* p;     // first row
  uint32_t pitch, rows, tail;  // bytes from row to row; rows; bytes of the last one
};
__device__ __forceinline__ RowSource row_source(const Heads& h, uint32_t first, uint32_t rows, uint32_t head, uint32_t dim) {
  return {reinterpret_cast<const uint8_t*>(h.p + (size_t)first * h.row + (size_t)head * h.head), (uint32_t)h.row * 2, rows, dim * 2};
}
// Rows [row, row + N) to LDS address `to`, by WAVES waves of which this is number `wave`.  What a lane adds to a load's first row, its row and chunk, is
// kept: the same for all of a wave's loads, but that with fewer than four waves their rows' swizzles differ.
template <int DP, uint32_t N, uint32_t WAVES>
struct Fetch {
  using R = Rows<DP>;
  static constexpr uint32_t FORMS = WAVES % 4 == 0 ? 1 : 4;
  uint32_t lane_at[FORMS];
  __device__ __forceinline__ Fetch(const RowSource& s, uint32_t wave) {
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (uint32_t i = 0; i < FORMS; ++i) {
      const uint32_t chunk = (lane % R::CHUNKS) ^ R::swizzle((i * WAVES + wave) * R::PER_LOAD + lane / R::CHUNKS);
      lane_at[i] = (lane / R::CHUNKS * s.pitch + chunk * 16) | (chunk * 16 < s.tail ? 0u : OOB);
    }
  }
  __device__ __forceinline__ void operator()(const RowSource& s, uint32_t row, uint32_t to, uint32_t wave) const {
    const uint32_t left = row < s.rows ? min(s.rows - row, N) : 0u, bytes = left ? (left - 1) * s.pitch + s.tail : 0u;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(s.p) + (size_t)row * s.pitch, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (uint32_t i = 0; i < N / R::PER_LOAD / WAVES; ++i) {
      const uint32_t n = i * WAVES + wave;
      lds_dma16(rsrc, to + n * 1024, lane_at[i % FORMS] + n * R::PER_LOAD * s.pitch);
    }
  }
};

// Where a lane reads its operands in a tile: along the rows (A or B of row lane % 32, step s of 16 values), or across them.
template <int DP>
struct Reader {
  uint32_t along0, across0;
  __device__ __forceinline__ Reader() {
    const uint32_t lane = threadIdx.x & 63u, r = lane & 31u, g = lane >> 5, r4 = (lane >> 2) & 3u;
    along0 = r * Rows<DP>::PITCH + ((g ^ Rows<DP>::swizzle(r)) << 4);
    // row 4 g + r4, value 16 ((lane / 16) % 2) + 4 (lane % 4)
    across0 = (4 * g + r4) * Rows<DP>::PITCH + (((2 * ((lane >> 4) & 1u) + ((lane & 3u) >> 1)) ^ Rows<DP>::swizzle(4 * g + r4)) << 4) + (lane & 1u) * 8;
  }
  // rows of block `block` of 32, values 16 s + 8 (lane / 32) ..
  __device__ __forceinline__ v8bf along(const uint8_t* tile, uint32_t block, uint32_t s) const {
    return *reinterpret_cast<const v8bf*>(tile + ((along0 ^ (s << 5)) + block * 32 * Rows<DP>::PITCH));
  }
  // values 32 d + lane % 32, rows 16 s + 8 a + 4 (lane / 32) + b in place 4 a + b
  __device__ __forceinline__ v8bf across(const uint8_t* tile, uint32_t s, uint32_t d) const {
    // (eight rows on, the swizzle's third bit, of the row's, changes: chunk ^ 2)
    const uint32_t at = (across0 ^ (d << 6)) + s * 16 * Rows<DP>::PITCH;
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + at));
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + ((at ^ 32u) + 8 * Rows<DP>::PITCH)));
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ v16f mfma(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b}); }
// Registers 8 s .. 8 s + 7 as an operand.
__device__ __forceinline__ v8bf operand_of(const v16f& p, int s) {
  const v4u w = {pack(p[8 * s], p[8 * s + 1]), pack(p[8 * s + 2], p[8 * s + 3]), pack(p[8 * s + 4], p[8 * s + 5]), pack(p[8 * s + 6], p[8 * s + 7])};
  return __builtin_bit_cast(v8bf, w);
}
// The sum of an operand's eight values and of `sum`, in binary32.
__device__ __forceinline__ float sum_of(const v8bf& w, float sum) {
  const v4u x = __builtin_bit_cast(v4u, w);
  const v2bf ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, x[i]), ones, sum, false);
  return sum;
}
__device__ __forceinline__ v16f zeros() {
  v16f z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}
// Row of a tile of 32 that register r holds, but for 4 (lane / 32).
__device__ __forceinline__ constexpr int row_of(int r) { return 8 * (r / 4) + r % 4; }

// lane ^ 32's value
__device__ __forceinline__ float max_of_halves(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Operand from memory: a row of a head, in steps of 16 values; zeros behind the head's values and for rows that are not there.
template <int DP>
__device__ __forceinline__ void load_operand(v8bf (&x)[DP / 16], const Heads& h, size_t row, uint32_t head, uint32_t dim, bool there) {
  const uint32_t g = (threadIdx.x >> 5) & 1u;
  const uint16_t* const p = h.p + row * h.row + (size_t)head * h.head;
#pragma unroll
  for (uint32_t s = 0; s < DP / 16; ++s) {
    v4u v = {0, 0, 0, 0};
    const uint32_t d = 16 * s + 8 * g;
    if (there && d < dim) v = *reinterpret_cast<const v4u*>(p + d);
    x[s] = __builtin_bit_cast(v8bf, v);
  }
}
// A column of the result (DP values in the sums' order, times `factor`) to its row of a head, as bfloat16: the halves of the wave trade words, so that each
// stores eight neighbouring values.
template <int DP>
__device__ __forceinline__ void store_column(const v16f (&acc)[DP / 32], float factor, const Heads& h, size_t row, uint32_t head, uint32_t dim, bool there) {
  const uint32_t g = (threadIdx.x >> 5) & 1u;
  uint16_t* const p = h.p + row * h.row + (size_t)head * h.head;
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int a = 0; a < 4; a += 2) {
      const v16f& x = acc[b];
      const uint32_t w0 = pack(x[4 * a] * factor, x[4 * a + 1] * factor), w1 = pack(x[4 * a + 2] * factor, x[4 * a + 3] * factor);
      const uint32_t w2 = pack(x[4 * a + 4] * factor, x[4 * a + 5] * factor), w3 = pack(x[4 * a + 6] * factor, x[4 * a + 7] * factor);
      const auto lo = __builtin_amdgcn_permlane32_swap(w0, w2, false, false), hi = __builtin_amdgcn_permlane32_swap(w1, w3, false, false);
      const uint32_t d = 32 * b + 8 * a + 8 * g;
      if (there && d < dim) *reinterpret_cast<v4u*>(p + d) = v4u{lo[0], hi[0], lo[1], hi[1]};
    }
}

}  // namespace attn
}  // namespace srq
