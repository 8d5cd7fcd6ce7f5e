// What the attention kernels share: which rows belong together, tiles of rows in LDS, and the products' operands.  gfx950 only.
//
// All products are bf16 matrix instructions of 16 x 16 x 32 with binary32 sums (the chip clocks higher under them than under the 32 x 32 ones).  Of C = A B a
// lane holds column lane % 16 and the four rows 4 (lane / 16) + r; of A and B one row / column, lane % 16, and eight places of the contraction.  Every
// kernel computes the scores so that what a softmax or its gradient belongs to (a query in the forward pass and for dq, a key for dk and dv) is a
// column: its statistics are one register a lane.  Two tiles of scores, rows 0 .. 15 and 16 .. 31, rounded to bfloat16, are then the B operand of the second
// product as they are, if A holds in place 4 a + b of lane group g the tile's row 16 a + 4 g + b: any order of a contraction will do.  A wave has 32
// columns, two of everything: an operand read from LDS serves two instructions.
// Tiles lie in LDS as they lie in memory, row by row; operands that run along the rows are read 16 bytes a lane, those that run across them by
// the transposing read (a group of sixteen lanes reads four rows of sixteen values, and lane i gets column i).
#pragma once
#include <algorithm>

#include "srq_decoder.hpp"
#include "srq_mma.hpp"

namespace srq {
namespace attn {

using mma::lds_void;
using mma::v4f;
using mma::v8bf;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr uint32_t OOB = 0x80000000u;  // beyond any tile: loads as zero
#define SRQ_INF __builtin_inff()

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// What is reckoned from this is reckoned where it is wanted, not kept in registers over a loop.
__device__ __forceinline__ uint32_t worked_out(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

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

// The sum, and the largest, of the wave's values, in all lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, F&& f) {
  v = f(v, moved<0xB1>(v));    // lane ^ 1
  v = f(v, moved<0x4E>(v));    // lane ^ 2
  v = f(v, moved<0x141>(v));   // 7 - lane of 8
  v = f(v, moved<0x140>(v));   // 15 - lane of 16
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return uniform(f(b[0], b[1]));
}
// The tiles of all sequences with the last ones first: all tiles of the highest index, then all of the one below, the place-th of them.  What a tile has to do
// goes by its index (of keys: by the tiles behind it, from_end), so a launch begins with the heaviest, whichever sequences they belong to, and ends
// with light ones.  Up to 256 sequences, four a lane; with more the slots are gone through from the last one, which mixes as well.
constexpr uint32_t RANKED = 256;
__device__ __forceinline__ Tile ranked_tile(const int32_t* offsets, uint32_t rows, uint32_t sequences, uint32_t bm, uint32_t slots, uint32_t place, bool from_end) {
  if (!offsets || sequences == 1 || sequences > RANKED) {
    Tile t = tile_of(offsets, rows, sequences, bm, from_end ? place : slots - 1 - place);
    return t;
  }
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t first[RANKED / 64], length[RANKED / 64], n[RANKED / 64], longest = 0;
#pragma unroll
  for (uint32_t c = 0; c < RANKED / 64; ++c) {
    first[c] = length[c] = n[c] = 0;
    if (64 * c < sequences && 64 * c + lane < sequences) {
      first[c] = within(offsets[64 * c + lane], rows);
      const uint32_t end = within(offsets[64 * c + lane + 1], rows);
      length[c] = end > first[c] ? end - first[c] : 0u;
      n[c] = (length[c] + bm - 1) / bm;
    }
    longest = max(longest, n[c]);
  }
  longest = over_wave(longest, [](uint32_t a, uint32_t b) { return max(a, b); });
  const auto tiles_from = [&](uint32_t i) {  // tiles of index i and above
    uint32_t sum = 0;
#pragma unroll
    for (uint32_t c = 0; c < RANKED / 64; ++c) sum += n[c] > i ? n[c] - i : 0u;
    return over_wave(sum, [](uint32_t a, uint32_t b) { return a + b; });
  };
  Tile t = {0, 0, 0, 0, false};
  if (place >= tiles_from(0)) return t;
  uint32_t lo = 0, hi = longest, above = 0;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2, count = tiles_from(mid);
    if (count > place) lo = mid;
    else hi = mid, above = count;
  }
  uint32_t left = place - above;  // of the tiles of index lo
#pragma unroll
  for (uint32_t c = 0; c < RANKED / 64; ++c) {
    const uint64_t have = __ballot(n[c] > lo);
    const uint32_t count = (uint32_t)__popcll(have);
    if (!t.valid && left < count) {
      const bool mine = n[c] > lo && __popcll(have & ((1ull << lane) - 1ull)) == left;
      const int at = __builtin_ctzll(__ballot(mine));
      t.sequence = 64 * c + at;
      t.first = (uint32_t)__builtin_amdgcn_readlane((int)first[c], at);
      t.rows = (uint32_t)__builtin_amdgcn_readlane((int)length[c], at);
      t.row = (from_end ? (t.rows + bm - 1) / bm - 1 - lo : lo) * bm;
      t.valid = true;
    }
    left -= t.valid ? 0u : count;
  }
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

// Slots that are cut into up to `pieces`: from slot to slot another comes first, as most have but the first one and neighbours fall to different XCDs.
struct PieceOf {
  uint32_t slot, piece;
  __device__ __forceinline__ PieceOf(uint32_t place, uint32_t pieces) : slot(place / pieces), piece((place % pieces + slot) % pieces) {}
};

// ---- the keys that rows see ---------------------------------------------------------------------------------------------------------
constexpr uint32_t KT = 64;  // keys of a tile
constexpr uint32_t MOST_PIECES = 8;
// A tile of queries with its keys, which may be cut into pieces, a workgroup each, whose sums a second launch puts together: a tile with many keys is a long
// way for one workgroup, where the others are done or not enough to fill the chip.
struct Cut {
  uint32_t pieces, quota;  // at most so many, of so many tiles at least
  // of `all` tiles: how many a piece takes, and the pieces
  __device__ __forceinline__ uint32_t each(uint32_t all) const {
    const uint32_t n = min(pieces, all / quota + 1);
    return max(1u, (all + n - 1) / n);
  }
  __device__ __forceinline__ uint32_t count(uint32_t all) const { return max(1u, (all + each(all) - 1) / each(all)); }
};
struct Queries {
  Tile t;
  Span keys;
  int lk, shift, causal;  // row i sees keys below i + shift, and lk
  uint32_t tiles;         // of keys
  __device__ __forceinline__ Queries(const AttentionShape& s, uint32_t bm, uint32_t slots, uint32_t place)
      : t(ranked_tile(s.offsets_q, s.rows_q, s.sequences, bm, slots, place, false)), causal(s.causal) {
    if (!t.valid) return;
    keys = keys_of(s, t.sequence);
    lk = (int)keys.rows;
    shift = lk - (int)t.rows + 1;
    const int end = limit_of((int)min(t.row + bm, t.rows) - 1);
    tiles = end > 0 ? ((uint32_t)end + KT - 1) / KT : 0u;
  }
  __device__ __forceinline__ int limit_of(int row) const { return causal ? min(lk, row + shift) : lk; }
};
// Of `slots` tiles of queries a head, where the chip holds `at_once` workgroups: what one has to do should not be far above its share of all the work, taking
// sequences of the mean length (those whose lengths are not known here may have up to four times their share of the rows).
inline Cut cut_of(const AttentionShape& s, uint32_t slots, size_t at_once) {
  const size_t mean = ((size_t)s.rows_k / s.sequences + KT - 1) / KT, most = s.offsets_k ? std::min<size_t>((s.rows_k + KT - 1) / KT, 4 * mean) : mean;
  const size_t share = (size_t)slots * s.heads_q * mean / (s.causal ? 2 : 1) / at_once, quota = std::max<size_t>(12, 2 * share);
  if (most < 2 * quota) return {1, 1};
  return {(uint32_t)std::min<size_t>(MOST_PIECES, (most + quota - 1) / quota), (uint32_t)quota};
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------------------------------
// Rows of DP values, chunk c (16 bytes) of row r at chunk c ^ swizzle(r).  A 16-byte read is served sixteen lanes at a time, lanes 0-3, 12-15 and 20-27 and so
// on: rows 0-3 and 12-15 in one chunk, 4-11 in its neighbour.  A transposing read is served in halves of the wave, eight rows of two chunks each.  With rows 4
// to 11 in chunks that are each other's neighbours, and rows that follow each other in different pairs of them, both are all 64 banks.
template <int DP>
struct Rows {
  static constexpr uint32_t PITCH = DP * 2, CHUNKS = DP / 8, PER_LOAD = 1024 / PITCH;  // bytes, chunks of a row; rows of a wave's load of 1 KiB
  static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
    const uint32_t t = (r >> 2) & 3u, f = (((t ^ (t >> 1)) & 1u) << 1) | (t >> 1);  // 0, 2, 3, 1
    if constexpr (DP == 128) return ((r & 3u) << 2) | f;
    else return (((r >> 1) & 1u) << 2) | f;
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
  __device__ __forceinline__ Fetch(const RowSource& s, uint32_t wave, uint32_t lane = threadIdx.x & 63u) {
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

// Where a lane reads its operands in a tile: along the rows (A of row lane % 16, step s of 32 values), or across them.
template <int DP>
struct Reader {
  uint32_t along0, across0;
  __device__ __forceinline__ explicit Reader(uint32_t lane = threadIdx.x & 63u) {
    const uint32_t r = lane & 15u, g = lane >> 4, r4 = 4 * g + ((lane >> 2) & 3u);
    along0 = r * Rows<DP>::PITCH + ((g ^ Rows<DP>::swizzle(r)) << 4);
    across0 = r4 * Rows<DP>::PITCH + ((((lane & 3u) >> 1) ^ Rows<DP>::swizzle(r4)) << 4) + (lane & 1u) * 8;
  }
  // rows of block `block` of 16, values 32 s + 8 (lane / 16) ..
  __device__ __forceinline__ v8bf along(const uint8_t* tile, uint32_t block, uint32_t s) const {
    return *reinterpret_cast<const v8bf*>(tile + ((along0 ^ (s << 6)) + block * 16 * Rows<DP>::PITCH));
  }
  // values 16 d + lane % 16, rows 32 s + 16 a + 4 (lane / 16) + b in place 4 a + b
  __device__ __forceinline__ v8bf across(const uint8_t* tile, uint32_t s, uint32_t d) const {
    const uint32_t at = (across0 ^ (d << 5)) + s * 32 * Rows<DP>::PITCH;
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + at));
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + (at + 16 * Rows<DP>::PITCH)));
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ v4f mfma(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b}); }

// 32 x 32 of a product: [rows 0-15, 16-31][columns 0-15, 16-31].  Register r of [i][j]: row 16 i + 4 (lane / 16) + r, column 16 j + lane % 16.
struct Block {
  v4f t[2][2];
};
// Rows of a tile's block of 32, times the columns' operands (B[column tile][step]).
template <int DP>
__device__ __forceinline__ Block product(const Reader<DP>& at, const uint8_t* tile, uint32_t block, const v8bf (&b)[2][DP / 32]) {
  Block p;
#pragma unroll
  for (int i = 0; i < 2; ++i) p.t[i][0] = p.t[i][1] = v4f{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < DP / 32; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v8bf a = at.along(tile, 2 * block + i, s);
#pragma unroll
      for (int j = 0; j < 2; ++j) p.t[i][j] = mfma(a, b[j][s], p.t[i][j]);
    }
  return p;
}
// Columns 16 j .. of a block as an operand.
__device__ __forceinline__ v8bf operand_of(const Block& p, int j) {
  const v4f &x = p.t[0][j], &y = p.t[1][j];
  return __builtin_bit_cast(v8bf, v4u{pack(x[0], x[1]), pack(x[2], x[3]), pack(y[0], y[1]), pack(y[2], y[3])});
}
// Sums (DP values of 32 columns) and what is added to them: a tile's block of 32 rows, turned, times the operands.
template <int DP>
struct Sums {
  v4f t[DP / 16][2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) t[d][0] = t[d][1] = v4f{0, 0, 0, 0};
  }
  __device__ __forceinline__ void add(const Reader<DP>& at, const uint8_t* tile, uint32_t block, const v8bf (&w)[2]) {
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
      const v8bf a = at.across(tile, block, d);
#pragma unroll
      for (int j = 0; j < 2; ++j) t[d][j] = mfma(a, w[j], t[d][j]);
    }
  }
  __device__ __forceinline__ void add(const Reader<DP>& at, const uint8_t* tile, uint32_t block, const v8bf (&w)[2], const v8bf (&rest)[2]) {
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
      const v8bf a = at.across(tile, block, d);
#pragma unroll
      for (int j = 0; j < 2; ++j) t[d][j] = mfma(a, w[j], t[d][j]);
#pragma unroll
      for (int j = 0; j < 2; ++j) t[d][j] = mfma(a, rest[j], t[d][j]);
    }
  }
  __device__ __forceinline__ void scale(const float (&factor)[2]) {
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
      for (int j = 0; j < 2; ++j) t[d][j] *= factor[j];
  }
};
// Columns that see a part of a tile give the rest weights of zero, and zero is what has to come of it, also where it holds infinities and NaN, which the
// product takes in.  So a pass whose sums are not all finite is gone through once more, with zeros in place of such values, and what the columns do see of
// them is added in the end, from memory.  (Looked for before each product that a column sees in part instead: 8 x 1024 rows, 12 heads of 64, forward and
// backward 106 us, so 99; with 128 channels dk and dv 30 % slower.)
template <int DP>
__device__ __forceinline__ bool finite(const Sums<DP>& s) {
  float zero = 0.0f;
#pragma unroll
  for (int d = 0; d < DP / 16; ++d)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(s.t[d][j][r], 0.0f, zero);
  return zero == 0.0f;
}
// A tile's stage, in the first pass or the second.
template <bool AGAIN>
struct Stage {
  static constexpr bool again = AGAIN;
  uint32_t value;
};
__device__ __forceinline__ uint32_t finite_of(uint32_t x) {  // two values; zeros for those that are not finite
  const uint32_t top = ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // (the exponent is all ones)
  return x & ~((top - (top >> 15)) | top);
}
// Sums::add so far.
template <int DP>
__device__ __forceinline__ void add_finite(Sums<DP>& s, const Reader<DP>& at, const uint8_t* tile, uint32_t block, const v8bf (&w)[2]) {
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) {
    v4u x = __builtin_bit_cast(v4u, at.across(tile, block, d));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = finite_of(x[i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) s.t[d][j] = mfma(__builtin_bit_cast(v8bf, x), w[j], s.t[d][j]);
    __builtin_amdgcn_sched_barrier(0);  // (one after the other: few registers)
  }
}
// Of a row the values that are not finite, to the columns that see it.
template <int DP>
__device__ __forceinline__ void add_rest(Sums<DP>& s, const Heads& h, size_t row, uint32_t head, uint32_t dim, bool seen0, bool seen1) {
  const uint16_t* const p = h.p + row * h.row + (size_t)head * h.head;
  const uint32_t g = (threadIdx.x >> 4) & 3u;
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) {
    v4f v;
    float zero = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t at = 16 * d + 4 * g + r;
      v[r] = at < dim ? __uint_as_float((uint32_t)p[at] << 16) : 0.0f;
      zero = __builtin_fmaf(v[r], 0.0f, zero);
    }
    if (!__any(zero != 0.0f)) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float x = __builtin_isfinite(v[r]) ? 0.0f : v[r];
      if (seen0) s.t[d][0][r] += x;
      if (seen1) s.t[d][1][r] += x;
    }
  }
}
// Over the four lanes of a column.
__device__ __forceinline__ float max_of_column(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_column(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Operand from memory: a row of a head, in steps of 32 values; zeros behind the head's values and for rows that are not there.
template <int DP>
__device__ __forceinline__ void load_operand(v8bf (&x)[DP / 32], const Heads& h, size_t row, uint32_t head, uint32_t dim, bool there) {
  const uint32_t g = (threadIdx.x >> 4) & 3u;
  const uint16_t* const p = h.p + row * h.row + (size_t)head * h.head;
#pragma unroll
  for (uint32_t s = 0; s < DP / 32; ++s) {
    v4u v = {0, 0, 0, 0};
    const uint32_t d = 32 * s + 8 * g;
    if (there && d < dim) v = *reinterpret_cast<const v4u*>(p + d);
    x[s] = __builtin_bit_cast(v8bf, v);
  }
}
// Values 16 d .. 16 d + 31 of a column (x, y: sixteen each), times `factor`, to its row of a head as bfloat16: neighbouring groups of lanes trade words, so
// that each stores eight neighbouring values.
__device__ __forceinline__ void store_values(v4f x, v4f y, uint32_t d, float factor, const Heads& h, size_t row, uint32_t head, uint32_t dim, bool there) {
  const uint32_t g = (threadIdx.x >> 4) & 3u, at = 16 * (d + (g & 1u)) + 8 * (g >> 1);
  x *= factor;
  y *= factor;
  const auto lo = __builtin_amdgcn_permlane16_swap(pack(x[0], x[1]), pack(y[0], y[1]), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(pack(x[2], x[3]), pack(y[2], y[3]), false, false);
  if (there && at < dim) *reinterpret_cast<v4u*>(h.p + row * h.row + (size_t)head * h.head + at) = v4u{lo[0], hi[0], lo[1], hi[1]};
}
// Columns 16 j .. of sums.
template <int DP>
__device__ __forceinline__ void store_column(const Sums<DP>& s, int j, float factor, const Heads& h, size_t row, uint32_t head, uint32_t dim, bool there) {
#pragma unroll
  for (uint32_t d = 0; d < DP / 16; d += 2) store_values(s.t[d][j], s.t[d + 1][j], d, factor, h, row, head, dim, there);
}

}  // namespace attn
}  // namespace srq
