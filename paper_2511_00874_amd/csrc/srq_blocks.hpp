// Block-scaled matrices: one byte a value (E4M3 or E5M2) and one power of two for every 128 consecutive values of a row.
// Device-side pieces that the kernels of this form share, and their launchers.  gfx950 only.
//
// The scale of a block is 2^(b - 127), b a byte: the least power of two with max|x| <= Qmax 2^(b - 127) over the block's finite
// values, b >= 27 (2^-100, the smallest step of the per-tensor quantizers too), no more than keeps Qmax 2^(b - 127) a finite binary32
// number (2^119 for E4M3, 2^112 for E5M2: larger values saturate), and 1 for a block of zeros.  Why a power of two:
//   - an 8-bit float has the same relative precision wherever the scale puts it, so rounding the scale up loses at most
//     one binade at the far end of the subnormals;
//   - x 2^-e and code 2^e are exact, in bfloat16 too, so the exact pipeline multiplies scaled values and never touches the sums;
//   - the matrix pipeline for codes takes such a scale with every operand row at no cost;
//   - a checkpoint whose blocks lie along the rows turns into one with blocks along the columns by shifting exponents.
#pragma once
#include <cstddef>

#include "srq_device.hpp"
#include "srq_internal.hpp"

namespace srq {

constexpr uint32_t SBLOCK = 128;  // values that share a scale
// Bytes of a row of codes: at least cols rounded up to 16; whole cache lines where the library's caller may choose.  (Turned rows are written
// 128 bytes by each tile: 12289 x 5632 turned into rows of 12304 bytes 80 us, of 12416 54.)
inline size_t block_pitch_least(size_t cols) { return (cols + 15) / 16 * 16; }
inline size_t block_pitch(size_t cols) { return (cols + 127) / 128 * 128; }
inline size_t scale_pitch(size_t cols) { return ((cols + SBLOCK - 1) / SBLOCK + 3) / 4 * 4; }   // bytes of a row of scales

// Source of a kernel that reads values: the dtypes of the C interface, and block-scaled codes.
enum BlockSource { BSRC_F32 = SRQ_F32, BSRC_BF16 = SRQ_BF16, BSRC_E4M3 = 2, BSRC_E5M2 = 3 };

struct Rounding {
  int sr;
  uint32_t k0, k1;
  uint64_t counter_offset;
  const uint64_t* counter_dev;
};

// ---- scales -----------------------------------------------------------------------------------------------------------
// The byte of a block whose largest finite |v| has these bits.
template <int KIND>
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  if (bits == 0) return 127u;  // nothing finite, or zeros alone
  constexpr int TOP = KIND == SRQ_E5M2 ? 15 : 8;  // Qmax = 1.75 * 2^TOP
  return (uint32_t)min(max((int)((bits + 0x1FFFFFu) >> 23) - TOP, 27), 254 - TOP);  // (carries where the fraction is above 0.75)
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float scale_value(uint32_t byte) { return byte ? __uint_as_float(byte << 23) : 0x1p-127f; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_of(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
// the largest within every 16 lanes, in all of them
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp_of<0xB1>(v));    // lane ^ 1
  v = max(v, dpp_of<0x4E>(v));    // lane ^ 2
  v = max(v, dpp_of<0x141>(v));   // 7 - lane of 8
  return max(v, dpp_of<0x140>(v));  // 15 - lane of 16
}
__device__ __forceinline__ float sum16(float v) {
  v += __uint_as_float(dpp_of<0xB1>(__float_as_uint(v)));
  v += __uint_as_float(dpp_of<0x4E>(__float_as_uint(v)));
  v += __uint_as_float(dpp_of<0x141>(__float_as_uint(v)));
  return v + __uint_as_float(dpp_of<0x140>(__float_as_uint(v)));
}
// over the four groups of 16 lanes
__device__ __forceinline__ float sum_of_rows(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ InvScale unit_scale(float inv) {
  InvScale s;
  s.inv = inv;
  s.inv16 = 0.0f;  // (integer formats only, as the rest)
  s.sub_m = 0;
  s.sub_qmax = 0.0f;
  s.sub_qi = 0;
  return s;
}

// grid of the kernels for a kind of the C interface
template <int KIND> struct BlockGrid;
template <> struct BlockGrid<SRQ_E4M3> { static constexpr int value = SRQ_E4M3_CONV; };
template <> struct BlockGrid<SRQ_E5M2> { static constexpr int value = SRQ_E5M2; };

// Largest and least magnitude of a group of eight values, NaN passed over by the one and kept by the other.
struct Extent {
  float most, least;
  __device__ __forceinline__ bool finite() const { return most < __builtin_inff() && least == least; }
};
__device__ __forceinline__ Extent extent_of(const float (&v)[8]) {
  Extent e = {fabsf(v[0]), fabsf(v[0])};
#pragma unroll
  for (int j = 1; j < 8; ++j) {
    e.most = fmaxf(e.most, fabsf(v[j]));
    e.least = __builtin_elementwise_minimum(e.least, fabsf(v[j]));
  }
  return e;
}
// Bits of the largest finite magnitude.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t most_finite(const float (&v)[8], const Extent& e) {
  uint32_t m = __float_as_uint(e.most);
  if (!e.finite()) {  // rare
    m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[j]));
  }
  return m;
}

// The smallest normal number of a kind's grid.
template <int KIND>
constexpr float LEAST_NORMAL = KIND == SRQ_E5M2 ? 0x1p-14f : 0x1p-6f;

// Eight values to codes, in units of 1 / inv: any values.
template <int KIND>
__device__ __forceinline__ u32x2 codes_of_any(const float (&v)[8], float inv, const uint32_t (&r)[4], bool sr) {
  return quantize_octet<BlockGrid<KIND>::value>({v[0], v[1], v[2], v[3]}, {v[4], v[5], v[6], v[7]}, unit_scale(inv), r, sr);
}
// The same for finite values whose results are normal numbers of the grid (a block's scale keeps them below Qmax): the conversions
// alone, with the seeds of convert_word.
template <int KIND, bool SR>
__device__ __forceinline__ u32x2 codes_of_normal(const float (&v)[8], float inv, const uint32_t (&r)[4]) {
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t n0 = ~r[2 * h], n1 = ~r[2 * h + 1];
    const uint32_t seed[4] = {(n0 << 16) | 0x8000u, (n0 & 0xFFFF0000u) | 0x8000u, (n1 << 16) | 0x8000u, (n1 & 0xFFFF0000u) | 0x8000u};
    int q = 0;
    int sd[4];
    float t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      t[e] = __fmul_rn(v[4 * h + e], inv);
      sd[e] = (int)(SR ? seed[e] : 0x80000000u) ^ ((int)__float_as_uint(t[e]) >> 31);
    }
    if constexpr (KIND == SRQ_E5M2) {
      q = __builtin_amdgcn_cvt_sr_bf8_f32(t[0], sd[0], q, 0);
      q = __builtin_amdgcn_cvt_sr_bf8_f32(t[1], sd[1], q, 1);
      q = __builtin_amdgcn_cvt_sr_bf8_f32(t[2], sd[2], q, 2);
      q = __builtin_amdgcn_cvt_sr_bf8_f32(t[3], sd[3], q, 3);
    } else {
      q = __builtin_amdgcn_cvt_sr_fp8_f32(t[0], sd[0], q, 0);
      q = __builtin_amdgcn_cvt_sr_fp8_f32(t[1], sd[1], q, 1);
      q = __builtin_amdgcn_cvt_sr_fp8_f32(t[2], sd[2], q, 2);
      q = __builtin_amdgcn_cvt_sr_fp8_f32(t[3], sd[3], q, 3);
    }
    w[h] = (uint32_t)q;
  }
  return w;
}
// The codes among them that are not normal numbers, or of the first normal binade, put right: by the spacing of the subnormal ones.  (What the lanes
// of a wave share stays one conversion; the general form for the groups that have such values would convert them anew.)
template <int KIND, bool SR>
__device__ __forceinline__ void small_codes(u32x2& w, const float (&v)[8], float inv, const uint32_t (&r)[4]) {
  constexpr uint32_t EXPONENT = KIND == SRQ_E5M2 ? 0x78787878u : 0x70707070u;  // without its last bit
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = __builtin_fmaf(v[4 * h + e], inv, 0.0f);  // (no negative zero)
    const uint32_t small = uniform_word<BlockGrid<KIND>::value>(t, r[2 * h], r[2 * h + 1], SR);
    const uint32_t normal = bytes_of_sign((w[h] & EXPONENT) + EXPONENT);
    w[h] = (w[h] & normal) | (small & ~normal);
  }
}
// A group of a row, its extent known.
template <int KIND, bool SR>
__device__ __forceinline__ u32x2 codes_of_octet(const float (&v)[8], const Extent& e, uint32_t byte, const uint32_t (&r)[4]) {
  const float inv = scale_inverse(byte);
  if (!e.finite() || byte == 254u - (KIND == SRQ_E5M2 ? 15 : 8)) return codes_of_any<KIND>(v, inv, r, SR);
  u32x2 w = codes_of_normal<KIND, SR>(v, inv, r);
  if (e.least < LEAST_NORMAL<KIND> * scale_value(byte)) small_codes<KIND, SR>(w, v, inv, r);
  return w;
}
template <bool SR>
__device__ __forceinline__ void thresholds(const Rounding& rnd, uint64_t block, uint32_t (&r)[4]) {
  r[0] = r[1] = r[2] = r[3] = RTN_WORD;
  if constexpr (SR) philox_block(block, rnd.k0, rnd.k1, r);
}

// Four codes times a power of two each (delta: the exponents, times the codes' unit of one, modulo 128, a byte each), all normal before and
// after: sums of seven bits a byte, beside the signs.
__device__ __forceinline__ uint32_t codes_shifted(uint32_t codes, uint32_t delta) {
  const uint32_t sum = (codes & 0x7F7F7F7Fu) + delta;
  return (sum & 0x7F7F7F7Fu) | (codes & 0x80808080u);
}

// Rows [first, first + most) of a matrix with rows of `pitch` bytes, as many as it has, as a buffer: what lies behind them reads as zeros.  Places
// in it are counted from the first row's begin in 32 bits (at most 2^21 columns, and 128 rows: under 2^31 bytes); OUT is beyond any.
constexpr uint32_t OUT = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void* x, size_t pitch, uint32_t first, uint32_t rows, uint32_t most) {
  const uint32_t n = first < rows ? min(rows - first, most) : 0u;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(static_cast<const uint8_t*>(x)) + first * pitch, 0, (int)(n * (uint32_t)pitch), 0x00020000);
}
constexpr int STREAMED = 2, KEPT = 0;  // cache policies of the fetches: not read again, or by another workgroup

// Eight values of a row as binary32: from the two dtypes, or from codes and the byte of their scale.
template <int SRC>
struct Octet;
template <> struct Octet<BSRC_F32> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void* x, size_t at) {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + at);
    a = __builtin_nontemporal_load(p);
    b = __builtin_nontemporal_load(p + 1);
  }
  template <int POLICY>
  __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at * 4, 0, POLICY));
    b = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at * 4 + 16, 0, POLICY));
  }
  __device__ __forceinline__ void zero() { a = b = f32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
template <> struct Octet<BSRC_BF16> {
  u32x4 a;
  __device__ __forceinline__ void load(const void* x, size_t at) {
    a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(x) + at));
  }
  template <int POLICY>
  __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    a = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at * 2, 0, POLICY));
  }
  __device__ __forceinline__ void zero() { a = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  }
};
template <int KIND>
struct CodeOctet {
  u32x2 a;
  __device__ __forceinline__ void load(const void* x, size_t at) {
    a = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(x) + at));
  }
  template <int POLICY>
  __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    a = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, POLICY));
  }
  __device__ __forceinline__ void get(float (&v)[8], float scale) const {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x2 lo, hi;
      if constexpr (KIND == SRQ_E5M2) {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8(a[i], false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8(a[i], true);
      } else {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], true);
      }
      v[4 * i] = __fmul_rn(lo[0], scale);
      v[4 * i + 1] = __fmul_rn(lo[1], scale);
      v[4 * i + 2] = __fmul_rn(hi[0], scale);
      v[4 * i + 3] = __fmul_rn(hi[1], scale);
    }
  }
};
template <> struct Octet<BSRC_E4M3> : CodeOctet<SRQ_E4M3> {};
template <> struct Octet<BSRC_E5M2> : CodeOctet<SRQ_E5M2> {};

// ---- one tile of 128 x 128 values to codes in one or both layouts ---------------------------------------------------------
// 512 threads; thread t holds columns 8 (t % 16) .. + 7 of rows 4 (t / 16) .. + 3, as v[row][column], zeros outside the matrix.
// Sixteen neighbouring lanes hold a whole block of a row; a block of a column is a thread's four rows, its wave's four
// groups of lanes and the eight waves, who meet in LDS.  Four rows of a thread are four neighbouring bytes of a turned row.
//
// Both layouts share one rounding: scales are powers of two and thresholds those of the element, so a value that is a normal number of the
// grid in both has the same significand in both, and the turned code is the other one with the difference of the scales' exponents added to
// its exponent -- three operations for four codes.  Groups with a value for which that does not hold (zeros and what is far below its block's
// largest, Inf, NaN) are rounded twice, by the general form; in E4M3, in whose short range most waves meet one, only what is small is put right
// (gradients of a gated block of 16384 x 5632: 298 -> 274 us; in E5M2 246 -> 250, and one layout alone 38 -> 39).
// What bounds it: vector work and memory alike (16384 x 2048 bfloat16 to E5M2 in both layouts, nearest: with each layout rounded by the
// general form 30 vector instructions a value, 28 of 44 us).
constexpr int TILE_THREADS = 512, TILE_ROWS = 4;
struct TileOut {
  uint8_t *codes, *scales, *codes_t, *scales_t;  // codes / codes_t null: that layout is not written
  uint32_t rows, cols;           // of the matrix
  size_t pitch, spitch, pitch_t, spitch_t;
};
constexpr uint32_t TURN_PITCH = SBLOCK + 16;  // (sixteen columns written at one row fall on different banks)
struct TileLds {                              // both parts are read 16 bytes at a time
  alignas(16) uint32_t top[SBLOCK];  // largest of every column
  alignas(16) uint8_t turned[SBLOCK * TURN_PITCH];
};
static_assert(alignof(TileLds) == 16 && offsetof(TileLds, turned) % 16 == 0 && TURN_PITCH % 16 == 0, "16-byte reads");
__device__ __forceinline__ void tile_begin(TileLds& lds) {
  if (threadIdx.x < SBLOCK) lds.top[threadIdx.x] = 0;
  __syncthreads();
}

// row0, col0: of the tile; first: index, in the tensor whose thresholds these are, of the element at (row0, col0), ld its row length.
// After tile_begin.
template <int KIND, bool SR, bool ROWS>
__device__ __forceinline__ void tile_to_codes(const float (&v)[TILE_ROWS][8], const TileOut& o, TileLds& lds, uint32_t row0, uint32_t col0,
                                              size_t first, size_t ld, const Rounding& rnd, uint64_t counter) {
  constexpr uint32_t CAP = 254u - (KIND == SRQ_E5M2 ? 15 : 8);  // (the largest scale: values may saturate)
  constexpr int M = KIND == SRQ_E5M2 ? 2 : 3;                   // fraction bits
  constexpr bool SHARED = ROWS && KIND == SRQ_E4M3;             // groups with small values: one conversion for the whole wave
  const uint32_t t = threadIdx.x, cg = t & 15u, rg = t >> 4;
  const uint32_t col = col0 + 8 * cg;
  Extent ext[TILE_ROWS];
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i) ext[i] = extent_of(v[i]);
  const bool finite = ext[0].finite() && ext[1].finite() && ext[2].finite() && ext[3].finite();
  // columns: this thread's rows, its wave's, all waves' (two columns to each group of lanes)
  {
    uint32_t key[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) key[j] = __float_as_uint(fmaxf(fmaxf(fabsf(v[0][j]), fabsf(v[1][j])), fmaxf(fabsf(v[2][j]), fabsf(v[3][j]))));
    if (!finite) {
#pragma unroll
      for (int j = 0; j < 8; ++j) key[j] = max(max(finite_bits(v[0][j]), finite_bits(v[1][j])), max(finite_bits(v[2][j]), finite_bits(v[3][j])));
    }
    // halves of the wave, then of the halves, each keeping half of the columns: two are left to each group of sixteen lanes
    uint32_t m[4], n[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto x = __builtin_amdgcn_permlane32_swap(key[j], key[j + 4], false, false);
      m[j] = max((uint32_t)x[0], (uint32_t)x[1]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const auto x = __builtin_amdgcn_permlane16_swap(m[j], m[j + 2], false, false);
      n[j] = max((uint32_t)x[0], (uint32_t)x[1]);
    }
    uint32_t* const at = lds.top + 8 * cg + ((rg & 1u) << 1) + ((rg & 2u) << 1);
    atomicMax(at, n[0]);  // (in LDS, of whole numbers: the same in any order)
    atomicMax(at + 1, n[1]);
  }
  __syncthreads();
  uint32_t byte_col[8], most_col = 0;
#pragma unroll
  for (int j = 0; j < 8; j += 4) {
    const u32x4 m = *reinterpret_cast<const u32x4*>(lds.top + 8 * cg + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      byte_col[j + e] = scale_byte<KIND>(m[e]);
      most_col = max(most_col, byte_col[j + e]);
    }
  }
  if (rg == 0 && col < o.cols) {
    const uint32_t b = row0 / SBLOCK;
    uint8_t* at = o.scales_t + col * o.spitch_t + b;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j, at += o.spitch_t) *at = (uint8_t)byte_col[j];
  }
  // what the columns' scales take from a code's exponent, four to a word
  uint32_t less[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    less[h] = (((0u - byte_col[4 * h]) << M) & 0x7Fu) | ((((0u - byte_col[4 * h + 1]) << M) & 0x7Fu) << 8) |
              ((((0u - byte_col[4 * h + 2]) << M) & 0x7Fu) << 16) | ((((0u - byte_col[4 * h + 3]) << M) & 0x7Fu) << 24);
  u32x2 w[TILE_ROWS];
  const uint64_t group = counter + first / 8;                           // of the tile's first element (rows are whole groups)
  const uint32_t lrow = TILE_ROWS * rg, ld8 = (uint32_t)(ld / 8);
  uint8_t* const out = o.codes + row0 * o.pitch + col0;                 // (not used without that layout)
  uint8_t* const out_scales = o.scales + row0 * o.spitch + col0 / SBLOCK;
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i) {
    uint32_t r[4];
    thresholds<SR>(rnd, group + ((lrow + i) * ld8 + cg), r);
    // (without the layout along the rows any scale will do for the one rounding)
    const uint32_t byte = ROWS ? scale_byte<KIND>(max16(most_finite(v[i], ext[i]))) : most_col;
    u32x2 c;
    const bool normal = ext[i].least >= LEAST_NORMAL<KIND> * scale_value(max(byte, most_col));
    if ((SHARED ? ext[i].finite() : normal && ext[i].most < __builtin_inff()) && max(byte, most_col) < CAP) {
      c = codes_of_normal<KIND, SR>(v[i], scale_inverse(byte), r);
      const uint32_t more = ((byte << M) & 0x7Fu) * 0x01010101u;
#pragma unroll
      for (int h = 0; h < 2; ++h) w[i][h] = codes_shifted(c[h], (more + less[h]) & 0x7F7F7F7Fu);
      if (SHARED && !normal) {
        small_codes<KIND, SR>(c, v[i], scale_inverse(byte), r);
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = __fmul_rn(v[i][j], scale_inverse(byte_col[j]));
        w[i] = codes_of_normal<KIND, SR>(s, 1.0f, r);
        small_codes<KIND, SR>(w[i], s, 1.0f, r);
      }
    } else {
      if constexpr (ROWS) c = codes_of_any<KIND>(v[i], scale_inverse(byte), r, SR);
      float s[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = __fmul_rn(v[i][j], scale_inverse(byte_col[j]));
      w[i] = codes_of_any<KIND>(s, 1.0f, r, SR);
    }
    if constexpr (ROWS) {
      if (row0 + lrow + i < o.rows && col < o.cols) {
        __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(out + ((lrow + i) * (uint32_t)o.pitch + 8 * cg)));
        if (cg == 0) out_scales[(lrow + i) * (uint32_t)o.spitch] = (uint8_t)byte;
      }
    }
  }
  // turned row c of the tile: 128 bytes, its 16-byte chunk k at chunk k ^ (c / 16)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t q[4];
    turn4x4(w[0][h], w[1][h], w[2][h], w[3][h], q);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint32_t*>(lds.turned + (8 * cg + 4 * h + j) * TURN_PITCH + (((rg >> 2) ^ (cg >> 1)) << 4) + ((rg & 3u) << 2)) = q[j];
  }
  __syncthreads();
  const uint32_t end = (o.rows + 15u) & ~15u;  // (up to there the bytes behind a turned row are zeros)
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const uint32_t id = n * TILE_THREADS + t, c = id >> 3, k = id & 7u;
    const u32x4 q = *reinterpret_cast<const u32x4*>(lds.turned + c * TURN_PITCH + ((k ^ (c >> 4)) << 4));
    if (col0 + c < o.cols && row0 + 16 * k < end)
      __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(o.codes_t + (size_t)(col0 + c) * o.pitch_t + row0 + 16 * k));
  }
}

// ---- activations of the gated block ---------------------------------------------------------------------------------------
// act(g) and act'(g).  SiLU: g s, s (1 + g (1 - s)) with s = 1 / (1 + e^-g).  GELU: g Phi(g), Phi(g) + g phi(g).
// Phi: of z = |g|, Phi(-z) = e^(-z^2 / 2) P(t) with t = 1 / (1 + 0.275 z), P a polynomial of degree 9 without a constant, fitted here for the least
// relative error over z in [0, 14] (3.9e-8); Phi(z) = 1 - Phi(-z).  No sum cancels below zero, where 1 + erf is 4 % off at -5 and
// has nothing left beyond -5.5: within 15 units of 2^-24 of Phi for g > -4 and 50 for g > -7 (the exponent's rounding), and the density is the same power.
// 16384 x 5632 backward, bfloat16 to E5M2 stochastically: 274 us (with erf 541); forward with checkpoint 680 (704).
template <int ACT>
__device__ __forceinline__ void activate(float g, float& a, float& da) {
  if constexpr (ACT == SRQ_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g));
    a = g * s;
    da = s * __builtin_fmaf(g, 1.0f - s, 1.0f);
  } else {
    const float z = fabsf(g), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.275f, z, 1.0f));
    const float density = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float q = 0.026249513f;
    for (const float c : {-0.106021337f, 0.12018393f, -0.0233457666f, 0.0796035826f, 0.082601741f, 0.10123615f, 0.109789461f, 0.109702744f})
      q = __builtin_fmaf(q, t, c);
    q *= t * density;
    const float p = g < 0.0f ? q : 1.0f - q;
    a = g * p;
    da = __builtin_fmaf(0.39894228f * g, density, p);
  }
}

// ---- launchers --------------------------------------------------------------------------------------------------------------
// A launch has fewer than 2^32 threads: `wgs` workgroups (of at most 1024) in launches of up to 2^21, f(the first, how many).
template <class F>
void in_launches(size_t wgs, F&& f) {
  constexpr size_t MOST = (size_t)1 << 21;
  for (size_t first = 0; first < wgs; first += MOST) f((uint32_t)first, (unsigned)(wgs - first < MOST ? wgs - first : MOST));
}

// Values to codes along the rows and / or turned.  src: BlockSource; of codes, scales and their pitch.
struct BlockQuantize {
  const void* x;
  const uint8_t* x_scales;
  size_t x_pitch, x_spitch;  // elements of x, bytes of scales
  int src, kind;
  TileOut out;
  Rounding rnd;
};
hipError_t launch_block_quantize(const BlockQuantize& q, hipStream_t stream);
hipError_t launch_block_restore(void* x, int dtype, const uint8_t* codes, size_t pitch, const uint8_t* scales, size_t rows, size_t cols,
                                int kind, hipStream_t stream);

// Gradients of G and U side by side (rows x 2 F) from dH and the checkpoint of G and U.
struct GatedBackward {
  const void* dh;
  int dtype, act, kind;
  const uint8_t *gu, *gu_scales;
  uint32_t F;
  TileOut out;
  Rounding rnd;
};
hipError_t launch_gated_backward(const GatedBackward& g, hipStream_t stream);

struct NormForward {
  const void *x, *residual;
  void *h, *y;
  const float* gamma;
  float* rstd;
  uint8_t* scales;   // not null: y takes E4M3 / E5M2 codes (kind)
  size_t y_pitch, spitch;
  int dtype, kind;
  uint32_t rows, cols;
  float eps;
  Rounding rnd;
};
hipError_t launch_norm_forward(const NormForward& n, hipStream_t stream);
struct NormBackward {
  const void *dy, *dh, *h;
  void* dx;
  const float *gamma, *rstd;
  float *dgamma, *partial;
  int dtype, accumulate;
  uint32_t rows, cols;
};
size_t norm_backward_partials(uint32_t rows, uint32_t cols);
hipError_t launch_norm_backward(const NormBackward& n, hipStream_t stream);

// out (P x Q) = alpha X Z^T (+ out), binary32 or bfloat16.
struct BlockOperand {
  const uint8_t *codes, *scales;
  size_t pitch, spitch;
};
struct BlockProduct {
  BlockOperand X, Z;
  int kindX, kindZ, f8;
  void* out;
  int out_bf16, accumulate;
  float alpha;
  size_t P, Q, R;
  float* partial;  // of block_product_workspace bytes
};
size_t block_product_workspace(size_t P, size_t Q, size_t R, int f8);
hipError_t launch_block_product(const BlockProduct& p, hipStream_t stream);

// H = act(X Wg^T) (X Wu^T), W = Wg over Wu; h: bfloat16, or codes with scales; gu: the checkpoint of both sums, or null.
struct GatedForward {
  BlockOperand X, W;
  int act, f8;
  void* h;
  uint8_t* h_scales;
  uint8_t *gu, *gu_scales;
  uint32_t M, F, K;
  Rounding rnd_h, rnd_gu;
  float* partial;
};
size_t gated_forward_workspace(size_t M, size_t F, size_t K, int f8);
hipError_t launch_gated_forward(const GatedForward& g, hipStream_t stream);

}  // namespace srq
