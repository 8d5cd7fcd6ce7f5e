// Attention, backward: the scores are computed again from q, k and lse, once for dq and once for dk and dv, so that every sum has one owner and one
// order.
#include "srq_attention.hpp"

namespace srq {
namespace {
using namespace attn;

struct Backward {
  AttentionBackward a;
  Cut cut_q, cut_k;    // of the keys of a tile of queries, and of the queries of a tile of keys
  float *partial_q, *partial_k;  // the pieces' sums, where there are several
  uint32_t* again;      // dk and dv, by workgroup: sums that are not finite
  float *lse2, *delta;  // heads_q x rows_q: lse log2 e (+inf where a row sees nothing: its p is 0 then), and sum of do o
};

__device__ __forceinline__ float dot(const v8bf& a, const v8bf& b, float sum) {
  const v4u x = __builtin_bit_cast(v4u, a), y = __builtin_bit_cast(v4u, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum = __builtin_fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum);
    sum = __builtin_fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(y[i] & 0xFFFF0000u), sum);
  }
  return sum;
}

// Sums over this lane's keys of the wave's 32 columns, of ds and p as they were rounded.
struct Totals {
  float s[2] = {0.0f, 0.0f}, p[2] = {0.0f, 0.0f};
};
__device__ __forceinline__ float add_two(uint32_t x, float sum) {  // two values of 16 bits
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, x), __builtin_bit_cast(v2bf, 0x3F803F80u), sum, false);
}
// A block of sixteen rows times the columns' operands.
template <int DP>
__device__ __forceinline__ void product16(const Reader<DP>& at, const uint8_t* tile, uint32_t block, const v8bf (&b)[2][DP / 32], v4f (&x)[2]) {
  x[0] = x[1] = v4f{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < DP / 32; ++s) {
    const v8bf a = at.along(tile, block, s);
#pragma unroll
    for (int j = 0; j < 2; ++j) x[j] = mfma(a, b[j][s], x[j]);
  }
}
struct Operands {  // of a block's two sets of columns
  v8bf x[2];
};
__device__ __forceinline__ Operands operands(const v4u (&w)[2]) { return {{__builtin_bit_cast(v8bf, w[0]), __builtin_bit_cast(v8bf, w[1])}}; }
// A block of rows times two operands.
template <int DP>
__device__ __forceinline__ void add_both(Sums<DP>& x, Sums<DP>& y, const Reader<DP>& at, const uint8_t* tile, uint32_t block, const Operands& wx, const Operands& wy) {
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) {
    const v8bf a = at.across(tile, block, d);
#pragma unroll
    for (int j = 0; j < 2; ++j) x.t[d][j] = mfma(a, wx.x[j], x.t[d][j]);
#pragma unroll
    for (int j = 0; j < 2; ++j) y.t[d][j] = mfma(a, wy.x[j], y.t[d][j]);
  }
}
// The first pass over a tile, of keys that all rows see or not; the second, for dq and the mean by themselves: registers.
enum { WHOLE, BOTH, DQ, MEAN };
template <int PART>
struct Part {
  static constexpr int part = PART;
  uint32_t value;
};
// What a piece of a row's keys leaves.
template <int DP>
struct Partial {
  float *dq, *mean, *totals;
  __device__ __forceinline__ Partial(const Backward& f, uint32_t piece, size_t row, uint32_t head) {
    const AttentionShape& s = f.a.shape;
    const size_t each = (size_t)s.rows_q * s.heads_q, at = piece * each + row * s.heads_q + head;
    dq = f.partial_q + 2 * at * DP;
    mean = dq + DP;
    totals = f.partial_q + 2 * f.cut_q.pieces * each * DP + 2 * at;
  }
};

// ---- dq ---------------------------------------------------------------------------------------------------------------------------
// As the forward pass: a wave has 32 rows, the columns of
//   S^T = K Q^T,  dP^T = V dO^T,  P = 2^(c S - lse2),  dS = P (dP - delta),  dQ^T = K^T dS^T - K^T P^T (sum dS / sum P).
// A row of dS has the sum 0, but not with delta from an o of 16 bits: with delta - e in place of delta, each dS_j is P_j e too large, and dQ has e times
// the row's mean key too much, which is far larger than what tells the keys apart where they have an offset, and larger than the row's dQ where one key has
// nearly all the weight.  So the mean K^T P^T is summed beside dQ, and what the rounded dS and P add up to says how much of it to take off:
// of the row's own keys, so that nothing else has a part in dq, and good to the roundings of dS however the weights lie.  (dQ is 2.3e-3 off with scores of any
// size, as one rounding of dS and one of dQ leave it.  The mean of a tile of keys in place of the row's, and dS as two values of 16 bits: as many
// products, 2.3e-3, but 8e-3 with queries ten times as large, single rows by 17 times their size.)  The other kernel gets delta + e.
// Rows that see up to one tile of keys have dS as two values, itself and what its rounding leaves: there a row's gradient can hang on a difference of two.
// 9 packed sequences of up to 4095 rows, 16 heads of 128 over 4: 244 us, 0.68 PFLOP/s of S, dP and dQ under the diagonal (0.91 with the mean), at all 256
// registers of two waves a SIMD, matrix instructions in 47 % of the cycles and vector ones in 50 %; 8 x 1024 rows, 12 heads of 64, 47 us, three waves a SIMD
// (with two, 56).  (Tiles that all rows see by themselves, without the branch for what is hidden: 128 channels 250 us to 244.)
template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP == 64 ? 3 : 2) void attention_dq_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BM = NW * 32, STAGE = 2 * KT * Rows<DP>::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const AttentionShape& s = f.a.shape;
  const Place place = place_of(s.heads_q, slots * f.cut_q.pieces);
  if (!place.valid) return;
  const uint32_t head = place.head, head_k = head / (s.heads_q / s.heads_kv);
  const PieceOf of(place.slot, f.cut_q.pieces);
  const uint32_t piece = of.piece;
  const Queries rows(s, BM, slots, of.slot);
  if (!rows.t.valid) return;
  const Tile& t = rows.t;
  const Span& keys = rows.keys;
  const uint32_t pieces = f.cut_q.count(rows.tiles), each = f.cut_q.each(rows.tiles);
  const uint32_t begin = piece * each, tiles = min(begin + each, rows.tiles);
  if (piece && begin >= tiles) return;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int row0 = (int)(t.row + wave * 32), row[2] = {row0 + (int)(lane & 15u), row0 + 16 + (int)(lane & 15u)};
  const bool there[2] = {row[0] < (int)t.rows, row[1] < (int)t.rows};
  const int most = row0 < (int)t.rows ? rows.limit_of(min(row0 + 31, (int)t.rows - 1)) : 0;
  const int least = rows.limit_of(row0);

  const RowSource ks = row_source(f.a.k, keys.first, keys.rows, head_k, s.dim), vs = row_source(f.a.v, keys.first, keys.rows, head_k, s.dim);
  const uint32_t base = lds_address(lds);
  const auto fetch = [&](uint32_t kt, uint32_t stage) {
    const uint32_t to = base + stage * STAGE, at_lane = worked_out(lane);
    Fetch<DP, KT, NW>(ks, wave, at_lane)(ks, kt * KT, to, wave);
    Fetch<DP, KT, NW>(vs, wave, at_lane)(vs, kt * KT, to + KT * Rows<DP>::PITCH, wave);
  };
  if (begin < tiles) fetch(begin, 0);
  const size_t out[2] = {(size_t)t.first + (there[0] ? row[0] : 0), (size_t)t.first + (there[1] ? row[1] : 0)};
  v8bf q[2][DP / 32], dout[2][DP / 32];
  float lse2[2], delta[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    v8bf o[DP / 32];
    load_operand<DP>(dout[j], f.a.dout, out[j], head, s.dim, there[j]);
    load_operand<DP>(o, f.a.o, out[j], head, s.dim, there[j]);
    load_operand<DP>(q[j], f.a.q, out[j], head, s.dim, there[j]);
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < DP / 32; ++n) sum = dot(dout[j][n], o[n], sum);
    delta[j] = sum_of_column(sum);
    lse2[j] = SRQ_INF;
    if (there[j]) {
      const float v = f.a.lse[(size_t)head * s.rows_q + out[j]];
      lse2[j] = v == -SRQ_INF ? SRQ_INF : v * LOG2E;
      if (g == 0 && piece == 0) f.lse2[(size_t)head * s.rows_q + out[j]] = lse2[j];
    }
  }
  Sums<DP> dq, mean;
  dq.clear();
  mean.clear();
  Totals totals;
  const float c = s.scale * LOG2E;
  const bool few = rows.limit_of((int)t.row) <= (int)KT;

  const auto tile = [&](uint32_t kt, auto stage) __attribute__((always_inline)) {  // (its places in LDS are constants)
    landed_everywhere();
    if (kt + 1 < tiles) fetch(kt + 1, 1 - stage.value);
    const uint8_t* const kl = lds + stage.value * STAGE;
    const uint8_t* const vl = kl + KT * Rows<DP>::PITCH;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int key0 = (int)(kt * KT) + 32 * n;
      if (key0 >= most) return;
      const Reader<DP> at(worked_out(lane));
      v4u wp[2], ws[2], rest[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // (sixteen keys after the others: registers)
        v4f p[2], ds[2];
        product16(at, kl, 2 * n + i, q, p);
        if (stage.part != MEAN) product16(at, vl, 2 * n + i, dout, ds);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p[j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[j][r], c, -lse2[j]));
            if (stage.part != MEAN) ds[j][r] = p[j][r] * (ds[j][r] - delta[j]);
          }
        if (stage.part != WHOLE && (DP > 64 || key0 + 32 > least)) {  // (with 128 channels a branch here costs registers: 280 us for 252)
          const int at_lane = (int)worked_out(lane), first = row0 + (at_lane & 15), behind = key0 + 4 * (at_lane >> 4);
          const int left[2] = {rows.limit_of(first) - behind, rows.limit_of(first + 16) - behind};
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              p[j][r] = 16 * i + r < left[j] ? p[j][r] : 0.0f;
              if (stage.part != MEAN) ds[j][r] = 16 * i + r < left[j] ? ds[j][r] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t at_word = 2 * i + h;
            if (stage.part != DQ) {
              wp[j][at_word] = pack(p[j][2 * h], p[j][2 * h + 1]);
              totals.p[j] = add_two(wp[j][at_word], totals.p[j]);
            }
            if (stage.part != MEAN) {
              const uint32_t w = ws[j][at_word] = pack(ds[j][2 * h], ds[j][2 * h + 1]);
              totals.s[j] = add_two(w, totals.s[j]);
              if (stage.part == DQ && few) {
                rest[j][at_word] = pack(ds[j][2 * h] - __uint_as_float(w << 16), ds[j][2 * h + 1] - __uint_as_float(w & 0xFFFF0000u));
                totals.s[j] = add_two(rest[j][at_word], totals.s[j]);
              }
            }
          }
      }
      if (stage.part == WHOLE || stage.part == BOTH) add_both(dq, mean, at, kl, n, operands(ws), operands(wp));
      if (stage.part == DQ) {  // (a row that sees a key which is not finite has NaN for weights, or zeros)
        add_finite(dq, at, kl, n, operands(ws).x);
        if (few) add_finite(dq, at, kl, n, operands(rest).x);
      }
      if (stage.part == MEAN) add_finite(mean, at, kl, n, operands(wp).x);
    }
  };
  if (!few) {
    const uint32_t whole = min(tiles, max(begin, (uint32_t)max(0, rows.limit_of((int)t.row)) / KT));
    for (uint32_t kt = begin; kt < whole; kt += 2) {
      tile(kt, Part<WHOLE>{0});
      if (kt + 1 < whole) tile(kt + 1, Part<WHOLE>{1});
    }
#pragma unroll 1
    for (uint32_t kt = whole; kt < tiles; ++kt) tile(kt, Part<BOTH>{(kt - begin) & 1u});
  }
  if (few || __syncthreads_or(!finite(dq) || !finite(mean))) {
    if (!few) {
      dq.clear();
      fetch(begin, 0);
    }
    totals = Totals();
#pragma unroll 1
    for (uint32_t kt = begin; kt < tiles; ++kt) tile(kt, Part<DQ>{(kt - begin) & 1u});
    landed_everywhere();
    mean.clear();
    if (begin < tiles) fetch(begin, 0);
#pragma unroll 1
    for (uint32_t kt = begin; kt < tiles; ++kt) tile(kt, Part<MEAN>{(kt - begin) & 1u});
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const size_t at_row = (size_t)head * s.rows_q + out[j];
    const float of_ds = sum_of_column(totals.s[j]), of_p = sum_of_column(totals.p[j]);
    const float off = of_p == 0.0f ? 0.0f : of_ds / of_p;
    if (g == 0 && there[j] && piece == 0) f.delta[at_row] = delta[j] + (pieces == 1 ? off : 0.0f);
    if (pieces == 1) {
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) dq.t[d][j] -= mean.t[d][j] * off;
      store_column<DP>(dq, j, s.scale, f.a.dq, out[j], head, s.dim, there[j]);
    } else if (there[j]) {
      const Partial<DP> part(f, piece, out[j], head);
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        *reinterpret_cast<v4f*>(part.dq + 16 * d + 4 * g) = dq.t[d][j];
        *reinterpret_cast<v4f*>(part.mean + 16 * d + 4 * g) = mean.t[d][j];
      }
      if (g == 0) part.totals[0] = of_ds, part.totals[1] = of_p;
    }
  }
}

// The pieces of dq, one after the other: DP / 4 threads a row.
template <int DP, int NW>
__global__ __launch_bounds__(256) void attention_dq_join_kernel(Backward f) {
  constexpr uint32_t T = DP / 4, BM = NW * 32;
  const AttentionShape& s = f.a.shape;
  const Queries rows(s, BM, gridDim.x, blockIdx.x);
  if (!rows.t.valid) return;
  const uint32_t pieces = f.cut_q.count(rows.tiles), head = blockIdx.y, d = 4 * (threadIdx.x % T);
  if (pieces == 1 || d >= s.dim) return;
  const uint32_t i = rows.t.row + blockIdx.z * (256 / T) + threadIdx.x / T;
  if (i >= rows.t.rows) return;
  const size_t row = (size_t)rows.t.first + i;
  v4f v = {0, 0, 0, 0}, mean = {0, 0, 0, 0}, part[MOST_PIECES], part_mean[MOST_PIECES];
  float of_ds = 0.0f, of_p = 0.0f;
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p) {
    const Partial<DP> x(f, p < pieces ? p : 0, row, head);
    part[p] = *reinterpret_cast<const v4f*>(x.dq + d);
    part_mean[p] = *reinterpret_cast<const v4f*>(x.mean + d);
    of_ds += p < pieces ? x.totals[0] : 0.0f;
    of_p += p < pieces ? x.totals[1] : 0.0f;
  }
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p)
    if (p < pieces) v += part[p], mean += part_mean[p];
  const float off = of_p == 0.0f ? 0.0f : of_ds / of_p;
  v -= mean * off;
  if (d == 0) f.delta[(size_t)head * s.rows_q + row] += off;
  v *= s.scale;
  *reinterpret_cast<v2u*>(f.a.dq.p + row * f.a.dq.row + (size_t)head * f.a.dq.head + d) = v2u{pack(v[0], v[1]), pack(v[2], v[3])};
}

// ---- dk and dv ------------------------------------------------------------------------------------------------------------------------
// A workgroup has 32 NW keys of one key head, a wave 32 of them, the columns of
//   S = Q K^T,  dP = dO V^T,  dV^T = dO^T P,  dK^T = Q^T dS;
// the rows of q and do of all heads of the group go through LDS in tiles.  p and ds are rounded to bfloat16 for their products: what is summed there has no
// part in common, and dk and dv are 2.3e-3 to 2.4e-3 off, where a few rows have most of the gradient up to 2.6e-3 (their own rounding 1.7e-3).  (As two values
// of 16 bits each, which leaves 1.7e-3: 45 us to 59 and 307 to 398 in the cases below, an eighth of a step.)
// 9 packed sequences of up to 4095 rows, 16 heads of 128 over 4: 285 us, 0.78 PFLOP/s, one wave a SIMD (443 registers), matrix instructions in 40 % of the
// cycles, vector ones in 33 %; 8 x 1024 rows, 12 heads of 64, 44.5 us.
constexpr uint32_t QT = 64;

// The order of both sums' products: operands are read four ahead of the instructions that take them, as with one wave a SIMD nothing else covers the reads
// (the compiler's order has one ahead: 307 us to 285 in the larger case above, 45.5 to 44.5 in the smaller).
template <int DP>
__device__ __forceinline__ void reads_ahead() {
  constexpr int N = DP / 8, AHEAD = 4;  // operands
  __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
  for (int d = 0; d < N; ++d) {
    __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
    if (d + AHEAD < N) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}
struct Keys {
  Tile t;
  Span keys, queries;
  int lq, lk, shift;         // row i sees keys below i + shift
  uint32_t tile0, tiles;     // of the queries that see any of the keys: the first tile, how many
  bool valid;
  __device__ __forceinline__ Keys(const AttentionShape& s, uint32_t bn, uint32_t slots, uint32_t place)
      : t(ranked_tile(s.offsets_k, s.rows_k, s.sequences, bn, slots, place, true)) {
    valid = t.valid;
    if (!valid) return;
    keys = keys_of(s, t.sequence);
    queries = span_of(s.offsets_q, s.rows_q, s.sequences, t.sequence);
    lq = (int)queries.rows;
    lk = (int)keys.rows;
    shift = lk - lq + 1;
    valid = t.row < keys.rows;
    const int first = s.causal ? max(0, (int)t.row - shift + 1) : 0;
    tile0 = (uint32_t)first / QT;
    tiles = lq > first ? ((uint32_t)lq + QT - 1) / QT - tile0 : 0u;
  }
};
// With 128 channels the second pass is a launch of its own, for the workgroups that want it (4.5 us where none does): in the same kernel it costs the
// first its registers, 315 us to 360 for 9 packed sequences of up to 4095 rows, 16 heads over 4.  With 64 it costs nothing there.
template <int DP>
constexpr bool apart = DP > 64;
template <int DP, int NW, bool AGAIN>
__global__ __launch_bounds__(NW * 64, DP == 64 ? 2 : 1) void attention_dkv_kernel(Backward f, uint32_t slots) {
  constexpr bool APART = apart<DP>;
  constexpr uint32_t BN = NW * 32, TILE = QT * Rows<DP>::PITCH, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  __shared__ __attribute__((aligned(16))) float rows_lds[2][2][QT];  // lse2 and delta
  const AttentionShape& s = f.a.shape;
  const Place place = place_of(s.heads_kv * f.cut_k.pieces, slots);  // (a key head's pieces as heads of their own)
  if (!place.valid) return;
  const uint32_t head_k = place.head / f.cut_k.pieces, piece = place.head % f.cut_k.pieces, group = s.heads_q / s.heads_kv;
  if (AGAIN && !f.again[blockIdx.x]) return;  // (not written where there is nothing to sum)
  const Keys geometry(s, BN, slots, place.slot);
  if (!geometry.valid) return;
  const Span &keys = geometry.keys, &queries = geometry.queries;
  const int lq = geometry.lq, lk = geometry.lk, shift = geometry.shift;
  const uint32_t tile0 = geometry.tile0, tiles = geometry.tiles, all = tiles * group, pieces = f.cut_k.count(all), each = f.cut_k.each(all);
  const uint32_t begin = piece * each, end = min(begin + each, all);
  if ((piece || AGAIN) && begin >= end) return;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int key0 = (int)(geometry.t.row + wave * 32), key[2] = {key0 + (int)(lane & 15u), key0 + 16 + (int)(lane & 15u)};
  const bool there[2] = {key[0] < lk, key[1] < lk};
  const uint32_t base = lds_address(lds), rows_base = lds_address(&rows_lds[0][0][0]);
  const Fetch<DP, QT, NW> q_rows(row_source(f.a.q, 0, 0, 0, s.dim), wave), d_rows(row_source(f.a.dout, 0, 0, 0, s.dim), wave);
  const auto fetch = [&](uint32_t n, uint32_t parity) {
    const uint32_t head = head_k * group + n / tiles, row = (tile0 + n % tiles) * QT, to = base + parity * STAGE;
    q_rows(row_source(f.a.q, queries.first, queries.rows, head, s.dim), row, to, wave);
    d_rows(row_source(f.a.dout, queries.first, queries.rows, head, s.dim), row, to + TILE, wave);
    if (wave < 2) {  // (zeros behind the last row, as of q and do)
      const float* const from = (wave ? f.delta : f.lse2) + (size_t)head * s.rows_q + queries.first + row;
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, (int)(4 * min(queries.rows - row, QT)), 0x00020000);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                   : : "s"(rows_base + (parity * 2 + wave) * QT * 4), "v"(lane * 4), "s"(rsrc) : "memory");
    }
  };
  if (begin < end) fetch(begin, 0);
  const size_t out[2] = {(size_t)keys.first + (there[0] ? key[0] : 0), (size_t)keys.first + (there[1] ? key[1] : 0)};
  v8bf k[2][DP / 32], v[2][DP / 32];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    load_operand<DP>(k[j], f.a.k, out[j], head_k, s.dim, there[j]);
    load_operand<DP>(v[j], f.a.v, out[j], head_k, s.dim, there[j]);
  }
  const Reader<DP> at;
  Sums<DP> dk, dv;
  dk.clear();
  dv.clear();
  const float c = s.scale * LOG2E;


  const auto tile = [&](uint32_t n, auto stage) __attribute__((always_inline)) {  // (its places in LDS are constants)
    landed_everywhere();
    if (n + 1 < end) fetch(n + 1, 1 - stage.value);
    const uint8_t* const ql = lds + stage.value * STAGE;
    const uint8_t* const dl = ql + TILE;
    const float* const rl = rows_lds[stage.value][0];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int row0 = (int)((tile0 + n % tiles) * QT) + 32 * x;
      if (row0 >= lq) return;
      if (s.causal && row0 + 31 + shift <= key0) continue;
      Block p = product(at, ql, x, k), dp = product(at, dl, x, v);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const v4f lse2 = *reinterpret_cast<const v4f*>(rl + 32 * x + 16 * i + 4 * g);
        const v4f delta = *reinterpret_cast<const v4f*>(rl + QT + 32 * x + 16 * i + 4 * g);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p.t[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p.t[i][j][r], c, -lse2[r]));
            dp.t[i][j][r] = p.t[i][j][r] * (dp.t[i][j][r] - delta[r]);
          }
      }
      if (max(s.causal ? key0 + 32 - row0 - shift : 0, row0 + 32 - lq) > 0) {  // (rows behind the last are zeros, of which an infinite key makes NaN)
        const int at_lane = (int)worked_out(lane), at_row = row0 + 4 * (at_lane >> 4), end = lq - at_row;  // rows [from, end) see a column's key
        int from[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) from[j] = min(end, s.causal ? max(0, key0 + 16 * j + (at_lane & 15) - shift - at_row + 1) : 0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool seen = (uint32_t)(16 * i + r - from[j]) < (uint32_t)(end - from[j]);
              p.t[i][j][r] = seen ? p.t[i][j][r] : 0.0f;
              dp.t[i][j][r] = seen ? dp.t[i][j][r] : 0.0f;
            }
      }
      const v8bf wp[2] = {operand_of(p, 0), operand_of(p, 1)}, ws[2] = {operand_of(dp, 0), operand_of(dp, 1)};
      if (stage.again) {
        add_finite(dv, at, dl, x, wp);
        add_finite(dk, at, ql, x, ws);  // (keys that a row which is not finite is not hidden from have NaN for weights)
      } else {
        __builtin_amdgcn_sched_barrier(0);
        dv.add(at, dl, x, wp);
        dk.add(at, ql, x, ws);
        reads_ahead<DP>();
      }
    }
  };
  if (!AGAIN) {
    for (uint32_t n = begin; n < end; n += 2) {
      tile(n, Stage<false>{0});
      if (n + 1 < end) tile(n + 1, Stage<false>{1});
    }
    if (APART) {  // (the sums are in accumulation registers already, and read from there as they are asked for; else registers are spilled)
#pragma unroll
      for (int d = 0; d < DP / 16; ++d)
#pragma unroll
        for (int j = 0; j < 2; ++j) asm volatile("" : "+a"(dk.t[d][j]), "+a"(dv.t[d][j]));
    }
  }
  const bool again = AGAIN || __syncthreads_or(!finite(dk) || !finite(dv));
  if (!AGAIN && APART) {
    if (threadIdx.x == 0 && begin < end) f.again[blockIdx.x] = again;
  } else if (again) {
    if (!AGAIN) {
      dk.clear();
      dv.clear();
      fetch(begin, 0);
    }
#pragma unroll 1
    for (uint32_t n = begin; n < end; ++n) tile(n, Stage<true>{(n - begin) & 1u});
    for (uint32_t n = begin; n < end; ++n)
      for (int x = 0; x < 2; ++x) {
        const int row0 = (int)((tile0 + n % tiles) * QT) + 32 * x;
        for (int row = row0; row < min(row0 + 32, lq); ++row)
          add_rest(dv, f.a.dout, (size_t)queries.first + row, head_k * group + n / tiles, s.dim, !s.causal || key[0] < row + shift, !s.causal || key[1] < row + shift);
      }
  }
  if (pieces == 1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      store_column<DP>(dk, j, s.scale, f.a.dk, out[j], head_k, s.dim, there[j]);
      store_column<DP>(dv, j, 1.0f, f.a.dv, out[j], head_k, s.dim, there[j]);
    }
  } else {  // in the sums' own order, 64 lanes' values side by side
    float* const to = f.partial_k + ((((size_t)place.slot * s.heads_kv + head_k) * f.cut_k.pieces + piece) * NW + wave) * (DP * 64) + lane * 4;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        *reinterpret_cast<v4f*>(to + (2 * d + j) * 256) = dk.t[d][j];
        *reinterpret_cast<v4f*>(to + (DP / 8 + 2 * d + j) * 256) = dv.t[d][j];
      }
  }
}

// The pieces' sums, one after the other.
template <int DP, int NW>
__global__ __launch_bounds__(NW * 64) void attention_dkv_join_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BN = NW * 32;
  const AttentionShape& s = f.a.shape;
  const uint32_t head_k = blockIdx.x % s.heads_kv, slot = blockIdx.x / s.heads_kv, lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
  const Keys geometry(s, BN, slots, slot);
  if (!geometry.valid) return;
  const Tile& t = geometry.t;
  const Span& keys = geometry.keys;
  const uint32_t pieces = f.cut_k.count(geometry.tiles * (s.heads_q / s.heads_kv));
  if (pieces == 1 || t.row + wave * 32 >= keys.rows) return;
  const uint32_t of_v = blockIdx.y / (DP / 32), d = 2 * (blockIdx.y % (DP / 32));  // dk or dv, of it values 16 d ..
  const float* const from = f.partial_k + (((size_t)slot * s.heads_kv + head_k) * f.cut_k.pieces * NW + wave) * (DP * 64) + of_v * (DP * 32) + 2 * d * 256 + lane * 4;
  v4f v[4] = {}, part[MOST_PIECES][4];
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[p][i] = *reinterpret_cast<const v4f*>(from + (p < pieces ? p : 0) * (size_t)(NW * DP * 64) + i * 256);
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p < pieces) v[i] += part[p][i];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t key = t.row + wave * 32 + 16 * j + (lane & 15u);
    const bool there = key < keys.rows;
    store_values(v[j], v[2 + j], d, of_v ? 1.0f : s.scale, of_v ? f.a.dv : f.a.dk, (size_t)keys.first + (there ? key : 0), head_k, s.dim, there);
  }
}

constexpr int NW = 4;  // waves of a workgroup, 32 columns each
Cut cut_q(const AttentionShape& s) {
  return cut_of(s, slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32), s.dim <= 64 ? 1024 : 512);
}
Cut cut_k(const AttentionShape& s) {
  // All tiles alike, so that some thousand workgroups share the work; where a group has as many heads as there are pieces, each is about one head's, whose
  // rows stay in its XCD's L2 (8192 rows, 16 heads of 128 over 4, forward and backward: cut by a tile's length 1331 us and more, so 1280).
  const size_t wgs = std::max<size_t>(1, (size_t)slots_of(s.offsets_k, s.rows_k, s.sequences, NW * 32) * s.heads_kv);
  return {(uint32_t)std::max<size_t>(1, std::min<size_t>(MOST_PIECES, 1024 / wgs)), 1};
}
struct Layout {
  size_t rows, again, partial_q, partial_k, floats;
};
Layout layout(const AttentionShape& s, const Cut& q, const Cut& k) {
  const size_t dp = s.dim <= 64 ? 64 : 128;
  Layout l;
  l.rows = (size_t)s.heads_q * s.rows_q;
  l.again = 2 * l.rows;
  l.partial_q = (l.again + (dp > 64 && s.rows_k ? workgroups_of(s.heads_kv * k.pieces, slots_of(s.offsets_k, s.rows_k, s.sequences, NW * 32)) : 0) + 3) / 4 * 4;
  l.partial_k = l.partial_q + (q.pieces > 1 ? (q.pieces * l.rows * (2 * dp + 2) + 3) / 4 * 4 : 0);
  l.floats = l.partial_k + (k.pieces > 1 ? (size_t)k.pieces * slots_of(s.offsets_k, s.rows_k, s.sequences, NW * 32) * s.heads_kv * NW * 64 * dp : 0);
  return l;
}

template <int DP>
void backward_as(const Backward& f, hipStream_t stream) {
  const AttentionShape& s = f.a.shape;
  if (s.rows_q) {
    const uint32_t slots = slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32);
    attention_dq_kernel<DP, NW><<<workgroups_of(s.heads_q, slots * f.cut_q.pieces), NW * 64, 0, stream>>>(f, slots);
    if (f.cut_q.pieces > 1) attention_dq_join_kernel<DP, NW><<<dim3(slots, s.heads_q, NW * 32 * DP / 1024), 256, 0, stream>>>(f);
  }
  if (s.rows_k) {
    const uint32_t slots = slots_of(s.offsets_k, s.rows_k, s.sequences, NW * 32);
    attention_dkv_kernel<DP, NW, false><<<workgroups_of(s.heads_kv * f.cut_k.pieces, slots), NW * 64, 0, stream>>>(f, slots);
    if constexpr (apart<DP>)
      if (s.rows_q) attention_dkv_kernel<DP, NW, true><<<workgroups_of(s.heads_kv * f.cut_k.pieces, slots), NW * 64, 0, stream>>>(f, slots);
    if (f.cut_k.pieces > 1) attention_dkv_join_kernel<DP, NW><<<dim3(slots * s.heads_kv, DP / 16), NW * 64, 0, stream>>>(f, slots);
  }
}

}  // namespace

size_t attention_backward_workspace(const AttentionShape& s) {
  return layout(s, cut_q(s), s.rows_k ? cut_k(s) : Cut{1, 1}).floats * sizeof(float);
}

hipError_t launch_attention_backward(const AttentionBackward& b, hipStream_t stream) {
  const AttentionShape& s = b.shape;
  Backward f = {};
  f.a = b;
  f.cut_q = f.cut_k = {1, 1};
  if (s.rows_q) {  // (without queries there is no workspace, and nothing to cut)
    f.cut_q = cut_q(s);
    if (s.rows_k) f.cut_k = cut_k(s);
    const Layout l = layout(s, f.cut_q, f.cut_k);
    f.lse2 = static_cast<float*>(b.workspace);
    f.delta = f.lse2 + l.rows;
    f.again = reinterpret_cast<uint32_t*>(f.lse2 + l.again);
    f.partial_q = f.lse2 + l.partial_q;
    f.partial_k = f.lse2 + l.partial_k;
  }
  if (s.dim <= 64) backward_as<64>(f, stream);
  else backward_as<128>(f, stream);
  return hipGetLastError();
}

}  // namespace srq
