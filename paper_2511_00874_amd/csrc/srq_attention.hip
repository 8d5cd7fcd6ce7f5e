// Attention, forward: one pass over the keys with a running maximum and sum.
#include <algorithm>

#include "srq_attention.hpp"

namespace srq {
namespace {
using namespace attn;
// ---- many rows --------------------------------------------------------------------------------------------------------------------
// A workgroup has 32 NW rows of one query head, a wave 32 of them, the columns of its products; tiles of 64 keys and values go through LDS, the next
// one under way while one is worked on.
//   S^T = K Q^T (keys x rows),  m' = max(m, max S),  P = 2^(c (S - m')),  l = l 2^(c (m - m')) + sum P,  O^T = O^T 2^(c (m - m')) + V^T P^T
// with c = scale log2 e.  The maximum is only moved when a score is more than 2^GROW above what it stands for: until then P stays far from overflow and
// the sums keep their precision, and O^T is not multiplied.
constexpr float GROW = 8.0f;

// The running maximum and sum of a wave's 32 columns, two a lane.
struct Softmax {
  // of column 16 j + lane % 16: the maximum, in the scores' units, c times it (0 as long as there is none), from where on it is moved; this lane's part of the sum
  float m[2] = {-SRQ_INF, -SRQ_INF}, mc[2] = {0.0f, 0.0f}, move[2] = {-SRQ_INF, -SRQ_INF}, l[2] = {0.0f, 0.0f};
  // The maximum takes in these scores; where it moves, so do the sums.
  template <int DP, int N>
  __device__ __forceinline__ void take(const Block (&p)[N], float c, Sums<DP>& o) {
    float top[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      top[j] = p[0].t[0][j][0];
#pragma unroll
      for (int r = 1; r < 8 * N; ++r) top[j] = fmaxf(top[j], p[r / 8].t[r / 4 % 2][j][r % 4]);
      top[j] = max_of_column(top[j]);
    }
    if (__any(top[0] > move[0] || top[1] > move[1])) {
      asm volatile("");  // (a branch, no selects)
      float factor[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {  // (a column by itself: its result does not hang on its neighbours)
        const float to = top[j] > move[j] ? top[j] : m[j], toc =  to == -SRQ_INF ? 0.0f : to * c;
        move[j] = to + GROW / c;
        factor[j] = __builtin_amdgcn_exp2f(m[j] * c - toc);
        m[j] = to;
        mc[j] = toc;
        l[j] *= factor[j];
      }
      o.scale(factor);
    }
  }
  // Scores to weights, as operands; times `shrink`, a power of two, if they are to be SMALL.
  template <bool SMALL>
  __device__ __forceinline__ void weights(Block& p, float c, v8bf (&w)[2], const float (&shrink)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p.t[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p.t[i][j][r], c, -mc[j]));
          l[j] += p.t[i][j][r];  // (before they are rounded: lse is good to binary32)
          if (SMALL) p.t[i][j][r] *= shrink[j];
        }
      w[j] = operand_of(p, j);
    }
  }
};
// Scores of keys that a column does not see: the block's first row, seen from its register 0, is `left` keys in front of the first of them.
__device__ __forceinline__ void hide(Block& p, const int (&left)[2], int first) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) p.t[i][j][r] = first + 16 * i + r < left[j] ? p.t[i][j][r] : -SRQ_INF;
}

// A weight is up to 2^GROW, so that the sums of many with values near the largest of the type can pass it, though their mean does not.  Then the pass
// is gone through a third time, with the weights of such columns 2^-40 as large, which changes no bit of what does not overflow.
constexpr float SHRINK = 0x1p-40f;
template <int DP>
__device__ __forceinline__ void shrink_where(const Sums<DP>& o, float (&shrink)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float zero = 0.0f;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(o.t[d][j][r], 0.0f, zero);
    shrink[j] = sum_of_column(zero) == 0.0f ? 1.0f : SHRINK;
  }
}

// What a piece of a row's keys leaves: the mean of its values, what the weights are taken from (c times the maximum) and their sum.
template <int DP>
struct Partial {
  float *means, *stats;
  __device__ __forceinline__ Partial(const AttentionForward& f, uint32_t pieces, uint32_t piece, size_t row, uint32_t head) {
    const size_t each = (size_t)f.shape.rows_q * f.shape.heads_q, at = piece * each + row * f.shape.heads_q + head;
    means = f.partial + at * DP;
    stats = f.partial + pieces * each * DP + 2 * at;
  }
};

// 16384 rows, 16 heads of 128 over 4, causal: 960 to 995 us from card to card, 1.10 to 1.14 PFLOP/s: matrix instructions in 54 % of the cycles, vector ones in
// 55 %, the clock down to 1.7 to 1.9 GHz under both.  Heads of 64 have as many exponentials for half the products: 23 sequences of up to 1999 rows, 32 heads
// over 8, 87 to 90 us, 0.63 PFLOP/s, vector instructions in 79 %.  (32 rows a wave: with 64 the sums leave no registers for the scores of a tile; the instruction of 32 x 32
// x 16 is as fast here and slower backward; scores of the next tile beside this one's products cost more vector work than they hide.)
template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_forward_kernel(AttentionForward f, uint32_t slots, Cut cut) {
  constexpr uint32_t BM = NW * 32, STAGE = 2 * KT * Rows<DP>::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const AttentionShape& s = f.shape;
  const Place place = place_of(s.heads_q, slots * cut.pieces);
  if (!place.valid) return;
  const uint32_t head = place.head, head_k = head / (s.heads_q / s.heads_kv);
  const PieceOf of(place.slot, cut.pieces);
  const uint32_t piece = of.piece;
  const Queries rows(s, BM, slots, of.slot);
  if (!rows.t.valid) return;
  const Tile& t = rows.t;
  const Span& keys = rows.keys;
  const uint32_t pieces = cut.count(rows.tiles), each = cut.each(rows.tiles);
  const uint32_t begin = piece * each, tiles = min(begin + each, rows.tiles);  // of keys: this piece's
  if (piece && begin >= tiles) return;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int row0 = (int)(t.row + wave * 32), row[2] = {row0 + (int)(lane & 15u), row0 + 16 + (int)(lane & 15u)};
  const bool there[2] = {row[0] < (int)t.rows, row[1] < (int)t.rows};
  const int most = row0 < (int)t.rows ? rows.limit_of(min(row0 + 31, (int)t.rows - 1)) : 0;  // keys that any of the wave's rows sees
  const int least = rows.limit_of(row0);

  const RowSource ks = row_source(f.k, keys.first, keys.rows, head_k, s.dim), vs = row_source(f.v, keys.first, keys.rows, head_k, s.dim);
  const uint32_t base = lds_address(lds);
  const Fetch<DP, KT, NW> k_rows(ks, wave), v_rows(vs, wave);
  const auto fetch = [&](uint32_t kt, uint32_t stage) {
    const uint32_t to = base + stage * STAGE;
    k_rows(ks, kt * KT, to, wave);
    v_rows(vs, kt * KT, to + KT * Rows<DP>::PITCH, wave);
  };
  if (begin < tiles) fetch(begin, 0);
  v8bf q[2][DP / 32];
#pragma unroll
  for (int j = 0; j < 2; ++j) load_operand<DP>(q[j], f.q, t.first + (there[j] ? row[j] : 0), head, s.dim, there[j]);
  const Reader<DP> at;
  Sums<DP> o;
  o.clear();
  const float c = s.scale * LOG2E;
  Softmax sm;
  float shrink[2] = {1.0f, 1.0f};

  const auto tile = [&](uint32_t kt, auto stage) __attribute__((always_inline)) {  // (its places in LDS are constants)
    landed_everywhere();
    if (kt + 1 < tiles) fetch(kt + 1, 1 - stage.value);
    const uint8_t* const kl = lds + stage.value * STAGE;
    const uint8_t* const vl = kl + KT * Rows<DP>::PITCH;
    const int key0 = (int)(kt * KT);
    if (key0 >= most) return;
    Block p[2] = {product(at, kl, 0, q), product(at, kl, 1, q)};
    if (key0 + (int)KT > least) {  // some of the wave's rows do not see all of it
      asm volatile("");  // (a branch, no selects)
      const int left[2] = {rows.limit_of(row[0]) - key0 - 4 * (int)g, rows.limit_of(row[1]) - key0 - 4 * (int)g};
      hide(p[0], left, 0);
      hide(p[1], left, 32);
    }
    sm.take(p, c, o);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      v8bf w[2];
      sm.template weights<stage.again>(p[n], c, w, shrink);
      if (stage.again) add_finite(o, at, vl, n, w);
      else o.add(at, vl, n, w);
    }
  };
  for (uint32_t kt = begin; kt < tiles; kt += 2) {
    tile(kt, Stage<false>{0});
    if (kt + 1 < tiles) tile(kt + 1, Stage<false>{1});
  }
  if (__syncthreads_or(!finite(o))) {
    const auto again = [&]() __attribute__((always_inline)) {
      o.clear();
      sm = Softmax();
      fetch(begin, 0);
#pragma unroll 1
      for (uint32_t kt = begin; kt < tiles; ++kt) tile(kt, Stage<true>{(kt - begin) & 1u});
    };
    again();
    if (__syncthreads_or(!finite(o))) {
      shrink_where(o, shrink);
      again();
    }
    for (int key = (int)(begin * KT); key < min(most, (int)(tiles * KT)); ++key)
      add_rest(o, f.v, (size_t)keys.first + key, head_k, s.dim, key < rows.limit_of(row[0]), key < rows.limit_of(row[1]));
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float l = sum_of_column(sm.l[j]), inv = l == 0.0f ? 0.0f : 1.0f / l * (1.0f / shrink[j]);
    const size_t out = (size_t)t.first + (there[j] ? row[j] : 0);
    if (pieces > 1) {
      const Partial<DP> part(f, cut.pieces, piece, out, head);
      if (!there[j]) continue;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) *reinterpret_cast<v4f*>(part.means + 16 * d + 4 * g) = o.t[d][j] * inv;
      if (g == 0) part.stats[0] = sm.m[j] == -SRQ_INF ? -SRQ_INF : sm.mc[j], part.stats[1] = l;
      continue;
    }
    store_column<DP>(o, j, inv, f.o, out, head, s.dim, there[j]);
    if (there[j] && g == 0) f.lse[(size_t)head * s.rows_q + out] = l == 0.0f ? -SRQ_INF : (sm.mc[j] + __builtin_amdgcn_logf(l)) * LN2;
  }
}

// The pieces of a row: DP / 4 threads with four values each.
template <int DP>
__device__ __forceinline__ void join_row(const AttentionForward& f, uint32_t most, uint32_t pieces, size_t row, uint32_t head, uint32_t d) {
  float top = -SRQ_INF, l = 0.0f, from[MOST_PIECES], sum[MOST_PIECES];
  v4f part[MOST_PIECES], v = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p) {  // (all loads under way together)
    const Partial<DP> x(f, most, p < pieces ? p : 0, row, head);
    from[p] = x.stats[0];
    sum[p] = x.stats[1];
    part[p] = *reinterpret_cast<const v4f*>(x.means + d);
  }
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p) top = fmaxf(top, from[p]);
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p) {
    sum[p] *= p >= pieces ? 0.0f : top == -SRQ_INF ? 1.0f : __builtin_amdgcn_exp2f(from[p] - top);
    if (p < pieces) l += sum[p];
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (uint32_t p = 0; p < MOST_PIECES; ++p)
    if (p < pieces) v += part[p] * (sum[p] * inv);
  if (d < f.shape.dim) *reinterpret_cast<v2u*>(f.o.p + row * f.o.row + (size_t)head * f.o.head + d) = v2u{pack(v[0], v[1]), pack(v[2], v[3])};
  if (d == 0) f.lse[(size_t)head * f.shape.rows_q + row] = l == 0.0f ? -SRQ_INF : (top + __builtin_amdgcn_logf(l)) * LN2;
}
template <int DP, int NW>
__global__ __launch_bounds__(256) void attention_forward_join_kernel(AttentionForward f, Cut cut) {
  constexpr uint32_t T = DP / 4, BM = NW * 32;
  const Queries rows(f.shape, BM, gridDim.x, blockIdx.x);
  if (!rows.t.valid) return;
  const uint32_t pieces = cut.count(rows.tiles);
  if (pieces == 1) return;
  const uint32_t row = rows.t.row + blockIdx.z * (256 / T) + threadIdx.x / T;
  if (row < rows.t.rows) join_row<DP>(f, cut.pieces, pieces, (size_t)rows.t.first + row, blockIdx.y, 4 * (threadIdx.x % T));
}

// ---- few rows ---------------------------------------------------------------------------------------------------------------------
// Single tokens, and up to some: memory-bound, so the heads that share a key head share the columns of one wave's products, and the keys of a sequence
// are cut into chunks, a workgroup each, whose waves take tiles of 32 keys in turn, each by itself: a wave's loads run ahead of it through its own two
// stages in LDS, with no barrier before the end.  The waves' results meet in LDS, the chunks' in a second launch.  24 caches of up to 32768, 16 heads of 128
// over 4, one row each: 68 us, 4.9 TB/s (equal ones 5.6), and 9 the second launch.  (Workgroups of one wave or four, chunks from 512 on: slower.)
struct Few {
  AttentionForward a;
  uint32_t slots, waves;           // of a workgroup
  uint32_t splits, chunk;          // chunks a sequence has at most, and keys of one at least
  uint32_t per, parts, rows;       // heads a column set takes of a group; sets of a group; rows of a tile
};
constexpr uint32_t FT = 32;
template <int DP>
constexpr uint32_t MOST_WAVES = DP == 64 ? 8 : 4;  // whose stages a CU holds
// Keys of a chunk of a sequence with lk: whole turns of the waves, so many that `splits` chunks hold all.
__device__ __forceinline__ uint32_t chunk_of(const Few& f, uint32_t lk) {
  const uint32_t turn = FT * f.waves, least = ((lk + f.splits - 1) / f.splits + turn - 1) / turn * turn;
  return max(f.chunk, least);
}

template <int DP, uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void attention_few_kernel(Few f) {
  constexpr uint32_t STAGE = 2 * FT * Rows<DP>::PITCH, OWN = 2 * STAGE;
  constexpr int ND = DP / 16, LOADS = 2 * FT / Rows<DP>::PER_LOAD;
  static_assert(OWN >= ND * 8 * 64 * 4, "the waves' sums in place of the tiles");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[WAVES * OWN];
  __shared__ float stats[2][WAVES][32];
  const AttentionShape& s = f.a.shape;
  // Neighbours take the heads of the same rows, which lie side by side in memory; then come the other sequences, and then their next chunks, which not all
  // have.  Workgroups go to the eight XCDs in turn: from chunk to chunk the list moves on by one, so that a long sequence's do not all meet on one.
  const uint32_t sets = s.heads_kv * f.parts, turn = sets * f.slots, split = blockIdx.x / turn;
  const uint32_t at_turn = (blockIdx.x - split * turn + (turn & 1u ? 0u : split)) % turn, set = at_turn % sets, slot = at_turn / sets;
  const uint32_t head_k = set / f.parts, group = s.heads_q / s.heads_kv, in_group = set % f.parts * f.per;
  const Tile t = tile_of(s.offsets_q, s.rows_q, s.sequences, f.rows, slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t chunk = chunk_of(f, keys.rows);
  if (split && split * chunk >= keys.rows) return;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int lk = (int)keys.rows, shift = lk - (int)t.rows + 1;  // row i sees keys below i + shift
  const auto limit_of = [&](int r) { return s.causal ? min(lk, r + shift) : lk; };
  uint32_t row[2], head[2];
  bool there[2];
  int limit[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t col = 16 * j + (lane & 15u), head_at = in_group + col % f.per;
    row[j] = t.row + col / f.per;
    there[j] = col / f.per < f.rows && row[j] < t.rows && head_at < group;
    row[j] = there[j] ? row[j] : 0;
    head[j] = there[j] ? head_k * group + head_at : 0;
    limit[j] = there[j] ? limit_of((int)row[j]) : 0;
  }
  const int end = min(limit_of((int)min(t.row + f.rows, t.rows) - 1), (int)((split + 1) * chunk));
  const int least = limit_of((int)t.row);
  const uint32_t begin = split * chunk + wave * FT;
  const uint32_t tiles = end > (int)begin ? ((uint32_t)end - begin + FT * WAVES - 1) / (FT * WAVES) : 0u;

  const RowSource ks = row_source(f.a.k, keys.first, keys.rows, head_k, s.dim), vs = row_source(f.a.v, keys.first, keys.rows, head_k, s.dim);
  const uint32_t base = lds_address(lds) + wave * OWN;
  const Fetch<DP, FT, 1> k_rows(ks, 0), v_rows(vs, 0);
  const auto fetch = [&](uint32_t n) {
    const uint32_t to = base + (n & 1u) * STAGE, from = begin + n * FT * WAVES;
    k_rows(ks, from, to, 0);
    v_rows(vs, from, to + FT * Rows<DP>::PITCH, 0);
  };
  if (tiles) fetch(0);
  v8bf q[2][DP / 32];
#pragma unroll
  for (int j = 0; j < 2; ++j) load_operand<DP>(q[j], f.a.q, (size_t)t.first + row[j], head[j], s.dim, there[j]);
  wait_vmcnt<0>();
  if (tiles > 1) fetch(1);
  const Reader<DP> at;
  Sums<DP> o;
  o.clear();
  const float c = s.scale * LOG2E;
  Softmax sm;
  float shrink[2] = {1.0f, 1.0f};
  const auto tile = [&](uint32_t n, auto stage) __attribute__((always_inline)) {
    if (n + 1 < tiles) wait_vmcnt<LOADS>();
    else wait_vmcnt<0>();
    const uint8_t* const kl = lds + wave * OWN + stage.value * STAGE;
    const uint8_t* const vl = kl + FT * Rows<DP>::PITCH;
    const int key0 = (int)(begin + n * FT * WAVES);
    Block p[1] = {product(at, kl, 0, q)};
    if (key0 + (int)FT > least) {
      const int left[2] = {limit[0] - key0 - 4 * (int)g, limit[1] - key0 - 4 * (int)g};
      hide(p[0], left, 0);
    }
    sm.take(p, c, o);
    v8bf w[2];
    sm.template weights<stage.again>(p[0], c, w, shrink);
    if (stage.again) add_finite(o, at, vl, 0, w);
    else o.add(at, vl, 0, w);
    wait_lds();  // the stage has been read
    if (n + 2 < tiles) fetch(n + 2);
  };
  for (uint32_t n = 0; n < tiles; ++n) tile(n, Stage<false>{n & 1u});
  if (__any(!finite(o))) {
    const auto again = [&]() __attribute__((always_inline)) {
      o.clear();
      sm = Softmax();
      fetch(0);
      if (tiles > 1) fetch(1);
#pragma unroll 1
      for (uint32_t n = 0; n < tiles; ++n) tile(n, Stage<true>{n & 1u});
    };
    again();
    if (__any(!finite(o))) {
      shrink_where(o, shrink);
      again();
    }
    for (uint32_t n = 0; n < tiles; ++n) {
      const int key0 = (int)(begin + n * FT * WAVES);
      for (int key = key0; key < min(key0 + (int)FT, end); ++key)
        add_rest(o, f.a.v, (size_t)keys.first + key, head_k, s.dim, key < limit[0], key < limit[1]);
    }
  }
  // the waves' means, in place of their tiles: wave w puts together every WAVES-th sixteen values
  __syncthreads();
  float* const means = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float l = sum_of_column(sm.l[j]), inv = l == 0.0f ? 0.0f : 1.0f / l * (1.0f / shrink[j]);
#pragma unroll
    for (int d = 0; d < ND; ++d) *reinterpret_cast<v4f*>(means + (((wave * ND + d) * 2 + j) * 64 + lane) * 4) = o.t[d][j] * inv;
    if (g == 0) {
      stats[0][wave][16 * j + lane] = sm.m[j] == -SRQ_INF ? -SRQ_INF : sm.mc[j];
      stats[1][wave][16 * j + lane] = l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t col = 16 * j + (lane & 15u);
    float top = stats[0][0][col], factor[WAVES], l = 0.0f;
#pragma unroll
    for (uint32_t w = 1; w < WAVES; ++w) top = fmaxf(top, stats[0][w][col]);
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) {
      factor[w] = stats[1][w][col] * (top == -SRQ_INF ? 1.0f : __builtin_amdgcn_exp2f(stats[0][w][col] - top));
      l += factor[w];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) factor[w] *= inv;
    if (!there[j]) continue;
    const size_t out = (size_t)t.first + row[j], at_part = ((size_t)split * s.rows_q + out) * s.heads_q + head[j];
    const bool whole = f.splits == 1;
#pragma unroll
    for (uint32_t d0 = 0; d0 < ND; d0 += WAVES) {
      if (d0 + wave >= ND) continue;
      v4f v = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t w = 0; w < WAVES; ++w) v += *reinterpret_cast<const v4f*>(means + (((w * ND + d0 + wave) * 2 + j) * 64 + lane) * 4) * factor[w];
      const uint32_t d = 16 * (d0 + wave) + 4 * g;
      if (d >= s.dim) continue;
      if (whole) *reinterpret_cast<v2u*>(f.a.o.p + out * f.a.o.row + (size_t)head[j] * f.a.o.head + d) = v2u{pack(v[0], v[1]), pack(v[2], v[3])};
      else *reinterpret_cast<v4f*>(f.a.partial + at_part * DP + d) = v;
    }
    if (wave == 0 && g == 0) {
      if (whole) {
        f.a.lse[(size_t)head[j] * s.rows_q + out] = l == 0.0f ? -SRQ_INF : (top + __builtin_amdgcn_logf(l)) * LN2;
      } else {
        float* const st = f.a.partial + (size_t)f.splits * s.rows_q * s.heads_q * DP + 2 * at_part;
        st[0] = top;
        st[1] = l;
      }
    }
  }
}

// The chunks of a row and head, up to 64 of them, a wave's work: a lane has a chunk's maximum and sum, then four values of every chunk of its lanes' turn.
constexpr uint32_t MOST_SPLITS = 64;
template <int DP>
__global__ __launch_bounds__(256) void attention_join_kernel(Few f) {
  constexpr uint32_t T = DP / 4, TURNS = 64 / T;
  const AttentionShape& s = f.a.shape;
  const uint32_t across = (s.heads_q + 3) / 4, lane = threadIdx.x & 63u, head = uniform(blockIdx.x % across * 4 + (threadIdx.x >> 6));
  const Tile t = tile_of(s.offsets_q, s.rows_q, s.sequences, f.rows, blockIdx.x / across);
  if (!t.valid || head >= s.heads_q) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t chunk = chunk_of(f, keys.rows), chunks = max(1u, (keys.rows + chunk - 1) / chunk), d = 4 * (lane % T), turn = lane / T;
  const float* const stats = f.a.partial + (size_t)f.splits * s.rows_q * s.heads_q * DP;
  const size_t step = (size_t)s.rows_q * s.heads_q;
  for (uint32_t row = t.row; row < min(t.row + f.rows, t.rows); ++row) {
    const size_t out = (size_t)t.first + row, at = out * s.heads_q + head;
    float own = -SRQ_INF, l = 0.0f;
    if (lane < chunks) {
      own = stats[2 * (at + lane * step)];
      l = stats[2 * (at + lane * step) + 1];
    }
    float top = own;
#pragma unroll
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    float factor = l * (top == -SRQ_INF ? 1.0f : __builtin_amdgcn_exp2f(own - top));
    l = factor;
#pragma unroll
    for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
    factor *= l == 0.0f ? 0.0f : 1.0f / l;
    v4f v = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t k0 = 0; k0 < chunks; k0 += TURNS) {
      const uint32_t k = k0 + turn;
      const float w = __shfl(factor, (int)(k & 63u));
      if (k < chunks && d < s.dim) v += w * *reinterpret_cast<const v4f*>(f.a.partial + (at + k * step) * DP + d);
    }
#pragma unroll
    for (uint32_t x = T; x < 64; x <<= 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], (int)x);
    if (d < s.dim && turn == 0)
      *reinterpret_cast<v2u*>(f.a.o.p + out * f.a.o.row + (size_t)head * f.a.o.head + d) = v2u{pack(v[0], v[1]), pack(v[2], v[3])};
    if (lane == 0) f.a.lse[(size_t)head * s.rows_q + out] = l == 0.0f ? -SRQ_INF : (top + __builtin_amdgcn_logf(l)) * LN2;
  }
}

// Which form, and how the keys are cut: few rows where those of a sequence and group fill two sets of columns at most.
bool few_rows(const AttentionShape& s) {
  return (size_t)s.rows_q * (s.heads_q / s.heads_kv) <= (size_t)64 * s.sequences;
}
Few few_of(const AttentionShape& s) {
  Few f = {};
  f.a.shape = s;
  const uint32_t group = s.heads_q / s.heads_kv;
  f.parts = (group + 31) / 32;
  f.per = (group + f.parts - 1) / f.parts;
  f.rows = 32 / f.per;
  f.slots = slots_of(s.offsets_q, s.rows_q, s.sequences, f.rows);
  // Chunks: of 1024 keys, or fewer where that leaves the chip to less than a thousand workgroups.  Where the sequences' lengths are not known here, one
  // is taken to have up to four times its share; what a chunk holds at last is settled where they are known.
  const size_t share = s.rows_k / s.sequences, most = s.offsets_k ? std::min<size_t>(s.rows_k, 4 * share + 1024) : share;
  const size_t sets = std::max<size_t>(1, (size_t)f.slots * s.heads_kv * f.parts);
  f.waves = 2;
  f.chunk = 1024;
  while (f.chunk > 128 && sets * ((most + f.chunk - 1) / f.chunk) < 1024) f.chunk /= 2;
  f.splits = (uint32_t)std::max<size_t>(1, std::min<size_t>(std::min<size_t>(MOST_SPLITS, 65536 / sets), (most + f.chunk - 1) / f.chunk));
  // Up to four tiles a wave of the largest workgroup, a CU's whole, are not cut where all workgroups run in two turns: 4 caches of 1024, 12 heads of 64 from
  // Python 15.2 us, so 18.0 with the second launch (40 of them 15.7 and 18.2; 80, in four turns, 23.6 and 19.4).
  const uint32_t waves = s.dim <= 64 ? MOST_WAVES<64> : MOST_WAVES<128>;
  if (f.splits > 1 && most <= 4 * FT * waves && sets <= 512) f.waves = waves, f.splits = 1;
  return f;
}

template <int DP>
void few_as(const AttentionForward& a, hipStream_t stream) {
  Few f = few_of(a.shape);
  f.a = a;
  const AttentionShape& s = a.shape;
  const uint32_t wgs = f.slots * s.heads_kv * f.parts * f.splits;
  if (f.waves == 2) attention_few_kernel<DP, 2><<<wgs, 128, 0, stream>>>(f);
  else attention_few_kernel<DP, MOST_WAVES<DP>><<<wgs, 64 * MOST_WAVES<DP>, 0, stream>>>(f);
  if (f.splits > 1) attention_join_kernel<DP><<<f.slots * ((s.heads_q + 3) / 4), 256, 0, stream>>>(f);
}

constexpr int NW = 4;  // waves of a workgroup, 32 rows each
// (two workgroups a CU with heads of up to 128 values, four of up to 64)
Cut forward_cut(const AttentionShape& s) {
  return cut_of(s, slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32), s.dim <= 64 ? 1024 : 512);
}

template <int DP>
void forward_as(const AttentionForward& f, hipStream_t stream) {
  const AttentionShape& s = f.shape;
  if (few_rows(s)) return few_as<DP>(f, stream);
  const uint32_t slots = slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32);
  const Cut cut = forward_cut(s);
  attention_forward_kernel<DP, NW><<<workgroups_of(s.heads_q, slots * cut.pieces), NW * 64, 0, stream>>>(f, slots, cut);
  if (cut.pieces > 1) attention_forward_join_kernel<DP, NW><<<dim3(slots, s.heads_q, NW * 32 * DP / 1024), 256, 0, stream>>>(f, cut);
}

}  // namespace

size_t attention_forward_workspace(const AttentionShape& s) {
  const size_t pieces = few_rows(s) ? few_of(s).splits : forward_cut(s).pieces;
  return pieces > 1 ? pieces * s.rows_q * s.heads_q * ((s.dim <= 64 ? 64 : 128) + 2) * sizeof(float) : 0;
}

hipError_t launch_attention_forward(const AttentionForward& f, hipStream_t stream) {
  if (f.shape.dim <= 64) forward_as<64>(f, stream);
  else forward_as<128>(f, stream);
  return hipGetLastError();
}

}  // namespace srq
