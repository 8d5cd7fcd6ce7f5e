// Attention, backward: the scores are computed again from q, k and lse, once for dq and once for dk and dv, so that every sum has one owner and one
// order.
#include <algorithm>

#include "srq_attention.hpp"

namespace srq {
namespace {
using namespace attn;

struct Backward {
  AttentionBackward a;
  uint32_t pieces;   // that the rows of a tile of keys are cut into
  float* partial;    // their sums of dk and dv, where there are several
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

// Zeros where a register's row, counted from the lane's first, is not below `left`.
__device__ __forceinline__ void clear_unseen(Block& p, const int (&left)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) p.t[i][j][r] = 16 * i + r < left[j] ? p.t[i][j][r] : 0.0f;
}

// ---- dq ---------------------------------------------------------------------------------------------------------------------------
// As the forward pass: a wave has 32 rows, the columns of
//   S^T = K Q^T,  dP^T = V dO^T,  P = 2^(c S - lse2),  dS = P (dP - delta),  dQ^T = K^T dS^T.
// Also writes lse2 and delta, which the other kernel reads.
constexpr uint32_t KT = 64;

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_dq_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BM = NW * 32, STAGE = 2 * KT * Rows<DP>::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const AttentionShape& s = f.a.shape;
  const Place place = place_of(s.heads_q, slots);
  if (!place.valid) return;
  const uint32_t head = place.head, head_k = head / (s.heads_q / s.heads_kv);
  const Tile t = tile_of(s.offsets_q, s.rows_q, s.sequences, BM, slots - 1 - place.slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int lk = (int)keys.rows, shift = lk - (int)t.rows + 1;  // row i sees keys below i + shift
  const auto limit_of = [&](int row) { return s.causal ? min(lk, row + shift) : lk; };
  const int row0 = (int)(t.row + wave * 32), row[2] = {row0 + (int)(lane & 15u), row0 + 16 + (int)(lane & 15u)};
  const bool there[2] = {row[0] < (int)t.rows, row[1] < (int)t.rows};
  const int most = row0 < (int)t.rows ? limit_of(min(row0 + 31, (int)t.rows - 1)) : 0;
  const int least = limit_of(row0);
  const int end = limit_of(min((int)(t.row + BM), (int)t.rows) - 1);
  const uint32_t tiles = end > 0 ? ((uint32_t)end + KT - 1) / KT : 0u;

  const RowSource ks = row_source(f.a.k, keys.first, keys.rows, head_k, s.dim), vs = row_source(f.a.v, keys.first, keys.rows, head_k, s.dim);
  const uint32_t base = lds_address(lds);
  const Fetch<DP, KT, NW> k_rows(ks, wave), v_rows(vs, wave);
  const auto fetch = [&](uint32_t kt) {
    const uint32_t to = base + (kt & 1u) * STAGE;
    k_rows(ks, kt * KT, to, wave);
    v_rows(vs, kt * KT, to + KT * Rows<DP>::PITCH, wave);
  };
  if (tiles) fetch(0);
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
      if (g == 0) {
        f.lse2[(size_t)head * s.rows_q + out[j]] = lse2[j];
        f.delta[(size_t)head * s.rows_q + out[j]] = delta[j];
      }
    }
  }
  const Reader<DP> at;
  Sums<DP> dq;
  dq.clear();
  const float c = s.scale * LOG2E;

  const auto tile = [&](uint32_t kt, auto parity) {  // (its places in LDS are constants)
    landed_everywhere();
    if (kt + 1 < tiles) fetch(kt + 1);
    const uint8_t* const kl = lds + parity.value * STAGE;
    const uint8_t* const vl = kl + KT * Rows<DP>::PITCH;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int key0 = (int)(kt * KT) + 32 * n;
      if (key0 >= most) return;
      Block p = product(at, kl, n, q);
      const Block dp = product(at, vl, n, dout);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            p.t[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p.t[i][j][r], c, -lse2[j])) * (dp.t[i][j][r] - delta[j]);
      if (key0 + 32 > least) {
        asm volatile("");  // (a branch, no selects)
        const int left[2] = {limit_of(row[0]) - key0 - 4 * (int)g, limit_of(row[1]) - key0 - 4 * (int)g};
        clear_unseen(p, left);
      }
      const v8bf w[2] = {operand_of(p, 0), operand_of(p, 1)};
      dq.add(at, kl, n, w);
    }
  };
  for (uint32_t kt = 0; kt < tiles; kt += 2) {
    tile(kt, std::integral_constant<uint32_t, 0>{});
    if (kt + 1 < tiles) tile(kt + 1, std::integral_constant<uint32_t, 1>{});
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) store_column<DP>(dq, j, s.scale, f.a.dq, out[j], head, s.dim, there[j]);
}

// ---- dk and dv ------------------------------------------------------------------------------------------------------------------------
// A workgroup has 32 NW keys of one key head, a wave 32 of them, the columns of
//   S = Q K^T,  dP = dO V^T,  dV^T = dO^T P,  dK^T = Q^T dS;
// the rows of q and do of all heads of the group go through LDS in tiles.
constexpr uint32_t QT = 64;

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP == 64 ? 2 : 1) void attention_dkv_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BN = NW * 32, TILE = QT * Rows<DP>::PITCH, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  __shared__ __attribute__((aligned(16))) float rows_lds[2][2][QT];  // lse2 and delta
  const AttentionShape& s = f.a.shape;
  const Place place = place_of(s.heads_kv * f.pieces, slots);  // (a key head's pieces as heads of their own)
  if (!place.valid) return;
  const uint32_t head_k = place.head / f.pieces, piece = place.head % f.pieces, group = s.heads_q / s.heads_kv;
  const Tile t = tile_of(s.offsets_k, s.rows_k, s.sequences, BN, place.slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence), queries = span_of(s.offsets_q, s.rows_q, s.sequences, t.sequence);
  if (t.row >= keys.rows) return;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = lane >> 4;
  const int lq = (int)queries.rows, lk = (int)keys.rows, shift = lk - lq + 1;  // row i sees keys below i + shift
  const int key0 = (int)(t.row + wave * 32), key[2] = {key0 + (int)(lane & 15u), key0 + 16 + (int)(lane & 15u)};
  const bool there[2] = {key[0] < lk, key[1] < lk};
  const int first = s.causal ? max(0, (int)t.row - shift + 1) : 0;  // the first row that sees the workgroup's first key
  const uint32_t tile0 = (uint32_t)first / QT, tiles = lq > first ? ((uint32_t)lq + QT - 1) / QT - tile0 : 0u;
  const uint32_t all = tiles * group, begin = (uint32_t)((uint64_t)all * piece / f.pieces), end = (uint32_t)((uint64_t)all * (piece + 1) / f.pieces);
  const uint32_t base = lds_address(lds), rows_base = lds_address(&rows_lds[0][0][0]);
  const Fetch<DP, QT, NW> q_rows(row_source(f.a.q, 0, 0, 0, s.dim), wave), d_rows(row_source(f.a.dout, 0, 0, 0, s.dim), wave);
  const auto fetch = [&](uint32_t n, uint32_t parity) {
    const uint32_t head = head_k * group + n / tiles, row = (tile0 + n % tiles) * QT, to = base + parity * STAGE;
    q_rows(row_source(f.a.q, queries.first, queries.rows, head, s.dim), row, to, wave);
    d_rows(row_source(f.a.dout, queries.first, queries.rows, head, s.dim), row, to + TILE, wave);
    if (wave < 2) {  // (zeros behind the last row, whose q and do are zeros too: nothing comes of them)
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

  const auto tile = [&](uint32_t n, auto parity) {  // (its places in LDS are constants)
    landed_everywhere();
    if (n + 1 < end) fetch(n + 1, 1 - parity.value);
    const uint8_t* const ql = lds + parity.value * STAGE;
    const uint8_t* const dl = ql + TILE;
    const float* const rl = rows_lds[parity.value][0];
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
      if (s.causal && row0 + shift < key0 + 32) {
        asm volatile("");  // (a branch, no selects)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool seen = key[j] - shift - row0 - 4 * (int)g < 16 * i + r;
              p.t[i][j][r] = seen ? p.t[i][j][r] : 0.0f;
              dp.t[i][j][r] = seen ? dp.t[i][j][r] : 0.0f;
            }
      }
      const v8bf wp[2] = {operand_of(p, 0), operand_of(p, 1)}, ws[2] = {operand_of(dp, 0), operand_of(dp, 1)};
      dv.add(at, dl, x, wp);
      dk.add(at, ql, x, ws);
    }
  };
  for (uint32_t n = begin; n < end; n += 2) {
    tile(n, std::integral_constant<uint32_t, 0>{});
    if (n + 1 < end) tile(n + 1, std::integral_constant<uint32_t, 1>{});
  }
  if (f.pieces == 1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      store_column<DP>(dk, j, s.scale, f.a.dk, out[j], head_k, s.dim, there[j]);
      store_column<DP>(dv, j, 1.0f, f.a.dv, out[j], head_k, s.dim, there[j]);
    }
  } else {  // in the sums' own order, 64 lanes' values side by side
    float* const to = f.partial + ((((size_t)place.slot * s.heads_kv + head_k) * f.pieces + piece) * NW + wave) * (DP * 64) + lane * 4;
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
  const Tile t = tile_of(s.offsets_k, s.rows_k, s.sequences, BN, slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  if (t.row + wave * 32 >= keys.rows) return;
  const uint32_t of_v = blockIdx.y;  // dk or dv
  const float* from = f.partial + (((size_t)slot * s.heads_kv + head_k) * f.pieces * NW + wave) * (DP * 64) + of_v * (DP * 32) + lane * 4;
  Sums<DP> d;
  d.clear();
  for (uint32_t p = 0; p < f.pieces; ++p, from += NW * (DP * 64))
#pragma unroll
    for (int b = 0; b < DP / 16; ++b)
#pragma unroll
      for (int j = 0; j < 2; ++j) d.t[b][j] += *reinterpret_cast<const v4f*>(from + (2 * b + j) * 256);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t key = t.row + wave * 32 + 16 * j + (lane & 15u);
    const bool there = key < keys.rows;
    store_column<DP>(d, j, of_v ? 1.0f : s.scale, of_v ? f.a.dv : f.a.dk, (size_t)keys.first + (there ? key : 0), head_k, s.dim, there);
  }
}

// Pieces that the rows of a tile of keys are cut into, so that some thousand workgroups share the work.
constexpr uint32_t KEY_TILE = 128;
uint32_t pieces_of(const AttentionShape& s) {
  const size_t wgs = std::max<size_t>(1, (size_t)slots_of(s.offsets_k, s.rows_k, s.sequences, KEY_TILE) * s.heads_kv);
  const size_t most = (size_t)s.heads_q / s.heads_kv * std::max<size_t>(1, s.rows_q / QT / s.sequences);  // of a stage at least
  return (uint32_t)std::max<size_t>(1, std::min<size_t>({8, most, 1024 / wgs}));
}
size_t partial_floats(const AttentionShape& s) {
  const size_t pieces = pieces_of(s), each = (size_t)KEY_TILE * 2 * (s.dim <= 64 ? 64 : 128);
  return pieces > 1 ? pieces * slots_of(s.offsets_k, s.rows_k, s.sequences, KEY_TILE) * s.heads_kv * each : 0;
}

template <int DP>
void backward_as(const Backward& f, hipStream_t stream) {
  constexpr int NW = 4;
  const AttentionShape& s = f.a.shape;
  if (s.rows_q) {
    const uint32_t slots = slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32);
    attention_dq_kernel<DP, NW><<<workgroups_of(s.heads_q, slots), NW * 64, 0, stream>>>(f, slots);
  }
  if (s.rows_k) {
    static_assert(NW * 32 == KEY_TILE, "tiles of keys");
    const uint32_t slots = slots_of(s.offsets_k, s.rows_k, s.sequences, KEY_TILE);
    attention_dkv_kernel<DP, NW><<<workgroups_of(s.heads_kv * f.pieces, slots), NW * 64, 0, stream>>>(f, slots);
    if (f.pieces > 1) attention_dkv_join_kernel<DP, NW><<<dim3(slots * s.heads_kv, 2), NW * 64, 0, stream>>>(f, slots);
  }
}

}  // namespace

size_t attention_backward_workspace(const AttentionShape& s) {
  return (((size_t)s.heads_q * s.rows_q * 2 + 3) / 4 * 4 + (s.rows_k ? partial_floats(s) : 0)) * sizeof(float);
}

hipError_t launch_attention_backward(const AttentionBackward& b, hipStream_t stream) {
  Backward f = {};
  f.a = b;
  const size_t rows = (size_t)b.shape.heads_q * b.shape.rows_q;
  f.lse2 = static_cast<float*>(b.workspace);
  f.delta = f.lse2 + rows;
  f.partial = f.lse2 + (2 * rows + 3) / 4 * 4;
  f.pieces = b.shape.rows_q && b.shape.rows_k ? pieces_of(b.shape) : 1;
  if (b.shape.dim <= 64) backward_as<64>(f, stream);
  else backward_as<128>(f, stream);
  return hipGetLastError();
}

}  // namespace srq
