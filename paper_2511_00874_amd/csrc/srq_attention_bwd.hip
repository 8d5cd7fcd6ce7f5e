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

// ---- dq ---------------------------------------------------------------------------------------------------------------------------
// As the forward pass: a wave has 32 rows, the columns of
//   S^T = K Q^T,  dP^T = V dO^T,  P = 2^(c S - lse2),  dS = P (dP - delta),  dQ^T = K^T dS^T.
// Also writes lse2 and delta, which the other kernel reads.
constexpr uint32_t KT = 64;

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_dq_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BM = NW * 32, STAGE = 2 * KT * Rows<DP>::PITCH;
  constexpr int NB = DP / 32, NS = DP / 16;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const AttentionShape& s = f.a.shape;
  const Place place = place_of(s.heads_q, slots);
  if (!place.valid) return;
  const uint32_t head = place.head, head_k = head / (s.heads_q / s.heads_kv);
  const Tile t = tile_of(s.offsets_q, s.rows_q, s.sequences, BM, slots - 1 - place.slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), col = lane & 31u, g = lane >> 5;
  const int lk = (int)keys.rows, shift = lk - (int)t.rows + 1;  // row i sees keys below i + shift
  const auto limit_of = [&](int row) { return s.causal ? min(lk, row + shift) : lk; };
  const int row0 = (int)(t.row + wave * 32), row = row0 + (int)col;
  const bool there = row < (int)t.rows;
  const int limit = limit_of(row);
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
  const size_t out = (size_t)t.first + (there ? row : 0);
  v8bf q[NS], dout[NS];
  float lse2 = SRQ_INF, delta = 0.0f;
  {
    v8bf o[NS];
    load_operand<DP>(dout, f.a.dout, out, head, s.dim, there);
    load_operand<DP>(o, f.a.o, out, head, s.dim, there);
#pragma unroll
    for (int n = 0; n < NS; ++n) delta = dot(dout[n], o[n], delta);
    delta = sum_of_halves(delta);
    if (there) {
      const float v = f.a.lse[(size_t)head * s.rows_q + out];
      lse2 = v == -SRQ_INF ? SRQ_INF : v * LOG2E;
      if (g == 0) {
        f.lse2[(size_t)head * s.rows_q + out] = lse2;
        f.delta[(size_t)head * s.rows_q + out] = delta;
      }
    }
  }
  load_operand<DP>(q, f.a.q, out, head, s.dim, there);
  const Reader<DP> at;
  v16f dq[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) dq[b] = zeros();
  const float c = s.scale * LOG2E;

  for (uint32_t kt = 0; kt < tiles; ++kt) {
    landed_everywhere();
    if (kt + 1 < tiles) fetch(kt + 1);
    const uint8_t* const kl = lds + (kt & 1u) * STAGE;
    const uint8_t* const vl = kl + KT * Rows<DP>::PITCH;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key0 = (int)(kt * KT) + 32 * i;
      if (key0 >= most) continue;
      v16f p = zeros(), dp = zeros();
#pragma unroll
      for (int n = 0; n < NS; ++n) p = mfma(at.along(kl, i, n), q[n], p);
#pragma unroll
      for (int n = 0; n < NS; ++n) dp = mfma(at.along(vl, i, n), dout[n], dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -lse2)) * (dp[r] - delta);
      if (key0 + 32 > least) {
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = key0 + row_of(r) + 4 * (int)g < limit ? p[r] : 0.0f;
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const v8bf w = operand_of(p, n);
#pragma unroll
        for (int b = 0; b < NB; ++b) dq[b] = mfma(at.across(kl, 2 * i + n, b), w, dq[b]);
      }
    }
  }
  store_column<DP>(dq, s.scale, f.a.dq, out, head, s.dim, there);
}

// ---- dk and dv ------------------------------------------------------------------------------------------------------------------------
// A workgroup has 32 NW keys of one key head, a wave 32 of them, the columns of
//   S = Q K^T,  dP = dO V^T,  dV^T = dO^T P,  dK^T = Q^T dS;
// the rows of q and do of all heads of the group go through LDS in tiles.
constexpr uint32_t QT = 64;

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP == 64 ? 2 : 1) void attention_dkv_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BN = NW * 32, TILE = QT * Rows<DP>::PITCH, STAGE = 2 * TILE;
  constexpr int NB = DP / 32, NS = DP / 16;
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
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), col = lane & 31u, g = lane >> 5;
  const int lq = (int)queries.rows, lk = (int)keys.rows, shift = lk - lq + 1;  // row i sees keys below i + shift
  const int key0 = (int)(t.row + wave * 32), key = key0 + (int)col;
  const bool there = key < lk;
  const int first = s.causal ? max(0, (int)t.row - shift + 1) : 0;  // the first row that sees the workgroup's first key
  const uint32_t tile0 = (uint32_t)first / QT, tiles = lq > first ? ((uint32_t)lq + QT - 1) / QT - tile0 : 0u;
  const uint32_t all = tiles * group, begin = (uint32_t)((uint64_t)all * piece / f.pieces), end = (uint32_t)((uint64_t)all * (piece + 1) / f.pieces);
  const uint32_t base = lds_address(lds), rows_base = lds_address(&rows_lds[0][0][0]);
  const Fetch<DP, QT, NW> q_rows(row_source(f.a.q, 0, 0, 0, s.dim), wave), d_rows(row_source(f.a.dout, 0, 0, 0, s.dim), wave);
  const auto fetch = [&](uint32_t n) {
    const uint32_t head = head_k * group + n / tiles, row = (tile0 + n % tiles) * QT, to = base + (n & 1u) * STAGE;
    q_rows(row_source(f.a.q, queries.first, queries.rows, head, s.dim), row, to, wave);
    d_rows(row_source(f.a.dout, queries.first, queries.rows, head, s.dim), row, to + TILE, wave);
    if (wave < 2) {  // (zeros behind the last row, whose q and do are zeros too: nothing comes of them)
      const float* const from = (wave ? f.delta : f.lse2) + (size_t)head * s.rows_q + queries.first + row;
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, (int)(4 * min(queries.rows - row, QT)), 0x00020000);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                   : : "s"(rows_base + ((n & 1u) * 2 + wave) * QT * 4), "v"(lane * 4), "s"(rsrc) : "memory");
    }
  };
  if (begin < end) fetch(begin);
  const size_t out = (size_t)keys.first + (there ? key : 0);
  v8bf k[NS], v[NS];
  load_operand<DP>(k, f.a.k, out, head_k, s.dim, there);
  load_operand<DP>(v, f.a.v, out, head_k, s.dim, there);
  const Reader<DP> at;
  v16f dk[NB], dv[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) dk[b] = dv[b] = zeros();
  const float c = s.scale * LOG2E;

  for (uint32_t n = begin; n < end; ++n) {
    landed_everywhere();
    if (n + 1 < end) fetch(n + 1);
    const uint8_t* const ql = lds + (n & 1u) * STAGE;
    const uint8_t* const dl = ql + TILE;
    const float* const rl = rows_lds[n & 1u][0];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row0 = (int)((tile0 + n % tiles) * QT) + 32 * i;
      if (row0 >= lq || (s.causal && row0 + 31 + shift <= key0)) continue;
      v16f p = zeros(), dp = zeros();
#pragma unroll
      for (int x = 0; x < NS; ++x) p = mfma(at.along(ql, i, x), k[x], p);
#pragma unroll
      for (int x = 0; x < NS; ++x) dp = mfma(at.along(dl, i, x), v[x], dp);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const mma::v4f lse2 = *reinterpret_cast<const mma::v4f*>(rl + 32 * i + 8 * a + 4 * g);
        const mma::v4f delta = *reinterpret_cast<const mma::v4f*>(rl + QT + 32 * i + 8 * a + 4 * g);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int r = 4 * a + b;
          p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -lse2[b]));
          dp[r] = p[r] * (dp[r] - delta[b]);
        }
      }
      if (s.causal && row0 + shift < key0 + 32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool seen = key < row0 + row_of(r) + 4 * (int)g + shift;
          p[r] = seen ? p[r] : 0.0f;
          dp[r] = seen ? dp[r] : 0.0f;
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const v8bf wp = operand_of(p, x), ws = operand_of(dp, x);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          dv[b] = mfma(at.across(dl, 2 * i + x, b), wp, dv[b]);
          dk[b] = mfma(at.across(ql, 2 * i + x, b), ws, dk[b]);
        }
      }
    }
  }
  if (f.pieces == 1) {
    store_column<DP>(dk, s.scale, f.a.dk, out, head_k, s.dim, there);
    store_column<DP>(dv, 1.0f, f.a.dv, out, head_k, s.dim, there);
  } else {  // in the sums' own order, 64 lanes' values side by side
    float* const to = f.partial + ((((size_t)place.slot * s.heads_kv + head_k) * f.pieces + piece) * NW + wave) * (2 * NB * 16 * 64) + lane * 4;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        *reinterpret_cast<mma::v4f*>(to + (b * 4 + a) * 256) = mma::v4f{dk[b][4 * a], dk[b][4 * a + 1], dk[b][4 * a + 2], dk[b][4 * a + 3]};
        *reinterpret_cast<mma::v4f*>(to + ((NB + b) * 4 + a) * 256) = mma::v4f{dv[b][4 * a], dv[b][4 * a + 1], dv[b][4 * a + 2], dv[b][4 * a + 3]};
      }
  }
}

// The pieces' sums, one after the other.
template <int DP, int NW>
__global__ __launch_bounds__(NW * 64) void attention_dkv_join_kernel(Backward f, uint32_t slots) {
  constexpr uint32_t BN = NW * 32;
  constexpr int NB = DP / 32;
  const AttentionShape& s = f.a.shape;
  const uint32_t head_k = blockIdx.x % s.heads_kv, slot = blockIdx.x / s.heads_kv, lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
  const Tile t = tile_of(s.offsets_k, s.rows_k, s.sequences, BN, slot);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t key = t.row + wave * 32 + (lane & 31u);
  const bool there = key < keys.rows;
  if (t.row + wave * 32 >= keys.rows) return;
  const float* from = f.partial + (((size_t)slot * s.heads_kv + head_k) * f.pieces * NW + wave) * (2 * NB * 16 * 64) + lane * 4;
  v16f d[2 * NB];
#pragma unroll
  for (int b = 0; b < 2 * NB; ++b) d[b] = zeros();
  for (uint32_t p = 0; p < f.pieces; ++p, from += NW * (2 * NB * 16 * 64))
#pragma unroll
    for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const mma::v4f v = *reinterpret_cast<const mma::v4f*>(from + (b * 4 + a) * 256);
#pragma unroll
        for (int j = 0; j < 4; ++j) d[b][4 * a + j] += v[j];
      }
  const size_t out = (size_t)keys.first + (there ? key : 0);
  v16f dk[NB], dv[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    dk[b] = d[b];
    dv[b] = d[NB + b];
  }
  store_column<DP>(dk, s.scale, f.a.dk, out, head_k, s.dim, there);
  store_column<DP>(dv, 1.0f, f.a.dv, out, head_k, s.dim, there);
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
    if (f.pieces > 1) attention_dkv_join_kernel<DP, NW><<<slots * s.heads_kv, NW * 64, 0, stream>>>(f, slots);
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
