// Attention, forward: one pass over the keys with a running maximum and sum.
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
constexpr uint32_t KT = 64;
constexpr float GROW = 8.0f;

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_forward_kernel(AttentionForward f, uint32_t slots, uint32_t total) {
  constexpr uint32_t BM = NW * 32, STAGE = 2 * KT * Rows<DP>::PITCH;
  constexpr int NB = DP / 32, NS = DP / 16;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const AttentionShape& s = f.shape;
  const uint32_t place = place_in_list(total);
  if (place >= total) return;
  const uint32_t head = place / slots, head_k = head / (s.heads_q / s.heads_kv);
  // (the last rows of a sequence see most: they begin first)
  const Tile t = tile_of<BM>(s.offsets_q, s.rows_q, s.sequences, slots - 1 - place % slots);
  if (!t.valid) return;
  const Span keys = keys_of(s, t.sequence);
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), col = lane & 31u, g = lane >> 5;
  const int lk = (int)keys.rows, shift = lk - (int)t.rows + 1;  // row i sees keys below i + shift
  const auto limit_of = [&](int row) { return s.causal ? min(lk, row + shift) : lk; };
  const int row0 = (int)(t.row + wave * 32), row = row0 + (int)col;
  const bool there = row < (int)t.rows;
  const int limit = limit_of(row);
  const int most = row0 < (int)t.rows ? limit_of(min(row0 + 31, (int)t.rows - 1)) : 0;  // keys that any of the wave's rows sees
  const int least = limit_of(row0);
  const int end = limit_of(min((int)(t.row + BM), (int)t.rows) - 1);                     // and of the workgroup's
  const uint32_t tiles = end > 0 ? ((uint32_t)end + KT - 1) / KT : 0u;

  const RowSource ks = row_source(f.k, keys.first, keys.rows, head_k, s.dim), vs = row_source(f.v, keys.first, keys.rows, head_k, s.dim);
  const uint32_t base = lds_address(lds);
  const auto fetch = [&](uint32_t kt) {
    const uint32_t to = base + (kt & 1u) * STAGE;
    fetch_rows<DP, KT, NW>(ks, kt * KT, to, wave);
    fetch_rows<DP, KT, NW>(vs, kt * KT, to + KT * Rows<DP>::PITCH, wave);
  };
  if (tiles) fetch(0);
  v8bf q[NS];
  load_operand<DP>(q, f.q, t.first + (there ? row : 0), head, s.dim, there);
  const Reader<DP> at;
  v16f o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = zeros();
  const float c = s.scale * LOG2E;
  // the maximum, in the scores' units, c times it (0 as long as there is none), and from where on it is moved; this lane's part of the sum
  float m = -SRQ_INF, mc = 0.0f, move = -SRQ_INF, l = 0.0f;

  for (uint32_t kt = 0; kt < tiles; ++kt) {
    landed_everywhere();
    if (kt + 1 < tiles) fetch(kt + 1);
    const uint8_t* const kl = lds + (kt & 1u) * STAGE;
    const uint8_t* const vl = kl + KT * Rows<DP>::PITCH;
    const int key0 = (int)(kt * KT);
    if (key0 >= most) continue;
    v16f p[2] = {zeros(), zeros()};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NS; ++n) p[i] = mfma(at.along(kl, i, n), q[n], p[i]);
    if (key0 + (int)KT > least) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[i][r] = key0 + 32 * i + row_of(r) + 4 * (int)g < limit ? p[i][r] : -SRQ_INF;
    }
    float top = p[0][0];
#pragma unroll
    for (int r = 1; r < 32; ++r) top = fmaxf(top, p[r / 16][r % 16]);
    top = max_of_halves(top);
    if (__any(top > move)) {
      const float to = fmaxf(m, top), toc = to == -SRQ_INF ? 0.0f : to * c;
      move = to + GROW / c;
      const float factor = __builtin_amdgcn_exp2f(m * c - toc);
      m = to;
      mc = toc;
      l *= factor;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= factor;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[i][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i][r], c, -mc));
        l += p[i][r];
      }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const v8bf w = operand_of(p[n / 2], n % 2);
#pragma unroll
      for (int b = 0; b < NB; ++b) o[b] = mfma(at.across(vl, n, b), w, o[b]);
    }
  }
  l = sum_of_halves(l);
  const size_t out = (size_t)t.first + (there ? row : 0);
  store_column<DP>(o, l == 0.0f ? 0.0f : 1.0f / l, f.o, out, head, s.dim, there);
  if (there && g == 0) f.lse[(size_t)head * s.rows_q + out] = l == 0.0f ? -SRQ_INF : (mc + __builtin_amdgcn_logf(l)) * LN2;
}

template <int DP>
void forward_as(const AttentionForward& f, hipStream_t stream) {
  constexpr int NW = 4;
  const AttentionShape& s = f.shape;
  const uint32_t slots = slots_of(s.offsets_q, s.rows_q, s.sequences, NW * 32), total = slots * s.heads_q;
  attention_forward_kernel<DP, NW><<<workgroups_of(total), NW * 64, 0, stream>>>(f, slots, total);
}

}  // namespace

size_t attention_forward_workspace(const AttentionShape&) { return 0; }

hipError_t launch_attention_forward(const AttentionForward& f, hipStream_t stream) {
  if (f.shape.dim <= 64) forward_as<64>(f, stream);
  else forward_as<128>(f, stream);
  return hipGetLastError();
}

}  // namespace srq
