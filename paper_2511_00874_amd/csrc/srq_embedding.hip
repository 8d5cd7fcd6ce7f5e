// Embedding: rows of a table, scaled, and the gradient of the table.  gfx950 only.
//   out_m = scale table[id_m],   dtable_v = scale * sum over {m : id_m = v} of dy_m (+ dtable_v)
// Memory-bound both ways.  The gradient sorts the places m by their ids (stable, so that every sum has one order), adds up runs of equal ids in
// pieces of the sorted list, and joins the pieces of a run: whatever the ids, no atomics, and a token that fills the batch is as much work as
// any other.
#include <algorithm>

#include "srq_blocks.hpp"
#include "srq_decoder.hpp"

namespace srq {
namespace {

constexpr uint32_t THREADS = 256;

__device__ __forceinline__ int64_t id_at(const void* ids, int wide, size_t i) {
  return wide ? static_cast<const int64_t*>(ids)[i] : (int64_t) static_cast<const int32_t*>(ids)[i];
}
template <int DTYPE>
__device__ __forceinline__ void put_octet(void* p, size_t at, const float (&v)[8]) {
  if constexpr (DTYPE == SRQ_F32) {
    f32x4* const q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + at);
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, q);
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, q + 1);
  } else {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (__bf16)v[j];
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + at));
  }
}
// Rows of a table are met again: cached loads.
template <int DTYPE>
__device__ __forceinline__ void get_octet(float (&v)[8], const void* p, size_t at) {
  if constexpr (DTYPE == SRQ_F32) {
    const f32x4* const q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
    const f32x4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  }
}

// T threads a row (a power of two), ROWS rows a thread.  7 rows of 2048: 2.5 us, a launch and two latencies, id and row.
template <int TABLE, int OUT_, int ROWS>
__global__ __launch_bounds__(THREADS) void embed_forward_kernel(EmbedForward e, uint32_t threads_log2, uint32_t first) {
  const uint32_t t = threadIdx.x & ((1u << threads_log2) - 1u), teams = THREADS >> threads_log2;
  const size_t row0 = ((size_t)first + blockIdx.x) * teams * ROWS + (threadIdx.x >> threads_log2);
  int64_t id[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const size_t row = row0 + r * teams;
    id[r] = row < e.rows ? id_at(e.ids, e.wide, row) : -1;
  }
  for (uint32_t col = 8 * t; col < e.cols; col += 8u << threads_log2) {
    float v[ROWS][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool there = id[r] >= 0 && (uint64_t)id[r] < e.vocab;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[r][j] = __builtin_nanf("");
      if (there) get_octet<TABLE>(v[r], e.table, (size_t)id[r] * e.cols + col);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const size_t row = row0 + r * teams;
      if (row >= e.rows) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[r][j] = __fmul_rn(v[r][j], e.scale);
      put_octet<OUT_>(e.out, row * e.cols + col, v[r]);
    }
  }
}

// ---- the sort: few keys by their ranks, many least digit first, up to 9 bits a pass ------------------------------------------------------------------------
constexpr uint32_t SORT_THREADS = 1024, SORT_WAVES = 16, BINS = 512, ROUNDS = 4, SUB = SORT_THREADS * ROUNDS;  // keys of a sub-block
constexpr uint32_t ONE_ROUNDS = 16, ONE_TILE = SORT_THREADS * ONE_ROUNDS;  // up to so many places are sorted in one launch
constexpr uint32_t MOST_TILES = 64;   // workgroups of a pass otherwise; each finds its bins' begins from all counts
struct Keys {  // source and target of a pass; ids: the source of the first one
  const void* ids;
  int wide;
  uint32_t vocab;
  int64_t padding;
  const uint32_t *key_in, *place_in;
  uint32_t *key_out, *place_out;
};
// Key of place m: its id, or vocab (behind all others) where it has no row.
__device__ __forceinline__ uint32_t key_of(const Keys& k, uint32_t m) {
  if (k.key_in) return k.key_in[m];
  const int64_t id = id_at(k.ids, k.wide, m);
  return id < 0 || id >= (int64_t)k.vocab || id == k.padding ? k.vocab : (uint32_t)id;
}

// The sort leaves the memory idle; other workgroups of its launches clear a part of the table each: rows without a token are zeros, and the few others
// are written again (8191 places, 32000 x 768: 20 us for both, of which clearing alone takes 15; sums beside a search for the empty rows took 44).
struct Fill {
  float* p;
  size_t n;  // a multiple of 4
};
__device__ __forceinline__ void fill(const Fill& f, uint32_t wg, uint32_t wgs) {
  for (size_t i = 4 * ((size_t)wg * SORT_THREADS + threadIdx.x); i < f.n; i += (size_t)4 * wgs * SORT_THREADS)
    __builtin_nontemporal_store(f32x4{0, 0, 0, 0}, reinterpret_cast<f32x4*>(f.p + i));
}
uint32_t fill_workgroups(const Fill& f) { return (uint32_t)std::min<size_t>(512, (f.n + 16 * SORT_THREADS - 1) / (16 * SORT_THREADS)); }

typedef uint16_t Counts[SORT_WAVES][BINS];
__device__ __forceinline__ void clear(Counts& counts) {
  for (uint32_t i = threadIdx.x; i < sizeof(Counts) / 4; i += SORT_THREADS) reinterpret_cast<uint32_t*>(&counts[0][0])[i] = 0;
}
// Place of this lane's key among the wave's of its digit so far, which are then one round more.
__device__ __forceinline__ uint32_t rank_of(uint16_t (&counts)[BINS], uint32_t digit, bool live, uint32_t bits) {
  const uint32_t lane = threadIdx.x & 63u;
  uint64_t same = __ballot(live);  // lanes with this digit
  for (uint32_t b = 0; b < bits; ++b) {
    const bool set = (digit >> b) & 1u;
    const uint64_t all = __ballot(set);
    same &= set ? all : ~all;
  }
  const uint32_t before = __popcll(same & ((1ull << lane) - 1ull)), rank = live ? counts[digit] + before : 0u;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (all lanes of the wave have read; then: one of each digit has written)
  if (live && before == 0) counts[digit] = (uint16_t)(rank + __popcll(same));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return rank;
}
// The waves' counts become the places, within the block, of each wave's first key of a bin; returns the bin's count (threads below BINS).
__device__ __forceinline__ uint32_t waves_begin(Counts& counts) {
  uint32_t total = 0;
  if (threadIdx.x < BINS) {
#pragma unroll
    for (uint32_t w = 0; w < SORT_WAVES; ++w) {
      const uint32_t c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = (uint16_t)total;
      total += c;
    }
  }
  return total;
}
// Exclusive sums over all bins of the threads' values (0 from BINS on).
__device__ __forceinline__ uint32_t sums_before(uint32_t v, uint32_t (&sums)[SORT_WAVES]) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(s, d);
    if (lane >= (uint32_t)d) s += up;
  }
  if (lane == 63) sums[wave] = s;
  __syncthreads();
  uint32_t before = 0;
  for (uint32_t w = 0; w < wave; ++w) before += sums[w];
  return before + s - v;
}

// Few keys: each is told its place by counting those that go in front of it, all pairs.  A workgroup has RANKED of the keys and all of them in LDS; its half
// waves, with a key a lane, go through a part of them each (a comparison and an addition a pair: 8191 keys 4 us of the chip's issue).  A call with 8191
// places of 768 columns takes 38.0 us, 41.5 with one workgroup that sorts by digits in registers and LDS; 4096 of 2048 25.3, so 32.3; 16384 of 768 64, so 68.
constexpr uint32_t RANKED = 32, PARTS = SORT_THREADS / RANKED;
__global__ __launch_bounds__(SORT_THREADS) void sort_rank_kernel(Keys k, uint32_t n, uint32_t wgs, Fill f) {
  __shared__ __attribute__((aligned(16))) uint32_t key[ONE_TILE];
  __shared__ uint32_t counts[PARTS][RANKED];
  if (blockIdx.x >= wgs) return fill(f, blockIdx.x - wgs, gridDim.x - wgs);
  const uint32_t part = threadIdx.x / RANKED, i = threadIdx.x % RANKED, first = blockIdx.x * RANKED, each = (n + 4 * PARTS - 1) / (4 * PARTS) * 4;
#pragma unroll 4
  for (uint32_t m = threadIdx.x; m < each * PARTS; m += SORT_THREADS) key[m] = m < n ? key_of(k, m) : ~0u;  // (in front of none)
  __syncthreads();
  const uint32_t own = key[min(first + i, n - 1)];
  uint32_t count = 0;
#pragma unroll 4
  for (uint32_t m = part * each; m < (part + 1) * each; m += 4) {
    const u32x4 four = *reinterpret_cast<const u32x4*>(key + m);
    const uint32_t below = own + (m < first ? 1u : 0u);  // of equal keys the places in front
#pragma unroll
    for (int e = 0; e < 4; ++e) count += four[e] < below ? 1u : 0u;
  }
  if (part == 0)
    for (uint32_t m = 0; m < i; ++m) count += key[min(first + m, n - 1)] == own ? 1u : 0u;
  counts[part][i] = count;
  __syncthreads();
  if (threadIdx.x < RANKED && first + i < n) {
    uint32_t to = 0;
#pragma unroll
    for (uint32_t p = 0; p < PARTS; ++p) to += counts[p][i];
    k.key_out[to] = own;
    k.place_out[to] = first + i;
  }
}

// Many: a launch that counts and one that moves for every pass, a tile a workgroup.
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(Keys k, uint32_t* counts, uint32_t n, uint32_t tile, uint32_t tiles, uint32_t shift,
                                                                  uint32_t bits, Fill f) {
  __shared__ uint32_t bins[BINS];
  if (blockIdx.x >= tiles) return fill(f, blockIdx.x - tiles, gridDim.x - tiles);
  const uint32_t begin = blockIdx.x * tile, end = min(n, begin + tile);
  if (threadIdx.x < BINS) bins[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll 4
  for (uint32_t m = begin + threadIdx.x; m < end; m += SORT_THREADS) atomicAdd(&bins[(key_of(k, m) >> shift) & ((1u << bits) - 1u)], 1u);
  __syncthreads();
  if (threadIdx.x < BINS) counts[blockIdx.x * BINS + threadIdx.x] = bins[threadIdx.x];
}
__global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(Keys k, const uint32_t* counts, uint32_t n, uint32_t tile, uint32_t tiles, uint32_t shift,
                                                                    uint32_t bits, Fill f) {
  __shared__ Counts waves;
  __shared__ uint32_t base[BINS], sums[SORT_WAVES];  // base: where the next key of a bin goes
  if (blockIdx.x >= tiles) return fill(f, blockIdx.x - tiles, gridDim.x - tiles);
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, mask = (1u << bits) - 1u;
  uint32_t before = 0, all = 0;
  if (threadIdx.x < BINS) {
#pragma unroll 8
    for (uint32_t w = 0; w < tiles; ++w) {
      const uint32_t c = counts[w * BINS + threadIdx.x];
      all += c;
      before += w < blockIdx.x ? c : 0u;
    }
  }
  const uint32_t from = sums_before(all, sums);
  if (threadIdx.x < BINS) base[threadIdx.x] = from + before;
  const uint32_t begin = blockIdx.x * tile, end = min(n, begin + tile);
  for (uint32_t sub = begin; sub < end; sub += SUB) {
    clear(waves);
    __syncthreads();
    uint32_t key[ROUNDS], place[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
      const uint32_t m = sub + wave * (64 * ROUNDS) + r * 64 + lane;
      key[r] = m < end ? key_of(k, m) : 0u;
      place[r] = m < end && k.place_in ? k.place_in[m] : m;
    }
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) rank[r] = rank_of(waves[wave], (key[r] >> shift) & mask, sub + wave * (64 * ROUNDS) + r * 64 + lane < end, bits);
    __syncthreads();
    const uint32_t total = waves_begin(waves);
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
      if (sub + wave * (64 * ROUNDS) + r * 64 + lane >= end) continue;
      const uint32_t digit = (key[r] >> shift) & mask, to = base[digit] + waves[wave][digit] + rank[r];
      k.key_out[to] = key[r];
      k.place_out[to] = place[r];
    }
    __syncthreads();
    if (threadIdx.x < BINS) base[threadIdx.x] += total;
    __syncthreads();
  }
}

// ---- sums of runs --------------------------------------------------------------------------------------------------------------
struct Runs {
  const uint32_t *keys, *places;  // sorted
  float *head, *tail;             // of every piece: the sum of its part of a run that began before it, and of one that goes on behind it
  uint32_t n, piece, pieces;
};

constexpr uint32_t AHEAD = 8;     // rows of dy under way

// The runs of a piece, T threads with 8 columns each, blockIdx.y the block of 8 T columns.  65536 places of 2048 bfloat16: 89 us, 4 TB/s of what is read and
// written; 8191 of 768 binary32 11.  (Four rows under way or sixteen, pieces of 16: as fast or slower.)
template <int DTYPE>
__global__ __launch_bounds__(THREADS) void embed_sum_kernel(EmbedBackward e, Runs r) {
  const uint32_t col = 8 * (blockIdx.y * blockDim.x + threadIdx.x);
  const bool mine = col < e.cols;
  const uint32_t begin = blockIdx.x * r.piece, end = min(r.n, begin + r.piece);
  const uint32_t before = begin ? r.keys[begin - 1] : ~0u, behind = end < r.n ? r.keys[end] : ~0u;
  float acc[8] = {};
  uint32_t key = r.keys[begin];
  bool head = key == before;
  const auto flush = [&](bool goes_on) {
    if (key >= e.vocab || !mine) return;  // (places without a row)
    if (head || goes_on) {
      float* const to = (head ? r.head : r.tail) + (size_t)blockIdx.x * e.cols + col;
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j] = acc[j];
      return;
    }
    float v[8];
    const size_t at = (size_t)key * e.cols + col;
    if (e.accumulate) get_octet<SRQ_F32>(v, e.dtable, at);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e.accumulate ? __fadd_rn(v[j], __fmul_rn(acc[j], e.scale)) : __fmul_rn(acc[j], e.scale);
    put_octet<SRQ_F32>(e.dtable, at, v);
  };
  for (uint32_t i = begin; i < end; i += AHEAD) {
    Octet<DTYPE> row[AHEAD];
#pragma unroll
    for (uint32_t u = 0; u < AHEAD; ++u) {
      row[u].zero();
      if (i + u < end && mine) row[u].load(e.dy, (size_t)r.places[i + u] * e.cols + col);
    }
#pragma unroll
    for (uint32_t u = 0; u < AHEAD; ++u) {
      if (i + u >= end) break;
      const uint32_t next = r.keys[i + u];
      if (next != key) {
        flush(false);
        key = next;
        head = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
      }
      float v[8];
      row[u].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[j];
    }
  }
  flush(key == behind);
}

// A run that goes on behind the piece it begins in: the piece's tail and the heads of those it reaches, waves of 64 threads with 8 columns each
// taking every fourth, always in one order.  (Most pieces have none: few threads.)  65536 places of 2048: 12 us.
constexpr uint32_t JOIN_WAVES = 4;
__global__ __launch_bounds__(64 * JOIN_WAVES) void embed_join_kernel(EmbedBackward e, Runs r) {
  const uint32_t begin = blockIdx.x * r.piece, end = min(r.n, begin + r.piece);
  if (end >= r.n) return;
  const uint32_t key = r.keys[end];
  if (key >= e.vocab || r.keys[end - 1] != key) return;     // nothing goes on
  if (begin && r.keys[begin - 1] == key) return;            // it began before
  __shared__ __attribute__((aligned(16))) float sums[JOIN_WAVES][64 * 8 + 8];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = 8 * (blockIdx.y * 64 + lane);
  const bool mine = col < e.cols;
  uint32_t last = blockIdx.x;                               // the piece in which it ends: the last that begins with it, 64 looked at a time
  for (uint32_t more = 64; more == 64; last += more) {
    const uint32_t p = last + 1 + lane;
    const uint64_t others = ~__ballot(p < r.pieces && r.keys[(size_t)p * r.piece] == key);
    more = others ? (uint32_t)__builtin_ctzll(others) : 64u;
  }
  float acc[8] = {};
  if (mine)
#pragma unroll 4
    for (uint32_t p = blockIdx.x + wave; p <= last; p += JOIN_WAVES) {
      float v[8];
      get_octet<SRQ_F32>(v, p == blockIdx.x ? r.tail : r.head, (size_t)p * e.cols + col);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[j];
    }
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[wave][lane * 8 + j] = acc[j];
  __syncthreads();
  if (wave == 0 && mine) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j] = 0.0f;
      for (uint32_t w = 0; w < JOIN_WAVES; ++w) acc[j] += sums[w][lane * 8 + j];
    }
    float v[8];
    const size_t at = (size_t)key * e.cols + col;
    if (e.accumulate) get_octet<SRQ_F32>(v, e.dtable, at);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e.accumulate ? __fadd_rn(v[j], __fmul_rn(acc[j], e.scale)) : __fmul_rn(acc[j], e.scale);
    put_octet<SRQ_F32>(e.dtable, at, v);
  }
}

uint32_t threads_of(uint32_t cols) {  // a row's threads, 8 columns each: whole waves
  uint32_t t = 64;
  while (t < THREADS && 8 * t < cols) t *= 2;
  return t;
}
// Places of a piece: so many that some two thousand workgroups share them, 8 at least (a thread's rows under way), 64 at most.
uint32_t piece_of(uint32_t rows) {
  uint32_t p = 8;
  while (p < 64 && rows / p > 2048) p *= 2;
  return p;
}
struct Layout {
  uint32_t *key_a, *place_a, *key_b, *place_b, *counts;
  float *head, *tail;
  size_t bytes;
};
Layout layout(void* ws, uint32_t rows, uint32_t cols) {
  Layout l;
  const size_t n = ((size_t)rows + 3) / 4 * 4, pieces = ((size_t)rows + piece_of(rows) - 1) / piece_of(rows);
  uint32_t* const at = static_cast<uint32_t*>(ws);
  l.key_a = at;
  l.place_a = at + n;
  l.key_b = at + 2 * n;
  l.place_b = at + 3 * n;
  l.counts = at + 4 * n;
  l.head = reinterpret_cast<float*>(at + 4 * n + MOST_TILES * BINS);
  l.tail = l.head + pieces * cols;
  l.bytes = 4 * (4 * n + MOST_TILES * BINS + 2 * pieces * cols);
  return l;
}

template <int TABLE, int OUT_>
void embed_forward_as(const EmbedForward& e, hipStream_t stream) {
  uint32_t log2 = 0;
  while ((1u << log2) < THREADS && (8u << log2) < e.cols) ++log2;
  const uint32_t teams = THREADS >> log2;
  // four rows a thread where the rows fill the chip four times over
  const bool four = e.rows / teams >= 4096;
  const size_t per = (size_t)teams * (four ? 4 : 1);
  in_launches((e.rows + per - 1) / per, [&](uint32_t first, unsigned wgs) {
    if (four) embed_forward_kernel<TABLE, OUT_, 4><<<wgs, THREADS, 0, stream>>>(e, log2, first);
    else embed_forward_kernel<TABLE, OUT_, 1><<<wgs, THREADS, 0, stream>>>(e, log2, first);
  });
}

}  // namespace

hipError_t launch_embed_forward(const EmbedForward& e, hipStream_t stream) {
  if (e.dtype == SRQ_F32) {
    if (e.out_dtype == SRQ_F32) embed_forward_as<SRQ_F32, SRQ_F32>(e, stream);
    else embed_forward_as<SRQ_F32, SRQ_BF16>(e, stream);
  } else {
    if (e.out_dtype == SRQ_F32) embed_forward_as<SRQ_BF16, SRQ_F32>(e, stream);
    else embed_forward_as<SRQ_BF16, SRQ_BF16>(e, stream);
  }
  return hipGetLastError();
}

size_t embed_backward_workspace(uint32_t rows, uint32_t cols) { return layout(nullptr, rows, cols).bytes; }

hipError_t launch_embed_backward(const EmbedBackward& e, hipStream_t stream) {
  const Layout l = layout(e.workspace, e.rows, e.cols);
  Runs r = {};
  r.keys = l.key_b;
  r.places = l.place_b;
  r.head = l.head;
  r.tail = l.tail;
  r.n = e.rows;
  r.piece = piece_of(e.rows);
  r.pieces = (e.rows + r.piece - 1) / r.piece;
  const size_t table = e.accumulate ? 0 : (size_t)e.vocab * e.cols;
  uint32_t width = 1;  // bits of a key (vocab among them)
  while (width < 32 && (e.vocab >> width)) ++width;
  const uint32_t passes = (width + 8) / 9, bits = (width + passes - 1) / passes;
  Keys k = {};
  k.ids = e.ids;
  k.wide = e.wide;
  k.vocab = e.vocab;
  k.padding = e.padding;
  if (e.rows <= ONE_TILE) {
    k.key_out = l.key_b;
    k.place_out = l.place_b;
    const Fill f = {e.dtable, table};
    const uint32_t wgs = (e.rows + RANKED - 1) / RANKED, all = wgs + fill_workgroups(f);
    if (all) sort_rank_kernel<<<all, SORT_THREADS, 0, stream>>>(k, e.rows, wgs, f);
  } else {
    uint32_t tile = SUB, part = 0;
    while ((e.rows + tile - 1) / tile > MOST_TILES) tile += SUB;
    const uint32_t tiles = (e.rows + tile - 1) / tile;
    const auto fill_part = [&]() {  // the next of as many parts as there are launches
      const size_t from = table / 4 * part / (2 * passes) * 4, to = table / 4 * (part + 1) / (2 * passes) * 4;
      ++part;
      return Fill{e.dtable + from, to - from};
    };
    for (uint32_t p = 0; p < passes; ++p) {
      const bool to_b = ((passes - p) & 1u) != 0;
      k.key_out = to_b ? l.key_b : l.key_a;
      k.place_out = to_b ? l.place_b : l.place_a;
      Fill f = fill_part();
      sort_count_kernel<<<tiles + fill_workgroups(f), SORT_THREADS, 0, stream>>>(k, l.counts, e.rows, tile, tiles, p * bits, bits, f);
      f = fill_part();
      sort_scatter_kernel<<<tiles + fill_workgroups(f), SORT_THREADS, 0, stream>>>(k, l.counts, e.rows, tile, tiles, p * bits, bits, f);
      k.key_in = k.key_out;
      k.place_in = k.place_out;
    }
  }
  if (r.pieces) {
    const uint32_t threads = threads_of(e.cols);
    const dim3 grid(r.pieces, (e.cols + 8 * threads - 1) / (8 * threads));
    if (e.dtype == SRQ_F32) embed_sum_kernel<SRQ_F32><<<grid, threads, 0, stream>>>(e, r);
    else embed_sum_kernel<SRQ_BF16><<<grid, threads, 0, stream>>>(e, r);
  }
  if (r.pieces > 1) embed_join_kernel<<<dim3(r.pieces - 1, (e.cols + 511) / 512), 64 * JOIN_WAVES, 0, stream>>>(e, r);
  return hipGetLastError();
}

}  // namespace srq
