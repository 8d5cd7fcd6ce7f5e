// AdamW over many tensors at once, in place:
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   w' = w - lr (m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps) + decay w)
// Weights in binary32, or bfloat16 rounded as by sr_update_bf16 (to nearest or stochastically); moments in binary32 or block-scaled E4M3.
// gfx950 only.
//
// Moments in 8 bits.  A scale belongs to 128 neighbouring values, which sixteen lanes hold, eight each.  m is quantized as any block-scaled
// matrix.  The second moment spans twice as many binades as the format has for it, so its root r is held, and rounding is by squares: with q D
// and (q + 1) D the neighbours of r / scale, r is rounded up where the threshold eps of Eq. 1 satisfies
//   (r^2 / scale^2 - q^2 D^2) >= eps ((q + 1)^2 - q^2) D^2,
// so that over the thresholds the expectation of the stored square is v' itself; rounding the root without bias would add its variance to v'
// at every step, which for b2 near 1 outgrows what b2 takes away.  An r above zero is never stored as zero: it would be divided by eps.
// The weights are updated with m' and v' as computed, before they are rounded for storage.
#include "srq_blocks.hpp"
#include "srq_decoder.hpp"

namespace srq {
namespace {

constexpr uint32_t THREADS = 256, PIECE = THREADS * 8;  // values of a workgroup's iteration

// Tensors of one launch, by value: arguments of a kernel take up to 4 KiB.
struct Wide {  // moments in binary32
  static constexpr int MOST = 60;
  struct Entry {
    void* w;
    const void* g;
    void *m, *v;
    uint64_t n, counter;
    float decay;
    uint32_t pad;
  };
};
struct Narrow {  // in E4M3
  static constexpr int MOST = 46;
  struct Entry {
    void* w;
    const void* g;
    void *m, *v;
    uint64_t n, counter;
    float decay;
    uint32_t pad;
    uint8_t *ms, *vs;
  };
};
template <class C>
struct Batch {
  AdamWOptions o;
  uint32_t count, piece;         // piece: values of a workgroup, a multiple of PIECE
  uint32_t first[C::MOST];       // each tensor's first workgroup
  typename C::Entry entry[C::MOST];
};
static_assert(sizeof(Batch<Wide>) <= 4096 && sizeof(Batch<Narrow>) <= 4096, "kernel arguments");

__device__ __forceinline__ float value_of(const float* p, uint64_t i) { return p[i]; }
__device__ __forceinline__ float value_of(const uint16_t* p, uint64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }

// Values [at, at + 8) of a tensor of n, zeros behind its end.
template <int DTYPE>
__device__ __forceinline__ void load_octet(float (&x)[8], const void* p, uint64_t at, uint64_t n) {
  if (at + 8 <= n) {
    Octet<DTYPE> o;
    o.load(p, at);
    o.get(x);
  } else {
    typedef typename std::conditional<DTYPE == SRQ_F32, float, uint16_t>::type T;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = at + j < n ? value_of(static_cast<const T*>(p), at + j) : 0.0f;
  }
}
// Four of them, `whole`: all of the wave's lie within the tensor.
template <int DTYPE>
__device__ __forceinline__ void load_quad(float (&x)[4], const void* p, uint64_t at, uint64_t n, bool whole) {
  if (whole) {
    if constexpr (DTYPE == SRQ_F32) {
      const f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at));
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + at));
      x[0] = __uint_as_float(v.x << 16);
      x[1] = __uint_as_float(v.x & 0xFFFF0000u);
      x[2] = __uint_as_float(v.y << 16);
      x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
  } else {
    typedef typename std::conditional<DTYPE == SRQ_F32, float, uint16_t>::type T;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = at + j < n ? value_of(static_cast<const T*>(p), at + j) : 0.0f;
  }
}
// (bfloat16: of values that are numbers of its grid)
template <int DTYPE>
__device__ __forceinline__ void store_quad(void* p, uint64_t at, uint64_t n, bool whole, const float (&x)[4]) {
  if (whole) {
    if constexpr (DTYPE == SRQ_F32) {
      __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4*>(static_cast<float*>(p) + at));
    } else {
      const auto two = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
      __builtin_nontemporal_store(u32x2{two(x[0], x[1]), two(x[2], x[3])}, reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p) + at));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (at + j >= n) continue;
      if constexpr (DTYPE == SRQ_F32) static_cast<float*>(p)[at + j] = x[j];
      else static_cast<uint16_t*>(p)[at + j] = (uint16_t)(__float_as_uint(x[j]) >> 16);
    }
  }
}
__device__ __forceinline__ void store_floats(float* p, uint64_t at, uint64_t n, const float (&x)[8]) {
  if (at + 8 <= n) {
    f32x4* const q = reinterpret_cast<f32x4*>(p + at);
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, q);
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, q + 1);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (at + j < n) p[at + j] = x[j];
  }
}
__device__ __forceinline__ u32x2 load_codes(const void* p, uint64_t at, uint64_t n) {
  const uint8_t* const q = static_cast<const uint8_t*>(p) + at;
  if (at + 8 <= n) return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(q));
  u32x2 c = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (at + j < n) c[j / 4] |= (uint32_t)q[j] << (8 * (j % 4));
  return c;
}
__device__ __forceinline__ void store_codes(void* p, uint64_t at, uint64_t n, u32x2 c) {
  uint8_t* const q = static_cast<uint8_t*>(p) + at;
  if (at + 8 <= n) {
    __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(q));
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (at + j < n) q[j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
}

// x to the bfloat16 grid, as sr_update_bf16 rounds (r: two thresholds a word, RTN_WORD for nearest).
__device__ __forceinline__ uint32_t to_grid(float x, uint32_t r16, bool sr) {
  const uint32_t bits = __float_as_uint(x), sign = bits & 0x80000000u;
  uint32_t mag = bits & 0x7FFFFFFFu;
  if (mag > 0x7F800000u) return 0x7FC0u;
  mag = min(mag, 0x7F7F0000u);
  const uint32_t add = sign ? (sr ? r16 : 0x7FFFu) : (sr ? 65535u - r16 : 0x8000u);
  const uint32_t q = (mag + add) >> 16;
  return q ? (q | (sign >> 16)) : 0u;
}

// Codes of the roots of eight values v >= 0, r = sqrt(v), in units of 1 / inv, rounded by squares.  2^-120 takes E4M3's numbers to those binary32
// numbers, subnormals included, whose bits 20 to 26 are their codes.
template <bool SR>
__device__ __forceinline__ u32x2 codes_of_roots(const float (&v)[8], const float (&r)[8], float inv, const uint32_t (&w)[4]) {
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t code = min(__float_as_uint(__fmul_rn(__fmul_rn(r[j], inv), 0x1p-120f)) >> 20, 0x7Eu);  // (inv 2^-120 need be no normal number)
    const float low = __fmul_rn(__uint_as_float(code << 20), 0x1p+120f), high = __fmul_rn(__uint_as_float((code + 1) << 20), 0x1p+120f);
    const float from = __fmul_rn(low, low), u = __fmul_rn(__fmul_rn(v[j], inv), inv);
    const float eps = SR ? __builtin_fmaf((float)((w[j / 2] >> (16 * (j & 1))) & 0xFFFFu), 0x1p-16f, 0x1p-17f) : 0.5f;
    code += __fsub_rn(u, from) >= __fmul_rn(eps, __fsub_rn(__fmul_rn(high, high), from)) ? 1u : 0u;
    code = min(max(code, v[j] > 0.0f ? 1u : 0u), 0x7Eu);
    c[j] = v[j] != v[j] ? 0x7Fu : code;
  }
  return u32x2{c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24};
}

// What the workgroup has to do: its tensor (as many begin at or before it), where in it, and the step's constants.
template <class C>
struct Job {
  const typename C::Entry& e;
  uint64_t begin, end;
  float lr, inv1, inv2;  // inv2: of the second moment's root
  __device__ __forceinline__ Job(const Batch<C>& b, uint32_t which) : e(b.entry[which]) {
    begin = (uint64_t)(blockIdx.x - b.first[which]) * b.piece;
    end = min(begin + b.piece, e.n);
    const AdamWOptions& o = b.o;
    const float t = (float)(o.step_dev ? *o.step_dev : o.step);
    lr = o.lr_dev ? *o.lr_dev : o.lr;
    inv1 = __fdiv_rn(1.0f, -expm1f(t * o.log_beta1));
    inv2 = __fsqrt_rn(__fdiv_rn(1.0f, -expm1f(t * o.log_beta2)));
  }
};
template <class C>
__device__ __forceinline__ uint32_t tensor_of(const Batch<C>& b) {
  const uint32_t lane = threadIdx.x & 63u;
  return (uint32_t)__builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < b.count && b.first[lane < b.count ? lane : 0] <= blockIdx.x)) - 1);
}
// m and v become what they are after the step; root: of the new v.  (The root and the reciprocal are good to a unit in the last place.)
__device__ __forceinline__ void moments_of(const AdamWOptions& o, float g, float& m, float& v, float& root) {
  m = __fadd_rn(__fmul_rn(m, o.beta1), __fmul_rn(g, o.rest1));
  v = __fadd_rn(__fmul_rn(v, o.beta2), __fmul_rn(__fmul_rn(g, g), o.rest2));
  root = __builtin_amdgcn_sqrtf(v);
}
// The instruction's root of what is below the normal numbers is 0: looked for where a root is.
template <int N>
__device__ __forceinline__ void small_roots(const float (&v)[N], float (&root)[N]) {
  float least = root[0];
#pragma unroll
  for (int j = 1; j < N; ++j) least = fminf(least, root[j]);
  if (!__any(least == 0.0f)) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (root[j] == 0.0f) root[j] = __fmul_rn(__builtin_amdgcn_sqrtf(__fmul_rn(v[j], 0x1p64f)), 0x1p-32f);
}
template <class C>
__device__ __forceinline__ float weight_of(const Job<C>& j, const AdamWOptions& o, float m, float root, float w) {
  const float step = __fmul_rn(__fmul_rn(m, j.inv1), __builtin_amdgcn_rcpf(__builtin_fmaf(root, j.inv2, o.eps)));
  return __fsub_rn(w, __fmul_rn(j.lr, __builtin_fmaf(j.e.decay, w, step)));
}

// Moments in binary32.  A wave takes 512 values at a time, a lane four of the first and four of the second half of them (a pair of lanes trades words of two
// Philox blocks): 16-byte accesses of neighbouring lanes lie side by side.  Bound by memory: 48 tensors of 85 million weights in bfloat16 366 us, 5.6 TB/s;
// 50 tensors of 768 5.2, a launch and its latencies.
template <int W, int G, bool SR>
__global__ __launch_bounds__(THREADS) void adamw_kernel(Batch<Wide> b) {
  const uint32_t lane = threadIdx.x & 63u;
  const bool odd = lane & 1u;
  const Job<Wide> job(b, tensor_of(b));
  const Wide::Entry& e = job.e;
  const uint64_t counter = SR && W == SRQ_BF16 ? first_block(e.counter, b.o.counter_dev) : 0;
  for (uint64_t at = job.begin + (threadIdx.x >> 6) * CHUNK; at < job.end; at += PIECE) {
    uint32_t x[4] = {RTN_WORD, RTN_WORD, RTN_WORD, RTN_WORD};
    if constexpr (SR && W == SRQ_BF16) round_words_of_neighbours(counter + at / 8 + (odd ? 32u : 0u) + (lane >> 1), b.o.k0, b.o.k1, x, odd);
    const uint64_t from[2] = {at + 4 * lane, at + 256 + 4 * lane};
    float g[2][4], w[2][4], m[2][4], v[2][4];
    const bool whole = at + CHUNK <= e.n;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      load_quad<G>(g[h], e.g, from[h], e.n, whole);
      load_quad<W>(w[h], e.w, from[h], e.n, whole);
      load_quad<SRQ_F32>(m[h], e.m, from[h], e.n, whole);
      load_quad<SRQ_F32>(v[h], e.v, from[h], e.n, whole);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float root[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) moments_of(b.o, g[h][j], m[h][j], v[h][j], root[j]);
      small_roots(v[h], root);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[h][j] = weight_of(job, b.o, m[h][j], root[j], w[h][j]);
        if constexpr (W == SRQ_BF16) w[h][j] = __uint_as_float(to_grid(w[h][j], (x[2 * h + j / 2] >> (16 * (j & 1))) & 0xFFFFu, SR) << 16);
      }
      store_quad<W>(e.w, from[h], e.n, whole, w[h]);
      store_quad<SRQ_F32>(e.m, from[h], e.n, whole, m[h]);
      store_quad<SRQ_F32>(e.v, from[h], e.n, whole, v[h]);
    }
  }
}

// Moments in 8 bits: a lane has eight neighbouring values, sixteen lanes a block.  28 tensors of 206 million weights in bfloat16 520 us, 4.8 TB/s: three
// Philox blocks and two quantizations for eight values are nearly as long as the memory.
template <int W, int G, bool SR>
__global__ __launch_bounds__(THREADS) void adamw_kernel(Batch<Narrow> b) {
  const uint32_t lane = threadIdx.x & 63u;
  const Job<Narrow> job(b, tensor_of(b));
  const Narrow::Entry& e = job.e;
  const uint64_t n = e.n, blocks = (n + 7) / 8, counter = SR ? first_block(e.counter, b.o.counter_dev) : 0;
  for (uint64_t at = job.begin + 8 * threadIdx.x; at - 8 * lane < job.end; at += PIECE) {
    const bool live = at < n;
    float g[8], w[8], m[8], v[8], root[8];
    load_octet<G>(g, e.g, at, n);
    load_octet<W>(w, e.w, at, n);
    Octet<BSRC_E4M3> om, ov;
    om.a = load_codes(e.m, at, n);
    ov.a = load_codes(e.v, at, n);
    om.get(m, scale_value(live ? e.ms[at / SBLOCK] : 127u));
    ov.get(v, scale_value(live ? e.vs[at / SBLOCK] : 127u));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = __fmul_rn(v[j], v[j]);
      moments_of(b.o, g[j], m[j], v[j], root[j]);
    }
    small_roots(v, root);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = weight_of(job, b.o, m[j], root[j], w[j]);
    uint32_t r[4] = {RTN_WORD, RTN_WORD, RTN_WORD, RTN_WORD};
    if constexpr (W == SRQ_F32) {
      store_floats(static_cast<float*>(e.w), at, n, w);
    } else {
      uint32_t c[8];
      if constexpr (SR) philox_block(counter + at / 8, b.o.k0, b.o.k1, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = to_grid(w[j], (r[j / 2] >> (16 * (j & 1))) & 0xFFFFu, SR);
      uint16_t* const p = static_cast<uint16_t*>(e.w) + at;
      if (at + 8 <= n) {
        *reinterpret_cast<u32x4*>(p) = u32x4{c[0] | c[1] << 16, c[2] | c[3] << 16, c[4] | c[5] << 16, c[6] | c[7] << 16};
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (at + j < n) p[j] = (uint16_t)c[j];
      }
    }
    const Extent em = extent_of(m), ev = extent_of(root);
    const uint32_t bm = scale_byte<SRQ_E4M3>(max16(most_finite(m, em))), bv = scale_byte<SRQ_E4M3>(max16(most_finite(root, ev)));
    r[0] = r[1] = r[2] = r[3] = RTN_WORD;
    if constexpr (SR) philox_block(counter + blocks + at / 8, b.o.k0, b.o.k1, r);
    const u32x2 cm = codes_of_octet<SRQ_E4M3, SR>(m, em, bm, r);
    if constexpr (SR) philox_block(counter + 2 * blocks + at / 8, b.o.k0, b.o.k1, r);
    const u32x2 cv = codes_of_roots<SR>(v, root, scale_inverse(bv), r);
    store_codes(e.m, at, n, cm);
    store_codes(e.v, at, n, cv);
    if ((lane & 15u) == 0 && live) {
      e.ms[at / SBLOCK] = (uint8_t)bm;
      e.vs[at / SBLOCK] = (uint8_t)bv;
    }
  }
}

template <class C, int W, int G>
hipError_t run_class(const srq_adamw_tensor* tensors, int count, const AdamWOptions& o, hipStream_t stream) {
  constexpr bool NARROW = std::is_same<C, Narrow>::value;
  Batch<C> b;
  b.o = o;
  const auto fits = [&](const srq_adamw_tensor& t) {
    return t.n && (t.state_kind != SRQ_NONE) == NARROW && t.w_dtype == W && t.g_dtype == G;
  };
  for (int i = 0; i < count;) {
    // as many tensors as a launch takes, and what a workgroup does of them
    uint64_t values = 0;
    b.count = 0;
    for (; i < count && b.count < (uint32_t)C::MOST; ++i) {
      const srq_adamw_tensor& t = tensors[i];
      if (!fits(t)) continue;
      auto& e = b.entry[b.count++];
      e.w = t.w;
      e.g = t.g;
      e.m = t.m;
      e.v = t.v;
      e.n = t.n;
      e.counter = t.counter_offset;
      e.decay = t.weight_decay;
      e.pad = 0;
      if constexpr (NARROW) {
        e.ms = t.m_scales;
        e.vs = t.v_scales;
      }
      values += t.n;
    }
    if (b.count == 0) break;
    uint64_t piece = PIECE;
    while (values / piece > 1u << 14) piece *= 2;
    b.piece = (uint32_t)piece;
    uint32_t wgs = 0;
    for (uint32_t k = 0; k < b.count; ++k) {
      b.first[k] = wgs;
      wgs += (uint32_t)((b.entry[k].n + piece - 1) / piece);
    }
    if (o.sr) adamw_kernel<W, G, true><<<wgs, THREADS, 0, stream>>>(b);
    else adamw_kernel<W, G, false><<<wgs, THREADS, 0, stream>>>(b);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(const srq_adamw_tensor* tensors, int count, const AdamWOptions& o, hipStream_t stream) {
  bool there[2][2][2] = {};
  for (int i = 0; i < count; ++i)
    if (tensors[i].n) there[tensors[i].state_kind != SRQ_NONE][tensors[i].w_dtype == SRQ_BF16][tensors[i].g_dtype == SRQ_BF16] = true;
  hipError_t e = hipSuccess;
  const auto run = [&](bool is, auto f) {
    if (is && e == hipSuccess) e = f(tensors, count, o, stream);
  };
  run(there[0][0][0], run_class<Wide, SRQ_F32, SRQ_F32>);
  run(there[0][0][1], run_class<Wide, SRQ_F32, SRQ_BF16>);
  run(there[0][1][0], run_class<Wide, SRQ_BF16, SRQ_F32>);
  run(there[0][1][1], run_class<Wide, SRQ_BF16, SRQ_BF16>);
  run(there[1][0][0], run_class<Narrow, SRQ_F32, SRQ_F32>);
  run(there[1][0][1], run_class<Narrow, SRQ_F32, SRQ_BF16>);
  run(there[1][1][0], run_class<Narrow, SRQ_BF16, SRQ_F32>);
  run(there[1][1][1], run_class<Narrow, SRQ_BF16, SRQ_BF16>);
  return e;
}

}  // namespace srq
