// Root-mean-square norm with the residual's addition, and its backward pass.
//   h = x + r (rounded to the stream's dtype: the norm is that of the value the stream holds)
//   rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd gamma
//   d = dy gamma,  c = mean(d h rstd),  dx = rstd (d - h rstd c) + dh,  dgamma = sum over rows of dy h rstd
// Sums in binary32.  Memory-bound: a row is read once and stays in registers between its sum and its results.
#include "srq_blocks.hpp"

namespace srq {
namespace {

// ---- a row on T threads, groups of eight neighbouring values: group i of thread t starts at column 8 (i T + t) -----------
template <int DTYPE>
__device__ __forceinline__ void store_octet(void* p, size_t at, const float (&v)[8]) {
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

// The sum of one value a thread over the T threads of a row, in all of them, always in the same order.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = sum_of_rows(sum16(v));
  if constexpr (T > 64) {
    const uint32_t wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63u) == 0) lds[wave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += lds[w];
  }
  return v;
}

// Q: 0 values of the stream's dtype, else codes of that kind; SR: rounded stochastically.  16384 x 2048 bfloat16 with residual to E4M3: 39.9 us
// (5.9 TB/s); one row 2.8, its launch and three latencies (row, sum, gain).
template <int DTYPE, int Q, bool SR, int T, int NC>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_forward_kernel(NormForward n, uint32_t first) {
  __shared__ float lds[T / 64];
  constexpr uint32_t TEAMS = T < 256 ? 256 / T : 1;
  const uint32_t t = threadIdx.x % T;
  const size_t row = ((size_t)first + blockIdx.x) * TEAMS + threadIdx.x / T;
  if (TEAMS > 1 && row >= n.rows) return;  // (whole waves, and no barrier below where there are several teams)
  const size_t base = row * n.cols;
  Octet<DTYPE> x[NC], r[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const uint32_t col = 8 * (i * T + t);
    x[i].zero();
    r[i].zero();
    if (col < n.cols) {
      x[i].load(n.x, base + col);
      if (n.residual) r[i].load(n.residual, base + col);
    }
  }
  float h[NC][8], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const uint32_t col = 8 * (i * T + t);
    x[i].get(h[i]);
    if (n.residual) {
      float b[8];
      r[i].get(b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i][j] = __fadd_rn(h[i][j], b[j]);
        if constexpr (DTYPE == SRQ_BF16) h[i][j] = (float)(__bf16)h[i][j];
      }
      if (col < n.cols) store_octet<DTYPE>(n.h, base + col, h[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(h[i][j], h[i][j], sum);
  }
  sum = row_sum<T>(sum, lds);
  const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)n.cols), n.eps)));
  if (t == 0) n.rstd[row] = rstd;
  uint64_t counter = 0;
  if constexpr (SR) counter = first_block(n.rnd.counter_offset, n.rnd.counter_dev);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const uint32_t col = 8 * (i * T + t);
    const bool live = col < n.cols;
    float y[8];
    f32x4 g0 = {0, 0, 0, 0}, g1 = {0, 0, 0, 0};
    if (live) {
      g0 = *reinterpret_cast<const f32x4*>(n.gamma + col);
      g1 = *reinterpret_cast<const f32x4*>(n.gamma + col + 4);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = __fmul_rn(__fmul_rn(h[i][j], rstd), j < 4 ? g0[j & 3] : g1[j & 3]);
    if constexpr (Q == 0) {
      if (live) store_octet<DTYPE>(n.y, base + col, y);
    } else {
      // sixteen neighbouring lanes hold one block; those beyond the row zeros
      if (!live) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = 0.0f;  // (an infinite rstd times zero is not one)
      }
      const Extent e = extent_of(y);
      const uint32_t byte = scale_byte<Q>(max16(most_finite(y, e)));
      uint32_t w[4];
      thresholds<SR>(n.rnd, counter + (base + col) / 8, w);
      const u32x2 c = codes_of_octet<Q, SR>(y, e, byte, w);
      if (live) __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(static_cast<uint8_t*>(n.y) + row * n.y_pitch + col));
      if ((t & 15u) == 0 && live) n.scales[row * n.spitch + col / SBLOCK] = (uint8_t)byte;
    }
  }
}

// A workgroup's rows are a contiguous piece; every thread keeps the sums of its columns' dgamma over its team's rows.  8191 x 2048 binary32 with
// dh: 61.8 us (4.3 TB/s), of them 5 the second launch.
template <int DTYPE, int T, int NC>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_backward_kernel(NormBackward n, uint32_t rows_per_wg) {
  constexpr uint32_t TEAMS = T < 256 ? 256 / T : 1;
  constexpr int WIDTH = NC * T * 8;
  __shared__ float lds[2][T / 64];
  __shared__ __attribute__((aligned(16))) float sums[TEAMS > 1 ? WIDTH : 4];
  const uint32_t t = threadIdx.x % T, team = threadIdx.x / T;
  const uint32_t begin = blockIdx.x * rows_per_wg, end = min(n.rows, begin + rows_per_wg);
  const float inv_cols = __fdiv_rn(1.0f, (float)n.cols);
  float dg[NC][8], gamma[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const uint32_t col = 8 * (i * T + t);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dg[i][j] = 0.0f;
      gamma[i][j] = col < n.cols ? n.gamma[col + j] : 0.0f;
    }
  }
  // The next row's loads are under way while one is worked on, where registers allow.
  constexpr bool AHEAD = NC == 1 || T <= 256;
  struct Row {
    Octet<DTYPE> dy[NC], h[NC], dh[NC];
    float rstd;
  };
  auto fetch = [&](Row& r, uint32_t row) {
    const size_t base = (size_t)row * n.cols;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint32_t col = 8 * (i * T + t);
      r.dy[i].zero();
      r.h[i].zero();
      r.dh[i].zero();
      if (col < n.cols) {
        r.dy[i].load(n.dy, base + col);
        r.h[i].load(n.h, base + col);
        if (n.dh) r.dh[i].load(n.dh, base + col);
      }
    }
    r.rstd = n.rstd[row];
  };
  uint32_t turn = 0;
  Row next;
  if (AHEAD && begin + team < end) fetch(next, begin + team);
  for (uint32_t row = begin + team; row < end; row += TEAMS, turn ^= 1u) {
    Row cur;
    if constexpr (AHEAD) {
      cur = next;
      if (row + TEAMS < end) fetch(next, row + TEAMS);
    } else {
      fetch(cur, row);
    }
    float along = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float a[8], b[8];
      cur.dy[i].get(a);
      cur.h[i].get(b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float xhat = b[j] * cur.rstd;
        dg[i][j] = __builtin_fmaf(a[j], xhat, dg[i][j]);
        along = __builtin_fmaf(a[j] * gamma[i][j], xhat, along);
      }
    }
    const float c = row_sum<T>(along, lds[turn]) * inv_cols;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint32_t col = 8 * (i * T + t);
      float a[8], b[8], o[8];
      cur.dy[i].get(a);
      cur.h[i].get(b);
      cur.dh[i].get(o);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(cur.rstd, a[j] * gamma[i][j] - (b[j] * cur.rstd) * c, o[j]);
      if (col < n.cols) store_octet<DTYPE>(n.dx, (size_t)row * n.cols + col, o);
    }
  }
  if constexpr (TEAMS > 1) {  // the teams' sums one after the other
    for (uint32_t k = 0; k + 1 < TEAMS; ++k) {
      if (team == k) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int j = 0; j < 8; j += 4) {
            f32x4* const at = reinterpret_cast<f32x4*>(sums + 8 * (i * T + t) + j);
            f32x4 s = {dg[i][j], dg[i][j + 1], dg[i][j + 2], dg[i][j + 3]};
            if (k) s += *at;
            *at = s;
          }
      }
      __syncthreads();
    }
    if (team + 1 == TEAMS) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[i][j] += sums[8 * (i * T + t) + j];
    }
  }
  if (team + 1 == TEAMS) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint32_t col = 8 * (i * T + t);
      if (col >= n.cols) continue;
      f32x4* const at = reinterpret_cast<f32x4*>(n.partial + (size_t)blockIdx.x * n.cols + col);
      at[0] = f32x4{dg[i][0], dg[i][1], dg[i][2], dg[i][3]};
      at[1] = f32x4{dg[i][4], dg[i][5], dg[i][6], dg[i][7]};
    }
  }
}

// dgamma: the workgroups' sums in a fixed order, 64 columns a workgroup on sixteen waves, each with every sixteenth sum.
__global__ __launch_bounds__(1024) void norm_gain_kernel(float* dgamma, const float* partial, uint32_t parts, uint32_t cols, int accumulate) {
  __shared__ float lds[16][64];
  const uint32_t c = threadIdx.x & 63u, s = threadIdx.x >> 6, col = blockIdx.x * 64 + c;
  float v = 0.0f;
  if (col < cols) {
#pragma unroll 8
    for (uint32_t p = s; p < parts; p += 16) v += partial[(size_t)p * cols + col];
  }
  lds[s][c] = v;
  __syncthreads();
  if (s == 0 && col < cols) {
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += lds[k][c];
    dgamma[col] = accumulate ? dgamma[col] + v : v;
  }
}

// Threads a row and groups a thread, of which a thread's registers hold four.  64 threads (four rows a workgroup, no barrier) for rows of one
// group a thread, and of two where the rows alone fill the chip; else 256 and, beyond 8192 values, 1024.  bfloat16, 64 | 256 threads a row, us:
// 16384 x 512 11.8 | 25.6, 16384 x 1024 22.1 | 28.7, 512 x 1024 4.1 | 3.6, 16384 x 1536 33.6 | 32.8, 16384 x 2048 41.7 | 39.8, 1 x 2048 4.2 | 2.7.
template <class F>
void with_row_form(uint32_t rows, uint32_t cols, F&& f) {
  using std::integral_constant;
  const auto nc = [&](auto T, uint32_t groups) {
    if (groups <= 1) f(T, integral_constant<int, 1>{});
    else if (T.value == 64 || groups <= 2) f(T, integral_constant<int, 2>{});
    else if constexpr (T.value > 64) f(T, integral_constant<int, 4>{});
  };
  if (cols <= 512 || (cols <= 1024 && rows >= 2048)) nc(integral_constant<int, 64>{}, (cols + 511) / 512);
  else if (cols <= 8192) nc(integral_constant<int, 256>{}, (cols + 2047) / 2048);
  else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

template <int DTYPE>
void norm_forward_as(const NormForward& n, hipStream_t stream) {
  with_row_form(n.rows, n.cols, [&](auto T, auto NC) {
    constexpr unsigned threads = T.value < 256 ? 256 : T.value, teams = threads / T.value;
    const auto run = [&](auto kernel) {
      in_launches((n.rows + teams - 1) / teams, [&](uint32_t first, unsigned wgs) { kernel<<<wgs, threads, 0, stream>>>(n, first); });
    };
    constexpr int t = T.value, nc = NC.value;
    if (!n.scales) run(norm_forward_kernel<DTYPE, 0, false, t, nc>);
    else if (n.kind == SRQ_E5M2) run(n.rnd.sr ? norm_forward_kernel<DTYPE, SRQ_E5M2, true, t, nc> : norm_forward_kernel<DTYPE, SRQ_E5M2, false, t, nc>);
    else run(n.rnd.sr ? norm_forward_kernel<DTYPE, SRQ_E4M3, true, t, nc> : norm_forward_kernel<DTYPE, SRQ_E4M3, false, t, nc>);
  });
}

// Backward: a thread holds its columns' gain and the sums of its gradient over all of its rows, so few columns a thread and more threads a
// row: 256 from 528 columns on (8191 x 2048 binary32: with 64 threads a row and 32 columns each 225 registers, two waves a SIMD and two
// rows a wave, 87 us).
bool one_wave(uint32_t cols) { return cols <= 512; }
template <class F>
void with_backward_form(uint32_t cols, F&& f) {
  using std::integral_constant;
  if (one_wave(cols)) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (cols <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (cols <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (cols <= 8192) f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
uint32_t backward_rows(uint32_t rows, uint32_t cols) {
  // up to 1024 workgroups, and rows enough in each that its sums of dgamma weigh little beside them
  const uint32_t per = (rows + 1023) / 1024, least = one_wave(cols) ? 8 : 2;
  return per < least ? least : per;
}

template <int DTYPE>
void norm_backward_as(const NormBackward& n, uint32_t parts, uint32_t per, hipStream_t stream) {
  with_backward_form(n.cols, [&](auto T, auto NC) {
    constexpr unsigned threads = T.value < 256 ? 256 : T.value;
    norm_backward_kernel<DTYPE, T.value, NC.value><<<parts, threads, 0, stream>>>(n, per);
  });
}

}  // namespace

hipError_t launch_norm_forward(const NormForward& n, hipStream_t stream) {
  if (n.dtype == SRQ_F32) norm_forward_as<SRQ_F32>(n, stream);
  else norm_forward_as<SRQ_BF16>(n, stream);
  return hipGetLastError();
}

size_t norm_backward_partials(uint32_t rows, uint32_t cols) {
  const uint32_t per = backward_rows(rows, cols);
  return ((size_t)rows + per - 1) / per * cols;
}

hipError_t launch_norm_backward(const NormBackward& n, hipStream_t stream) {
  const uint32_t per = backward_rows(n.rows, n.cols), parts = (n.rows + per - 1) / per;
  if (parts == 0) {}  // (no rows: dgamma is still written)
  else if (n.dtype == SRQ_F32) norm_backward_as<SRQ_F32>(n, parts, per, stream);
  else norm_backward_as<SRQ_BF16>(n, parts, per, stream);
  norm_gain_kernel<<<(n.cols + 63) / 64, 1024, 0, stream>>>(n.dgamma, n.partial, parts, n.cols, n.accumulate);
  return hipGetLastError();
}

}  // namespace srq
