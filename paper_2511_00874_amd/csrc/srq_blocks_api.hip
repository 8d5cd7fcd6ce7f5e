// C ABI of the block-scaled operators: argument checks and one launch (or two) each.
#include <cmath>

#include "srq_blocks.hpp"

using namespace srq;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool dtype_ok(int d) { return d == SRQ_F32 || d == SRQ_BF16; }
bool act_ok(int a) { return a == SRQ_ACT_SILU || a == SRQ_ACT_GELU; }

// What the kernels' 32-bit indexes hold: rows, and tiles of 128 x 128, under 2^30 (up to two workgroups a tile; more threads than a launch has: in_launches).
constexpr size_t MOST = 0x3FFFFFFF;
bool size_ok(size_t rows, size_t cols) {
  return rows <= MOST && cols <= MOST && ((rows + 127) / 128) * ((cols + 127) / 128) <= MOST;
}
// Columns of a matrix that is quantized, turned or restored: 128 rows of binary32 within 2^30 bytes.
constexpr size_t WIDEST = (size_t)1 << 21;
bool features_ok(size_t rows, size_t cols) { return cols <= WIDEST && size_ok(rows, cols); }
// Tiles of the gated block's gradients, two workgroups of 512 threads each in sixteens: one launch, of fewer than 2^32 threads (550 GB to move).
constexpr size_t MOST_PAIRS = ((size_t)1 << 22) - 8;

int check_kind(int kind) {
  if (kind == SRQ_E4M3 || kind == SRQ_E5M2) return SRQ_OK;
  return kind >= SRQ_NONE && kind <= SRQ_E4M0 ? SRQ_ERR_UNSUPPORTED : SRQ_ERR_FORMAT;
}

int check_quantizer(const srq_quant* q) {
  if (!q) return SRQ_ERR_NULL;
  if (const int st = check_kind(q->kind); st != SRQ_OK) return st;
  if (q->round != SRQ_SR && q->round != SRQ_RTN) return SRQ_ERR_FORMAT;
  if (q->flags & ~(uint32_t)SRQ_FLAG_COUNTER_DEV) return SRQ_ERR_FORMAT;
  if ((q->flags & SRQ_FLAG_COUNTER_DEV) && (q->counter_offset == 0 || (q->counter_offset & 7u))) return SRQ_ERR_ALIGN;
  return SRQ_OK;
}

Rounding rounding(const srq_quant* q) {
  Rounding r = {};
  if (!q) return r;
  const bool dev = q->flags & SRQ_FLAG_COUNTER_DEV;
  r.sr = q->round == SRQ_SR;
  r.k0 = (uint32_t)q->seed;
  r.k1 = (uint32_t)(q->seed >> 32);
  r.counter_offset = dev ? 0 : q->counter_offset;
  r.counter_dev = dev && r.sr ? reinterpret_cast<const uint64_t*>(static_cast<uintptr_t>(q->counter_offset)) : nullptr;
  return r;
}

// The longest contraction of a product: a tile's rows of both operands then lie within the 31 bits of a buffer's offsets.
constexpr size_t LONGEST = (size_t)1 << 22;

// A block-scaled matrix of `cols` columns: both parts, and rows that hold them, or an error.
int check_blocks(const void* codes, size_t pitch, const void* scales, size_t cols) {
  if (!codes || !scales) return SRQ_ERR_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4) || pitch % 16) return SRQ_ERR_ALIGN;
  return pitch >= block_pitch_least(cols) ? SRQ_OK : SRQ_ERR_SHAPE;
}

TileOut tile_out(void* codes, size_t pitch, void* scales, void* codes_t, size_t pitch_t, void* scales_t, size_t rows, size_t cols) {
  TileOut o;
  o.codes = static_cast<uint8_t*>(codes);
  o.scales = static_cast<uint8_t*>(scales);
  o.codes_t = static_cast<uint8_t*>(codes_t);
  o.scales_t = static_cast<uint8_t*>(scales_t);
  o.rows = (uint32_t)rows;
  o.cols = (uint32_t)cols;
  o.pitch = pitch;
  o.spitch = scale_pitch(cols);
  o.pitch_t = pitch_t;
  o.spitch_t = scale_pitch(rows);
  return o;
}

BlockOperand operand(const void* codes, size_t pitch, const void* scales, size_t cols) {
  return {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), pitch, scale_pitch(cols)};
}

int done(hipError_t e) { return e == hipSuccess ? SRQ_OK : SRQ_ERR_HIP; }

}  // namespace

extern "C" {

size_t sr_block_pitch(size_t cols) { return block_pitch(cols); }
size_t sr_block_scale_pitch(size_t cols) { return scale_pitch(cols); }

int sr_block_quantize(void* codes, size_t pitch, void* scales, void* codes_t, size_t pitch_t, void* scales_t, const void* x, int dtype,
                      size_t rows, size_t cols, const srq_quant* q, void* stream) {
  if (const int st = check_quantizer(q); st != SRQ_OK) return st;
  if (!dtype_ok(dtype)) return SRQ_ERR_FORMAT;
  if (!features_ok(rows, cols)) return SRQ_ERR_SHAPE;
  if (cols % 16) return SRQ_ERR_ALIGN;
  if (rows == 0 || cols == 0) return SRQ_OK;
  if (!x || (!codes && !codes_t)) return SRQ_ERR_NULL;
  if (codes)
    if (const int st = check_blocks(codes, pitch, scales, cols); st != SRQ_OK) return st;
  if (codes && pitch > 2 * WIDEST) return SRQ_ERR_SHAPE;
  if (codes_t)
    if (const int st = check_blocks(codes_t, pitch_t, scales_t, rows); st != SRQ_OK) return st;
  if (!aligned(x, 16)) return SRQ_ERR_ALIGN;
  BlockQuantize b = {};
  b.x = x;
  b.x_pitch = cols;
  b.src = dtype;
  b.kind = q->kind;
  b.out = tile_out(codes, pitch, scales, codes_t, pitch_t, scales_t, rows, cols);
  b.rnd = rounding(q);
  return done(launch_block_quantize(b, static_cast<hipStream_t>(stream)));
}

int sr_block_turn(void* codes_t, size_t pitch_t, void* scales_t, const void* codes, size_t pitch, const void* scales, int kind, size_t rows,
                  size_t cols, const srq_quant* q, void* stream) {
  if (const int st = check_quantizer(q); st != SRQ_OK) return st;
  if (const int st = check_kind(kind); st != SRQ_OK) return st;
  if (!features_ok(rows, cols)) return SRQ_ERR_SHAPE;
  if (cols % 16) return SRQ_ERR_ALIGN;
  if (rows == 0 || cols == 0) return SRQ_OK;
  if (const int st = check_blocks(codes, pitch, scales, cols); st != SRQ_OK) return st;
  if (pitch > 2 * WIDEST) return SRQ_ERR_SHAPE;
  if (const int st = check_blocks(codes_t, pitch_t, scales_t, rows); st != SRQ_OK) return st;
  BlockQuantize b = {};
  b.x = codes;
  b.x_scales = static_cast<const uint8_t*>(scales);
  b.x_pitch = pitch;
  b.x_spitch = scale_pitch(cols);
  b.src = kind == SRQ_E5M2 ? BSRC_E5M2 : BSRC_E4M3;
  b.kind = q->kind;
  b.out = tile_out(nullptr, 0, nullptr, codes_t, pitch_t, scales_t, rows, cols);
  b.rnd = rounding(q);
  return done(launch_block_quantize(b, static_cast<hipStream_t>(stream)));
}

int sr_block_restore(void* x, int dtype, const void* codes, size_t pitch, const void* scales, int kind, size_t rows, size_t cols,
                     void* stream) {
  if (const int st = check_kind(kind); st != SRQ_OK) return st;
  if (!dtype_ok(dtype)) return SRQ_ERR_FORMAT;
  if (!features_ok(rows, cols)) return SRQ_ERR_SHAPE;
  if (cols % 16) return SRQ_ERR_ALIGN;
  if (rows == 0 || cols == 0) return SRQ_OK;
  if (!x) return SRQ_ERR_NULL;
  if (const int st = check_blocks(codes, pitch, scales, cols); st != SRQ_OK) return st;
  if (!aligned(x, 16)) return SRQ_ERR_ALIGN;
  return done(launch_block_restore(x, dtype, static_cast<const uint8_t*>(codes), pitch, static_cast<const uint8_t*>(scales), rows, cols, kind,
                                   static_cast<hipStream_t>(stream)));
}

size_t sr_gemm_blocks_workspace_bytes(size_t P, size_t Q, size_t R, uint32_t flags) {
  if (!size_ok(P, Q) || R > LONGEST) return 0;
  return block_product_workspace(P, Q, R, (flags & SRQ_FLAG_F8_PIPELINE) != 0);
}

int sr_gemm_blocks(void* out, int dtype, const void* X, size_t pitchX, const void* scalesX, int kindX, const void* Z, size_t pitchZ,
                   const void* scalesZ, int kindZ, size_t P, size_t Q, size_t R, float alpha, float beta, uint32_t flags, void* workspace,
                   size_t workspace_bytes, void* stream) {
  for (const int kind : {kindX, kindZ})
    if (const int st = check_kind(kind); st != SRQ_OK) return st;
  if (!dtype_ok(dtype) || !std::isfinite(alpha) || (flags & ~(uint32_t)SRQ_FLAG_F8_PIPELINE)) return SRQ_ERR_FORMAT;
  if (beta != 0.0f && (beta != 1.0f || dtype != SRQ_F32)) return SRQ_ERR_UNSUPPORTED;
  if (!size_ok(P, Q) || R > LONGEST) return SRQ_ERR_SHAPE;
  if (P == 0 || Q == 0) return SRQ_OK;
  if (!out) return SRQ_ERR_NULL;
  if (!aligned(out, 16)) return SRQ_ERR_ALIGN;
  if (R) {
    if (const int st = check_blocks(X, pitchX, scalesX, R); st != SRQ_OK) return st;
    if (const int st = check_blocks(Z, pitchZ, scalesZ, R); st != SRQ_OK) return st;
    if (pitchX > LONGEST || pitchZ > LONGEST) return SRQ_ERR_SHAPE;
  }
  BlockProduct p = {};
  p.f8 = (flags & SRQ_FLAG_F8_PIPELINE) != 0;
  const size_t need = block_product_workspace(P, Q, R, p.f8);
  if (need && (!workspace || workspace_bytes < need)) return SRQ_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  p.X = operand(X, pitchX, scalesX, R);
  p.Z = operand(Z, pitchZ, scalesZ, R);
  p.kindX = kindX;
  p.kindZ = kindZ;
  p.out = out;
  p.out_bf16 = dtype == SRQ_BF16;
  p.accumulate = beta != 0.0f;
  p.alpha = alpha;
  p.P = P;
  p.Q = Q;
  p.R = R;
  p.partial = static_cast<float*>(workspace);
  return done(launch_block_product(p, static_cast<hipStream_t>(stream)));
}

// Results that are quantized again are made from exact sums.
static bool gated_f8(uint32_t flags, bool codes, bool kept) { return (flags & SRQ_FLAG_F8_PIPELINE) && !codes && !kept; }

size_t sr_gated_fwd_workspace_bytes(size_t M, size_t F, size_t K, uint32_t flags) {
  if (F == 0 || K == 0 || F > WIDEST || !features_ok(M, 2 * F) || K > LONGEST) return 0;
  return std::max(gated_forward_workspace(M, F, K, 0), flags & SRQ_FLAG_F8_PIPELINE ? gated_forward_workspace(M, F, K, 1) : 0);
}

int sr_gated_fwd(void* h, void* h_scales, void* gu, void* gu_scales, const void* X, size_t pitchX, const void* scalesX, const void* W,
                 size_t pitchW, const void* scalesW, size_t M, size_t F, size_t K, int act, const srq_quant* qh, const srq_quant* qgu,
                 uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  for (const srq_quant* q : {qh, qgu}) {
    if (!q) continue;
    if (const int st = check_quantizer(q); st != SRQ_OK) return st;
    if (q->kind != SRQ_E4M3) return SRQ_ERR_UNSUPPORTED;
  }
  if (!act_ok(act) || (flags & ~(uint32_t)SRQ_FLAG_F8_PIPELINE)) return SRQ_ERR_FORMAT;
  if (F == 0 || K == 0 || F > WIDEST || !features_ok(M, 2 * F) || K > LONGEST) return SRQ_ERR_SHAPE;
  if (F % SBLOCK || K % 16) return SRQ_ERR_ALIGN;
  if (M == 0) return SRQ_OK;
  if (!h) return SRQ_ERR_NULL;
  if (!aligned(h, 16)) return SRQ_ERR_ALIGN;
  if (qh)
    if (const int st = check_blocks(h, F, h_scales, F); st != SRQ_OK) return st;
  if (qgu)
    if (const int st = check_blocks(gu, 2 * F, gu_scales, 2 * F); st != SRQ_OK) return st;
  if (const int st = check_blocks(X, pitchX, scalesX, K); st != SRQ_OK) return st;
  if (const int st = check_blocks(W, pitchW, scalesW, K); st != SRQ_OK) return st;
  if (pitchX > LONGEST || pitchW > LONGEST) return SRQ_ERR_SHAPE;
  GatedForward g = {};
  g.f8 = gated_f8(flags, qh != nullptr, qgu != nullptr);
  const size_t need = gated_forward_workspace(M, F, K, g.f8);
  if (need && (!workspace || workspace_bytes < need)) return SRQ_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  g.partial = static_cast<float*>(workspace);
  g.X = operand(X, pitchX, scalesX, K);
  g.W = operand(W, pitchW, scalesW, K);
  g.act = act;
  g.h = h;
  g.h_scales = qh ? static_cast<uint8_t*>(h_scales) : nullptr;
  g.gu = qgu ? static_cast<uint8_t*>(gu) : nullptr;
  g.gu_scales = qgu ? static_cast<uint8_t*>(gu_scales) : nullptr;
  g.M = (uint32_t)M;
  g.F = (uint32_t)F;
  g.K = (uint32_t)K;
  g.rnd_h = rounding(qh);
  g.rnd_gu = rounding(qgu);
  return done(launch_gated_forward(g, static_cast<hipStream_t>(stream)));
}

int sr_gated_bwd(void* dz, void* dz_scales, void* dz_t, size_t dz_t_pitch, void* dz_t_scales, const void* dH, int dtype, const void* gu,
                 const void* gu_scales, size_t M, size_t F, int act, const srq_quant* q, void* stream) {
  if (const int st = check_quantizer(q); st != SRQ_OK) return st;
  if (!dtype_ok(dtype) || !act_ok(act)) return SRQ_ERR_FORMAT;
  if (F == 0 || F > WIDEST || !features_ok(M, 2 * F) || (M + 127) / 128 * ((F + 127) / 128) > MOST_PAIRS) return SRQ_ERR_SHAPE;
  if (F % SBLOCK) return SRQ_ERR_ALIGN;
  if (M == 0) return SRQ_OK;
  if (!dH) return SRQ_ERR_NULL;
  if (!aligned(dH, 16)) return SRQ_ERR_ALIGN;
  if (const int st = check_blocks(dz, 2 * F, dz_scales, 2 * F); st != SRQ_OK) return st;
  if (const int st = check_blocks(dz_t, dz_t_pitch, dz_t_scales, M); st != SRQ_OK) return st;
  if (const int st = check_blocks(gu, 2 * F, gu_scales, 2 * F); st != SRQ_OK) return st;
  GatedBackward g = {};
  g.dh = dH;
  g.dtype = dtype;
  g.act = act;
  g.kind = q->kind;
  g.gu = static_cast<const uint8_t*>(gu);
  g.gu_scales = static_cast<const uint8_t*>(gu_scales);
  g.F = (uint32_t)F;
  g.out = tile_out(dz, 2 * F, dz_scales, dz_t, dz_t_pitch, dz_t_scales, M, 2 * F);
  g.rnd = rounding(q);
  return done(launch_gated_backward(g, static_cast<hipStream_t>(stream)));
}

int sr_rmsnorm_fwd(void* y, size_t y_pitch, void* y_scales, void* h, float* rstd, const void* x, const void* residual, const float* gamma,
                   int dtype, size_t M, size_t D, float eps, const srq_quant* q, void* stream) {
  if (q)
    if (const int st = check_quantizer(q); st != SRQ_OK) return st;
  if (!dtype_ok(dtype) || !(eps > 0.0f) || !std::isfinite(eps)) return SRQ_ERR_FORMAT;
  if (D == 0 || !size_ok(M, D)) return SRQ_ERR_SHAPE;
  if (D % 16) return SRQ_ERR_ALIGN;
  if (D > SRQ_RMSNORM_LONGEST) return SRQ_ERR_UNSUPPORTED;
  if (M == 0) return SRQ_OK;
  if (!y || !rstd || !x || !gamma || (residual && !h)) return SRQ_ERR_NULL;
  if (q)
    if (const int st = check_blocks(y, y_pitch, y_scales, D); st != SRQ_OK) return st;
  if (!aligned(y, 16) || !aligned(x, 16) || !aligned(gamma, 16) || !aligned(rstd, 4) || (residual && (!aligned(residual, 16) || !aligned(h, 16))))
    return SRQ_ERR_ALIGN;
  NormForward n = {};
  n.x = x;
  n.residual = residual;
  n.h = h;
  n.y = y;
  n.gamma = gamma;
  n.rstd = rstd;
  n.scales = q ? static_cast<uint8_t*>(y_scales) : nullptr;
  n.y_pitch = y_pitch;
  n.spitch = scale_pitch(D);
  n.dtype = dtype;
  n.kind = q ? q->kind : 0;
  n.rows = (uint32_t)M;
  n.cols = (uint32_t)D;
  n.eps = eps;
  n.rnd = rounding(q);
  return done(launch_norm_forward(n, static_cast<hipStream_t>(stream)));
}

size_t sr_rmsnorm_bwd_workspace_bytes(size_t M, size_t D) {
  if (D == 0 || !size_ok(M, D) || D > SRQ_RMSNORM_LONGEST) return 0;
  return norm_backward_partials((uint32_t)M, (uint32_t)D) * sizeof(float);
}

int sr_rmsnorm_bwd(void* dx, float* dgamma, const void* dy, const void* dh, const void* h, const float* rstd, const float* gamma, int dtype,
                   size_t M, size_t D, float beta, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype)) return SRQ_ERR_FORMAT;
  if (beta != 0.0f && beta != 1.0f) return SRQ_ERR_UNSUPPORTED;
  if (D == 0 || !size_ok(M, D)) return SRQ_ERR_SHAPE;
  if (D % 16) return SRQ_ERR_ALIGN;
  if (D > SRQ_RMSNORM_LONGEST) return SRQ_ERR_UNSUPPORTED;
  if (!dgamma || (M && (!dx || !dy || !h || !rstd || !gamma))) return SRQ_ERR_NULL;
  if (M && (!aligned(dx, 16) || !aligned(dy, 16) || !aligned(h, 16) || !aligned(gamma, 16) || !aligned(rstd, 4) || (dh && !aligned(dh, 16))))
    return SRQ_ERR_ALIGN;
  if (!aligned(dgamma, 4)) return SRQ_ERR_ALIGN;
  if (M && (!workspace || workspace_bytes < sr_rmsnorm_bwd_workspace_bytes(M, D))) return SRQ_ERR_WORKSPACE;
  if (M && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  NormBackward n = {};
  n.dy = dy;
  n.dh = dh;
  n.h = h;
  n.dx = dx;
  n.gamma = gamma;
  n.rstd = rstd;
  n.dgamma = dgamma;
  n.partial = static_cast<float*>(workspace);
  n.dtype = dtype;
  n.accumulate = beta != 0.0f;
  n.rows = (uint32_t)M;
  n.cols = (uint32_t)D;
  return done(launch_norm_backward(n, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
