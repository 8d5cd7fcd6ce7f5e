// C ABI of the operators around a decoder's products: argument checks and the launches.
#include <algorithm>
#include <cmath>
#include <vector>

#include "srq_decoder.hpp"

using namespace srq;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool dtype_ok(int d) { return d == SRQ_F32 || d == SRQ_BF16; }
int done(hipError_t e) { return e == hipSuccess ? SRQ_OK : SRQ_ERR_HIP; }

// What the kernels' 32-bit indexes hold.
constexpr size_t MOST = 0x3FFFFFFF;

// ---- attention
int check_shape(const srq_attention* a) {
  if (!a) return SRQ_ERR_NULL;
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale) || (a->causal != 0 && a->causal != 1)) return SRQ_ERR_FORMAT;
  if (a->sequences == 0 || a->heads_q == 0 || a->heads_kv == 0 || a->dim == 0) return SRQ_ERR_SHAPE;
  if (a->sequences > MOST || a->rows_q > MOST || a->rows_k > MOST || a->heads_q > 65535 || a->heads_q % a->heads_kv) return SRQ_ERR_SHAPE;
  // (a launch, of fewer than 2^32 threads, has a workgroup for every head and piece of its rows: up to five times as many as this, of 256 threads)
  if ((a->rows_q / 32 + a->sequences + 1) * a->heads_q > MOST / 512 || (a->rows_k / 32 + a->sequences + 1) * a->heads_kv > MOST / 512) return SRQ_ERR_SHAPE;
  const bool same = a->offsets_q && !a->offsets_k;
  if (same && a->rows_q != a->rows_k) return SRQ_ERR_SHAPE;
  if ((!a->offsets_q && a->rows_q % a->sequences) || (!a->offsets_k && !same && a->rows_k % a->sequences)) return SRQ_ERR_SHAPE;
  if (a->dim % 8 || !aligned(a->offsets_q, 4) || !aligned(a->offsets_k, 4) || !aligned(a->lengths_k, 4)) return SRQ_ERR_ALIGN;
  return a->dim > 128 ? SRQ_ERR_UNSUPPORTED : SRQ_OK;
}
// A tensor of `rows` rows of heads; written: no two values at one place.
int check_heads(const srq_heads* h, size_t rows, size_t heads, size_t dim, bool written) {
  if (!h) return SRQ_ERR_NULL;
  if (rows == 0) return SRQ_OK;
  if (!h->p) return SRQ_ERR_NULL;
  if (!aligned(h->p, 16) || h->row % 8 || h->head % 8) return SRQ_ERR_ALIGN;
  if ((rows > 1 && h->row < dim) || (rows > 1 && h->row > SRQ_ATTENTION_WIDEST) || h->head > ((size_t)1 << 40)) return SRQ_ERR_SHAPE;
  if (written && heads > 1) {
    const bool within = h->head >= dim && (rows == 1 || (heads - 1) * h->head + dim <= h->row);  // the heads of a row side by side
    const bool apart = h->head >= (rows - 1) * h->row + dim;                                     // all rows of a head, then the next
    if (!within && !apart) return SRQ_ERR_SHAPE;
  }
  return SRQ_OK;
}
// (of a single row the stride is not looked at)
Heads heads(const srq_heads* h, size_t rows, size_t dim) { return {static_cast<uint16_t*>(h->p), rows > 1 ? h->row : dim, h->head}; }
AttentionShape shape(const srq_attention* a) {
  AttentionShape s = {};
  s.offsets_q = a->offsets_q;
  s.offsets_k = a->offsets_k ? a->offsets_k : a->offsets_q;
  s.lengths_k = a->lengths_k;
  s.sequences = (uint32_t)a->sequences;
  s.rows_q = (uint32_t)a->rows_q;
  s.rows_k = (uint32_t)a->rows_k;
  s.heads_q = (uint32_t)a->heads_q;
  s.heads_kv = (uint32_t)a->heads_kv;
  s.dim = (uint32_t)a->dim;
  s.scale = a->scale;
  s.causal = a->causal;
  return s;
}

}  // namespace

extern "C" {

size_t sr_attention_fwd_workspace_bytes(const srq_attention* a) {
  return check_shape(a) == SRQ_OK && a->rows_q ? attention_forward_workspace(shape(a)) : 0;
}

int sr_attention_fwd(const srq_heads* o, float* lse, const srq_heads* q, const srq_heads* k, const srq_heads* v, const srq_attention* a,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (const int st = check_shape(a); st != SRQ_OK) return st;
  if (const int st = check_heads(o, a->rows_q, a->heads_q, a->dim, true); st != SRQ_OK) return st;
  if (const int st = check_heads(q, a->rows_q, a->heads_q, a->dim, false); st != SRQ_OK) return st;
  for (const srq_heads* h : {k, v})
    if (const int st = check_heads(h, a->rows_k, a->heads_kv, a->dim, false); st != SRQ_OK) return st;
  if (a->rows_q == 0) return SRQ_OK;
  if (!lse) return SRQ_ERR_NULL;
  if (!aligned(lse, 4)) return SRQ_ERR_ALIGN;
  AttentionForward f = {};
  f.shape = shape(a);
  const size_t need = attention_forward_workspace(f.shape);
  if (need && (!workspace || workspace_bytes < need)) return SRQ_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  f.o = heads(o, a->rows_q, a->dim);
  f.q = heads(q, a->rows_q, a->dim);
  f.k = heads(k, a->rows_k, a->dim);
  f.v = heads(v, a->rows_k, a->dim);
  f.lse = lse;
  f.partial = static_cast<float*>(workspace);
  return done(launch_attention_forward(f, static_cast<hipStream_t>(stream)));
}

size_t sr_attention_bwd_workspace_bytes(const srq_attention* a) {
  return check_shape(a) == SRQ_OK && a->rows_q ? attention_backward_workspace(shape(a)) : 0;
}

int sr_attention_bwd(const srq_heads* dq, const srq_heads* dk, const srq_heads* dv, const srq_heads* do_, const srq_heads* q, const srq_heads* k,
                     const srq_heads* v, const srq_heads* o, const float* lse, const srq_attention* a, void* workspace, size_t workspace_bytes,
                     void* stream) {
  if (const int st = check_shape(a); st != SRQ_OK) return st;
  if (const int st = check_heads(dq, a->rows_q, a->heads_q, a->dim, true); st != SRQ_OK) return st;
  for (const srq_heads* h : {dk, dv})
    if (const int st = check_heads(h, a->rows_k, a->heads_kv, a->dim, true); st != SRQ_OK) return st;
  for (const srq_heads* h : {do_, q, o})
    if (const int st = check_heads(h, a->rows_q, a->heads_q, a->dim, false); st != SRQ_OK) return st;
  for (const srq_heads* h : {k, v})
    if (const int st = check_heads(h, a->rows_k, a->heads_kv, a->dim, false); st != SRQ_OK) return st;
  if (a->rows_q == 0 && a->rows_k == 0) return SRQ_OK;
  if (a->rows_q && !lse) return SRQ_ERR_NULL;
  if (!aligned(lse, 4)) return SRQ_ERR_ALIGN;
  AttentionBackward b = {};
  b.shape = shape(a);
  const size_t need = a->rows_q ? attention_backward_workspace(b.shape) : 0;
  if (need && (!workspace || workspace_bytes < need)) return SRQ_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  b.dq = heads(dq, a->rows_q, a->dim);
  b.dk = heads(dk, a->rows_k, a->dim);
  b.dv = heads(dv, a->rows_k, a->dim);
  b.dout = heads(do_, a->rows_q, a->dim);
  b.q = heads(q, a->rows_q, a->dim);
  b.k = heads(k, a->rows_k, a->dim);
  b.v = heads(v, a->rows_k, a->dim);
  b.o = heads(o, a->rows_q, a->dim);
  b.lse = lse;
  b.workspace = workspace;
  return done(launch_attention_backward(b, static_cast<hipStream_t>(stream)));
}

// ---- embedding

int sr_embedding_fwd(void* out, int out_dtype, const void* table, int dtype, const void* ids, int id_bytes, size_t M, size_t V, size_t D, float scale,
                     void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || (id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale)) return SRQ_ERR_FORMAT;
  if (V == 0 || D == 0 || M > MOST || V > MOST || D > MOST) return SRQ_ERR_SHAPE;
  if (D % 8) return SRQ_ERR_ALIGN;
  if (M == 0) return SRQ_OK;
  if (!out || !table || !ids) return SRQ_ERR_NULL;
  if (!aligned(out, 16) || !aligned(table, 16) || !aligned(ids, (size_t)id_bytes)) return SRQ_ERR_ALIGN;
  EmbedForward e = {};
  e.out = out;
  e.table = table;
  e.ids = ids;
  e.out_dtype = out_dtype;
  e.dtype = dtype;
  e.wide = id_bytes == 8;
  e.rows = M;
  e.vocab = V;
  e.cols = (uint32_t)D;
  e.scale = scale;
  return done(launch_embed_forward(e, static_cast<hipStream_t>(stream)));
}

size_t sr_embedding_bwd_workspace_bytes(size_t M, size_t D) {
  return M == 0 || D == 0 || M > MOST || D > MOST ? 0 : embed_backward_workspace((uint32_t)M, (uint32_t)D);
}

int sr_embedding_bwd(float* dtable, const void* dy, int dtype, const void* ids, int id_bytes, size_t M, size_t V, size_t D, float scale, int64_t padding,
                     float beta, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || (id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale) || padding < -1) return SRQ_ERR_FORMAT;
  if (beta != 0.0f && beta != 1.0f) return SRQ_ERR_UNSUPPORTED;
  // (blocks of 512 columns are the second dimension of a launch, of at most 65535; rows and table share the first)
  if (V == 0 || D == 0 || M > MOST || V > MOST || D > ((size_t)1 << 22) || (M / 8 + V / 64 + 2) * ((D + 2047) / 2048) > MOST / 64) return SRQ_ERR_SHAPE;
  if (D % 8) return SRQ_ERR_ALIGN;
  if (!dtable || (M && (!dy || !ids))) return SRQ_ERR_NULL;
  if (!aligned(dtable, 16) || (M && (!aligned(dy, 16) || !aligned(ids, (size_t)id_bytes)))) return SRQ_ERR_ALIGN;
  const size_t need = sr_embedding_bwd_workspace_bytes(M, D);
  if (need && (!workspace || workspace_bytes < need)) return SRQ_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return SRQ_ERR_ALIGN;
  EmbedBackward e = {};
  e.dtable = dtable;
  e.dy = dy;
  e.ids = ids;
  e.dtype = dtype;
  e.wide = id_bytes == 8;
  e.accumulate = beta != 0.0f;
  e.rows = (uint32_t)M;
  e.vocab = (uint32_t)V;
  e.cols = (uint32_t)D;
  e.scale = scale;
  e.padding = padding;
  e.workspace = workspace;
  return done(launch_embed_backward(e, static_cast<hipStream_t>(stream)));
}

// ---- AdamW

int sr_adamw(const srq_adamw_tensor* tensors, int count, const srq_adamw* options, void* stream) {
  if (!options || (count > 0 && !tensors)) return SRQ_ERR_NULL;
  const srq_adamw& p = *options;
  if (count < 0) return SRQ_ERR_SHAPE;
  const auto beta_ok = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!beta_ok(p.beta1) || !beta_ok(p.beta2) || !std::isfinite(p.lr) || !std::isfinite(p.eps) || p.eps < 0.0f || p.reserved) return SRQ_ERR_FORMAT;
  if (p.round != SRQ_SR && p.round != SRQ_RTN) return SRQ_ERR_FORMAT;
  if (!p.step_dev && p.step == 0) return SRQ_ERR_FORMAT;
  if (!aligned(p.lr_dev, 4) || !aligned(p.step_dev, 8) || !aligned(p.counter_dev, 8)) return SRQ_ERR_ALIGN;
  typedef std::pair<uintptr_t, uintptr_t> Range;
  std::vector<Range> written;
  try {
    written.reserve((size_t)count * 5);
  } catch (...) {
    return SRQ_ERR_SHAPE;
  }
  const auto add = [&](const void* at, size_t bytes) { written.push_back({reinterpret_cast<uintptr_t>(at), reinterpret_cast<uintptr_t>(at) + bytes}); };
  for (int i = 0; i < count; ++i) {
    const srq_adamw_tensor& t = tensors[i];
    if (!dtype_ok(t.w_dtype) || !dtype_ok(t.g_dtype) || !std::isfinite(t.weight_decay)) return SRQ_ERR_FORMAT;
    if (t.state_kind != SRQ_NONE && t.state_kind != SRQ_E4M3) return t.state_kind > SRQ_NONE && t.state_kind <= SRQ_E4M0 ? SRQ_ERR_UNSUPPORTED : SRQ_ERR_FORMAT;
    if (t.n > (size_t)1 << 40) return SRQ_ERR_SHAPE;
    if (t.n == 0) continue;
    const bool narrow = t.state_kind != SRQ_NONE;
    if (!t.w || !t.g || !t.m || !t.v || (narrow && (!t.m_scales || !t.v_scales))) return SRQ_ERR_NULL;
    if (!aligned(t.w, 16) || !aligned(t.g, 16) || !aligned(t.m, 16) || !aligned(t.v, 16)) return SRQ_ERR_ALIGN;
    add(t.w, t.n * (t.w_dtype == SRQ_F32 ? 4 : 2));
    add(t.m, t.n * (narrow ? 1 : 4));
    add(t.v, t.n * (narrow ? 1 : 4));
    if (narrow) add(t.m_scales, (t.n + 127) / 128), add(t.v_scales, (t.n + 127) / 128);
  }
  std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].first < written[i - 1].second) return SRQ_ERR_UNSUPPORTED;
  AdamWOptions o = {};
  o.lr = p.lr;
  o.eps = p.eps;
  o.beta1 = (float)p.beta1;
  o.rest1 = (float)(1.0 - p.beta1);
  o.beta2 = (float)p.beta2;
  o.rest2 = (float)(1.0 - p.beta2);
  o.log_beta1 = (float)std::log(p.beta1);
  o.log_beta2 = (float)std::log(p.beta2);
  o.lr_dev = p.lr_dev;
  o.step = p.step;
  o.step_dev = p.step_dev;
  o.counter_dev = p.counter_dev;
  o.k0 = (uint32_t)p.seed;
  o.k1 = (uint32_t)(p.seed >> 32);
  o.sr = p.round == SRQ_SR;
  return done(launch_adamw(tensors, count, o, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
