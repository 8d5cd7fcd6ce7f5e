// Operators of a decoder around its products: attention, embedding, AdamW.  What the C interface hands to their launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/srq.h"

namespace srq {

// ---- attention --------------------------------------------------------------------------------------------------------
struct Heads {  // value d of head h at row t: p[t * row + h * head + d]
  uint16_t* p;
  size_t row, head;
};
struct AttentionShape {
  const int32_t *offsets_q, *offsets_k, *lengths_k;
  uint32_t sequences, rows_q, rows_k, heads_q, heads_kv, dim;
  float scale;
  int causal;
};
struct AttentionForward {
  AttentionShape shape;
  Heads o, q, k, v;
  float* lse;      // heads_q x rows_q
  float* partial;  // of the pieces of a sequence's keys, where they are cut
};
struct AttentionBackward {
  AttentionShape shape;
  Heads dq, dk, dv, dout, q, k, v, o;
  const float* lse;
  void* workspace;
};
size_t attention_forward_workspace(const AttentionShape& s);
hipError_t launch_attention_forward(const AttentionForward& f, hipStream_t stream);
size_t attention_backward_workspace(const AttentionShape& s);
hipError_t launch_attention_backward(const AttentionBackward& b, hipStream_t stream);

// ---- embedding --------------------------------------------------------------------------------------------------------
struct EmbedForward {
  void* out;
  const void* table;
  const void* ids;
  int out_dtype, dtype, wide;  // wide: ids of 8 bytes
  size_t rows, vocab;
  uint32_t cols;
  float scale;
};
hipError_t launch_embed_forward(const EmbedForward& e, hipStream_t stream);

struct EmbedBackward {
  float* dtable;
  const void* dy;
  const void* ids;
  int dtype, wide, accumulate;
  uint32_t rows, vocab, cols;
  float scale;
  int64_t padding;
  void* workspace;
};
size_t embed_backward_workspace(uint32_t rows, uint32_t cols);
hipError_t launch_embed_backward(const EmbedBackward& e, hipStream_t stream);

// ---- AdamW ------------------------------------------------------------------------------------------------------------
struct AdamWOptions {
  float lr, eps, beta1, rest1, beta2, rest2;  // rest: 1 - beta
  float log_beta1, log_beta2;
  const float* lr_dev;
  uint64_t step;
  const uint64_t* step_dev;
  const uint64_t* counter_dev;
  uint32_t k0, k1;
  int sr;
};
hipError_t launch_adamw(const srq_adamw_tensor* tensors, int count, const AdamWOptions& o, hipStream_t stream);

}  // namespace srq
