// decode_internal.h -- launch interfaces of the decode step's kernels
// (include/stride_decode.h), between the C-ABI layer and the kernels.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "stride_decode.h"
#include "stride_internal.h"

namespace stride {

// One set of head rows of a norm-and-rotation kernel: where they are read and
// written.
struct RowSet {
  const void* x;
  void* y;
  const void* w;   // [D] or NULL
  const void* dy;  // backward: gradient of the output
  int64_t x_tok, x_head, y_tok, y_head, dy_tok, dy_head;
  int32_t heads;
};

struct PagedCache {
  void* k;
  void* v;
  int64_t page_stride, row_stride, head_stride;
  int32_t n_pages, page_size, n_heads, n_seqs;
  const int32_t* block_table;
  int64_t table_stride;
  const int32_t* ctx_len;
  const int32_t* tok_off;
};

struct NormRopeParams {
  RowSet q, k;
  const void* v;  // append: values, copied as they are
  int64_t v_tok, v_head;
  int64_t n_tokens;
  int32_t D;
  float eps;
  int32_t interleaved, rot_dim;
  const int32_t* pos;
  const float* cos_table;
  const float* sin_table;
  int64_t table_rows;
  int32_t* dev_status;
  PagedCache cache;     // append: where the k and v rows go
  float* partials;      // backward: [blocks][D] weight-gradient sums
  float* dq_weight;     // backward, nullable
  float* dk_weight;
};

// Blocks of the backward kernel at most: partial weight gradients are one row
// of D floats each.
constexpr int kNormRopeBackwardBlocks = 608;

// chunk: elements per load that every row, pair half and stride is a multiple
// of (8, 4 or 1).
cudaError_t launch_norm_rope(const NormRopeParams& p, int dtype, int chunk, bool append, int sms, cudaStream_t stream);
cudaError_t launch_norm_rope_backward(const NormRopeParams& p, int dtype, int chunk, cudaStream_t stream);

struct AttentionParams {
  const void* q;
  int64_t q_tok, q_head;
  void* out;
  int64_t out_tok, out_head;
  float* lse;
  int64_t n_tokens;
  int32_t Hq, D;
  float scale;
  const uint64_t* tree_mask;
  PagedCache cache;
  int32_t* dev_status;
  void* workspace;
};
size_t attention_workspace_bytes(int64_t n_tokens, int Hq, int Hk, int D);
cudaError_t launch_tree_attention(const AttentionParams& p, int dtype, int sms, cudaStream_t stream);

struct SampleParams {
  const void* x;
  int64_t ld;
  int32_t V, rows;
  const float* noise;
  int64_t ld_noise;
  stride_sample_params how;
  int32_t* tokens;
  float* logp;
  int32_t* dev_status;
  bool long_first;  // rows without a top_k are started first
};
cudaError_t launch_sample(const SampleParams& p, int dtype, int sms, cudaStream_t stream);

}  // namespace stride
