// decode_api.cu -- the C ABI of include/stride_decode.h: host-side argument
// checks and kernel launches.  No allocation, no synchronisation, no CPU
// fallback.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "decode_internal.h"

namespace {

using namespace stride;

size_t elem_bytes(int32_t dtype) {
  return dtype == STRIDE_DTYPE_BF16 || dtype == STRIDE_DTYPE_F16 ? 2 : dtype == STRIDE_DTYPE_F32 ? 4 : 0;
}

bool multiple(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Checked head rows; an absent set is one without heads.
struct Rows {
  stride_head_rows r = {nullptr, 0, 0, 0};
  explicit Rows(const stride_head_rows* p) {
    if (p) r = *p;
  }
  bool valid(int64_t n_tokens, size_t e) const {
    return r.n_heads >= 0 && (r.n_heads == 0 || n_tokens == 0 || (r.data && multiple(r.data, e)));
  }
  // Every row starts at a multiple of c elements.
  bool whole(int64_t n_tokens, int c, size_t e) const {
    if (r.n_heads == 0) return true;
    return multiple(r.data, c * e) && (n_tokens <= 1 || r.token_stride % c == 0) && (r.n_heads <= 1 || r.head_stride % c == 0);
  }
};

int check_how(const stride_norm_rope& how, int32_t D) {
  if (how.rot_dim < 0 || how.rot_dim > D || how.rot_dim % 2 != 0) return STRIDE_ERR_INVALID_ARG;
  if (how.rot_dim > 0 && (!how.pos || !how.cos_table || !how.sin_table || how.table_rows < 1)) return STRIDE_ERR_INVALID_ARG;
  if ((how.q_weight || how.k_weight) && !(how.eps >= 0.f)) return STRIDE_ERR_INVALID_ARG;
  return STRIDE_OK;
}

int check_shape(int32_t dtype, int64_t n_tokens, int32_t D) {
  if (elem_bytes(dtype) == 0) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (n_tokens < 0 || n_tokens > INT32_MAX || D < 1 || D > STRIDE_MAX_HEAD_DIM) return STRIDE_ERR_INVALID_ARG;
  return STRIDE_OK;
}

int check_cache(const stride_paged_cache* c, size_t e) {
  if (!c || !c->k || !c->v || !multiple(c->k, e) || !multiple(c->v, e) || c->n_pages < 1 || c->page_size < 1 || c->n_heads < 1 || c->n_seqs < 1 || c->table_stride < 1 ||
      !c->block_table || !c->ctx_len || !c->tok_off)
    return STRIDE_ERR_INVALID_ARG;
  return STRIDE_OK;
}

PagedCache view(const stride_paged_cache& c) {
  return {c.k,      c.v,        c.page_stride,  c.row_stride,   c.head_stride, c.n_pages, c.page_size,
          c.n_heads, c.n_seqs, c.block_table, c.table_stride, c.ctx_len,     c.tok_off};
}

bool cache_whole(const stride_paged_cache& c, int n, size_t e) {
  return multiple(c.k, n * e) && multiple(c.v, n * e) && (c.n_pages <= 1 || c.page_stride % n == 0) &&
         (c.page_size <= 1 || c.row_stride % n == 0) && (c.n_heads <= 1 || c.head_stride % n == 0);
}

RowSet row_set(const Rows& x, const Rows& y, const void* w, const Rows* dy = nullptr) {
  RowSet s = {};
  s.x = x.r.data;
  s.x_tok = x.r.token_stride;
  s.x_head = x.r.head_stride;
  s.y = y.r.data;
  s.y_tok = y.r.token_stride;
  s.y_head = y.r.head_stride;
  s.w = w;
  s.heads = x.r.n_heads;
  if (dy) {
    s.dy = dy->r.data;
    s.dy_tok = dy->r.token_stride;
    s.dy_head = dy->r.head_stride;
  }
  return s;
}

void fill(NormRopeParams& p, const stride_norm_rope& how, int64_t n_tokens, int32_t D, int32_t* dev_status) {
  p.n_tokens = n_tokens;
  p.D = D;
  p.eps = how.eps;
  p.interleaved = how.interleaved != 0;
  p.rot_dim = how.rot_dim;
  p.pos = how.pos;
  p.cos_table = how.cos_table;
  p.sin_table = how.sin_table;
  p.table_rows = how.table_rows;
  p.dev_status = dev_status;
}

// The largest chunk (elements) that divides a row and, where halves are
// rotated, its halves.
int row_chunk(const stride_norm_rope& how, int32_t D, int c) {
  const int half = how.interleaved ? 0 : how.rot_dim / 2;
  while (c > 1 && (D % c != 0 || half % c != 0)) c /= 2;
  return c;
}

int done(cudaError_t e) { return e == cudaSuccess ? STRIDE_OK : STRIDE_ERR_CUDA; }

const stride_norm_rope kPlain = {nullptr, nullptr, 0.f, 0, 0, nullptr, nullptr, nullptr, 0};

}  // namespace

extern "C" {

int stride_qk_norm_rope(const stride_head_rows* q, const stride_head_rows* k, const stride_head_rows* q_out,
                        const stride_head_rows* k_out, int32_t dtype, int64_t n_tokens, int32_t D,
                        const stride_norm_rope* how, int32_t* dev_status, void* stream) {
  int rc = check_shape(dtype, n_tokens, D);
  if (rc != STRIDE_OK) return rc;
  const Rows Q(q), K(k), Qo(q_out), Ko(k_out);
  if (!how || !Q.valid(n_tokens, elem_bytes(dtype)) || !K.valid(n_tokens, elem_bytes(dtype)) || !Qo.valid(n_tokens, elem_bytes(dtype)) || !Ko.valid(n_tokens, elem_bytes(dtype)) || Q.r.n_heads != Qo.r.n_heads || K.r.n_heads != Ko.r.n_heads)
    return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_how(*how, D)) != STRIDE_OK) return rc;
  if (n_tokens == 0 || Q.r.n_heads + K.r.n_heads == 0) return STRIDE_OK;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  NormRopeParams p = {};
  p.q = row_set(Q, Qo, how->q_weight);
  p.k = row_set(K, Ko, how->k_weight);
  fill(p, *how, n_tokens, D, dev_status);
  const size_t es = elem_bytes(dtype);
  int c = row_chunk(*how, D, es == 2 ? 8 : 4);
  for (; c > 1; c /= 2)
    if (Q.whole(n_tokens, c, es) && K.whole(n_tokens, c, es) && Qo.whole(n_tokens, c, es) && Ko.whole(n_tokens, c, es) &&
        multiple(how->q_weight, c * es) && multiple(how->k_weight, c * es))
      break;
  return done(launch_norm_rope(p, dtype, c, false, sms, (cudaStream_t)stream));
}

size_t stride_qk_norm_rope_backward_workspace_size(int64_t n_tokens, int32_t Hq, int32_t Hk, int32_t D) {
  if (n_tokens <= 0 || D < 1 || D > STRIDE_MAX_HEAD_DIM || Hq < 0 || Hk < 0 || Hq + (int64_t)Hk == 0) return 0;
  return ((size_t)kNormRopeBackwardBlocks * D * sizeof(float) + 255) & ~(size_t)255;
}

int stride_qk_norm_rope_backward(const stride_head_rows* dq_out, const stride_head_rows* dk_out, const stride_head_rows* q,
                                 const stride_head_rows* k, const stride_head_rows* dq, const stride_head_rows* dk,
                                 int32_t dtype, int64_t n_tokens, int32_t D, const stride_norm_rope* how, float* dq_weight,
                                 float* dk_weight, int32_t* dev_status, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_shape(dtype, n_tokens, D);
  if (rc != STRIDE_OK) return rc;
  const Rows Q(q), K(k), Go(dq_out), Ho(dk_out), G(dq), H(dk);
  if (!how || !Q.valid(n_tokens, elem_bytes(dtype)) || !K.valid(n_tokens, elem_bytes(dtype)) || !Go.valid(n_tokens, elem_bytes(dtype)) || !Ho.valid(n_tokens, elem_bytes(dtype)) || !G.valid(n_tokens, elem_bytes(dtype)) || !H.valid(n_tokens, elem_bytes(dtype)) || Q.r.n_heads != Go.r.n_heads ||
      Q.r.n_heads != G.r.n_heads || K.r.n_heads != Ho.r.n_heads || K.r.n_heads != H.r.n_heads)
    return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_how(*how, D)) != STRIDE_OK) return rc;
  if ((dq_weight && !how->q_weight) || (dk_weight && !how->k_weight)) return STRIDE_ERR_INVALID_ARG;
  const bool rows = n_tokens > 0 && Q.r.n_heads + K.r.n_heads > 0;
  if (!rows && !dq_weight && !dk_weight) return STRIDE_OK;
  if (rows && (!workspace || workspace_bytes < stride_qk_norm_rope_backward_workspace_size(n_tokens, Q.r.n_heads, K.r.n_heads, D) ||
               !multiple(workspace, 256)))
    return STRIDE_ERR_WORKSPACE;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  NormRopeParams p = {};
  p.q = row_set(Q, G, how->q_weight, &Go);
  p.k = row_set(K, H, how->k_weight, &Ho);
  fill(p, *how, n_tokens, D, dev_status);
  p.dq_weight = dq_weight;
  p.dk_weight = dk_weight;
  p.partials = static_cast<float*>(workspace);
  const size_t es = elem_bytes(dtype);
  int c = row_chunk(*how, D, es == 2 ? 8 : 4);
  for (; c > 1; c /= 2) {
    bool ok = true;
    for (const Rows* r : {&Q, &K, &Go, &Ho, &G, &H}) ok = ok && r->whole(n_tokens, c, es);
    if (ok) break;
  }
  return done(launch_norm_rope_backward(p, dtype, c, (cudaStream_t)stream));
}

int stride_kv_append(const stride_head_rows* k, const stride_head_rows* v, const stride_head_rows* q,
                     const stride_head_rows* q_out, int32_t dtype, int64_t n_tokens, int32_t D, const stride_norm_rope* how,
                     const stride_paged_cache* cache, int32_t* dev_status, void* stream) {
  int rc = check_shape(dtype, n_tokens, D);
  if (rc != STRIDE_OK) return rc;
  if (!how) how = &kPlain;
  const Rows K(k), V(v), Q(q), Qo(q_out);
  if (!K.valid(n_tokens, elem_bytes(dtype)) || !V.valid(n_tokens, elem_bytes(dtype)) || !Q.valid(n_tokens, elem_bytes(dtype)) || !Qo.valid(n_tokens, elem_bytes(dtype)) || Q.r.n_heads != Qo.r.n_heads) return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_cache(cache, elem_bytes(dtype))) != STRIDE_OK) return rc;
  if (K.r.n_heads != cache->n_heads || V.r.n_heads != cache->n_heads) return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_how(*how, D)) != STRIDE_OK) return rc;
  if (n_tokens == 0) return STRIDE_OK;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  NormRopeParams p = {};
  p.q = row_set(Q, Qo, how->q_weight);
  p.k = row_set(K, K, how->k_weight);
  p.v = V.r.data;
  p.v_tok = V.r.token_stride;
  p.v_head = V.r.head_stride;
  p.cache = view(*cache);
  fill(p, *how, n_tokens, D, dev_status);
  const size_t es = elem_bytes(dtype);
  int c = row_chunk(*how, D, es == 2 ? 8 : 4);
  for (; c > 1; c /= 2)
    if (Q.whole(n_tokens, c, es) && K.whole(n_tokens, c, es) && V.whole(n_tokens, c, es) && Qo.whole(n_tokens, c, es) &&
        cache_whole(*cache, c, es) && multiple(how->q_weight, c * es) && multiple(how->k_weight, c * es))
      break;
  return done(launch_norm_rope(p, dtype, c, true, sms, (cudaStream_t)stream));
}

size_t stride_tree_attention_workspace_size(int64_t n_tokens, int32_t Hq, int32_t Hk, int32_t D) {
  if (n_tokens <= 0 || Hq < 1 || Hk < 1 || Hq % Hk != 0 || D < 8 || D > STRIDE_MAX_ATTENTION_DIM || D % 8 != 0) return 0;
  return attention_workspace_bytes(n_tokens, Hq, Hk, D);
}

int stride_tree_attention(const stride_head_rows* q, const stride_head_rows* out, float* lse, int32_t dtype, int64_t n_tokens,
                          int32_t D, float scale, const uint64_t* tree_mask, const stride_paged_cache* cache,
                          int32_t* dev_status, void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != STRIDE_DTYPE_BF16 && dtype != STRIDE_DTYPE_F16) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (n_tokens < 0 || n_tokens > INT32_MAX || D < 8 || D > STRIDE_MAX_ATTENTION_DIM || D % 8 != 0 || !isfinite(scale)) return STRIDE_ERR_INVALID_ARG;
  const Rows Q(q), O(out);
  int rc = check_cache(cache, elem_bytes(dtype));
  if (rc != STRIDE_OK) return rc;
  if (!Q.valid(n_tokens, elem_bytes(dtype)) || !O.valid(n_tokens, elem_bytes(dtype)) || Q.r.n_heads < 1 || O.r.n_heads != Q.r.n_heads || Q.r.n_heads % cache->n_heads != 0)
    return STRIDE_ERR_INVALID_ARG;
  if (!Q.whole(n_tokens, 8, 2) || !O.whole(n_tokens, 8, 2) || !cache_whole(*cache, 8, 2)) return STRIDE_ERR_INVALID_ARG;
  if (n_tokens * (Q.r.n_heads / cache->n_heads) > INT32_MAX - 256) return STRIDE_ERR_INVALID_ARG;
  if (n_tokens == 0) return STRIDE_OK;
  if (!workspace || workspace_bytes < attention_workspace_bytes(n_tokens, Q.r.n_heads, cache->n_heads, D) || !multiple(workspace, 256))
    return STRIDE_ERR_WORKSPACE;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  AttentionParams p = {};
  p.q = Q.r.data;
  p.q_tok = Q.r.token_stride;
  p.q_head = Q.r.head_stride;
  p.out = O.r.data;
  p.out_tok = O.r.token_stride;
  p.out_head = O.r.head_stride;
  p.lse = lse;
  p.n_tokens = n_tokens;
  p.Hq = Q.r.n_heads;
  p.D = D;
  p.scale = scale;
  p.tree_mask = tree_mask;
  p.cache = view(*cache);
  p.dev_status = dev_status;
  p.workspace = workspace;
  return done(launch_tree_attention(p, dtype, sms, (cudaStream_t)stream));
}

int stride_sample(const void* logits, int32_t dtype, int64_t ld, int64_t V, int32_t rows, const float* noise, int64_t ld_noise,
                  const stride_sample_params* params, int32_t* tokens, float* logp, int32_t* dev_status, void* stream) {
  if (elem_bytes(dtype) == 0) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (!params || rows < 0 || V < 1 || V > STRIDE_MAX_VOCAB || ld < V || (rows > 0 && (!logits || !tokens || !multiple(logits, elem_bytes(dtype)) || !multiple(noise, sizeof(float))))) return STRIDE_ERR_INVALID_ARG;
  const bool greedy = !params->temperature && params->temperature_all == 0.f;
  if (!greedy && V > STRIDE_MAX_TOP_P_VOCAB && (params->top_p || params->top_p_all < 1.f)) return STRIDE_ERR_INVALID_ARG;
  if (!greedy && ((rows > 0 && !noise) || ld_noise < V)) return STRIDE_ERR_INVALID_ARG;
  if (!params->temperature && !(params->temperature_all >= 0.f && isfinite(params->temperature_all))) return STRIDE_ERR_INVALID_ARG;
  if ((!params->top_p && isnan(params->top_p_all)) || (!params->min_p && isnan(params->min_p_all))) return STRIDE_ERR_INVALID_ARG;
  if (rows == 0) return STRIDE_OK;
  const int dc = check_device();
  if (dc != STRIDE_OK) return dc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  SampleParams p = {};
  p.x = logits;
  p.ld = ld;
  p.V = (int32_t)V;
  p.rows = rows;
  p.noise = noise;
  p.ld_noise = ld_noise;
  p.how = *params;
  p.tokens = tokens;
  p.logp = logp;
  p.dev_status = dev_status;
  return done(launch_sample(p, dtype, sms, (cudaStream_t)stream));
}

}  // extern "C"
