// decode_api.cu -- the C ABI of include/stride_decode.h: host-side argument
// checks and kernel launches.  No allocation, no synchronisation, no CPU
// fallback.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <utility>

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

int check_mass(const stride_slot_mass* m) {
  return !m || !m->data || !multiple(m->data, sizeof(float)) || m->slots < 1 ? STRIDE_ERR_INVALID_ARG : STRIDE_OK;
}

// Sequences' and heads' slots, where they are written, are apart.
bool apart(const stride_slot_mass& m, const stride_paged_cache& c) {
  const auto size = [](int64_t x) { return x < 0 ? -x : x; };
  int64_t a = size(m.seq_stride), b = size(m.head_stride), n = c.n_heads;  // a: the larger of two
  if (c.n_seqs <= 1) return n <= 1 || b >= m.slots;
  if (n <= 1) return a >= m.slots;
  if (a < b) {
    std::swap(a, b);
    n = c.n_seqs;
  }
  return b >= m.slots && a >= m.slots && (a - m.slots) / b >= n - 1;
}

SlotMass view(const stride_slot_mass& m) { return {m.data, m.seq_stride, m.head_stride, m.slots}; }

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

int stride_attention_mass(const stride_head_rows* q, const float* lse, int32_t dtype, int64_t n_tokens, int32_t D, float scale,
                          const uint64_t* tree_mask, const stride_paged_cache* cache, float decay, const stride_slot_mass* mass,
                          int32_t* dev_status, void* stream) {
  if (dtype != STRIDE_DTYPE_BF16 && dtype != STRIDE_DTYPE_F16) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (n_tokens < 0 || n_tokens > INT32_MAX || D < 8 || D > STRIDE_MAX_ATTENTION_DIM || D % 8 != 0 || !isfinite(scale)) return STRIDE_ERR_INVALID_ARG;
  if (!cache || !(decay >= 0.f && isfinite(decay))) return STRIDE_ERR_INVALID_ARG;
  stride_paged_cache keys = *cache;
  keys.v = keys.k;
  const Rows Q(q);
  int rc = check_cache(&keys, elem_bytes(dtype));
  if (rc != STRIDE_OK) return rc;
  if ((rc = check_mass(mass)) != STRIDE_OK) return rc;
  if (!apart(*mass, keys)) return STRIDE_ERR_INVALID_ARG;
  if (!Q.valid(n_tokens, elem_bytes(dtype)) || Q.r.n_heads < 1 || Q.r.n_heads % keys.n_heads != 0) return STRIDE_ERR_INVALID_ARG;
  if (!Q.whole(n_tokens, 8, 2) || !cache_whole(keys, 8, 2)) return STRIDE_ERR_INVALID_ARG;
  if (n_tokens * (Q.r.n_heads / keys.n_heads) > (1 << 30)) return STRIDE_ERR_INVALID_ARG;
  if (n_tokens == 0) return STRIDE_OK;
  if (!lse || !multiple(lse, sizeof(float))) return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  MassParams p = {};
  p.a.q = Q.r.data;
  p.a.q_tok = Q.r.token_stride;
  p.a.q_head = Q.r.head_stride;
  p.a.n_tokens = n_tokens;
  p.a.Hq = Q.r.n_heads;
  p.a.D = D;
  p.a.scale = scale;
  p.a.tree_mask = tree_mask;
  p.a.cache = view(keys);
  p.a.dev_status = dev_status;
  p.lse = lse;
  p.decay = decay;
  p.mass = view(*mass);
  return done(launch_attention_mass(p, dtype, sms, (cudaStream_t)stream));
}

int stride_kv_evict(const stride_paged_cache* from, const stride_slot_mass* mass, const stride_paged_cache* to, int32_t dtype,
                    int32_t D, const stride_evict_params* how, int32_t* new_len, int32_t* kept, const stride_slot_mass* mass_to,
                    int32_t* dev_status, void* stream) {
  const size_t es = elem_bytes(dtype);
  if (es == 0) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (D < 1 || D > STRIDE_MAX_HEAD_DIM || !from || !to || !how || !new_len || !kept || new_len == from->ctx_len || new_len == how->budget) return STRIDE_ERR_INVALID_ARG;
  stride_paged_cache f = *from, t = *to;
  f.tok_off = f.ctx_len;  // (not used)
  t.tok_off = t.ctx_len = f.ctx_len;
  int rc = check_cache(&f, es);
  if (rc != STRIDE_OK) return rc;
  if ((rc = check_cache(&t, es)) != STRIDE_OK) return rc;
  if ((rc = check_mass(mass)) != STRIDE_OK || (mass_to && (rc = check_mass(mass_to)) != STRIDE_OK)) return rc;
  if (f.n_heads != t.n_heads || f.n_seqs != t.n_seqs || how->sink < 0 || how->recent < 0 || how->most < 1) return STRIDE_ERR_INVALID_ARG;
  if (mass_to && (mass_to->slots < how->most || mass_to->data == mass->data || !apart(*mass_to, f))) return STRIDE_ERR_INVALID_ARG;
  if ((int64_t)f.n_seqs * f.n_heads > INT32_MAX / 16) return STRIDE_ERR_INVALID_ARG;
  if ((rc = check_device()) != STRIDE_OK) return rc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  EvictParams p = {};
  p.from = view(f);
  p.to = view(t);
  p.mass = view(*mass);
  if (mass_to) p.mass_to = view(*mass_to);
  p.row_bytes = (int32_t)(D * es);
  p.how = *how;
  p.new_len = new_len;
  p.kept = kept;
  p.dev_status = dev_status;
  const int n = (int)(16 / es);
  const bool whole = D % n == 0 && cache_whole(f, n, es) && cache_whole(t, n, es);
  return done(launch_kv_evict(p, (int)es, whole ? 16 : (int)es, sms, (cudaStream_t)stream));
}

int stride_logit_controls(const void* logits, int64_t ld, void* out, int64_t ld_out, int32_t dtype, int64_t V, int32_t rows,
                          const stride_logit_rules* rules, int32_t* dev_status, void* stream) {
  const size_t es = elem_bytes(dtype);
  if (es == 0) return STRIDE_ERR_UNSUPPORTED_DTYPE;
  if (!rules || rows < 0 || V < 1 || V > STRIDE_MAX_VOCAB || ld < V || ld_out < V) return STRIDE_ERR_INVALID_ARG;
  const stride_logit_rules& r = *rules;
  if (rows > 0 && (!logits || !out || !multiple(logits, es) || !multiple(out, es))) return STRIDE_ERR_INVALID_ARG;
  if (logits == out && rows > 1 && ld != ld_out) return STRIDE_ERR_INVALID_ARG;
  if (r.history) {
    if (r.history_most < 0 || r.history_most >= (1 << 30) || (rows > 1 && r.history_stride < r.history_most) || !r.history_len) return STRIDE_ERR_INVALID_ARG;
    if (!r.repetition && !(r.repetition_all > 0.f && isfinite(r.repetition_all))) return STRIDE_ERR_INVALID_ARG;
    if ((!r.frequency && !isfinite(r.frequency_all)) || (!r.presence && !isfinite(r.presence_all))) return STRIDE_ERR_INVALID_ARG;
  }
  if (r.bias_off && (r.n_bias < 0 || (r.n_bias > 0 && (!r.bias_token || !r.bias)))) return STRIDE_ERR_INVALID_ARG;
  if (r.allowed && r.allowed_stride != 0 && r.allowed_stride < (V + 31) / 32) return STRIDE_ERR_INVALID_ARG;
  if (rows == 0) return STRIDE_OK;
  const int dc = check_device();
  if (dc != STRIDE_OK) return dc;
  cudaError_t e = cudaSuccess;
  const int sms = current_device_sms(nullptr, &e);
  if (sms <= 0) return STRIDE_ERR_CUDA;
  ControlParams p = {};
  p.x = logits;
  p.ld = ld;
  p.out = out;
  p.ld_out = ld_out;
  p.V = (int32_t)V;
  p.rows = rows;
  p.how = r;
  p.dev_status = dev_status;
  return done(launch_logit_controls(p, dtype, sms, (cudaStream_t)stream));
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
