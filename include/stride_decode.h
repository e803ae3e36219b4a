/*
 * stride_decode.h -- C ABI of the rollout's decode step around the scoring
 * path: what turns a layer's projections into attention over the cached prefix
 * and a step's logits into the tokens that stride_score_step then scores.
 *
 *   stride_qk_norm_rope(_backward)  norms of queries and keys for each head,
 *                                   with the position rotation (training);
 *   stride_kv_append                keys and values into a paged cache, norm
 *                                   and rotation on the way (serving);
 *   stride_tree_attention           attention of one token, a chain or a tree
 *                                   of drafted tokens over that cache;
 *   stride_attention_mass           what attention weight each cached slot gets,
 *                                   added up over steps;
 *   stride_kv_evict                 the slots of most weight into fewer pages;
 *   stride_logit_controls           penalties for repeated tokens, biases and
 *                                   grammar masks on logits;
 *   stride_sample                   temperature, top-k, top-p and min-p from
 *                                   given random numbers.
 *
 * The paper leaves this step to its rollout engine (Sec. 4.2 step 3: a restart
 * resumes from the cached prefix; Algorithm 1, inner turn loop).  The
 * conventions of stride.h hold: device pointers owned by the caller, host
 * structs read during the call only, no allocation, calls asynchronous on
 * `stream` and capturable, errors found on the device OR-ed into *dev_status,
 * kernels that never trap.
 *
 * Types: STRIDE_DTYPE_BF16 and STRIDE_DTYPE_F16 everywhere, STRIDE_DTYPE_F32
 * where a call says so.  Products, sums, norms and softmax statistics are held
 * in 32 bits; each result is rounded once to its type.  Attention rounds one
 * thing more: the softmax weights that its second product takes are of the
 * rows' type (see there).
 */
#ifndef STRIDE_DECODE_H_
#define STRIDE_DECODE_H_

#include "stride.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STRIDE_DTYPE_F16 2 /* IEEE half; this header's calls only */

#define STRIDE_DEV_POSITION 0x8 /* a position outside the rotation's tables: that token's rows are NaN, and sums over them */
#define STRIDE_DEV_NO_TOKEN 0x10 /* a row that has no token to sample: token -1, NaN log-prob */

#define STRIDE_DEV_BAD_CONTROL 0x20 /* a row's penalty that stride_logit_controls does not take: that row is NaN */

#define STRIDE_MAX_HEAD_DIM 1024 /* D of the norm, rotation and append calls */
#define STRIDE_MAX_ATTENTION_DIM 128 /* D of the attention call */
#define STRIDE_MAX_TREE 64       /* drafted tokens of a sequence under a tree mask (one bit each) */
#define STRIDE_MAX_TOP_P_VOCAB (1 << 23) /* V of a sampling call with a top_p: its masses are sums of 64 bits in units of 2^-40 */

/* Head rows [n_tokens, n_heads, D]: unit stride along D, any other strides (in
 * elements), so q, k and v may be views of one fused projection. */
typedef struct stride_head_rows {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
  int32_t n_heads;
} stride_head_rows;

/* What happens to a head row x of D components (host struct):
 *   u = x * (mean(x^2) + eps)^(-1/2) * weight   (u = x where weight is NULL)
 *   y = u, its first rot_dim components rotated in pairs by the angles of the
 *       token's position: (a, b) -> (a cos - b sin, a sin + b cos)
 * Pairs are (i, i + rot_dim/2), or (2i, 2i + 1) if interleaved; angle i, whose
 * cosine and sine are cos_table[pos * rot_dim/2 + i] and sin_table[...].  No
 * tables (NULL, rot_dim 0): no rotation.  Weights: [D], the rows' type. */
typedef struct stride_norm_rope {
  const void* q_weight; /* NULL: queries are not normalised */
  const void* k_weight; /* NULL: keys are not normalised */
  float eps;
  int32_t interleaved;
  int32_t rot_dim;        /* even, 0 <= rot_dim <= D */
  const int32_t* pos;     /* [n_tokens] position of each token, 0 <= pos < table_rows */
  const float* cos_table; /* [table_rows, rot_dim / 2] */
  const float* sin_table;
  int64_t table_rows;
} stride_norm_rope;

/* A paged cache of keys and values and the sequences in it (host struct).
 * Slot s of sequence b is row s % page_size of page
 * block_table[b * table_stride + s / page_size].  A page's element (row, head,
 * component) lies at page * page_stride + row * row_stride + head *
 * head_stride + component, in k as in v: either order of rows and heads.
 * Sequence b holds ctx_len[b] committed tokens; tokens tok_off[b] ..
 * tok_off[b+1]-1 of a call are its new ones, in slots ctx_len[b], ctx_len[b] + 1,
 * ...  (A sequence may have none.)  What lies in slots past those is not used,
 * whatever it holds. */
typedef struct stride_paged_cache {
  void* k;
  void* v;
  int64_t page_stride;
  int64_t row_stride;
  int64_t head_stride;
  int32_t n_pages;
  int32_t page_size;
  int32_t n_heads;            /* key/value heads */
  int32_t n_seqs;
  const int32_t* block_table; /* [n_seqs, table_stride] */
  int64_t table_stride;       /* pages that a sequence's row can hold */
  const int32_t* ctx_len;     /* [n_seqs] */
  const int32_t* tok_off;     /* [n_seqs + 1], tok_off[0] = 0, tok_off[n_seqs] = n_tokens */
} stride_paged_cache;

/* q_out = rotated, normed q; k_out likewise (see stride_norm_rope).  Types
 * BF16, F16, F32; D <= STRIDE_MAX_HEAD_DIM.  q or k may have no heads
 * (n_heads 0); an output may be its input. */
STRIDE_API int stride_qk_norm_rope(const stride_head_rows* q, const stride_head_rows* k,
                                   const stride_head_rows* q_out, const stride_head_rows* k_out,
                                   int32_t dtype, int64_t n_tokens, int32_t D,
                                   const stride_norm_rope* how, int32_t* dev_status, void* stream);

/* Workspace bytes of the backward call (256-byte aligned). */
STRIDE_API size_t stride_qk_norm_rope_backward_workspace_size(int64_t n_tokens, int32_t Hq,
                                                              int32_t Hk, int32_t D);

/* Gradients of the forward call at q, k (its inputs) given those of its
 * outputs: dq, dk (the rows' type) and, where the weight is given, dq_weight,
 * dk_weight (float [D], summed over tokens and heads in a fixed order;
 * nullable).  With r = (mean(x^2) + eps)^(-1/2), n = r x, R the rotation:
 *   du = R^T dy,  dweight = sum du * n,  g = du * weight,  dx = r (g - n mean(g n));
 *   dx = du without a weight.  dq may be dq_out, dk may be dk_out. */
STRIDE_API int stride_qk_norm_rope_backward(const stride_head_rows* dq_out, const stride_head_rows* dk_out,
                                            const stride_head_rows* q, const stride_head_rows* k,
                                            const stride_head_rows* dq, const stride_head_rows* dk,
                                            int32_t dtype, int64_t n_tokens, int32_t D,
                                            const stride_norm_rope* how, float* dq_weight,
                                            float* dk_weight, int32_t* dev_status, void* workspace,
                                            size_t workspace_bytes, void* stream);

/* Writes the new tokens' keys (normed with how->k_weight, rotated) and values
 * (as they are) into their slots.  In the same launch, where q has heads,
 * q_out = rotated, normed q.  Types BF16, F16, F32, the cache's and the rows'
 * alike; D <= STRIDE_MAX_HEAD_DIM; how NULL: plain copies.  A token whose slot
 * the block table does not hold (no such entry, or a page outside
 * [0, n_pages)), of no sequence, or of one of a negative ctx_len is not written
 * and sets STRIDE_DEV_BAD_LAYOUT.  Slots of two
 * tokens must differ. */
STRIDE_API int stride_kv_append(const stride_head_rows* k, const stride_head_rows* v,
                                const stride_head_rows* q, const stride_head_rows* q_out,
                                int32_t dtype, int64_t n_tokens, int32_t D,
                                const stride_norm_rope* how, const stride_paged_cache* cache,
                                int32_t* dev_status, void* stream);

/* Workspace bytes of stride_tree_attention for a call of n_tokens tokens
 * (256-byte aligned). */
STRIDE_API size_t stride_tree_attention_workspace_size(int64_t n_tokens, int32_t Hq, int32_t Hk, int32_t D);

/* Attention of the new tokens over the cache, the new tokens' own keys and
 * values in it (append them first).
 *
 * Token i of sequence b, query head h (of q->n_heads, a multiple of
 * cache->n_heads; kv head h / (n_heads / cache->n_heads)):
 *   s_j = scale * q . k_j  over the ctx_len[b] committed slots and the new
 *         tokens that it may see; out = sum_j softmax(s)_j v_j;
 *   lse = ln sum_j exp(s_j).
 * tree_mask NULL: a chain, token i sees the new tokens up to itself (any
 * number of them: also the prefill of a restart's new tokens over its reused
 * prefix).  Else tree_mask[i] (uint64 [n_tokens]): bit j set, it sees new
 * token j of its sequence, of which there are at most STRIDE_MAX_TREE (more:
 * STRIDE_DEV_BAD_LAYOUT, that sequence's rows NaN).  A row that sees nothing:
 * out 0, lse -inf.  Keys and values that a row does not see may hold anything,
 * NaN and infinities too: they change nothing in it.  A slot without a page:
 * STRIDE_DEV_BAD_LAYOUT and NaN rows.  STRIDE_DEV_TIMEOUT (a wait inside the
 * kernel ran out: not known to happen): out and lse of the whole call hold
 * nothing of use, and some of their rows may not have been written.
 *
 * The weights exp(s_j - max s) go into the second product rounded to the rows'
 * type (both operands of a tensor-core product are of one); their sum, and with
 * it lse, takes them unrounded.  A component of out is so
 * within u sum_j p_j |v_j| of the one that 32-bit weights give, p = softmax(s), u
 * half a unit in the last place (2^-8 BF16, 2^-11 F16), before its own rounding
 * (F16: plus 2^-38 max p sum_j |v_j|, its weights being whole from 2^-27 of the
 * largest on).
 *
 * One kernel takes the whole call, chosen by its mean of rows a sequence: a long
 * chain is best not in one call with many single tokens.
 *
 * Types BF16, F16; D a multiple of 8, at most STRIDE_MAX_ATTENTION_DIM; the
 * caches' base and strides whole 16-byte vectors (q and out too); n_tokens times
 * the group of query heads under 2^31 - 256.  lse: float [n_tokens, n_heads] or
 * NULL. */
STRIDE_API int stride_tree_attention(const stride_head_rows* q, const stride_head_rows* out, float* lse,
                                     int32_t dtype, int64_t n_tokens, int32_t D, float scale,
                                     const uint64_t* tree_mask, const stride_paged_cache* cache,
                                     int32_t* dev_status, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* Attention weight of cached slots (host struct): float [n_seqs, heads, slots]
 * of unit stride along the slots, other strides in elements; where it is written no two rows overlap.  Slot s is the
 * sequence's s-th, not a place in a page: sequences that share pages of a prefix
 * have weights of their own. */
typedef struct stride_slot_mass {
  float* data;
  int64_t seq_stride;
  int64_t head_stride;
  int64_t slots;
} stride_slot_mass;

/* Adds the attention weights of the call's new tokens to their sequences' slots.
 * Arguments as of stride_tree_attention, after it: lse is what it wrote.  For
 * sequence b and kv head h, over the new tokens i and the query heads g of h's
 * group, where i sees slot j:
 *   w_j = sum_i sum_g exp(scale * q_ig . k_j - lse_ig)
 *   mass_j = decay * mass_j + w_j   for the ctx_len[b] committed slots
 *            w_j                    for those of the new tokens
 * Slots past those, and sequences without new tokens, stay as they are.  decay >= 0; with 0
 * mass is not read (it may hold anything).  A row whose lse is -inf sees nothing
 * and adds nothing; keys that a row does not see may hold anything and change nothing
 * in its weights.  Sums are held in 32 bits, in an order that follows from the
 * sequence and from the mean of new tokens over the call's sequences alone: the same call gives the same bits.
 * Of itself a weight is off by what its score is, and 2^-24 (|score| + |lse|) + 2^-23 |score - lse| + 2^-22 at most.
 *
 * A slot without a page: NaN and STRIDE_DEV_BAD_LAYOUT.  Sequences of a length that
 * the block table or mass->slots does not hold, or, under a tree mask, of more than
 * STRIDE_MAX_TREE new tokens: STRIDE_DEV_BAD_LAYOUT, their mass stays as it is.
 * STRIDE_DEV_TIMEOUT (as of stride_tree_attention): masses of the whole call hold
 * nothing of use.
 *
 * One kernel takes the call, by the mean of new tokens: sequences of one token each and
 * long chains are faster in calls of their own.
 *
 * To let a prompt's last tokens alone vote, pass their rows of q and lse with ctx_len
 * moved on over the others and a decay of 0.
 *
 * Types and bounds of q and the cache as of stride_tree_attention (cache->v is not
 * used and may be NULL), n_tokens times the group of query heads at most 2^30; lse:
 * float [n_tokens, q->n_heads]. */
STRIDE_API int stride_attention_mass(const stride_head_rows* q, const float* lse, int32_t dtype, int64_t n_tokens,
                                     int32_t D, float scale, const uint64_t* tree_mask,
                                     const stride_paged_cache* cache, float decay, const stride_slot_mass* mass,
                                     int32_t* dev_status, void* stream);

/* What stride_kv_evict keeps of each sequence and kv head (host struct). */
typedef struct stride_evict_params {
  const int32_t* budget; /* [n_seqs] slots that remain, or NULL: budget_all for each.  Negative: the sequence is left out */
  int32_t budget_all;
  int32_t sink;          /* >= 0: of them, the first ones */
  int32_t recent;        /* >= 0: of them, the last ones */
  int32_t most;          /* slots that a row of `kept` and of mass_to holds */
} stride_evict_params;

/* Copies of each sequence of `from`, for each kv head by itself, the slots that
 * remain into the pages of `to`, in order.
 *
 * With n = from->ctx_len[b] and m = min(n, budget): the first a = min(m, sink)
 * slots, the last z = min(m - a, recent), and the m - a - z others of the largest
 * mass (ties: the lower slot; a NaN is below every number).  Slot number i of those,
 * counted from 0 in rising order of slots, goes to slot i of sequence b in `to`, and
 *   kept[b, h, i] = its slot in `from`,  mass_to[b, h, i] = its mass,  new_len[b] = m.
 * new_len is another array than from->ctx_len and budget.  kept: int32 [n_seqs, heads, most] and required; mass_to: stride_slot_mass of at least
 * `most` slots, nullable, not over mass.  What lies past m in kept, mass_to and the pages stays as
 * it is, and `from` is read only: pages that several sequences share (the prefix
 * that restarts reuse) stay whole.  So no page of `to` may be one that the call reads;
 * the pools may be the same.  The heads' slots hold different tokens from there on,
 * which attention does not mind (keys are rotated before they are cached): the next
 * tokens' positions go on counting, ctx_len goes on from new_len.
 *
 * A sequence that is left out: new_len[b] = ctx_len[b], nothing else is touched.  A
 * negative ctx_len, one that from's block table or mass->slots does not hold, an m above most or
 * what to's block table holds: STRIDE_DEV_BAD_LAYOUT, new_len[b] = -1, nothing else
 * is touched.  A slot without a page, on either side: STRIDE_DEV_BAD_LAYOUT, its row is
 * not copied.
 *
 * Types BF16, F16, F32; D <= STRIDE_MAX_HEAD_DIM; `to` has from's heads and sequences (page sizes and
 * strides may differ); tok_off of both and to->ctx_len are not used and may be NULL. */
STRIDE_API int stride_kv_evict(const stride_paged_cache* from, const stride_slot_mass* mass, const stride_paged_cache* to,
                               int32_t dtype, int32_t D, const stride_evict_params* how, int32_t* new_len,
                               int32_t* kept, const stride_slot_mass* mass_to, int32_t* dev_status, void* stream);

/* What stride_logit_controls does to a row of logits (host struct); every part
 * may be absent.  Per-row numbers are arrays [rows] or, where NULL, one value for all. */
typedef struct stride_logit_rules {
  const int32_t* history;     /* [rows, history_stride] tokens of each row's sequence; NULL: no penalties */
  int64_t history_stride;
  int32_t history_most;       /* columns that a row has: below 2^30 */
  const int32_t* history_len; /* [rows], 0 <= history_len <= history_most */
  const int32_t* prompt_len;  /* [rows] of which the prompt's; NULL: 0 */
  const float* repetition;    /* > 0; 1: none */
  float repetition_all;
  const float* frequency;     /* 0: none */
  float frequency_all;
  const float* presence;      /* 0: none */
  float presence_all;
  const int32_t* bias_off;    /* [rows + 1] each row's entries of bias_token and bias; NULL: no biases */
  const int32_t* bias_token;  /* [n_bias] */
  const float* bias;          /* [n_bias] */
  int32_t n_bias;
  const uint32_t* allowed;    /* [rows, allowed_stride]: bit j % 32 of word j / 32 set, token j is allowed; NULL: all */
  int64_t allowed_stride;     /* words; 0: one row for all */
} stride_logit_rules;

/* out = logits ([rows, ld], [rows, ld_out]; BF16, F16, F32; V at most STRIDE_MAX_VOCAB)
 * with these in turn, in 32 bits, rounded once:
 *   x = x > 0 ? x / repetition : x * repetition   tokens of the history
 *   x = x - frequency * count - presence          tokens generated (past the prompt) `count` > 0 times
 *   x = x + bias                                  listed tokens (of several entries the last)
 *   x = -inf                                      tokens that are not allowed
 * out may be logits, and must not overlap them otherwise; in place, logits that nothing applies to are
 * not read.  Separate, the raw logits stay for the scoring call.  A negative token in a history
 * or a list is padding.  One of V or more: STRIDE_DEV_TOKEN_RANGE, nothing else.  A
 * row's repetition that is not positive and finite, a frequency or presence that is
 * not finite: STRIDE_DEV_BAD_CONTROL; a history_len or a row's part of the lists out of
 * bounds: STRIDE_DEV_BAD_LAYOUT; the row is NaN. */
STRIDE_API int stride_logit_controls(const void* logits, int64_t ld, void* out, int64_t ld_out, int32_t dtype, int64_t V,
                                     int32_t rows, const stride_logit_rules* rules, int32_t* dev_status, void* stream);

/* A row's sampling parameters: each an array [rows] or, where that is NULL,
 * one value for all rows (host struct). */
typedef struct stride_sample_params {
  const float* temperature; /* >= 0; 0: the largest logit */
  float temperature_all;
  const int32_t* top_k; /* <= 0 or >= V: all */
  int32_t top_k_all;
  const float* top_p; /* >= 1: all */
  float top_p_all;
  const float* min_p; /* <= 0: all */
  float min_p_all;
} stride_sample_params;

/* Samples a token of each row of logits ([rows, ld], BF16, F16 or F32; V at
 * most STRIDE_MAX_VOCAB, STRIDE_MAX_TOP_P_VOCAB where a top_p is given, as an array
 * or a number below 1, and not all rows are of temperature 0).
 *
 * With m the row's largest logit, d_i = (x_i - m) / temperature and w_i =
 * exp(d_i), tokens ordered by falling logit, equal ones by rising index:
 *   A: the first top_k;  B: of A, those before which less than top_p of A's
 *   mass lies (the first always);  C: of B, those with w >= min(min_p, 1).
 * token = argmax over C of w_i / noise_i (ties: lowest index): with noise
 * (float [rows, ld_noise], > 0) of independent Exp(1) numbers, i is drawn with
 * probability w_i / sum_C w.  logp (nullable) = d_token - ln sum_C w, the
 * log-probability it was drawn with (temperature 0: the first token of the
 * order, logp 0; noise is not read, and may be NULL if temperature_all is 0 and
 * no array is given).
 * A logit of -inf is never drawn.  The type's lowest value is a logit like any
 * other: as a mask it has weight 0 where it lies 104 temperatures or more below
 * the row's largest logit (F16's -65504 beside logits around 0: at temperatures
 * up to 600).  Masses, and the weights that min_p is compared with, are of
 * approximate exponentials: a token whose weight is within 1e-5 (relative) of min_p
 * may fall on either side, as may one before which the mass is within 1e-5 of
 * top_p.  A row without a finite logit, with a NaN or +inf logit, a NaN, negative
 * or infinite temperature, a NaN top_p or min_p, or no positive ratio: token -1,
 * logp NaN, STRIDE_DEV_NO_TOKEN. */
STRIDE_API int stride_sample(const void* logits, int32_t dtype, int64_t ld, int64_t V, int32_t rows,
                             const float* noise, int64_t ld_noise, const stride_sample_params* params,
                             int32_t* tokens, float* logp, int32_t* dev_status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STRIDE_DECODE_H_ */
