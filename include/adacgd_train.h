/*
 * adacgd_train.h -- operators of a worker's local training step.
 *
 * adacgd.h starts from a worker's gradient X_i = grad f_i(x).  When f_i is the loss of a language model the worker
 * fine-tunes, that gradient comes out of matrix products (a library's) and of the operators below, which stand between
 * and behind those products: the embedding lookup and its gradient, norm and rotation of queries and keys, attention,
 * layer norm with the residual sum and dropout in front of it, dropout on its own, the
 * log-probabilities of given tokens, and the two losses a fine-tuning worker minimises -- the preference loss over
 * pairs of answers (the logistic loss of a margin, as in Section 6 of the paper, with a.x replaced by a paired log
 * ratio) and the clipped policy loss with a KL term -- with their gradients with respect to the logits.
 *
 * Conventions, where they differ from or add to those of adacgd.h
 *   - A context (adacgd_train) owns nothing on the device: the caller gives it a workspace, which it must not share
 *     with another context.  All work is enqueued on the stream given to adacgd_train_init; no call synchronises.
 *     Inputs have to be ready, and outputs are ready, in that stream's order.  One call at a time per context, captured
 *     ones too: graphs with calls of one context are replayed one after the other.
 *   - A context is bound to the device that was current at adacgd_train_init, as adacgd_ctx is.
 *   - Matrices are row-major with a row stride in elements and unit column stride; vectors are contiguous.  No
 *     alignment beyond the element's own is needed; rows aligned to 16 bytes
 *     (32 for binary32), or misaligned alike, are faster.
 *   - Element types: binary32, binary16, bfloat16 (ADACGD_F32, _F16, _BF16).  All sums, statistics, probabilities and
 *     logarithms are kept in binary32 or binary64 and a result is rounded once, to its own type, when it is stored.
 *   - An output may be the very same matrix (pointer and stride) as an input unless a call says otherwise; other
 *     overlaps of an output with anything return ADACGD_ERR_INVALID_ARG.
 *   - Results do not depend on the order in which blocks run: there are no floating-point atomics, and the same call
 *     on the same inputs gives the same bits.
 *   - Zero rows are valid: sums are then zero.  Inf and NaN follow the formulas, row by row; rows that a mask excludes
 *     are never read, so nothing in them reaches a result.
 */
#ifndef ADACGD_TRAIN_H
#define ADACGD_TRAIN_H

#include "adacgd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct adacgd_train adacgd_train; /* opaque; created by adacgd_train_init, released by adacgd_train_destroy */

#define ADACGD_F32 0
#define ADACGD_F16 1
#define ADACGD_BF16 2

#define ADACGD_TRAIN_MAX_COLS 32768 /* widest row of adacgd_layer_norm and its backward pass */
#define ADACGD_TRAIN_MAX_RUN (2147483648ll - 16777216ll) /* most tokens of a lookup's gradient, of attention and its backward pass: 2^31 - 2^24 */

/* Bytes of device workspace for calls of at most max_tokens rows (of a norm's backward pass, or of logits; sequences
 * count as rows too) and norms of at most max_cols columns. */
adacgd_status adacgd_train_workspace_bytes(int64_t max_tokens, int64_t max_cols, size_t* bytes_out);

/* workspace_dev: dev, 256-byte aligned, caller-owned, must outlive the context.  Clears a part of it on the stream. */
adacgd_status adacgd_train_init(adacgd_train** out, int64_t max_tokens, int64_t max_cols, void* workspace_dev,
                                size_t workspace_bytes, void* cuda_stream);
void adacgd_train_destroy(adacgd_train* t);

/* Message of the last failure on this context (NULL: of the last failed call without one on this thread).  Never NULL. */
const char* adacgd_train_last_error(const adacgd_train* t);

/* Number of kernels launched on behalf of t since init. */
int64_t adacgd_train_launch_count(const adacgd_train* t);

/* Dropout.  No mask is stored: whether an element is kept is a function of (seed, offset, its number).  Element number
 * i = row * cols + col belongs to block i / 8; the block's 128 random bits are Philox4x32-10 (Salmon, Moraes, Dror,
 * Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) of the counter (i / 8, offset), two 64-bit numbers, low
 * words first, under the key `seed`; element i takes the (i mod 8)-th 16-bit half, low halves first, and is kept when it
 * is at least thr = floor(65536 p + 1/2).  Kept elements are multiplied by 65536 / (65536 - thr), so the expectation is
 * exact for the probability thr / 65536 that is realised; p below 2^-17 drops nothing, p = 1 everything.  A dropped
 * element is 0 even where the input is Inf or NaN.  The backward pass is the same call on the gradient, with the same
 * seed and offset.  Calls that should be independent take different offsets (or seeds). */
typedef struct {
  double p;        /* in [0, 1] */
  uint64_t seed;
  uint64_t offset;
} adacgd_drop;

/* out = [residual +] drop(x). */
typedef struct {
  int64_t rows, cols;
  const void* x;        int64_t x_stride;
  const void* residual; int64_t residual_stride; /* or NULL */
  void* out;            int64_t out_stride;
  int32_t dtype;        /* of x, residual and out */
  int32_t reserved;     /* must be 0 */
  adacgd_drop drop;
} adacgd_dropout_args;
adacgd_status adacgd_dropout(adacgd_train* t, const adacgd_dropout_args* a);

/* Layer norm of each row of s = residual + drop(x):
 *   mu = mean(s), rstd = (mean((s - mu)^2) + eps)^(-1/2), out = (s - mu) rstd weight + bias. */
typedef struct {
  int64_t rows, cols;   /* cols <= ADACGD_TRAIN_MAX_COLS */
  const void* x;        int64_t x_stride;
  const void* residual; int64_t residual_stride; /* or NULL: s = drop(x) */
  void* out;            int64_t out_stride;
  void* sum;            int64_t sum_stride;      /* s, for the next block's residual and the backward pass; or NULL */
  const void* weight;   /* [cols] or NULL (1) */
  const void* bias;     /* [cols] or NULL (0) */
  float* mean;          /* [rows] or NULL */
  float* rstd;          /* [rows] or NULL */
  int32_t dtype;        /* of x, residual, out and sum */
  int32_t param_dtype;  /* of weight and bias: dtype or ADACGD_F32 */
  float eps;
  int32_t reserved;     /* must be 0 */
  adacgd_drop drop;     /* p = 0: none */
} adacgd_norm_args;
adacgd_status adacgd_layer_norm(adacgd_train* t, const adacgd_norm_args* a);

/* Backward pass.  s, mean and rstd are what the forward pass stored (s = x where there was neither residual nor dropout):
 *   h = (s - mean) rstd,  g = dout weight,  ds = rstd (g - mean(g) - h mean(g h)) + dsum,
 *   dresidual = ds,  dx = drop(ds),  dweight = sum_rows dout h,  dbias = sum_rows dout.
 * Row sums run in a fixed order in binary32 chains, which are joined in binary64. */
typedef struct {
  int64_t rows, cols;
  const void* dout;     int64_t dout_stride;
  const void* s;        int64_t s_stride;
  const void* dsum;     int64_t dsum_stride;      /* gradient that reaches s from elsewhere (the residual stream), or NULL */
  void* dx;             int64_t dx_stride;
  void* dresidual;      int64_t dresidual_stride; /* or NULL (p = 0: dx is the same) */
  const float* mean;    /* [rows] */
  const float* rstd;    /* [rows] */
  const void* weight;   /* [cols] or NULL (1) */
  void* dweight;        /* [cols] or NULL, param_dtype */
  void* dbias;          /* [cols] or NULL, param_dtype */
  int32_t dtype;        /* of dout, s, dsum, dx and dresidual */
  int32_t param_dtype;
  adacgd_drop drop;     /* as in the forward pass */
} adacgd_norm_backward_args;
adacgd_status adacgd_layer_norm_backward(adacgd_train* t, const adacgd_norm_backward_args* a);

/* Logits of `tokens` rows over a vocabulary, the token each row should predict, and which rows count.  The tokens of
 * sequence q are rows [seq_start[q], seq_start[q + 1]), or, with seq_start = NULL, rows [q L, (q + 1) L) with
 * L = tokens / sequences (which must divide).  seq_start lives on the device and is trusted to ascend from 0 to `tokens`
 * as far as results go; positions outside [0, tokens] are cut off there, nothing is read out of bounds.
 * A label outside [0, vocab) on a row that counts makes that row's log-probability, and what depends on it, NaN. */
typedef struct {
  int64_t tokens, vocab;
  const void* logits;   int64_t logits_stride;
  const void* labels;   /* [tokens] int64 or int32 */
  const uint8_t* mask;  /* [tokens], non-zero = counts; NULL: all count */
  const int32_t* seq_start; /* [sequences + 1] or NULL */
  int64_t sequences;    /* >= 1; not used by adacgd_token_logp */
  int32_t dtype;        /* of logits and dlogits */
  int32_t label_bytes;  /* 8 or 4 */
} adacgd_token_rows;

/* logp[t] = logits[t][label] - log sum_j exp(logits[t][j]) for rows that count, 0 for the others.  lse (the logarithm
 * of the sum, 0 for rows that do not count) may be NULL. */
adacgd_status adacgd_token_logp(adacgd_train* t, const adacgd_token_rows* rows, float* logp, float* lse);

/* Preference loss.  Sequences 0 .. S/2 - 1 are the preferred answers, S/2 + p the rejected answer of pair p.  With
 * d_q = sum over q's counted tokens of (logp - ref_logp) (their mean if length_normalized),
 *   h_p = beta (d_p - d_{S/2 + p}),   loss = mean_p l(h_p),
 *   SIGMOID  l = -(1 - e) log sigma(h) - e log sigma(-h), e = label_smoothing
 *   HINGE    l = max(0, 1 - h)
 *   SQUARE   l = (h / beta - 1 / (2 beta))^2
 * A sequence without counted tokens has d_q = 0.  With e = 0 the second logarithm is left out, infinite or not.  The
 * differences are taken token by token because the two sums are large and nearly equal. */
#define ADACGD_PREF_SIGMOID 0
#define ADACGD_PREF_HINGE 1
#define ADACGD_PREF_SQUARE 2
typedef struct {
  adacgd_token_rows rows;   /* sequences even */
  const float* ref_logp;    /* [tokens] the reference model's log-probabilities (adacgd_token_logp) */
  void* dlogits;            int64_t dlogits_stride; /* grad_scale * dloss/dlogits, or NULL (loss only) */
  float* loss;              /* [1] */
  float* margin;            /* [sequences / 2] h_p, or NULL */
  float* seq_logp;          /* [sequences] sum (mean) of logp, or NULL */
  float beta;               /* > 0 */
  float label_smoothing;    /* in [0, 0.5], SIGMOID only */
  float grad_scale;
  int32_t kind;             /* ADACGD_PREF_* */
  int32_t length_normalized;
  int32_t reserved;         /* must be 0 */
} adacgd_preference_args;
adacgd_status adacgd_preference_loss(adacgd_train* t, const adacgd_preference_args* a);

/* Clipped policy loss with a KL term.  With r = exp(logp - old_logp), A the token's advantage and u = ref_logp - logp,
 *   l_t = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_beta (exp(u) - u - 1),   loss = sum_t w_t l_t,
 * w_t = 1 / (counted tokens), or with per_sequence 1 / (sequences with a counted token * counted tokens of t's sequence).
 * Where the clipped term is the smaller one its gradient is zero; where the two are equal the gradient is the first's.
 * No counted token: loss 0.  kl_beta = 0 leaves the KL term out of loss and gradient, with ref_logp or without. */
typedef struct {
  adacgd_token_rows rows;
  const float* old_logp;    /* [tokens] log-probabilities under the policy that answered */
  const float* advantages;  /* [tokens] */
  const float* ref_logp;    /* [tokens] or NULL */
  void* dlogits;            int64_t dlogits_stride; /* grad_scale * dloss/dlogits, or NULL */
  float* loss;              /* [1] */
  float* logp;              /* [tokens] as adacgd_token_logp, or NULL */
  float* stats;             /* [3] or NULL: over counted tokens the mean of exp(u) - u - 1 (0 without ref_logp), the share
                               whose gradient is clipped away, and their number */
  float clip_low, clip_high; /* in [0, 1] and >= 0 */
  float kl_beta;            /* >= 0 */
  float grad_scale;
  int32_t per_sequence;
  int32_t reserved;         /* must be 0 */
} adacgd_policy_args;
adacgd_status adacgd_policy_loss(adacgd_train* t, const adacgd_policy_args* a);

/* Embedding lookup: out[t] = scale * table[ids[t]] for tokens that count, 0 for the others.  An id outside [0, vocab) on a
 * token that counts makes that row NaN. */
typedef struct {
  int64_t tokens, vocab, cols;
  const void* ids;      /* [tokens] int64 or int32 */
  const uint8_t* mask;  /* [tokens], non-zero = counts; NULL: all count */
  const void* table;    int64_t table_stride;
  void* out;            int64_t out_stride;
  float scale;          /* finite */
  int32_t dtype;        /* of table and out */
  int32_t id_bytes;     /* 8 or 4 */
  int32_t reserved;     /* must be 0 */
} adacgd_embedding_args;
adacgd_status adacgd_embedding(adacgd_train* t, const adacgd_embedding_args* a);

/* Gradient of the lookup: dtable[v] = [base[v] +] scale * sum of dout[t] over the tokens t that count and have ids[t] = v.
 * The tokens of one id are summed in the order of the batch, in pieces: binary32 chains of at most max(16, tokens / 592) rows (1024 where
 * tokens <= 1024 and cols <= 1024), joined in binary32 in order.  Ids outside [0, vocab) add to nothing.  Every row of dtable is written,
 * unless base is the very same matrix: then rows without tokens stay as they are.  tokens <= max_tokens and ADACGD_TRAIN_MAX_RUN, cols <= max_cols. */
typedef struct {
  int64_t tokens, vocab, cols;
  const void* ids;
  const uint8_t* mask;
  const void* dout;     int64_t dout_stride;
  const void* base;     int64_t base_stride;     /* or NULL */
  void* dtable;         int64_t dtable_stride;
  float scale;
  int32_t dtype;        /* of dout */
  int32_t table_dtype;  /* of base and dtable: dtype or ADACGD_F32 */
  int32_t id_bytes;
} adacgd_embedding_backward_args;
adacgd_status adacgd_embedding_backward(adacgd_train* t, const adacgd_embedding_backward_args* a);

/* Norm and rotation of queries and keys.  A row holds its heads side by side, head_dim elements each.  With x a head,
 *   n = x (mean(x^2) + eps)^(-1/2) weight,
 * and the first 2 pairs elements of n are turned in pairs (a, b), by the angle position * freq[i] for pair i:
 *   a' = a cos - b sin,  b' = b cos + a sin;   (a, b) = elements (i, pairs + i), or with interleaved (2 i, 2 i + 1).
 * The angle is the product of the position and the binary32 number freq[i], formed and reduced in binary64.  k may be NULL
 * with key_heads = 0; pairs = 0 is the norm alone.  The mean of the squares is a binary32 number: it is infinite for elements beyond 1.8e19, and 0 below 1e-23. */
typedef struct {
  int64_t tokens, heads, key_heads;
  int32_t head_dim;        /* in [1, ADACGD_TRAIN_MAX_HEAD] */
  int32_t pairs;           /* in [0, head_dim / 2] */
  const void* q;           int64_t q_stride;       /* [tokens, heads * head_dim] */
  const void* k;           int64_t k_stride;       /* [tokens, key_heads * head_dim] */
  void* q_out;             int64_t q_out_stride;
  void* k_out;             int64_t k_out_stride;
  const void* q_weight;    /* [head_dim] or NULL (1) */
  const void* k_weight;
  const void* positions;   /* [tokens] int64 or int32; NULL where pairs = 0 */
  const float* freq;       /* [pairs] */
  float eps;               /* finite, >= 0 */
  int32_t dtype;           /* of the matrices */
  int32_t param_dtype;     /* of the weights: dtype or ADACGD_F32 */
  int32_t position_bytes;  /* 8 or 4 */
  int32_t interleaved;
  int32_t reserved;        /* must be 0 */
} adacgd_qk_norm_args;
#define ADACGD_TRAIN_MAX_HEAD 512
adacgd_status adacgd_qk_norm(adacgd_train* t, const adacgd_qk_norm_args* a);

/* Its backward pass, from the inputs of the forward pass.  `f` describes the forward call; its q_out and k_out are read and hold the
 * gradients with respect to the outputs.  With dn those gradients turned back, r = (mean(x^2) + eps)^(-1/2), g = dn weight:
 *   dx = r (g - x r mean(g x r)),   dweight = sum over tokens and heads of dn x r.
 * cols of q and k <= max_cols, tokens <= max_tokens. */
typedef struct {
  adacgd_qk_norm_args f;
  void* dq;                int64_t dq_stride;
  void* dk;                int64_t dk_stride;
  void* dq_weight;         /* [head_dim] or NULL, param_dtype */
  void* dk_weight;
} adacgd_qk_norm_backward_args;
adacgd_status adacgd_qk_norm_backward(adacgd_train* t, const adacgd_qk_norm_backward_args* a);

/* Attention over the tokens of each sequence.  Sequences are rows [seq_start[q], seq_start[q + 1]), or equal runs, as in
 * adacgd_token_rows; rows that belong to none are left as they are in every output.  Query head h reads key head h / (heads / key_heads).  Token i sees token j of its own
 * sequence if both count (mask) and, where causal, j <= i.  With s_ij = scale q_i.k_j over those j,
 *   lse_i = log sum_j exp(s_ij),   out_i = sum_j exp(s_ij - lse_i) v_j;
 * tokens that do not count have out = 0 and lse = -inf.  Products and sums are kept in binary32; for the 16-bit types
 * exp(s_ij - c) is rounded to that type as an operand of the second product, with a power of two c near the row's largest s that keeps it in range.
 * What is stored in rows of tokens that do not count, or of other sequences, reaches no result; Inf or NaN in a token that counts may reach
 * every row of its sequence.  No output may overlap anything.
 * The tensor cores take the 16-bit types where head_dim is a multiple of 8 up to 128 and every matrix has rows on 16 bytes (pointer and
 * stride); everything else goes to the general cores, at a thirtieth to a hundredth of the rate. */
typedef struct {
  int64_t tokens, sequences; /* tokens <= ADACGD_TRAIN_MAX_RUN */
  const int32_t* seq_start; /* [sequences + 1] or NULL */
  const uint8_t* mask;      /* [tokens] or NULL */
  const void* q;            int64_t q_stride;     /* [tokens, heads * head_dim] */
  const void* k;            int64_t k_stride;     /* [tokens, key_heads * head_dim] */
  const void* v;            int64_t v_stride;     /* [tokens, key_heads * head_dim] */
  int32_t heads, key_heads; /* key_heads divides heads */
  int32_t head_dim;         /* in [1, ADACGD_ATTENTION_MAX_HEAD] */
  int32_t causal;
  float scale;              /* finite, > 0 */
  int32_t dtype;
} adacgd_attention_inputs;
#define ADACGD_ATTENTION_MAX_HEAD 256
typedef struct {
  adacgd_attention_inputs in;
  void* out;                int64_t out_stride;   /* [tokens, heads * head_dim] */
  float* lse;               /* [heads][tokens] or NULL */
} adacgd_attention_args;
adacgd_status adacgd_attention(adacgd_train* t, const adacgd_attention_args* a);

/* Backward pass, from what the forward pass stored; the probabilities p_ij = exp(s_ij - lse_i) are computed again.
 *   d_i = dout_i.out_i,   ds_ij = p_ij (dout_i.v_j - d_i),
 *   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij dout_i,
 * the sums over i running over the query heads that share the key head too.  row_dot receives d (0 for tokens that do not count).
 * p and ds are rounded to the 16-bit types as operands of products.  Rows of tokens that do not count are 0 in dq, dk and dv. */
typedef struct {
  adacgd_attention_inputs in;
  const void* out;          int64_t out_stride;
  const void* dout;         int64_t dout_stride;
  const float* lse;         /* [heads][tokens] */
  float* row_dot;           /* [heads][tokens] */
  void* dq;                 int64_t dq_stride;
  void* dk;                 int64_t dk_stride;
  void* dv;                 int64_t dv_stride;     /* dq, dk and dv hold other numbers while the call runs */
} adacgd_attention_backward_args;
adacgd_status adacgd_attention_backward(adacgd_train* t, const adacgd_attention_backward_args* a);

#ifdef __cplusplus
}
#endif
#endif /* ADACGD_TRAIN_H */
