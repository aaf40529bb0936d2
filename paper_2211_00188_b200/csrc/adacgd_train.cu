// C ABI of the training operators (adacgd_train.h): contexts and the checks of arguments.  The kernels are in
// adacgd_train_norm.cu (dropout, layer norm) and adacgd_train_loss.cu (log-probabilities and the losses).
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "adacgd_train.cuh"

using namespace adacgd;

struct adacgd_train {
  TrainScratch s;
  Where at;
  long long launches;
  char err[256];
};

namespace {

thread_local char g_train_err[256] = "";

// No entry point throws: messages go to fixed buffers.
adacgd_status fail(adacgd_train* t, adacgd_status s, const char* entry, const char* what) {
  snprintf(t ? t->err : g_train_err, sizeof(g_train_err), "%s: %s", entry, what);
  return s;
}
adacgd_status invalid(adacgd_train* t, const char* entry, const char* what) {
  return fail(t, ADACGD_ERR_INVALID_ARG, entry, what);
}
adacgd_status cuda_fail(adacgd_train* t, const char* entry, cudaError_t e) {
  cudaGetLastError();
  return fail(t, ADACGD_ERR_CUDA, entry, cudaGetErrorString(e));
}

adacgd_status check_device(adacgd_train* t, const char* entry) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(t, entry, e);
  if (dev != t->at.device) return invalid(t, entry, "the current CUDA device is not the one the context was created on");
  return ADACGD_OK;
}

adacgd_status launched(adacgd_train* t, const char* entry, int n) {
  if (n < 0) {
    const cudaError_t e = cudaGetLastError();
    return fail(t, ADACGD_ERR_CUDA, entry, e == cudaSuccess ? "kernel launch failed" : cudaGetErrorString(e));
  }
  t->launches += n;
  return ADACGD_OK;
}

size_t size_of(int32_t dtype) { return dtype == ADACGD_F32 ? 4 : 2; }
bool good_type(int32_t dtype) { return dtype == ADACGD_F32 || dtype == ADACGD_F16 || dtype == ADACGD_BF16; }

// A matrix argument in bytes.
struct Region {
  const char* p;
  long long stride, width, rows;
  bool out;
  bool matrix;  // an output may be the very same matrix as an input
};
Region region(const void* p, long long stride, long long cols, long long rows, size_t es, bool out) {
  return Region{(const char*)p, stride * (long long)es, cols * (long long)es, rows, out, true};
}
Region vec(const void* p, long long n, size_t es, bool out) {
  return Region{(const char*)p, n * (long long)es, n * (long long)es, 1, out, false};
}

bool conflict(const Region& a, const Region& b) {
  if (!a.p || !b.p || !(a.out || b.out) || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  const char* ae = a.p + (a.rows - 1) * a.stride + a.width;
  const char* be = b.p + (b.rows - 1) * b.stride + b.width;
  if (ae <= b.p || be <= a.p) return false;
  if (a.matrix && b.matrix && a.out != b.out && a.p == b.p && a.width == b.width && a.rows == b.rows && (a.stride == b.stride || a.rows == 1))
    return false;                                     // in place: every element is read before it is written
  if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {  // columns of one larger matrix
    long long d = (b.p - a.p) % a.stride;
    if (d < 0) d += a.stride;
    if (d >= a.width && d + b.width <= a.stride) return false;
  }
  return true;
}
bool any_conflict(const Region* r, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j)
      if (conflict(r[i], r[j])) return true;
  return false;
}

const char* check_matrix(const void* p, long long stride, long long rows, long long cols, int32_t dtype, bool optional) {
  if (!p) return optional || rows == 0 ? nullptr : "a matrix that is needed is NULL";
  if (((uintptr_t)p) % size_of(dtype)) return "a matrix is not aligned to its element";
  if (rows > 1 && stride < cols) return "a row stride is smaller than the row";
  if (stride > (1ll << 40)) return "a row stride is out of range";
  return nullptr;
}
const char* check_drop(const adacgd_drop& d) {
  return d.p >= 0.0 && d.p <= 1.0 ? nullptr : "p must be in [0, 1]";
}

const char* check_rows(const adacgd_train* t, const adacgd_token_rows& r, bool sequences) {
  if (r.tokens < 0 || r.tokens > t->s.max_tokens) return "tokens must be in [0, max_tokens]";
  if (r.vocab < 1 || r.vocab >= (1ll << 31)) return "vocab must be in [1, 2^31)";
  if (!good_type(r.dtype)) return "unknown dtype";
  if (r.label_bytes != 4 && r.label_bytes != 8) return "label_bytes must be 4 or 8";
  const char* m = check_matrix(r.logits, r.logits_stride, r.tokens, r.vocab, r.dtype, false);
  if (m) return m;
  if (r.tokens > 0 && (!r.labels || ((uintptr_t)r.labels) % r.label_bytes)) return "labels must be non-NULL and aligned";
  if (!sequences) return nullptr;
  if (r.sequences < 1 || r.sequences > t->s.max_tokens) return "sequences must be in [1, max_tokens]";
  if (((uintptr_t)r.seq_start) & 3) return "seq_start is not aligned";
  if (!r.seq_start && r.tokens % r.sequences) return "without seq_start, sequences must divide tokens";
  return nullptr;
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

namespace adacgd {

static size_t up256(size_t v) { return (v + 255) / 256 * 256; }

size_t train_scratch_bytes(long long max_tokens, long long max_cols) {
  const size_t n = (size_t)max_tokens;
  return up256(NTRAIN_TICKETS * 4) + 3 * up256(n * 4) + up256((n + 1) * 4) + up256((n + 3) * 8) + up256(3ull * MAX_SMALL_CTAS * 8) +
         up256((size_t)NORM_PARTS * 2 * (size_t)max_cols * 4);
}

void carve_train_scratch(TrainScratch* s, void* base, long long max_tokens, long long max_cols) {
  char* b = (char*)base;
  const size_t n = (size_t)max_tokens;
  auto take = [&](size_t bytes) { char* p = b; b += up256(bytes); return p; };
  s->tickets = (u32*)take(NTRAIN_TICKETS * 4);
  s->tok_a = (float*)take(n * 4);
  s->tok_b = (float*)take(n * 4);
  s->tok_c = (float*)take(n * 4);
  s->seq = (float*)take((n + 1) * 4);
  s->part = (double*)take((n + 3) * 8);
  s->own = (double*)take(3ull * MAX_SMALL_CTAS * 8);
  s->norm_part = (float*)take((size_t)NORM_PARTS * 2 * (size_t)max_cols * 4);
  s->max_tokens = max_tokens;
  s->max_cols = max_cols;
}

}  // namespace adacgd

extern "C" {

adacgd_status adacgd_train_workspace_bytes(int64_t max_tokens, int64_t max_cols, size_t* bytes_out) {
  const char* entry = "adacgd_train_workspace_bytes";
  if (!bytes_out) return invalid(nullptr, entry, "bytes_out is NULL");
  if (max_tokens < 1 || max_tokens >= (1ll << 31)) return invalid(nullptr, entry, "max_tokens must be in [1, 2^31)");
  if (max_cols < 1 || max_cols > ADACGD_TRAIN_MAX_COLS)
    return invalid(nullptr, entry, "max_cols must be in [1, ADACGD_TRAIN_MAX_COLS = 32768]");
  *bytes_out = train_scratch_bytes(max_tokens, max_cols);
  return ADACGD_OK;
}

adacgd_status adacgd_train_init(adacgd_train** out, int64_t max_tokens, int64_t max_cols, void* workspace_dev,
                                size_t workspace_bytes, void* cuda_stream) {
  const char* entry = "adacgd_train_init";
  if (!out) return invalid(nullptr, entry, "out is NULL");
  *out = nullptr;
  size_t need = 0;
  const adacgd_status st = adacgd_train_workspace_bytes(max_tokens, max_cols, &need);
  if (st != ADACGD_OK) return st;
  if (!workspace_dev || ((uintptr_t)workspace_dev & 255))
    return invalid(nullptr, entry, "workspace_dev must be non-NULL and 256-byte aligned");
  if (workspace_bytes < need)
    return fail(nullptr, ADACGD_ERR_WORKSPACE, entry, "workspace smaller than adacgd_train_workspace_bytes reports");
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(nullptr, entry, e);
  const DevProps* dp = current_device();
  if (!dp) return fail(nullptr, ADACGD_ERR_CUDA, entry, "no usable current device");
  adacgd_train* t = new (std::nothrow) adacgd_train();
  if (!t) return invalid(nullptr, entry, "out of host memory");
  carve_train_scratch(&t->s, workspace_dev, max_tokens, max_cols);
  t->at.stream = (cudaStream_t)cuda_stream;
  t->at.device = dev;
  t->at.sms = dp->sms;
  t->launches = 0;
  t->err[0] = 0;
  e = cudaMemsetAsync(t->s.tickets, 0, NTRAIN_TICKETS * 4, t->at.stream);
  if (e != cudaSuccess) {
    delete t;
    return cuda_fail(nullptr, entry, e);
  }
  *out = t;
  return ADACGD_OK;
}

void adacgd_train_destroy(adacgd_train* t) { delete t; }

const char* adacgd_train_last_error(const adacgd_train* t) { return t ? t->err : g_train_err; }

int64_t adacgd_train_launch_count(const adacgd_train* t) { return t ? t->launches : 0; }

adacgd_status adacgd_dropout(adacgd_train* t, const adacgd_dropout_args* a) {
  const char* entry = "adacgd_dropout";
  if (!t || !a) return invalid(t, entry, "context or arguments are NULL");
  if (a->rows < 0 || a->cols < 1 || a->rows > (1ll << 40) || a->cols > (1ll << 40) ||
      (a->rows > 0 && a->cols > (1ll << 50) / a->rows))
    return invalid(t, entry, "rows must be >= 0 and cols >= 1, at most 2^50 elements");
  if (!good_type(a->dtype)) return invalid(t, entry, "unknown dtype");
  if (a->reserved) return invalid(t, entry, "reserved must be 0");
  const char* m = check_drop(a->drop);
  if (!m) m = check_matrix(a->x, a->x_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->residual, a->residual_stride, a->rows, a->cols, a->dtype, true);
  if (!m) m = check_matrix(a->out, a->out_stride, a->rows, a->cols, a->dtype, false);
  if (m) return invalid(t, entry, m);
  const size_t es = size_of(a->dtype);
  const Region r[] = {region(a->x, a->x_stride, a->cols, a->rows, es, false),
                      region(a->residual, a->residual_stride, a->cols, a->rows, es, false),
                      region(a->out, a->out_stride, a->cols, a->rows, es, true)};
  if (any_conflict(r, 3)) return invalid(t, entry, "out overlaps an input without being the same matrix");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  if (a->rows == 0) return ADACGD_OK;
  return launched(t, entry, launch_dropout(*a, t->at));
}

adacgd_status adacgd_layer_norm(adacgd_train* t, const adacgd_norm_args* a) {
  const char* entry = "adacgd_layer_norm";
  if (!t || !a) return invalid(t, entry, "context or arguments are NULL");
  if (a->rows < 0 || a->rows >= (1ll << 31)) return invalid(t, entry, "rows must be in [0, 2^31)");
  if (a->cols < 1 || a->cols > ADACGD_TRAIN_MAX_COLS)
    return invalid(t, entry, "cols must be in [1, ADACGD_TRAIN_MAX_COLS = 32768]");
  if (!good_type(a->dtype)) return invalid(t, entry, "unknown dtype");
  if (a->param_dtype != a->dtype && a->param_dtype != ADACGD_F32)
    return invalid(t, entry, "param_dtype must be dtype or ADACGD_F32");
  if (a->reserved) return invalid(t, entry, "reserved must be 0");
  if (!(a->eps >= 0.f) || isinf(a->eps)) return invalid(t, entry, "eps must be finite and >= 0");
  const char* m = check_drop(a->drop);
  if (!m) m = check_matrix(a->x, a->x_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->residual, a->residual_stride, a->rows, a->cols, a->dtype, true);
  if (!m) m = check_matrix(a->out, a->out_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->sum, a->sum_stride, a->rows, a->cols, a->dtype, true);
  if (!m && (((uintptr_t)a->weight | (uintptr_t)a->bias) % size_of(a->param_dtype))) m = "weight or bias is not aligned to its element";
  if (!m && !(aligned4(a->mean) && aligned4(a->rstd))) m = "mean or rstd is not aligned";
  if (m) return invalid(t, entry, m);
  const size_t es = size_of(a->dtype), ps = size_of(a->param_dtype);
  const Region r[] = {region(a->x, a->x_stride, a->cols, a->rows, es, false),
                      region(a->residual, a->residual_stride, a->cols, a->rows, es, false),
                      region(a->out, a->out_stride, a->cols, a->rows, es, true),
                      region(a->sum, a->sum_stride, a->cols, a->rows, es, true),
                      vec(a->weight, a->cols, ps, false), vec(a->bias, a->cols, ps, false),
                      vec(a->mean, a->rows, 4, true), vec(a->rstd, a->rows, 4, true)};
  if (any_conflict(r, 8))
    return invalid(t, entry, "an output overlaps another argument without being the same matrix as x or residual");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  if (a->rows == 0) return ADACGD_OK;
  return launched(t, entry, launch_layer_norm(*a, t->at));
}

adacgd_status adacgd_layer_norm_backward(adacgd_train* t, const adacgd_norm_backward_args* a) {
  const char* entry = "adacgd_layer_norm_backward";
  if (!t || !a) return invalid(t, entry, "context or arguments are NULL");
  if (a->rows < 0 || a->rows > t->s.max_tokens) return invalid(t, entry, "rows must be in [0, max_tokens]");
  if (a->cols < 1 || a->cols > t->s.max_cols) return invalid(t, entry, "cols must be in [1, max_cols]");
  if (!good_type(a->dtype)) return invalid(t, entry, "unknown dtype");
  if (a->param_dtype != a->dtype && a->param_dtype != ADACGD_F32)
    return invalid(t, entry, "param_dtype must be dtype or ADACGD_F32");
  const char* m = check_drop(a->drop);
  if (!m) m = check_matrix(a->dout, a->dout_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->s, a->s_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->dsum, a->dsum_stride, a->rows, a->cols, a->dtype, true);
  if (!m) m = check_matrix(a->dx, a->dx_stride, a->rows, a->cols, a->dtype, false);
  if (!m) m = check_matrix(a->dresidual, a->dresidual_stride, a->rows, a->cols, a->dtype, true);
  if (!m && a->rows > 0 && (!a->mean || !a->rstd)) m = "mean and rstd must be non-NULL";
  if (!m && !(aligned4(a->mean) && aligned4(a->rstd))) m = "mean or rstd is not aligned";
  if (!m && (((uintptr_t)a->weight | (uintptr_t)a->dweight | (uintptr_t)a->dbias) % size_of(a->param_dtype)))
    m = "weight, dweight or dbias is not aligned to its element";
  if (m) return invalid(t, entry, m);
  const size_t es = size_of(a->dtype), ps = size_of(a->param_dtype);
  const Region r[] = {region(a->dout, a->dout_stride, a->cols, a->rows, es, false),
                      region(a->s, a->s_stride, a->cols, a->rows, es, false),
                      region(a->dsum, a->dsum_stride, a->cols, a->rows, es, false),
                      region(a->dx, a->dx_stride, a->cols, a->rows, es, true),
                      region(a->dresidual, a->dresidual_stride, a->cols, a->rows, es, true),
                      vec(a->mean, a->rows, 4, false), vec(a->rstd, a->rows, 4, false),
                      vec(a->weight, a->cols, ps, false), vec(a->dweight, a->cols, ps, true), vec(a->dbias, a->cols, ps, true)};
  if (any_conflict(r, 10))
    return invalid(t, entry, "an output overlaps another argument without being the same matrix as dout, s or dsum");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  if (a->rows == 0) {
    cudaError_t e = cudaSuccess;
    if (a->dweight) e = cudaMemsetAsync(a->dweight, 0, a->cols * ps, t->at.stream);
    if (e == cudaSuccess && a->dbias) e = cudaMemsetAsync(a->dbias, 0, a->cols * ps, t->at.stream);
    return e == cudaSuccess ? ADACGD_OK : cuda_fail(t, entry, e);
  }
  return launched(t, entry, launch_layer_norm_backward(t->s, *a, t->at));
}

adacgd_status adacgd_token_logp(adacgd_train* t, const adacgd_token_rows* rows, float* logp, float* lse) {
  const char* entry = "adacgd_token_logp";
  if (!t || !rows) return invalid(t, entry, "context or arguments are NULL");
  const char* m = check_rows(t, *rows, false);
  if (!m && rows->tokens > 0 && !logp) m = "logp must be non-NULL";
  if (!m && !(aligned4(logp) && aligned4(lse))) m = "logp or lse is not aligned";
  if (m) return invalid(t, entry, m);
  const long long n = rows->tokens;
  const Region r[] = {region(rows->logits, rows->logits_stride, rows->vocab, n, size_of(rows->dtype), false),
                      vec(rows->labels, n, rows->label_bytes, false), vec(rows->mask, n, 1, false),
                      vec(logp, n, 4, true), vec(lse, n, 4, true)};
  if (any_conflict(r, 5)) return invalid(t, entry, "an output overlaps another argument");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  if (n == 0) return ADACGD_OK;
  return launched(t, entry, launch_token_logp(*rows, logp, lse, t->at));
}

adacgd_status adacgd_preference_loss(adacgd_train* t, const adacgd_preference_args* a) {
  const char* entry = "adacgd_preference_loss";
  if (!t || !a) return invalid(t, entry, "context or arguments are NULL");
  const char* m = check_rows(t, a->rows, true);
  const long long n = a->rows.tokens, q = a->rows.sequences;
  if (!m && (q & 1)) m = "sequences must be even: the preferred answers, then the rejected ones";
  if (!m && !a->loss) m = "loss must be non-NULL";
  if (!m && n > 0 && !a->ref_logp) m = "ref_logp must be non-NULL";
  if (!m && !(aligned4(a->loss) && aligned4(a->ref_logp) && aligned4(a->margin) && aligned4(a->seq_logp))) m = "a vector is not aligned";
  if (!m) m = check_matrix(a->dlogits, a->dlogits_stride, n, a->rows.vocab, a->rows.dtype, true);
  if (!m && (a->kind < ADACGD_PREF_SIGMOID || a->kind > ADACGD_PREF_SQUARE)) m = "unknown kind";
  if (!m && !(a->beta > 0.f && !isinf(a->beta))) m = "beta must be finite and > 0";
  if (!m && !(a->label_smoothing >= 0.f && a->label_smoothing <= 0.5f)) m = "label_smoothing must be in [0, 0.5]";
  if (!m && a->label_smoothing != 0.f && a->kind != ADACGD_PREF_SIGMOID) m = "label_smoothing goes with the sigmoid kind only";
  if (!m && (isnan(a->grad_scale) || isinf(a->grad_scale))) m = "grad_scale must be finite";
  if (!m && a->reserved) m = "reserved must be 0";
  if (m) return invalid(t, entry, m);
  const size_t es = size_of(a->rows.dtype);
  const Region r[] = {region(a->rows.logits, a->rows.logits_stride, a->rows.vocab, n, es, false),
                      region(a->dlogits, a->dlogits_stride, a->rows.vocab, n, es, true),
                      vec(a->rows.labels, n, a->rows.label_bytes, false), vec(a->rows.mask, n, 1, false),
                      vec(a->rows.seq_start, q + 1, 4, false), vec(a->ref_logp, n, 4, false),
                      vec(a->loss, 1, 4, true), vec(a->margin, q / 2, 4, true), vec(a->seq_logp, q, 4, true)};
  if (any_conflict(r, 9))
    return invalid(t, entry, "an output overlaps another argument without dlogits being the same matrix as logits");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  return launched(t, entry, launch_preference(t->s, *a, t->at));
}

adacgd_status adacgd_policy_loss(adacgd_train* t, const adacgd_policy_args* a) {
  const char* entry = "adacgd_policy_loss";
  if (!t || !a) return invalid(t, entry, "context or arguments are NULL");
  const char* m = check_rows(t, a->rows, true);
  const long long n = a->rows.tokens, q = a->rows.sequences;
  if (!m && !a->loss) m = "loss must be non-NULL";
  if (!m && n > 0 && (!a->old_logp || !a->advantages)) m = "old_logp and advantages must be non-NULL";
  if (!m && !(aligned4(a->loss) && aligned4(a->old_logp) && aligned4(a->advantages) && aligned4(a->ref_logp) &&
              aligned4(a->logp) && aligned4(a->stats)))
    m = "a vector is not aligned";
  if (!m) m = check_matrix(a->dlogits, a->dlogits_stride, n, a->rows.vocab, a->rows.dtype, true);
  if (!m && !(a->clip_low >= 0.f && a->clip_low <= 1.f)) m = "clip_low must be in [0, 1]";
  if (!m && !(a->clip_high >= 0.f && !isinf(a->clip_high))) m = "clip_high must be finite and >= 0";
  if (!m && !(a->kl_beta >= 0.f && !isinf(a->kl_beta))) m = "kl_beta must be finite and >= 0";
  if (!m && a->kl_beta > 0.f && !a->ref_logp && n > 0) m = "kl_beta > 0 needs ref_logp";
  if (!m && (isnan(a->grad_scale) || isinf(a->grad_scale))) m = "grad_scale must be finite";
  if (!m && a->reserved) m = "reserved must be 0";
  if (m) return invalid(t, entry, m);
  const size_t es = size_of(a->rows.dtype);
  const Region r[] = {region(a->rows.logits, a->rows.logits_stride, a->rows.vocab, n, es, false),
                      region(a->dlogits, a->dlogits_stride, a->rows.vocab, n, es, true),
                      vec(a->rows.labels, n, a->rows.label_bytes, false), vec(a->rows.mask, n, 1, false),
                      vec(a->rows.seq_start, q + 1, 4, false), vec(a->old_logp, n, 4, false),
                      vec(a->advantages, n, 4, false), vec(a->ref_logp, n, 4, false),
                      vec(a->loss, 1, 4, true), vec(a->logp, n, 4, true), vec(a->stats, 3, 4, true)};
  if (any_conflict(r, 11))
    return invalid(t, entry, "an output overlaps another argument without dlogits being the same matrix as logits");
  const adacgd_status st = check_device(t, entry);
  if (st != ADACGD_OK) return st;
  return launched(t, entry, launch_policy(t->s, *a, t->at));
}

}  // extern "C"
