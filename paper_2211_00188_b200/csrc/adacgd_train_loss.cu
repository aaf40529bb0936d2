// Token log-probabilities, the preference loss and the clipped policy loss with their gradients (adacgd_train.h).
#include "adacgd_train.cuh"

namespace adacgd {

namespace {

constexpr int NT = 256;

// Running maximum and sum of exponentials of a set of numbers: sum_j exp(x_j) = s exp(m).  m = -inf: nothing but -inf.
struct Soft { float m, s; };
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  Soft r;
  r.m = fmaxf(a.m, b.m);
  const float base = base_of(r.m);
  r.s = a.s * exp_fast(a.m - base) + b.s * exp_fast(b.m - base);
  return r;
}
__device__ __forceinline__ void add(Soft& a, float x) {
  if (x > a.m) {
    a.s = a.s * exp_fast(a.m - x);
    a.m = x;
  }
  a.s += exp_fast(x - base_of(a.m));
}

__device__ __forceinline__ long long label_at(const adacgd_token_rows& r, long long t) {
  return r.label_bytes == 8 ? (long long)((const int64_t*)r.labels)[t] : (long long)((const int32_t*)r.labels)[t];
}

__device__ Soft block_soft(Soft v, Soft* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Soft w;
    w.m = __shfl_xor_sync(0xffffffffu, v.m, o);
    w.s = __shfl_xor_sync(0xffffffffu, v.s, o);
    v = join(v, w);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  Soft t = sh[0];
#pragma unroll
  for (int w = 1; w < NT / 32; ++w) t = join(t, sh[w]);
  return t;
}

template <typename T>
__device__ Soft row_soft(const T* x, int vocab, Soft* sh) {
  Soft v = {-INFINITY, 0.f};
  for (int j = threadIdx.x; j < vocab; j += NT) add(v, to_f(x[j]));
  return block_soft(v, sh);
}

// The row's gradient c (1{j = label} - softmax_j), softmax_j = exp(x_j - base) inv.  Not exp(x_j - lse): in a row of the
// type's lowest values the logarithm of the sum is lost against the maximum.
template <typename T>
__device__ void row_grad(const T* x, T* d, int vocab, long long label, float c, float base, float inv) {
  for (int j = threadIdx.x; j < vocab; j += NT) {
    const float p = exp_fast(to_f(x[j]) - base) * inv;
    d[j] = from_f<T>(j == label ? c * (1.f - p) : -c * p);
  }
}
template <typename T>
__device__ void row_zero(T* d, int vocab) {
  for (int j = threadIdx.x; j < vocab; j += NT) d[j] = from_f<T>(0.f);
}

template <typename T>
__global__ void __launch_bounds__(NT) k_logp(adacgd_token_rows r, float* __restrict__ logp, float* __restrict__ lse,
                                             float* __restrict__ base_out, float* __restrict__ inv_out) {
  __shared__ Soft sh[NT / 32];
  const long long t = blockIdx.x;
  if (r.mask && !r.mask[t]) {
    if (threadIdx.x == 0) {
      logp[t] = 0.f;
      if (lse) lse[t] = 0.f;
    }
    return;
  }
  const T* x = (const T*)r.logits + t * r.logits_stride;
  const Soft v = row_soft(x, (int)r.vocab, sh);
  if (threadIdx.x == 0) {
    const long long y = label_at(r, t);
    const float z = y >= 0 && y < r.vocab ? to_f(x[y]) : NAN, base = base_of(v.m), l = logf(v.s);
    logp[t] = (z - base) - l;
    if (lse) lse[t] = base + l;
    if (base_out) {
      base_out[t] = base;
      inv_out[t] = 1.f / v.s;
    }
  }
}

template <int NTH>
__device__ double block_sum_f64(double v, double* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < NTH / 32; ++w) t += sh[w];
  return t;
}

// One CTA a pair: margin, loss and the coefficient of the pair's two sequences.
__global__ void __launch_bounds__(NT) k_pairs(adacgd_preference_args a, const float* __restrict__ logp, float* __restrict__ coef,
                                              double* __restrict__ part) {
  __shared__ double sh[NT / 32];
  const long long pairs = a.rows.sequences / 2, each = a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences;
  const long long p = blockIdx.x;
  double d[2], inv[2];
  for (int k = 0; k < 2; ++k) {
    const long long q = p + k * pairs;
    long long lo, hi;
    seq_bounds(a.rows.seq_start, q, a.rows.tokens, each, &lo, &hi);
    double sum = 0.0, diff = 0.0, cnt = 0.0;
    for (long long t = lo + threadIdx.x; t < hi; t += NT) {
      if (a.rows.mask && !a.rows.mask[t]) continue;
      cnt += 1.0;
      sum += (double)logp[t];
      diff += (double)logp[t] - (double)a.ref_logp[t];
    }
    sum = block_sum_f64<NT>(sum, sh);
    diff = block_sum_f64<NT>(diff, sh);
    cnt = block_sum_f64<NT>(cnt, sh);
    inv[k] = a.length_normalized && cnt > 0.0 ? 1.0 / cnt : 1.0;
    d[k] = diff * inv[k];
    if (threadIdx.x == 0 && a.seq_logp) a.seq_logp[q] = (float)(sum * inv[k]);
  }
  if (threadIdx.x) return;
  const double beta = (double)a.beta, h = beta * (d[0] - d[1]), e = (double)a.label_smoothing;
  double l, g;
  if (a.kind == ADACGD_PREF_SIGMOID) {
    const double tail = log1p(exp(-fabs(h)));               // -log sigma(|h|)
    l = (1.0 - e) * (tail + fmax(-h, 0.0)) + e * (tail + fmax(h, 0.0));
    const double sg = 1.0 / (1.0 + exp(-h)), sn = 1.0 / (1.0 + exp(h));
    g = e * sg - (1.0 - e) * sn;
    if (h != h) l = h;
  } else if (a.kind == ADACGD_PREF_HINGE) {
    l = h < 1.0 ? 1.0 - h : (h != h ? h : 0.0);
    g = h < 1.0 ? -1.0 : (h != h ? h : 0.0);
  } else {
    const double u = h / beta - 0.5 / beta;
    l = u * u;
    g = 2.0 * u / beta;
  }
  const double c = (double)a.grad_scale * g * beta / (double)pairs;
  coef[p] = (float)(c * inv[0]);
  coef[p + pairs] = (float)(-c * inv[1]);
  if (a.margin) a.margin[p] = (float)h;
  part[p] = l;
}

__global__ void __launch_bounds__(NT) k_mean_pairs(const double* __restrict__ part, long long pairs, float* __restrict__ loss) {
  __shared__ double sh[NT / 32];
  double v = 0.0;
  for (long long p = threadIdx.x; p < pairs; p += NT) v += part[p];
  v = block_sum_f64<NT>(v, sh);
  if (threadIdx.x == 0) *loss = (float)(v / (double)pairs);
}

template <typename T>
__global__ void __launch_bounds__(NT) k_preference_grad(adacgd_preference_args a, const float* __restrict__ coef,
                                                        const float* __restrict__ base, const float* __restrict__ inv) {
  const long long t = blockIdx.x;
  T* d = (T*)a.dlogits + t * a.dlogits_stride;
  if (a.rows.mask && !a.rows.mask[t]) return row_zero(d, (int)a.rows.vocab);
  const long long q = seq_of(a.rows.seq_start, t, a.rows.sequences, a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences);
  row_grad((const T*)a.rows.logits + t * a.rows.logits_stride, d, (int)a.rows.vocab, label_at(a.rows, t), coef[q],
           base[t], inv[t]);
}

// Weight of every sequence's tokens; one CTA walks all of them.  weight[sequences] = counted tokens.
__global__ void __launch_bounds__(1024) k_policy_weights(adacgd_policy_args a, float* __restrict__ weight) {
  __shared__ double sh[32];
  const long long S = a.rows.sequences, n = a.rows.tokens, each = a.rows.seq_start ? 0 : n / S;
  double total = 0.0, used = 0.0;
  if (a.per_sequence) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long q = warp; q < S; q += 32) {
      long long lo, hi, c = 0;
      seq_bounds(a.rows.seq_start, q, n, each, &lo, &hi);
      for (long long t = lo + lane; t < hi; t += 32) c += !a.rows.mask || a.rows.mask[t];
      for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if (lane == 0) weight[q] = (float)c;
      if (lane == 0) { total += (double)c; used += c > 0 ? 1.0 : 0.0; }
    }
  } else {
    for (long long t = threadIdx.x; t < n; t += 1024) total += !a.rows.mask || a.rows.mask[t];
  }
  total = block_sum_f64<1024>(total, sh);
  used = block_sum_f64<1024>(used, sh);
  for (long long q = threadIdx.x; q < S; q += 1024) {
    if (a.per_sequence) weight[q] = weight[q] > 0.f ? (float)(1.0 / (used * (double)weight[q])) : 0.f;
    else weight[q] = total > 0.0 ? (float)(1.0 / total) : 0.f;
  }
  if (threadIdx.x == 0) weight[S] = (float)total;
}

template <typename T>
__global__ void __launch_bounds__(NT) k_policy(adacgd_policy_args a, const float* __restrict__ weight, float* __restrict__ tl,
                                               float* __restrict__ tk, float* __restrict__ tc) {
  __shared__ Soft sh[NT / 32];
  const long long t = blockIdx.x;
  const int vocab = (int)a.rows.vocab;
  T* d = a.dlogits ? (T*)a.dlogits + t * a.dlogits_stride : nullptr;
  if (a.rows.mask && !a.rows.mask[t]) {
    if (threadIdx.x == 0) {
      tl[t] = tk[t] = tc[t] = 0.f;
      if (a.logp) a.logp[t] = 0.f;
    }
    if (d) row_zero(d, vocab);
    return;
  }
  const T* x = (const T*)a.rows.logits + t * a.rows.logits_stride;
  const long long y = label_at(a.rows, t);
  const float z = y >= 0 && y < vocab ? to_f(x[y]) : NAN;
  const Soft v = row_soft(x, vocab, sh);
  const float base = base_of(v.m), l = logf(v.s), logp = (z - base) - l;
  const long long q = seq_of(a.rows.seq_start, t, a.rows.sequences, a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences);
  const float w = weight[q], A = a.advantages[t], r = expf(logp - a.old_logp[t]);
  const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
  const float held = (r < lo ? lo : (r > hi ? hi : r)) * A, gain = r * A;   // NaN goes through
  float c = gain <= held ? -gain : 0.f, tok = gain <= held ? -gain : -held, kl = 0.f;
  if (a.ref_logp) {
    const float u = a.ref_logp[t] - logp, e1 = expm1f(u);   // exp(u) - 1 without cancellation near 0
    kl = e1 - u;
    c = c - a.kl_beta * e1;
    tok = tok + a.kl_beta * kl;
  }
  if (d) row_grad(x, d, vocab, y, a.grad_scale * (w * c), base, 1.f / v.s);
  if (threadIdx.x == 0) {
    if (a.logp) a.logp[t] = logp;
    tl[t] = w * tok;
    tk[t] = kl;
    tc[t] = gain > held ? 1.f : 0.f;
  }
}

__global__ void __launch_bounds__(1024) k_policy_sum(adacgd_policy_args a, const float* __restrict__ weight,
                                                     const float* __restrict__ tl, const float* __restrict__ tk,
                                                     const float* __restrict__ tc) {
  __shared__ double sh[32];
  double l = 0.0, k = 0.0, c = 0.0;
  for (long long t = threadIdx.x; t < a.rows.tokens; t += 1024) {
    l += (double)tl[t];
    k += (double)tk[t];
    c += (double)tc[t];
  }
  l = block_sum_f64<1024>(l, sh);
  k = block_sum_f64<1024>(k, sh);
  c = block_sum_f64<1024>(c, sh);
  if (threadIdx.x) return;
  const double total = (double)weight[a.rows.sequences];
  *a.loss = (float)l;
  if (a.stats) {
    a.stats[0] = total > 0.0 ? (float)(k / total) : 0.f;
    a.stats[1] = total > 0.0 ? (float)(c / total) : 0.f;
    a.stats[2] = (float)total;
  }
}

int done(int n) { return cudaGetLastError() == cudaSuccess ? n : -1; }

template <typename T>
int logp_t(const adacgd_token_rows& r, float* logp, float* lse, cudaStream_t st) {
  k_logp<T><<<(unsigned)r.tokens, NT, 0, st>>>(r, logp, lse, nullptr, nullptr);
  return done(1);
}

template <typename T>
int preference_t(const TrainScratch& s, const adacgd_preference_args& a, cudaStream_t st) {
  int n = 2;
  const long long pairs = a.rows.sequences / 2;
  if (a.rows.tokens) k_logp<T><<<(unsigned)a.rows.tokens, NT, 0, st>>>(a.rows, s.logp, nullptr, s.tok_a, s.tok_b), ++n;
  k_pairs<<<(unsigned)pairs, NT, 0, st>>>(a, s.logp, s.seq, s.part);
  k_mean_pairs<<<1, NT, 0, st>>>(s.part, pairs, a.loss);
  if (a.dlogits && a.rows.tokens) k_preference_grad<T><<<(unsigned)a.rows.tokens, NT, 0, st>>>(a, s.seq, s.tok_a, s.tok_b), ++n;
  return done(n);
}

template <typename T>
int policy_t(const TrainScratch& s, const adacgd_policy_args& a, cudaStream_t st) {
  int n = 2;
  k_policy_weights<<<1, 1024, 0, st>>>(a, s.seq);
  if (a.rows.tokens) k_policy<T><<<(unsigned)a.rows.tokens, NT, 0, st>>>(a, s.seq, s.tok_a, s.tok_b, s.tok_c), ++n;
  k_policy_sum<<<1, 1024, 0, st>>>(a, s.seq, s.tok_a, s.tok_b, s.tok_c);
  return done(n);
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_token_logp(const adacgd_token_rows& r, float* logp, float* lse, int sms, cudaStream_t st) {
  BY_TYPE(r.dtype, (logp_t<T>(r, logp, lse, st)))
}
int launch_preference(const TrainScratch& s, const adacgd_preference_args& a, int sms, cudaStream_t st) {
  BY_TYPE(a.rows.dtype, (preference_t<T>(s, a, st)))
}
int launch_policy(const TrainScratch& s, const adacgd_policy_args& a, int sms, cudaStream_t st) {
  BY_TYPE(a.rows.dtype, (policy_t<T>(s, a, st)))
}

}  // namespace adacgd
