// Dropout and layer norm with the residual sum and dropout in front of it, forward and backward (adacgd_train.h).
#include "adacgd_train.cuh"

namespace adacgd {

namespace {

constexpr int NT = 256;

template <typename T>
__global__ void __launch_bounds__(NT) k_dropout(const T* __restrict__ x, long long xs, const T* __restrict__ res, long long rs,
                                                T* __restrict__ out, long long os, long long rows, long long cols, Drop d) {
  const long long n = rows * cols;
  for (long long i = (long long)blockIdx.x * NT + threadIdx.x; i < n; i += (long long)gridDim.x * NT) {
    const long long r = i / cols, c = i - r * cols;
    const float b = res ? to_f(res[r * rs + c]) : 0.f;
    float v = to_f(x[r * xs + c]);
    if (d.thr) v = drop_one(v, b, (u64)i, d);
    else if (res) v = b + v;
    out[r * os + c] = from_f<T>(v);
  }
}

template <typename T, typename P>
__global__ void __launch_bounds__(NT) k_norm(adacgd_norm_args a, Drop d) {
  extern __shared__ float srow[];
  __shared__ float sh[NT / 32];
  const long long row = blockIdx.x;
  const int cols = (int)a.cols;
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* res = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  float acc = 0.f;
  for (int c = threadIdx.x; c < cols; c += NT) {
    const float b = res ? to_f(res[c]) : 0.f;
    float v = to_f(x[c]);
    if (d.thr) v = drop_one(v, b, (u64)(row * cols + c), d);
    else if (res) v = b + v;
    srow[c] = v;
    acc += v;
  }
  const float mean = block_sum<NT>(acc, sh) / (float)cols;
  acc = 0.f;
  for (int c = threadIdx.x; c < cols; c += NT) acc = fmaf(srow[c] - mean, srow[c] - mean, acc);
  const float rstd = 1.f / sqrtf(block_sum<NT>(acc, sh) / (float)cols + a.eps);
  T* out = (T*)a.out + row * a.out_stride;
  T* sum = a.sum ? (T*)a.sum + row * a.sum_stride : nullptr;
  const P* w = (const P*)a.weight;
  const P* b = (const P*)a.bias;
  for (int c = threadIdx.x; c < cols; c += NT) {
    const float v = srow[c];
    if (sum) sum[c] = from_f<T>(v);
    out[c] = from_f<T>(fmaf((v - mean) * rstd, w ? to_f(w[c]) : 1.f, b ? to_f(b[c]) : 0.f));
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

template <typename T, typename P>
__global__ void __launch_bounds__(NT) k_norm_bwd(adacgd_norm_backward_args a, Drop d) {
  __shared__ float sh[NT / 32];
  const long long row = blockIdx.x;
  const int cols = (int)a.cols;
  const T* dy = (const T*)a.dout + row * a.dout_stride;
  const T* s = (const T*)a.s + row * a.s_stride;
  const T* ds = a.dsum ? (const T*)a.dsum + row * a.dsum_stride : nullptr;
  T* dx = (T*)a.dx + row * a.dx_stride;
  T* dr = a.dresidual ? (T*)a.dresidual + row * a.dresidual_stride : nullptr;
  const P* w = (const P*)a.weight;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float p = 0.f, q = 0.f;
  for (int c = threadIdx.x; c < cols; c += NT) {
    const float g = to_f(dy[c]) * (w ? to_f(w[c]) : 1.f);
    p += g;
    q = fmaf(g, (to_f(s[c]) - mean) * rstd, q);
  }
  p = block_sum<NT>(p, sh) / (float)cols;
  q = block_sum<NT>(q, sh) / (float)cols;
  for (int c = threadIdx.x; c < cols; c += NT) {
    const float g = to_f(dy[c]) * (w ? to_f(w[c]) : 1.f);
    const float h = (to_f(s[c]) - mean) * rstd;
    float v = rstd * (g - p - h * q);
    if (ds) v += to_f(ds[c]);
    if (dr) dr[c] = from_f<T>(v);
    dx[c] = from_f<T>(d.thr ? drop_one(v, 0.f, (u64)(row * cols + c), d) : v);
  }
}

// Partial weight and bias gradients: a thread a column, a slice of rows a CTA row.
template <typename T>
__global__ void __launch_bounds__(NT) k_norm_dw(adacgd_norm_backward_args a, float* __restrict__ part, long long max_cols) {
  const int c = blockIdx.x * NT + threadIdx.x;
  if (c >= a.cols) return;
  const long long lo = a.rows * blockIdx.y / gridDim.y, hi = a.rows * (blockIdx.y + 1) / gridDim.y;
  float dw = 0.f, db = 0.f;
  for (long long r = lo; r < hi; ++r) {
    const float g = to_f(((const T*)a.dout)[r * a.dout_stride + c]);
    dw = fmaf(g, (to_f(((const T*)a.s)[r * a.s_stride + c]) - a.mean[r]) * a.rstd[r], dw);
    db += g;
  }
  part[(2ll * blockIdx.y) * max_cols + c] = dw;
  part[(2ll * blockIdx.y + 1) * max_cols + c] = db;
}

template <typename P>
__global__ void __launch_bounds__(NT) k_norm_dw_sum(const float* __restrict__ part, long long max_cols, int parts, int cols,
                                                    P* __restrict__ dw, P* __restrict__ db) {
  const int c = blockIdx.x * NT + threadIdx.x;
  if (c >= cols) return;
  double a = 0.0, b = 0.0;
  for (int k = 0; k < parts; ++k) {
    a += (double)part[2ll * k * max_cols + c];
    b += (double)part[(2ll * k + 1) * max_cols + c];
  }
  if (dw) dw[c] = from_f<P>((float)a);
  if (db) db[c] = from_f<P>((float)b);
}

template <typename T>
int dropout_t(const adacgd_dropout_args& a, int sms, cudaStream_t st) {
  const long long n = a.rows * a.cols;
  long long g = (n + NT - 1) / NT;
  if (g > 16ll * sms) g = 16ll * sms;
  k_dropout<T><<<(unsigned)g, NT, 0, st>>>((const T*)a.x, a.x_stride, (const T*)a.residual, a.residual_stride, (T*)a.out,
                                           a.out_stride, a.rows, a.cols, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, typename P>
int norm_t(const adacgd_norm_args& a, cudaStream_t st) {
  const int smem = (int)a.cols * 4;
  if (cudaFuncSetAttribute(k_norm<T, P>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return -1;
  k_norm<T, P><<<(unsigned)a.rows, NT, smem, st>>>(a, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, typename P>
int norm_bwd_t(const TrainScratch& s, const adacgd_norm_backward_args& a, int sms, cudaStream_t st) {
  const int cols = (int)a.cols, tiles = (cols + NT - 1) / NT;
  int n = 0;
  if (a.dweight || a.dbias) {   // before dx is written: it may be the same matrix as dout or s
    long long parts = 4ll * sms / tiles + 1;
    if (parts > NORM_PARTS) parts = NORM_PARTS;
    if (parts > a.rows) parts = a.rows;
    k_norm_dw<T><<<dim3(tiles, (unsigned)parts), NT, 0, st>>>(a, s.norm_part, s.max_cols);
    k_norm_dw_sum<P><<<tiles, NT, 0, st>>>(s.norm_part, s.max_cols, (int)parts, cols, (P*)a.dweight, (P*)a.dbias);
    n += 2;
  }
  k_norm_bwd<T, P><<<(unsigned)a.rows, NT, 0, st>>>(a, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? n + 1 : -1;
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_dropout(const adacgd_dropout_args& a, int sms, cudaStream_t st) { BY_TYPE(a.dtype, (dropout_t<T>(a, sms, st))) }

int launch_layer_norm(const adacgd_norm_args& a, int sms, cudaStream_t st) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_t<T, float>(a, st)))
  BY_TYPE(a.dtype, (norm_t<T, T>(a, st)))
}

int launch_layer_norm_backward(const TrainScratch& s, const adacgd_norm_backward_args& a, int sms, cudaStream_t st) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_bwd_t<T, float>(s, a, sms, st)))
  BY_TYPE(a.dtype, (norm_bwd_t<T, T>(s, a, sms, st)))
}

}  // namespace adacgd
