// Declarations and device helpers shared by the units of the training operators (adacgd_train.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "adacgd_internal.cuh"
#include "adacgd_train.h"

namespace adacgd {

constexpr int NORM_PARTS = 592;  // most partial rows of a weight gradient: four CTAs on each of 148 SMs

// The context's workspace, carved by carve_train_scratch.
struct TrainScratch {
  u32* tickets;    // [NTRAIN_TICKETS] completion counts, zero between calls
  float* logp;     // [tokens] log-probabilities (where the caller wants none)
  float* lse;      // [tokens] log of the sum of exponentials
  float* tok_a;    // [tokens] a token's weighted loss
  float* tok_b;    // [tokens] its KL estimate
  float* tok_c;    // [tokens] 1 where the clipped term has taken the gradient
  float* seq;      // [tokens + 1] per sequence: weight or gradient coefficient; the last is the total
  double* part;    // [tokens] per pair: loss
  float* norm_part; // [NORM_PARTS][2][max_cols] partial weight and bias gradients
  long long max_tokens, max_cols;
};
constexpr int NTRAIN_TICKETS = 1024;

size_t train_scratch_bytes(long long max_tokens, long long max_cols);
void carve_train_scratch(TrainScratch* s, void* base, long long max_tokens, long long max_cols);

// Each returns the number of kernels launched, or -1 after a failed launch.
int launch_dropout(const adacgd_dropout_args& a, int sms, cudaStream_t stream);
int launch_layer_norm(const adacgd_norm_args& a, int sms, cudaStream_t stream);
int launch_layer_norm_backward(const TrainScratch& s, const adacgd_norm_backward_args& a, int sms, cudaStream_t stream);
int launch_token_logp(const adacgd_token_rows& r, float* logp, float* lse, int sms, cudaStream_t stream);
int launch_preference(const TrainScratch& s, const adacgd_preference_args& a, int sms, cudaStream_t stream);
int launch_policy(const TrainScratch& s, const adacgd_policy_args& a, int sms, cudaStream_t stream);

// ---- element types ----
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ---- dropout's random bits: Philox4x32-10 (Salmon et al., SC 2011) ----
struct Drop {     // what the kernels need of adacgd_drop
  u32 thr;        // kept iff the 16-bit number is at least this; 0: nothing is dropped
  float scale;    // 65536 / (65536 - thr) rounded down, and what is missing: a sum with a residual that nearly cancels
  float scale_lo; // the product would otherwise show the scale's own rounding
  u32 k0, k1, o0, o1;
};
inline Drop make_drop(const adacgd_drop& d) {
  Drop r;
  r.thr = (u32)(d.p * 65536.0 + 0.5);
  const double scale = r.thr < 65536u ? 65536.0 / (65536.0 - (double)r.thr) : 0.0;
  r.scale = (float)scale;
  if ((double)r.scale > scale) r.scale = nextafterf(r.scale, 0.f);   // scale_lo >= 0: an infinite input stays infinite
  r.scale_lo = (float)(scale - (double)r.scale);
  r.k0 = (u32)d.seed; r.k1 = (u32)(d.seed >> 32);
  r.o0 = (u32)d.offset; r.o1 = (u32)(d.offset >> 32);
  return r;
}
__device__ __forceinline__ uint4 philox(u64 block, const Drop& d) {
  u32 c0 = (u32)block, c1 = (u32)(block >> 32), c2 = d.o0, c3 = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const u64 a = (u64)c0 * 0xD2511F53u, b = (u64)c2 * 0xCD9E8D57u;
    c0 = (u32)(b >> 32) ^ c1 ^ k0;
    c1 = (u32)b;
    c2 = (u32)(a >> 32) ^ c3 ^ k1;
    c3 = (u32)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
// The 16-bit number of element j (0 .. 7) of a block.
__device__ __forceinline__ u32 half_of(const uint4& w, int j) {
  const u32 v = j < 4 ? (j < 2 ? w.x : w.y) : (j < 6 ? w.z : w.w);
  return (j & 1) ? v >> 16 : v & 0xffffu;
}
// base + scale v, rounded as if the scale were exact (d.thr > 0)
__device__ __forceinline__ float scaled(float v, float base, const Drop& d) {
  const float t = fmaf(v, d.scale, base);
  return d.scale_lo > 0.f ? fmaf(v, d.scale_lo, t) : t;
}
__device__ __forceinline__ float drop_one(float v, float base, u64 i, const Drop& d) {
  return half_of(philox(i >> 3, d), (int)(i & 7)) >= d.thr ? scaled(v, base, d) : base;
}

// 2^x by the hardware's approximation (relative error about 2^-22, subnormal results flushed to zero)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float exp_fast(float x) { return ex2(x * LOG2E); }

// Sum over the CTA (NT threads), the same bits in every thread; the order is fixed.  sh: NT / 32 floats per value.
template <int NT>
__device__ __forceinline__ float block_sum(float v, float* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) t += sh[w];
  return t;
}

// The first token of sequence q and the one behind its last, cut off at the ends of the batch.
__device__ __forceinline__ void seq_bounds(const int32_t* start, long long q, long long tokens, long long each,
                                           long long* lo, long long* hi) {
  if (start) {
    long long a = start[q], b = start[q + 1];
    a = a < 0 ? 0 : (a > tokens ? tokens : a);
    b = b < a ? a : (b > tokens ? tokens : b);
    *lo = a; *hi = b;
  } else {
    *lo = q * each; *hi = (q + 1) * each;
  }
}
// The sequence a token belongs to.
__device__ __forceinline__ long long seq_of(const int32_t* start, long long t, long long seqs, long long each) {
  if (!start) return t / each;
  long long lo = 0, hi = seqs;       // the last q with start[q] <= t
  while (hi - lo > 1) {
    const long long mid = (lo + hi) >> 1;
    if ((long long)start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace adacgd
