// Declarations and device helpers shared by the units of the training operators (adacgd_train.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>

#include "adacgd_internal.cuh"
#include "adacgd_train.h"

namespace adacgd {

constexpr int NORM_PARTS = 592;  // most partial rows of a weight gradient: four CTAs on each of 148 SMs

// The context's workspace, carved by carve_train_scratch.
struct TrainScratch {
  u32* tickets;    // [NTRAIN_TICKETS] completion counts, zero between calls
  float* tok_a;    // [tokens] a token's loss;                      in the gradient of a lookup these four are the tokens' ids and
  float* tok_b;    // [tokens] its KL estimate;                     numbers, being sorted
  float* tok_c;    // [tokens] 1 where the clipped term has taken the gradient
  float* seq;      // [tokens + 1] per sequence: weight or gradient coefficient; the last is the total
  double* part;    // [tokens + 3] per pair: loss; per CTA of the token sums: three of them
  double* own;     // [MAX_SMALL_CTAS][3] sums of the CTAs of a small policy loss
  float* norm_part; // [NORM_PARTS][2][max_cols] partial weight and bias gradients, or partial rows of a table's gradient
  long long max_tokens, max_cols;
};
constexpr int NTRAIN_TICKETS = 64;
constexpr int MAX_SMALL_CTAS = 2048;   // of a small policy loss: a row each at most

// Where a call runs.
struct Where {
  int device, sms;
  cudaStream_t stream;
};

// CTAs of a kernel that fit on an SM; the first call on a device also raises its limit of dynamic shared memory.  One table
// per kernel.  0 after an error.
constexpr int TRAIN_DEVICES = 64;
template <typename K>
int resident_ctas(K kern, std::atomic<int> (&table)[TRAIN_DEVICES], int device, int threads, int smem) {
  if (device < 0 || device >= TRAIN_DEVICES) return 0;
  int n = table[device].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (smem > 0 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, threads, smem) != cudaSuccess || n < 1) return 0;
  table[device].store(n, std::memory_order_relaxed);
  return n;
}

size_t train_scratch_bytes(long long max_tokens, long long max_cols);
void carve_train_scratch(TrainScratch* s, void* base, long long max_tokens, long long max_cols);

// Each returns the number of kernels launched, or -1 after a failed launch.
int launch_dropout(const adacgd_dropout_args& a, const Where& at);
int launch_layer_norm(const adacgd_norm_args& a, const Where& at);
int launch_layer_norm_backward(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& at);
int launch_token_logp(const adacgd_token_rows& r, float* logp, float* lse, const Where& at);
int launch_preference(const TrainScratch& s, const adacgd_preference_args& a, const Where& at);
int launch_policy(const TrainScratch& s, const adacgd_policy_args& a, const Where& at);
int launch_embedding(const adacgd_embedding_args& a, const Where& at);
int launch_embedding_backward(const TrainScratch& s, const adacgd_embedding_backward_args& a, const Where& at);
int launch_qk_norm(const adacgd_qk_norm_args& a, const Where& at);
int launch_qk_norm_backward(const TrainScratch& s, const adacgd_qk_norm_backward_args& a, const Where& at);
int launch_attention(const adacgd_attention_args& a, const Where& at);
int launch_attention_backward(const adacgd_attention_backward_args& a, const Where& at);

// ---- element types ----
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ---- eight consecutive elements: 16 bytes, or 32 of binary32, aligned to their size ----
template <typename T> struct Run { uint4 v[sizeof(T) / 2]; };

template <typename T> __device__ __forceinline__ Run<T> load_run(const T* p) {
  Run<T> r;
  r.v[0] = *reinterpret_cast<const uint4*>(p);
  return r;
}
// one 32-byte access: two of 16 bytes would each use half of every sector they touch
template <> __device__ __forceinline__ Run<float> load_run<float>(const float* p) {
  Run<float> r;
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r.v[0].x), "=r"(r.v[0].y), "=r"(r.v[0].z), "=r"(r.v[0].w), "=r"(r.v[1].x), "=r"(r.v[1].y), "=r"(r.v[1].z), "=r"(r.v[1].w)
               : "l"(p)
               : "memory");
  return r;
}
__device__ __forceinline__ void unpack(const Run<float>& r, float (&o)[8]) {
  o[0] = __uint_as_float(r.v[0].x); o[1] = __uint_as_float(r.v[0].y); o[2] = __uint_as_float(r.v[0].z); o[3] = __uint_as_float(r.v[0].w);
  o[4] = __uint_as_float(r.v[1].x); o[5] = __uint_as_float(r.v[1].y); o[6] = __uint_as_float(r.v[1].z); o[7] = __uint_as_float(r.v[1].w);
}
__device__ __forceinline__ void unpack(const Run<__nv_bfloat16>& r, float (&o)[8]) {
  const u32 w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = __uint_as_float(w[i] << 16);
    o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Run<__half>& r, float (&o)[8]) {
  const u32 w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    o[2 * i] = f.x;
    o[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void store_run(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
               "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
// Eight elements of a 16-bit type in 16 bytes, each rounded to nearest.
template <typename T> __device__ __forceinline__ uint4 pack_run(const float (&v)[8]);
template <> __device__ __forceinline__ uint4 pack_run<__nv_bfloat16>(const float (&v)[8]) {
  u32 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const u32*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <> __device__ __forceinline__ uint4 pack_run<__half>(const float (&v)[8]) {
  u32 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 b = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const u32*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T> __device__ __forceinline__ void store_run(T* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = pack_run<T>(v);
}

// ---- packed binary32 ----
// Two binary32 numbers in a register pair: one instruction for both.
struct F2 { u64 v; };
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(F2 a, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
// Eight numbers as four pairs.
__device__ __forceinline__ void pairs_of(const float (&x)[8], F2 (&o)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f2(x[2 * i], x[2 * i + 1]);
}
__device__ __forceinline__ void floats_of(const F2 (&x)[4], float (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) split(x[i], o[2 * i], o[2 * i + 1]);
}

// ---- dropout's random bits: Philox4x32-10 (Salmon et al., SC 2011) ----
struct Drop {        // what the kernels need of adacgd_drop
  bool on;
  u32 lim;           // 65536 thr - 1: a 16-bit number in the upper half of a word keeps its element iff the word exceeds this
  float scale;       // 65536 / (65536 - thr), nearest
  float hi, lo;      // the same as hi + lo, both positive: see scaled()
  u32 ka[10], kb[10];  // the rounds' keys
  u32 o0, o1;
};
inline Drop make_drop(const adacgd_drop& d) {
  Drop r;
  const u32 thr = (u32)(d.p * 65536.0 + 0.5);
  r.on = thr > 0;
  r.lim = thr << 16;
  r.lim -= 1u;       // thr = 65536: nothing exceeds 2^32 - 1
  const double scale = thr < 65536u ? 65536.0 / (65536.0 - (double)thr) : 1.0;
  r.scale = (float)scale;
  r.hi = (float)scale;
  if ((double)r.hi >= scale) r.hi = nextafterf(r.hi, 0.f);
  r.lo = (float)(scale - (double)r.hi);
  u32 k0 = (u32)d.seed, k1 = (u32)(d.seed >> 32);
  for (int i = 0; i < 10; ++i, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) {
    r.ka[i] = k0;
    r.kb[i] = k1;
  }
  r.o0 = (u32)d.offset; r.o1 = (u32)(d.offset >> 32);
  return r;
}
// One call costs 20 wide products, which run at a quarter of the rate of additions: 0.62 clocks of an SM measured, against
// 1.4 clocks that eight 16-bit elements take to be read and written.  The keys come from the host: 20 additions less.
__device__ __forceinline__ uint4 philox(u64 block, const Drop& d) {
  u32 c0 = (u32)block, c1 = (u32)(block >> 32), c2 = d.o0, c3 = d.o1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const u64 a = (u64)c0 * 0xD2511F53u, b = (u64)c2 * 0xCD9E8D57u;
    c0 = (u32)(b >> 32) ^ c1 ^ d.ka[r];
    c1 = (u32)b;
    c2 = (u32)(a >> 32) ^ c3 ^ d.kb[r];
    c3 = (u32)a;
  }
  return make_uint4(c0, c1, c2, c3);
}
// Whether element j (0 .. 7) of a block is kept.
__device__ __forceinline__ bool kept(const uint4& w, int j, const Drop& d) {
  const u32 v = j < 4 ? (j < 2 ? w.x : w.y) : (j < 6 ? w.z : w.w);
  return ((j & 1) ? v : v << 16) > d.lim;   // what lies below an upper half does not change the comparison
}
// base + scale v, as if the scale were exact: where the two nearly cancel, its rounding would show.  hi and lo are both
// positive, so an infinite v stays infinite.
__device__ __forceinline__ float scaled(float v, float base, const Drop& d) { return fmaf(v, d.lo, fmaf(v, d.hi, base)); }
// [base +] dropout of element number i
__device__ __forceinline__ float drop_one(float v, u64 i, const Drop& d) {
  return kept(philox(i >> 3, d), (int)(i & 7), d) ? v * d.scale : 0.f;
}
__device__ __forceinline__ float drop_one(float v, float base, u64 i, const Drop& d) {
  return kept(philox(i >> 3, d), (int)(i & 7), d) ? scaled(v, base, d) : base;
}

// 2^x by the hardware's approximation (relative error about 2^-22, subnormal results flushed to zero)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float LOG2E = 1.4426950408889634f;

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
