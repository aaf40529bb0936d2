// Token log-probabilities, the preference loss and the clipped policy loss with their gradients (adacgd_train.h).
//
// Everything here is passes over rows of logits, a few operations and one exponential an element and pass: memory sets the time of
// the first pass (the exponential unit, 16 a clock and SM, is at 70 % when 16-bit logits arrive at the copy rate), memory and the
// exponential together that of the second, which also writes.
//   statistics   one pass with the running maximum and sum: sum_j exp(z_j) = s exp(m)
//   gradient     c (1{j = label} - exp(z_j - m) / s); for the policy loss c is known as soon as the row's log-probability
//                is, so the same kernel reads the row again, now from the cache, and writes it; the preference loss first
//                needs the sums of both answers of the pair
// m and s are kept apart to the end: in a row of the type's lowest values the logarithm of s is lost against m.
#include <cooperative_groups.h>
#include "adacgd_train.cuh"

namespace cg = cooperative_groups;
namespace adacgd {

namespace {

// Programmatic dependent launch: the kernels of a call may become resident early and wait for their predecessors' results
// where they need them.  What a predecessor writes is never taken as const __restrict__: that promises data which nobody writes
// while the kernel runs, and lets its loads go ahead of the wait.
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// m: a reference at most SLACK below the maximum; s: sum of exponentials relative to it (to its offset, see below).  m = -inf: nothing but -inf, s = 0.
struct Soft { float m, s; };
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// Exponents are base 2: exp(z - m) is taken as 2^(z L - o), L = log2 e, one fused operation an element.  The offset o is m L to the
// nearest integer: as good as m L, because the logarithm is taken against the same number, and sums kept relative to different m
// differ by a power of two, which costs no rounding.  Beyond |m| = 2^21, where integers beside m L become coarse (a row that a mask
// has filled with -1e10), z - m is formed first.
constexpr float BIG = 2097152.f;

__device__ __forceinline__ bool plain_range(float m) { return fabsf(m) <= BIG; }
// Added to a number below 2^22 and taken off again, 1.5 2^23 leaves the nearest integer.
__device__ __forceinline__ float offset_of(float m) { return fmaf(m, LOG2E, 12582912.f) - 12582912.f; }
// x_i = 2^(x_i L + off)
template <int N>
__device__ __forceinline__ void exp_plain(float (&x)[N], float off) {
  const F2 l2 = f2(LOG2E, LOG2E), o2 = f2(off, off);
#pragma unroll
  for (int i = 0; i + 1 < N; i += 2) {
    float a, b;
    split(fma2(f2(x[i], x[i + 1]), l2, o2), a, b);
    x[i] = ex2(a);
    x[i + 1] = ex2(b);
  }
  if (N & 1) x[N - 1] = ex2(fmaf(x[N - 1], LOG2E, off));
}
template <int N>
__device__ __forceinline__ void exp_all(float (&x)[N], float m) {
  if (plain_range(m)) {
    exp_plain(x, -offset_of(m));
  } else {
    const float b = base_of(m);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = ex2((x[i] - b) * LOG2E);
  }
}
// what a sum kept relative to a is worth relative to m >= a
__device__ __forceinline__ float rel(float a, float m) {
  if (m == -INFINITY) return 0.f;
  const bool pa = plain_range(a), pm = plain_range(m);
  if (pa && pm) {
    const float k = offset_of(a) - offset_of(m);     // an integer, at most 0
    return k < -126.f ? 0.f : __int_as_float(((int)k + 127) << 23);
  }
  if (pm) return ex2(fmaf(a, LOG2E, -offset_of(m)));
  if (pa) return ex2(fmaf(-m, LOG2E, offset_of(a)));
  return ex2((a - m) * LOG2E);
}
// log2 of exp(z) relative to m
__device__ __forceinline__ float log2_rel(float z, float m) {
  return plain_range(m) ? fmaf(z, LOG2E, -offset_of(m)) : (z - base_of(m)) * LOG2E;
}

// log softmax of a row's entry z, and the logarithm of its sum of exponentials, from the reference and the sum.  Added up in 64 bits:
// where the row's largest entry is SLACK above m, both terms have that size and nearly cancel, and z L may pass binary32's range.  The
// sum's exponent k is split off and joins the offset, an integer too; what remains, log2f of [0.75, 1.5), is off by less than 2^-24.
struct Log2 { float k, f; };
__device__ __forceinline__ Log2 log2_sum(float s) {
  const int b = __float_as_int(s), k = b >= 0x00800000 && b < 0x7f800000 ? (b - 0x3f400000) >> 23 : 0;     // not of 0, inf and NaN
  return {(float)k, log2f(__int_as_float(b - (k << 23)))};
}
constexpr double LN2 = 0.6931471805599453;
__device__ __forceinline__ double logp64(float z, const Soft& a) {
  const Log2 l = log2_sum(a.s);
  const double t = plain_range(a.m) ? fma((double)z, (double)LOG2E, -(double)(offset_of(a.m) + l.k))
                                    : ((double)z - (double)base_of(a.m)) * (double)LOG2E - (double)l.k;
  return (t - (double)l.f) * LN2;
}
__device__ __forceinline__ double lse64(const Soft& a) {
  const Log2 l = log2_sum(a.s);
  const double b = (double)base_of(a.m), o = plain_range(a.m) ? fma(b, -(double)LOG2E, (double)(offset_of(a.m) + l.k)) : (double)l.k;
  return b + (o + (double)l.f) * LN2;
}
// logp less another model's, which comes rounded to 32 bits.  Beyond 2^10, as of a label that a mask has set to -1e9, that rounding
// would be most of the difference, so there both are taken rounded.
__device__ __forceinline__ double logp_less(double logp, float other) {
  return (fabs(logp) > 1024.0 ? (double)(float)logp : logp) - (double)other;
}

__device__ __forceinline__ long long label_at(const adacgd_token_rows& r, long long t) {
  return r.label_bytes == 8 ? (long long)((const int64_t*)r.labels)[t] : (long long)((const int32_t*)r.labels)[t];
}

// A row, or a cluster part of it, cut at run boundaries: elements [first, first + 8 runs) in whole runs of eight,
// [begin, first) and [first + 8 runs, end) one by one (at most seven each).
struct Cut {
  int begin, first, runs, end;
};
template <typename T>
__device__ __forceinline__ Cut cut_row(const T* row, int vocab, int part, int parts) {
  constexpr int ALIGN = 8;
  const int head = min(vocab, (int)((ALIGN - ((uintptr_t)row / sizeof(T)) % ALIGN) % ALIGN));
  const int runs = (vocab - head) >> 3;
  const int r0 = (int)((long long)runs * part / parts), r1 = (int)((long long)runs * (part + 1) / parts);
  Cut c;
  c.first = head + 8 * r0;
  c.runs = r1 - r0;
  c.begin = part == 0 ? 0 : c.first;
  c.end = part == parts - 1 ? vocab : head + 8 * r1;
  return c;
}
// Element number t of the ragged ends, or -1.  Fourteen at most, so a thread handles EDGES of them: numbers t, t + NTH.
template <int NTH> constexpr int EDGES = NTH < 14 ? 2 : 1;
__device__ __forceinline__ int edge_of(const Cut& c, int t) {
  const int head = c.first - c.begin, tail0 = c.first + 8 * c.runs;
  if (t < head) return c.begin + t;
  t -= head;
  return t < c.end - tail0 ? tail0 + t : -1;
}

// The reference m only follows the maximum when that is ahead by more than SLACK: exponentials up to e^SLACK do no harm, and
// after the first batch the sum is hardly ever rescaled.  10: the exponents, SLACK L and half a unit, stay below 16, so the largest
// terms are off by 2^-21 L^-1 at most from their arguments' rounding; 16 gave twice that and 8 no measured gain.
constexpr float SLACK = 10.f;
template <int N>
__device__ __forceinline__ void absorb(Soft& a, float (&x)[N]) {
  float m[2] = {x[0], x[N > 1 ? 1 : 0]};
#pragma unroll
  for (int j = 2; j < N; ++j) m[j & 1] = fmaxf(m[j & 1], x[j]);
  const float top = fmaxf(m[0], m[1]);
  if (top > a.m + SLACK) {
    a.s *= rel(a.m, top);          // a.m = -inf: s is 0 and stays 0
    a.m = top;
  }
  exp_all(x, a.m);
  if (N == 1) {
    a.s += x[0];
  } else {
    F2 s = f2(x[0], x[N > 1 ? 1 : 0]);
#pragma unroll
    for (int j = 2; j + 1 < N; j += 2) s = add2(s, f2(x[j], x[j + 1]));
    float u, v;
    split(s, u, v);
    a.s += u + v;
  }
}

// Runs of eight elements that a thread has under way: 64 bytes, loaded before the batch in front of it is worked on, so that
// loads and exponentials overlap within the thread.  LAST: nobody reads these lines again, nor soon what is stored, so both
// are first to leave the cache and rows that still wait for their second pass stay in it.
template <typename T, bool LAST> __device__ __forceinline__ Run<T> load_hint(const T* p) {
  if constexpr (LAST && sizeof(T) == 2) {
    Run<T> r;
    r.v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
    return r;
  }
  return load_run(p);
}
template <typename T, bool LAST> __device__ __forceinline__ void store_hint(T* p, const float (&v)[8]) {
  if constexpr (LAST && sizeof(T) == 2) __stcs(reinterpret_cast<uint4*>(p), pack_run<T>(v));
  else store_run(p, v);
}
template <typename T> struct Batch {
  static constexpr int U = sizeof(T) == 2 ? 4 : 2;
  Run<T> r[U];
};
template <typename T, int NTH, bool LAST>
__device__ __forceinline__ void load_batch(Batch<T>& b, const T* p) {   // p: this thread's first run of the batch
#pragma unroll
  for (int u = 0; u < Batch<T>::U; ++u) b.r[u] = load_hint<T, LAST>(p + 8 * u * NTH);
}

// This thread's share of the statistics.
template <typename T, int NTH>
__device__ __forceinline__ Soft thread_soft(const T* row, const Cut& c, int t) {
  constexpr int U = Batch<T>::U;
  Soft a = {-INFINITY, 0.f};
  const T* p = row + c.first + 8 * t;
  const int whole = c.runs / (U * NTH);      // batches that all threads have in full
  auto take = [&](const Batch<T>& b) {
#pragma unroll
    for (int u = 0; u < U; u += 2) {
      float x[16];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[8];
        unpack(b.r[u + h], y);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[h * 8 + j] = y[j];
      }
      absorb(a, x);
    }
  };
  Batch<T> b0, b1;
  if (whole > 0) load_batch<T, NTH, false>(b0, p);
#pragma unroll
  for (int k = 0; k < EDGES<NTH>; ++k) {
    const int e = edge_of(c, t + k * NTH);
    if (e >= 0) {
      float x[1] = {to_f(row[e])};
      absorb(a, x);
    }
  }
  int k = 0;
  for (; k + 2 <= whole; k += 2) {           // two batches take turns: no copies between registers
    load_batch<T, NTH, false>(b1, p + 8 * U * NTH);
    take(b0);
    p += 16 * U * NTH;
    if (k + 2 < whole) load_batch<T, NTH, false>(b0, p);
    take(b1);
  }
  if (k < whole) {
    take(b0);
    p += 8 * U * NTH;
  }
  const int r0 = whole * U * NTH + t;
  if (r0 < c.runs) {      // the rest: up to U runs, loaded together
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + u * NTH < c.runs) b0.r[u] = load_run(p + 8 * u * NTH);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * NTH >= c.runs) break;
      float x[8];
      unpack(b0.r[u], x);
      absorb(a, x);
    }
  }
  return a;
}

// Before thread_soft: the CTAs of a cluster announce themselves.
template <bool CLUSTER>
__device__ __forceinline__ void row_begin() {
  if (CLUSTER) cg::this_cluster().barrier_arrive();
}

// The lanes of a warp that share a row; the others may have another one, or none.
template <int NTH>
__device__ __forceinline__ u32 row_lanes() {
  return NTH >= 32 ? 0xffffffffu : ((1u << (NTH & 31)) - 1u) << (threadIdx.x & 31 & ~(NTH - 1));
}
// The statistics of the row's threads joined, the same bits in each: lanes of a warp, a CTA or a cluster.
template <int NTH, bool CLUSTER>
__device__ __forceinline__ Soft row_soft(Soft a, Soft* sh, Soft* xch) {
  // maxima first, then the sums against the largest: one exponential instead of two a step
  constexpr int HALF = (NTH < 32 ? NTH : 32) / 2;
  const u32 lanes = row_lanes<NTH>();
  const float mine = a.m;
#pragma unroll
  for (int o = HALF; o > 0; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(lanes, a.m, o));
  a.s *= rel(mine, a.m);
#pragma unroll
  for (int o = HALF; o > 0; o >>= 1) a.s += __shfl_xor_sync(lanes, a.s, o);
  if (NTH <= 32) {
    __syncwarp(lanes);   // what the lanes have read of the row they may now write
    return a;
  }
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = a;
  __syncthreads();
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int w = 0; w < NTH / 32; ++w) m = fmaxf(m, sh[w].m);
  const int lane = threadIdx.x & 31;
  float f = lane < NTH / 32 ? sh[lane].s * rel(sh[lane].m, m) : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) f += __shfl_xor_sync(0xffffffffu, f, o);
  s = __shfl_sync(0xffffffffu, f, 0);
  a.m = m;
  a.s = s;
  if (CLUSTER) {
    cg::cluster_group cl = cg::this_cluster();
    const int parts = (int)cl.num_blocks();
    cl.barrier_wait();   // of row_begin: the other CTAs have started
    if (threadIdx.x < parts) *cl.map_shared_rank(&xch[cl.block_rank()], threadIdx.x) = a;
    cl.sync();      // every CTA's writes have arrived; nobody writes to another CTA after this
    m = -INFINITY;
    for (int k = 0; k < parts; ++k) m = fmaxf(m, xch[k].m);
    s = 0.f;
    for (int k = 0; k < parts; ++k) s += xch[k].s * rel(xch[k].m, m);
    a.m = m;
    a.s = s;
  }
  return a;
}

// c (1{j = label} - softmax_j) for this thread's share, softmax_j = 2^(x_j L) relative to m, over sum.  `same`: the gradient's row
// is aligned as the logits' is.  The label's entry (tz: its log2_rel) is written once more, by the thread that wrote it first.
template <typename T, int NTH, bool LAST>
__device__ __forceinline__ void thread_grad(const T* row, T* d, const Cut& c, int t, bool same, int label, float tz, float coef, float m,
                                            float sum) {
  constexpr int U = Batch<T>::U;
  const float neg = -coef / sum;
  int e[EDGES<NTH>];
  float edge[EDGES<NTH>];
#pragma unroll
  for (int k = 0; k < EDGES<NTH>; ++k) {
    e[k] = edge_of(c, t + k * NTH);
    edge[k] = e[k] >= 0 ? to_f(row[e[k]]) : 0.f;
  }
  const T* p = row + c.first + 8 * t;
  T* q = d + c.first + 8 * t;
  int r = t;                                 // this thread's next run
  if (same && plain_range(m)) {              // as good as always: whole batches, nothing to ask in between
    const int whole = c.runs / (U * NTH);
    const float off = -offset_of(m);
    auto put = [&](const Batch<T>& b) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[8];
        unpack(b.r[u], x);
        exp_plain(x, off);
#pragma unroll
        for (int j = 0; j < 8; j += 2) split(mul2(f2(x[j], x[j + 1]), f2(neg, neg)), x[j], x[j + 1]);
        store_hint<T, LAST>(q + 8 * u * NTH, x);
      }
      q += 8 * U * NTH;
    };
    Batch<T> b0, b1;
    if (whole > 0) load_batch<T, NTH, LAST>(b0, p);
    int k = 0;
    for (; k + 2 <= whole; k += 2) {
      load_batch<T, NTH, LAST>(b1, p + 8 * U * NTH);
      put(b0);
      p += 16 * U * NTH;
      if (k + 2 < whole) load_batch<T, NTH, LAST>(b0, p);
      put(b1);
    }
    if (k < whole) {
      put(b0);
      p += 8 * U * NTH;
    }
    r += whole * U * NTH;
  }
  for (; r < c.runs; r += U * NTH, p += 8 * U * NTH, q += 8 * U * NTH) {
    Batch<T> b;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r + u * NTH < c.runs) b.r[u] = load_hint<T, LAST>(p + 8 * u * NTH);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r + u * NTH >= c.runs) break;
      float x[8];
      unpack(b.r[u], x);
      exp_all(x, m);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= neg;
      if (same) {
        store_hint<T, LAST>(q + 8 * u * NTH, x);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[8 * u * NTH + j] = from_f<T>(x[j]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < EDGES<NTH>; ++k) {
    if (e[k] >= 0) {
      float x[1] = {edge[k]};
      exp_all(x, m);
      d[e[k]] = from_f<T>(neg * x[0]);
    }
  }
  if (label >= c.begin && label < c.end) {
    const int in = label - c.first;
    bool mine = in >= 0 && in < 8 * c.runs && (in >> 3) % NTH == t;
#pragma unroll
    for (int k = 0; k < EDGES<NTH>; ++k) mine = mine || label == e[k];
    if (mine) d[label] = from_f<T>(fmaf(neg, ex2(tz), coef));
  }
}
template <typename T, int NTH>
__device__ __forceinline__ void thread_zero(T* d, const Cut& c, int t) {   // c cut by the gradient's own alignment
  const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < EDGES<NTH>; ++k) {
    const int e = edge_of(c, t + k * NTH);
    if (e >= 0) d[e] = from_f<T>(0.f);
  }
  for (int r = t; r < c.runs; r += NTH) store_run(d + c.first + 8ll * r, z);
}
template <typename T>
__device__ __forceinline__ bool same_phase(const T* a, const T* b) {
  return (((uintptr_t)a ^ (uintptr_t)b) & (8 * sizeof(T) - 1)) == 0;
}

// Where a thread stands: its row, its number among the row's threads, the row's part it works on.
template <int NTH, bool CLUSTER> struct Place {
  static constexpr int CTA = NTH < 128 ? 128 : NTH;
  static constexpr int ROWS = CTA / NTH;
  static constexpr int CTAS = 1024 / CTA;   // an SM: 64 registers a thread
  long long row;
  int t, part, parts;
  __device__ __forceinline__ Place() {
    t = NTH < 128 ? (int)threadIdx.x % NTH : (int)threadIdx.x;
    part = 0;
    parts = 1;
    if (CLUSTER) {
      part = (int)cg::this_cluster().block_rank();
      parts = (int)cg::this_cluster().num_blocks();
    }
    row = (long long)(blockIdx.x / parts) * ROWS + (NTH < 128 ? threadIdx.x / NTH : 0);
  }
};

// --------------------------------------------------------------------------
// log-probabilities
// --------------------------------------------------------------------------
//   logp = z_label - m - log s
// One pass, two 64-byte batches a thread under way.  4096 rows x 65536 bfloat16 91 us = 5.9 TB/s, 91 % of the copy rate; 131072 x 512,
// where a row is one memory latency and two reductions, 31 us = 4.3 TB/s.  Rows walked by as many CTAs as fit lost to CTAs handed out
// by the hardware: no gain on full batches, 140 against 113 us with a third of the rows masked.
// zl, sum, top: the label's entry, the sum and the reference, from which the preference loss has its log-probabilities in 64 bits and
// its gradient.  Either these or logp.
template <typename T, int NTH, bool CLUSTER>
__global__ void __launch_bounds__(Place<NTH, CLUSTER>::CTA, Place<NTH, CLUSTER>::CTAS) k_logp(adacgd_token_rows r, float* __restrict__ logp, float* __restrict__ lse,
                                                                   float* __restrict__ zl, float* __restrict__ sum,
                                                                   float* __restrict__ top) {
  __shared__ Soft sh[32], xch[8];
  pdl_trigger();
  const Place<NTH, CLUSTER> at;
  const long long row = at.row;
  if (row >= r.tokens) return;       // all of the row's lanes; only where NTH <= 32
  const bool counts = !r.mask || r.mask[row];      // fetched together with the label, not one after the other
  const long long y = label_at(r, row);
  const int vocab = (int)r.vocab;
  const T* x = (const T*)r.logits + row * r.logits_stride;
  if (!counts) {                     // the same in the whole cluster
    if (at.t == 0 && at.part == 0) {
      if (logp) logp[row] = 0.f;
      if (lse) lse[row] = 0.f;
    }
    return;
  }
  row_begin<CLUSTER>();
  const float z = y >= 0 && y < vocab ? to_f(x[y]) : NAN;
  const Soft a = row_soft<NTH, CLUSTER>(thread_soft<T, NTH>(x, cut_row(x, vocab, at.part, at.parts), at.t), sh, xch);
  if (at.t == 0 && at.part == 0) {
    if (logp) {
      logp[row] = (float)logp64(z, a);
      if (lse) lse[row] = (float)lse64(a);
    } else {
      zl[row] = z;
      sum[row] = a.s;
      top[row] = a.m;
    }
  }
}

template <int NTH>
__device__ __forceinline__ double block_sum_f64(double v, double* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll 8
  for (int w = 0; w < NTH / 32; ++w) t += sh[w];
  return t;
}

// True in every thread of the CTA that is the last of `n` to arrive; the counter is zero again then.
__device__ __forceinline__ bool last_to_arrive(u32* ticket, u32 n) {
  __shared__ u32 last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicAdd(ticket, 1u) == n - 1u;
    if (last) *ticket = 0u;
  }
  __syncthreads();
  if (last) __threadfence();
  return last != 0u;
}

// --------------------------------------------------------------------------
// preference loss
// --------------------------------------------------------------------------
constexpr int PAIR_NT = 256;

// A pair's margin, loss and the coefficients of its two sequences, from the sums of log-probabilities, of their differences to the
// reference and of counted tokens over the preferred ([0]) and the rejected ([1]) answer.
__device__ __forceinline__ double finish_pair(const adacgd_preference_args& a, long long p, long long pairs, const double (&total)[2],
                                              const double (&diff)[2], const double (&cnt)[2], float* __restrict__ coef) {
  double d[2], inv[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    inv[k] = a.length_normalized && cnt[k] > 0.0 ? 1.0 / cnt[k] : 1.0;
    d[k] = diff[k] * inv[k];
    if (a.seq_logp) a.seq_logp[p + k * pairs] = (float)(total[k] * inv[k]);
  }
  const double beta = (double)a.beta, h = beta * (d[0] - d[1]), e = (double)a.label_smoothing;
  double l, g;
  if (a.kind == ADACGD_PREF_SIGMOID) {
    const double tail = log1p(exp(-fabs(h)));               // -log sigma(|h|)
    l = (1.0 - e) * (tail + fmax(-h, 0.0)) + (e > 0.0 ? e * (tail + fmax(h, 0.0)) : 0.0);   // h = inf: no 0 inf
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
  return l;
}

// `slices` CTAs a pair.  One: it also finishes the pair, and the last CTA of all takes the mean of the losses.  More: the last CTA
// adds the slices' six sums of each pair and finishes the pairs.
__global__ void __launch_bounds__(PAIR_NT) k_pairs(adacgd_preference_args a, const float* zl, const float* sum,
                                                   const float* top, float* __restrict__ coef, double* __restrict__ part, u32 slices, u32* ticket) {
  __shared__ double sh[PAIR_NT / 32];
  pdl_wait();
  pdl_trigger();   // the gradient kernel is large: it is let in when this one has its operands
  const long long pairs = a.rows.sequences / 2, each = a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences;
  const long long p = blockIdx.x / slices, slice = blockIdx.x - p * slices;
  double total[2], diff[2], cnt[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    long long lo, hi;
    seq_bounds(a.rows.seq_start, p + k * pairs, a.rows.tokens, each, &lo, &hi);
    total[k] = diff[k] = cnt[k] = 0.0;
    for (long long t = lo + slice * PAIR_NT + threadIdx.x; t < hi; t += (long long)slices * PAIR_NT) {
      if (a.rows.mask && !a.rows.mask[t]) continue;
      const double logp = logp64(zl[t], Soft{top[t], sum[t]});
      cnt[k] += 1.0;
      total[k] += logp;
      diff[k] += logp_less(logp, a.ref_logp[t]);
    }
    total[k] = block_sum_f64<PAIR_NT>(total[k], sh);
    diff[k] = block_sum_f64<PAIR_NT>(diff[k], sh);
    cnt[k] = block_sum_f64<PAIR_NT>(cnt[k], sh);
  }
  if (threadIdx.x == 0) {
    if (slices == 1) {
      part[p] = finish_pair(a, p, pairs, total, diff, cnt, coef);
    } else {
      double* const q = part + 6ll * blockIdx.x;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        q[k] = total[k];
        q[2 + k] = diff[k];
        q[4 + k] = cnt[k];
      }
    }
  }
  if (!last_to_arrive(ticket, gridDim.x)) return;
  double v = 0.0;
  for (long long q = threadIdx.x; q < pairs; q += PAIR_NT) {
    if (slices == 1) {
      v += __ldcg(&part[q]);
      continue;
    }
    double s[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
    for (u32 k = 0; k < slices; ++k) {
#pragma unroll
      for (int i = 0; i < 6; ++i) s[i] += __ldcg(&part[6 * (q * slices + k) + i]);
    }
    total[0] = s[0]; total[1] = s[1];
    diff[0] = s[2]; diff[1] = s[3];
    cnt[0] = s[4]; cnt[1] = s[5];
    v += finish_pair(a, q, pairs, total, diff, cnt, coef);
  }
  v = block_sum_f64<PAIR_NT>(v, sh);
  if (threadIdx.x == 0) *a.loss = (float)(v / (double)pairs);
}

// The gradient once the pairs' coefficients are known: element by element, `parts` places a row.  The logits have to be read again
// (512 MB do not stay in the cache), so the call moves three units where log-probabilities of the policy kind move two: 4096 x 32000
// bfloat16, two thirds of the tokens counted, 117 us against a floor of 67 for one read and one write, 94 for the two reads.
template <typename T, int NTH>
__global__ void __launch_bounds__(Place<NTH, false>::CTA, Place<NTH, false>::CTAS) k_preference_grad(adacgd_preference_args a, const float* coef,
                                                                            const float* zl, const float* sum,
                                                                            const float* top, u32 parts) {
  const Place<NTH, false> at;
  const long long turn = parts == 1 ? at.row : at.row / parts;
  const int part = parts == 1 ? 0 : (int)(at.row - turn * parts);
  if (turn >= a.rows.tokens) return;
  const long long row = a.rows.tokens - 1 - turn;      // backwards: the rows read last are still in the cache
  T* d = (T*)a.dlogits + row * a.dlogits_stride;
  const int vocab = (int)a.rows.vocab;
  const bool counts = !a.rows.mask || a.rows.mask[row];
  const long long y = label_at(a.rows, row);
  const long long q = seq_of(a.rows.seq_start, row, a.rows.sequences, a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences);
  pdl_wait();      // before anything is written: dlogits may be the logits that the first kernel reads
  if (!counts) {
    thread_zero<T, NTH>(d, cut_row(d, vocab, part, (int)parts), at.t);
    return;
  }
  const T* x = (const T*)a.rows.logits + row * a.rows.logits_stride;
  thread_grad<T, NTH, false>(x, d, cut_row(x, vocab, part, (int)parts), at.t, same_phase(x, d), y >= 0 && y < vocab ? (int)y : -1,
                             log2_rel(zl[row], top[row]), coef[q], top[row], sum[row]);
}

// --------------------------------------------------------------------------
// policy loss
// --------------------------------------------------------------------------
// Weight of every sequence's tokens; one CTA walks all of them.  weight[sequences] = counted tokens.
__global__ void __launch_bounds__(1024) k_policy_weights(adacgd_policy_args a, float* __restrict__ weight) {
  __shared__ double sh[32];
  pdl_trigger();
  const long long S = a.rows.sequences, n = a.rows.tokens, each = a.rows.seq_start ? 0 : n / S;
  double total = 0.0, used = 0.0;
  if (a.per_sequence) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long q = warp; q < S; q += 32) {
      long long lo, hi, c = 0;
      seq_bounds(a.rows.seq_start, q, n, each, &lo, &hi);
      for (long long t = lo + lane; t < hi; t += 32) c += !a.rows.mask || a.rows.mask[t];
      for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if (lane == 0) {
        weight[q] = (float)c;
        total += (double)c;
        used += c > 0 ? 1.0 : 0.0;
      }
    }
  } else if (a.rows.mask) {
    long long c = 0;
    for (long long t = threadIdx.x; t < n; t += 1024) c += a.rows.mask[t] != 0;
    total = (double)c;
  } else {
    total = threadIdx.x == 0 ? (double)n : 0.0;
  }
  total = block_sum_f64<1024>(total, sh);
  used = block_sum_f64<1024>(used, sh);
  for (long long q = threadIdx.x; q < S; q += 1024) {
    if (a.per_sequence) weight[q] = weight[q] > 0.f ? (float)(1.0 / (used * (double)weight[q])) : 0.f;
    else weight[q] = total > 0.0 ? (float)(1.0 / total) : 0.f;
  }
  if (threadIdx.x == 0) weight[S] = (float)total;
  if (n > 0) return;
  if (threadIdx.x == 0) *a.loss = 0.f;      // no rows: no other kernel follows
  if (threadIdx.x < 3 && a.stats) a.stats[threadIdx.x] = 0.f;
}

// A token's loss and its slope with respect to the log-probability, before the token's weight.  The differences of log-probabilities
// are small beside them, so they are taken before the rounding to 32 bits.
struct Token { float loss, slope, kl; bool clipped; };
__device__ __forceinline__ Token token_loss(double logp, float old, float A, bool with_ref, float ref, float clip_low, float clip_high,
                                            float kl_beta) {
  const float x = (float)logp_less(logp, old), r = expf(x), lo = 1.f - clip_low, hi = 1.f + clip_high;
  // NaN goes through, but not inf * 0 where r has only passed binary32's range
  const float held = (r < lo ? lo : (r > hi ? hi : r)) * A, gain = A == 0.f && fabsf(x) < INFINITY ? 0.f : r * A;
  Token k;
  k.clipped = gain > held;
  k.slope = k.clipped ? 0.f : -gain;     // a NaN is not clipped away: it reaches loss and gradient
  k.loss = k.clipped ? -held : -gain;
  k.kl = 0.f;
  if (with_ref) {
    const float u = -(float)logp_less(logp, ref), e1 = expm1f(u);   // exp(u) - 1 without cancellation near 0
    k.kl = e1 - u;
    if (kl_beta > 0.f) {                          // else the term is a statistic alone, which may overflow
      k.slope = k.slope - kl_beta * e1;
      k.loss = k.loss + kl_beta * k.kl;
    }
  }
  return k;
}
__device__ __forceinline__ void write_policy(float* loss, float* stats, double l, double k, double c, double total) {
  *loss = (float)l;
  if (stats) {
    stats[0] = total > 0.0 ? (float)(k / total) : 0.f;
    stats[1] = total > 0.0 ? (float)(c / total) : 0.f;
    stats[2] = (float)total;
  }
}

// Counted tokens among `n`, a share of them for each of NTH threads.
template <int NTH>
__device__ __forceinline__ int count_share(const uint8_t* mask, int n, int t) {
  int c = 0;
  if (((uintptr_t)mask & 15) == 0) {
    for (int i = t * 16; i + 16 <= n; i += NTH * 16) {
      const uint4 v = *reinterpret_cast<const uint4*>(mask + i);
      const u32 w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        u32 x = w[k];             // the lowest bit of each byte becomes the disjunction of its eight
        x |= x >> 4;
        x |= x >> 2;
        x |= x >> 1;
        c += __popc(x & 0x01010101u);
      }
    }
    for (int i = n / 16 * 16 + t; i < n; i += NTH) c += mask[i] != 0;   // up to fifteen, which can be more than NTH
  } else {
    for (int i = t; i < n; i += NTH) c += mask[i] != 0;
  }
  return c;
}

// A row's loss and, from the cache, its gradient.  4096 x 131072 bfloat16, two thirds of the rows counted: 345 us = 5.2 TB/s of DRAM
// traffic, beside which a third as much again comes from the cache.  Rows kept in shared memory between the passes: 521 against 420 us
// with all rows counted, for want of threads; an asynchronous ring instead of the register batches 55 to 62 % of the copy rate.
// SMALL: every row counts the tokens itself and the last CTA adds the CTAs' sums; otherwise a kernel before gives the weights and one
// behind takes the sums.  One kernel instead of three in a call of little work, us in a graph: 528 rows x 1001 7.1 against 8.3, 2048 x
// 256 7.0 against 8.0.  Not for long rows, where the CTAs' fence and count at the end cost more: 16 x 32000 8.9 against 8.3, 2000 x
// 32000 52 against 48; nor for weights by sequence, whose kernel stays: no difference.
constexpr long long SMALL_ELEMENTS = 1 << 21;
template <typename T, int NTH, bool CLUSTER, bool SMALL>
__global__ void __launch_bounds__(Place<NTH, CLUSTER>::CTA, Place<NTH, CLUSTER>::CTAS) k_policy(adacgd_policy_args a, const float* weight, float* tl,
                                                                     float* tk, float* tc, double* own, u32* ticket) {
  constexpr int CTA = Place<NTH, CLUSTER>::CTA, ROWS = Place<NTH, CLUSTER>::ROWS;
  __shared__ Soft sh[32], xch[8];
  __shared__ int counted[32];
  __shared__ double mine[3][ROWS];
  pdl_trigger();
  const Place<NTH, CLUSTER> at;
  const long long row = at.row;
  if (!SMALL && row >= a.rows.tokens) return;       // all of the row's lanes; only where NTH <= 32
  const int vocab = (int)a.rows.vocab, slot = NTH < 128 ? threadIdx.x / NTH : 0;
  const bool here = row < a.rows.tokens;
  // fetched together, not one after the other
  const bool counts = here && (!a.rows.mask || a.rows.mask[row]);
  const long long y = here ? label_at(a.rows, row) : -1;
  const float A = here ? a.advantages[row] : 0.f, old = here ? a.old_logp[row] : 0.f, ref = here && a.ref_logp ? a.ref_logp[row] : 0.f;
  T* d = a.dlogits ? (T*)a.dlogits + row * a.dlogits_stride : nullptr;
  int total = 0;
  if (SMALL) {
    total = (int)a.rows.tokens;
    if (a.rows.mask) {
      int c = count_share<NTH>(a.rows.mask, total, at.t);
#pragma unroll
      for (int o = (NTH < 32 ? NTH : 32) / 2; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      total = c;
      if (NTH > 32) {
        if ((threadIdx.x & 31) == 0) counted[threadIdx.x >> 5] = c;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < NTH / 32; ++w) total += counted[w];
      }
    }
  }
  if (SMALL && at.t == 0) mine[0][slot] = mine[1][slot] = mine[2][slot] = 0.0;
  if (!counts) {
    if (here && at.t == 0 && at.part == 0) {
      if (!SMALL) tl[row] = tk[row] = tc[row] = 0.f;
      if (a.logp) a.logp[row] = 0.f;
    }
    if (here && d) thread_zero<T, NTH>(d, cut_row(d, vocab, at.part, at.parts), at.t);
    pdl_wait();
    if (!SMALL) return;
  } else {
    row_begin<CLUSTER>();
    const T* x = (const T*)a.rows.logits + row * a.rows.logits_stride;
    const int label = y >= 0 && y < vocab ? (int)y : -1;
    const float z = label >= 0 ? to_f(x[label]) : NAN;
    const Cut cut = cut_row(x, vocab, at.part, at.parts);
    const Soft v = row_soft<NTH, CLUSTER>(thread_soft<T, NTH>(x, cut, at.t), sh, xch);
    const double logp = logp64(z, v);
    // the same weight for all, or the sequence's
    const long long q = a.per_sequence ? seq_of(a.rows.seq_start, row, a.rows.sequences, a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences) : 0;
    pdl_wait();
    const float w = SMALL ? (float)(1.0 / (double)total) : weight[q];
    const Token tok = token_loss(logp, old, A, a.ref_logp != nullptr, ref, a.clip_low, a.clip_high, a.kl_beta);
    if (at.t == 0 && at.part == 0) {
      if (a.logp) a.logp[row] = (float)logp;
      if (SMALL) {
        mine[0][slot] = (double)w * (double)tok.loss;
        mine[1][slot] = (double)tok.kl;
        mine[2][slot] = tok.clipped ? 1.0 : 0.0;
      } else {
        tl[row] = tok.loss;
        tk[row] = tok.kl;
        tc[row] = tok.clipped ? 1.f : 0.f;
      }
    }
    if (d) thread_grad<T, NTH, true>(x, d, cut, at.t, same_phase(x, d), label, log2_rel(z, v.m), a.grad_scale * (w * tok.slope), v.m, v.s);
  }
  if (!SMALL) return;
  __syncthreads();
  if (threadIdx.x < 3) {
    double v = 0.0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) v += mine[threadIdx.x][r];
    own[3ll * blockIdx.x + threadIdx.x] = v;
  }
  if (!last_to_arrive(ticket, gridDim.x)) return;
  __shared__ double shd[CTA / 32];
  double v[3] = {0.0, 0.0, 0.0};
#pragma unroll 4
  for (u32 k = threadIdx.x; k < gridDim.x; k += CTA) {
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] += __ldcg(&own[3ll * k + i]);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) v[i] = block_sum_f64<CTA>(v[i], shd);
  if (threadIdx.x == 0) write_policy(a.loss, a.stats, v[0], v[1], v[2], (double)total);
}

// The sums over tokens, in a fixed order: a CTA takes SUM_ROWS of them, the last one adds the CTAs'.
constexpr int SUM_ROWS = 4096, SUM_NT = 512;
__global__ void __launch_bounds__(SUM_NT) k_policy_sum(adacgd_policy_args a, const float* weight, const float* tl,
                                                       const float* tk, const float* tc, double* own, u32* ticket) {
  __shared__ double sh[SUM_NT / 32];
  pdl_wait();
  const long long lo = (long long)blockIdx.x * SUM_ROWS, hi = min((long long)a.rows.tokens, lo + SUM_ROWS);
  double v[3] = {0.0, 0.0, 0.0};
  for (long long t = lo + threadIdx.x; t < hi; t += SUM_NT) {
    const long long q = a.per_sequence ? seq_of(a.rows.seq_start, t, a.rows.sequences, a.rows.seq_start ? 0 : a.rows.tokens / a.rows.sequences) : 0;
    v[0] += (double)weight[q] * (double)tl[t];     // weighted here: losses of both signs cancel, a product rounded before would show
    v[1] += (double)tk[t];
    v[2] += (double)tc[t];
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    v[i] = block_sum_f64<SUM_NT>(v[i], sh);
    if (threadIdx.x == 0) own[3ll * blockIdx.x + i] = v[i];
  }
  if (gridDim.x > 1) {
    if (!last_to_arrive(ticket, gridDim.x)) return;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      v[i] = 0.0;
      for (u32 k = threadIdx.x; k < gridDim.x; k += SUM_NT) v[i] += __ldcg(&own[3ll * k + i]);
      v[i] = block_sum_f64<SUM_NT>(v[i], sh);
    }
  }
  if (threadIdx.x == 0) write_policy(a.loss, a.stats, v[0], v[1], v[2], (double)weight[a.rows.sequences]);
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
// Launches with optional cluster and programmatic dependence on the kernel before.
template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kern)(KArgs...), unsigned grid, int block, int cluster, bool pdl, cudaStream_t st, int smem, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = cluster;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}

unsigned ctas(long long rows, int rows_per_cta, int cluster) {
  return (unsigned)((rows + rows_per_cta - 1) / rows_per_cta * cluster);
}

// Threads a row and CTAs a row (a cluster, only where rows would leave SMs idle).
struct Split { int threads, cluster; };
Split split_of(long long rows, long long vocab, int threads, const Where& at) {
  Split s = {threads, 1};   // with rows for all SMs
  while (s.threads < 512 && rows * s.threads < 1024ll * at.sms && vocab > 8 * s.threads) s.threads = s.threads < 32 ? 32 : s.threads * 4;
  if (s.threads >= 512)
    while (s.cluster < 8 && rows * s.cluster * 2 <= 2 * at.sms && vocab / (s.cluster * 2) >= 4096) s.cluster *= 2;
  if (s.threads > 512 && s.cluster > 1) s.threads = 512;
  return s;
}
// One pass: a row's two reductions cost every warp the same, about what 128 elements a thread do, and many rows on an SM hide them; so
// as few threads a row as that.  Log-probabilities of 2^28 elements, us at 8 / 32 / 128 / 512 threads a row: bfloat16 512 wide 101 / 283 /
// - / -; 1536 90 / 127 / - / -; 2048 91 / 97 / 292 / -; 4096 95 / 89 / 144 / -; 8192 96 / 88 / 101 / 330; 16384 - / 89 / 86 / 170; 32768 - /
// 101 / 86 / 113; 131072 - / - / 93 / 87; binary32, 131072 rows, 1024 wide 82 / 88; 1536 121 / 119.
Split split_once(long long rows, long long vocab, int size, const Where& at) {
  return split_of(rows, vocab, vocab * size <= 4096 ? 8 : vocab <= 8192 ? 32 : (vocab <= 65536 ? 128 : 512), at);
}
// Two passes, the second from the cache: what the resident threads hold between their passes (1024 an SM) has to stay in it beside
// what is written, so a thread may have 400 bytes of a row, and 640 where more threads a row cost more than the cache gives.
// Policy loss, us at 8 / 32 / 128 / 256 / 512 / 1024 threads a row, bfloat16: 131072 x 1024 110 / 143; 131072 x 1536 160 / 195; 131072 x
// 2048 218 / 209; 65536 x 4096 - / 194 / 273; 32768 x 8192 - / 213 / 208; 8192 x 32000 - / - / 211 / 200 / 248; 8192 x 50001 368 / 313 /
// 351 / 537 from 128 on; 4096 x 65536 255 / 212 / 209 from 128 on; 4096 x 131072 416 / 467 and 2048 x 262145 511 / 464 at 512 / 1024;
// binary32: 131072 x 512 109 / 136; 131072 x 1024 251 / 197; 65536 x 4096 - / 474 / 378.
constexpr int PASS_BYTES = 400, PASS_BYTES_WIDE = 640;
Split split_twice(long long rows, long long vocab, int size, const Where& at) {
  const long long bytes = vocab * size;
  for (int threads : {8, 32, 128, 256})
    if (bytes <= threads * PASS_BYTES) return split_of(rows, vocab, threads, at);
  return split_of(rows, vocab, bytes <= 512 * PASS_BYTES_WIDE ? 512 : 1024, at);
}
#define BY_THREADS(s, call)                                                                            \
  (s.threads == 512 ? ([&] { constexpr int NTH = 512; constexpr bool CL = false; return call; }())     \
   : s.threads == 128 ? ([&] { constexpr int NTH = 128; constexpr bool CL = false; return call; }())   \
   : s.threads == 32 ? ([&] { constexpr int NTH = 32; constexpr bool CL = false; return call; }())     \
                     : ([&] { constexpr int NTH = 8; constexpr bool CL = false; return call; }()))
#define BY_SPLIT_ONCE(s, call) \
  (s.cluster > 1 ? ([&] { constexpr int NTH = 512; constexpr bool CL = true; return call; }()) : BY_THREADS(s, call))
#define BY_SPLIT_TWICE(s, call)                                                                        \
  (s.cluster > 1 ? ([&] { constexpr int NTH = 512; constexpr bool CL = true; return call; }())         \
   : s.threads == 1024 ? ([&] { constexpr int NTH = 1024; constexpr bool CL = false; return call; }()) \
   : s.threads == 256 ? ([&] { constexpr int NTH = 256; constexpr bool CL = false; return call; }())   \
                      : BY_THREADS(s, call))

template <typename T>
cudaError_t logp_t(const adacgd_token_rows& r, float* logp, float* lse, float* zl, float* sum, float* top, const Where& at) {
  const Split s = split_once(r.tokens, r.vocab, (int)sizeof(T), at);
  return BY_SPLIT_ONCE(s, (launch(k_logp<T, NTH, CL>, ctas(r.tokens, Place<NTH, CL>::ROWS, s.cluster), Place<NTH, CL>::CTA, s.cluster, false,
                             at.stream, 0, r, logp, lse, zl, sum, top)));
}

template <typename T>
int preference_t(const TrainScratch& s, const adacgd_preference_args& a, const Where& at) {
  int n = 1;
  const long long rows = a.rows.tokens;
  if (rows) {
    if (logp_t<T>(a.rows, nullptr, nullptr, s.tok_a, s.tok_b, s.tok_c, at) != cudaSuccess) return -1;
    ++n;
  }
  // Slices of at least two tokens a thread, as long as SMs are free.  The six sums of each fit: 6 pairs slices <= 6 tokens / 1024.
  const long long pairs = a.rows.sequences / 2;
  long long slices = rows / a.rows.sequences / (2 * PAIR_NT);
  if (slices * pairs > at.sms) slices = at.sms / pairs;
  if (slices < 1) slices = 1;
  if (launch(k_pairs, (unsigned)(pairs * slices), PAIR_NT, 1, rows > 0, at.stream, 0, a, s.tok_a, s.tok_b, s.tok_c, s.seq, s.part, (u32)slices,
             s.tickets) != cudaSuccess)
    return -1;
  if (a.dlogits && rows) {
    Split sp = split_once(rows, a.rows.vocab, (int)sizeof(T), at);
    const u32 parts = (u32)sp.cluster;      // no reduction: parts of a row need no cluster
    sp.cluster = 1;
    const cudaError_t e = BY_SPLIT_ONCE(sp, (launch(k_preference_grad<T, NTH>, ctas(rows * parts, Place<NTH, false>::ROWS, 1), Place<NTH, false>::CTA,
                                               1, true, at.stream, 0, a, s.seq, s.tok_a, s.tok_b, s.tok_c, parts)));
    if (e != cudaSuccess) return -1;
    ++n;
  }
  return n;
}

template <typename T>
int policy_t(const TrainScratch& s, const adacgd_policy_args& a, const Where& at) {
  const Split sp = split_twice(a.rows.tokens, a.rows.vocab, (int)sizeof(T), at);
  if (!a.per_sequence && sp.cluster == 1 && a.rows.tokens > 0 && a.rows.tokens <= MAX_SMALL_CTAS &&
      a.rows.tokens * a.rows.vocab <= SMALL_ELEMENTS &&
      sp.threads != 256 && sp.threads != 1024)      // rows so long have clusters when they are so few
    return BY_THREADS(sp, (launch(k_policy<T, NTH, CL, true>, ctas(a.rows.tokens, Place<NTH, CL>::ROWS, 1), Place<NTH, CL>::CTA, 1, false, at.stream, 0,
                                  a, (const float*)nullptr, s.tok_a, s.tok_b, s.tok_c, s.own, s.tickets + 1))) == cudaSuccess
               ? 1
               : -1;
  if (launch(k_policy_weights, 1u, 1024, 1, false, at.stream, 0, a, s.seq) != cudaSuccess) return -1;
  if (!a.rows.tokens) return 1;
  cudaError_t e = BY_SPLIT_TWICE(sp, (launch(k_policy<T, NTH, CL, false>, ctas(a.rows.tokens, Place<NTH, CL>::ROWS, sp.cluster), Place<NTH, CL>::CTA, sp.cluster,
                                       true, at.stream, 0, a, s.seq, s.tok_a, s.tok_b, s.tok_c, s.own, s.tickets + 1)));
  if (e == cudaSuccess)
    e = launch(k_policy_sum, (unsigned)((a.rows.tokens + SUM_ROWS - 1) / SUM_ROWS), SUM_NT, 1, true, at.stream, 0, a, s.seq, s.tok_a, s.tok_b,
               s.tok_c, s.part, s.tickets + 1);
  return e == cudaSuccess ? 3 : -1;
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_token_logp(const adacgd_token_rows& r, float* logp, float* lse, const Where& at) {
  BY_TYPE(r.dtype, (logp_t<T>(r, logp, lse, nullptr, nullptr, nullptr, at) == cudaSuccess ? 1 : -1))
}
int launch_preference(const TrainScratch& s, const adacgd_preference_args& a, const Where& at) {
  BY_TYPE(a.rows.dtype, (preference_t<T>(s, a, at)))
}
int launch_policy(const TrainScratch& s, const adacgd_policy_args& a, const Where& at) { BY_TYPE(a.rows.dtype, (policy_t<T>(s, a, at))) }

}  // namespace adacgd
