// Dropout and layer norm with the residual sum and dropout in front of it, forward and backward (adacgd_train.h).
//
// All three are bound by memory: a few operations an element against 4 to 20 bytes of traffic.  So every element is read
// once and written once, a row stays on the SM between its statistics and its result (forward in registers, backward in shared
// memory), and what is left is to keep enough loads in flight.
//
// The unit is a run of eight elements, which is 16 bytes (32 of binary32) and one block of the dropout generator.  Matrices whose
// rows do not lie on runs (gaps or alignments that shift from row to row) take kernels that go element by element.
#include <cooperative_groups.h>

#include "adacgd_train.cuh"

namespace cg = cooperative_groups;

namespace adacgd {

namespace {

// Bit j set: element j of the block is kept.
__device__ __forceinline__ u32 keep_bits(u64 block, const Drop& d) {
  const uint4 w = philox(block, d);
  u32 m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m |= (kept(w, j, d) ? 1u : 0u) << j;
  return m;
}

// --------------------------------------------------------------------------
// dropout
// --------------------------------------------------------------------------
// Two blocks a thread and 48 registers (five CTAs an SM).  32768 x 8192 bfloat16, p = 0.1, measured: the generator after the
// loads' first use 216 us, before it 185 us; one block a thread 208 to 220 us; four blocks 182 to 185 us but for the smallest
// calls half the threads.  p = 0 takes 163 us, the copy itself 164 us at the measured copy rate: what is left of the
// difference is the comparisons, selections and conversions of the elements, which fill the integer pipe to two thirds.
constexpr int DROP_NT = 256, DROP_RUNS = 2;

// A thread takes DROP_RUNS blocks of eight elements.  VEC: every block is eight aligned columns of one row, or the rows
// are one long run.
template <typename T, bool VEC>
__global__ void __launch_bounds__(DROP_NT, 5) k_dropout(const T* x, long long xs, const T* res, long long rs, T* out, long long os,
                                                     long long rows, long long cols, Drop d) {
  const long long n = rows * cols, blocks = (n + 7) >> 3;
  const long long b0 = (long long)blockIdx.x * (DROP_NT * DROP_RUNS) + threadIdx.x;
  if (VEC) {
    Run<T> a[DROP_RUNS], r[DROP_RUNS];
    long long off_o[DROP_RUNS];
#pragma unroll
    for (int u = 0; u < DROP_RUNS; ++u) {
      const long long b = b0 + u * DROP_NT, i = b << 3;
      if (i + 8 > n) continue;
      long long row = 0, c = i;
      if (rows > 1) {
        row = (n >> 32) ? i / cols : (long long)((u32)i / (u32)cols);
        c = i - row * cols;
      }
      a[u] = load_run(x + row * xs + c);
      if (res) r[u] = load_run(res + row * rs + c);
      off_o[u] = row * os + c;
    }
    uint4 w[DROP_RUNS];      // made while the loads are under way
    if (d.on) {
#pragma unroll
      for (int u = 0; u < DROP_RUNS; ++u) w[u] = philox((u64)(b0 + u * DROP_NT), d);
    }
#pragma unroll
    for (int u = 0; u < DROP_RUNS; ++u) {
      const long long b = b0 + u * DROP_NT;
      if ((b << 3) + 8 > n) continue;
      float v[8], base[8];
      unpack(a[u], v);
      if (res) unpack(r[u], base);
      if (d.on) {
        if (res) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = kept(w[u], j, d) ? scaled(v[j], base[j], d) : base[j];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = kept(w[u], j, d) ? v[j] * d.scale : 0.f;
        }
      } else if (res) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = base[j] + v[j];
      }
      store_run(out + off_o[u], v);
    }
    if ((n & 7) && rows == 1) {           // the last, shorter block of one long run
      const long long b = n >> 3;
      if (b >= b0 - threadIdx.x && b < b0 - threadIdx.x + DROP_NT * DROP_RUNS && threadIdx.x < (n & 7)) {
        const long long i = (b << 3) + threadIdx.x;
        const float base = res ? to_f(res[i]) : 0.f, v = to_f(x[i]);
        out[i] = from_f<T>(!d.on ? (res ? base + v : v) : res ? drop_one(v, base, (u64)i, d) : drop_one(v, (u64)i, d));
      }
    }
    return;
  }
  for (int u = 0; u < DROP_RUNS; ++u) {
    const long long b = b0 + u * DROP_NT;
    if (b >= blocks) return;
    const u32 m = d.on ? keep_bits((u64)b, d) : 0xffu;
    long long i = b << 3;
    long long row = i / cols, c = i - row * cols;
    for (int j = 0; j < 8 && i < n; ++j, ++i) {
      const float base = res ? to_f(res[row * rs + c]) : 0.f;
      float v = to_f(x[row * xs + c]);
      if (d.on) v = (m >> j) & 1u ? (res ? scaled(v, base, d) : v * d.scale) : base;
      else if (res) v = base + v;
      out[row * os + c] = from_f<T>(v);
      if (++c == cols) { c = 0; ++row; }
    }
  }
}

// --------------------------------------------------------------------------
// rows of runs
// --------------------------------------------------------------------------
// The fast form.  A run is eight elements whose number (row * cols + col) begins at a multiple of eight, which is also a block
// of the dropout generator.  In matrices without gaps between rows, and in aligned ones whose width is a multiple of eight, a
// run is aligned to its size in memory, whatever the width.  A row is its whole runs and, with EDGE (other widths), up to seven
// elements in front of them and seven behind, which threads take one each: a warp would execute a run that only partly belongs
// to the row element by element, for every row.
// `ph` = where in its run a row begins.  Rows whose numbers differ by a multiple of PERIOD = 8 / gcd(cols, 8) have the same ph, so
// a walker (NTH threads) that takes such rows only finds the same columns in the same registers for every one of them: weights
// are loaded once, weight gradients summed in place.
constexpr int MAX_PERIOD = 8;

__host__ __device__ constexpr int walk_cta(int nth) { return nth < 256 ? 256 : nth; }   // narrow rows: several walkers a CTA, whose partial sums it adds
template <typename T, int NTH, int R, int ARRAYS> struct Walk {   // R: runs a thread
  static constexpr int CTA = walk_cta(NTH);
  static constexpr int ROWS = CTA / NTH;
  static constexpr int PIECES = sizeof(T) / 2;                    // 16-byte pieces of a run
  static constexpr int STAGE = ARRAYS * R * PIECES * CTA * 16;    // bytes
  // registers allow 512 threads on an SM; 32-bit rows have half the elements a byte, so half of those threads keep up
  static constexpr int THREADS = sizeof(T) == 4 ? 256 : 512;
  static constexpr int FIT = 200 * 1024 / (STAGE * (THREADS > CTA ? THREADS / CTA : 1));
  static constexpr int STAGES = FIT >= 4 ? 4 : FIT >= 2 ? FIT : 1;
  static constexpr int SMEM = STAGES * STAGE;
};

// A row's whole runs, and the column outside them that a thread takes (-1: none).
struct Lie {
  int first, runs, edge;
};
template <bool EDGE>
__device__ __forceinline__ Lie lie_of(int ph, int cols, int t) {
  Lie l;
  l.first = EDGE ? min(cols, (8 - ph) & 7) : 0;
  l.runs = (cols - l.first) >> 3;
  l.edge = -1;
  if (EDGE) {
    const int c = t < l.first ? t : 8 * l.runs + t;      // behind the runs: first + 8 runs + (t - first)
    if (c < cols) l.edge = c;
    if (t >= 16) l.edge = -1;
  }
  return l;
}

struct Walker {
  long long row, step;
  int t, slot, ph;
};
// Which rows a thread's walker takes: those of one class modulo the period, evenly dealt among the class's walkers.
template <int NTH>
__device__ __forceinline__ Walker walker_of(int cols, int group, int groups) {
  constexpr int ROWS = walk_cta(NTH) / NTH;
  const int period = MAX_PERIOD / (cols & 1 ? 1 : (cols & 2 ? 2 : (cols & 4 ? 4 : 8)));
  Walker w;
  w.t = threadIdx.x % NTH;
  w.slot = threadIdx.x / NTH;
  const long long id = (long long)group * ROWS + w.slot, all = (long long)groups * ROWS;   // all: a multiple of the period
  w.row = id;
  w.step = all;
  w.ph = (int)((id % period) * cols & 7);
  return w;
}

__device__ __forceinline__ void copy16(u32 to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sends a row's runs of one array on their way.
// Binary32: the lanes of a row's warp copy each other's pieces, consecutive ones together, because a lane's own two would be
// halves of sectors; they meet at warp_meets() before they read and before they send again.
template <typename T>
__device__ __forceinline__ void warp_meets() {
  if (sizeof(T) == 4) __syncwarp();
}
template <typename T, int NTH, int R, int CTA>
__device__ __forceinline__ void send_runs(u32 ring32, const T* first, int runs, int t) {
  constexpr int L = NTH < 32 ? NTH : 32, PIECES = sizeof(T) / 2, E = 16 / (int)sizeof(T);
  const int tl = t % L;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int q = PIECES * (r * NTH + t - tl) + tl + i * L;          // piece of the row
      if (q < PIECES * runs) copy16(ring32 + (u32)(r * PIECES * CTA + PIECES * ((int)threadIdx.x - tl) + tl + i * L) * 16, first + q * E);
    }
  }
}
// A thread's r-th run of an array's stage.
template <typename T, int CTA>
__device__ __forceinline__ void take_run(const uint4* stage, int r, float (&o)[8]) {
  constexpr int PIECES = sizeof(T) / 2;
  Run<T> v;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) v.v[i] = stage[r * PIECES * CTA + PIECES * threadIdx.x + i];
  unpack(v, o);
}
// The walker's own barrier where its CTA has several.
template <int NTH, int CTA>
__device__ __forceinline__ void walker_sync() {
  if (NTH == CTA) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / NTH), "n"(NTH) : "memory");
}

// Sum over a walker's threads, the same bits in each; `sh` alternates.  NTH <= 32: within the warp.
template <int NTH>
__device__ __forceinline__ float walker_sum(float v, float* sh) {
#pragma unroll
  for (int o = (NTH < 32 ? NTH : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (NTH <= 32) return v;
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NTH / 32; ++w) t += sh[w];
  return t;
}

// Eight weights of a 16-byte aligned vector from any column c on: the aligned pieces around them, shifted.
__device__ __forceinline__ void shift_weights(const float* w, int c, float (&o)[8]) {
  const int off = c & 3;
  const float4* p = reinterpret_cast<const float4*>(w + (c - off));
  const float4 x = p[0], y = p[1];
  if (off == 0) {
    o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w; o[4] = y.x; o[5] = y.y; o[6] = y.z; o[7] = y.w;
    return;
  }
  const float4 z = p[2];
  if (off == 1) {
    o[0] = x.y; o[1] = x.z; o[2] = x.w; o[3] = y.x; o[4] = y.y; o[5] = y.z; o[6] = y.w; o[7] = z.x;
  } else if (off == 2) {
    o[0] = x.z; o[1] = x.w; o[2] = y.x; o[3] = y.y; o[4] = y.z; o[5] = y.w; o[6] = z.x; o[7] = z.y;
  } else {
    o[0] = x.w; o[1] = y.x; o[2] = y.y; o[3] = y.z; o[4] = y.w; o[5] = z.x; o[6] = z.y; o[7] = z.z;
  }
}
template <typename P>
__device__ __forceinline__ void shift_weights(const P* w, int c, float (&o)[8]) {
  const int off = c & 7;
  const uint4* p = reinterpret_cast<const uint4*>(w + (c - off));
  const uint4 x = p[0];
  const uint4 y = off ? p[1] : x;
  u32 a[5];
  switch (off >> 1) {
    case 0: a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w; a[4] = y.x; break;
    case 1: a[0] = x.y; a[1] = x.z; a[2] = x.w; a[3] = y.x; a[4] = y.y; break;
    case 2: a[0] = x.z; a[1] = x.w; a[2] = y.x; a[3] = y.y; a[4] = y.z; break;
    default: a[0] = x.w; a[1] = y.x; a[2] = y.y; a[3] = y.z; a[4] = y.w; break;
  }
  const u32 by = (off & 1) * 16;
  Run<P> r;
  r.v[0] = make_uint4(__funnelshift_r(a[0], a[1], by), __funnelshift_r(a[1], a[2], by), __funnelshift_r(a[2], a[3], by),
                      __funnelshift_r(a[3], a[4], by));
  unpack(r, o);
}

// Eight weights from column c on (c + 8 <= cols), `other` without a vector.
template <typename P>
__device__ __forceinline__ void load_weights(const P* w, int c, int cols, float other, float (&o)[8]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = other;
  } else if (((uintptr_t)w & 15) == 0 && c + 16 <= cols) {     // the pieces read end within 15 elements
    shift_weights(w, c, o);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = to_f(w[c + j]);
  }
}
// Kept in the parameter's own type: half the registers.
template <typename P> struct Held {
  uint4 v;
  __device__ __forceinline__ void set(const float (&x)[8]) { v = pack_run<P>(x); }   // exact: x came from P
  __device__ __forceinline__ void get(float (&x)[8]) const {
    Run<P> r;
    r.v[0] = v;
    unpack(r, x);
  }
};
template <> struct Held<float> {
  float v[8];
  __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x[j];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[j];
  }
};

// --------------------------------------------------------------------------
// layer norm
// --------------------------------------------------------------------------
//   v = dropout(x) + residual,  mean = sum v / n,  rstd = 1 / sqrt(sum (v - mean)^2 / n + eps),  out = (v - mean) rstd weight + bias
// NTH threads take one row, CTAs are handed out by the hardware: the row's two sums and the loads of other rows on the SM hide each
// other (a grid of as many CTAs as fit, with rows through an asynchronous ring, took 404 us where this took 374).  The mean first,
// then the squares about it, over registers: no cancellation.
// 32768 x 8192 bfloat16 with residual and sum (four arrays, 2.1 GB): 316 us = 6.8 TB/s, the copy rate; with dropout 353 us, where
// the generator's products and the selections fill the issue slots.
template <int NTH> struct Group {
  static constexpr int CTA = NTH <= 32 ? 128 : NTH;
  static constexpr int ROWS = CTA / NTH;
};
template <typename T, typename P, int NTH, int R, bool EDGE>
__global__ void __launch_bounds__(Group<NTH>::CTA) k_norm(const __grid_constant__ adacgd_norm_args a, const __grid_constant__ Drop d) {
  __shared__ float sh[2][NTH < 32 ? 1 : NTH / 32];
  const int cols = (int)a.cols, t = threadIdx.x % NTH;
  const long long row = (long long)blockIdx.x * Group<NTH>::ROWS + threadIdx.x / NTH;
  if (NTH >= 32 && row >= a.rows) return;          // whole warps; no barrier follows where a CTA has several rows
  const bool live = row < a.rows;
  const u64 i0 = (u64)row * (u64)cols;
  Lie l = lie_of<EDGE>((int)(i0 & 7), cols, t);
  if (!live) {
    l.runs = 0;
    l.edge = -1;
  }
  const T* const x = (const T*)a.x + row * a.x_stride;
  const T* const res = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  Run<T> raw[R], rest[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int g = r * NTH + t;
    if (g < l.runs) {
      raw[r] = load_run(x + l.first + 8 * g);
      if (res) rest[r] = load_run(res + l.first + 8 * g);
    }
  }
  float ev = 0.f, er = 0.f;
  if (EDGE && l.edge >= 0) {
    ev = to_f(x[l.edge]);
    if (res) er = to_f(res[l.edge]);
  }
  uint4 bits[R];                                   // made while the loads are under way
  if (d.on) {
#pragma unroll
    for (int r = 0; r < R; ++r) bits[r] = philox(((i0 + l.first) >> 3) + (u64)(r * NTH + t), d);
  }
  F2 v[R][4], acc = f2(0.f, 0.f);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r * NTH + t < l.runs) {
      float u[8], b[8];
      unpack(raw[r], u);
      if (res) unpack(rest[r], b);
      if (d.on) {
        if (res) {
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = kept(bits[r], j, d) ? scaled(u[j], b[j], d) : b[j];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = kept(bits[r], j, d) ? u[j] * d.scale : 0.f;
        }
      }
      pairs_of(u, v[r]);
      if (res && !d.on) {
        F2 b2[4];
        pairs_of(b, b2);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[r][j] = add2(v[r][j], b2[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = add2(acc, v[r][j]);
    }
  }
  if (EDGE && l.edge >= 0) {
    if (!d.on) ev = er + ev;
    else ev = res ? drop_one(ev, er, i0 + l.edge, d) : drop_one(ev, i0 + l.edge, d);
  }
  float lo, hi;
  split(acc, lo, hi);
  const float mean = walker_sum<NTH>(lo + hi + ev, sh[0]) / (float)cols;
  const F2 minus = f2(-mean, -mean);
  acc = f2(0.f, 0.f);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r * NTH + t < l.runs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const F2 z = add2(v[r][j], minus);
        acc = fma2(z, z, acc);
      }
    }
  }
  split(acc, lo, hi);
  if (EDGE && l.edge >= 0) lo = fmaf(ev - mean, ev - mean, lo);
  const float rstd = 1.f / sqrtf(walker_sum<NTH>(lo + hi, sh[1]) / (float)cols + a.eps);
  if (!live) return;
  T* const out = (T*)a.out + row * a.out_stride;
  T* const sum = a.sum ? (T*)a.sum + row * a.sum_stride : nullptr;
  const P* const weight = (const P*)a.weight;
  const P* const bias = (const P*)a.bias;
  const F2 scale = f2(rstd, rstd);
  const bool even = !EDGE && (((uintptr_t)weight | (uintptr_t)bias) & (8 * sizeof(P) - 1)) == 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int g = r * NTH + t, c = l.first + 8 * g;
    if (g < l.runs) {
      float u[8], p[8], q[8];
      if (sum) {
        floats_of(v[r], u);
        store_run(sum + c, u);
      }
      if (even) {
        if (weight) unpack(load_run(weight + c), p);
        if (bias) unpack(load_run(bias + c), q);
      } else {
        if (weight) load_weights(weight, c, cols, 1.f, p);
        if (bias) load_weights(bias, c, cols, 0.f, q);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        F2 z = mul2(add2(v[r][j], minus), scale);
        if (weight && bias) z = fma2(z, f2(p[2 * j], p[2 * j + 1]), f2(q[2 * j], q[2 * j + 1]));
        else if (weight) z = mul2(z, f2(p[2 * j], p[2 * j + 1]));
        else if (bias) z = add2(z, f2(q[2 * j], q[2 * j + 1]));
        split(z, u[2 * j], u[2 * j + 1]);
      }
      store_run(out + c, u);
    }
  }
  if (EDGE && l.edge >= 0) {
    if (sum) sum[l.edge] = from_f<T>(ev);
    out[l.edge] = from_f<T>(fmaf((ev - mean) * rstd, weight ? to_f(weight[l.edge]) : 1.f, bias ? to_f(bias[l.edge]) : 0.f));
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// --------------------------------------------------------------------------
// layer norm, backward
// --------------------------------------------------------------------------
//   h = (s - mean) rstd,  g = dout weight,  ds = rstd (g - mean(g) - h mean(g h)) + dsum
//   dresidual = ds,  dx = the forward pass's dropout of ds,  dweight = sum over rows of dout h,  dbias = sum over rows of dout
// dout and s are read once for all results: first for the two sums and the weight gradients, then, from shared memory, for ds.
// Rows wider than NTH * R runs are cut into as many column parts as the cluster has CTAs; the two sums then meet in distributed
// shared memory.
// K rows go through the two phases together, so that their reductions share one barrier: 465 -> 341 us at 32768 x 8192 bfloat16,
// K = 1 -> 2; now 325 us = 6.6 TB/s, the copy rate, and 440 us = 6.1 TB/s with dropout (five arrays).  The weight gradients of a
// column stay in the registers of the thread that always meets it, so the grid is as many CTAs as fit, and rows come through a ring
// of asynchronous copies because registers hold no second row.
template <typename T, typename P, int NTH, int R, bool CLUSTER, bool EDGE, int ARRAYS>
__global__ void __launch_bounds__(Walk<T, NTH, R, ARRAYS>::CTA) k_norm_bwd(const __grid_constant__ adacgd_norm_backward_args a,
                                                                      const __grid_constant__ Drop d, float* __restrict__ part,
                                                                      long long max_cols) {
  typedef Walk<T, NTH, R, ARRAYS> W;      // ARRAYS: 3 with dsum, 2 without
  constexpr int CTA = W::CTA, S = W::STAGES, A = R * W::PIECES * CTA, K = S >= 4 ? 2 : 1, WARPS = NTH < 32 ? 1 : NTH / 32;
  extern __shared__ uint4 ring[];
  __shared__ float sh_all[W::ROWS][2][2 * K][WARPS];
  __shared__ float xch[2][8][2 * K];
  asm volatile("griddepcontrol.launch_dependents;");     // the sum of the partials may take its place and wait
  int nparts = 1, rank = 0;
  if (CLUSTER) {
    nparts = (int)cg::this_cluster().num_blocks();
    rank = (int)cg::this_cluster().block_rank();
    cg::this_cluster().sync();   // every CTA has started before any writes into another's shared memory
  }
  const int cols = (int)a.cols;
  const Walker w = walker_of<NTH>(cols, blockIdx.x / nparts, gridDim.x / nparts);
  float (&sh)[2][2 * K][WARPS] = sh_all[w.slot];
  const Lie l = lie_of<EDGE>(w.ph, cols, w.t);
  const int g0 = CLUSTER ? (int)((long long)l.runs * rank / nparts) : 0;                  // this part's first run and their number
  const int runs = CLUSTER ? (int)((long long)l.runs * (rank + 1) / nparts) - g0 : l.runs;
  const int first = l.first + 8 * g0;
  const int edge = rank == 0 ? l.edge : -1;                                               // the first part takes the edges
  const T* const dout = (const T*)a.dout;
  const T* const s_in = (const T*)a.s;
  const T* const dsum = (const T*)a.dsum;
  const u32 ring32 = (u32)__cvta_generic_to_shared(ring);
  const float inv = 1.f / (float)cols, less = fmaf(-inv, (float)cols, 1.f) * inv;
  auto mean_of = [&](float sum) {      // sum / cols with one rounding, 1 / cols being inv + less: a constant's mean is the constant
    const float m = sum * inv;
    return fabsf(m) < INFINITY ? fmaf(sum, inv, sum * less) : m;
  };
  Held<P> wt[R];
  F2 dw[R][4], db[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int g = r * NTH + w.t;
    if (g < runs) load_weights((const P*)a.weight, first + 8 * g, cols, 1.f, o);
    wt[r].set(o);
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[r][j] = db[r][j] = f2(0.f, 0.f);
  }
  const float ew = EDGE && edge >= 0 && a.weight ? to_f(((const P*)a.weight)[edge]) : 1.f;
  float edw = 0.f, edb = 0.f;
  auto send = [&](long long row, int stage) {
    if (row < a.rows) {
      const u32 to = ring32 + (u32)(stage * ARRAYS * A * 16);
      send_runs<T, NTH, R, CTA>(to, dout + row * a.dout_stride + first, runs, w.t);
      send_runs<T, NTH, R, CTA>(to + A * 16, s_in + row * a.s_stride + first, runs, w.t);
      if (ARRAYS == 3) send_runs<T, NTH, R, CTA>(to + 2 * A * 16, dsum + row * a.dsum_stride + first, runs, w.t);
    }
    copy_commit();
  };
#pragma unroll
  for (int s = 0; s < S; ++s) send(w.row + s * w.step, s);
  // what comes through registers: statistics and edges of the rows next in turn
  float mean[K], rstd[K], ny[K], ns[K], nd[K];
  auto ask = [&](int k, long long row) {
    if (row < a.rows) {
      mean[k] = a.mean[row];
      rstd[k] = a.rstd[row];
      if (EDGE && edge >= 0) {
        ny[k] = to_f(dout[row * a.dout_stride + edge]);
        ns[k] = to_f(s_in[row * a.s_stride + edge]);
        if (ARRAYS == 3) nd[k] = to_f(dsum[row * a.dsum_stride + edge]);
      }
    }
  };
#pragma unroll
  for (int k = 0; k < K; ++k) {
    mean[k] = rstd[k] = ny[k] = ns[k] = nd[k] = 0.f;
    ask(k, w.row + k * w.step);
  }
  int stage = 0, parity = 0;
  // walkers of one warp go on together, also when the last ones have no row left
  for (long long row = w.row, lead = w.row - w.slot % (NTH < 32 ? 32 / NTH : 1); lead < a.rows; row += K * w.step, lead += K * w.step) {
    float mu[K], rs[K], ey[K], es[K], ed[K], sums[2 * K];
    bool live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      live[k] = row + k * w.step < a.rows;
      mu[k] = mean[k];
      rs[k] = rstd[k];
      ey[k] = ny[k];
      es[k] = ns[k];
      ed[k] = nd[k];
      ask(k, row + (K + k) * w.step);
    }
    copy_wait<S - K>();
    warp_meets<T>();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint4* const at = ring + (stage + k) * ARRAYS * A;
      F2 p2 = f2(0.f, 0.f), q2 = p2;
      const F2 mu2 = f2(-mu[k], -mu[k]), rs2 = f2(rs[k], rs[k]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r * NTH + w.t < runs && live[k]) {
          float y[8], h[8], v[8];
          take_run<T, CTA>(at, r, y);
          take_run<T, CTA>(at + A, r, h);
          wt[r].get(v);
          F2 y2[4], h2[4], v2[4];
          pairs_of(y, y2);
          pairs_of(h, h2);
          pairs_of(v, v2);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            h2[j] = mul2(add2(h2[j], mu2), rs2);
            dw[r][j] = fma2(y2[j], h2[j], dw[r][j]);
            db[r][j] = add2(db[r][j], y2[j]);
            v2[j] = mul2(v2[j], y2[j]);
            p2 = add2(p2, v2[j]);
            q2 = fma2(v2[j], h2[j], q2);
          }
        }
      }
      float odd;
      split(p2, sums[2 * k], odd);
      sums[2 * k] += odd;
      split(q2, sums[2 * k + 1], odd);
      sums[2 * k + 1] += odd;
      if (EDGE && edge >= 0 && live[k]) {
        const float h = (es[k] - mu[k]) * rs[k], g = ey[k] * ew;
        edw = fmaf(ey[k], h, edw);
        edb += ey[k];
        sums[2 * k] += g;
        sums[2 * k + 1] = fmaf(g, h, sums[2 * k + 1]);
      }
    }
#pragma unroll
    for (int o = (NTH < 32 ? NTH : 32) / 2; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < 2 * K; ++i) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], o);
    }
    if (NTH > 32) {
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) sh[parity][i][w.t >> 5] = sums[i];
      }
      walker_sync<NTH, CTA>();
#pragma unroll
      for (int i = 0; i < 2 * K; ++i) {
        sums[i] = 0.f;
#pragma unroll
        for (int j = 0; j < WARPS; ++j) sums[i] += sh[parity][i][j];
      }
      if (CLUSTER) {
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x < nparts) {
          float* const to = cl.map_shared_rank(&xch[parity][rank][0], threadIdx.x);
#pragma unroll
          for (int i = 0; i < 2 * K; ++i) to[i] = sums[i];
        }
        cl.sync();     // the slots of this parity are written again only behind the next rows' barrier
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) {
          sums[i] = 0.f;
          for (int j = 0; j < nparts; ++j) sums[i] += xch[parity][j][i];
        }
      }
      parity ^= 1;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const long long now = row + k * w.step;
      if (live[k]) {
        const uint4* const at = ring + (stage + k) * ARRAYS * A;
        const float p = mean_of(sums[2 * k]), cq = -rs[k] * mean_of(sums[2 * k + 1]);
        const F2 mu2 = f2(-mu[k], -mu[k]), rs2 = f2(rs[k], rs[k]), cq2 = f2(cq, cq), p2 = f2(-p, -p);
        T* const dx = (T*)a.dx + now * a.dx_stride;
        T* const dr = a.dresidual ? (T*)a.dresidual + now * a.dresidual_stride : nullptr;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int g = r * NTH + w.t, c = first + 8 * g;
          if (g < runs) {
            float y[8], h[8], v[8];
            uint4 bits;
            if (d.on) bits = philox((((u64)now * (u64)cols + first) >> 3) + (u64)g, d);
            take_run<T, CTA>(at, r, y);
            take_run<T, CTA>(at + A, r, h);
            wt[r].get(v);
            F2 y2[4], h2[4], v2[4];
            pairs_of(y, y2);
            pairs_of(h, h2);
            pairs_of(v, v2);
            // rs ((g - p) - (s - mu) (rs q)) [+ dsum]: rs^2 may be out of range where rs is not
#pragma unroll
            for (int j = 0; j < 4; ++j) y2[j] = mul2(fma2(add2(h2[j], mu2), cq2, fma2(y2[j], v2[j], p2)), rs2);
            if (ARRAYS == 3) {
              take_run<T, CTA>(at + 2 * A, r, v);
              pairs_of(v, v2);
#pragma unroll
              for (int j = 0; j < 4; ++j) y2[j] = add2(y2[j], v2[j]);
            }
            floats_of(y2, y);
            if (dr) store_run(dr + c, y);
            if (d.on) {
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = kept(bits, j, d) ? y[j] * d.scale : 0.f;
            }
            store_run(dx + c, y);
          }
        }
        if (EDGE && edge >= 0) {
          float y = fmaf(es[k] - mu[k], cq, fmaf(ey[k], ew, -p)) * rs[k];
          if (ARRAYS == 3) y += ed[k];
          if (dr) dr[edge] = from_f<T>(y);
          dx[edge] = from_f<T>(d.on ? drop_one(y, (u64)now * (u64)cols + edge, d) : y);
        }
      }
    }
    warp_meets<T>();
#pragma unroll
    for (int k = 0; k < K; ++k) send(row + (S + k) * w.step, stage + k);
    stage = stage + K == S ? 0 : stage + K;
  }
  copy_wait<0>();
  if (CLUSTER) cg::this_cluster().sync();   // no CTA leaves while another may still write into its shared memory
  if (!part) return;
  float* const pw = part + 2ll * (blockIdx.x / nparts) * max_cols;
  float* const pb = pw + max_cols;
  if (CLUSTER) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float u[8], v[8];
      floats_of(dw[r], u);
      floats_of(db[r], v);
      const int g = r * NTH + w.t;
      if (g < runs) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          pw[first + 8 * g + j] = u[j];
          pb[first + 8 * g + j] = v[j];
        }
      }
    }
    if (EDGE && edge >= 0) {
      pw[edge] = edw;
      pb[edge] = edb;
    }
    return;
  }
  // The CTA's walkers one after the other, through shared memory (the ring is empty now): written from the registers, every
  // store would touch a sector for four bytes of it.
  float* const acc = reinterpret_cast<float*>(ring);
  // Without edges the walkers of a warp have the same columns: they are added first, eight turns instead of up to 32.
  constexpr int TOGETHER = !EDGE && NTH < 32 ? 32 / NTH : 1;
#pragma unroll
  for (int o = NTH; o < NTH * TOGETHER; o <<= 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        F2 u, v;
        u.v = __shfl_xor_sync(0xffffffffu, dw[r][j].v, o);
        v.v = __shfl_xor_sync(0xffffffffu, db[r][j].v, o);
        dw[r][j] = add2(dw[r][j], u);
        db[r][j] = add2(db[r][j], v);
      }
    }
  }
  for (int k = 0; k < W::ROWS; k += TOGETHER) {
    __syncthreads();
    if (w.slot == k) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float u[8], v[8];
        floats_of(dw[r], u);
        floats_of(db[r], v);
        const int g = r * NTH + w.t, c = first + 8 * g;
        if (g < runs) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            acc[c + j] = k ? acc[c + j] + u[j] : u[j];
            acc[cols + c + j] = k ? acc[cols + c + j] + v[j] : v[j];
          }
        }
      }
      if (EDGE && edge >= 0) {
        acc[edge] = k ? acc[edge] + edw : edw;
        acc[cols + edge] = k ? acc[cols + edge] + edb : edb;
      }
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < cols; c += CTA) {
    pw[c] = acc[c];
    pb[c] = acc[cols + c];
  }
}

// --------------------------------------------------------------------------
// rows that lie on no runs
// --------------------------------------------------------------------------
// Any stride, any alignment: a thread owns every NTH-th column and loads elements one by one.  The generator's bits for a row are
// made block by block and passed through shared memory.
__host__ __device__ constexpr int bits_of(int cols) { return ((cols + 14) / 8 + 15) / 16 * 16; }
constexpr int ANY_NT = 256;

__device__ __forceinline__ void fill_bits(unsigned char* bits, int cols, u64 i0, const Drop& d) {
  const int nb = ((int)(i0 & 7) + cols + 7) >> 3;
  for (int b = threadIdx.x; b < nb; b += ANY_NT) bits[b] = (unsigned char)keep_bits((i0 >> 3) + b, d);
  __syncthreads();
}
__device__ __forceinline__ bool bit_at(const unsigned char* bits, int c, u64 i0) {
  const int i = c + (int)(i0 & 7);
  return (bits[i >> 3] >> (i & 7)) & 1;
}

// One CTA a row, which waits in shared memory.
template <typename T, typename P>
__global__ void __launch_bounds__(ANY_NT) k_norm_any(const __grid_constant__ adacgd_norm_args a, const __grid_constant__ Drop d) {
  extern __shared__ uint4 dyn[];
  __shared__ float sh[2][ANY_NT / 32];
  const long long row = blockIdx.x;
  const int cols = (int)a.cols;
  float* const srow = reinterpret_cast<float*>(dyn);
  unsigned char* const bits = reinterpret_cast<unsigned char*>(srow + (cols + 3) / 4 * 4);
  const u64 i0 = (u64)row * (u64)cols;
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* res = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  if (d.on) fill_bits(bits, cols, i0, d);
  float acc = 0.f;
#pragma unroll 4
  for (int c = threadIdx.x; c < cols; c += ANY_NT) {
    const float b = res ? to_f(res[c]) : 0.f;
    float v = to_f(x[c]);
    if (d.on) v = !bit_at(bits, c, i0) ? b : (res ? scaled(v, b, d) : v * d.scale);
    else if (res) v = b + v;
    srow[c] = v;
    acc += v;
  }
  const float mean = walker_sum<ANY_NT>(acc, sh[0]) / (float)cols;
  acc = 0.f;
  for (int c = threadIdx.x; c < cols; c += ANY_NT) acc = fmaf(srow[c] - mean, srow[c] - mean, acc);
  const float rstd = 1.f / sqrtf(walker_sum<ANY_NT>(acc, sh[1]) / (float)cols + a.eps);
  T* out = (T*)a.out + row * a.out_stride;
  T* sum = a.sum ? (T*)a.sum + row * a.sum_stride : nullptr;
  const P* w = (const P*)a.weight;
  const P* b = (const P*)a.bias;
#pragma unroll 4
  for (int c = threadIdx.x; c < cols; c += ANY_NT) {
    const float v = srow[c];
    if (sum) sum[c] = from_f<T>(v);
    out[c] = from_f<T>(fmaf((v - mean) * rstd, w ? to_f(w[c]) : 1.f, b ? to_f(b[c]) : 0.f));
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// One CTA a row, read twice.
template <typename T, typename P>
__global__ void __launch_bounds__(ANY_NT) k_norm_bwd_any(const __grid_constant__ adacgd_norm_backward_args a, const __grid_constant__ Drop d) {
  extern __shared__ uint4 dyn[];
  __shared__ float sh[2][ANY_NT / 32];
  const long long row = blockIdx.x;
  const int cols = (int)a.cols;
  unsigned char* const bits = reinterpret_cast<unsigned char*>(dyn);
  const u64 i0 = (u64)row * (u64)cols;
  const T* dy = (const T*)a.dout + row * a.dout_stride;
  const T* s = (const T*)a.s + row * a.s_stride;
  const T* ds = a.dsum ? (const T*)a.dsum + row * a.dsum_stride : nullptr;
  T* dx = (T*)a.dx + row * a.dx_stride;
  T* dr = a.dresidual ? (T*)a.dresidual + row * a.dresidual_stride : nullptr;
  const P* w = (const P*)a.weight;
  const float mean = a.mean[row], rstd = a.rstd[row];
  if (d.on) fill_bits(bits, cols, i0, d);
  float p = 0.f, q = 0.f;
#pragma unroll 4
  for (int c = threadIdx.x; c < cols; c += ANY_NT) {
    const float g = to_f(dy[c]) * (w ? to_f(w[c]) : 1.f);
    p += g;
    q = fmaf(g, (to_f(s[c]) - mean) * rstd, q);
  }
  p = walker_sum<ANY_NT>(p, sh[0]) / (float)cols;
  q = walker_sum<ANY_NT>(q, sh[1]) / (float)cols;
#pragma unroll 4
  for (int c = threadIdx.x; c < cols; c += ANY_NT) {
    float v = rstd * (fmaf(to_f(dy[c]), w ? to_f(w[c]) : 1.f, -p) - ((to_f(s[c]) - mean) * rstd) * q);
    if (ds) v += to_f(ds[c]);
    if (dr) dr[c] = from_f<T>(v);
    if (d.on) v = bit_at(bits, c, i0) ? v * d.scale : 0.f;
    dx[c] = from_f<T>(v);
  }
}
// Its partial weight gradients, before dx is written (it may be dout or s): a thread a column, a slice of rows a CTA row.
template <typename T>
__global__ void __launch_bounds__(ANY_NT) k_norm_dw_any(const __grid_constant__ adacgd_norm_backward_args a, float* __restrict__ part, long long max_cols) {
  const int c = blockIdx.x * ANY_NT + threadIdx.x;
  if (c >= a.cols) return;
  const long long lo = a.rows * blockIdx.y / gridDim.y, hi = a.rows * (blockIdx.y + 1) / gridDim.y;
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (long long r = lo; r < hi; ++r) {
    const float g = to_f(((const T*)a.dout)[r * a.dout_stride + c]);
    dw = fmaf(g, (to_f(((const T*)a.s)[r * a.s_stride + c]) - a.mean[r]) * a.rstd[r], dw);
    db += g;
  }
  part[(2ll * blockIdx.y) * max_cols + c] = dw;
  part[(2ll * blockIdx.y + 1) * max_cols + c] = db;
}

// Adds the CTAs' partial weight gradients: SUM_COLS columns a CTA, SUM_SLICES threads share a column's partials.  Few columns a CTA,
// so that the partials, which still lie in the cache, are fetched by many SMs at once.  In 64 bits and in a fixed order: the result
// repeats bit for bit.  One tenth of the time at 32768 x 8192, half of it where there are few rows.
constexpr int SUM_COLS = 8, SUM_SLICES = 64;
template <typename P>
__global__ void __launch_bounds__(SUM_COLS* SUM_SLICES) k_norm_dw_sum(const float* part, long long max_cols, int parts,
                                                                      int cols, P* __restrict__ dw, P* __restrict__ db) {
  __shared__ double sh[2][SUM_SLICES][SUM_COLS];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int x = threadIdx.x % SUM_COLS, s = threadIdx.x / SUM_COLS, c = blockIdx.x * SUM_COLS + x;
  double a = 0.0, b = 0.0;
  if (c < cols) {
#pragma unroll 4
    for (int k = s; k < parts; k += SUM_SLICES) {
      a += (double)part[2ll * k * max_cols + c];
      b += (double)part[(2ll * k + 1) * max_cols + c];
    }
  }
  sh[0][s][x] = a;
  sh[1][s][x] = b;
#pragma unroll
  for (int w = SUM_SLICES / 8; w >= 1; w /= 8) {      // eight neighbours at a time, in order
    __syncthreads();
    if (s < w) {
      a = b = 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        a += sh[0][s * 8 + k][x];
        b += sh[1][s * 8 + k][x];
      }
    }
    __syncthreads();
    if (s < w) {
      sh[0][s][x] = a;
      sh[1][s][x] = b;
    }
  }
  if (s || c >= cols) return;
  if (dw) dw[c] = from_f<P>((float)a);
  if (db) db[c] = from_f<P>((float)b);
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
template <typename T>
bool run_aligned(const void* p, long long stride, long long rows) {
  return !p || ((uintptr_t)p % (8 * sizeof(T)) == 0 && (rows == 1 || stride % 8 == 0));
}

template <typename T>
int dropout_t(adacgd_dropout_args a, cudaStream_t st) {
  if (a.x_stride == a.cols && a.out_stride == a.cols && (!a.residual || a.residual_stride == a.cols)) {
    a.cols *= a.rows;   // one long run
    a.rows = 1;
  }
  const long long blocks = (a.rows * a.cols + 7) / 8, per = DROP_NT * DROP_RUNS;
  const unsigned grid = (unsigned)((blocks + per - 1) / per);
  const bool vec = (a.rows == 1 || a.cols % 8 == 0) && run_aligned<T>(a.x, a.x_stride, a.rows) &&
                   run_aligned<T>(a.residual, a.residual_stride, a.rows) && run_aligned<T>(a.out, a.out_stride, a.rows);
  auto kern = vec ? k_dropout<T, true> : k_dropout<T, false>;
  kern<<<grid, DROP_NT, 0, st>>>((const T*)a.x, a.x_stride, (const T*)a.residual, a.residual_stride, (T*)a.out, a.out_stride,
                                 a.rows, a.cols, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

// Whether a call's matrices lie on runs: no gaps between rows, or aligned rows of a multiple of eight columns.
struct Runs {
  bool whole, flat;
  long long cols, rows;
  template <typename T> void look(const void* p, long long stride) {
    if (!p) return;
    flat = flat && (uintptr_t)p % (8 * sizeof(T)) == 0 && (stride == cols || rows == 1);
    whole = whole && run_aligned<T>(p, stride, rows);
  }
  bool good() const { return flat || (whole && cols % 8 == 0); }
};

template <typename T, typename P, int NTH, int R>
int norm_launch(const adacgd_norm_args& a, const Where& at) {
  constexpr int ROWS = Group<NTH>::ROWS;
  auto kern = a.cols % 8 ? k_norm<T, P, NTH, R, (NTH >= 16)> : k_norm<T, P, NTH, R, false>;      // edges take sixteen threads
  kern<<<(unsigned)((a.rows + ROWS - 1) / ROWS), Group<NTH>::CTA, 0, at.stream>>>(a, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, typename P>
int norm_t(const adacgd_norm_args& a, const Where& at) {
  Runs k = {true, true, a.cols, a.rows};
  k.look<T>(a.x, a.x_stride);
  k.look<T>(a.residual, a.residual_stride);
  k.look<T>(a.out, a.out_stride);
  k.look<T>(a.sum, a.sum_stride);
  const long long n = a.cols / 8;      // the most runs of a row
  if (!k.good()) {
    static std::atomic<int> table[TRAIN_DEVICES];
    const int smem = (int)((a.cols + 3) / 4 * 16) + (a.drop.p > 0.0 ? bits_of((int)a.cols) : 0);
    auto kern = k_norm_any<T, P>;
    if (resident_ctas(kern, table, at.device, ANY_NT, ADACGD_TRAIN_MAX_COLS * 4 + bits_of(ADACGD_TRAIN_MAX_COLS)) < 1) return -1;
    kern<<<(unsigned)a.rows, ANY_NT, smem, at.stream>>>(a, make_drop(a.drop));
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  }
  // Few rows: more threads a row, a shorter chain each.  us in a graph, 1 / 148 / 296 rows of bfloat16, so and as below: 1024 columns
  // 2.06 / 2.36 / 2.49 and 3.11 / 3.50 / 3.51; 4096 2.49 / 2.84 / 3.26 and 3.25 / 3.62 / 4.05.  8192 columns over 1024 threads gain
  // 0.13 us for one row and lose 1.8 for 296.
  if (a.rows <= 2 * at.sms && n > 32) {
    if (n <= 128) return norm_launch<T, P, 128, 1>(a, at);
    if (n <= 512) return norm_launch<T, P, 512, 1>(a, at);
  }
  // As few threads a row as its length in registers allows: the reductions cost every warp the same.  us for 2^27 elements with a
  // residual, bfloat16, p = 0 / p = 0.1, here and at twice the threads: 64 columns 160 / 181 and 185 / 220; 128 162 / 183, 185 / 222;
  // 256 161 / 183, 187 / 222; 4096 161 / 170, 177 / 193; 8192 164 / 181, 190 / 205; 16384 241 / 251, 249 / 251.  Four runs of binary32
  // take twice the registers: 8192 columns 316 (344 at 8185) against 312 (325) with two.
  const bool edge = a.cols % 8 != 0;                                         // takes sixteen threads
  if (n <= 8 && !edge) return norm_launch<T, P, 4, 2>(a, at);
  if (n <= 16 && !edge) return norm_launch<T, P, 8, 2>(a, at);
  if (n <= 32) return norm_launch<T, P, 16, 2>(a, at);
  if (n <= 64) return norm_launch<T, P, 32, 2>(a, at);
  if (n <= 128) return norm_launch<T, P, 32, 4>(a, at);
  if (n <= 256) return norm_launch<T, P, 128, 2>(a, at);
  if (n <= 512) return norm_launch<T, P, 128, 4>(a, at);
  if (sizeof(T) == 2 && n <= 1024) return norm_launch<T, P, 256, 4>(a, at);
  if (n <= 1024) return norm_launch<T, P, 512, 2>(a, at);
  if (n <= 2048) return norm_launch<T, P, 512, 4>(a, at);
  return norm_launch<T, P, 1024, 4>(a, at);
}

template <typename P>
int sum_parts(const TrainScratch& s, const adacgd_norm_backward_args& a, long long parts, const Where& at) {
  const int cols = (int)a.cols;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((cols + SUM_COLS - 1) / SUM_COLS));
  cfg.blockDim = dim3(SUM_COLS * SUM_SLICES);
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_norm_dw_sum<P>, (const float*)s.norm_part, s.max_cols, (int)parts, cols, (P*)a.dweight, (P*)a.dbias) == cudaSuccess
             ? 2
             : -1;
}

template <typename T, typename P, int NTH, int R, bool CLUSTER, bool EDGE, int ARRAYS>
int norm_bwd_arrays(const TrainScratch& s, const adacgd_norm_backward_args& a, int cluster, const Where& at) {
  typedef Walk<T, NTH, R, ARRAYS> W;
  static std::atomic<int> table[TRAIN_DEVICES];
  auto kern = k_norm_bwd<T, P, NTH, R, CLUSTER, EDGE, ARRAYS>;
  const int per_sm = resident_ctas(kern, table, at.device, W::CTA, W::SMEM);
  if (per_sm < 1) return -1;
  long long groups = (a.rows + W::ROWS - 1) / W::ROWS, most = (long long)per_sm * at.sms / cluster;
  if (most > NORM_PARTS) most = NORM_PARTS;
  if (groups > most) groups = most;
  const int need = MAX_PERIOD / W::ROWS > 1 ? MAX_PERIOD / W::ROWS : 1;
  if (EDGE) groups = groups < need ? need : groups / need * need;
  const bool grads = a.dweight || a.dbias;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * cluster));
  cfg.blockDim = dim3(W::CTA);
  cfg.dynamicSmemBytes = W::SMEM;
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CLUSTER ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, a, make_drop(a.drop), grads ? s.norm_part : (float*)nullptr, s.max_cols) != cudaSuccess) return -1;
  return grads ? sum_parts<P>(s, a, groups, at) : 1;
}

template <typename T, typename P, int NTH, int R, bool CLUSTER, bool EDGE>
int norm_bwd_launch(const TrainScratch& s, const adacgd_norm_backward_args& a, int cluster, const Where& at) {
  return a.dsum ? norm_bwd_arrays<T, P, NTH, R, CLUSTER, EDGE, 3>(s, a, cluster, at)
                : norm_bwd_arrays<T, P, NTH, R, CLUSTER, EDGE, 2>(s, a, cluster, at);
}

template <typename T, typename P, bool EDGE>
int norm_bwd_by_width(const TrainScratch& s, const adacgd_norm_backward_args& a, long long n, const Where& at) {
  // Up to 64 columns, us at 8 / 16 threads a row: bfloat16 512 rows 8.4 / 8.7, 16384 11.1 / 12.5, 131072 20.6 / 30.9; binary32 16384 rows 10.9 /
  // 12.5, 131072 23.1 / 28.3 and with dsum 31.1 / 32.1.  Edges take sixteen threads.
  if (!EDGE && n <= 8) return norm_bwd_launch<T, P, 8, 1, false, false>(s, a, 1, at);
  if (n <= 16) return norm_bwd_launch<T, P, 16, 1, false, EDGE>(s, a, 1, at);
  if (n <= 32) return norm_bwd_launch<T, P, 32, 1, false, EDGE>(s, a, 1, at);
  // One run a thread for binary32, of which an SM holds half as many rows, and where a walker gets few rows; else two, which share a
  // reduction.  us, one / two, with dsum: bfloat16 1024 columns, 512 rows 9.8 / 12.7, 4096 15.2 / 18.6, 8192 22.9 / 21.4, 65536 121 /
  // 98; 4096 columns, 512 rows 12.9 / 14.7, 4096 39 / 35, 16384 121 / 94; binary32 1024 columns, 512 rows 10.8 / 12.7, 16384 53 / 56.
  if (sizeof(T) == 4 || a.rows * a.cols <= 32768ll * at.sms) {
    if (n <= 64) return norm_bwd_launch<T, P, 64, 1, false, EDGE>(s, a, 1, at);
    if (n <= 128) return norm_bwd_launch<T, P, 128, 1, false, EDGE>(s, a, 1, at);
    if (n <= 256) return norm_bwd_launch<T, P, 256, 1, false, EDGE>(s, a, 1, at);
    if (n <= 512) return norm_bwd_launch<T, P, 512, 1, false, EDGE>(s, a, 1, at);
  } else {
    if (n <= 64) return norm_bwd_launch<T, P, 32, 2, false, EDGE>(s, a, 1, at);
    if (n <= 128) return norm_bwd_launch<T, P, 64, 2, false, EDGE>(s, a, 1, at);
    if (n <= 256) return norm_bwd_launch<T, P, 128, 2, false, EDGE>(s, a, 1, at);
    if (n <= 512) return norm_bwd_launch<T, P, 256, 2, false, EDGE>(s, a, 1, at);
  }
  if (n <= 1024) return norm_bwd_launch<T, P, 512, 2, false, EDGE>(s, a, 1, at);
  return norm_bwd_launch<T, P, 512, 2, true, EDGE>(s, a, (int)((n + 1023) / 1024), at);
}

template <typename T, typename P>
int norm_bwd_t(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& at) {
  Runs k = {true, true, a.cols, a.rows};
  k.look<T>(a.dout, a.dout_stride);
  k.look<T>(a.s, a.s_stride);
  k.look<T>(a.dsum, a.dsum_stride);
  k.look<T>(a.dx, a.dx_stride);
  k.look<T>(a.dresidual, a.dresidual_stride);
  const long long n = a.cols / 8;
  if (!k.good()) {
    int launched = 1;
    if (a.dweight || a.dbias) {
      const int tiles = (int)((a.cols + ANY_NT - 1) / ANY_NT);
      long long parts = 8ll * at.sms / tiles + 1;
      if (parts > NORM_PARTS) parts = NORM_PARTS;
      if (parts > a.rows) parts = a.rows;
      k_norm_dw_any<T><<<dim3(tiles, (unsigned)parts), ANY_NT, 0, at.stream>>>(a, s.norm_part, s.max_cols);
      if (sum_parts<P>(s, a, parts, at) < 0) return -1;
      launched = 3;
    }
    k_norm_bwd_any<T, P><<<(unsigned)a.rows, ANY_NT, a.drop.p > 0.0 ? bits_of((int)a.cols) : 0, at.stream>>>(a, make_drop(a.drop));
    return cudaGetLastError() == cudaSuccess ? launched : -1;
  }
  return a.cols % 8 ? norm_bwd_by_width<T, P, true>(s, a, n, at) : norm_bwd_by_width<T, P, false>(s, a, n, at);
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_dropout(const adacgd_dropout_args& a, const Where& at) { BY_TYPE(a.dtype, (dropout_t<T>(a, at.stream))) }

int launch_layer_norm(const adacgd_norm_args& a, const Where& at) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_t<T, float>(a, at)))
  BY_TYPE(a.dtype, (norm_t<T, T>(a, at)))
}

int launch_layer_norm_backward(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& at) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_bwd_t<T, float>(s, a, at)))
  BY_TYPE(a.dtype, (norm_bwd_t<T, T>(s, a, at)))
}

}  // namespace adacgd
