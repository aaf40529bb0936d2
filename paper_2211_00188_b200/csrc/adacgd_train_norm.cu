// Dropout and layer norm with the residual sum and dropout in front of it, forward and backward (adacgd_train.h).
//
// All three are bound by memory: a few operations an element against 4 to 20 bytes of traffic.  So every element is read
// once and written once, a row stays in registers between its statistics and its result, and what is left is to keep
// enough loads in flight.
//
// Two ways to spread a row over threads:
//   VEC   a thread owns runs of eight consecutive columns and moves them in 16-byte pieces.  Eight columns are also one
//         block of the dropout generator, so a run costs one call of it.  Needs 16-byte aligned rows (base, stride, weight)
//         and a multiple of eight columns.
//   else  a thread owns every NTH-th column, loaded one by one: a warp's 32 elements are consecutive, whatever the
//         alignment.  The generator's bits for the row are made once, block by block, and passed through shared memory.
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
// a row spread over NTH threads, E elements each
// --------------------------------------------------------------------------
template <int NTH> struct Shape {
  static constexpr int CTA = NTH < 128 ? 128 : NTH;   // a row of one warp shares its CTA with three others
  static constexpr int ROWS = CTA / NTH;
};

template <int NTH, bool VEC>
__device__ __forceinline__ int col_of(int e, int t) { return VEC ? ((e >> 3) * NTH + t) * 8 + (e & 7) : e * NTH + t; }

// The row's elements in 32 bits; columns at or past `cols` are 0.
template <typename T, int NTH, int E, bool VEC>
__device__ __forceinline__ void load_row(const T* row, int cols, int t, float (&o)[E]) {
  if (VEC) {
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
      const int c = (g * NTH + t) * 8;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
      if (c < cols) unpack(load_run(row + c), v);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[g * 8 + j] = v[j];
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = e * NTH + t;
      o[e] = c < cols ? to_f(row[c]) : 0.f;
    }
  }
}

template <typename T, int NTH, int E, bool VEC>
__device__ __forceinline__ void store_row(T* row, int cols, int t, const float (&v)[E]) {
  if (VEC) {
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
      const int c = (g * NTH + t) * 8;
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = v[g * 8 + j];
      if (c < cols) store_run(row + c, w);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = e * NTH + t;
      if (c < cols) row[c] = from_f<T>(v[e]);
    }
  }
}

// v[e] = dropout of v[e], or with BASE base[e] + dropout of v[e]; i0 = number of the element in the row's first column.  bits: the row's share of shared
// memory (one byte a block), filled by fill_bits before the last barrier.
template <int NTH, int E, bool VEC, bool BASE>
__device__ __forceinline__ void drop_row(float (&v)[E], const float (&base)[E], int cols, int t, u64 i0, const Drop& d,
                                         const unsigned char* bits) {
  if (VEC) {
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
      const int c = (g * NTH + t) * 8;
      if (c < cols) {
        const uint4 w = philox((i0 + c) >> 3, d);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[g * 8 + j] = !kept(w, j, d) ? (BASE ? base[g * 8 + j] : 0.f)
                                        : (BASE ? scaled(v[g * 8 + j], base[g * 8 + j], d) : v[g * 8 + j] * d.scale);
      }
    }
  } else {
    const int ph = (int)(i0 & 7);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = e * NTH + t;
      if (c < cols) v[e] = (bits[(c + ph) >> 3] >> ((c + ph) & 7)) & 1 ? (BASE ? scaled(v[e], base[e], d) : v[e] * d.scale) : (BASE ? base[e] : 0.f);
    }
  }
}
template <int NTH>
__device__ __forceinline__ void fill_bits(unsigned char* bits, int cols, int t, u64 i0, const Drop& d) {
  const int nb = ((int)(i0 & 7) + cols + 7) >> 3;
  for (int b = t; b < nb; b += NTH) bits[b] = (unsigned char)keep_bits((i0 >> 3) + b, d);
}
__host__ __device__ constexpr int bits_of(int cols) { return ((cols + 14) / 8 + 15) / 16 * 16; }

template <int NTH>
__device__ __forceinline__ void row_sync() {
  if (NTH == 32) __syncwarp();
  else __syncthreads();
}

// Sum over the row's threads, the same bits in each; `sh` must not be in use by an earlier sum.
template <int NTH>
__device__ __forceinline__ float row_sum(float v, float* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (NTH == 32) return v;
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NTH / 32; ++w) t += sh[w];
  return t;
}

// --------------------------------------------------------------------------
// layer norm
// --------------------------------------------------------------------------
// The mean first, then the squares about it: two sums over registers, no cancellation.
template <typename T, typename P, int NTH, int E, bool VEC>
__global__ void __launch_bounds__(Shape<NTH>::CTA) k_norm(adacgd_norm_args a, Drop d) {
  __shared__ float sh[2][32];
  extern __shared__ unsigned char dyn[];
  const int t = NTH == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const long long row = (long long)blockIdx.x * Shape<NTH>::ROWS + (NTH == 32 ? threadIdx.x >> 5 : 0);
  if (row >= a.rows) return;               // whole warps, and only where NTH == 32: no barrier follows then
  const int cols = (int)a.cols;
  const u64 i0 = (u64)row * (u64)cols;
  unsigned char* bits = dyn + (NTH == 32 ? (threadIdx.x >> 5) * bits_of(cols) : 0);
  float v[E], base[E];
  load_row<T, NTH, E, VEC>((const T*)a.x + row * a.x_stride, cols, t, v);
#pragma unroll
  for (int e = 0; e < E; ++e) base[e] = 0.f;
  if (a.residual) load_row<T, NTH, E, VEC>((const T*)a.residual + row * a.residual_stride, cols, t, base);
  if (d.on) {
    if (!VEC) {
      fill_bits<NTH>(bits, cols, t, i0, d);
      row_sync<NTH>();
    }
    if (a.residual) drop_row<NTH, E, VEC, true>(v, base, cols, t, i0, d, bits);
    else drop_row<NTH, E, VEC, false>(v, base, cols, t, i0, d, bits);
  } else if (a.residual) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = base[e] + v[e];
  }
  float acc = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc += v[e];
  const float mean = row_sum<NTH>(acc, sh[0]) / (float)cols;
  acc = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (col_of<NTH, VEC>(e, t) < cols) acc = fmaf(v[e] - mean, v[e] - mean, acc);
  const float rstd = 1.f / sqrtf(row_sum<NTH>(acc, sh[1]) / (float)cols + a.eps);
  if (a.sum) store_row<T, NTH, E, VEC>((T*)a.sum + row * a.sum_stride, cols, t, v);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (v[e] - mean) * rstd;
  if (a.weight) {
    load_row<P, NTH, E, VEC>((const P*)a.weight, cols, t, base);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= base[e];
  }
  if (a.bias) {
    load_row<P, NTH, E, VEC>((const P*)a.bias, cols, t, base);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += base[e];
  }
  store_row<T, NTH, E, VEC>((T*)a.out + row * a.out_stride, cols, t, v);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// --------------------------------------------------------------------------
// layer norm, backward
// --------------------------------------------------------------------------
// What a thread has loaded of one row of one matrix.
template <typename T, int E, bool VEC> struct Raw;
template <typename T, int E> struct Raw<T, E, true> {
  Run<T> r[E / 8];
  template <int NTH> __device__ __forceinline__ void load(const T* row, int cols, int t) {
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
      const int c = (g * NTH + t) * 8;
      if (c < cols) r[g] = load_run(row + c);
    }
  }
  __device__ __forceinline__ void get(int g, float (&o)[8]) const { unpack(r[g], o); }
};
template <typename T, int E> struct Raw<T, E, false> {
  T r[E];
  template <int NTH> __device__ __forceinline__ void load(const T* row, int cols, int t) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = e * NTH + t;
      if (c < cols) r[e] = row[c];
    }
  }
  __device__ __forceinline__ void get(int g, float (&o)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = to_f(r[g * 8 + j]);
  }
};

// A CTA walks rows and keeps the weight gradients of its columns in registers: dout and s are read once for both results.
// The next row's loads are issued as soon as the current row has been unpacked, so they are under way while the row's two
// sums are formed and its gradient is written.  Rows wider than NTH * E are cut into as many column parts as the cluster
// has CTAs; the two sums then meet in distributed shared memory.
//   ds = rstd g + dsum - rstd mean(g) - h rstd mean(g h)
template <typename T, typename P, int NTH, int E, bool VEC, bool CLUSTER>
__global__ void __launch_bounds__(Shape<NTH>::CTA) k_norm_bwd(adacgd_norm_backward_args a, Drop d, float* __restrict__ part,
                                                              long long max_cols) {
  constexpr int CTA = Shape<NTH>::CTA, ROWS = Shape<NTH>::ROWS;
  __shared__ float sh[2][2][32];
  __shared__ float2 xch[2][8];
  extern __shared__ unsigned char dyn[];
  const int t = NTH == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const int warp = threadIdx.x >> 5;
  int nparts = 1, rank = 0;
  if (CLUSTER) {
    nparts = (int)cg::this_cluster().num_blocks();
    rank = (int)cg::this_cluster().block_rank();
  }
  if (CLUSTER) cg::this_cluster().sync();   // every CTA has started before any writes into another's shared memory
  const int all = (int)a.cols;
  const int span = CLUSTER ? ((all + nparts - 1) / nparts + 7) / 8 * 8 : all;   // columns of a part, a multiple of eight
  const int c0 = rank * span, cols = min(span, all - c0) < 0 ? 0 : min(span, all - c0);
  const long long group = blockIdx.x / nparts, step = (long long)(gridDim.x / nparts) * ROWS;
  const bool grads = part != nullptr;
  float dw[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
  unsigned char* bits = dyn + (NTH == 32 ? warp * bits_of(cols) : 0);

  Raw<T, E, VEC> rdy, rs, rds;
  float mean = 0.f, rstd = 0.f;
  long long row = group * ROWS + (NTH == 32 ? warp : 0);
  const T* dout = (const T*)a.dout + c0;
  const T* s = (const T*)a.s + c0;
  const T* dsum = a.dsum ? (const T*)a.dsum + c0 : nullptr;
  const P* weight = a.weight ? (const P*)a.weight + c0 : nullptr;
  if (row < a.rows) {
    rdy.template load<NTH>(dout + row * a.dout_stride, cols, t);
    rs.template load<NTH>(s + row * a.s_stride, cols, t);
    if (dsum) rds.template load<NTH>(dsum + row * a.dsum_stride, cols, t);
    mean = a.mean[row];
    rstd = a.rstd[row];
  }
  int parity = 0;
  for (; row < a.rows; row += step, parity ^= 1) {
    float v[E], h[E], p = 0.f, q = 0.f;
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
      float x[8], y[8], w[8], z[8];
      rdy.get(g, y);
      rs.get(g, x);
      if (dsum) rds.get(g, z);
      if (VEC) {
        const int c = (g * NTH + t) * 8;
        if (weight && c < cols) unpack(load_run(weight + c), w);
      } else if (weight) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = (g * 8 + j) * NTH + t;
          if (c < cols) w[j] = to_f(weight[c]);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = g * 8 + j;
        const bool in = col_of<NTH, VEC>(e, t) < cols;
        const float hh = in ? (x[j] - mean) * rstd : 0.f, dy = in ? y[j] : 0.f;
        const float gw = weight && in ? dy * w[j] : dy;
        p += gw;
        q = fmaf(gw, hh, q);
        dw[e] = fmaf(dy, hh, dw[e]);
        db[e] += dy;
        h[e] = hh;
        v[e] = dsum && in ? fmaf(rstd, gw, z[j]) : rstd * gw;
      }
    }
    const float rs_now = rstd;
    const long long next = row + step;
    if (next < a.rows) {
      rdy.template load<NTH>(dout + next * a.dout_stride, cols, t);
      rs.template load<NTH>(s + next * a.s_stride, cols, t);
      if (dsum) rds.template load<NTH>(dsum + next * a.dsum_stride, cols, t);
      mean = a.mean[next];
      rstd = a.rstd[next];
    }
    const u64 i0 = (u64)row * (u64)all + (u64)c0;
    if (!VEC && d.on) fill_bits<NTH>(bits, cols, t, i0, d);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      p += __shfl_xor_sync(0xffffffffu, p, o);
      q += __shfl_xor_sync(0xffffffffu, q, o);
    }
    if (NTH > 32) {
      if ((threadIdx.x & 31) == 0) {
        sh[parity][0][warp] = p;
        sh[parity][1][warp] = q;
      }
      __syncthreads();
      p = q = 0.f;
#pragma unroll
      for (int w = 0; w < NTH / 32; ++w) {
        p += sh[parity][0][w];
        q += sh[parity][1][w];
      }
      if (CLUSTER) {
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x < nparts) *cl.map_shared_rank(&xch[parity][rank], threadIdx.x) = make_float2(p, q);
        cl.sync();     // the slots of this parity are written again only behind the next row's barrier
        p = q = 0.f;
        for (int k = 0; k < nparts; ++k) {
          p += xch[parity][k].x;
          q += xch[parity][k].y;
        }
      }
    } else {
      __syncwarp();
    }
    p = rs_now * (p / (float)all);
    q = rs_now * (q / (float)all);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = fmaf(-h[e], q, v[e] - p);
    if (a.dresidual) store_row<T, NTH, E, VEC>((T*)a.dresidual + row * a.dresidual_stride + c0, cols, t, v);
    if (d.on) {
      drop_row<NTH, E, VEC, false>(v, v, cols, t, i0, d, bits);
      if (!VEC) row_sync<NTH>();   // the bits are written again for the next row
    }
    store_row<T, NTH, E, VEC>((T*)a.dx + row * a.dx_stride + c0, cols, t, v);
  }
  if (CLUSTER) cg::this_cluster().sync();   // no CTA leaves while another may still write into its shared memory
  if (!grads) return;
  float* pw = part + 2ll * group * max_cols + c0;
  float* pb = pw + max_cols;
  if (ROWS == 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = col_of<NTH, VEC>(e, t);
      if (c < cols) {
        pw[c] = dw[e];
        pb[c] = db[e];
      }
    }
  } else {   // the four warps' sums, in warp order
    __shared__ float acc[ROWS == 1 ? 1 : 2][ROWS == 1 ? 1 : NTH * E];
    for (int w = 0; w < ROWS; ++w) {
      if (warp == w) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int i = e * 32 + t;
          acc[0][i] = w ? acc[0][i] + dw[e] : dw[e];
          acc[1][i] = w ? acc[1][i] + db[e] : db[e];
        }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < NTH * E; i += CTA) {
      const int c = col_of<NTH, VEC>(i / 32, i & 31);
      if (c < cols) {
        pw[c] = acc[0][i];
        pb[c] = acc[1][i];
      }
    }
  }
}

// Adds the CTAs' partial weight gradients: a column a thread of the x dimension, SLICES threads share its partials.
constexpr int SUM_COLS = 32, SUM_SLICES = 16;
template <typename P>
__global__ void __launch_bounds__(SUM_COLS* SUM_SLICES) k_norm_dw_sum(const float* __restrict__ part, long long max_cols, int parts,
                                                                      int cols, P* __restrict__ dw, P* __restrict__ db) {
  __shared__ double sh[2][SUM_SLICES][SUM_COLS];
  const int c = blockIdx.x * SUM_COLS + threadIdx.x, s = threadIdx.y;
  double a = 0.0, b = 0.0;
  if (c < cols) {
#pragma unroll 4
    for (int k = s; k < parts; k += SUM_SLICES) {
      a += (double)part[2ll * k * max_cols + c];
      b += (double)part[(2ll * k + 1) * max_cols + c];
    }
  }
  sh[0][s][threadIdx.x] = a;
  sh[1][s][threadIdx.x] = b;
  __syncthreads();
  if (s || c >= cols) return;
  a = b = 0.0;
#pragma unroll
  for (int k = 0; k < SUM_SLICES; ++k) {
    a += sh[0][k][threadIdx.x];
    b += sh[1][k][threadIdx.x];
  }
  if (dw) dw[c] = from_f<P>((float)a);
  if (db) db[c] = from_f<P>((float)b);
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
template <typename T>
bool run_aligned(const void* p, long long stride, long long rows) {
  return !p || (((uintptr_t)p & 15) == 0 && (rows == 1 || (stride * (long long)sizeof(T)) % 16 == 0));
}
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

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

template <typename T, typename P, int NTH, int E, bool VEC>
int norm_launch(const adacgd_norm_args& a, cudaStream_t st) {
  constexpr int R = Shape<NTH>::ROWS;
  const int smem = VEC || a.drop.p == 0.0 ? 0 : R * bits_of((int)a.cols);
  k_norm<T, P, NTH, E, VEC><<<(unsigned)((a.rows + R - 1) / R), Shape<NTH>::CTA, smem, st>>>(a, make_drop(a.drop));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, typename P, bool VEC>
int norm_by_width(const adacgd_norm_args& a, int sms, cudaStream_t st) {
  const long long c = a.cols;
  if (a.rows <= 2 * sms && c > 256) {   // few rows: more threads a row, a shorter chain each
    if (c <= 1024) return norm_launch<T, P, 128, 8, VEC>(a, st);
    if (c <= 4096) return norm_launch<T, P, 512, 8, VEC>(a, st);
    if (c <= 8192) return norm_launch<T, P, 1024, 8, VEC>(a, st);
  }
  if (c <= 256) return norm_launch<T, P, 32, 8, VEC>(a, st);
  if (c <= 1024) return norm_launch<T, P, 32, 32, VEC>(a, st);
  if (c <= 2048) return norm_launch<T, P, 128, 16, VEC>(a, st);
  if (c <= 4096) return norm_launch<T, P, 256, 16, VEC>(a, st);
  if (c <= 8192) return norm_launch<T, P, 512, 16, VEC>(a, st);
  if (c <= 16384) return norm_launch<T, P, 1024, 16, VEC>(a, st);
  return norm_launch<T, P, 1024, 32, VEC>(a, st);
}

template <typename T, typename P>
int norm_t(const adacgd_norm_args& a, int sms, cudaStream_t st) {
  const bool vec = a.cols % 8 == 0 && run_aligned<T>(a.x, a.x_stride, a.rows) && run_aligned<T>(a.residual, a.residual_stride, a.rows) &&
                   run_aligned<T>(a.out, a.out_stride, a.rows) && run_aligned<T>(a.sum, a.sum_stride, a.rows) &&
                   aligned16(a.weight) && aligned16(a.bias);
  return vec ? norm_by_width<T, P, true>(a, sms, st) : norm_by_width<T, P, false>(a, sms, st);
}

template <typename T, typename P, int NTH, int E, bool VEC, bool CLUSTER>
int norm_bwd_launch(const TrainScratch& s, const adacgd_norm_backward_args& a, int cluster, const Where& at_, cudaStream_t st) {
  constexpr int R = Shape<NTH>::ROWS, CTA = Shape<NTH>::CTA;
  auto kern = k_norm_bwd<T, P, NTH, E, VEC, CLUSTER>;
  const int span = CLUSTER ? ((int)a.cols + cluster - 1) / cluster + 8 : (int)a.cols;
  const int smem = VEC || a.drop.p == 0.0 ? 0 : R * bits_of(span);
  static std::atomic<int> table[TRAIN_DEVICES];
  const int per_sm = resident_ctas(kern, table, at_.device, CTA, VEC ? 0 : R * bits_of(NTH * E));
  if (per_sm < 1) return -1;
  long long groups = (long long)at_.sms * per_sm / cluster;
  if (groups > NORM_PARTS) groups = NORM_PARTS;
  if (groups > (a.rows + R - 1) / R) groups = (a.rows + R - 1) / R;
  const bool grads = a.dweight || a.dbias;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * cluster));
  cfg.blockDim = dim3(CTA);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = CLUSTER ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, a, make_drop(a.drop), grads ? s.norm_part : (float*)nullptr, s.max_cols) != cudaSuccess) return -1;
  if (!grads) return 1;
  const int cols = (int)a.cols;
  k_norm_dw_sum<P><<<(cols + SUM_COLS - 1) / SUM_COLS, dim3(SUM_COLS, SUM_SLICES), 0, st>>>(s.norm_part, s.max_cols, (int)groups, cols,
                                                                                       (P*)a.dweight, (P*)a.dbias);
  return cudaGetLastError() == cudaSuccess ? 2 : -1;
}

template <typename T, typename P, bool VEC>
int norm_bwd_by_width(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& sms, cudaStream_t st) {
  const long long c = a.cols;
  if (c <= 256) return norm_bwd_launch<T, P, 32, 8, VEC, false>(s, a, 1, sms, st);
  if (c <= 1024) return norm_bwd_launch<T, P, 128, 8, VEC, false>(s, a, 1, sms, st);
  if (c <= 2048) return norm_bwd_launch<T, P, 128, 16, VEC, false>(s, a, 1, sms, st);
  if (c <= 4096) return norm_bwd_launch<T, P, 256, 16, VEC, false>(s, a, 1, sms, st);
  if (c <= 8192) return norm_bwd_launch<T, P, 512, 16, VEC, false>(s, a, 1, sms, st);
  return norm_bwd_launch<T, P, 512, 16, VEC, true>(s, a, c <= 16384 ? 2 : 4, sms, st);
}

template <typename T, typename P>
int norm_bwd_t(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& sms, cudaStream_t st) {
  const bool vec = a.cols % 8 == 0 && run_aligned<T>(a.dout, a.dout_stride, a.rows) && run_aligned<T>(a.s, a.s_stride, a.rows) &&
                   run_aligned<T>(a.dsum, a.dsum_stride, a.rows) && run_aligned<T>(a.dx, a.dx_stride, a.rows) &&
                   run_aligned<T>(a.dresidual, a.dresidual_stride, a.rows) && aligned16(a.weight);
  return vec ? norm_bwd_by_width<T, P, true>(s, a, sms, st) : norm_bwd_by_width<T, P, false>(s, a, sms, st);
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
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_t<T, float>(a, at.sms, at.stream)))
  BY_TYPE(a.dtype, (norm_t<T, T>(a, at.sms, at.stream)))
}

int launch_layer_norm_backward(const TrainScratch& s, const adacgd_norm_backward_args& a, const Where& at) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_bwd_t<T, float>(s, a, at, at.stream)))
  BY_TYPE(a.dtype, (norm_bwd_t<T, T>(s, a, at, at.stream)))
}

}  // namespace adacgd
