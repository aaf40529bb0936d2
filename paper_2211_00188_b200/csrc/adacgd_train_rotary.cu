// Norm and rotation of queries and keys, and its backward pass (adacgd_train.h).  Every element is read once and written once.  Heads of a multiple of
// 16 elements are bound by memory; the kernels for other lengths by a token's chain of latencies: position, angles, tables, barrier, heads.
// A head is held by the lanes of a part of a warp, eight elements each, so its mean of squares is a few
// shuffles; the cosines and sines of a token are made once (in binary64: position times frequency, reduced to a turn) and used by all its heads.
#include "adacgd_train.cuh"

namespace adacgd {
namespace {

__device__ __forceinline__ long long position_at(const adacgd_qk_norm_args& a, long long t) {
  return a.position_bytes == 8 ? reinterpret_cast<const long long*>(a.positions)[t] : (long long)reinterpret_cast<const int32_t*>(a.positions)[t];
}

// Cosine and sine of position * freq.  Position times frequency and that in turns are each rounded to binary64, as 1 / (2 pi) is; the reduction is
// exact: the angle is off by 2^-51 of itself at most, 5e-9 rad at ten million rad.  Rounding what is left of the turn to binary32 adds up to 2^-26 of a
// turn, 9.4e-8 rad, at any position.
__device__ __forceinline__ void turn(long long position, float freq, float* c, float* s) {
  const double turns = (double)position * (double)freq * 0.15915494309189535;   // 1 / (2 pi)
  sincospif(2.f * (float)(turns - rint(turns)), s, c);
}

// Tables of a token: for each element of a head the cosine, and the sine with the sign it has for that element (0 behind the rotated
// ones, whose cosine is 1).
__device__ __forceinline__ void fill_turns(const adacgd_qk_norm_args& a, long long t, int i, float* cs, float* sn, bool back) {
  float c, s;
  turn(position_at(a, t), a.freq[i], &c, &s);
  if (back) s = -s;
  const int p = a.interleaved ? 2 * i : i, q = a.interleaved ? 2 * i + 1 : a.pairs + i;
  cs[p] = cs[q] = c;
  sn[p] = -s;
  sn[q] = s;
}
// The other element of e's pair; e < 2 pairs.
__device__ __forceinline__ int partner(const adacgd_qk_norm_args& a, int e) {
  if (a.interleaved) return e ^ 1;
  return e < a.pairs ? e + a.pairs : e - a.pairs;
}

template <typename P> __device__ __forceinline__ float param(const void* w, int e) { return w ? to_f(((const P*)w)[e]) : 1.f; }

// Where head h of token t lies; heads behind the queries' are the keys'.
__device__ __forceinline__ long long place(long long stride, long long t, int h, int dim) { return t * stride + (long long)h * dim; }

// --------------------------------------------------------------------------
// heads of whole aligned runs
// --------------------------------------------------------------------------
constexpr int ROT_CTA = 256;
constexpr int ROT_MAX_TOKENS = 8;

// How the partner of a pair is reached: NEAR within the lane (neighbours, whole heads), PART the same of a front of the head or none of it, LANE in
// another lane at the same place, ROW through shared memory (halves whose distance is no whole number of runs).  Behind the rotated front a
// partner counts as 0, so that an infinity there stays where it is: its product with a sine of 0 would be NaN.  (PART for whole heads too took 79 registers
// instead of 64, 51.5 instead of 45.4 us for 16384 x 16 heads of 72.)
enum Reach { NEAR, LANE, ROW, PART };

// The lane's eight elements turned.  cs, sn: the lane's entries of the token's tables.
template <int LPH, int REACH>
__device__ __forceinline__ void rotate(const adacgd_qk_norm_args& a, const float* cs, const float* sn, int e0, float* row, float (&x)[8]) {
  __align__(16) float c[8], s[8], y[8];
#pragma unroll
  for (int j = 0; j < 8; j += 4) {
    *reinterpret_cast<float4*>(c + j) = *reinterpret_cast<const float4*>(cs + e0 + j);
    *reinterpret_cast<float4*>(s + j) = *reinterpret_cast<const float4*>(sn + e0 + j);
  }
  if (REACH == NEAR || REACH == PART) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = REACH == NEAR || e0 + j < 2 * a.pairs ? x[j ^ 1] : 0.f;
  } else if (REACH == LANE) {
    const int d = a.pairs / 8, me = e0 / 8;
    const int from = me < d ? me + d : (me < 2 * d ? me - d : me);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      y[j] = __shfl_sync(0xffffffffu, x[j], from, LPH);
      if (me >= 2 * d) y[j] = 0.f;
    }
  } else {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4*>(row + e0 + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
    __syncwarp();
    if (a.pairs % 4 == 0) {                           // four elements have their partners side by side
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<float4*>(y + j) = e0 + j < 2 * a.pairs ? *reinterpret_cast<const float4*>(row + partner(a, e0 + j)) : make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = e0 + j < 2 * a.pairs ? row[partner(a, e0 + j)] : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = fmaf(y[j], s[j], x[j] * c[j]);
}

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int LPH> struct HeadSmem {          // shared memory of a CTA, in floats
  static constexpr int DIM = LPH * 8, SLOTS = ROT_CTA / LPH;
  static constexpr int TURNS = 2 * ROT_MAX_TOKENS * DIM, WEIGHTS = 2 * DIM, ROWS = SLOTS * DIM;
};

// A CTA takes `each` tokens (of all heads, or with grid.y of a part of them): their tables, then their heads, LPH lanes a head and BATCH heads in
// flight.
template <typename T, typename P, int LPH, int REACH, int BATCH>
__global__ void __launch_bounds__(ROT_CTA) k_qk_norm(adacgd_qk_norm_args a, int each) {
  typedef HeadSmem<LPH> S;
  __shared__ __align__(16) float turns[S::TURNS], weights[S::WEIGHTS], rows[REACH == ROW ? S::ROWS : 1];
  const int dim = a.head_dim, lane = threadIdx.x % LPH, slot = threadIdx.x / LPH, e0 = lane * 8;
  const long long t0 = (long long)blockIdx.x * each;
  const int tokens = (int)min((long long)each, a.tokens - t0);
  const int heads = (int)(a.heads + a.key_heads), items = tokens * heads;
  const int per = (items + gridDim.y - 1) / gridDim.y, first = blockIdx.y * per, last = min(items, first + per);
  const bool in = e0 < dim;
  Run<T> x[BATCH];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * S::SLOTS + slot;
      if (i < last && in) {
        const int t = i / heads, h = i - t * heads;
        x[b] = h < a.heads ? load_run((const T*)a.q + place(a.q_stride, t0 + t, h, dim) + e0)
                           : load_run((const T*)a.k + place(a.k_stride, t0 + t, h - (int)a.heads, dim) + e0);
      }
    }
  };
  fetch(first);
  for (int i = threadIdx.x; i < S::DIM; i += ROT_CTA) {
    weights[i] = i < dim ? param<P>(a.q_weight, i) : 0.f;
    weights[S::DIM + i] = i < dim ? param<P>(a.k_weight, i) : 0.f;
  }
  const int rest = S::DIM - 2 * a.pairs;
  for (int i = threadIdx.x; i < tokens * rest; i += ROT_CTA) {
    float* const c = turns + (i / rest) * 2 * S::DIM + 2 * a.pairs + i % rest;
    c[0] = 1.f;
    c[S::DIM] = 0.f;
  }
  for (int i = threadIdx.x; i < tokens * a.pairs; i += ROT_CTA) {
    const int t = i / a.pairs;
    fill_turns(a, t0 + t, i - t * a.pairs, turns + t * 2 * S::DIM, turns + t * 2 * S::DIM + S::DIM, false);
  }
  __syncthreads();
  const float inv = 1.f / (float)dim;
  for (int i0 = first; i0 < last; i0 += BATCH * S::SLOTS) {
    Run<T> now[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) now[b] = x[b];
    fetch(i0 + BATCH * S::SLOTS);
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * S::SLOTS + slot;
      const bool live = i < last;
      const int t = live ? i / heads : 0, h = live ? i - t * heads : 0;
      float v[8];
      if (live && in) {
        unpack(now[b], v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
      }
      float q = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) q = fmaf(v[j], v[j], q);
      const float r = rsqrtf(fmaf(head_sum<LPH>(q), inv, a.eps));
      const float* const w = weights + (h < a.heads ? 0 : S::DIM) + e0;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * r * w[j];
      const float* const cs = turns + t * 2 * S::DIM;
      rotate<LPH, REACH>(a, cs, cs + S::DIM, e0, rows + (REACH == ROW ? slot * S::DIM : 0), v);
      if (live && in) {
        T* const out = h < a.heads ? (T*)a.q_out + place(a.q_out_stride, t0 + t, h, dim)
                                   : (T*)a.k_out + place(a.k_out_stride, t0 + t, h - (int)a.heads, dim);
        store_run(out + e0, v);
      }
    }
  }
}

// Backward: persistent CTAs, the weights' gradients in registers until the end; the CTA's heads are then added through shared memory.
template <typename T, typename P, int LPH, int REACH, int BATCH>
__global__ void __launch_bounds__(ROT_CTA) k_qk_norm_bwd(adacgd_qk_norm_backward_args g, int each, float* part, long long part_stride) {
  typedef HeadSmem<LPH> S;
  const adacgd_qk_norm_args& a = g.f;
  __shared__ __align__(16) float turns[S::TURNS], weights[S::WEIGHTS], rows[S::ROWS];
  const int dim = a.head_dim, lane = threadIdx.x % LPH, slot = threadIdx.x / LPH, e0 = lane * 8;
  const int heads = (int)(a.heads + a.key_heads);
  const bool in = e0 < dim;
  for (int i = threadIdx.x; i < S::DIM; i += ROT_CTA) {
    weights[i] = i < dim ? param<P>(a.q_weight, i) : 0.f;
    weights[S::DIM + i] = i < dim ? param<P>(a.k_weight, i) : 0.f;
  }
  float dwq[8], dwk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) dwq[j] = dwk[j] = 0.f;
  const float inv = 1.f / (float)dim;
  for (long long t0 = (long long)blockIdx.x * each; t0 < a.tokens; t0 += (long long)gridDim.x * each) {
    const int tokens = (int)min((long long)each, a.tokens - t0), items = tokens * heads;
    Run<T> x[BATCH], y[BATCH];
    auto fetch = [&](int i0) {
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int i = i0 + b * S::SLOTS + slot;
        if (i < items && in) {
          const int t = i / heads, h = i - t * heads;
          if (h < a.heads) {
            x[b] = load_run((const T*)a.q + place(a.q_stride, t0 + t, h, dim) + e0);
            y[b] = load_run((const T*)a.q_out + place(a.q_out_stride, t0 + t, h, dim) + e0);
          } else {
            x[b] = load_run((const T*)a.k + place(a.k_stride, t0 + t, h - (int)a.heads, dim) + e0);
            y[b] = load_run((const T*)a.k_out + place(a.k_out_stride, t0 + t, h - (int)a.heads, dim) + e0);
          }
        }
      }
    };
    fetch(0);
    __syncthreads();       // the tables of the tokens before are not needed any more
    const int rest = S::DIM - 2 * a.pairs;
    for (int i = threadIdx.x; i < tokens * rest; i += ROT_CTA) {
      float* const c = turns + (i / rest) * 2 * S::DIM + 2 * a.pairs + i % rest;
      c[0] = 1.f;
      c[S::DIM] = 0.f;
    }
    for (int i = threadIdx.x; i < tokens * a.pairs; i += ROT_CTA) {
      const int t = i / a.pairs;
      fill_turns(a, t0 + t, i - t * a.pairs, turns + t * 2 * S::DIM, turns + t * 2 * S::DIM + S::DIM, true);
    }
    __syncthreads();
    for (int i0 = 0; i0 < items; i0 += BATCH * S::SLOTS) {
      Run<T> nx[BATCH], ny[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        nx[b] = x[b];
        ny[b] = y[b];
      }
      fetch(i0 + BATCH * S::SLOTS);
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int i = i0 + b * S::SLOTS + slot;
        const bool live = i < items;
        const int t = live ? i / heads : 0, h = live ? i - t * heads : 0;
        float v[8], d[8];
        if (live && in) {
          unpack(nx[b], v);
          unpack(ny[b], d);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = d[j] = 0.f;
        }
        const float* const cs = turns + t * 2 * S::DIM;
        rotate<LPH, REACH>(a, cs, cs + S::DIM, e0, rows + (REACH == ROW ? slot * S::DIM : 0), d);
        const bool query = h < a.heads;
        const float* const w = weights + (query ? 0 : S::DIM) + e0;
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(v[j], v[j], q);
        const float r = rsqrtf(fmaf(head_sum<LPH>(q), inv, a.eps));
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] *= r;                                     // x r
          const float dw = live ? d[j] * v[j] : 0.f;
          if (query) dwq[j] += dw; else dwk[j] += dw;
          d[j] *= w[j];                                  // g
          dot = fmaf(d[j], v[j], dot);
        }
        const float m = head_sum<LPH>(dot) * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = r * fmaf(-m, v[j], d[j]);
        if (live && in) {
          T* const out = query ? (T*)g.dq + place(g.dq_stride, t0 + t, h, dim) : (T*)g.dk + place(g.dk_stride, t0 + t, h - (int)a.heads, dim);
          store_run(out + e0, d);
        }
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) rows[slot * S::DIM + e0 + j] = k ? dwk[j] : dwq[j];
    __syncthreads();
    for (int e = threadIdx.x; e < dim; e += ROT_CTA) {
      float sum = 0.f;
      for (int i = 0; i < S::SLOTS; ++i) sum += rows[i * S::DIM + e];
      part[(2ll * blockIdx.x + k) * part_stride + e] = sum;
    }
  }
}

// --------------------------------------------------------------------------
// heads of two runs a lane
// --------------------------------------------------------------------------
// Where a head is a multiple of 16 long, a lane takes run l and the run half a head further: with the usual rotation, of whole
// heads in halves, both elements of a pair are its own, and so they are with neighbours.  A warp takes a token, or a part of its heads where
// there are few tokens, makes the token's cosines and sines once and keeps its lanes' in registers, as it does the weights.
constexpr int TWO_CTA = 128, TWO_WARPS = TWO_CTA / 32, MAX_PAIRS = 128;

// Cosines and sines of the lane's pairs, packed in twos.  HALVES: pair 8 l + j couples the runs' j-th elements.  NEIGHBOURS: pair 4 l + i is
// elements 2 i and 2 i + 1 of the first run, and those of the second follow.  FRONT: halves of at most the head's first half, by whole
// runs: pair 8 (l mod pairs / 8) + j is the first run's j-th element here and pairs / 8 lanes further; the sine has the element's sign.  PARTLY:
// neighbours in a front of the head.  NONE: no pairs.  (One kernel for the last two and NEIGHBOURS: 131 instead of 127 us for 32768 x 40 heads of 128.)
enum Turn { HALVES, NEIGHBOURS, FRONT, PARTLY, NONE };
template <int TURN>
__device__ __forceinline__ void lane_turns(const adacgd_qk_norm_args& a, long long t, int l, bool in, float* table, bool back, F2 (&c)[4], F2 (&s)[4]) {
  if (TURN == NONE) return;
  float* const sines = table + MAX_PAIRS;
  __syncwarp();
  const long long position = position_at(a, t);
  for (int i = threadIdx.x & 31; i < a.head_dim / 2; i += 32) {
    float x = 1.f, y = 0.f;
    if (i < a.pairs) turn(position, a.freq[i], &x, &y);
    table[i] = x;
    sines[i] = back ? -y : y;
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int d = a.pairs / 8;
    const int i = TURN == HALVES ? 8 * l + 2 * j
                : TURN == FRONT  ? 8 * (l < d ? l : l - d) + 2 * j
                                 : (j < 2 ? 4 * l + 2 * j : 4 * (l + a.head_dim / 16) + 2 * (j - 2));
    const bool has = in && (TURN != FRONT || l < 2 * d);
    c[j] = has ? *reinterpret_cast<const F2*>(table + i) : f2(1.f, 1.f);
    s[j] = has ? *reinterpret_cast<const F2*>(sines + i) : f2(0.f, 0.f);
    if (TURN == FRONT && l < d) s[j].v ^= 0x8000000080000000ull;
  }
}
__device__ __forceinline__ F2 minus(F2 a) {
  F2 r;
  r.v = a.v ^ 0x8000000080000000ull;
  return r;
}
// Turns the lane's sixteen elements, of a head of `dim`: four packed pairs a run.  See Reach for what lies behind the rotated front.
template <int TURN, int LPH> __device__ __forceinline__ void turn_two(F2 (&x)[8], const F2 (&c)[4], const F2 (&s)[4], int l, int pairs, int dim) {
  if (TURN == NONE) return;
  if (TURN == FRONT) {
    const int d = pairs / 8;
    const int from = l < d ? l + d : (l < 2 * d ? l - d : l);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      F2 y;
      y.v = __shfl_sync(0xffffffffu, x[j].v, from, LPH);
      if (l >= 2 * d) y.v = 0;
      x[j] = fma2(y, s[j], mul2(x[j], c[j]));
    }
  } else if (TURN == HALVES) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const F2 a = x[j], b = x[4 + j];
      x[j] = fma2(a, c[j], mul2(b, minus(s[j])));
      x[4 + j] = fma2(b, c[j], mul2(a, s[j]));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {                     // element pair j: its turn is half of c[j / 2]
      float a, b, cx, cy, sx, sy;
      split(x[j], a, b);
      split(c[j / 2], cx, cy);
      split(s[j / 2], sx, sy);
      const float u = j & 1 ? cy : cx, v = j & 1 ? sy : sx;
      const bool on = TURN == NEIGHBOURS || 4 * l + (j < 4 ? j : dim / 4 + j - 4) < pairs;
      x[j] = f2(fmaf(a, u, -((on ? b : 0.f) * v)), fmaf(b, u, (on ? a : 0.f) * v));
    }
  }
}
template <typename T> __device__ __forceinline__ void runs_of(const Run<T>& a, const Run<T>& b, F2 (&x)[8]) {
  float v[8];
  unpack(a, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f2(v[2 * j], v[2 * j + 1]);
  unpack(b, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[4 + j] = f2(v[2 * j], v[2 * j + 1]);
}
template <typename T> __device__ __forceinline__ void store_two(T* first, T* second, const F2 (&x)[8]) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) split(x[j], v[2 * j], v[2 * j + 1]);
  store_run(first, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) split(x[4 + j], v[2 * j], v[2 * j + 1]);
  store_run(second, v);
}
template <typename P> __device__ __forceinline__ void lane_weights(const void* w, int e, int half, bool in, F2 (&out)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int at = (j < 4 ? e : e + half) + 2 * (j & 3);
    out[j] = in ? f2(param<P>(w, at), param<P>(w, at + 1)) : f2(0.f, 0.f);
  }
}
__device__ __forceinline__ float dot16(const F2 (&x)[8], const F2 (&y)[8]) {
  F2 s = mul2(x[0], y[0]), u = mul2(x[1], y[1]);
#pragma unroll
  for (int j = 2; j < 8; j += 2) {
    s = fma2(x[j], y[j], s);
    u = fma2(x[j + 1], y[j + 1], u);
  }
  float a, b;
  split(add2(s, u), a, b);
  return a + b;
}

// Heads [lo, hi) of one matrix row, LPH lanes a head and BATCH rounds of loads ahead.  `ready` makes w, c and s, behind the first loads.
template <typename T, int LPH, int TURN, int BATCH, typename R>
__device__ __forceinline__ void norm_heads(const T* x, T* out, int lo, int hi, int dim, float eps, int group, int e, int pairs, bool in, const F2 (&w)[8],
                                           const F2 (&c)[4], const F2 (&s)[4], R ready) {
  constexpr int G = 32 / LPH;
  const int half = dim / 2;
  const float inv = 1.f / (float)dim;
  Run<T> a[BATCH], b[BATCH];
  auto fetch = [&](int k, int h) {
    if (h < hi && in) {
      a[k] = load_run(x + (long long)h * dim + e);
      b[k] = load_run(x + (long long)h * dim + e + half);
    } else {
#pragma unroll
      for (int j = 0; j < (int)sizeof(T) / 2; ++j) a[k].v[j] = b[k].v[j] = make_uint4(0, 0, 0, 0);
    }
  };
#pragma unroll
  for (int k = 0; k < BATCH; ++k) fetch(k, lo + k * G + group);
  ready();
  for (int h0 = lo; h0 < hi; h0 += BATCH * G) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int h = h0 + k * G + group;
      F2 v[8];
      runs_of(a[k], b[k], v);
      fetch(k, h + BATCH * G);
      const float r = rsqrtf(fmaf(head_sum<LPH>(dot16(v, v)), inv, eps));
      const F2 r2 = f2(r, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = mul2(mul2(v[j], r2), w[j]);
      turn_two<TURN, LPH>(v, c, s, e / 8, pairs, dim);
      if (h < hi && in) store_two(out + (long long)h * dim + e, out + (long long)h * dim + e + half, v);
    }
  }
}

// parts: warps a token.
template <typename T, typename P, int LPH, int TURN>
__global__ void __launch_bounds__(TWO_CTA) k_qk_norm_two(adacgd_qk_norm_args a, int parts) {
  constexpr int BATCH = sizeof(T) == 4 ? 1 : 2;
  __shared__ __align__(16) float tables[TWO_WARPS][2 * MAX_PAIRS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, group = lane / LPH, e = 8 * l;
  const long long item = (long long)blockIdx.x * TWO_WARPS + warp, t = item / parts;
  if (t >= a.tokens) return;
  const bool in = l < a.head_dim / 16;
  const int heads = (int)(a.heads + a.key_heads), part = (int)(item % parts);
  const int lo = (int)((long long)heads * part / parts), hi = (int)((long long)heads * (part + 1) / parts), nq = (int)a.heads;
  F2 c[4], s[4], w[8];
  if (lo < nq) {
    norm_heads<T, LPH, TURN, BATCH>((const T*)a.q + t * a.q_stride, (T*)a.q_out + t * a.q_out_stride, lo, min(hi, nq), a.head_dim, a.eps, group, e, a.pairs, in, w, c, s, [&] {
      lane_weights<P>(a.q_weight, e, a.head_dim / 2, in, w);
      lane_turns<TURN>(a, t, l, in, tables[warp], false, c, s);
    });
  }
  if (hi > nq) {
    norm_heads<T, LPH, TURN, BATCH>((const T*)a.k + t * a.k_stride, (T*)a.k_out + t * a.k_out_stride, max(lo, nq) - nq, hi - nq, a.head_dim, a.eps, group, e,
                                      a.pairs, in, w, c, s, [&] {
      lane_weights<P>(a.k_weight, e, a.head_dim / 2, in, w);
      if (lo >= nq) lane_turns<TURN>(a, t, l, in, tables[warp], false, c, s);
    });
  }
}

template <typename T, int LPH, int TURN, int BATCH, typename R>
__device__ __forceinline__ void norm_heads_bwd(const T* x, const T* y, T* out, int lo, int hi, int dim, float eps, int group, int e, int pairs, bool in,
                                               const F2 (&w)[8], const F2 (&c)[4], const F2 (&s)[4], F2 (&dw)[8], R ready) {
  constexpr int G = 32 / LPH;
  const int half = dim / 2;
  const float inv = 1.f / (float)dim;
  Run<T> a[BATCH], b[BATCH], p[BATCH], q[BATCH];
  auto fetch = [&](int k, int h) {
    if (h < hi && in) {
      const long long at = (long long)h * dim + e;
      a[k] = load_run(x + at);
      b[k] = load_run(x + at + half);
      p[k] = load_run(y + at);
      q[k] = load_run(y + at + half);
    } else {
#pragma unroll
      for (int j = 0; j < (int)sizeof(T) / 2; ++j) a[k].v[j] = b[k].v[j] = p[k].v[j] = q[k].v[j] = make_uint4(0, 0, 0, 0);
    }
  };
#pragma unroll
  for (int k = 0; k < BATCH; ++k) fetch(k, lo + k * G + group);
  ready();
  for (int h0 = lo; h0 < hi; h0 += BATCH * G) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int h = h0 + k * G + group;
      F2 v[8], d[8];
      runs_of(a[k], b[k], v);
      runs_of(p[k], q[k], d);
      fetch(k, h + BATCH * G);
      turn_two<TURN, LPH>(d, c, s, e / 8, pairs, dim);
      const float r = rsqrtf(fmaf(head_sum<LPH>(dot16(v, v)), inv, eps));
      const F2 r2 = f2(r, r);
      const bool live = h < hi && in;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = mul2(v[j], r2);                       // x r
        if (live) dw[j] = fma2(d[j], v[j], dw[j]);
        d[j] = mul2(d[j], w[j]);                     // g
      }
      const float m = -head_sum<LPH>(dot16(d, v)) * inv;
      const F2 m2 = f2(m, m);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = mul2(r2, fma2(m2, v[j], d[j]));
      if (live) store_two(out + (long long)h * dim + e, out + (long long)h * dim + e + half, d);
    }
  }
}

template <typename T, typename P, int LPH, int TURN>
__global__ void __launch_bounds__(TWO_CTA, sizeof(T) == 4 ? 3 : 4) k_qk_norm_two_bwd(adacgd_qk_norm_backward_args g, int parts, float* part, long long part_stride) {
  constexpr int BATCH = 1, DIM = 16 * LPH, SLOTS = TWO_CTA / LPH;
  const adacgd_qk_norm_args& a = g.f;
  __shared__ __align__(16) float tables[TWO_WARPS][2 * MAX_PAIRS], rows[SLOTS * DIM];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, group = lane / LPH, e = 8 * l, half = a.head_dim / 2;
  const bool in = l < a.head_dim / 16;
  const int heads = (int)(a.heads + a.key_heads), nq = (int)a.heads;
  F2 dwq[8], dwk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) dwq[j] = dwk[j] = f2(0.f, 0.f);
  const long long items = a.tokens * parts;
  for (long long item = (long long)blockIdx.x * TWO_WARPS + warp; item < items; item += (long long)gridDim.x * TWO_WARPS) {
    const long long t = item / parts;
    const int mine = (int)(item % parts), lo = (int)((long long)heads * mine / parts), hi = (int)((long long)heads * (mine + 1) / parts);
    F2 c[4], s[4], w[8];
    if (lo < nq) {
      norm_heads_bwd<T, LPH, TURN, BATCH>((const T*)a.q + t * a.q_stride, (const T*)a.q_out + t * a.q_out_stride, (T*)g.dq + t * g.dq_stride, lo,
                                            min(hi, nq), a.head_dim, a.eps, group, e, a.pairs, in, w, c, s, dwq, [&] {
        lane_weights<P>(a.q_weight, e, half, in, w);
        lane_turns<TURN>(a, t, l, in, tables[warp], true, c, s);
      });
    }
    if (hi > nq) {
      norm_heads_bwd<T, LPH, TURN, BATCH>((const T*)a.k + t * a.k_stride, (const T*)a.k_out + t * a.k_out_stride, (T*)g.dk + t * g.dk_stride,
                                            max(lo, nq) - nq, hi - nq, a.head_dim, a.eps, group, e, a.pairs, in, w, c, s, dwk, [&] {
        lane_weights<P>(a.k_weight, e, half, in, w);
        if (lo >= nq) lane_turns<TURN>(a, t, l, in, tables[warp], true, c, s);
      });
    }
  }
  if (!part) return;
  const int slot = threadIdx.x / LPH;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
    if (in) {
#pragma unroll
      for (int j = 0; j < 8; ++j) *reinterpret_cast<F2*>(rows + slot * DIM + (j < 4 ? e : e + half) + 2 * (j & 3)) = k ? dwk[j] : dwq[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.head_dim; i += TWO_CTA) {
      float sum = 0.f;
      for (int j = 0; j < SLOTS; ++j) sum += rows[j * DIM + i];
      part[(2ll * blockIdx.x + k) * part_stride + i] = sum;
    }
  }
}

// Joins the CTAs' partial gradients in order, in binary64: a warp a column.
template <typename P>
__global__ void __launch_bounds__(256) k_qk_norm_dw(const float* part, long long part_stride, int parts, int dim, void* dqw, void* dkw) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, e = blockIdx.x * 8 + (threadIdx.x >> 5), k = blockIdx.y;
  if (e >= dim) return;
  double sum = 0.0;
#pragma unroll 8
  for (int i = lane; i < parts; i += 32) sum += (double)__ldcg(part + (2ll * i + k) * part_stride + e);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  void* const to = k ? dkw : dqw;
  if (lane == 0 && to) ((P*)to)[e] = from_f<P>((float)sum);
}

// --------------------------------------------------------------------------
// any head length and alignment
// --------------------------------------------------------------------------
// A warp a head, element by element; the row waits in shared memory for the rotation.
constexpr int ANY_CTA = 256, ANY_WARPS = ANY_CTA / 32;

// K elements a lane: heads of up to 32 K.  The next head's are loaded ahead.
template <typename T, int K> struct Lane {
  float v[K];
  __device__ __forceinline__ void load(const T* p, int dim, bool on) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = (threadIdx.x & 31) + 32 * k;
      v[k] = on && e < dim ? to_f(p[e]) : 0.f;
    }
  }
};
template <typename T> __device__ __forceinline__ T* head_at(const adacgd_qk_norm_args& a, const void* q, long long qs, const void* k, long long ks, long long t, int h) {
  return h < a.heads ? (T*)q + place(qs, t, h, a.head_dim) : (T*)k + place(ks, t, h - (int)a.heads, a.head_dim);
}

template <typename T, typename P, int K>
__global__ void __launch_bounds__(ANY_CTA) k_qk_norm_any(adacgd_qk_norm_args a) {
  extern __shared__ float any_smem[];
  const int dim = a.head_dim, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* const cs = any_smem;
  float* const sn = cs + dim;
  float* const row = sn + dim + warp * dim;
  const long long t = blockIdx.x;
  const int heads = (int)(a.heads + a.key_heads);
  auto at = [&](int h) { return head_at<const T>(a, a.q, a.q_stride, a.k, a.k_stride, t, h); };
  Lane<T, K> x;
  if (warp < heads) x.load(at(warp), dim, true);
  for (int i = 2 * a.pairs + threadIdx.x; i < dim; i += ANY_CTA) {
    cs[i] = 1.f;
    sn[i] = 0.f;
  }
  for (int i = threadIdx.x; i < a.pairs; i += ANY_CTA) fill_turns(a, t, i, cs, sn, false);
  __syncthreads();
  for (int h = warp; h < heads; h += ANY_WARPS) {
    const Lane<T, K> now = x;
    if (h + ANY_WARPS < heads) x.load(at(h + ANY_WARPS), dim, true);
    const bool query = h < a.heads;
    T* const out = head_at<T>(a, a.q_out, a.q_out_stride, a.k_out, a.k_out_stride, t, h);
    const void* const w = query ? a.q_weight : a.k_weight;
    float q = 0.f;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = lane + 32 * k;
      q = fmaf(now.v[k], now.v[k], q);
      if (e < dim) row[e] = now.v[k] * param<P>(w, e);
    }
    const float r = rsqrtf(fmaf(head_sum<32>(q), 1.f / (float)dim, a.eps));
    __syncwarp();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = lane + 32 * k;
      if (e < dim) out[e] = from_f<T>(r * fmaf(e < 2 * a.pairs ? row[partner(a, e)] : 0.f, sn[e], row[e] * cs[e]));
    }
  }
}

// The weights' gradients stay with the lane, and are added up in shared memory at the end.
template <typename T, typename P, int K>
__global__ void __launch_bounds__(ANY_CTA) k_qk_norm_bwd_any(adacgd_qk_norm_backward_args g, float* part, long long part_stride) {
  extern __shared__ float any_smem[];
  const adacgd_qk_norm_args& a = g.f;
  const int dim = a.head_dim, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* const cs = any_smem;
  float* const sn = cs + dim;
  float* const sums = sn + dim;                        // [warps][2][dim]
  float* const row = sums + 2 * ANY_WARPS * dim + warp * dim;
  const int heads = (int)(a.heads + a.key_heads);
  float dwq[K], dwk[K];
#pragma unroll
  for (int k = 0; k < K; ++k) dwq[k] = dwk[k] = 0.f;
  for (long long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    auto x_at = [&](int h) { return head_at<const T>(a, a.q, a.q_stride, a.k, a.k_stride, t, h); };
    auto y_at = [&](int h) { return head_at<const T>(a, a.q_out, a.q_out_stride, a.k_out, a.k_out_stride, t, h); };
    Lane<T, K> x, y;
    if (warp < heads) {
      x.load(x_at(warp), dim, true);
      y.load(y_at(warp), dim, true);
    }
    __syncthreads();
    for (int i = 2 * a.pairs + threadIdx.x; i < dim; i += ANY_CTA) {
      cs[i] = 1.f;
      sn[i] = 0.f;
    }
    for (int i = threadIdx.x; i < a.pairs; i += ANY_CTA) fill_turns(a, t, i, cs, sn, true);
    __syncthreads();
    for (int h = warp; h < heads; h += ANY_WARPS) {
      const Lane<T, K> v = x, u = y;
      if (h + ANY_WARPS < heads) {
        x.load(x_at(h + ANY_WARPS), dim, true);
        y.load(y_at(h + ANY_WARPS), dim, true);
      }
      const bool query = h < a.heads;
      T* const out = head_at<T>(a, g.dq, g.dq_stride, g.dk, g.dk_stride, t, h);
      const void* const w = query ? a.q_weight : a.k_weight;
      float q = 0.f;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int e = lane + 32 * k;
        q = fmaf(v.v[k], v.v[k], q);
        if (e < dim) row[e] = u.v[k];
      }
      const float r = rsqrtf(fmaf(head_sum<32>(q), 1.f / (float)dim, a.eps));
      __syncwarp();
      float dot = 0.f, dn[K];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int e = lane + 32 * k;
        dn[k] = 0.f;
        if (e < dim) {
          const float d = fmaf(e < 2 * a.pairs ? row[partner(a, e)] : 0.f, sn[e], u.v[k] * cs[e]), xr = v.v[k] * r;
          if (query) dwq[k] = fmaf(d, xr, dwq[k]); else dwk[k] = fmaf(d, xr, dwk[k]);
          dn[k] = d * param<P>(w, e);
          dot = fmaf(dn[k], xr, dot);
        }
      }
      const float m = head_sum<32>(dot) * (1.f / (float)dim);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int e = lane + 32 * k;
        if (e < dim) out[e] = from_f<T>(r * fmaf(-m, v.v[k] * r, dn[k]));
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = lane + 32 * k;
    if (e < dim) {
      sums[2 * warp * dim + e] = dwq[k];
      sums[(2 * warp + 1) * dim + e] = dwk[k];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * dim; i += ANY_CTA) {
    float sum = 0.f;
    for (int w = 0; w < ANY_WARPS; ++w) sum += sums[2 * w * dim + i];
    const int k = i >= dim;
    part[(2ll * blockIdx.x + k) * part_stride + i - k * dim] = sum;
  }
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
template <typename T> bool on_runs(const void* p, long long stride, long long tokens) {
  const size_t step = 8 * sizeof(T);
  return !p || ((uintptr_t)p % step == 0 && (tokens <= 1 || stride * sizeof(T) % step == 0));
}
template <typename T> bool head_runs(const adacgd_qk_norm_args& a) {
  return a.head_dim % 8 == 0 && a.head_dim <= 256 && on_runs<T>(a.q, a.q_stride, a.tokens) && on_runs<T>(a.k, a.k_stride, a.tokens) &&
         on_runs<T>(a.q_out, a.q_out_stride, a.tokens) && on_runs<T>(a.k_out, a.k_out_stride, a.tokens);
}
Reach reach_of(const adacgd_qk_norm_args& a) {
  if (a.interleaved && 2 * a.pairs == a.head_dim) return NEAR;
  if (a.interleaved || a.pairs == 0) return PART;
  return a.pairs % 8 == 0 ? LANE : ROW;
}

template <typename T, typename P, int LPH, int REACH>
int norm_launch(const adacgd_qk_norm_args& a, const Where& at) {
  constexpr int BATCH = sizeof(T) == 4 ? 2 : 4, SLOTS = ROT_CTA / LPH;
  const long long heads = a.heads + a.key_heads;
  // as many tokens a CTA as make a table for every thread, where there are that many
  long long each = a.pairs ? ROT_CTA / a.pairs : ROT_MAX_TOKENS;
  if (each < 1) each = 1;
  if (each > ROT_MAX_TOKENS) each = ROT_MAX_TOKENS;
  while (each > 1 && (a.tokens + each - 1) / each < 4ll * at.sms) each /= 2;
  long long ctas = (a.tokens + each - 1) / each, cut = 1;
  if (ctas < at.sms) {                       // few tokens: their heads over several CTAs
    cut = (each * heads + SLOTS - 1) / SLOTS;
    if (cut > 2 * at.sms / ctas) cut = 2 * at.sms / ctas;
    if (cut < 1) cut = 1;
  }
  k_qk_norm<T, P, LPH, REACH, BATCH><<<dim3((unsigned)ctas, (unsigned)cut), ROT_CTA, 0, at.stream>>>(a, (int)each);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename P>
int join_weights(const adacgd_qk_norm_backward_args& g, const TrainScratch& s, int parts, const Where& at) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((g.f.head_dim + 7) / 8), 2);
  cfg.blockDim = dim3(256);
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_qk_norm_dw<P>, (const float*)s.norm_part, s.max_cols, parts, (int)g.f.head_dim, g.dq_weight, g.dk_weight) ==
                 cudaSuccess
             ? 2
             : -1;
}

template <typename T, typename P, int LPH, int REACH>
int norm_bwd_launch(const TrainScratch& s, const adacgd_qk_norm_backward_args& g, const Where& at) {
  constexpr int BATCH = 2;
  const adacgd_qk_norm_args& a = g.f;
  static std::atomic<int> table[TRAIN_DEVICES];
  auto kern = k_qk_norm_bwd<T, P, LPH, REACH, BATCH>;
  const int per_sm = resident_ctas(kern, table, at.device, ROT_CTA, 0);
  if (per_sm < 1) return -1;
  long long most = (long long)per_sm * at.sms;
  if (most > NORM_PARTS) most = NORM_PARTS;
  long long each = a.pairs ? ROT_CTA / a.pairs : ROT_MAX_TOKENS;
  if (each < 1) each = 1;
  if (each > ROT_MAX_TOKENS) each = ROT_MAX_TOKENS;
  while (each > 1 && (a.tokens + each - 1) / each < most) each /= 2;
  long long ctas = (a.tokens + each - 1) / each;
  if (ctas > most) ctas = most;
  const bool grads = g.dq_weight || g.dk_weight;
  kern<<<(unsigned)ctas, ROT_CTA, 0, at.stream>>>(g, (int)each, grads ? s.norm_part : (float*)nullptr, s.max_cols);
  if (cudaGetLastError() != cudaSuccess) return -1;
  return grads ? join_weights<P>(g, s, (int)ctas, at) : 1;
}

template <typename T, typename P, int K>
int any_bwd_launch(const TrainScratch& s, const adacgd_qk_norm_backward_args& g, const Where& at) {
  static std::atomic<int> table[TRAIN_DEVICES];
  constexpr int MOST = (2 + 3 * ANY_WARPS) * 32 * K * 4;
  if (resident_ctas(k_qk_norm_bwd_any<T, P, K>, table, at.device, ANY_CTA, MOST) < 1) return -1;
  const bool grads = g.dq_weight || g.dk_weight;
  const int ctas = (int)(g.f.tokens < NORM_PARTS ? g.f.tokens : NORM_PARTS);
  k_qk_norm_bwd_any<T, P, K><<<ctas, ANY_CTA, (2 + 3 * ANY_WARPS) * g.f.head_dim * 4, at.stream>>>(g, grads ? s.norm_part : (float*)nullptr, s.max_cols);
  if (cudaGetLastError() != cudaSuccess) return -1;
  return grads ? join_weights<P>(g, s, ctas, at) : 1;
}

// Heads of two runs a lane: lengths by 16, turned in neighbours, or in halves of the whole head or of whole runs of its first half.
bool in_front(const adacgd_qk_norm_args& a) { return a.pairs % 8 == 0 && 4 * a.pairs <= a.head_dim; }
bool two_runs(const adacgd_qk_norm_args& a) { return a.head_dim % 16 == 0 && (a.interleaved || 2 * a.pairs == a.head_dim || in_front(a)); }
// Warps a token: one where that gives every SM sixteen of them.
int parts_of(const adacgd_qk_norm_args& a, int lph, const Where& at) {
  const long long heads = a.heads + a.key_heads, most = (heads + 32 / lph - 1) / (32 / lph);
  long long parts = 16ll * at.sms / a.tokens;
  if (parts > most) parts = most;
  return (int)(parts < 1 ? 1 : parts);
}

template <typename T, typename P, int LPH, int TURN>
int two_launch(const adacgd_qk_norm_args& a, const Where& at) {
  const int parts = parts_of(a, LPH, at);
  const long long ctas = (a.tokens * parts + TWO_WARPS - 1) / TWO_WARPS;
  k_qk_norm_two<T, P, LPH, TURN><<<(unsigned)ctas, TWO_CTA, 0, at.stream>>>(a, parts);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}
template <typename T, typename P, int LPH, int TURN>
int two_bwd_launch(const TrainScratch& s, const adacgd_qk_norm_backward_args& g, const Where& at) {
  const int parts = parts_of(g.f, LPH, at);
  long long ctas = (g.f.tokens * parts + TWO_WARPS - 1) / TWO_WARPS;
  if (ctas > (sizeof(T) == 4 ? 3ll : 4ll) * at.sms) ctas = (sizeof(T) == 4 ? 3ll : 4ll) * at.sms;
  if (ctas > NORM_PARTS) ctas = NORM_PARTS;
  const bool grads = g.dq_weight || g.dk_weight;
  k_qk_norm_two_bwd<T, P, LPH, TURN><<<(unsigned)ctas, TWO_CTA, 0, at.stream>>>(g, parts, grads ? s.norm_part : (float*)nullptr, s.max_cols);
  if (cudaGetLastError() != cudaSuccess) return -1;
  return grads ? join_weights<P>(g, s, (int)ctas, at) : 1;
}

#define BY_LANES(call)                                                                                 \
  if (a.head_dim <= 32) { constexpr int LPH = 2; BY_TURN(call) }                                       \
  if (a.head_dim <= 64) { constexpr int LPH = 4; BY_TURN(call) }                                       \
  if (a.head_dim <= 128) { constexpr int LPH = 8; BY_TURN(call) }                                      \
  { constexpr int LPH = 16; BY_TURN(call) }
#define BY_TURN(call)                                                                                  \
  if (a.pairs == 0) { constexpr int TURN = NONE; return call; }                                        \
  if (a.interleaved && 2 * a.pairs < a.head_dim) { constexpr int TURN = PARTLY; return call; }         \
  if (a.interleaved) { constexpr int TURN = NEIGHBOURS; return call; }                                 \
  if (2 * a.pairs == a.head_dim) { constexpr int TURN = HALVES; return call; }                         \
  { constexpr int TURN = FRONT; return call; }

#define BY_HEAD(call)                                                                                  \
  const Reach reach = reach_of(a);                                                                     \
  if (a.head_dim <= 64) { constexpr int LPH = 8; BY_REACH(call) }                                      \
  if (a.head_dim <= 128) { constexpr int LPH = 16; BY_REACH(call) }                                    \
  { constexpr int LPH = 32; BY_REACH(call) }
#define BY_REACH(call)                                                                                 \
  if (reach == NEAR) { constexpr int REACH = NEAR; return call; }                                      \
  if (reach == PART) { constexpr int REACH = PART; return call; }                                      \
  if (reach == LANE) { constexpr int REACH = LANE; return call; }                                      \
  { constexpr int REACH = ROW; return call; }

template <typename T, typename P>
int norm_t(const adacgd_qk_norm_args& a, const Where& at) {
  if (!head_runs<T>(a)) {
    const int smem = (2 + ANY_WARPS) * a.head_dim * 4;
    if (a.head_dim <= 64) k_qk_norm_any<T, P, 2><<<(unsigned)a.tokens, ANY_CTA, smem, at.stream>>>(a);
    else if (a.head_dim <= 128) k_qk_norm_any<T, P, 4><<<(unsigned)a.tokens, ANY_CTA, smem, at.stream>>>(a);
    else k_qk_norm_any<T, P, 16><<<(unsigned)a.tokens, ANY_CTA, smem, at.stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  }
  if (two_runs(a)) { BY_LANES((two_launch<T, P, LPH, TURN>(a, at))) }
  BY_HEAD((norm_launch<T, P, LPH, REACH>(a, at)))
}

template <typename T, typename P>
int norm_bwd_t(const TrainScratch& s, const adacgd_qk_norm_backward_args& g, const Where& at) {
  const adacgd_qk_norm_args& a = g.f;
  if (!head_runs<T>(a) || !on_runs<T>(g.dq, g.dq_stride, a.tokens) || !on_runs<T>(g.dk, g.dk_stride, a.tokens)) {
    if (a.head_dim <= 64) return any_bwd_launch<T, P, 2>(s, g, at);
    if (a.head_dim <= 128) return any_bwd_launch<T, P, 4>(s, g, at);
    return any_bwd_launch<T, P, 16>(s, g, at);
  }
  if (two_runs(a)) { BY_LANES((two_bwd_launch<T, P, LPH, TURN>(s, g, at))) }
  BY_HEAD((norm_bwd_launch<T, P, LPH, REACH>(s, g, at)))
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_qk_norm(const adacgd_qk_norm_args& a, const Where& at) {
  if (a.param_dtype == ADACGD_F32) BY_TYPE(a.dtype, (norm_t<T, float>(a, at)))
  BY_TYPE(a.dtype, (norm_t<T, T>(a, at)))
}

int launch_qk_norm_backward(const TrainScratch& s, const adacgd_qk_norm_backward_args& a, const Where& at) {
  if (a.f.param_dtype == ADACGD_F32) BY_TYPE(a.f.dtype, (norm_bwd_t<T, float>(s, a, at)))
  BY_TYPE(a.f.dtype, (norm_bwd_t<T, T>(s, a, at)))
}

}  // namespace adacgd
