// Norm and rotation of queries and keys, and its backward pass (adacgd_train.h).  Bound by memory: every element is read once and
// written once.  A head is held by the lanes of a part of a warp, eight elements each, so its mean of squares is a few
// shuffles; the cosines and sines of a token are made once (in binary64: position times frequency, reduced to a turn) and used by all its heads.
#include "adacgd_train.cuh"

namespace adacgd {
namespace {

__device__ __forceinline__ long long position_at(const adacgd_qk_norm_args& a, long long t) {
  return a.position_bytes == 8 ? reinterpret_cast<const long long*>(a.positions)[t] : (long long)reinterpret_cast<const int32_t*>(a.positions)[t];
}

// Cosine and sine of position * freq.  The product of a 53-bit and a 24-bit number is rounded once in binary64; as turns it is reduced exactly, so the
// angle is off by 2^-52 of itself: 1e-9 rad at ten million rad.
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
__device__ __forceinline__ int partner(const adacgd_qk_norm_args& a, int e) {
  if (e >= 2 * a.pairs) return e;
  if (a.interleaved) return e ^ 1;
  return e < a.pairs ? e + a.pairs : e - a.pairs;
}

template <typename P> __device__ __forceinline__ float param(const void* w, int e) { return w ? to_f(((const P*)w)[e]) : 1.f; }

// Where head h of token t lies; heads behind the queries' are the keys'.
__device__ __forceinline__ long long place(long long stride, long long t, int h, int dim) { return t * stride + (long long)h * dim; }

// --------------------------------------------------------------------------
// heads of whole aligned runs
// --------------------------------------------------------------------------
constexpr int ROT_CTA = 256, ROT_WARPS = ROT_CTA / 32;
constexpr int ROT_MAX_TOKENS = 8;

// How the partner of a pair is reached: NEAR within the lane (neighbours), LANE in another lane at the same place, ROW through shared
// memory (halves whose distance is no whole number of runs).
enum Reach { NEAR, LANE, ROW };

// The lane's eight elements turned.  cs, sn: the lane's entries of the token's tables.
template <int LPH, int REACH>
__device__ __forceinline__ void rotate(const adacgd_qk_norm_args& a, const float* cs, const float* sn, int e0, float* row, float (&x)[8]) {
  float c[8], s[8], y[8];
#pragma unroll
  for (int j = 0; j < 8; j += 4) {
    *reinterpret_cast<float4*>(c + j) = *reinterpret_cast<const float4*>(cs + e0 + j);
    *reinterpret_cast<float4*>(s + j) = *reinterpret_cast<const float4*>(sn + e0 + j);
  }
  if (REACH == NEAR) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j ^ 1];
  } else if (REACH == LANE) {
    const int d = a.pairs / 8, me = e0 / 8;
    const int from = me < d ? me + d : (me < 2 * d ? me - d : me);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = __shfl_sync(0xffffffffu, x[j], from, LPH);
  } else {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) row[e0 + j] = x[j];
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = e0 + j < a.head_dim ? row[partner(a, e0 + j)] : 0.f;
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

// Joins the CTAs' partial gradients in order, in binary64: a warp a column.
template <typename P>
__global__ void __launch_bounds__(256) k_qk_norm_dw(const float* part, long long part_stride, int parts, int dim, void* dqw, void* dkw) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, e = blockIdx.x * 8 + (threadIdx.x >> 5), k = blockIdx.y;
  if (e >= dim) return;
  double sum = 0.0;
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

template <typename T, typename P>
__global__ void __launch_bounds__(ANY_CTA) k_qk_norm_any(adacgd_qk_norm_args a) {
  extern __shared__ float any_smem[];
  const int dim = a.head_dim, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* const cs = any_smem;
  float* const sn = cs + dim;
  float* const row = sn + dim + warp * dim;
  const long long t = blockIdx.x;
  for (int i = 2 * a.pairs + threadIdx.x; i < dim; i += ANY_CTA) {
    cs[i] = 1.f;
    sn[i] = 0.f;
  }
  for (int i = threadIdx.x; i < a.pairs; i += ANY_CTA) fill_turns(a, t, i, cs, sn, false);
  __syncthreads();
  const int heads = (int)(a.heads + a.key_heads);
  for (int h = warp; h < heads; h += ANY_WARPS) {
    const bool query = h < a.heads;
    const T* const x = query ? (const T*)a.q + place(a.q_stride, t, h, dim) : (const T*)a.k + place(a.k_stride, t, h - (int)a.heads, dim);
    T* const out = query ? (T*)a.q_out + place(a.q_out_stride, t, h, dim) : (T*)a.k_out + place(a.k_out_stride, t, h - (int)a.heads, dim);
    const void* const w = query ? a.q_weight : a.k_weight;
    float q = 0.f;
    __syncwarp();
    for (int e = lane; e < dim; e += 32) {
      const float v = to_f(x[e]);
      q = fmaf(v, v, q);
      row[e] = v * param<P>(w, e);
    }
    const float r = rsqrtf(fmaf(head_sum<32>(q), 1.f / (float)dim, a.eps));
    __syncwarp();
    for (int e = lane; e < dim; e += 32) out[e] = from_f<T>(r * fmaf(row[partner(a, e)], sn[e], row[e] * cs[e]));
  }
}

// The weights' gradients are added up in the warp's own row of shared memory, the warps' rows at the end.
template <typename T, typename P>
__global__ void __launch_bounds__(ANY_CTA) k_qk_norm_bwd_any(adacgd_qk_norm_backward_args g, float* part, long long part_stride) {
  extern __shared__ float any_smem[];
  const adacgd_qk_norm_args& a = g.f;
  const int dim = a.head_dim, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* const cs = any_smem;
  float* const sn = cs + dim;
  float* const sums = sn + dim;                        // [warps][2][dim]
  float* const row = sums + 2 * ANY_WARPS * dim + warp * dim;
  float* const mine = sums + 2 * warp * dim;
  for (int i = lane; i < 2 * dim; i += 32) mine[i] = 0.f;
  const int heads = (int)(a.heads + a.key_heads);
  for (long long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    __syncthreads();
    for (int i = 2 * a.pairs + threadIdx.x; i < dim; i += ANY_CTA) {
      cs[i] = 1.f;
      sn[i] = 0.f;
    }
    for (int i = threadIdx.x; i < a.pairs; i += ANY_CTA) fill_turns(a, t, i, cs, sn, true);
    __syncthreads();
    for (int h = warp; h < heads; h += ANY_WARPS) {
      const bool query = h < a.heads;
      const int kh = h - (int)a.heads;
      const T* const x = query ? (const T*)a.q + place(a.q_stride, t, h, dim) : (const T*)a.k + place(a.k_stride, t, kh, dim);
      const T* const y = query ? (const T*)a.q_out + place(a.q_out_stride, t, h, dim) : (const T*)a.k_out + place(a.k_out_stride, t, kh, dim);
      T* const out = query ? (T*)g.dq + place(g.dq_stride, t, h, dim) : (T*)g.dk + place(g.dk_stride, t, kh, dim);
      const void* const w = query ? a.q_weight : a.k_weight;
      float q = 0.f;
      __syncwarp();
      for (int e = lane; e < dim; e += 32) {
        const float v = to_f(x[e]);
        q = fmaf(v, v, q);
        row[e] = to_f(y[e]);
      }
      const float r = rsqrtf(fmaf(head_sum<32>(q), 1.f / (float)dim, a.eps));
      __syncwarp();
      float dot = 0.f;
      float dn[ADACGD_TRAIN_MAX_HEAD / 32];            // the lane's elements
#pragma unroll
      for (int k = 0; k < ADACGD_TRAIN_MAX_HEAD / 32; ++k) {
        const int e = lane + 32 * k;
        if (e < dim) {
          const float d = fmaf(row[partner(a, e)], sn[e], row[e] * cs[e]), v = to_f(x[e]) * r;
          mine[(query ? 0 : dim) + e] += d * v;
          dn[k] = d * param<P>(w, e);
          dot = fmaf(dn[k], v, dot);
        }
      }
      const float m = head_sum<32>(dot) * (1.f / (float)dim);
#pragma unroll
      for (int k = 0; k < ADACGD_TRAIN_MAX_HEAD / 32; ++k) {
        const int e = lane + 32 * k;
        if (e < dim) out[e] = from_f<T>(r * fmaf(-m, to_f(x[e]) * r, dn[k]));
      }
    }
  }
  __syncthreads();
  if (!part) return;
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
  if (a.interleaved || a.pairs == 0) return NEAR;
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

#define BY_HEAD(call)                                                                                  \
  const Reach reach = reach_of(a);                                                                     \
  if (a.head_dim <= 64) { constexpr int LPH = 8; BY_REACH(call) }                                      \
  if (a.head_dim <= 128) { constexpr int LPH = 16; BY_REACH(call) }                                    \
  { constexpr int LPH = 32; BY_REACH(call) }
#define BY_REACH(call)                                                                                 \
  if (reach == NEAR) { constexpr int REACH = NEAR; return call; }                                      \
  if (reach == LANE) { constexpr int REACH = LANE; return call; }                                      \
  { constexpr int REACH = ROW; return call; }

template <typename T, typename P>
int norm_t(const adacgd_qk_norm_args& a, const Where& at) {
  if (!head_runs<T>(a)) {
    k_qk_norm_any<T, P><<<(unsigned)a.tokens, ANY_CTA, (2 + ANY_WARPS) * a.head_dim * 4, at.stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  }
  BY_HEAD((norm_launch<T, P, LPH, REACH>(a, at)))
}

template <typename T, typename P>
int norm_bwd_t(const TrainScratch& s, const adacgd_qk_norm_backward_args& g, const Where& at) {
  const adacgd_qk_norm_args& a = g.f;
  if (!head_runs<T>(a) || !on_runs<T>(g.dq, g.dq_stride, a.tokens) || !on_runs<T>(g.dk, g.dk_stride, a.tokens)) {
    static std::atomic<int> table[TRAIN_DEVICES];
    constexpr int MOST = (2 + 3 * ANY_WARPS) * ADACGD_TRAIN_MAX_HEAD * 4;
    if (resident_ctas(k_qk_norm_bwd_any<T, P>, table, at.device, ANY_CTA, MOST) < 1) return -1;
    const bool grads = g.dq_weight || g.dk_weight;
    const int ctas = (int)(a.tokens < NORM_PARTS ? a.tokens : NORM_PARTS);
    k_qk_norm_bwd_any<T, P><<<ctas, ANY_CTA, (2 + 3 * ANY_WARPS) * a.head_dim * 4, at.stream>>>(g, grads ? s.norm_part : (float*)nullptr, s.max_cols);
    if (cudaGetLastError() != cudaSuccess) return -1;
    return grads ? join_weights<P>(g, s, ctas, at) : 1;
  }
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
