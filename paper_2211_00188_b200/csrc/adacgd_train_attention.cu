// Attention and its backward pass (adacgd_train.h) for any element type, alignment and head length: binary32 products on the
// general cores.  One pass over the keys with the running maximum and sum of each row; the scores never leave the SM.  The backward pass computes
// the probabilities again, once by query tiles for dq and once by key tiles for dk and dv, so that every sum has one owner and a
// fixed order.  Bound by shared memory reads beside the multiplications (a thread holds a 4 x 4 part of a score tile).
#include "adacgd_train_attention.cuh"

namespace adacgd {
namespace {

constexpr int ATT_CTA = 256;   // 16 x 16 threads over a tile of scores

// Rows [first, first + ROWS) of a sequence as binary32, zero where they do not count or lie behind its end.
template <typename T, int DM, int ROWS>
__device__ __forceinline__ void load_tile(float* sm, const void* base, long long stride, long long row, int head, int dim, const uint8_t* counts, int first) {
  for (int i = threadIdx.x; i < ROWS * DM; i += ATT_CTA) {
    const int r = i / DM, d = i - r * DM;
    float v = 0.f;
    if (d < dim && counts[r]) v = to_f(((const T*)base)[(row + first + r) * stride + (long long)head * dim + d]);
    sm[r * (DM + 4) + d] = v;
  }
}
template <int ROWS>
__device__ __forceinline__ void load_counts(uint8_t* counts, const adacgd_attention_inputs& a, const Tile& t, int first) {
  for (int r = threadIdx.x; r < ROWS; r += ATT_CTA) {
    const int i = first + r;
    counts[r] = i < t.length && (!a.mask || a.mask[t.row + i]);
  }
}

// s[r][c] = x_i . y_j with i = ty + 16 r, j = tx + 16 c
template <int DM, int RM, int RN>
__device__ __forceinline__ void products(const float* x, const float* y, float (&s)[RM][RN]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int r = 0; r < RM; ++r)
#pragma unroll
    for (int c = 0; c < RN; ++c) s[r][c] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DM; d += 4) {
    float4 u[RM], v[RN];
#pragma unroll
    for (int r = 0; r < RM; ++r) u[r] = *reinterpret_cast<const float4*>(x + (ty + 16 * r) * (DM + 4) + d);
#pragma unroll
    for (int c = 0; c < RN; ++c) v[c] = *reinterpret_cast<const float4*>(y + (tx + 16 * c) * (DM + 4) + d);
#pragma unroll
    for (int r = 0; r < RM; ++r)
#pragma unroll
      for (int c = 0; c < RN; ++c) {
        s[r][c] = fmaf(u[r].x, v[c].x, s[r][c]);
        s[r][c] = fmaf(u[r].y, v[c].y, s[r][c]);
        s[r][c] = fmaf(u[r].z, v[c].z, s[r][c]);
        s[r][c] = fmaf(u[r].w, v[c].w, s[r][c]);
      }
  }
}

// o[r] (rows ty + 16 r, columns 4 tx + 64 k ..) += sum over j of p(row, j) y_j.  BY_ROW: p is stored [row][j], else [j][row].
template <int DM, int R, int N, int PS, bool BY_ROW>
__device__ __forceinline__ void accumulate(const float* p, const float* y, float (&o)[R][DM / 16]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 4
  for (int j = 0; j < N; ++j) {
    float w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = BY_ROW ? p[(ty + 16 * r) * PS + j] : p[j * PS + ty + 16 * r];
#pragma unroll
    for (int k = 0; k < DM / 64; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(y + j * (DM + 4) + 64 * k + 4 * tx);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        o[r][4 * k] = fmaf(w[r], v.x, o[r][4 * k]);
        o[r][4 * k + 1] = fmaf(w[r], v.y, o[r][4 * k + 1]);
        o[r][4 * k + 2] = fmaf(w[r], v.z, o[r][4 * k + 2]);
        o[r][4 * k + 3] = fmaf(w[r], v.w, o[r][4 * k + 3]);
      }
    }
  }
}

// Stores factor * o to rows of the sequence; rows inside it that do not count get 0.
template <typename T, int DM, int R>
__device__ __forceinline__ void store_tile(void* base, long long stride, const Tile& t, int first, int head, int dim, const uint8_t* counts,
                                           const float (&factor)[R], const float (&o)[R][DM / 16]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = ty + 16 * r;
    if (first + i >= t.length) continue;
    T* const to = (T*)base + (t.row + first + i) * stride + (long long)head * dim;
#pragma unroll
    for (int k = 0; k < DM / 16; ++k) {
      const int d = 64 * (k / 4) + 4 * tx + k % 4;
      if (d < dim) to[d] = from_f<T>(counts[i] ? o[r][k] * factor[r] : 0.f);
    }
  }
}

__device__ __forceinline__ float max16(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = !(v >= u) && !(v != v) ? u : v;      // a NaN stays
  }
  return v;
}
__device__ __forceinline__ float sum16(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

constexpr float NONE = -INFINITY;

template <int DM, int BM, int BN> struct FwdSmem {
  static constexpr int PS = BN + 4, FLOATS = (BM + 2 * BN) * (DM + 4) + BM * PS;
  static constexpr int BYTES = FLOATS * 4 + BM + BN;
};

template <typename T, int DM, int BM, int BN>
__global__ void __launch_bounds__(ATT_CTA) k_attention_any(adacgd_attention_args g) {
  typedef FwdSmem<DM, BM, BN> S;
  constexpr int RM = BM / 16, RN = BN / 16;
  extern __shared__ __align__(16) float att_smem[];
  float* const q = att_smem;
  float* const k = q + BM * (DM + 4);
  float* const v = k + BN * (DM + 4);
  float* const p = v + BN * (DM + 4);
  uint8_t* const cq = (uint8_t*)(p + BM * S::PS);
  uint8_t* const ck = cq + BM;
  const adacgd_attention_inputs& a = g.in;
  Tile t;
  if (!tile_of(a, blockIdx.x, BM, &t)) return;
  const int head = blockIdx.y, kh = head / (a.heads / a.key_heads), dim = a.head_dim;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_counts<BM>(cq, a, t, t.first);
  __syncthreads();
  load_tile<T, DM, BM>(q, a.q, a.q_stride, t.row, head, dim, cq, t.first);
  float top[RM], sum[RM], o[RM][DM / 16];
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    top[r] = NONE;
    sum[r] = 0.f;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) o[r][c] = 0.f;
  }
  const int end = a.causal ? min(t.length, t.first + BM) : t.length;
  for (int j0 = 0; j0 < end; j0 += BN) {
    __syncthreads();
    load_counts<BN>(ck, a, t, j0);
    __syncthreads();
    load_tile<T, DM, BN>(k, a.k, a.k_stride, t.row, kh, dim, ck, j0);
    load_tile<T, DM, BN>(v, a.v, a.v_stride, t.row, kh, dim, ck, j0);
    __syncthreads();
    float s[RM][RN];
    products<DM, RM, RN>(q, k, s);
#pragma unroll
    for (int r = 0; r < RM; ++r) {
      const int i = t.first + ty + 16 * r;
      float m = NONE;
#pragma unroll
      for (int c = 0; c < RN; ++c) {
        const int j = tx + 16 * c;
        const bool sees = ck[j] && (!a.causal || j0 + j <= i);
        s[r][c] = sees ? s[r][c] * a.scale : NONE;
        m = !(m >= s[r][c]) && !(m != m) ? s[r][c] : m;
      }
      m = max16(m);
      const float now = !(top[r] >= m) && !(top[r] != top[r]) ? m : top[r];
      const float base = now == NONE ? 0.f : now;
      const float shrink = ex2((top[r] - base) * LOG2E);
      float add = 0.f;
#pragma unroll
      for (int c = 0; c < RN; ++c) {
        const float e = ex2((s[r][c] - base) * LOG2E);
        p[(ty + 16 * r) * S::PS + tx + 16 * c] = e;
        add += e;
      }
      sum[r] = fmaf(sum[r], shrink, sum16(add));
      top[r] = now;
#pragma unroll
      for (int c = 0; c < DM / 16; ++c) o[r][c] *= shrink;
    }
    __syncthreads();
    accumulate<DM, RM, BN, S::PS, true>(p, v, o);
  }
  float inv[RM];
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    inv[r] = 1.f / sum[r];
    const int i = ty + 16 * r;
    if (g.lse && tx == 0 && t.first + i < t.length)
      g.lse[(long long)head * a.tokens + t.row + t.first + i] = cq[i] ? (float)((double)top[r] + log((double)sum[r])) : NONE;
  }
  store_tile<T, DM, RM>(g.out, g.out_stride, t, t.first, head, dim, cq, inv, o);
}

template <int DM, int BM, int BN> struct BwdSmem {
  static constexpr int PS = BN + 4, FLOATS = 2 * (BM + BN) * (DM + 4) + 2 * BM * PS + 2 * BM;
  static constexpr int BYTES = FLOATS * 4 + BM + BN;
};

// p_ij and ds_ij of a tile into shared memory ([query][key]).  Rows that do not count have lse = +inf, so p = 0, and row_dot = 0.
template <int DM, int BM, int BN>
__device__ __forceinline__ void probabilities(const float* q, const float* k, const float* dout, const float* v, const float* lse, const float* dot,
                                              const uint8_t* cq, const uint8_t* ck, float scale, bool causal, int i0, int j0, float* p, float* ds) {
  constexpr int RM = BM / 16, RN = BN / 16, PS = BN + 4;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float s[RM][RN], d[RM][RN];
  products<DM, RM, RN>(q, k, s);
  products<DM, RM, RN>(dout, v, d);
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    const int i = ty + 16 * r;
#pragma unroll
    for (int c = 0; c < RN; ++c) {
      const int j = tx + 16 * c;
      const bool sees = cq[i] && ck[j] && (!causal || j0 + j <= i0 + i);
      const float e = sees ? ex2(fmaf(s[r][c], scale, -lse[i]) * LOG2E) : 0.f;
      if (p) p[i * PS + j] = e;
      ds[i * PS + j] = sees ? e * (d[r][c] - dot[i]) : 0.f;
    }
  }
}

// dq of a query tile; leaves row_dot.
template <typename T, int DM, int BM, int BN>
__global__ void __launch_bounds__(ATT_CTA) k_attention_dq_any(adacgd_attention_backward_args g) {
  typedef BwdSmem<DM, BM, BN> S;
  constexpr int RM = BM / 16;
  extern __shared__ __align__(16) float att_smem[];
  float* const q = att_smem;
  float* const dout = q + BM * (DM + 4);
  float* const k = dout + BM * (DM + 4);
  float* const v = k + BN * (DM + 4);
  float* const ds = v + BN * (DM + 4);
  float* const lse = ds + 2 * BM * S::PS;
  float* const dot = lse + BM;
  uint8_t* const cq = (uint8_t*)(dot + BM);
  uint8_t* const ck = cq + BM;
  const adacgd_attention_inputs& a = g.in;
  Tile t;
  if (!tile_of(a, blockIdx.x, BM, &t)) return;
  const int head = blockIdx.y, kh = head / (a.heads / a.key_heads), dim = a.head_dim;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_counts<BM>(cq, a, t, t.first);
  __syncthreads();
  load_tile<T, DM, BM>(q, a.q, a.q_stride, t.row, head, dim, cq, t.first);
  load_tile<T, DM, BM>(dout, g.dout, g.dout_stride, t.row, head, dim, cq, t.first);
  __syncthreads();
  for (int i = ty; i < BM; i += 16) {           // sixteen threads a row
    float sum = 0.f;
    const long long row = t.row + t.first + i;
    if (cq[i])
      for (int d = tx; d < dim; d += 16) sum = fmaf(dout[i * (DM + 4) + d], to_f(((const T*)g.out)[row * g.out_stride + (long long)head * dim + d]), sum);
    sum = sum16(sum);
    if (tx == 0) {
      const long long at = (long long)head * a.tokens + row;
      dot[i] = sum;
      lse[i] = cq[i] ? g.lse[at] : INFINITY;
      if (t.first + i < t.length) g.row_dot[at] = sum;
    }
  }
  float o[RM][DM / 16], factor[RM];
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    factor[r] = a.scale;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) o[r][c] = 0.f;
  }
  const int end = a.causal ? min(t.length, t.first + BM) : t.length;
  for (int j0 = 0; j0 < end; j0 += BN) {
    __syncthreads();
    load_counts<BN>(ck, a, t, j0);
    __syncthreads();
    load_tile<T, DM, BN>(k, a.k, a.k_stride, t.row, kh, dim, ck, j0);
    load_tile<T, DM, BN>(v, a.v, a.v_stride, t.row, kh, dim, ck, j0);
    __syncthreads();
    probabilities<DM, BM, BN>(q, k, dout, v, lse, dot, cq, ck, a.scale, a.causal, t.first, j0, nullptr, ds);
    __syncthreads();
    accumulate<DM, RM, BN, S::PS, true>(ds, k, o);
  }
  store_tile<T, DM, RM>(g.dq, g.dq_stride, t, t.first, head, dim, cq, factor, o);
}

// dk and dv of a key tile, over the query heads that share it.
template <typename T, int DM, int BM, int BN>
__global__ void __launch_bounds__(ATT_CTA) k_attention_dkv_any(adacgd_attention_backward_args g) {
  typedef BwdSmem<DM, BM, BN> S;
  constexpr int RN = BN / 16;
  extern __shared__ __align__(16) float att_smem[];
  float* const q = att_smem;
  float* const dout = q + BM * (DM + 4);
  float* const k = dout + BM * (DM + 4);
  float* const v = k + BN * (DM + 4);
  float* const p = v + BN * (DM + 4);
  float* const ds = p + BM * S::PS;
  float* const lse = ds + BM * S::PS;
  float* const dot = lse + BM;
  uint8_t* const cq = (uint8_t*)(dot + BM);
  uint8_t* const ck = cq + BM;
  const adacgd_attention_inputs& a = g.in;
  Tile t;
  if (!tile_of(a, blockIdx.x, BN, &t)) return;
  const int kh = blockIdx.y, group = a.heads / a.key_heads, dim = a.head_dim;
  load_counts<BN>(ck, a, t, t.first);
  __syncthreads();
  load_tile<T, DM, BN>(k, a.k, a.k_stride, t.row, kh, dim, ck, t.first);
  load_tile<T, DM, BN>(v, a.v, a.v_stride, t.row, kh, dim, ck, t.first);
  float dk[RN][DM / 16], dv[RN][DM / 16], one[RN], factor[RN];
#pragma unroll
  for (int r = 0; r < RN; ++r) {
    one[r] = 1.f;
    factor[r] = a.scale;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) dk[r][c] = dv[r][c] = 0.f;
  }
  const int begin = a.causal ? t.first / BM * BM : 0;
  for (int h = 0; h < group; ++h) {
    const int head = kh * group + h;
    for (int i0 = begin; i0 < t.length; i0 += BM) {
      __syncthreads();
      load_counts<BM>(cq, a, t, i0);
      __syncthreads();
      load_tile<T, DM, BM>(q, a.q, a.q_stride, t.row, head, dim, cq, i0);
      load_tile<T, DM, BM>(dout, g.dout, g.dout_stride, t.row, head, dim, cq, i0);
      for (int i = threadIdx.x; i < BM; i += ATT_CTA) {
        const long long at = (long long)head * a.tokens + t.row + i0 + i;
        lse[i] = cq[i] ? g.lse[at] : INFINITY;
        dot[i] = cq[i] ? g.row_dot[at] : 0.f;
      }
      __syncthreads();
      probabilities<DM, BM, BN>(q, k, dout, v, lse, dot, cq, ck, a.scale, a.causal, i0, t.first, p, ds);
      __syncthreads();
      accumulate<DM, RN, BM, S::PS, false>(p, dout, dv);
      accumulate<DM, RN, BM, S::PS, false>(ds, q, dk);
    }
  }
  store_tile<T, DM, RN>(g.dk, g.dk_stride, t, t.first, kh, dim, ck, factor, dk);
  store_tile<T, DM, RN>(g.dv, g.dv_stride, t, t.first, kh, dim, ck, one, dv);
}

template <typename T, int DM, int BM, int BN>
int fwd_any(const adacgd_attention_args& g, const Where& at) {
  static std::atomic<int> table[TRAIN_DEVICES];
  constexpr int BYTES = FwdSmem<DM, BM, BN>::BYTES;
  auto kern = k_attention_any<T, DM, BM, BN>;
  if (resident_ctas(kern, table, at.device, ATT_CTA, BYTES) < 1) return -1;
  kern<<<dim3((unsigned)tile_slots(g.in, BM), (unsigned)g.in.heads), ATT_CTA, BYTES, at.stream>>>(g);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}
template <typename T, int DM, int BM, int BN>
int bwd_any(const adacgd_attention_backward_args& g, const Where& at) {
  static std::atomic<int> table[2][TRAIN_DEVICES];
  constexpr int BYTES = BwdSmem<DM, BM, BN>::BYTES;
  auto dq = k_attention_dq_any<T, DM, BM, BN>;
  auto dkv = k_attention_dkv_any<T, DM, BM, BN>;
  if (resident_ctas(dq, table[0], at.device, ATT_CTA, BYTES) < 1 || resident_ctas(dkv, table[1], at.device, ATT_CTA, BYTES) < 1) return -1;
  dq<<<dim3((unsigned)tile_slots(g.in, BM), (unsigned)g.in.heads), ATT_CTA, BYTES, at.stream>>>(g);
  if (cudaGetLastError() != cudaSuccess) return -1;
  dkv<<<dim3((unsigned)tile_slots(g.in, BN), (unsigned)g.in.key_heads), ATT_CTA, BYTES, at.stream>>>(g);
  return cudaGetLastError() == cudaSuccess ? 2 : -1;
}

template <typename T> int fwd_t(const adacgd_attention_args& g, const Where& at) {
  if (g.in.head_dim <= 64) return fwd_any<T, 64, 64, 64>(g, at);
  if (g.in.head_dim <= 128) return fwd_any<T, 128, 64, 64>(g, at);
  return fwd_any<T, 256, 64, 32>(g, at);
}
template <typename T> int bwd_t(const adacgd_attention_backward_args& g, const Where& at) {
  if (g.in.head_dim <= 64) return bwd_any<T, 64, 64, 64>(g, at);
  if (g.in.head_dim <= 128) return bwd_any<T, 128, 64, 32>(g, at);
  return bwd_any<T, 256, 32, 32>(g, at);
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_attention(const adacgd_attention_args& a, const Where& at) {
  const int n = launch_attention_mma(a, at);
  if (n) return n;
  BY_TYPE(a.in.dtype, (fwd_t<T>(a, at)))
}

int launch_attention_backward(const adacgd_attention_backward_args& a, const Where& at) {
  const int n = launch_attention_backward_mma(a, at);
  if (n) return n;
  BY_TYPE(a.in.dtype, (bwd_t<T>(a, at)))
}

}  // namespace adacgd
