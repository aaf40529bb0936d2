// Attention and its backward pass for the 16-bit types on the tensor cores: heads of up to 128 elements (a multiple of 8), rows on
// 16 bytes.  Bound by the products and, beside them, by the exponentials (16 a clock and SM, where a product of 128 x 128 x 128 takes
// 512 clocks and its scores' exponentials 1024).
//
// Common to the three kernels.  A CTA holds one tile of rows and walks over the tiles it meets; tiles are 128 rows of 64 or
// 128 columns in shared memory, rows of 128 bytes, swizzled, brought by one warp's tensor copies, which fill columns behind a
// head's end with zeros.  One thread issues the products; their operands are tiles and, for probabilities and ds, tensor memory, where
// the row warps put them in place of the scores they were made from: forward eight of them, a thread a row, backward sixteen, four threads a row.
// A row that does not count, or belongs to another sequence, must not reach a sum over rows even as 0 x NaN: where a tile that is summed over has
// such rows, the copying warp sets them to zero before it hands the tile on.
// p and ds are rounded to the matrices' type, as an operand of a product is of the other one's type; the errors of the results are 1.2 to 1.45 times
// those of a computation in 32 bits that rounds them alone.
//
// The backward pass is two kernels that each compute the scores again, seven products for the five that are needed: every sum stays in one
// CTA's tensor memory, without atomics, and dq needs no binary32 array.
#include <type_traits>

#include "adacgd_tcgen05.cuh"
#include "adacgd_train_attention.cuh"

namespace adacgd {
namespace {

constexpr int TILE = 128, HALF = TILE * 128;       // rows of a tile; bytes of 64 of its columns
constexpr int FWD_CTA = 384, FWD_ROWS = 8;         // threads; warps that hold rows, before the product and the copying warp
constexpr int BWD_CTA = 576, BWD_ROWS = 16;
constexpr int MOST_SMEM = 227 * 1024;              // a CTA's shared memory

struct Maps {
  CUtensorMap q, k, v, dout;
};

// ---- the copying warp ----
template <int DP> __device__ __forceinline__ void copy_tile(u32 dst, const CUtensorMap* map, int head, long long row, u32 bar) {
#pragma unroll
  for (int h = 0; h < DP / 64; ++h) tma_load_3d(dst + h * HALF, map, 64 * h, head, (int)row, bar);
}
// Which of the rows first .. first + 127 count: read a tile ahead (a byte of the mask a lane and 32 rows), put together where they are needed.
struct Counts {
  bool on[4];
};
__device__ __forceinline__ void read_counts(const adacgd_attention_inputs& a, const Tile& t, int first, Counts& c) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int i = first + 32 * w + (threadIdx.x & 31);
    c.on[w] = i >= 0 && i < t.length && (!a.mask || a.mask[t.row + i]);
  }
}
__device__ __forceinline__ void words_of(const Counts& c, u32 (&words)[4]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) words[w] = __ballot_sync(0xffffffffu, c.on[w]);
}
__device__ __forceinline__ bool all_count(const u32 (&words)[4]) { return (words[0] & words[1] & words[2] & words[3]) == 0xffffffffu; }

// Brings a tile and hands it on by `full`.  Rows whose bit is not set are zeroed where `clean`: then the copy arrives at `aside` first.
template <int DP>
__device__ __forceinline__ bool bring(u32 dst, const CUtensorMap* map, int head, long long row, const u32 (&words)[4], bool clean, u32 full, u32 aside,
                                      u32& aside_parity, volatile int* dead) {
  const int lane = threadIdx.x & 31;
  const bool fix = clean && !all_count(words);
  if (lane == 0) {
    mbar_expect(fix ? aside : full, DP * 256);
    copy_tile<DP>(dst, map, head, row, fix ? aside : full);
  }
  if (!fix) return true;
  if (!mbar_wait(aside, aside_parity, dead)) return false;
  aside_parity ^= 1;
#pragma unroll 1
  for (int r = lane >> 3; r < TILE; r += 4) {
    if (words[r >> 5] >> (r & 31) & 1) continue;
#pragma unroll
    for (int h = 0; h < DP / 64; ++h)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + h * HALF + r * 128 + (lane & 7) * 16), "r"(0) : "memory");
  }
  fence_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(full);
  return true;
}

// After a wait that ran out: the copies under way must have ended before the CTA's memory goes to another.
__device__ __forceinline__ void settle(u32 bar, u32 parity) { mbar_wait(bar, parity, nullptr); }

// The tiles of the item's sequence between its first and its last token that counts: [begin, end), none if nothing counts.  A padded
// batch has nothing but padding in the others.  By the whole CTA.  The scratch lies where no tensor copy arrives: nothing orders these accesses
// before a copy's writes.
__device__ __forceinline__ void trim(const adacgd_attention_inputs& a, const Tile& t, int* scratch, int* begin, int* end) {
  *begin = 0;
  *end = (t.length + TILE - 1) / TILE;
  if (!a.mask) return;
  if (threadIdx.x == 0) {
    scratch[0] = t.length;
    scratch[1] = 0;
  }
  __syncthreads();
  int lo = t.length, hi = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < t.length; i += blockDim.x)
    if (a.mask[t.row + i]) {
      lo = min(lo, i);
      hi = i + 1;
    }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((threadIdx.x & 31) == 0) {
    atomicMin(scratch, lo);
    atomicMax(scratch + 1, hi);
  }
  __syncthreads();
  *begin = scratch[0] / TILE;
  *end = scratch[1] ? (scratch[1] + TILE - 1) / TILE : *begin;
  __syncthreads();
}
// Zeros in a row.
__device__ __forceinline__ void zero_row(void* base, long long stride, long long row, int head, int dim) {
  uint4* const to = reinterpret_cast<uint4*>((char*)base + (row * stride + (long long)head * dim) * 2);
  for (int d = 0; d < dim / 8; ++d) to[d] = make_uint4(0, 0, 0, 0);
}

// ---- the product warp ----
// d = a b^T over 16 * STEPS columns of both tiles.
template <bool BF16, int DP> __device__ __forceinline__ void product_nt(u32 leader, u32 d, u32 a, u32 b) {
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) {
    const u32 off = (k / 4) * HALF + (k % 4) * 32;
    mma_ss(leader, d, operand(a + off, 16), operand(b + off, 16), product_of(BF16, TILE, false), k > 0);
  }
}
// d [128 x DP] += p tile, p in tensor memory: 16 rows of the tile a step.  p was put in the place of 128 columns of scores, by parts of
// them: 16 PER numbers in the first half of a part's columns.
template <bool BF16, int DP, int PER> __device__ __forceinline__ void product_pn(u32 leader, u32 d, u32 p, u32 tile, bool add) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    mma_ts(leader, d, p + (k / PER) * PER * 16 + (k % PER) * 8, operand(tile + k * 2048, HALF), product_of(BF16, DP, true), add || k > 0);
}

// ---- rows of results ----
// Stores factor * (32 columns of tensor memory) as elements c .. c + 31 of a row of `dim`, or zeros.
template <bool BF16>
__device__ __forceinline__ void store_cols(void* base, long long stride, long long row, int head, int dim, int c, u32 tmem, float factor, bool inside, bool zero) {
  char* const to = (char*)base + (row * stride + (long long)head * dim) * 2;
  u32 r[32];
  __syncwarp();
  tmem_ld32(tmem + c, r);
  tmem_wait_ld();
  tmem_hold(r);
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    if (!inside || c + j >= dim) continue;
    u32 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = zero ? 0u : pack2<BF16>(__uint_as_float(r[j + 2 * i]) * factor, __uint_as_float(r[j + 2 * i + 1]) * factor);
    *reinterpret_cast<uint4*>(to + (c + j) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// What a kernel leaves whose wait has run out: NaN in either type.
__device__ __forceinline__ void poison_row(void* base, long long stride, long long row, int head, int dim) {
  unsigned short* const to = (unsigned short*)base + row * stride + (long long)head * dim;
  for (int d = 0; d < dim; ++d) to[d] = 0x7fff;
}

// 2^x of a pair on the multiplying units: x = n + f with n the nearest integer, 2^f by the polynomial of degree 4 with the least relative error on
// [-1/2, 1/2] (2.7e-6, computed by exchange; its mean is 4e-8), 2^n as a factor so that NaN stays NaN.  x is held at -127, where the factor's bits
// come out as those of 0: what is below 2^-126.5 is exactly 0, as the hardware's function has it below 2^-126.
__device__ __forceinline__ float at_least(float x, float low) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(low));
  return r;
}
__device__ __forceinline__ F2 exp2_by_products(float x0, float x1) {
  const float big = 12582912.f;                                // 1.5 2^23: adding it rounds to an integer, in the low bits of the sum
  const F2 x = f2(at_least(x0, -127.f), at_least(x1, -127.f)), t = add2(x, f2(big, big)), n = add2(t, f2(-big, -big));
  const F2 f = fma2(n, f2(-1.f, -1.f), x);
  F2 y = fma2(f2(0x1.3997d6p-7f, 0x1.3997d6p-7f), f, f2(0x1.ca1440p-5f, 0x1.ca1440p-5f));
  y = fma2(y, f, f2(0x1.ec06dap-3f, 0x1.ec06dap-3f));
  y = fma2(y, f, f2(0x1.62e0dcp-1f, 0x1.62e0dcp-1f));
  y = fma2(y, f, f2(0x1.ffffe8p-1f, 0x1.ffffe8p-1f));
  float t0, t1;
  split(t, t0, t1);
  return mul2(y, f2(__uint_as_float((__float_as_uint(t0) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(t1) << 23) + 0x3f800000u)));
}
__device__ __forceinline__ F2 exp2_pair(F2 x) {
  float a, b;
  split(x, a, b);
  return f2(ex2(a), ex2(b));
}
// The pair with this number of a row: the hardware's function gives four a clock and scheduler, half of the products' pace, so in the
// forward pass three pairs of eight take the other way (453 -> 443 us; backward there was nothing in it).
template <bool MIXED> __device__ __forceinline__ F2 exp2_pair(F2 x, int number) {
  const int i = MIXED ? number & 7 : 0;
  if (i != 1 && i != 4 && i != 6) return exp2_pair(x);
  float a, b;
  split(x, a, b);
  return exp2_by_products(a, b);
}

typedef std::integral_constant<bool, false> No;
typedef std::integral_constant<bool, true> Yes;

__device__ __forceinline__ u32 low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }

// --------------------------------------------------------------------------
// forward
// --------------------------------------------------------------------------
// A CTA takes two tiles of queries of a head, A and B.  While the products of one run, four warps turn the scores of the other into
// probabilities: S = Q K^T, the row's maximum, p = 2^(c s - c max) in S's place, O += p V.  The maximum that p is taken against is
// moved only when it has grown by more than 2^8, so O, which stays in tensor memory, is hardly ever rescaled; p is at most 256 then, and the
// division by the sum at the end takes it out.  (Rows of other sequences and rows that do not count have no say in that: a rescaling changes roundings.)  binary16 has few numbers below 1: there p is taken 2^7 times larger, at most 2^15.
template <int DP> struct FwdLayout {
  static constexpr int BYTES = DP * 256, STAGES = DP == 128 ? 5 : 8, RING = 2 * BYTES, BARS = RING + STAGES * BYTES;
  static constexpr int TOTAL = BARS + 256, SCRATCH = TOTAL - 8;
  static_assert(64 + 16 * STAGES + 8 <= SCRATCH - BARS && TOTAL <= MOST_SMEM, "barriers, trim's scratch, the CTA's shared memory");
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(FWD_CTA, 1) k_attention_mma(const __grid_constant__ Maps maps, adacgd_attention_args g) {
  typedef FwdLayout<DP> L;
  extern __shared__ __align__(1024) unsigned char mma_smem[];
  const adacgd_attention_inputs& a = g.in;
  const int head = (int)(blockIdx.x % a.heads);
  Tile t;
  if (!tile_of(a, gridDim.x / a.heads - 1 - blockIdx.x / a.heads, 2 * TILE, &t)) return;   // long ones first where causal
  const u32 base = smem_addr(mma_smem), bars = base + L::BARS;
  const u32 q_full = bars, aside = bars + 8, s_full = bars + 16, p_full = bars + 32, o_full = bars + 48, full = bars + 64, empty = full + 8 * L::STAGES;
  u32* const tmem_at = reinterpret_cast<u32*>(mma_smem + L::BARS + 64 + 16 * L::STAGES);
  volatile int* const dead = reinterpret_cast<int*>(tmem_at + 1);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int kh = head / (a.heads / a.key_heads);
  int begin, end, count[2];                                    // tiles of keys; how many of them A and B meet
  trim(a, t, reinterpret_cast<int*>(mma_smem + L::SCRATCH), &begin, &end);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int mine = t.first / TILE + x;                       // without a row that counts: none
    count[x] = mine < begin || mine >= end ? 0 : (a.causal ? mine + 1 : end) - begin;
  }
  const int n = max(count[0], count[1]), last = a.causal ? begin + n : end;   // the walk goes from the last tile down to the first
  if (n == 0) {
    const int i = t.first + (int)threadIdx.x;
    if (threadIdx.x < 2 * TILE && i < t.length) {
      zero_row(g.out, g.out_stride, t.row + i, head, a.head_dim);
      if (g.lse) g.lse[(long long)head * a.tokens + t.row + i] = -INFINITY;
    }
    return;
  }
  if (warp == FWD_ROWS + 1 && lane == 0) {
    mbar_init(q_full, 1);
    mbar_init(aside, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full + 8 * x, 1);
      mbar_init(p_full + 8 * x, 128);
      mbar_init(o_full + 8 * x, 1);
    }
    for (int i = 0; i < L::STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    *dead = 0;
    mbar_init_fence();
    mbar_expect(q_full, ((count[0] ? 1 : 0) + (count[1] ? 1 : 0)) * L::BYTES);   // the first copies start before the CTA's warps have met
    if (count[0]) copy_tile<DP>(base, &maps.q, head, t.row + t.first, q_full);
    if (count[1]) copy_tile<DP>(base + L::BYTES, &maps.q, head, t.row + t.first + TILE, q_full);
  }
  if (warp == FWD_ROWS) tmem_alloc(smem_addr(tmem_at), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = __shfl_sync(0xffffffffu, *tmem_at, 0);
  // A row's 128 scores are held at once: of the CTA's 384 x 168 registers the row warps get 208 each, the others 88.
  if (warp >= FWD_ROWS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == FWD_ROWS + 1) {
      u32 side = 0, words[4];
      Counts ahead;
      read_counts(a, t, (last - 1) * TILE, ahead);
      int i = 0;
      bool ok = true;
      for (; ok && i < 2 * n; ++i) {                             // tiles of keys and values in turn, the last ones first
        const int st = i % L::STAGES, first = (last - 1 - i / 2) * TILE;
        if (i >= L::STAGES && !mbar_wait(empty + 8 * st, (i / L::STAGES - 1) & 1, dead)) break;
        if (i & 1) {                                           // only values are summed over
          words_of(ahead, words);
          read_counts(a, t, first - TILE, ahead);
        }
        ok = bring<DP>(base + L::RING + st * L::BYTES, i & 1 ? &maps.v : &maps.k, kh, t.row + first, words, i & 1, full + 8 * st, aside, side, dead);
      }
      if (*dead) {
        settle(q_full, 0);
        for (int b = max(0, i - L::STAGES); b < i; ++b) settle(full + 8 * (b % L::STAGES), (b / L::STAGES) & 1);
      }
    } else if (warp == FWD_ROWS) {
      {
      const u32 leader = elect_leader();
        bool ok = mbar_wait_warp(q_full, 0, dead);
        for (int j = 0; ok && j <= n; ++j) {
          const int ik = 2 * j, iv = 2 * j - 1, sk = ik % L::STAGES, sv = iv % L::STAGES;
          if (j < n && !(ok = mbar_wait_warp(full + 8 * sk, (ik / L::STAGES) & 1, dead))) break;
          if (j > 0 && !(ok = mbar_wait_warp(full + 8 * sv, (iv / L::STAGES) & 1, dead))) break;
          for (int x = 0; ok && x < 2; ++x) {
            const int u = j - (n - count[x]);                    // the step as x counts
            if (u < 0 || count[x] == 0) continue;
            const u32 s = tmem + x * TILE, o = tmem + 2 * TILE + x * DP;
            if (u > 0) {
              if (!(ok = mbar_wait_warp(p_full + 8 * x, (u - 1) & 1, dead))) break;
              tc_fence_after();
              product_pn<BF16, DP, 8>(leader, o, s, base + L::RING + sv * L::BYTES, u > 1);
            }
            if (j < n) {
              tc_fence_after();
              product_nt<BF16, DP>(leader, s, base + x * L::BYTES, base + L::RING + sk * L::BYTES);
              mma_commit(leader, s_full + 8 * x);
            } else {
              mma_commit(leader, o_full + 8 * x);
            }
          }
          if (!ok) break;
          if (j < n) mma_commit(leader, empty + 8 * sk);
          if (j > 0) mma_commit(leader, empty + 8 * sv);
        }
        if (*dead) {
          mma_commit(leader, aside);                                     // nobody else uses it any more, or its wait has run out too
          settle(aside, 0);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int x = warp >> 2, i = t.first + x * TILE + (warp & 3) * 32 + lane;
    const u32 lanes = (u32)(warp & 3) << 21, s_at = tmem + x * TILE + lanes, o_at = tmem + 2 * TILE + x * DP + lanes;
    const float c = a.scale * LOG2E;
    const bool inside = i < t.length, on = inside && (!a.mask || a.mask[t.row + i]);
    float top = -INFINITY, sum = 0.f;
    bool ok = true;
    // A and B end with the same tile; where causal, A's walk begins a tile later
    const int top_tile = begin + count[x];
    Counts ahead;
    if (count[x]) read_counts(a, t, (top_tile - 1) * TILE, ahead);
    for (int u = 0; u < count[x]; ++u) {
      const int j0 = (top_tile - 1 - u) * TILE;
      u32 words[4];
      words_of(ahead, words);
      if (u + 1 < count[x]) read_counts(a, t, j0 - TILE, ahead);
      const bool edge = a.causal && j0 + TILE > t.first + x * TILE, mask = edge || !all_count(words);
      if (edge)
#pragma unroll
        for (int w = 0; w < 4; ++w) words[w] &= low_bits(i + 1 - j0 - 32 * w);
      if (!(ok = mbar_wait(s_full + 8 * x, u & 1, dead))) break;
      tc_fence_after();
      u32 s[4][32];
#pragma unroll
      for (int w = 0; w < 4; ++w) tmem_ld32(s_at + 32 * w, s[w]);
      tmem_wait_ld();
#pragma unroll
      for (int w = 0; w < 4; ++w) tmem_hold(s[w]);
      if (mask)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int k = 0; k < 32; ++k) s[w][k] = words[w] >> k & 1 ? s[w][k] : 0xff800000u;
      float m[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        m[w] = __uint_as_float(s[w][0]);
#pragma unroll
        for (int k = 1; k < 32; ++k) m[w] = fmaxf(m[w], __uint_as_float(s[w][k]));
      }
      const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
      if (u == 0) {
        top = most;
      } else if (__any_sync(0xffffffffu, on && (most - top) * c > 8.f)) {   // only rows that count decide; -inf - -inf is NaN: no
        const float now = fmaxf(top, most), f = now == -INFINITY ? 1.f : ex2((top - now) * c);
        sum *= f;
        top = now;
#pragma unroll
        for (int d = 0; d < DP; d += 32) {
          u32 o[32];
          tmem_ld32(o_at + d, o);
          tmem_wait_ld();
          tmem_hold(o);
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
          tmem_st32(o_at + d, o);
        }
      }
      const float low = (top == -INFINITY ? 0.f : -top * c) + (BF16 ? 0.f : 7.f);
      const F2 c2 = f2(c, c), low2 = f2(low, low);
      F2 sum2 = f2(sum, 0.f);
      auto shares = [&](auto mixed) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          u32 p[16];
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const F2 y = exp2_pair<decltype(mixed)::value>(fma2(f2(__uint_as_float(s[w][k]), __uint_as_float(s[w][k + 1])), c2, low2), k / 2);
            float y0, y1;
            split(y, y0, y1);
            sum2 = add2(sum2, y);
            p[k / 2] = pack2<BF16>(y0, y1);
          }
          tmem_st16(s_at + 16 * w, p);
        }
      };
      if (mask) shares(No{});                                  // what is hidden has to be exactly zero
      else shares(Yes{});
      float e0, e1;
      split(sum2, e0, e1);
      sum = e0 + e1;
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(p_full + 8 * x);
    }
    if (count[x] == 0 && i < t.length) {
      zero_row(g.out, g.out_stride, t.row + i, head, a.head_dim);
      if (g.lse) g.lse[(long long)head * a.tokens + t.row + i] = -INFINITY;
    }
    if (count[x] && ok && mbar_wait(o_full + 8 * x, 0, dead)) {
      tc_fence_after();
#pragma unroll
      for (int d = 0; d < DP; d += 32) store_cols<BF16>(g.out, g.out_stride, t.row + i, head, a.head_dim, d, o_at, 1.f / sum, inside, !on);
      if (inside && g.lse) g.lse[(long long)head * a.tokens + t.row + i] = on ? fmaf(top, a.scale, logf(BF16 ? sum : sum * 0.0078125f)) : -INFINITY;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == FWD_ROWS) tmem_free(tmem, 512);
  if (*dead && threadIdx.x < 2 * TILE && t.first + (int)threadIdx.x < t.length)
    poison_row(g.out, g.out_stride, t.row + t.first + threadIdx.x, head, a.head_dim);
}

// --------------------------------------------------------------------------
// backward: the range of ds
// --------------------------------------------------------------------------
// bfloat16 holds ds as it is.  binary16 would lose what is below 2^-14, and gradients are often that small, so there ds is multiplied by a power
// of two that brings the largest one possible, |dout_i| (|v_j| + |out_i|) <= 2 |dout_i| max|v|, below 2^14.  For dq that is a factor a row: the
// row's own |dout_i| and the largest |v| of its sequence and key head.  dk sums over the rows, so there it is the largest |dout| of the sequence and of the
// heads that share the key head.  What other sequences and key heads hold has no part in it.
// This kernel takes the rows' products dout.out, their |dout|^2 and the maxima of a tile, a CTA one tile, key head and part of the heads that share it;
// LPR lanes take a head's row, four rows at a time.  What the others need waits where it is overwritten last:
//   |dout_i|^2 in the row's own columns of dq, read and overwritten by one CTA;
//   the maxima in dv, in the tile's first row and the key head's columns: the parts' ones of |dout|^2, then that of |v|^2.  The kernel of dq joins those of
//   its sequence, and where it has a group's first head it leaves dk's factor in its tile's own first row of dk, read and overwritten by one CTA.
constexpr int RANGE_CTA = 256, RANGE_ROWS = 4;

// Parts of a group of heads: as many as there are heads, and room for their maxima.
__host__ __device__ __forceinline__ int range_parts(const adacgd_attention_inputs& a) {
  const int group = a.heads / a.key_heads, room = a.head_dim / 2 - 1;
  return group < room ? group : room;
}
__device__ __forceinline__ float* range_at(void* base, long long stride, long long row, int kh, int dim) {
  return reinterpret_cast<float*>((char*)base + (row * stride + (long long)kh * dim) * 2);
}

template <int LPR>
__global__ void __launch_bounds__(RANGE_CTA) k_attention_range(adacgd_attention_backward_args g) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const adacgd_attention_inputs& a = g.in;
  constexpr int GROUPS = RANGE_CTA / LPR;
  Tile t;
  if (!tile_of(a, blockIdx.x, TILE, &t)) return;
  const int lane = threadIdx.x % LPR, mine = threadIdx.x / LPR, d = lane * 8, kh = (int)blockIdx.y, part = (int)blockIdx.z, parts = (int)gridDim.z;
  const bool in = d < a.head_dim;
  const int group = a.heads / a.key_heads, h0 = (int)((long long)group * part / parts), heads = (int)((long long)group * (part + 1) / parts) - h0;
  const int rows = min(TILE, t.length - t.first);
  const long long row = t.row + t.first;
  float mo = 0.f, mv = 0.f;
  auto sum = [](float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  for (int i0 = 0; i0 < rows * heads; i0 += GROUPS * RANGE_ROWS) {               // heads of a row lie side by side
    Run<__half> x[RANGE_ROWS], y[RANGE_ROWS];
    int r[RANGE_ROWS], head[RANGE_ROWS];
    bool on[RANGE_ROWS];
#pragma unroll
    for (int u = 0; u < RANGE_ROWS; ++u) {
      const int i = i0 + u * GROUPS + mine;
      r[u] = i / heads;
      head[u] = kh * group + h0 + i - r[u] * heads;
      on[u] = r[u] < rows && (!a.mask || a.mask[row + r[u]]);
      if (on[u] && in) {
        x[u] = load_run((const __half*)g.dout + (row + r[u]) * g.dout_stride + (long long)head[u] * a.head_dim + d);
        y[u] = load_run((const __half*)g.out + (row + r[u]) * g.out_stride + (long long)head[u] * a.head_dim + d);
      }
    }
#pragma unroll
    for (int u = 0; u < RANGE_ROWS; ++u) {
      float p[8], q[8], dot = 0.f, sq = 0.f;
      if (on[u] && in) {
        unpack(x[u], p);
        unpack(y[u], q);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          dot = fmaf(p[k], q[k], dot);
          sq = fmaf(p[k], p[k], sq);
        }
      }
      dot = sum(dot);
      sq = sum(sq);
      mo = fmaxf(mo, sq);
      if (lane == 0 && r[u] < rows) g.row_dot[(long long)head[u] * a.tokens + row + r[u]] = dot;
      if (lane == 0 && on[u]) *range_at(g.dq, g.dq_stride, row + r[u], head[u], a.head_dim) = sq;
    }
  }
  if (part == 0) {
#pragma unroll 4
    for (int r = mine; r < (rows + GROUPS - 1) / GROUPS * GROUPS; r += GROUPS) {
      float v[8], sq = 0.f;
      if (in && r < rows && (!a.mask || a.mask[row + r])) {
        unpack(load_run((const __half*)a.v + (row + r) * a.v_stride + (long long)kh * a.head_dim + d), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sq = fmaf(v[k], v[k], sq);
      }
      mv = fmaxf(mv, sum(sq));
    }
  }
  __shared__ float most[2][GROUPS];
  if (lane == 0) {
    most[0][mine] = mo;
    most[1][mine] = mv;
  }
  __syncthreads();
  if (threadIdx.x < (part == 0 ? 2 : 1)) {
    float m = 0.f;
    for (int i = 0; i < GROUPS; ++i) m = fmaxf(m, most[threadIdx.x][i]);
    __stcg(range_at(g.dv, g.dv_stride, row, kh, a.head_dim) + (threadIdx.x ? parts : part), m);
  }
}

// The power of two, of the squares of the largest |dout| and |v|: 2 |dout| |v| is at least 2^(half the exponent of 4 dout2 v2, rounded down).  The squares
// are in [2^-48, 2^40] or 0; 4.01 makes up for the roundings.
__device__ __forceinline__ float range_of(float dout2, float v2) {
  const float square = 4.01f * dout2 * v2;
  if (!(square > 0.f) || isinf(square)) return 1.f;
  const int half = ((__float_as_int(square) >> 23) - 127) >> 1;
  return __int_as_float((127 + min(13 - half, 60)) << 23);
}
// The largest of numbers [from, to) of the sequence's tiles begin .. end - 1: by a warp.
__device__ __forceinline__ float join_range(const adacgd_attention_backward_args& g, const Tile& t, int kh, int begin, int end, int from, int to) {
  float m = 0.f;
#pragma unroll 2
  for (int k = begin + (int)(threadIdx.x & 31); k < end; k += 32) {
    const float* const at = range_at(g.dv, g.dv_stride, t.row + (long long)k * TILE, kh, g.in.head_dim);
#pragma unroll 4
    for (int i = from; i < to; ++i) m = fmaxf(m, __ldcg(at + i));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

// --------------------------------------------------------------------------
// backward: dq
// --------------------------------------------------------------------------
// A CTA takes a tile of queries and walks over tiles of keys: S = Q K^T, dP = dO V^T, ds = p (dP - row_dot) in S's place, dQ += ds K.
// S has two places, so that the next one is there while this one's exponentials run; dP is free again once ds has been made.
// Sixteen warps share a tile by quarters of its columns: eight with twice the columns each left a scheduler two warps, whose chains of
// conversions and exponentials nothing filled (4600 clocks a step; 1536 of products).
template <int DP> struct DqLayout {
  static constexpr int BYTES = DP * 256, KS = DP == 128 ? 3 : 4, VS = DP == 128 ? 2 : 4, RING = 2 * BYTES;
  static constexpr int PART = RING + (KS + VS) * BYTES, BARS = PART + 4 * TILE * 4, TOTAL = BARS + 256, SCRATCH = TOTAL - 8;
  static_assert(64 + 16 * (KS + VS) + 8 <= SCRATCH - BARS && TOTAL <= MOST_SMEM, "barriers, trim's scratch, the CTA's shared memory");
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(BWD_CTA, 1) k_attention_dq_mma(const __grid_constant__ Maps maps, adacgd_attention_backward_args g) {
  typedef DqLayout<DP> L;
  extern __shared__ __align__(1024) unsigned char mma_smem[];
  const adacgd_attention_inputs& a = g.in;
  const int head = (int)(blockIdx.x % a.heads);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Tile t;
  if (!tile_of(a, gridDim.x / a.heads - 1 - blockIdx.x / a.heads, TILE, &t)) {
    if (!BF16) asm volatile("griddepcontrol.wait;" ::: "memory");   // this kernel ends after the one before it, whatever there is to do
    return;
  }
  int begin, end;                                              // tiles of keys
  trim(a, t, reinterpret_cast<int*>(mma_smem + L::SCRATCH), &begin, &end);
  if (t.first / TILE < begin || t.first / TILE >= end) {        // no row that counts
    const int i = t.first + (int)threadIdx.x;
    if (threadIdx.x < TILE && i < t.length) {
      zero_row(g.dq, g.dq_stride, t.row + i, head, a.head_dim);
      if (BF16) g.row_dot[(long long)head * a.tokens + t.row + i] = 0.f;
    }
    if (!BF16) asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  const int last = a.causal ? t.first / TILE + 1 : end, n = last - begin;
  const u32 base = smem_addr(mma_smem), bars = base + L::BARS;
  const u32 q_full = bars, aside = bars + 8, s_full = bars + 16, dp_full = bars + 32, ds_full = bars + 40, dq_full = bars + 48, k_full = bars + 64,
            k_empty = k_full + 8 * L::KS, v_full = k_empty + 8 * L::KS, v_empty = v_full + 8 * L::VS;
  u32* const tmem_at = reinterpret_cast<u32*>(mma_smem + L::BARS + 64 + 16 * (L::KS + L::VS));
  volatile int* const dead = reinterpret_cast<int*>(tmem_at + 1);
  float* const part = reinterpret_cast<float*>(mma_smem + L::PART);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (warp == BWD_ROWS + 1 && lane == 0) {
    mbar_init(q_full, 1);
    mbar_init(aside, 1);
    mbar_init(s_full, 1);
    mbar_init(s_full + 8, 1);
    mbar_init(dp_full, 1);
    mbar_init(ds_full, 32 * BWD_ROWS);
    mbar_init(dq_full, 1);
    for (int i = 0; i < L::KS; ++i) {
      mbar_init(k_full + 8 * i, 1);
      mbar_init(k_empty + 8 * i, 1);
    }
    for (int i = 0; i < L::VS; ++i) {
      mbar_init(v_full + 8 * i, 1);
      mbar_init(v_empty + 8 * i, 1);
    }
    *dead = 0;
    mbar_init_fence();
    mbar_expect(q_full, 2 * L::BYTES);                         // the first copies start before the CTA's warps have met
    copy_tile<DP>(base, &maps.q, head, t.row + t.first, q_full);
    copy_tile<DP>(base + L::BYTES, &maps.dout, head, t.row + t.first, q_full);
  }
  if (warp == BWD_ROWS) tmem_alloc(smem_addr(tmem_at), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = __shfl_sync(0xffffffffu, *tmem_at, 0), dp_at = tmem + 2 * TILE, dq_at = tmem + 3 * TILE;
  const u32 q_tile = base, do_tile = base + L::BYTES, k_tiles = base + L::RING, v_tiles = k_tiles + L::KS * L::BYTES;
  const int kh = head / (a.heads / a.key_heads);
  if (warp == BWD_ROWS + 1) {
    u32 side = 0, words[4];
    Counts ahead;
    read_counts(a, t, (last - 1) * TILE, ahead);
    int nk = 0, nv = 0;
    for (int j = 0; j < n; ++j) {
      const int first = (last - 1 - j) * TILE, sk = j % L::KS, sv = j % L::VS;
      words_of(ahead, words);
      read_counts(a, t, first - TILE, ahead);
      if (j >= L::KS && !mbar_wait(k_empty + 8 * sk, (j / L::KS - 1) & 1, dead)) break;
      ++nk;
      if (!bring<DP>(k_tiles + sk * L::BYTES, &maps.k, kh, t.row + first, words, true, k_full + 8 * sk, aside, side, dead)) break;
      if (j >= L::VS && !mbar_wait(v_empty + 8 * sv, (j / L::VS - 1) & 1, dead)) break;
      ++nv;
      bring<DP>(v_tiles + sv * L::BYTES, &maps.v, kh, t.row + first, words, false, v_full + 8 * sv, aside, side, dead);
    }
    if (!BF16 && head == kh * (a.heads / a.key_heads)) {         // for dk, under the last products
      asm volatile("griddepcontrol.wait;" ::: "memory");
      const int parts = range_parts(a);
      const float all = join_range(g, t, kh, begin, end, 0, parts), v = join_range(g, t, kh, begin, end, parts, parts + 1);
      if (lane == 0) __stcg(range_at(g.dk, g.dk_stride, t.row + t.first, kh, a.head_dim), range_of(all, v));
    }
    if (*dead) {
      settle(q_full, 0);
      for (int b = max(0, nk - L::KS); b < nk; ++b) settle(k_full + 8 * (b % L::KS), (b / L::KS) & 1);
      for (int b = max(0, nv - L::VS); b < nv; ++b) settle(v_full + 8 * (b % L::VS), (b / L::VS) & 1);
    }
  } else if (warp == BWD_ROWS) {
    {
      const u32 leader = elect_leader();
      auto scores = [&](int j) {                               // S of step j
        const int st = j % L::KS;
        if (!mbar_wait_warp(k_full + 8 * st, (j / L::KS) & 1, dead)) return false;
        tc_fence_after();
        product_nt<BF16, DP>(leader, tmem + (j & 1) * TILE, q_tile, k_tiles + st * L::BYTES);
        mma_commit(leader, s_full + 8 * (j & 1));
        return true;
      };
      auto shares = [&](int j) {                               // dP of step j
        const int st = j % L::VS;
        if (!mbar_wait_warp(v_full + 8 * st, (j / L::VS) & 1, dead)) return false;
        tc_fence_after();
        product_nt<BF16, DP>(leader, dp_at, do_tile, v_tiles + st * L::BYTES);
        mma_commit(leader, dp_full);
        mma_commit(leader, v_empty + 8 * st);
        return true;
      };
      bool ok = mbar_wait_warp(q_full, 0, dead) && scores(0) && shares(0) && (n < 2 || scores(1));
      for (int j = 0; ok && j < n; ++j) {
        if (!mbar_wait_warp(ds_full, j & 1, dead)) break;
        tc_fence_after();
        if (j + 1 < n && !shares(j + 1)) break;
        product_pn<BF16, DP, 2>(leader, dq_at, tmem + (j & 1) * TILE, k_tiles + (j % L::KS) * L::BYTES, j > 0);
        mma_commit(leader, k_empty + 8 * (j % L::KS));
        if (j + 1 == n) mma_commit(leader, dq_full);
        if (j + 2 < n && !scores(j + 2)) break;
      }
      if (*dead) {
        mma_commit(leader, aside);
        settle(aside, 0);
      }
    }
  } else {
    const int part_of = warp >> 2, r = (warp & 3) * 32 + lane, i = t.first + r;
    const u32 lanes = (u32)(warp & 3) << 21;
    const bool inside = i < t.length, on = inside && (!a.mask || a.mask[t.row + i]);
    const long long at = (long long)head * a.tokens + t.row + i;
    float dot = 0.f, range = 1.f;
    if (BF16) {
      if (on) {                                                // each quarter of the warps takes 32 of the head's elements
        const __nv_bfloat16* const x = (const __nv_bfloat16*)g.dout + (t.row + i) * g.dout_stride + (long long)head * a.head_dim;
        const __nv_bfloat16* const y = (const __nv_bfloat16*)g.out + (t.row + i) * g.out_stride + (long long)head * a.head_dim;
        for (int d = 32 * part_of; d < min(a.head_dim, 32 * part_of + 32); d += 8) {
          float u[8], v[8];
          unpack(load_run(x + d), u);
          unpack(load_run(y + d), v);
#pragma unroll
          for (int k = 0; k < 8; ++k) dot = fmaf(u[k], v[k], dot);
        }
      }
      part[part_of * TILE + r] = dot;
      asm volatile("bar.sync 1, 512;" ::: "memory");
      dot = (part[r] + part[TILE + r]) + (part[2 * TILE + r] + part[3 * TILE + r]);
      if (part_of == 0 && inside) g.row_dot[at] = dot;
    } else {
      asm volatile("griddepcontrol.wait;" ::: "memory");
      // each number is fetched once a CTA: their addresses lie a row of the matrix apart (by every thread that needs them: 644 against 615 us at 8192 tokens)
      if (on) dot = __ldcg(g.row_dot + at);
      if (part_of == 0) part[r] = on ? __ldcg(range_at(g.dq, g.dq_stride, t.row + i, head, a.head_dim)) : 0.f;
      if (warp == 4) part[TILE + lane] = join_range(g, t, kh, begin, end, range_parts(a), range_parts(a) + 1);
      asm volatile("bar.sync 1, 512;" ::: "memory");
      range = range_of(part[r], part[TILE]);
      dot *= range;
    }
    const float low = on ? -g.lse[at] * LOG2E : -INFINITY, c = a.scale * LOG2E;
    const F2 c2 = f2(c, c), low2 = f2(low, low), dot2 = f2(-dot, -dot), range2 = f2(range, range);
    bool ok = true;
    const int column = 32 * part_of + lane;
    auto counts = [&](int first) { return first + column >= 0 && first + column < t.length && (!a.mask || a.mask[t.row + first + column]); };
    bool ahead = counts((last - 1) * TILE);
    for (int j = 0; j < n; ++j) {
      const int j0 = (last - 1 - j) * TILE;
      const u32 s_at = tmem + (j & 1) * TILE + 32 * part_of + lanes;
      u32 bits = __ballot_sync(0xffffffffu, ahead);
      if (j + 1 < n) ahead = counts(j0 - TILE);
      const bool edge = a.causal && j0 + TILE > t.first, mask = edge || bits != 0xffffffffu;
      if (edge) bits &= low_bits(i + 1 - j0 - 32 * part_of);
      if (!(ok = mbar_wait(s_full + 8 * (j & 1), (j >> 1) & 1, dead))) break;
      tc_fence_after();
      u32 s[32];
      tmem_ld32(s_at, s);
      tmem_wait_ld();
      tmem_hold(s);
      F2 p[16];
#pragma unroll
      for (int k = 0; k < 32; k += 2) p[k / 2] = exp2_pair(fma2(f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, low2));
      if (!(ok = mbar_wait(dp_full, j & 1, dead))) break;
      tc_fence_after();
      tmem_ld32(dp_at + 32 * part_of + lanes, s);
      tmem_wait_ld();
      tmem_hold(s);
      u32 ds[16];
      auto products = [&](auto masked) {
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          float y0, y1;
          const F2 dp = f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1]));
          split(mul2(p[k / 2], BF16 ? add2(dp, dot2) : fma2(dp, range2, dot2)), y0, y1);
          if (decltype(masked)::value) {
            y0 = bits >> k & 1 ? y0 : 0.f;
            y1 = bits >> (k + 1) & 1 ? y1 : 0.f;
          }
          ds[k / 2] = pack2<BF16>(y0, y1);
        }
      };
      if (mask) products(Yes{});
      else products(No{});
      tmem_st16(s_at, ds);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(ds_full);
    }
    if (ok && mbar_wait(dq_full, 0, dead) && 32 * part_of < DP) {
      tc_fence_after();
      store_cols<BF16>(g.dq, g.dq_stride, t.row + i, head, a.head_dim, 32 * part_of, dq_at + lanes, a.scale / range, inside, !on);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == BWD_ROWS) tmem_free(tmem, 512);
  if (*dead && threadIdx.x < TILE && t.first + (int)threadIdx.x < t.length)
    poison_row(g.dq, g.dq_stride, t.row + t.first + threadIdx.x, head, a.head_dim);
}

// --------------------------------------------------------------------------
// backward: dk and dv
// --------------------------------------------------------------------------
// A CTA takes a tile of keys and walks over the tiles of queries, of all the heads that share it: S^T = K Q^T, dP^T = V dO^T, then p^T and ds^T
// side by side in dP's place, dV += p^T dO, dK += ds^T Q.  Transposed, p and ds are operands as they lie in tensor memory, and Q and dO
// serve as they were brought, once by rows and once by columns.  The rows' log sums and products lie in shared memory, where all threads
// read the same ones.  p waits in registers until dP has been read: so the next S is formed as soon as this one has been, under its exponentials, and
// the other three products run under those of the next step.  (p in the place of S, as soon as it is known, held the next S back behind dV: 3310 clocks
// a step, of which the products take 2048.)
template <int DP> struct DkvLayout {
  static constexpr int BYTES = DP * 256, STAGES = DP == 128 ? 5 : 8, RING = 2 * BYTES, STATS = RING + STAGES * BYTES;
  static constexpr int BARS = STATS + 2 * 2 * TILE * 4, TOTAL = BARS + 256, SCRATCH = TOTAL - 8;
  static_assert(56 + 16 * STAGES + 8 <= SCRATCH - BARS && TOTAL <= MOST_SMEM, "barriers, trim's scratch, the CTA's shared memory");
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(BWD_CTA, 1) k_attention_dkv_mma(const __grid_constant__ Maps maps, adacgd_attention_backward_args g) {
  typedef DkvLayout<DP> L;
  extern __shared__ __align__(1024) unsigned char mma_smem[];
  const adacgd_attention_inputs& a = g.in;
  const int kh = (int)(blockIdx.x % a.key_heads), group = a.heads / a.key_heads;
  Tile t;
  if (!tile_of(a, blockIdx.x / a.key_heads, TILE, &t)) {
    asm volatile("griddepcontrol.wait;" ::: "memory");           // this kernel ends after the one before it, whatever there is to do
    return;
  }
  int low_tile, high_tile;                                     // of queries
  trim(a, t, reinterpret_cast<int*>(mma_smem + L::SCRATCH), &low_tile, &high_tile);
  if (t.first / TILE < low_tile || t.first / TILE >= high_tile) {   // no key that counts
    const int i = t.first + (int)threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");           // dv still holds what the kernel before reads
    if (threadIdx.x < TILE && i < t.length) {
      zero_row(g.dk, g.dk_stride, t.row + i, kh, a.head_dim);
      zero_row(g.dv, g.dv_stride, t.row + i, kh, a.head_dim);
    }
    return;
  }
  const u32 base = smem_addr(mma_smem), bars = base + L::BARS;
  const u32 kv_full = bars, aside = bars + 8, s_full = bars + 16, dp_full = bars + 24, s_read = bars + 32, ds_full = bars + 40, end_full = bars + 48,
            full = bars + 56, empty = full + 8 * L::STAGES;
  u32* const tmem_at = reinterpret_cast<u32*>(mma_smem + L::BARS + 56 + 16 * L::STAGES);
  volatile int* const dead = reinterpret_cast<int*>(tmem_at + 1);
  float* const stats = reinterpret_cast<float*>(mma_smem + L::STATS);   // [2 steps][-lse log2 e, -row_dot][128], scaled as p and ds are
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (warp == BWD_ROWS + 1 && lane == 0) {
    mbar_init(kv_full, 1);
    mbar_init(aside, 1);
    mbar_init(s_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(s_read, 32 * BWD_ROWS);
    mbar_init(ds_full, 32 * BWD_ROWS);
    mbar_init(end_full, 1);
    for (int i = 0; i < L::STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    *dead = 0;
    mbar_init_fence();
    mbar_expect(kv_full, 2 * L::BYTES);                        // the first copies start before the CTA's warps have met
    copy_tile<DP>(base, &maps.k, kh, t.row + t.first, kv_full);
    copy_tile<DP>(base + L::BYTES, &maps.v, kh, t.row + t.first, kv_full);
  }
  if (warp == BWD_ROWS) tmem_alloc(smem_addr(tmem_at), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const u32 tmem = __shfl_sync(0xffffffffu, *tmem_at, 0), dp_at = tmem + TILE, dv_at = tmem + 2 * TILE, dk_at = dv_at + DP;
  const u32 k_tile = base, v_tile = base + L::BYTES, ring = base + L::RING;
  // binary16: p is taken 2^14 times larger, ds by its range (see above)
  const float shift = BF16 ? 0.f : 14.f, back = BF16 ? 1.f : 6.103515625e-05f;
  const int begin = a.causal ? t.first / TILE : low_tile, each = high_tile - begin, n = each * group;
  if (warp == BWD_ROWS + 1) {
    u32 side = 0, words[4];
    Counts ahead;
    read_counts(a, t, begin * TILE, ahead);
    int i = 0;
    bool ok = true;
    float range = 1.f;
    for (; ok && i < 2 * n; ++i) {                             // tiles of queries and of dout in turn
      const int st = i % L::STAGES, j = i / 2, head = kh * group + j / each, first = (begin + j % each) * TILE;
      if (i >= L::STAGES && !mbar_wait(empty + 8 * st, (i / L::STAGES - 1) & 1, dead)) break;
      if (!(i & 1)) {
        words_of(ahead, words);
        read_counts(a, t, (begin + (j + 1) % each) * TILE, ahead);
      } else {
        // With dout, whose slot was the queries' of two steps ago or later ones': the step that used these numbers before has ended.
        if (i >= 4 && L::STAGES > 5 && !mbar_wait(empty + 8 * ((i - 5) % L::STAGES), ((i - 5) / L::STAGES) & 1, dead)) break;
        if (i == 1) {                                          // row_dot comes from the kernel before this one
          asm volatile("griddepcontrol.wait;" ::: "memory");
          if (!BF16) range = __ldcg(range_at(g.dk, g.dk_stride, t.row + t.first, kh, a.head_dim));
        }
        float* const to = stats + (j & 1) * 2 * TILE;
        const long long at = (long long)head * a.tokens + t.row + first;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const bool on = words[w] >> lane & 1;
          to[32 * w + lane] = on ? fmaf(g.lse[at + 32 * w + lane], -LOG2E, shift) : -INFINITY;
          to[TILE + 32 * w + lane] = on ? -__ldcg(g.row_dot + at + 32 * w + lane) * (range * back) : 0.f;
        }
        __syncwarp();
      }
      ok = bring<DP>(ring + st * L::BYTES, i & 1 ? &maps.dout : &maps.q, head, t.row + first, words, true, full + 8 * st, aside, side, dead);
    }
    if (*dead) {
      settle(kv_full, 0);
      for (int b = max(0, i - L::STAGES); b < i; ++b) settle(full + 8 * (b % L::STAGES), (b / L::STAGES) & 1);
    }
  } else if (warp == BWD_ROWS) {
    {
      const u32 leader = elect_leader();
      auto tile = [&](int i) { return ring + (i % L::STAGES) * L::BYTES; };
      auto scores = [&](int j) {
        if (!mbar_wait_warp(full + 8 * (2 * j % L::STAGES), (2 * j / L::STAGES) & 1, dead)) return false;
        tc_fence_after();
        product_nt<BF16, DP>(leader, tmem, k_tile, tile(2 * j));
        mma_commit(leader, s_full);
        return true;
      };
      auto shares = [&](int j) {
        if (!mbar_wait_warp(full + 8 * ((2 * j + 1) % L::STAGES), ((2 * j + 1) / L::STAGES) & 1, dead)) return false;
        tc_fence_after();
        product_nt<BF16, DP>(leader, dp_at, v_tile, tile(2 * j + 1));
        mma_commit(leader, dp_full);
        return true;
      };
      bool ok = mbar_wait_warp(kv_full, 0, dead) && scores(0) && shares(0);
      for (int j = 0; ok && j < n; ++j) {
        if (j + 1 < n && !(mbar_wait_warp(s_read, j & 1, dead) && scores(j + 1))) break;
        if (!mbar_wait_warp(ds_full, j & 1, dead)) break;
        tc_fence_after();
        product_pn<BF16, DP, 2>(leader, dv_at, dp_at + 16, tile(2 * j + 1), j > 0);
        mma_commit(leader, empty + 8 * ((2 * j + 1) % L::STAGES));
        product_pn<BF16, DP, 2>(leader, dk_at, dp_at, tile(2 * j), j > 0);
        mma_commit(leader, empty + 8 * (2 * j % L::STAGES));
        if (j + 1 < n && !shares(j + 1)) break;
      }
      if (!*dead) mma_commit(leader, end_full);
      else {
        mma_commit(leader, aside);
        settle(aside, 0);
      }
    }
  } else {
    const int part_of = warp >> 2, i = t.first + (warp & 3) * 32 + lane;   // the thread's key
    const u32 lanes = (u32)(warp & 3) << 21, s_at = tmem + 32 * part_of + lanes, d_at = dp_at + 32 * part_of + lanes;
    float range = 1.f;
    if (!BF16) {
      asm volatile("griddepcontrol.wait;" ::: "memory");
      range = __ldcg(range_at(g.dk, g.dk_stride, t.row + t.first, kh, a.head_dim));
    }
    const float c = a.scale * LOG2E;
    const F2 c2 = f2(c, c), range2 = f2(range * back, range * back);
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      const int first = (begin + j % each) * TILE + 32 * part_of;
      const float* const low = stats + (j & 1) * 2 * TILE + 32 * part_of;
      const bool mask = a.causal && first < t.first + TILE;              // queries before the key
      // the log sums come with dout's tile
      if (!(ok = mbar_wait(full + 8 * ((2 * j + 1) % L::STAGES), ((2 * j + 1) / L::STAGES) & 1, dead))) break;
      if (!(ok = mbar_wait(s_full, j & 1, dead))) break;
      tc_fence_after();
      u32 s[32];
      tmem_ld32(s_at, s);
      tmem_wait_ld();
      tmem_hold(s);
      tc_fence_before();
      mbar_arrive(s_read);
      F2 p[16];
      auto shares = [&](auto masked) {
#pragma unroll
        for (int k = 0; k < 32; k += 4) {
          const float4 l = *reinterpret_cast<const float4*>(low + k);
          float y0, y1, y2, y3;
          split(exp2_pair(fma2(f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, f2(l.x, l.y))), y0, y1);
          split(exp2_pair(fma2(f2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, f2(l.z, l.w))), y2, y3);
          if (decltype(masked)::value) {
            const int q = first + k;
            y0 = q >= i ? y0 : 0.f;
            y1 = q + 1 >= i ? y1 : 0.f;
            y2 = q + 2 >= i ? y2 : 0.f;
            y3 = q + 3 >= i ? y3 : 0.f;
          }
          p[k / 2] = f2(y0, y1);
          p[k / 2 + 1] = f2(y2, y3);
        }
      };
      if (mask) shares(Yes{});
      else shares(No{});
      if (!(ok = mbar_wait(dp_full, j & 1, dead))) break;
      tc_fence_after();
      tmem_ld32(d_at, s);
      tmem_wait_ld();
      tmem_hold(s);
      u32 w16[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        float y0, y1;
        split(p[k], y0, y1);
        w16[k] = pack2<BF16>(y0, y1);
      }
      tmem_st16(d_at + 16, w16);
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 l = *reinterpret_cast<const float4*>(low + TILE + k);
        float y0, y1, y2, y3;
        const F2 u = f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), v = f2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
        split(mul2(p[k / 2], BF16 ? add2(u, f2(l.x, l.y)) : fma2(u, range2, f2(l.x, l.y))), y0, y1);
        split(mul2(p[k / 2 + 1], BF16 ? add2(v, f2(l.z, l.w)) : fma2(v, range2, f2(l.z, l.w))), y2, y3);
        w16[k / 2] = pack2<BF16>(y0, y1);
        w16[k / 2 + 1] = pack2<BF16>(y2, y3);
      }
      tmem_st16(d_at, w16);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(ds_full);
    }
    if (ok && mbar_wait(end_full, 0, dead)) {
      tc_fence_after();
      const bool inside = i < t.length, on = inside && (!a.mask || a.mask[t.row + i]);
      if (32 * part_of < DP) {
        store_cols<BF16>(g.dk, g.dk_stride, t.row + i, kh, a.head_dim, 32 * part_of, dk_at + lanes, a.scale / range, inside, !on);
        store_cols<BF16>(g.dv, g.dv_stride, t.row + i, kh, a.head_dim, 32 * part_of, dv_at + lanes, back, inside, !on);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == BWD_ROWS) tmem_free(tmem, 512);
  if (*dead && threadIdx.x < TILE && t.first + (int)threadIdx.x < t.length) {
    poison_row(g.dk, g.dk_stride, t.row + t.first + threadIdx.x, kh, a.head_dim);
    poison_row(g.dv, g.dv_stride, t.row + t.first + threadIdx.x, kh, a.head_dim);
  }
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) return (EncodeTiled) nullptr;
    return (EncodeTiled)p;
  }();
  return fn;
}

bool rows_on_16(const void* p, long long stride, long long rows) { return ((uintptr_t)p & 15) == 0 && (rows <= 1 || stride % 8 == 0); }

// Tokens x heads x elements; a box is 128 tokens of one head's 64 elements.
bool map_of(CUtensorMap* m, const void* p, long long stride, const adacgd_attention_inputs& a, int heads) {
  const long long row = (long long)heads * a.head_dim;
  if (a.tokens == 1 || stride < row) stride = row;             // of a single row it may be anything
  const cuuint64_t dims[3] = {(cuuint64_t)a.head_dim, (cuuint64_t)heads, (cuuint64_t)a.tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)a.head_dim * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, 1, TILE}, steps[3] = {1, 1, 1};
  return encoder()(m, a.dtype == ADACGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims,
                   strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool takes(const adacgd_attention_inputs& a) {
  return a.dtype != ADACGD_F32 && a.head_dim % 8 == 0 && a.head_dim <= 128 && rows_on_16(a.q, a.q_stride, a.tokens) &&
         rows_on_16(a.k, a.k_stride, a.tokens) && rows_on_16(a.v, a.v_stride, a.tokens) && tile_slots(a, TILE) * a.heads < (1ll << 31) && encoder();
}

// after: the kernel may begin before the one in front of it has ended (it waits for that itself).
template <typename K, typename... A>
bool launch_mma(K kern, std::atomic<int> (&table)[TRAIN_DEVICES], int threads, int smem, long long ctas, bool after, const Where& at, const A&... args) {
  if (resident_ctas(kern, table, at.device, threads, smem) < 1) return false;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, args...) == cudaSuccess;
}

template <bool BF16, int DP> int fwd_mma(const Maps& m, const adacgd_attention_args& g, const Where& at) {
  static std::atomic<int> table[TRAIN_DEVICES];
  return launch_mma(k_attention_mma<BF16, DP>, table, FWD_CTA, FwdLayout<DP>::TOTAL, tile_slots(g.in, 2 * TILE) * g.in.heads, false, at, m, g) ? 1 : -1;
}
template <bool BF16, int DP> int bwd_mma(const Maps& m, const adacgd_attention_backward_args& g, const Where& at) {
  static std::atomic<int> table[2][TRAIN_DEVICES];
  const long long slots = tile_slots(g.in, TILE);
  if (!BF16) {
    k_attention_range<DP / 8><<<dim3((unsigned)slots, (unsigned)g.in.key_heads, (unsigned)range_parts(g.in)), RANGE_CTA, 0, at.stream>>>(g);
    if (cudaGetLastError() != cudaSuccess) return -1;
  }
  if (!launch_mma(k_attention_dq_mma<BF16, DP>, table[0], BWD_CTA, DqLayout<DP>::TOTAL, slots * g.in.heads, !BF16, at, m, g)) return -1;
  if (!launch_mma(k_attention_dkv_mma<BF16, DP>, table[1], BWD_CTA, DkvLayout<DP>::TOTAL, slots * g.in.key_heads, true, at, m, g)) return -1;
  return BF16 ? 2 : 3;
}

}  // namespace

#define BY_KIND(call)                                                                                                    \
  if (a.dtype == ADACGD_BF16) { constexpr bool BF16 = true; BY_WIDTH(call) }                                             \
  { constexpr bool BF16 = false; BY_WIDTH(call) }
#define BY_WIDTH(call)                                                                                                   \
  if (a.head_dim <= 64) { constexpr int DP = 64; return call; }                                                          \
  { constexpr int DP = 128; return call; }

int launch_attention_mma(const adacgd_attention_args& g, const Where& at) {
  const adacgd_attention_inputs& a = g.in;
  if (!takes(a) || !rows_on_16(g.out, g.out_stride, a.tokens)) return 0;
  Maps m = {};
  if (!map_of(&m.q, a.q, a.q_stride, a, a.heads) || !map_of(&m.k, a.k, a.k_stride, a, a.key_heads) || !map_of(&m.v, a.v, a.v_stride, a, a.key_heads)) return 0;
  BY_KIND((fwd_mma<BF16, DP>(m, g, at)))
}

int launch_attention_backward_mma(const adacgd_attention_backward_args& g, const Where& at) {
  const adacgd_attention_inputs& a = g.in;
  if (!takes(a) || !rows_on_16(g.out, g.out_stride, a.tokens) || !rows_on_16(g.dout, g.dout_stride, a.tokens) ||
      !rows_on_16(g.dq, g.dq_stride, a.tokens) || !rows_on_16(g.dk, g.dk_stride, a.tokens) || !rows_on_16(g.dv, g.dv_stride, a.tokens))
    return 0;
  Maps m = {};
  if (!map_of(&m.q, a.q, a.q_stride, a, a.heads) || !map_of(&m.k, a.k, a.k_stride, a, a.key_heads) || !map_of(&m.v, a.v, a.v_stride, a, a.key_heads) ||
      !map_of(&m.dout, g.dout, g.dout_stride, a, a.heads))
    return 0;
  BY_KIND((bwd_mma<BF16, DP>(m, g, at)))
}

}  // namespace adacgd
