// Embedding lookup and its gradient (adacgd_train.h).
//
// The lookup is a copy of rows, bound by memory.  The gradient is a sum over the tokens of each id.  Sums in the order of the batch
// need the tokens of an id side by side, so tokens are sorted by id first: a stable radix sort by one cluster, whose CTAs
// see one another's digit counts through distributed shared memory (no second launch, no flag that anybody spins on).  Then CTAs take
// ranges of the table's rows, find their tokens by search and write every row once.  An id with very many tokens (frequent
// words: a twentieth of a batch may be one word) would leave one CTA with all the work; its run of sorted tokens is cut into
// windows, whose partial sums a last kernel adds in order.
#include <cooperative_groups.h>

#include "adacgd_train.cuh"

namespace cg = cooperative_groups;

namespace adacgd {
namespace {

// Vectors of N elements as floats: N = 8 takes whole runs, N = 1 any address.
template <typename T, int N> struct Elems {
  static __device__ __forceinline__ void load(const T* p, float (&v)[N]) {
    if constexpr (N == 8) unpack(load_run(p), v); else v[0] = to_f(p[0]);
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[N]) {
    if constexpr (N == 8) store_run(p, v); else p[0] = from_f<T>(v[0]);
  }
};

__device__ __forceinline__ long long id_at(const void* ids, int bytes, long long t) {
  return bytes == 8 ? reinterpret_cast<const long long*>(ids)[t] : (long long)reinterpret_cast<const int32_t*>(ids)[t];
}

// --------------------------------------------------------------------------
// lookup
// --------------------------------------------------------------------------
// TPR threads a row, each with up to four vectors in flight; grid.y cuts wide rows.
constexpr int LOOK_CTA = 128, LOOK_VECS = 4;

template <typename T, int N, int TPR>
__global__ void __launch_bounds__(LOOK_CTA) k_embedding(adacgd_embedding_args a) {
  const long long row = (long long)blockIdx.x * (LOOK_CTA / TPR) + threadIdx.x / TPR;
  if (row >= a.tokens) return;
  const int lane = threadIdx.x % TPR;
  const long long vecs = a.cols / N, first = (long long)blockIdx.y * (TPR * LOOK_VECS);
  const bool on = !a.mask || a.mask[row];
  const long long id = on ? id_at(a.ids, a.id_bytes, row) : 0;
  const bool known = id >= 0 && id < a.vocab;
  T* const out = (T*)a.out + row * a.out_stride;
  float v[LOOK_VECS][N];
  if (on && known) {
    const T* const src = (const T*)a.table + id * a.table_stride;
#pragma unroll
    for (int k = 0; k < LOOK_VECS; ++k) {
      const long long c = first + k * TPR + lane;
      if (c < vecs) Elems<T, N>::load(src + c * N, v[k]);
    }
  }
  const float other = on ? nanf("") : 0.f;
#pragma unroll
  for (int k = 0; k < LOOK_VECS; ++k) {
    const long long c = first + k * TPR + lane;
    if (c >= vecs) break;
#pragma unroll
    for (int j = 0; j < N; ++j) v[k][j] = on && known ? v[k][j] * a.scale : other;
    Elems<T, N>::store(out + c * N, v[k]);
  }
}

// Rows that consist of whole aligned runs.
template <typename T> bool whole_runs(const void* p, long long stride, long long rows, long long cols) {
  const size_t step = 8 * sizeof(T);
  return !p || (cols % 8 == 0 && (uintptr_t)p % step == 0 && (rows <= 1 || stride * sizeof(T) % step == 0));
}

template <typename T, int N, int TPR>
int lookup_launch(const adacgd_embedding_args& a, const Where& at) {
  const long long rows = LOOK_CTA / TPR, vecs = a.cols / N;
  const dim3 grid((unsigned)((a.tokens + rows - 1) / rows), (unsigned)((vecs + TPR * LOOK_VECS - 1) / (TPR * LOOK_VECS)));
  k_embedding<T, N, TPR><<<grid, LOOK_CTA, 0, at.stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}
template <typename T, int N>
int lookup_by_width(const adacgd_embedding_args& a, const Where& at) {
  const long long vecs = a.cols / N;
  if (vecs <= 32) return lookup_launch<T, N, 8>(a, at);
  if (vecs <= 128) return lookup_launch<T, N, 32>(a, at);
  return lookup_launch<T, N, 128>(a, at);
}
template <typename T>
int lookup_t(const adacgd_embedding_args& a, const Where& at) {
  const bool runs = whole_runs<T>(a.table, a.table_stride, a.vocab, a.cols) && whole_runs<T>(a.out, a.out_stride, a.tokens, a.cols);
  return runs ? lookup_by_width<T, 8>(a, at) : lookup_by_width<T, 1>(a, at);
}

// --------------------------------------------------------------------------
// sort of the tokens by id
// --------------------------------------------------------------------------
// Least significant digit first, 9 bits a pass: an id of 131072 words takes two.  The cluster's CTAs own consecutive parts of the
// array, their warps consecutive parts of those, so that (digit, CTA, warp, place) is the stable order.
constexpr int SORT_CTA = 1024, SORT_WARPS = SORT_CTA / 32, DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;

struct SortSmem {
  u32 hist[SORT_WARPS][DIGITS];   // a warp's counts, then where its next token of a digit goes
  u32 total[DIGITS];              // the CTA's counts, read by the others
  u32 scan[DIGITS / 32];
};

// Key of a token: its id, or `vocab` (which sorts last) where it adds to nothing.
__device__ __forceinline__ u32 key_of(const void* ids, int bytes, const uint8_t* mask, long long vocab, long long t) {
  if (mask && !mask[t]) return (u32)vocab;
  const long long id = id_at(ids, bytes, t);
  return id >= 0 && id < vocab ? (u32)id : (u32)vocab;
}

// (key, place) pairs alternate between (k0, p0) and (k1, p1); the last pass ends in (k1, p1).
__global__ void __launch_bounds__(SORT_CTA) k_sort_ids(const void* ids, int id_bytes, const uint8_t* mask, long long vocab, int n, int passes,
                                                       u32* k0, u32* p0, u32* k1, u32* p1) {
  extern __shared__ __align__(16) unsigned char sort_smem[];
  SortSmem& sh = *reinterpret_cast<SortSmem*>(sort_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), cta = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long parts = (long long)ctas * SORT_WARPS, part = (long long)cta * SORT_WARPS + warp;
  const int lo = (int)(part * n / parts), hi = (int)((part + 1) * n / parts);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * DIGIT_BITS;
    const bool odd = ((passes - pass) & 1) != 0;      // passes with an even distance to the end write (k1, p1)
    const u32* const ki = odd ? k0 : k1;
    const u32* const pi = odd ? p0 : p1;
    u32* const ko = odd ? k1 : k0;
    u32* const po = odd ? p1 : p0;
    for (int i = threadIdx.x; i < SORT_WARPS * DIGITS; i += SORT_CTA) (&sh.hist[0][0])[i] = 0;
    __syncthreads();
    for (int i = lo + lane; i < hi; i += 32) {
      const u32 key = pass ? __ldcg(ki + i) : key_of(ids, id_bytes, mask, vocab, i);
      atomicAdd(&sh.hist[warp][(key >> shift) & (DIGITS - 1)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < DIGITS) {                       // a digit's places among the CTA's warps
      u32 sum = 0;
#pragma unroll 8
      for (int w = 0; w < SORT_WARPS; ++w) {
        const u32 c = sh.hist[w][threadIdx.x];
        sh.hist[w][threadIdx.x] = sum;
        sum += c;
      }
      sh.total[threadIdx.x] = sum;
    }
    cluster.sync();
    u32 before = 0, all = 0;                          // of this digit: in the CTAs before this one, in all
    if (threadIdx.x < DIGITS) {
      for (int c = 0; c < ctas; ++c) {
        const u32 v = *cluster.map_shared_rank(&sh.total[threadIdx.x], c);
        if (c < cta) before += v;
        all += v;
      }
    }
    u32 incl = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u32 v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (threadIdx.x < DIGITS && lane == 31) sh.scan[warp] = incl;
    __syncthreads();
    if (threadIdx.x < DIGITS) {
      u32 base = incl - all + before;
      for (int w = 0; w < warp; ++w) base += sh.scan[w];
#pragma unroll 8
      for (int w = 0; w < SORT_WARPS; ++w) sh.hist[w][threadIdx.x] += base;
    }
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += 32) {
      const int i = i0 + lane;
      const bool in = i < hi;
      u32 key = 0, place = (u32)i;
      if (in) {
        key = pass ? __ldcg(ki + i) : key_of(ids, id_bytes, mask, vocab, i);
        if (pass) place = __ldcg(pi + i);
      }
      const u32 digit = in ? (key >> shift) & (DIGITS - 1) : DIGITS;   // lanes behind the end match none that is in
      const u32 same = __match_any_sync(0xffffffffu, digit);
      const int rank = __popc(same & ((1u << lane) - 1));
      u32 to = 0;
      if (in) to = sh.hist[warp][digit] + rank;
      __syncwarp();
      if (in && rank == 0) sh.hist[warp][digit] += __popc(same);
      __syncwarp();
      if (in) {
        __stcg(ko + to, key);
        __stcg(po + to, place);
      }
    }
    __threadfence();
    cluster.sync();     // the other CTAs' writes, and nobody's counts are still being read
  }
}

// --------------------------------------------------------------------------
// sums
// --------------------------------------------------------------------------
// The first place in the sorted keys whose key is at least `key`: a warp looks at 32 places a round.
__device__ __forceinline__ int lower_bound_warp(const u32* keys, int lo, int hi, u32 key) {
  const int lane = threadIdx.x & 31;
  while (hi - lo > 0) {                      // keys before lo are smaller, those from hi on are not
    const long long span = hi - lo;
    const int step = (int)((span + 31) / 32);
    const long long at = lo + (long long)lane * step;
    const bool less = at < hi && __ldcg(keys + at) < key;
    const int m = __popc(__ballot_sync(0xffffffffu, less));   // the first m probes are smaller
    if (m == 0) return lo;
    const long long from = lo + (long long)(m - 1) * step + 1, to = lo + (long long)m * step;
    hi = (int)(to < hi ? to : hi);
    lo = (int)from;
  }
  return lo;
}
__device__ __forceinline__ int lower_bound_lane(const u32* keys, int lo, int hi, u32 key) {
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (__ldcg(keys + mid) < key) lo = mid + 1; else hi = mid;
  }
  return lo;
}

constexpr int SUM_CTA = 256, SUM_ROWS = 32, SUM_MIN = 64, SUM_STAGE = 512;   // most rows of the table a CTA takes; tokens staged
constexpr int MAX_WINDOWS = NORM_PARTS;   // two partial sums a window

struct SumArgs {
  const void* dout; long long dout_stride;
  const void* base; long long base_stride;
  void* dtable;     long long dtable_stride;
  const u32* keys;
  const u32* places;
  float* part;      // [2 windows][part_stride]
  long long part_stride;
  long long vocab, cols;
  int n, most;      // tokens; rows of one id that one thread sums: longer runs go by windows of that length
  int windows, slices;   // CTAs of the long runs: windows * slices, a slice being SUM_CTA vectors of each row at a time
  int rows;         // of the table, that a CTA takes
  float scale;
  bool leave;       // rows without tokens stay as they are
};

// Sum of the rows places[lo .. hi) (a global or a shared array) in columns [N c, N c + N), four loads in flight.
template <typename T, int N>
__device__ __forceinline__ void sum_rows(const SumArgs& s, const u32* places, int lo, int hi, long long c, float (&acc)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) acc[j] = 0.f;
  int i = lo;
  for (; i + 4 <= hi; i += 4) {
    float v[4][N];
#pragma unroll
    for (int k = 0; k < 4; ++k) Elems<T, N>::load((const T*)s.dout + (long long)places[i + k] * s.dout_stride + c * N, v[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] += v[k][j];
  }
  for (; i < hi; ++i) {
    float v[N];
    Elems<T, N>::load((const T*)s.dout + (long long)places[i] * s.dout_stride + c * N, v);
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] += v[j];
  }
}

template <typename O, int N>
__device__ __forceinline__ void finish_row(const SumArgs& s, long long v, long long c, const float (&acc)[N]) {
  float o[N], b[N];
  if (s.base) Elems<O, N>::load((const O*)s.base + v * s.base_stride + c * N, b);
#pragma unroll
  for (int j = 0; j < N; ++j) o[j] = s.base ? fmaf(acc[j], s.scale, b[j]) : acc[j] * s.scale;
  Elems<O, N>::store((O*)s.dtable + v * s.dtable_stride + c * N, o);
}

// The first CTAs take a window of the sorted tokens each (and a slice of its columns), for ids with more than `most` tokens; the
// others `rows` rows of the table.  TPR threads a row.
template <typename T, typename O, int N, int TPR>
__global__ void __launch_bounds__(SUM_CTA) k_embedding_sum(SumArgs s) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int G = SUM_CTA / TPR;
  const long long vecs = s.cols / N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ int edge[SUM_ROWS + 1];
  __shared__ u32 staged[SUM_STAGE];
  const unsigned long_ctas = (unsigned)s.windows * s.slices;
  if (blockIdx.x < long_ctas) {
    const int w = (int)(blockIdx.x / s.slices), lo = w * s.most, hi = min(s.n, lo + s.most);
    const int slice = (int)(blockIdx.x % s.slices);
    // at most two long runs reach into a window: the one its first token belongs to and the one its last belongs to
    if (warp < 2) {
      const u32 key = __ldcg(s.keys + (warp ? hi - 1 : lo));
      const int a = lower_bound_warp(s.keys, 0, warp ? hi : lo + 1, key);
      const int b = lower_bound_warp(s.keys, warp ? hi - 1 : lo, s.n, key + 1);
      const bool longer = b - a > s.most && (long long)key < s.vocab;
      if (lane == 0) {
        edge[2 * warp] = longer ? max(a, lo) : 0;
        edge[2 * warp + 1] = longer ? min(b, hi) : 0;
      }
    }
    __syncthreads();
    const int from0 = edge[0], to0 = edge[1], from1 = edge[2], to1 = edge[3];
    for (int k = 0; k < 2; ++k) {
      const int from = k ? from1 : from0, to = k ? to1 : to0;
      if (to <= from || (k && from0 == from1 && to0 == to1)) continue;   // one run over the whole window: once
      float* const part = s.part + (2ll * w + k) * s.part_stride;
      for (long long c = (long long)slice * SUM_CTA + threadIdx.x; c < vecs; c += (long long)s.slices * SUM_CTA) {
        float acc[N];
        sum_rows<T, N>(s, s.places, from, to, c, acc);
#pragma unroll
        for (int j = 0; j < N; ++j) part[c * N + j] = acc[j];
      }
    }
    return;
  }
  const long long v0 = (long long)(blockIdx.x - long_ctas) * s.rows;
  const int rows = (int)min((long long)s.rows, s.vocab - v0);
  if (warp < 2) {
    const int e = lower_bound_warp(s.keys, 0, s.n, (u32)(v0 + (warp ? rows : 0)));
    if (lane == 0) edge[warp ? rows : 0] = e;
  }
  __syncthreads();
  const int lo = edge[0], hi = edge[rows];
  __syncthreads();
  const bool stage = hi - lo <= SUM_STAGE;            // the tokens' numbers ahead of the loads that need them
  if (stage)
    for (int i = threadIdx.x; i < hi - lo; i += SUM_CTA) staged[i] = __ldcg(s.places + lo + i);
  if (threadIdx.x < rows) edge[threadIdx.x] = lo == hi ? lo : lower_bound_lane(s.keys, lo, hi, (u32)(v0 + threadIdx.x));
  __syncthreads();
  const int t = threadIdx.x % TPR;
  for (int r = threadIdx.x / TPR; r < rows; r += G) {
    const int from = edge[r], to = edge[r + 1];
    if ((from == to && s.leave) || to - from > s.most) continue;
    for (long long c = t; c < vecs; c += TPR) {
      float acc[N];
      if (stage) sum_rows<T, N>(s, staged, from - lo, to - lo, c, acc);
      else sum_rows<T, N>(s, s.places, from, to, c, acc);
      finish_row<O, N>(s, v0 + r, c, acc);
    }
  }
}

// Adds the windows of a long run, in order, by the CTAs of the window in which it begins (in which no second one can begin:
// it would have to end there, and be short).
template <typename O, int N>
__global__ void __launch_bounds__(SUM_CTA) k_embedding_join(SumArgs s) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int w = (int)blockIdx.x, lo = w * s.most, hi = min(s.n, lo + s.most);
  __shared__ int ends[2];
  const u32 key = __ldcg(s.keys + hi - 1);
  if (threadIdx.x < 32) {
    const int a = lower_bound_warp(s.keys, 0, hi, key), b = lower_bound_warp(s.keys, hi - 1, s.n, key + 1);
    if (threadIdx.x == 0) {
      ends[0] = a;
      ends[1] = b;
    }
  }
  __syncthreads();
  const int a = ends[0], b = ends[1];
  if (b - a <= s.most || a < lo || (long long)key >= s.vocab) return;
  const int last = (b - 1) / s.most;
  const long long vecs = s.cols / N;
  for (long long c = (long long)blockIdx.y * SUM_CTA + threadIdx.x; c < vecs; c += (long long)gridDim.y * SUM_CTA) {
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    for (int i = w; i <= last; ++i) {
      // the run is its window's first one unless it begins behind the window's first token
      const float* const part = s.part + (2ll * i + (i == w && a > lo ? 1 : 0)) * s.part_stride + c * N;
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] += __ldcg(part + j);
    }
    finish_row<O, N>(s, (long long)key, c, acc);
  }
}

template <typename K, typename... A>
bool launch_dependent(K kern, dim3 grid, int threads, const Where& at, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...) == cudaSuccess;
}

template <typename T, typename O, int N, int TPR>
int sum_launch(SumArgs s, const Where& at) {
  const long long slices = (s.cols / N + SUM_CTA - 1) / SUM_CTA;
  s.slices = (int)(slices < 16 ? slices : 16);
  // Rows of the table one after the other are a chain of memory latencies: few of them a CTA as long as that gives every SM only a
  // few CTAs.
  s.rows = SUM_ROWS;
  while (s.rows > SUM_CTA / TPR && s.rows > 1 && s.vocab < 8ll * s.rows * at.sms) s.rows /= 2;
  const long long blocks = (long long)s.windows * s.slices + (s.vocab + s.rows - 1) / s.rows;
  if (!launch_dependent(k_embedding_sum<T, O, N, TPR>, dim3((unsigned)blocks), SUM_CTA, at, s)) return -1;
  if (!s.windows) return 1;
  return launch_dependent(k_embedding_join<O, N>, dim3((unsigned)s.windows, (unsigned)s.slices), SUM_CTA, at, s) ? 2 : -1;
}
template <typename T, typename O, int N>
int sum_by_width(const SumArgs& s, const Where& at) {
  const long long vecs = s.cols / N;
  if (vecs <= 16) return sum_launch<T, O, N, 8>(s, at);
  if (vecs <= 64) return sum_launch<T, O, N, 32>(s, at);
  return sum_launch<T, O, N, 256>(s, at);
}
template <typename T, typename O>
int sum_t(const SumArgs& s, const Where& at) {
  const bool runs = whole_runs<T>(s.dout, s.dout_stride, s.n, s.cols) && whole_runs<O>(s.base, s.base_stride, s.vocab, s.cols) &&
                    whole_runs<O>(s.dtable, s.dtable_stride, s.vocab, s.cols);
  return runs ? sum_by_width<T, O, 8>(s, at) : sum_by_width<T, O, 1>(s, at);
}

}  // namespace

#define BY_TYPE(dtype, call)                                   \
  switch (dtype) {                                             \
    case ADACGD_F32: { typedef float T; return call; }         \
    case ADACGD_F16: { typedef __half T; return call; }        \
    default: { typedef __nv_bfloat16 T; return call; }         \
  }

int launch_embedding(const adacgd_embedding_args& a, const Where& at) { BY_TYPE(a.dtype, (lookup_t<T>(a, at))) }

int launch_embedding_backward(const TrainScratch& ws, const adacgd_embedding_backward_args& a, const Where& at) {
  SumArgs s = {};
  s.dout = a.dout; s.dout_stride = a.dout_stride;
  s.base = a.base; s.base_stride = a.base_stride;
  s.dtable = a.dtable; s.dtable_stride = a.dtable_stride;
  s.vocab = a.vocab; s.cols = a.cols;
  s.n = (int)a.tokens;
  s.scale = a.scale;
  s.leave = a.base && a.base == a.dtable;
  u32 *k0 = (u32*)ws.tok_a, *p0 = (u32*)ws.tok_b, *k1 = (u32*)ws.tok_c, *p1 = (u32*)ws.seq;
  s.keys = k1;
  s.places = p1;
  s.part = ws.norm_part;
  s.part_stride = ws.max_cols;
  s.most = (s.n + MAX_WINDOWS - 1) / MAX_WINDOWS;
  if (s.most < SUM_MIN) s.most = SUM_MIN;
  s.windows = s.n > s.most ? (s.n + s.most - 1) / s.most : 0;
  int bits = 1;
  while ((1ll << bits) <= a.vocab) ++bits;           // keys up to `vocab` itself
  const int passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
  static std::atomic<int> table[TRAIN_DEVICES];
  if (resident_ctas(k_sort_ids, table, at.device, SORT_CTA, (int)sizeof(SortSmem)) < 1) return -1;
  // A CTA reads 32 numbers a warp and step; more CTAs cost a little in the counts they exchange.
  int ctas = 1;
  while (ctas < 8 && s.n > 2048 * ctas) ctas *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(SORT_CTA);
  cfg.dynamicSmemBytes = sizeof(SortSmem);
  cfg.stream = at.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, k_sort_ids, a.ids, (int)a.id_bytes, a.mask, (long long)a.vocab, s.n, passes, k0, p0, k1, p1) != cudaSuccess) return -1;
  int n = -1;
  if (a.table_dtype == ADACGD_F32 && a.dtype == ADACGD_F16) n = sum_t<__half, float>(s, at);
  else if (a.table_dtype == ADACGD_F32 && a.dtype == ADACGD_BF16) n = sum_t<__nv_bfloat16, float>(s, at);
  else if (a.dtype == ADACGD_F32) n = sum_t<float, float>(s, at);
  else if (a.dtype == ADACGD_F16) n = sum_t<__half, __half>(s, at);
  else n = sum_t<__nv_bfloat16, __nv_bfloat16>(s, at);
  return n < 0 ? -1 : n + 1;
}

}  // namespace adacgd
