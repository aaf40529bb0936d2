// Embedding lookup and its gradient (adacgd_train.h).
//
// The lookup is a copy of rows, bound by memory.  The gradient is a sum over the tokens of each id.  Sums in the order of the batch
// need the tokens of an id side by side, so tokens are sorted by id first: a stable radix sort by one cluster, whose CTAs
// see one another's digit counts through distributed shared memory (no second launch, no flag that anybody spins on).  Then CTAs take
// ranges of the table's rows, find their tokens by search and write every row once.  An id with very many tokens (frequent
// words: a twentieth of a batch may be one word) would leave one CTA with all the work; its run of sorted tokens is cut into
// windows, whose partial sums a last kernel adds in order.  (Adding them in the CTA that finishes last saved that kernel and cost more in the one
// before it: 311 against 288 us for 32768 tokens.)
#include <cooperative_groups.h>

#include <type_traits>

#include "adacgd_train.cuh"

namespace cg = cooperative_groups;

namespace adacgd {
namespace {

// Vectors of N elements: N = 8 takes whole runs, N = 1 any address.  Raw is what a load leaves.
template <typename T, int N> struct Elems {
  typedef typename std::conditional<N == 8, Run<T>, T>::type Raw;
  static __device__ __forceinline__ Raw fetch(const T* p) {
    if constexpr (N == 8) return load_run(p); else return p[0];
  }
  static __device__ __forceinline__ void floats(const Raw& r, float (&v)[N]) {
    if constexpr (N == 8) unpack(r, v); else v[0] = to_f(r);
  }
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
constexpr int SORT_CTA = 1024, SORT_WARPS = SORT_CTA / 32, DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS, SORT_CTAS = 8;
constexpr int SORT_KEEP = 8;      // (key, place) pairs a lane holds between counting and placing them

struct SortSmem {
  u32 hist[SORT_WARPS][DIGITS];   // a warp's counts, then where its next token of a digit goes
  u32 total[DIGITS];              // the CTA's counts, read by the others
  u32 scan[DIGITS / 32];
};

// Key of a token: its id, or `vocab` (which sorts last) where it adds to nothing.
__device__ __forceinline__ u32 key_of(const void* ids, int bytes, const uint8_t* mask, long long vocab, long long t) {
  const bool on = !mask || mask[t];
  const long long id = id_at(ids, bytes, t);
  return on && id >= 0 && id < vocab ? (u32)id : (u32)vocab;
}

// (key, place) pairs alternate between (k0, p0) and (k1, p1); the last pass ends in (k1, p1).  `warps` of each CTA take part: the
// counts of a digit are added up warp by warp, so few tokens take few warps.  KEEP: a warp's tokens fit its lanes' registers.
template <bool KEEP>
__global__ void __launch_bounds__(SORT_CTA) k_sort_ids(const void* ids, int id_bytes, const uint8_t* mask, long long vocab, int n, int passes, int warps,
                                                       u32* k0, u32* p0, u32* k1, u32* p1) {
  extern __shared__ __align__(16) unsigned char sort_smem[];
  SortSmem& sh = *reinterpret_cast<SortSmem*>(sort_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), cta = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long parts = (long long)ctas * warps, part = (long long)cta * warps + warp;
  const int lo = warp < warps ? (int)(part * n / parts) : n, hi = warp < warps ? (int)((part + 1) * n / parts) : n;
  u32 keys[SORT_KEEP], places[SORT_KEEP];
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * DIGIT_BITS;
    const bool odd = ((passes - pass) & 1) != 0;      // passes with an even distance to the end write (k1, p1)
    const u32* const ki = odd ? k0 : k1;
    const u32* const pi = odd ? p0 : p1;
    u32* const ko = odd ? k1 : k0;
    u32* const po = odd ? p1 : p0;
    auto key_at = [&](int i) { return pass ? __ldcg(ki + i) : key_of(ids, id_bytes, mask, vocab, i); };
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < SORT_KEEP; ++k) {
        const int i = lo + 32 * k + lane;
        keys[k] = i < hi ? key_at(i) : 0;
        places[k] = i < hi && pass ? __ldcg(pi + i) : (u32)i;
      }
    }
    for (int i = threadIdx.x; i < warps * DIGITS; i += SORT_CTA) (&sh.hist[0][0])[i] = 0;
    __syncthreads();
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < SORT_KEEP; ++k)
        if (lo + 32 * k + lane < hi) atomicAdd(&sh.hist[warp][(keys[k] >> shift) & (DIGITS - 1)], 1u);
    } else {
      for (int i = lo + lane; i < hi; i += 32) atomicAdd(&sh.hist[warp][(key_at(i) >> shift) & (DIGITS - 1)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < DIGITS) {                       // a digit's places among the CTA's warps
      u32 sum = 0;
#pragma unroll 8
      for (int w = 0; w < warps; ++w) {
        const u32 c = sh.hist[w][threadIdx.x];
        sh.hist[w][threadIdx.x] = sum;
        sum += c;
      }
      sh.total[threadIdx.x] = sum;
    }
    cluster.sync();
    u32 before = 0, all = 0;                          // of this digit: in the CTAs before this one, in all
    if (threadIdx.x < DIGITS) {
      u32 v[SORT_CTAS];
#pragma unroll
      for (int c = 0; c < SORT_CTAS; ++c) v[c] = c < ctas ? *cluster.map_shared_rank(&sh.total[threadIdx.x], c) : 0u;
#pragma unroll
      for (int c = 0; c < SORT_CTAS; ++c) {
        if (c < cta) before += v[c];
        all += v[c];
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
      for (int w = 0; w < warps; ++w) sh.hist[w][threadIdx.x] += base;
    }
    __syncthreads();
    auto put = [&](u32 key, u32 place, bool in) {     // 32 tokens of the warp, in order
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
    };
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < SORT_KEEP; ++k)
        if (lo + 32 * k < hi) put(keys[k], places[k], lo + 32 * k + lane < hi);
    } else {
      for (int i0 = lo; i0 < hi; i0 += 32) {
        const int i = i0 + lane;
        const bool in = i < hi;
        put(in ? key_at(i) : 0, in && pass ? __ldcg(pi + i) : (u32)i, in);
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

constexpr int SUM_CTA = 256, SUM_ROWS = 32, SUM_MIN = 16, SUM_STAGE = 512;   // most rows of the table a CTA takes; tokens staged
constexpr int MAX_WINDOWS = NORM_PARTS;   // two partial sums a window
// Places among the sorted tokens are 32-bit: none that is formed, a window or a CTA's stride behind the last token, may pass 2^31.
static_assert(ADACGD_TRAIN_MAX_RUN + (ADACGD_TRAIN_MAX_RUN + MAX_WINDOWS - 1) / MAX_WINDOWS + 32 * SORT_KEEP + SORT_CTA < (1ll << 31), "places fit in an int");

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
  bool few;         // the tokens are not sorted
};

// Sum of the rows places[lo .. hi) (a global or a shared array) in vector c of a row, AHEAD loads in flight.
template <typename T, int N, int AHEAD>
__device__ __forceinline__ void sum_rows(const SumArgs& s, const u32* places, int lo, int hi, long long c, float (&acc)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) acc[j] = 0.f;
  int i = lo;
  for (; i + AHEAD <= hi; i += AHEAD) {
    typename Elems<T, N>::Raw v[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) v[k] = Elems<T, N>::fetch((const T*)s.dout + (long long)places[i + k] * s.dout_stride + c * N);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      float f[N];
      Elems<T, N>::floats(v[k], f);
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] += f[j];
    }
  }
  for (; i < hi; ++i) {
    float f[N];
    Elems<T, N>::load((const T*)s.dout + (long long)places[i] * s.dout_stride + c * N, f);
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] += f[j];
  }
}

// Partial sums: N numbers at a multiple of N.
template <int N> __device__ __forceinline__ void store_part(float* p, const float (&v)[N]) {
  if constexpr (N == 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    p[0] = v[0];
  }
}
template <int N> __device__ __forceinline__ void load_part(const float* p, float (&v)[N]) {
  if constexpr (N == 8) {
    *reinterpret_cast<float4*>(v) = __ldcg(reinterpret_cast<const float4*>(p));
    *reinterpret_cast<float4*>(v + 4) = __ldcg(reinterpret_cast<const float4*>(p) + 1);
  } else {
    v[0] = __ldcg(p);
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

// Columns c0 .. c1 - 1 of a row without tokens: zeros, or the base's numbers.  Sixteen bytes at a time but for the ends; element by element such
// rows, most of a large table, took more instructions than the rest (118 us for 50257 rows of 1001).
template <typename O>
__device__ __forceinline__ void plain_row(const SumArgs& s, long long v, int c0, int c1, int t, int threads) {
  constexpr int V = 16 / sizeof(O);
  O* const to = (O*)s.dtable + v * s.dtable_stride;
  const O* const from = s.base ? (const O*)s.base + v * s.base_stride : nullptr;
  const int skew = (int)(((uintptr_t)(to + c0) & 15) / sizeof(O));
  const int head = min(c1, c0 + (skew ? V - skew : 0));
  const bool wide = !from || (((uintptr_t)from ^ (uintptr_t)to) & 15) == 0;
  const int tail = wide ? head + (c1 - head) / V * V : head;   // behind the whole groups of sixteen bytes
  for (int c = head + V * t; c < tail; c += V * threads)
    *reinterpret_cast<uint4*>(to + c) = from ? *reinterpret_cast<const uint4*>(from + c) : make_uint4(0, 0, 0, 0);
  for (int c = c0 + t; c < head; c += threads) to[c] = from ? from[c] : from_f<O>(0.f);
  for (int c = tail + t; c < c1; c += threads) to[c] = from ? from[c] : from_f<O>(0.f);
}

// Rows v0 .. v0 + rows - 1 of the table: the tokens of row r are places[edge[r] - lo .. edge[r + 1] - lo).  TPR threads a row; of its
// columns, every `of`-th part from `part` on.
template <typename T, typename O, int N, int TPR>
__device__ __forceinline__ void write_rows(const SumArgs& s, long long v0, int rows, const int* edge, const u32* places, int lo, int part, int of) {
  const long long vecs = s.cols / N;
  const int t = threadIdx.x % TPR;
  for (int r = threadIdx.x / TPR; r < rows; r += SUM_CTA / TPR) {
    const int from = edge[r], to = edge[r + 1];
    if ((from == to && s.leave) || to - from > s.most) continue;
    if (N == 1 && from == to) {
      plain_row<O>(s, v0 + r, (int)(s.cols * part / of), (int)(s.cols * (part + 1) / of), t, TPR);
      continue;
    }
    if (N == 8 || vecs <= 2 * of * TPR) {
      for (long long c = part * TPR + t; c < vecs; c += of * TPR) {
        float acc[N];
        sum_rows<T, N, N == 8 && sizeof(T) == 4 ? 4 : 8>(s, places, from - lo, to - lo, c, acc);
        finish_row<O, N>(s, v0 + r, c, acc);
      }
    } else if constexpr (N == 1) {                  // single elements of a long row: eight columns at a time, or their latencies add up
      constexpr int C = 8;
      const int cols = (int)s.cols, step = of * TPR;
      const O* const from_row = s.base ? (const O*)s.base + (v0 + r) * s.base_stride : nullptr;
      O* const to_row = (O*)s.dtable + (v0 + r) * s.dtable_stride;
      for (int c = part * TPR + t; c < cols; c += C * step) {
        float acc[C], base[C];
#pragma unroll
        for (int k = 0; k < C; ++k) {
          acc[k] = base[k] = 0.f;
          if (from_row && c + k * step < cols) base[k] = to_f(from_row[c + k * step]);
        }
#pragma unroll 2
        for (int i = from - lo; i < to - lo; ++i) {
          const T* const row = (const T*)s.dout + (long long)places[i] * s.dout_stride;
#pragma unroll
          for (int k = 0; k < C; ++k)
            if (c + k * step < cols) acc[k] += to_f(row[c + k * step]);
        }
#pragma unroll
        for (int k = 0; k < C; ++k)
          if (c + k * step < cols) to_row[c + k * step] = from_f<O>(from_row ? fmaf(acc[k], s.scale, base[k]) : acc[k] * s.scale);
      }
    }
  }
}

// The first CTAs take a window of the sorted tokens each (and a slice of its columns), for ids with more than `most` tokens; the
// others `rows` rows of the table.  TPR threads a row.
template <typename T, typename O, int N, int TPR>
__global__ void __launch_bounds__(SUM_CTA) k_embedding_sum(SumArgs s) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long vecs = s.cols / N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ int edge[SUM_ROWS + 1];
  __shared__ u32 staged[SUM_STAGE];
  __shared__ __align__(16) float shared[SUM_CTA * N];
  const unsigned long_ctas = (unsigned)s.windows * s.slices;
  if (blockIdx.x < long_ctas) {
    const int w = (int)(blockIdx.x / s.slices), lo = w * s.most, hi = min(s.n, lo + s.most);
    const int slice = (int)(blockIdx.x % s.slices);
    // Two runs at most are long and reach into a window: the one its first token belongs to and, another one or the same, the one that goes on
    // behind it.  A run is longer than `most` where the key `most` places before its end, or behind its start, is the same.
    const u32 key = __ldcg(s.keys + (warp ? hi - 1 : lo));
    const bool goes_on = hi < s.n && __ldcg(s.keys + hi) == __ldcg(s.keys + hi - 1);
    if (warp == 0) {
      const int end = lower_bound_warp(s.keys, lo, hi, key + 1);
      bool longer = end == hi && goes_on;
      if (!longer && end - s.most - 1 >= 0) longer = __ldcg(s.keys + end - s.most - 1) == key;
      if (lane == 0) {
        edge[0] = lo;
        edge[1] = longer && (long long)key < s.vocab ? end : lo;
        edge[4] = end == hi;
      }
    } else if (warp == 1) {
      const int start = lower_bound_warp(s.keys, lo, hi, key);
      const bool longer = goes_on && start + s.most < s.n && __ldcg(s.keys + start + s.most) == key;
      if (lane == 0) {
        edge[2] = start;
        edge[3] = longer && (long long)key < s.vocab ? hi : start;
      }
    }
    __syncthreads();
    for (int k = 0; k < 2; ++k) {
      const int from = edge[2 * k], to = edge[2 * k + 1];
      if (to <= from || (k && edge[4])) continue;                        // one run over the whole window: once
      float* const part = s.part + (2ll * w + k) * s.part_stride;
      if (vecs <= SUM_CTA / 2) {                      // groups of threads take parts of the tokens, in order
        int wide = 8;
        while (wide < vecs) wide *= 2;
        const int groups = SUM_CTA / wide, group = threadIdx.x / wide, c = threadIdx.x % wide;
        float acc[N];
        if (c < vecs) {
          sum_rows<T, N, 4>(s, s.places, from + (int)((long long)(to - from) * group / groups), from + (int)((long long)(to - from) * (group + 1) / groups), c, acc);
          store_part(shared + (group * wide + c) * N, acc);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < (int)vecs * N; e += SUM_CTA) {
          float sum = 0.f;
          for (int i = 0; i < groups; ++i) sum += shared[i * wide * N + e];
          __stcg(part + e, sum);
        }
        __syncthreads();
        continue;
      }
      for (long long c = (long long)slice * SUM_CTA + threadIdx.x; c < vecs; c += (long long)s.slices * SUM_CTA) {
        float acc[N];
        sum_rows<T, N, 4>(s, s.places, from, to, c, acc);
        store_part(part + c * N, acc);
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
  write_rows<T, O, N, TPR>(s, v0, rows, edge, stage ? staged : s.places + lo, lo, 0, 1);
}

// Few tokens: no sort, no search.  Every CTA looks at all of them, in order, keeps those of its rows, and puts them in the rows' order; one kernel
// instead of three, 24 -> 13 us for 1023 tokens and 1001 rows of 333.
constexpr int FEW_TOKENS = 1024, FEW_EACH = FEW_TOKENS / SUM_CTA, FEW_COLS = 1024;   // an id's tokens are one CTA's work there

template <typename T, typename O, int N, int TPR>
__global__ void __launch_bounds__(SUM_CTA) k_embedding_sum_few(SumArgs s, const void* ids, int id_bytes, const uint8_t* mask) {
  constexpr int WARPS = SUM_CTA / 32;
  __shared__ int count[FEW_EACH][WARPS], edge[SUM_ROWS + 1];
  __shared__ u32 found[FEW_TOKENS], staged[FEW_TOKENS];   // row in the CTA << 16 | token; tokens by row
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long v0 = (long long)blockIdx.x * s.rows;
  const int rows = (int)min((long long)s.rows, s.vocab - v0);
  u32 hit[FEW_EACH];
  int row[FEW_EACH];
#pragma unroll
  for (int k = 0; k < FEW_EACH; ++k) {
    const int i = k * SUM_CTA + threadIdx.x;
    const u32 key = i < s.n ? key_of(ids, id_bytes, mask, s.vocab, i) : (u32)s.vocab;
    row[k] = (long long)key >= v0 && (long long)key < v0 + rows ? (int)(key - v0) : -1;
    hit[k] = __ballot_sync(0xffffffffu, row[k] >= 0);
    if (lane == 0) count[k][warp] = __popc(hit[k]);
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int k = 0; k < FEW_EACH; ++k) {
    int at = 0;
    for (int w = 0; w < WARPS; ++w) {
      if (w == warp) at = total;
      total += count[k][w];
    }
    if (row[k] >= 0) found[at + __popc(hit[k] & ((1u << lane) - 1))] = (u32)row[k] << 16 | (u32)(k * SUM_CTA + threadIdx.x);
  }
  __syncthreads();
  for (int r = warp; r < rows; r += WARPS) {              // how many tokens the rows before have, and the row's own in order
    int before = 0;
    for (int i = lane; i < total; i += 32) before += (int)(found[i] >> 16) < r;
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) edge[r] = before;
    for (int i0 = 0; i0 < total; i0 += 32) {
      const u32 e = i0 + lane < total ? found[i0 + lane] : 0xffffffffu;
      const u32 mine = __ballot_sync(0xffffffffu, (int)(e >> 16) == r && i0 + lane < total);
      if (mine >> lane & 1) staged[before + __popc(mine & ((1u << lane) - 1))] = e & 0xffffu;
      before += __popc(mine);
    }
  }
  if (threadIdx.x == 0) edge[rows] = total;
  __syncthreads();
  write_rows<T, O, N, TPR>(s, v0, rows, edge, staged, 0, (int)blockIdx.y, (int)gridDim.y);
}

// Adds the windows of a long run, in order, by the CTAs of the window in which it begins (in which no second one can begin:
// it would have to end there, and be short).
template <typename O, int N>
__global__ void __launch_bounds__(SUM_CTA) k_embedding_join(SumArgs s) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int w = (int)blockIdx.x, lo = w * s.most, hi = min(s.n, lo + s.most);
  __shared__ int ends[2];
  const u32 key = __ldcg(s.keys + hi - 1);
  if (hi == s.n || __ldcg(s.keys + hi) != key) return;   // the run ends here, so it is short
  if (threadIdx.x < 64) {
    const bool behind = threadIdx.x >= 32;                // the run's beginning, its end
    const int e = behind ? lower_bound_warp(s.keys, hi - 1, s.n, key + 1) : lower_bound_warp(s.keys, lo, hi, key);
    if ((threadIdx.x & 31) == 0) ends[behind] = e;
  }
  __syncthreads();
  const int a = ends[0], b = ends[1];
  // a run that begins in front of the window is another window's
  if (a == lo && lo > 0 && __ldcg(s.keys + lo - 1) == key) return;
  if (b - a <= s.most || (long long)key >= s.vocab) return;
  const int last = (b - 1) / s.most;
  const long long vecs = s.cols / N;
  for (long long c = (long long)blockIdx.y * SUM_CTA + threadIdx.x; c < vecs; c += (long long)gridDim.y * SUM_CTA) {
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
#pragma unroll 8
    for (int i = w; i <= last; ++i) {
      // the run is its window's first one unless it begins behind the window's first token
      float v[N];
      load_part(s.part + (2ll * i + (i == w && a > lo ? 1 : 0)) * s.part_stride + c * N, v);
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] += v[j];
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
int sum_launch(SumArgs s, const adacgd_embedding_backward_args& a, const Where& at) {
  const long long slices = (s.cols / N + SUM_CTA - 1) / SUM_CTA;
  s.slices = (int)(slices < 16 ? slices : 16);
  // Rows of the table one after the other are a chain of memory latencies: few of them a CTA as long as that gives every SM only a
  // few CTAs.
  s.rows = SUM_ROWS;
  while (s.rows > SUM_CTA / TPR && s.rows > 1 && s.vocab < 8ll * s.rows * at.sms) s.rows /= 2;
  if (s.few) {
    const long long ctas = (s.vocab + s.rows - 1) / s.rows;
    long long parts = (s.cols / N + TPR - 1) / TPR, most = 16ll * at.sms / ctas;   // of the columns, where that does not make too many CTAs
    if (parts > most) parts = most;
    k_embedding_sum_few<T, O, N, TPR><<<dim3((unsigned)ctas, (unsigned)(parts < 1 ? 1 : parts)), SUM_CTA, 0, at.stream>>>(s, a.ids, (int)a.id_bytes, a.mask);
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  }
  const long long blocks = (long long)s.windows * s.slices + (s.vocab + s.rows - 1) / s.rows;
  if (!launch_dependent(k_embedding_sum<T, O, N, TPR>, dim3((unsigned)blocks), SUM_CTA, at, s)) return -1;
  if (!s.windows) return 1;
  return launch_dependent(k_embedding_join<O, N>, dim3((unsigned)s.windows, (unsigned)s.slices), SUM_CTA, at, s) ? 2 : -1;
}
template <typename T, typename O, int N>
int sum_by_width(const SumArgs& s, const adacgd_embedding_backward_args& a, const Where& at) {
  const long long vecs = s.cols / N;
  if (vecs <= 8) return sum_launch<T, O, N, 8>(s, a, at);
  if (vecs <= 32) return sum_launch<T, O, N, 32>(s, a, at);
  if (vecs <= 64) return sum_launch<T, O, N, 64>(s, a, at);
  return sum_launch<T, O, N, 256>(s, a, at);
}
template <typename T, typename O>
int sum_t(const SumArgs& s, const adacgd_embedding_backward_args& a, const Where& at) {
  const bool runs = whole_runs<T>(s.dout, s.dout_stride, s.n, s.cols) && whole_runs<O>(s.base, s.base_stride, s.vocab, s.cols) &&
                    whole_runs<O>(s.dtable, s.dtable_stride, s.vocab, s.cols);
  return runs ? sum_by_width<T, O, 8>(s, a, at) : sum_by_width<T, O, 1>(s, a, at);
}

// Sorts the tokens into s->keys and s->places.
bool sort_tokens(const TrainScratch& ws, const adacgd_embedding_backward_args& a, const Where& at, SumArgs* s) {
  u32 *k0 = (u32*)ws.tok_a, *p0 = (u32*)ws.tok_b, *k1 = (u32*)ws.tok_c, *p1 = (u32*)ws.seq;
  s->keys = k1;
  s->places = p1;
  int bits = 1;
  while ((1ll << bits) <= a.vocab) ++bits;           // keys up to `vocab` itself
  const int passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
  // A warp takes at least 128 tokens and then up to 256 in its registers; more CTAs cost a little in the counts they exchange.
  int ctas = 1, warps = 1;
  while (ctas < SORT_CTAS && s->n > 2048 * ctas) ctas *= 2;
  while (warps < SORT_WARPS && s->n > 128 * ctas * warps) warps *= 2;
  const bool keep = s->n <= 32ll * (SORT_KEEP - 1) * ctas * warps;   // shares differ by one
  auto sort = keep ? k_sort_ids<true> : k_sort_ids<false>;
  static std::atomic<int> table[2][TRAIN_DEVICES];
  if (resident_ctas(sort, table[keep], at.device, SORT_CTA, (int)sizeof(SortSmem)) < 1) return false;
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
  return cudaLaunchKernelEx(&cfg, sort, a.ids, (int)a.id_bytes, a.mask, (long long)a.vocab, s->n, passes, warps, k0, p0, k1, p1) == cudaSuccess;
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
  s.part = ws.norm_part;
  s.part_stride = a.cols;                            // at most max_cols; whole runs stay aligned
  s.most = (s.n + MAX_WINDOWS - 1) / MAX_WINDOWS;
  if (s.most < SUM_MIN) s.most = SUM_MIN;
  s.windows = s.n > s.most ? (s.n + s.most - 1) / s.most : 0;
  s.few = s.n <= FEW_TOKENS && s.cols <= FEW_COLS;
  if (s.few) s.most = FEW_TOKENS;
  else if (!sort_tokens(ws, a, at, &s)) return -1;
  int n = -1;
  if (a.table_dtype == ADACGD_F32 && a.dtype == ADACGD_F16) n = sum_t<__half, float>(s, a, at);
  else if (a.table_dtype == ADACGD_F32 && a.dtype == ADACGD_BF16) n = sum_t<__nv_bfloat16, float>(s, a, at);
  else if (a.dtype == ADACGD_F32) n = sum_t<float, float>(s, a, at);
  else if (a.dtype == ADACGD_F16) n = sum_t<__half, __half>(s, a, at);
  else n = sum_t<__nv_bfloat16, __nv_bfloat16>(s, a, at);
  return n < 0 || s.few ? n : n + 1;
}

}  // namespace adacgd
