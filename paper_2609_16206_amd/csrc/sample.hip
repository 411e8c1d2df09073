// rt_sample_tokens: one token per row of logits (temperature, top-k, top-p,
// min-p, then a draw by the running sum of the kept weights).
//
// Weights are w = 2^((l - l_max) log2(e) / T) in float64, held as integers in
// units of 2^-45: at most 2^18 of them add up in 64 bits without rounding, so
// no order of additions changes a sum, and the drawn token is the same however
// the work is cut.  The kept tokens are the front of the row's order by falling
// logit, lower index first, so they are given by a logit (its order key) and
// the last index that is kept among its equals.
//
// A row is cut into stretches of 2,048 elements, one a wave, four to a workgroup:
//   1. stats_kernel: every workgroup's largest logit (and its lowest index), the
//      smallest finite one, and maxima of small groups of tokens;
//   2. order_kernel, where the call has top-k or top-p:
//      - top_k <= kFewTokens: the k-th largest of the groups' maxima is a lower
//        bound of the k-th largest logit; the tokens above it, not many more
//        than k, go to a list, on which pick_kernel does everything else;
//      - otherwise counts, or sums of weights, over 4,096 ranges of logits;
//   3. weigh_kernel: the sums of the kept weights over the stretches, where the
//      range in which top-k or top-p ends counts only by a list of its tokens;
//   4. pick_kernel: the end within that list, the stretch the draw falls in, and
//      the token within the stretch.
// Bound by its passes over the row, the first at HBM's rate and the others from
// the last-level cache, by the weights' float64 operations (about 20 a logit), and for
// few rows by the chain of small kernels.  512 x 100,003 float32 logits by temperature
// alone 104 us (40 + 53 + 10 for kernels 1, 3, 4; one read at 4.9 TB/s is 42); 96 x
// 151,936 bfloat16 of every kind of setting 73 us; one row of 32,000 with top-k, top-p
// and min-p 28 us.
//
// What no list holds is left to whole_row, one workgroup that goes over the row
// again for every step: top_k beyond kFewTokens together with top-p (one row of
// 151,936 bfloat16 176 us, 96 rows 205 us, where top_k 50 takes 37 and 60),
// thousands of equal logits at the border (342 and 414 us), and more tokens than a
// list holds in fewer groups than top_k (a mask that leaves a block of 5,000, top_k
// 200: 96 and 141 us).
#include <algorithm>
#include <type_traits>

#include "serve_device.h"

namespace rt {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 4096;        // ranges of logits
constexpr int kStretch = 2048;     // elements of a wave's part of a row
constexpr int kSegThreads = 256;   // four stretches
constexpr int kMaxSegs = 34;       // 262,144 elements and a partial chunk at each end
constexpr int kList = 1024;
constexpr int kFewTokens = 256;
constexpr int kRows = 2048;        // rows of a launch: bounds the workspace
constexpr double kUnit = 35184372088832.0;  // 2^45
constexpr float kInf = __builtin_inff();

// Order of a float's bits as an unsigned number (no NaN); the zeros tie.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
constexpr uint32_t kNoKey = 0x007fffffu;  // order_key(-inf): no key of a masked token lies above
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

// Weights of a row: 2^x = 2^(i / 256) 2^r, i = round(256 x), |r| <= 1 / 512; the
// first factor from a table and an exponent, the second by its Taylor series
// to r^4 (the next term is below 2^-54).  32 entries in banks of their own and a
// term more: 111 us for 512 x 100,003 logits in place of 106.
constexpr int kTable = 256;
__device__ __forceinline__ double table_entry(int j) { return exp2((double)j / kTable) * kUnit; }

struct Weigher {
  const double* table;  // [256] 2^(j / 256) units, in LDS
  double top, scale;    // the largest logit; log2(e) / T
  double least;         // differences to the largest logit are taken as no less: 2^-1000
  float lmax;
  float low;  // logits below weigh nothing, and may be taken for this one: -inf if no float serves

  // Infinite logits share the row: they become 10^39, beyond every finite one,
  // and whatever lies below them has no weight.  At an infinite temperature
  // every finite logit weighs the same: 10^-300 times any difference is 0.
  __device__ __forceinline__ Weigher(const double* table, float lmax, float t)
      : table(table), top(lmax == kInf ? 1e39 : (double)lmax),
        scale(lmax == kInf ? 1.0 : fmax(1.4426950408889634074 / (double)t, 1e-300)), least(-1000.0 / scale), lmax(lmax) {
    // (60 powers of two down, well below 2^-46, where weights round to 0)
    low = (float)(top - 60.0 / scale);
    const double x = ((double)low - top) * scale;
    if (lmax == kInf || !(x >= -1000.0 && x <= -47.0)) low = -kInf;
  }

  // 2^(d scale) in units of 2^-45, not rounded; d scale >= -1000 (no branches:
  // neighbours overlap)
  __device__ __forceinline__ double power(double d) const {
    constexpr double kRound = 26388279066624.0;  // 1.5 * 2^44, whose last bit is 1 / 256
    const double u = __builtin_fma(d, scale, kRound);
    const int i = (int)(uint32_t)__double_as_longlong(u);
    const double r = __builtin_fma(d, scale, -(u - kRound));
    double p = __builtin_fma(r, 9.618129107628477e-3, 5.550410866482158e-2);  // ln(2)^n / n!
    p = __builtin_fma(r, p, 2.402265069591007e-1);
    p = __builtin_fma(r, p, 6.931471805599453e-1);
    const double t = table[i & (kTable - 1)];
    const double w = __builtin_fma(t * r, p, t);
    // times 2^(i >> 8), which stays a normal number
    return __longlong_as_double(__double_as_longlong(w) + ((int64_t)((i & -kTable) << (20 - 8)) << 32));
  }
  __device__ __forceinline__ double units(float l) const { return power(fmax(fmin((double)l, 1e39) - top, least)); }
  // The same for rows with a `low`, but for logits below it (another number that
  // rounds to 0).
  __device__ __forceinline__ double units_above(float l) const { return power((double)fmaxf(l, low) - top); }
  template <bool kLow>
  __device__ __forceinline__ double units_of(float l) const {
    return kLow ? units_above(l) : units(l);
  }
  static __device__ __forceinline__ uint64_t round(double w) {
    return (uint64_t)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull;  // + 2^52: to nearest
  }
  __device__ __forceinline__ uint64_t operator()(float l) const { return round(units(l)); }
};

template <class V>
__device__ __forceinline__ V wave_sum(V x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// f(index, logit) for the elements of 16-byte chunks [c0, c1) of a row, chunk
// c0 + lane first, `lanes` apart, kAhead loads under way.  Chunk 0 begins at the
// 16-byte border at or before the row's first element.
template <class T>
struct Row {
  const T* p;
  int n, lead;  // elements before the row in chunk 0
  static constexpr int kE = 16 / sizeof(T);

  __device__ __forceinline__ Row(const void* base, int64_t offset, int n)
      : p((const T*)base + offset), n(n), lead((int)(((uintptr_t)p & 15) / sizeof(T))) {}
  __device__ __forceinline__ int chunks() const { return (lead + n + kE - 1) / kE; }

  // Chunks c, c + lanes, ... below c1, as far as they lie in the row: loaded,
  // and used (what lies only partly in it is loaded there).
  template <int kN>
  __device__ __forceinline__ void load(u32x4 (&v)[kN], int c, int c1, int lanes) const {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int at = (c + j * lanes) * kE - lead;
      if (c + j * lanes < c1 && at >= 0 && at + kE <= n) v[j] = *(const u32x4*)(p + at);
    }
  }
  template <int kN, class F>
  __device__ __forceinline__ void use(const u32x4 (&v)[kN], int c, int c1, int lanes, F f) const {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int at = (c + j * lanes) * kE - lead;
      if (c + j * lanes >= c1) break;
      if (at >= 0 && at + kE <= n) {
        typedef T vec __attribute__((ext_vector_type(kE)));
        const vec x = __builtin_bit_cast(vec, v[j]);
#pragma unroll
        for (int e = 0; e < kE; ++e) f(at + e, (float)x[e]);
      } else {
        for (int e = 0; e < kE; ++e)
          if (at + e >= 0 && at + e < n) f(at + e, (float)p[at + e]);
      }
      __builtin_amdgcn_sched_barrier(0);  // (one chunk's work at a time: registers)
    }
  }
  template <int kAhead, class F>
  __device__ __forceinline__ void each(int c0, int c1, int lane, int lanes, F f) const {
    for (int c = c0 + lane; c < c1; c += kAhead * lanes) {
      u32x4 v[kAhead];
      load(v, c, c1, lanes);
      use(v, c, c1, lanes, f);
    }
  }
};

// The kept tokens: keys above `key`, and of its equals those up to `last`.  Masked
// tokens (-inf) stand last in the order and weigh nothing: they are in no list and
// no count, or a mask that leaves few tokens would fill both.
struct Kept {
  uint32_t key = kNoKey;
  int last = -1;
  __device__ __forceinline__ bool has(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

struct List {
  uint64_t hist[kBins];
  uint32_t list_key[kList];
  int list_idx[kList];
  uint64_t list_w[kList];
};
struct NoList {};

template <bool kOrder>  // the call has top-k or top-p settings
struct Shared : std::conditional_t<kOrder, List, NoList> {
  uint64_t sums[4 * kMaxSegs];
  int starts[kMaxSegs];
  double table[kTable];
  uint64_t part[kWaves];
  int n_list, found;
  uint32_t min_key, max_key;
  uint64_t above;
  int bin;
};

// The block's tokens with test(key, index, logit), into the list; more than
// kList are counted only.  Returns the count, with the smallest and largest of
// their keys in sh.min_key, sh.max_key.
template <class T, class F>
__device__ __forceinline__ int gather(const Row<T>& row, Shared<true>& sh, F test) {
  const int tid = (int)threadIdx.x;
  __syncthreads();
  if (tid == 0) sh.n_list = 0, sh.min_key = 0xffffffffu, sh.max_key = 0;
  __syncthreads();
  row.template each<4>(0, row.chunks(), tid, kThreads, [&](int i, float l) {
    const uint32_t k = order_key(l);
    if (!test(k, i, l)) return;
    const int at = atomicAdd(&sh.n_list, 1);
    if (at < kList) sh.list_key[at] = k, sh.list_idx[at] = i;
    if (k < sh.min_key) atomicMin(&sh.min_key, k);
    if (k > sh.max_key) atomicMax(&sh.max_key, k);
  });
  __syncthreads();
  return sh.n_list;
}

// How far below the largest logit ranges are laid.  Counts: to the smallest.
// Sums: the n tokens further down than log2(2 n / (1 - p)) powers of two have
// together less than half of the share 1 - p that top-p leaves out, so the end
// of top-p does not lie among them.
__device__ __forceinline__ float count_spread(float lmax, float low) { return lmax == kInf ? 0.0f : lmax - low; }
__device__ __forceinline__ float sum_spread(float lmax, float low, float tf, float pf, int n) {
  const float powers = fminf(46.0f, __log2f((float)n) + 1.5f - __log2f(fmaxf(1.0f - pf, 1e-9f)));
  return lmax == kInf ? 0.0f : fminf(lmax - low, powers * 0.6931472f * tf);
}

// The range of a logit, `bins` of them over `spread`.  (Both infinite: 0; an
// infinite difference, or 0 times it: the last.)
__device__ __forceinline__ int range_of(float l, float lmax, float s, int bins) {
  return (int)fminf(l == lmax ? 0.0f : (lmax - l) * s, (float)(bins - 1));
}

// Cut `kept` at the first token, in order, at which the running count (kMass
// false, goal: top_k) or sum of weights (goal: top_p, a share of the whole)
// reaches its goal.
template <class T, bool kMass>
__device__ __forceinline__ void cut(const Row<T>& row, Shared<true>& sh, const Weigher& weigh, double goal, float spread,
                                    Kept& kept) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float s = spread > 0.0f ? (float)kBins / spread : 0.0f;
  const float lmax = weigh.lmax;
  auto bin_of = [&](float l) { return range_of(l, lmax, s, kBins); };
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
  __syncthreads();
  row.template each<4>(0, row.chunks(), tid, kThreads, [&](int i, float l) {
    if (!kept.has(order_key(l), i)) return;
    const uint64_t w = kMass ? weigh(l) : 1;
    if (w) atomicAdd((unsigned long long*)&sh.hist[bin_of(l)], (unsigned long long)w);
  });
  __syncthreads();
  // the bin in which the running sum reaches the goal: four bins a thread
  constexpr int kMine = kBins / kThreads;
  uint64_t h[kMine], run = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) run += h[j] = sh.hist[kMine * tid + j];
  const uint64_t mine = run;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  if (lane == 63) sh.part[wave] = run;
  if (tid == 0) sh.bin = -1;
  __syncthreads();
  uint64_t total = 0;
  for (int v = 0; v < kWaves; ++v) {
    if (v < wave) run += sh.part[v];
    total += sh.part[v];
  }
  const double g = kMass ? goal * (double)total : goal;
  uint64_t above = run - mine;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    if ((double)above < g && (double)(above + h[j]) >= g) sh.bin = kMine * tid + j, sh.above = above;
    above += h[j];
  }
  __syncthreads();
  const int bin = sh.bin;
  if (bin < 0) return;  // (the goal lies behind all of them)
  above = sh.above;
  auto inside = [&](uint32_t k, int i, float l) { return bin_of(l) == bin && kept.has(k, i); };
  int n = gather(row, sh, inside);
  uint32_t lo = sh.min_key, hi = sh.max_key;
  if (n == 0) return;  // (nothing is left to cut)
  // More than the list holds: halve the range of keys, on counts or sums
  // above its middle, until the rest fits or is one key.
  while (n > kList && lo != hi) {
    const uint32_t mid = lo + (hi - lo) / 2;  // keys > mid are the upper half
    uint64_t w = 0;
    row.template each<1>(0, row.chunks(), tid, kThreads, [&](int i, float l) {
      const uint32_t k = order_key(l);
      if (k > mid && k <= hi && inside(k, i, l)) w += kMass ? weigh(l) : 1;
    });
    w = wave_sum(w);
    __syncthreads();
    if (lane == 0) sh.part[wave] = w;
    __syncthreads();
    w = 0;
    for (int v = 0; v < kWaves; ++v) w += sh.part[v];
    if ((double)(above + w) >= g) {
      lo = mid + 1;
    } else {
      above += w;
      hi = mid;
    }
    n = gather(row, sh, [&](uint32_t k, int i, float l) { return k >= lo && k <= hi && inside(k, i, l); });
    if (n == 0) return;
    lo = sh.min_key, hi = sh.max_key;
  }
  if (lo == hi) {
    // Equals: how many of them are needed, and the index of the last.
    const uint64_t each = kMass ? weigh(key_logit(lo)) : 1;
    uint64_t c = (uint64_t)n;
    if (each) {
      c = (uint64_t)fmin(fmax((g - (double)above) / (double)each, 1.0), (double)n);
      while (c < (uint64_t)n && (double)(above + c * each) < g) ++c;
      while (c > 1 && (double)(above + (c - 1) * each) >= g) --c;
    }
    int last = lo == kept.key ? kept.last : 0x7fffffff;
    if (c < (uint64_t)n) {
      // counts of the equals over the waves' stretches, then within one
      const int per = (row.chunks() + kWaves - 1) / kWaves, c0 = wave * per, c1 = min(c0 + per, row.chunks());
      int mine = 0;
      row.template each<1>(c0, c1, lane, 64, [&](int i, float l) { mine += order_key(l) == lo && kept.has(lo, i); });
      mine = wave_sum(mine);
      __syncthreads();
      if (lane == 0) sh.part[wave] = (uint64_t)mine;
      __syncthreads();
      uint64_t before = 0;
      int v = 0;
      while (v < kWaves - 1 && before + sh.part[v] < c) before += sh.part[v++];
      if (wave == v) {
        int need = (int)(c - before);  // the need-th equal of the stretch
        const int e0 = max(c0 * Row<T>::kE - row.lead, 0), e1 = min(c1 * Row<T>::kE - row.lead, row.n);
        for (int e = e0; e < e1; e += 64) {
          const bool eq = e + lane < e1 && order_key((float)row.p[e + lane]) == lo && kept.has(lo, e + lane);
          const uint64_t m = __ballot(eq);
          const int cnt = __popcll(m);
          if (cnt >= need) {
            if (eq && __popcll(m & ((2ull << lane) - 1)) == need) sh.found = e + lane;
            break;
          }
          need -= cnt;
        }
      }
      __syncthreads();
      last = sh.found;
    }
    kept.key = lo;
    kept.last = last;
    return;
  }
  // Few: every listed token finds what stands before it.
  const uint32_t k = tid < n ? sh.list_key[tid] : 0;
  const int idx = tid < n ? sh.list_idx[tid] : 0;
  const uint64_t w = tid < n ? (kMass ? weigh(key_logit(k)) : 1) : 0;
  __syncthreads();
  if (tid < n) sh.list_w[tid] = w;
  if (tid == 0) sh.found = -1;
  __syncthreads();
  uint64_t before = above;
  for (int j = 0; j < n; ++j) {
    const uint32_t kj = sh.list_key[j];
    if (kj > k || (kj == k && sh.list_idx[j] < idx)) before += sh.list_w[j];
  }
  // the last kept token: what stands before it is short of the goal, with it no more
  if (tid < n && (double)before < g && (double)(before + w) >= g) sh.found = tid;
  __syncthreads();
  const int at = sh.found;
  if (at < 0) return;  // (the goal lies behind all of them)
  kept.key = sh.list_key[at];
  kept.last = sh.list_idx[at];
}

// Everything for one row by one workgroup, from the kept tokens on.
template <class T>
__device__ __forceinline__ void whole_row(const SampleArgs& a, const Row<T>& row, Shared<true>& sh, const Weigher& weigh,
                                          int64_t r, int kk, float pf, float tf, float low, int besti, double floor_w) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, n = row.n;
  const float lmax = weigh.lmax;
  Kept kept;
  if (kk > 0 && kk < n) cut<T, false>(row, sh, weigh, (double)kk, count_spread(lmax, low), kept);
  if (pf < 1.0f) cut<T, true>(row, sh, weigh, (double)pf, sum_spread(lmax, low, tf, pf, n), kept);

  const int per = (row.chunks() + kWaves - 1) / kWaves;
  auto kept_units = [&](int i, float l) -> uint64_t {
    if (!kept.has(order_key(l), i)) return 0;
    const double w = weigh.units(l);
    return w >= floor_w || i == besti ? Weigher::round(w) : 0;
  };
  uint64_t sum = 0;
  row.template each<4>(min(wave * per, row.chunks()), min((wave + 1) * per, row.chunks()), lane, 64,
           [&](int i, float l) { sum += kept_units(i, l); });
  sum = wave_sum(sum);
  __syncthreads();
  if (lane == 0) sh.part[wave] = sum;
  __syncthreads();
  uint64_t total = 0;
  for (int v = 0; v < kWaves; ++v) total += sh.part[v];
  uint64_t goal = __umul64hi(total, a.bits[r]);
  int v = 0;
  while (v < kWaves - 1 && goal >= sh.part[v]) goal -= sh.part[v++];
  // the stretch's tokens, a run of them a thread
  const int e0 = max(v * per * Row<T>::kE - row.lead, 0), e1 = min((v + 1) * per * Row<T>::kE - row.lead, n);
  const int each = (e1 - e0 + kThreads - 1) / kThreads;
  const int i0 = min(e0 + tid * each, e1), i1 = min(i0 + each, e1);
  sum = 0;
  for (int i = i0; i < i1; ++i) sum += kept_units(i, (float)row.p[i]);
  uint64_t run = sum;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();
  if (lane == 63) sh.part[wave] = run;
  __syncthreads();
  for (int u = 0; u < wave; ++u) run += sh.part[u];
  if (run > goal && run - sum <= goal) {
    uint64_t at = run - sum;
    for (int i = i0; i < i1; ++i) {
      at += kept_units(i, (float)row.p[i]);
      if (at > goal) {
        a.out[r] = i;
        break;
      }
    }
  }
}

// The workspace, in this order (the parts of top-k and top-p only where the call
// has them).
struct Stats {
  uint32_t best;
  int32_t besti;
  float low;
  uint32_t nan;
};
struct Token {
  uint32_t key;
  int32_t idx;
};
struct Ws {
  Stats* stats;     // [rows][segs]
  uint64_t* sums;   // [rows][4 segs]
  uint32_t* count;  // [rows][segs] tokens listed
  uint64_t* hist;   // [rows][kBins]
  uint32_t* group;  // [rows][segs * kSegThreads / lanes] maxima of groups of `lanes` lanes' tokens
  Token* list;      // [rows][segs][cap]
  int segs, lanes, cap;
};

__host__ __device__ inline int segments(int vocab) {
  return (vocab + 7 + 4 * kStretch - 1) / (4 * kStretch);  // chunk 0 may hold 7 elements before the row
}

__host__ __device__ inline Ws workspace(char* p, int64_t rows, int vocab) {
  Ws w;
  w.segs = segments(vocab);
  w.lanes = w.segs <= 8 ? 1 : 4;
  w.cap = kList / (w.segs < 4 ? w.segs : 4);
  const int64_t n = rows * w.segs;
  w.stats = (Stats*)p;
  w.sums = (uint64_t*)(w.stats + n);
  w.hist = w.sums + 4 * n;
  w.list = (Token*)(w.hist + rows * kBins);
  w.group = (uint32_t*)(w.list + n * w.cap);
  w.count = w.group + n * (kSegThreads / w.lanes);
  return w;
}
inline int64_t workspace_bytes(int64_t rows, int vocab) {
  char* const base = (char*)256;
  const Ws w = workspace(base, rows, vocab);
  return (char*)(w.count + rows * w.segs) - base;
}

// What a row asks for, from its parts' stats.
enum Kind { kDone, kFew, kPlain, kSums, kCounts, kWhole };
struct Ask {
  uint32_t best;
  int besti, kk;
  float low, lmax, tf, pf, mf;
  Kind kind;
  int32_t token;  // kDone
};

__device__ __forceinline__ Ask ask_of(const SampleArgs& a, const Ws& w, int64_t r) {
  const int lane = (int)threadIdx.x & 63;
  Ask q;
  q.best = 0;
  q.besti = 0x7fffffff;
  q.low = kInf;
  bool nan = false;
  if (lane < w.segs) {
    const Stats st = w.stats[r * w.segs + lane];
    q.best = st.best, q.besti = st.besti, q.low = st.low, nan = st.nan;
  }
  for (int o = 32; o; o >>= 1) {
    const uint32_t k = __shfl_xor(q.best, o);
    const int i = __shfl_xor(q.besti, o);
    q.low = fminf(q.low, __shfl_xor(q.low, o));
    if (k > q.best || (k == q.best && i < q.besti)) q.best = k, q.besti = i;
  }
  nan = __ballot(nan) != 0;
  q.lmax = key_logit(q.best);
  q.tf = a.temperature ? a.temperature[r] : 1.0f;
  q.pf = a.top_p ? a.top_p[r] : 1.0f;
  q.mf = a.min_p ? a.min_p[r] : 0.0f;
  q.kk = a.top_k ? a.top_k[r] : 0;
  if (q.kk <= 0 || q.kk >= a.vocab) q.kk = 0;
  q.token = q.besti;
  if (nan || q.lmax == -kInf || !(q.tf >= 0.0f) || q.pf != q.pf || q.mf != q.mf) {
    q.kind = kDone;
    q.token = -1;
  } else if (q.tf == 0.0f || q.pf <= 0.0f || q.kk == 1) {  // the first token alone
    q.kind = kDone;
  } else if (q.kk > 0 && q.kk <= kFewTokens) {
    q.kind = kFew;
  } else if (q.kk > 0) {
    q.kind = q.pf < 1.0f ? kWhole : kCounts;
  } else {
    q.kind = q.pf < 1.0f ? kSums : kPlain;
  }
  return q;
}

__device__ __forceinline__ Weigher weigher_of(const Ask& q, const double* table) {
  return Weigher(table, q.lmax, q.tf);
}
__device__ __forceinline__ float range_scale(const Ask& q, int n) {
  const float spread =
      q.kind == kCounts ? count_spread(q.lmax, q.low) : sum_spread(q.lmax, q.low, q.tf, q.pf, n);
  return spread > 0.0f ? (float)kBins / spread : 0.0f;
}
__device__ __forceinline__ double floor_of(const Ask& q) { return fmin((double)q.mf, 4.0) * kUnit; }  // min-p, in units

// The range in which the running count, or sum, from the front reaches the
// goal, what stands before it, and the goal; range kBins if none does.
struct Border {
  int bin;
  uint64_t above;
  double goal;
};
template <int kN>  // threads
__device__ __forceinline__ Border border_of(const uint64_t* hist, const Ask& q, uint64_t* part, Border* out) {
  constexpr int kMine = kBins / kN;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t h[kMine], run = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) run += h[j] = hist[kMine * tid + j];
  const uint64_t mine = run;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = run;
  __syncthreads();
  uint64_t total = 0;
  for (int v = 0; v < kN / 64; ++v) {
    if (v < wave) run += part[v];
    total += part[v];
  }
  const double g = q.kind == kSums ? (double)q.pf * (double)total : (double)q.kk;
  if (tid == 0) *out = Border{kBins, 0, g};
  __syncthreads();
  uint64_t above = run - mine;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    if ((double)above < g && (double)(above + h[j]) >= g) *out = Border{kMine * tid + j, above, g};
    above += h[j];
  }
  __syncthreads();
  return *out;
}

template <class T, bool kOrder>
__global__ __launch_bounds__(kSegThreads) void stats_kernel(SampleArgs a) {
  const Ws w = workspace(a.ws, a.n_rows, a.vocab);
  const int64_t r = blockIdx.y;
  const int seg = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<T> row(a.logits, r * a.stride, a.vocab);
  constexpr int kC = kStretch / Row<T>::kE;
  const int c0 = (4 * seg + wave) * kC;
  uint32_t best = 0;
  float low = kInf;
  int besti = 0x7fffffff;
  bool nan = false;
  row.template each<kC / 64>(c0, min(c0 + kC, row.chunks()), lane, 64, [&](int i, float l) {
    nan = nan || l != l;
    const uint32_t k = order_key(l);
    besti = k > best ? i : besti;
    best = max(best, k);
    low = l > -kInf ? fminf(low, l) : low;
  });
  if (kOrder) {
    uint32_t g = best;
    for (int o = 1; o < w.lanes; o <<= 1) g = max(g, (uint32_t)__shfl_xor(g, o));
    if (lane % w.lanes == 0) w.group[(r * w.segs + seg) * (kSegThreads / w.lanes) + tid / w.lanes] = g > kNoKey ? g : 0;
    // ranges start at 0
    const int per = (kBins + w.segs - 1) / w.segs;
    for (int i = seg * per + tid; i < min((seg + 1) * per, kBins); i += kSegThreads) w.hist[r * kBins + i] = 0;
  }
  for (int o = 32; o; o >>= 1) {
    const uint32_t k = __shfl_xor(best, o);
    const int i = __shfl_xor(besti, o);
    low = fminf(low, __shfl_xor(low, o));
    if (k > best || (k == best && i < besti)) best = k, besti = i;
  }
  nan = __ballot(nan) != 0;
  __shared__ Stats st[4];
  if (lane == 0) st[wave] = Stats{best, besti, low, nan};
  __syncthreads();
  if (tid == 0) {
    Stats all = st[0];
    for (int v = 1; v < 4; ++v) {
      if (st[v].best > all.best) all.best = st[v].best, all.besti = st[v].besti;  // (equals: the earlier stretch)
      all.low = fminf(all.low, st[v].low);
      all.nan |= st[v].nan;
    }
    w.stats[r * w.segs + seg] = all;
    if (kOrder) w.count[r * w.segs + seg] = 0;
  }
}

template <class T>
__global__ __launch_bounds__(kSegThreads) void order_kernel(SampleArgs a) {
  const Ws w = workspace(a.ws, a.n_rows, a.vocab);
  const int64_t r = blockIdx.y;
  const int seg = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Ask q = ask_of(a, w, r);
  if (q.kind != kFew && q.kind != kSums && q.kind != kCounts) return;
  const Row<T> row(a.logits, r * a.stride, a.vocab);
  constexpr int kC = kStretch / Row<T>::kE;
  const int c0 = (4 * seg + wave) * kC, c1 = min(c0 + kC, row.chunks());
  __shared__ double table[kTable];
  __shared__ uint64_t hist[kBins];
  __shared__ int part[2][4], filled[4];
  __shared__ int count;
  if (q.kind == kFew) {
    // the kk-th largest of the groups' maxima, to the 12 bits below their common
    // ones (cut off below)
    constexpr int kMost = (kMaxSegs * 64 + 255) / 256 > 8 ? (kMaxSegs * 64 + 255) / 256 : 8;
    const int n = w.segs * (kSegThreads / w.lanes);
    uint32_t k[kMost], bound = 0;
#pragma unroll
    for (int j = 0; j < kMost; ++j)
      k[j] = j * kSegThreads + tid < n ? w.group[r * (int64_t)n + j * kSegThreads + tid] : 0;
    // bits that all of them share need no search
    uint32_t any = 0, all = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < kMost; ++j)
      if (k[j]) any |= k[j], all &= k[j];
    for (int o = 32; o; o >>= 1) any |= __shfl_xor(any, o), all &= __shfl_xor(all, o);
    if (tid == 0) count = 0;
    if (lane == 0) part[0][wave] = (int)any, part[1][wave] = (int)all;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) any |= (uint32_t)part[0][v], all &= (uint32_t)part[1][v];
    __syncthreads();
    const int top = 31 - __clz((int)((any & ~all) | 1u));
    bound = top == 31 ? 0 : all & ~((2u << top) - 1);
    {
      // fewer groups than tokens asked for: no bound
      int c = 0;
#pragma unroll
      for (int j = 0; j < kMost; ++j) c += __popcll(__ballot(k[j] != 0));
      if (lane == 0) filled[wave] = c;
      __syncthreads();
      if (filled[0] + filled[1] + filled[2] + filled[3] < q.kk) bound = 0;
    }
    for (int bit = top; bit >= max(top - 11, 0); --bit) {
      const uint32_t to = bound | 1u << bit;
      int c = 0;
#pragma unroll
      for (int j = 0; j < kMost; ++j) c += __popcll(__ballot(k[j] >= to));
      if (lane == 0) part[bit & 1][wave] = c;
      __syncthreads();  // (the next round writes the other half)
      if (part[bit & 1][0] + part[bit & 1][1] + part[bit & 1][2] + part[bit & 1][3] >= q.kk) bound = to;
    }
    bound = max(bound, kNoKey + 1);
    Token* list = w.list + (r * w.segs + seg) * w.cap;
    row.template each<kC / 64>(c0, c1, lane, 64, [&](int i, float l) {
      const uint32_t key = order_key(l);
      if (key >= bound) {
        const int at = atomicAdd(&count, 1);
        if (at < w.cap) list[at] = Token{key, i};
      }
    });
    __syncthreads();
    if (tid == 0) w.count[r * w.segs + seg] = count;
    return;
  }
  if (tid < kTable) table[tid] = table_entry(tid);
  for (int i = tid; i < kBins; i += kSegThreads) hist[i] = 0;
  __syncthreads();
  const Weigher weigh = weigher_of(q, table);
  const float s = range_scale(q, a.vocab);
  if (q.kind == kSums)
    row.template each<kC / 128>(c0, c1, lane, 64, [&](int, float l) {
      const uint64_t x = Weigher::round(weigh.low > -kInf ? weigh.units_above(l) : weigh.units(l));
      if (x) atomicAdd((unsigned long long*)&hist[range_of(l, q.lmax, s, kBins)], (unsigned long long)x);
    });
  else
    row.template each<4>(c0, c1, lane, 64, [&](int, float l) {
      if (l > -kInf) atomicAdd((unsigned long long*)&hist[range_of(l, q.lmax, s, kBins)], 1ull);
    });
  __syncthreads();
  // (whole numbers: the order of these additions changes nothing)
  for (int i = tid; i < kBins; i += kSegThreads)
    if (hist[i]) atomicAdd((unsigned long long*)&w.hist[r * kBins + i], (unsigned long long)hist[i]);
}

template <class T, bool kOrder>
__global__ __launch_bounds__(kSegThreads) void weigh_kernel(SampleArgs a) {
  const Ws w = workspace(a.ws, a.n_rows, a.vocab);
  const int64_t r = blockIdx.y;
  const int seg = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<T> row(a.logits, r * a.stride, a.vocab);
  constexpr int kC = kStretch / Row<T>::kE;
  const int c0 = (4 * seg + wave) * kC, c1 = min(c0 + kC, row.chunks());
  // the stretch is under way before the row's settings and statistics are known
  // (with top-k or top-p settings most stretches need less: 74 us for 96 x 151,936,
  // held as well 77)
  u32x4 held[kOrder ? 1 : kC / 64];
  if constexpr (!kOrder) row.load(held, c0 + lane, c1, 64);
  const Ask q = ask_of(a, w, r);
  const bool ranges = kOrder && (q.kind == kSums || q.kind == kCounts);
  if (q.kind != kPlain && !ranges) return;
  __shared__ double table[kTable];
  __shared__ uint64_t part[kSegThreads / 64];
  __shared__ Border border;
  __shared__ int count;
  if (tid < kTable) table[tid] = table_entry(tid);
  if (tid == 0) count = 0;
  __syncthreads();
  const Weigher weigh = weigher_of(q, table);
  const double floor_w = floor_of(q);
  // (a lane's few dozen whole numbers up to 2^45 add up exactly in float64)
  double acc = 0.0;
  auto pass = [&](auto above) {
    auto stretch = [&](auto f) {
      if constexpr (kOrder)
        row.template each<kC / 128>(c0, c1, lane, 64, f);
      else
        row.use(held, c0 + lane, c1, 64, f);
    };
    auto units = [&](float l) { return weigh.template units_of<decltype(above)::value>(l); };
    if (!ranges) {
      if (floor_w <= 0.0)
        stretch([&](int, float l) { acc += __builtin_rint(units(l)); });
      else
        stretch([&](int i, float l) {
          const double x = units(l);
          acc += x >= floor_w || i == q.besti ? __builtin_rint(x) : 0.0;
        });
    } else {
      const int bin = border_of<kSegThreads>(w.hist + r * kBins, q, part, &border).bin;
      const float s = range_scale(q, a.vocab);
      Token* list = w.list + (r * w.segs + seg) * w.cap;
      row.template each<4>(c0, c1, lane, 64, [&](int i, float l) {
        const int b = range_of(l, q.lmax, s, kBins);
        if (b > bin || l == -kInf) return;
        if (b == bin) {
          const int at = atomicAdd(&count, 1);
          if (at < w.cap) list[at] = Token{order_key(l), i};
          return;
        }
        const double x = units(l);
        acc += x >= floor_w || i == q.besti ? __builtin_rint(x) : 0.0;
      });
      __syncthreads();
      if (tid == 0) w.count[r * w.segs + seg] = count;
    }
  };
  if (weigh.low > -kInf)
    pass(std::true_type{});
  else
    pass(std::false_type{});
  uint64_t sum = (uint64_t)acc;
  sum = wave_sum(sum);
  if (lane == 0) w.sums[(r * w.segs + seg) * 4 + wave] = sum;
}

template <class T, bool kOrder>
__global__ __launch_bounds__(kThreads) void pick_kernel(SampleArgs a) {
  __shared__ Shared<kOrder> sh;
  __shared__ Border border;
  const Ws w = workspace(a.ws, a.n_rows, a.vocab);
  const int64_t r = blockIdx.x;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Ask q = ask_of(a, w, r);
  if (q.kind == kDone) {
    if (tid == 0) a.out[r] = q.token;
    return;
  }
  const Row<T> row(a.logits, r * a.stride, a.vocab);
  if (tid < kTable) sh.table[tid] = table_entry(tid);
  const Weigher weigh = weigher_of(q, sh.table);
  const double floor_w = floor_of(q);
  const int n_sums = 4 * w.segs;
  if (tid < n_sums) sh.sums[tid] = q.kind == kFew || q.kind == kWhole ? 0 : w.sums[r * n_sums + tid];
  __syncthreads();

  Kept kept;
  if constexpr (kOrder) {
    if (q.kind != kPlain) {
      // the parts' lists as one
      int m = 0, most = 0;
      if (q.kind != kWhole) {
        if (tid < w.segs) sh.starts[tid] = (int)w.count[r * w.segs + tid];
        __syncthreads();
        int from = 0, part = -1;  // where this thread's token stands
        for (int v = 0; v < w.segs; ++v) {
          const int c = sh.starts[v];
          most = max(most, c);
          if (tid >= m && tid < m + c) part = v, from = tid - m;
          m += min(c, kList + 1);
        }
        if (part >= 0 && most <= w.cap && m <= kList) {
          const Token t = w.list[(r * w.segs + part) * w.cap + from];
          sh.list_key[tid] = t.key;
          sh.list_idx[tid] = t.idx;
        }
      }
      if (q.kind == kWhole || most > w.cap || m > kList) {
        whole_row<T>(a, row, sh, weigh, r, q.kk, q.pf, q.tf, q.low, q.besti, floor_w);
        return;
      }
      __syncthreads();
      // in order: falling key, then rising index, a token a thread
      uint64_t v = tid < m ? (uint64_t)~sh.list_key[tid] << 32 | (uint32_t)sh.list_idx[tid] : ~0ull;
      for (int size = 2; size < 2 * m; size *= 2)
        for (int j = size / 2; j > 0; j /= 2) {
          uint64_t other;
          if (j < 64) {
            other = __shfl_xor(v, j);
          } else {
            __syncthreads();
            sh.list_w[tid] = v;
            __syncthreads();
            other = sh.list_w[tid ^ j];
          }
          v = ((tid & j) == 0) == ((tid & size) == 0) ? min(v, other) : max(v, other);
        }
      const uint32_t k = ~(uint32_t)(v >> 32);
      const int idx = (int)(uint32_t)v;
      const double wf = tid < m ? weigh.units(key_logit(k)) : 0.0;
      const uint64_t x = Weigher::round(wf);
      // what the order counts: tokens of the first kk, their weights, or weights
      // from the range's start on
      Border bd{0, 0, 0.0};
      if (q.kind != kFew) bd = border_of<kThreads>(w.hist + r * kBins, q, sh.part, &border);
      const uint64_t step = tid >= m || (q.kind == kFew && tid >= q.kk) ? 0 : q.kind == kCounts ? 1 : x;
      uint64_t run = step;
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t y = __shfl_up(run, o);
        if (lane >= o) run += y;
      }
      __syncthreads();
      if (lane == 63) sh.part[wave] = run;
      if (tid == 0) sh.found = -1;
      __syncthreads();
      uint64_t total = 0;
      for (int u = 0; u < kWaves; ++u) {
        if (u < wave) run += sh.part[u];
        total += sh.part[u];
      }
      const uint64_t before = bd.above + run - step;
      bool keep;
      if (q.kind == kFew)
        keep = tid < min(m, q.kk) && (tid == 0 || q.pf >= 1.0f || (double)before < (double)q.pf * (double)total);
      else
        keep = tid < m && (double)before < bd.goal;
      if (keep) atomicMax(&sh.found, tid);
      if (keep && (wf >= floor_w || idx == q.besti))
        atomicAdd((unsigned long long*)&sh.sums[(idx + row.lead) / kStretch], (unsigned long long)x);
      __syncthreads();
      if (tid == sh.found) sh.max_key = k, sh.list_idx[0] = idx;
      __syncthreads();
      if (sh.found >= 0) {
        kept.key = sh.max_key;
        kept.last = sh.list_idx[0];
      }
    }
  }

  // the stretch in which the running sum of the kept weights passes the draw
  static_assert(4 * kMaxSegs <= kThreads, "a sum a thread");
  const uint64_t mine = tid < n_sums ? sh.sums[tid] : 0;
  uint64_t run = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  if (lane == 63) sh.part[wave] = run;
  __syncthreads();
  uint64_t total = 0;
  for (int v = 0; v < kWaves; ++v) {
    if (v < wave) run += sh.part[v];
    total += sh.part[v];
  }
  const uint64_t goal = __umul64hi(total, a.bits[r]);
  if (run > goal && run - mine <= goal) sh.found = tid, sh.above = run - mine;
  __syncthreads();
  // its tokens, a run of them a thread
  auto kept_units = [&](int i, float l) -> uint64_t {
    const double x = weigh.units(l);
    return kept.has(order_key(l), i) && (x >= floor_w || i == q.besti) ? Weigher::round(x) : 0;
  };
  constexpr int kEach = kStretch / kThreads;
  const int i0 = sh.found * kStretch - row.lead + tid * kEach;
  uint64_t x[kEach], sum = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    sum += x[e] = i0 + e >= 0 && i0 + e < row.n ? kept_units(i0 + e, (float)row.p[i0 + e]) : 0;
  run = sum;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();
  if (lane == 63) sh.part[wave] = run;
  __syncthreads();
  run += sh.above;
  for (int v = 0; v < wave; ++v) run += sh.part[v];
  uint64_t at = run - sum;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    if (at <= goal && at + x[e] > goal) a.out[r] = i0 + e;
    at += x[e];
  }
}

template <class T>
void launch(const SampleArgs& a, hipStream_t stream) {
  for (int64_t r0 = 0; r0 < a.n_rows; r0 += kRows) {
    SampleArgs b = a;
    b.n_rows = std::min<int64_t>(a.n_rows - r0, kRows);
    b.logits = (const T*)a.logits + r0 * a.stride;
    b.bits += r0;
    b.out += r0;
    if (a.temperature) b.temperature += r0;
    if (a.top_k) b.top_k += r0;
    if (a.top_p) b.top_p += r0;
    if (a.min_p) b.min_p += r0;
    const dim3 g((uint32_t)segments(a.vocab), (uint32_t)b.n_rows);
    if (a.top_k || a.top_p) {
      stats_kernel<T, true><<<g, kSegThreads, 0, stream>>>(b);
      order_kernel<T><<<g, kSegThreads, 0, stream>>>(b);
      weigh_kernel<T, true><<<g, kSegThreads, 0, stream>>>(b);
      pick_kernel<T, true><<<(uint32_t)b.n_rows, kThreads, 0, stream>>>(b);
    } else {
      stats_kernel<T, false><<<g, kSegThreads, 0, stream>>>(b);
      weigh_kernel<T, false><<<g, kSegThreads, 0, stream>>>(b);
      pick_kernel<T, false><<<(uint32_t)b.n_rows, kThreads, 0, stream>>>(b);
    }
  }
}

}  // namespace

int64_t sample_workspace(int64_t n_rows, int32_t vocab) {
  return workspace_bytes(std::min<int64_t>(n_rows, kRows), vocab);
}

hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t stream) {
  if (dtype == 0)
    launch<__bf16>(a, stream);
  else if (dtype == 1)
    launch<_Float16>(a, stream);
  else
    launch<float>(a, stream);
  return hipGetLastError();
}

}  // namespace rt
