// rt_paged_attention, kernel for many rows per sequence and KV head (prompts,
// prompt chunks, wide trees).
//
// A workgroup is four waves of 32 rows each (rows as in attend_few.hip) on
// one run of the cache.  Tiles of 64 tokens of K and V go from the pages
// straight into LDS, the next one while the present one is worked on; a wave
// takes 32 tokens at a time with 32 x 32 x 16 products,
//   S^T = K Q^T (32 tokens x 32 rows),  O^T = V^T P^T (32 d x 32 rows),
// a lane's column being one row again.  A lane gets the scores of rows
// 8 (i / 4) + 4 h + i % 4 of the score tile (h its half of the wave) and needs
// the weights of 8 consecutive tokens per product: the token of K row r is r
// with bits 2 and 3 exchanged, so both are the same registers.
//
// Bound by the vector unit beside the matrix unit: a 64-token step of a wave is
// 32 products (1,024 cycles) with heads of 128 and about as many cycles of
// exponentials, maxima, sums and conversions, which two waves a SIMD overlap in
// part (3,800 cycles for both); heads of 64 halve the products alone.  Two prompts
// of 8,192 tokens, 16 heads of 128: 585 to 607 us, 905 to 940 TFLOP/s (a large
// matrix product reaches 1,407); four of 4,096, heads of 64: 179 us, 769 TFLOP/s.
// Short prompts pay about 6 us a workgroup for its start and end: 29 of 16 to 3,342
// tokens 152 us, 696 TFLOP/s (159 to 167 us replayed in a graph).  Raising the
// waves' priority around the products gains nothing (585 to 594 us).
#include "lane_ops.h"
#include "serve_device.h"

namespace rt {
namespace {

constexpr int kTile = 64;       // tokens of K and V in LDS
constexpr float kSlack = 6.0f;  // a reference may lag the maximum by this many powers of two
constexpr float kLag = kSlack + 1.0f;  // that and float32's steps at references up to kWhole (a half each for the
                                       // maximum and the limit)
// References beyond are too far apart in float32 (from the maximum by up to half a
// step, 32 at 10^9): the weights leave float16's range.
constexpr float kWhole = 8388608.0f;

typedef __attribute__((address_space(3))) void lds_void;

template <class T, int D>
struct Tile {
  T k[kTile * D];  // token t's chunk c (16 bytes) at t * D / 8 + (c ^ swizzle(t))
  T v[kTile * D];  // [token / 8][d][8], as in a page
};

// Rows of K are 16 or 8 chunks of 16 bytes; the 32 lanes of a read take one
// chunk each of 32 rows, so chunks change places by row to use all banks.
template <int D>
__device__ __forceinline__ int swizzle(int t) {
  return D == 128 ? t & 15 : (t >> 1) & 7;
}

// A wave's rows.  Weights are 2^(s scale2 - base), one fused operation and the
// exponential, base per row the running maximum of s scale2 (raised<T> below it)
// as it last moved: when a score is more than kSlack above, and first with the
// row's first seen score.  The largest weight is a power of two then, which T
// holds exactly (29 prompts 2.03e-3 off float64, trees 2.17e-3, chunks in float16
// 2.67e-4; from the nearest whole number 2.33e-3, 2.36e-3 and 2.93e-4).  Weights and sums carry the same
// factor, so a base below the maximum is no error, nor is a move's rounding.
template <class T, int D>
struct Rows {
  typedef typename Half<T>::x8 x8;
  x8 q[D / 16];
  f32x16 o[D / 32];
  float base, l;
  float limit;    // base moves when s scale2 is above: -inf before the first
  int see;        // places below are seen (tree: those before the new ones)
  uint64_t bits;  // tree word
};

// The page of place t0 + lane of the tile from t0 on (its last place's behind
// `stop`).
__device__ __forceinline__ int tile_pages(const int* page_s, int p0, int shift, int t0, int stop, int lane) {
  return page_s[(min(t0 + lane, stop - 1) >> shift) - p0];
}

// Bytes from a block of 16 tokens of K (or V) to the 16 bytes that a lane
// loads, the same for all of a wave's instructions: a tile's instruction
// 4 i + wave takes rows and groups of one such block, and 16 divides the page
// size.
template <int D>
__device__ __forceinline__ uint32_t k_offset(int wave, int lane) {
  const int t = 64 / (D / 8) * wave + lane / (D / 8);  // token of the instruction's 16 or 32
  return (t & 15) * 2 * D + 16 * ((lane % (D / 8)) ^ swizzle<D>(t));
}
template <int D>
__device__ __forceinline__ uint32_t v_offset(int wave, int lane) {
  return (64 * wave + lane) * 16 % (32 * D);
}

// The 64 tokens from t0 on, of pages pg (tile_pages), into a tile: 1,024 bytes
// per instruction and wave.  Blocks of 16 tokens behind the last before `stop`
// read that one instead.
template <class T, int D>
__device__ __forceinline__ void load_tile(const AttendArgs& a, Tile<T, D>& dst, int pg, int h, int t0, int stop, int wave,
                                          uint32_t off_k, uint32_t off_v) {
#ifdef __HIP_DEVICE_COMPILE__  // (buffer resources have no meaning in the host pass)
  constexpr int N = kTile * D / 2048;  // instructions of a wave: 4 or 2
  const int shift = a.c.shift;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int tk = min(t0 + kTile / N * i + (D == 64 ? wave / 2 * 16 : 0), (stop - 1) & ~15);
    const int64_t page = ((int64_t)__builtin_amdgcn_readlane(pg, tk - t0) * a.c.hkv + h) << shift;
    const int64_t at = (page + (tk & ((1 << shift) - 1))) * D;
    // (buffer loads, for their scalar base)
    const auto k = __builtin_amdgcn_make_buffer_rsrc((T*)a.c.k + at, 0, 32 * D, 0x00020000);
    const auto v = __builtin_amdgcn_make_buffer_rsrc((T*)a.c.v + at, 0, 32 * D, 0x00020000);
    const int n = (4 * i + wave) * 512;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(k, (lds_void*)(dst.k + n), 16, off_k, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(v, (lds_void*)(dst.v + n), 16, off_v, 0, 0, 0);
  }
#endif
}

// The larger of a lane's value and its other half's (lane ^ 32).
__device__ __forceinline__ float max_halves(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// The scores of a tile's 64 tokens for a wave's rows: score i is of the place
// 16 (i / 8) + 8 h + i % 8 of the tile, h the lane's half.
template <class T, int D>
__device__ __forceinline__ void scores(const Rows<T, D>& w, const Tile<T, D>& tile, int lane, f32x16 (&s)[2]) {
  typedef typename Half<T>::x8 x8;
  const int col = lane & 31, h = lane >> 5;
  const int kr = (col & 0x13) | ((col & 4) << 1) | ((col & 8) >> 1);
#pragma unroll
  for (int sub = 0; sub < 2; ++sub)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const x8 kf = *(const x8*)(tile.k + ((32 * sub + kr) * (D / 8) + ((2 * ks + h) ^ swizzle<D>(kr))) * 8);
      s[sub] = Half<T>::mma32(kf, w.q[ks], ks == 0 ? f32x16{} : s[sub]);
    }
  // reads of LDS stay half the products ahead of their use
  __builtin_amdgcn_sched_group_barrier(0x100, D / 16, 0);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, D / 16, 0);
}

// The largest of a row's scores, in powers of two.
template <class T, int D>
__device__ __forceinline__ float largest(const f32x16 (&s)[2], float scale2) {
  float mx = s[0][0];
#pragma unroll
  for (int i = 1; i < 32; ++i) mx = fmaxf(mx, s[i >> 4][i & 15]);
  return max_halves(mx) * scale2;
}

// Weights of the scores, and what they add to the sums and to O.
template <class T, int D>
__device__ __forceinline__ void add(Rows<T, D>& w, const Tile<T, D>& tile, float scale2, int lane, const f32x16 (&s)[2]) {
  typedef typename Half<T>::x8 x8;
  const int col = lane & 31, h = lane >> 5;
  x8 p[4];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 4][i & 15], scale2, -w.base));
    sum += e;
    p[i >> 3][i & 7] = (T)e;
  }
  w.l += sum;
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      const x8 vf = *(const x8*)(tile.v + ((2 * g + h) * D + 32 * d + col) * 8);
      w.o[d] = Half<T>::mma32(vf, p[g], w.o[d]);
    }
  // V's first values are read and the first half's weights formed (56 operations a
  // half: exponent, exponential, addition and half a conversion each); then the
  // second half's weights beside the first half's products
  __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
  __builtin_amdgcn_sched_group_barrier(0x002, 56, 0);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, 896 / D, 0);
    if (D == 128) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, D / 16, 0);
}

// A tile, from place t0 on, for a wave's rows; masked: some row of the
// workgroup does not see some of its tokens.  The next tile's loads are started
// first; `tile` and `next` are different tiles, which the compiler has to know
// lest every read of LDS waits for them.
template <class T, int D>
__device__ __forceinline__ void step(const AttendArgs& a, Rows<T, D>& w, const Tile<T, D>* __restrict tile,
                                     Tile<T, D>* __restrict next, int pg, int h, int t0, int stop, int wave,
                                     uint32_t off_k, uint32_t off_v, int first, bool masked, int lane, bool& huge) {
  if (t0 + kTile < stop) load_tile<T, D>(a, *next, pg, h, t0 + kTile, stop, wave, off_k, off_v);
  f32x16 s[2];
  for (;;) {
    // (nothing of a round is kept for the next: that would cost registers)
    const int half = lane >> 5;
    int see = w.see - t0 - 8 * half, new0 = t0 + 8 * half - first;
    asm volatile("" : "+v"(see), "+v"(new0));
    scores<T, D>(w, *tile, lane, s);
    if (masked) {
      // bit o of `sees`: the place o behind the lane's first is seen
      uint64_t sees = see >= 64 ? ~0ull : see > 0 ? (1ull << see) - 1 : 0ull;
      if (a.tree) {
        sees = new0 < 0 ? ~0ull : 0ull;
        if (new0 >= 0 && new0 < 64) sees = w.bits >> new0;
        if (new0 < 0 && new0 > -64) sees = w.bits << -new0 | ((1ull << -new0) - 1);
      }
#pragma unroll
      for (int i = 0; i < 32; ++i)
        s[i >> 4][i & 15] = (sees >> (16 * (i >> 3) + (i & 7)) & 1) ? s[i >> 4][i & 15] : kLowest;
    }
    const float mx = largest<T, D>(s, a.scale2);
    // A row whose base has to move: move it and form the scores again.  (Rare
    // after a row's first tile; with a branch around the move instead, the
    // compiler copies O for every tile.)
    const bool over = mx > w.limit;
    if (!__ballot(over)) break;
    const float to = over ? mx - raised<T>(kLag) : w.base;
    const float f = w.limit == kLowest ? 1.0f : __builtin_amdgcn_exp2f(w.base - to);
    w.limit = over ? fmaxf(to + (raised<T>(kLag) + kSlack), mx) : w.limit;
    w.base = to;
    w.l *= f;
    huge = huge || !(__builtin_fabsf(to) < kWhole);
    for (int d = 0; d < D / 32; ++d) w.o[d] *= f;
  }
  add<T, D>(w, *tile, a.scale2, lane, s);
}

// Places at or behind `stop` of a tile's V: zeroed, since what lies there may
// not be finite and a weight of 0 times it would not be 0.
template <class T, int D>
__device__ __forceinline__ void clear_behind(Tile<T, D>& tile, int t0, int stop, int tid) {
  for (int e = tid; e < kTile / 8 * D; e += 256) {
    const int n = stop - (t0 + e / D * 8);
    if (n < 8) *(u32x4*)(tile.v + 8 * e) = first_of8(*(const u32x4*)(tile.v + 8 * e), n);
  }
}

// Does a tile's V hold a value that is not finite?  (This thread's share.)
template <class T, int D>
__device__ __forceinline__ uint32_t odd_values(const Tile<T, D>& tile, int tid) {
  uint32_t odd = 0;
  for (int e = tid; e < kTile / 8 * D; e += 256) odd |= not_finite8<T>(*(const u32x4*)(tile.v + 8 * e));
  return odd;
}

__device__ __forceinline__ int wave_sum(int x) {
  x += (int)dpp<0xB1>((uint32_t)x);  // within rows of 16 lanes
  x += (int)dpp<0x4E>((uint32_t)x);
  x += (int)dpp<0x141>((uint32_t)x);
  x += (int)dpp<0x140>((uint32_t)x);
  return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) +
         __builtin_amdgcn_readlane(x, 48);
}

// The tile that is `rank`-th in the order of falling cost, of at most 64
// sequences, one a lane.  Tile t of sequence i costs b_i + t, b_i the places before
// its new ones in units of the new tokens of a tile; `above(e)` tiles cost e or
// more.  Ties go by sequence.  Longest first keeps the end of a launch short:
// 29 prompts of 16 to 3,342 tokens 167 us, in the order of the rows 187; 8 of up to
// 4,096 tokens 158, in the order of the rows 160, last rows first 174.
__device__ __forceinline__ RowTile costliest(const AttendArgs& a, int rank) {
  constexpr int R = 128;
  const int lane = (int)(threadIdx.x & 63), unit = R / a.group;
  int b = 0, t = 0;
  if (lane < a.b.n_seqs) {
    const int rows = rows_in(a.b, lane);
    const int kvl = a.b.kv_len[lane];
    t = (int)(((int64_t)rows * a.group + R - 1) / R);
    b = kvl >= rows && kvl <= a.b.max_kv ? (kvl - rows) / unit : 0;  // (else rejected)
  }
  auto above = [&](int e) { return wave_sum(min(max(b + t - e, 0), t)); };
  if (above(0) <= rank) return {-1, 0, false};
  // above(lo) > rank >= above(hi)
  int lo = 0, hi = wave_max_nonneg(b + t);
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (above(mid) > rank)
      lo = mid;
    else
      hi = mid;
  }
  const uint64_t at = __ballot(b <= lo && lo < b + t);  // those with a tile of this cost
  const int nth = rank - above(lo + 1);
  const uint64_t own = __ballot((at >> lane & 1) && __popcll(at & ((1ull << lane) - 1)) == nth);
  if (!own) return {-1, 0, false};
  const int s = __builtin_ctzll(own);
  const int64_t row0 = (int64_t)(lo - __builtin_amdgcn_readlane(b, s)) * R;
  if (row0 > kMostRows) return {-1, 0, false};
  return {s, (int)row0, false};
}

template <class T, int D>
__global__ __launch_bounds__(256, 2) void many_kernel(AttendArgs a) {
  typedef typename Half<T>::x8 x8;
  constexpr int R = 128;
  __shared__ Tile<T, D> tiles[2];
  extern __shared__ int page_s[];

  const int tid = (int)threadIdx.x, lane = tid & 63, col = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (heads of a tile side by side: a die's L2 holds fewer of them; 64 x 64 rows
  // 49 us, heads outermost 58)
  const int h = (int)(blockIdx.x % (uint32_t)a.c.hkv), G = a.group;
  const int rank = (int)(blockIdx.x / (uint32_t)a.c.hkv), last = (int)(gridDim.x / (uint32_t)a.c.hkv) - 1;
  const bool one = (int64_t)a.b.max_q * G <= R;
  int split = (int)blockIdx.y;
  RowTile rt;
  if (a.n_splits > 1 && gridDim.y == 1) {
    const Run r = nth_run(a, rank, one);
    rt = {r.s, r.tile * R, one};
    split = r.split;
  } else {
    // the costliest tiles start first (of many sequences: each one's last tiles)
    rt = !one && a.b.n_seqs <= 64 ? costliest(a, rank) : row_tile(a, last - rank, R);
  }
  const int s = rt.s;
  if (s < 0) return;
  const int row0 = rt.row0;
  const Seq sq = load_seq(a.b, s);
  if (!sq.ok) {
    if (split == 0) reject_rows<T, D>(a, sq, s, h, row0, rt.one ? INT64_MAX : row0 + R);
    return;
  }
  const int n_rows = sq.n * G;
  if (row0 >= n_rows) return;
  const int first = sq.kvl - sq.n;
  const int end = tile_end(a, sq, row0);
  const int c0 = split * a.chunk;
  if (c0 >= end && split > 0) return;
  const int c1 = min(end, c0 + a.chunk), run = end <= a.chunk ? -1 : split;
  const int p0 = c0 >> a.c.shift;
  bool bad = false;  // a page outside the cache
  for (int i = tid; i < ((c1 - 1) >> a.c.shift) - p0 + 1; i += 256) {
    const int pg = a.b.table[(int64_t)s * a.b.table_stride + p0 + i];
    const bool in = pg >= 0 && pg < a.c.n_pages;
    page_s[i] = in ? pg : 0;
    bad = bad || !in;
  }

  Rows<T, D> w;
  const int wrow = row0 + wave * 32;  // the wave's rows
  {
    const int rr = wrow + col;
    const bool in = rr < n_rows;
    const int t = in ? (int)((uint32_t)rr / (uint32_t)G) : 0, g = in ? rr - t * G : 0;
    const T* src = (const T*)a.q.data + (int64_t)(sq.q0 + t) * a.q.ts + (h * G + g) * a.q.hs + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) w.q[ks] = in ? *(const x8*)(src + 16 * ks) : as_half8<T>(u32x4{0, 0, 0, 0});
    w.bits = in && a.tree ? a.tree[sq.q0 + t] & ~0ull >> ((64 - sq.n) & 63) : 0;
    w.see = !in ? 0 : a.tree ? first : first + t + 1;
    w.limit = kLowest;
    w.base = w.l = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) w.o[d] = f32x16{};
  }
  const int whole = a.tree ? first : first + (int)((uint32_t)row0 / (uint32_t)G) + 1;  // places that all of the workgroup's rows see
  __syncthreads();

  const uint32_t off_k = k_offset<D>(wave, lane), off_v = v_offset<D>(wave, lane);
  uint32_t odd = 0;   // a value that is not finite at a place that some row may not see
  bool huge = false;  // scores beyond kWhole, or below float32 in powers of two
  load_tile<T, D>(a, tiles[0], tile_pages(page_s, p0, a.c.shift, c0, c1, lane), h, c0, c1, wave, off_k, off_v);
  int pg = tile_pages(page_s, p0, a.c.shift, c0 + kTile, c1, lane);  // of the next tile
  int at = 0;
  for (int t0 = c0; t0 < c1; t0 += kTile, at ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // this wave's loads have landed
    __syncthreads();                     // everyone's have, and nobody reads the other tile
    const bool masked = t0 + kTile > whole;
    if (masked) {
      if (t0 + kTile > c1) {
        clear_behind<T, D>(tiles[at], t0, c1, tid);
        __syncthreads();
      }
      odd |= odd_values<T, D>(tiles[at], tid);
    }
    const int now = pg;
    pg = tile_pages(page_s, p0, a.c.shift, t0 + 2 * kTile, c1, lane);
    step<T, D>(a, w, &tiles[at], &tiles[at ^ 1], now, h, t0, c1, wave, off_k, off_v, first, masked, lane, huge);
  }

  const float l = w.l + __shfl_xor(w.l, 32);
  // A row that sees places of the run, but no score above -inf: in powers of two
  // (1.44 to a score's unit) finite scores may have ended there.
  const bool some = w.see > c0 || (a.tree && (w.bits >> max(c0 - first, 0)) != 0);
  huge = huge || (some && w.limit == kLowest && l == 0.0f);
  if (__syncthreads_or(bad || huge || odd)) {
    for (int rr = row0 + wave; rr < min(row0 + R, n_rows); rr += 4)
      row_by_place<T, D, false>(a, sq, s, h, run, rr, c0, c1);
    return;
  }
  const int rr = wrow + col;
  if (rr >= n_rows) return;
  const RowOut<T, D> out(a, sq, h, run, rr);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      out.put4(32 * d + 8 * r + 4 * hf,
               f32x4{w.o[d][4 * r], w.o[d][4 * r + 1], w.o[d][4 * r + 2], w.o[d][4 * r + 3]}, inv);
  if (hf == 0) out.put_sum(w.limit == kLowest ? kLowest : w.base / kBaseUnit, l);
}

template <class T, int D>
void launch(const AttendPlan& p, const AttendArgs& a, hipStream_t stream) {
  const int pages = (min((int64_t)p.chunk, (int64_t)a.b.max_kv) >> a.c.shift) + 2;
  const bool row = p.runs_in_a_row(a.c.hkv, a.b.n_seqs);
  const dim3 grid((uint32_t)p.groups_x(a.c.hkv, a.b.n_seqs), row ? 1 : p.n_splits);
  many_kernel<T, D><<<grid, 256, pages * sizeof(int), stream>>>(a);
}

}  // namespace

void launch_attend_many(int dtype, int head_dim, const AttendPlan& p, const AttendArgs& a, hipStream_t stream) {
  if (dtype == 0)
    head_dim == 64 ? launch<__bf16, 64>(p, a, stream) : launch<__bf16, 128>(p, a, stream);
  else
    head_dim == 64 ? launch<_Float16, 64>(p, a, stream) : launch<_Float16, 128>(p, a, stream);
}

}  // namespace rt
