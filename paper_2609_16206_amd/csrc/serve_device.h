// Device helpers of the serving operators: 16-bit types and their matrix
// products, and the way from a row of a ragged batch to its sequence.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rt_internal.h"
#include "serve_internal.h"

namespace rt {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Half;
template <>
struct Half<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(x8 a, x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Half<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(x8 a, x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// 16 bytes as eight values of T.
template <class T>
__device__ __forceinline__ typename Half<T>::x8 as_half8(u32x4 u) {
  return __builtin_bit_cast(typename Half<T>::x8, u);
}

// Eight 16-bit values at once: adding one to an exponent that is all ones
// carries into the sign's place.  Bits 15 and 31 of the result say whether any
// value is NaN or infinite (OR of several results included).
template <class T>
__device__ __forceinline__ uint32_t not_finite8(u32x4 u) {
  constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7f807f80u : 0x7c007c00u;
  constexpr uint32_t kOne = __is_same(T, __bf16) ? 0x00800080u : 0x04000400u;
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (u[i] & kExp) + kOne;
  return r & 0x80008000u;
}

// The first n (0 .. 8) of eight 16-bit values, 0 in the place of the others.
__device__ __forceinline__ u32x4 first_of8(u32x4 u, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = n >= 2 * i + 2 ? u[i] : n == 2 * i + 1 ? u[i] & 0xffffu : 0u;
  return u;
}

// The number of i in [0, n) with f(i) <= x, f non-decreasing, found by the
// whole wave 64 values at a time (two rounds up to 4,096); whatever f holds,
// the loop ends and the result lies in [0, n].
template <class F>
__device__ __forceinline__ int wave_count_le(F f, int n, int64_t x) {
  const int lane = (int)(threadIdx.x & 63);
  int lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    const bool le = i < hi && f(i) <= x;
    const int c = __popcll(__ballot(le));
    if (c == 0) return lo;  // f(lo) > x
    const int top = lo + (c - 1) * step;  // f(top) <= x
    hi = min(hi, top + step);
    lo = top + 1;
    if (step == 1) return lo;
  }
  return lo;
}

// What a call uses of one sequence.
struct Seq {
  int q0, n, kvl;  // first row, new rows, cached tokens
  bool ok;         // not rejected
};

__device__ __forceinline__ bool accepted(const Batch& b, int q0, int q1, int kvl) {
  return q0 >= 0 && q1 >= q0 && q1 <= b.n_tokens && q1 - q0 <= b.max_q && kvl >= q1 - q0 && kvl <= b.max_kv;
}

// (s is the same for the whole wave)
__device__ __forceinline__ Seq load_seq(const Batch& b, int s) {
  Seq r;
  r.q0 = __builtin_amdgcn_readfirstlane(b.q_start[s]);
  const int q1 = __builtin_amdgcn_readfirstlane(b.q_start[s + 1]);
  r.kvl = __builtin_amdgcn_readfirstlane(b.kv_len[s]);
  r.ok = accepted(b, r.q0, q1, r.kvl);
  r.n = q1 - r.q0;
  return r;
}

// The sequence that holds a row, or -1 (whole wave, one row).  Decode batches
// have one row per sequence in order, which one pair of loads shows.
__device__ __forceinline__ int seq_of_row(const Batch& b, int row) {
  if (row < b.n_seqs && b.q_start[row] == row && b.q_start[row + 1] == row + 1) return row;
  const int32_t* q = b.q_start;
  const int s = wave_count_le([q](int i) { return (int64_t)q[i]; }, b.n_seqs + 1, row) - 1;
  if (s < 0 || s >= b.n_seqs) return -1;
  return row < q[s + 1] ? s : -1;
}

constexpr float kLowest = -__builtin_inff();

// 2^((s - base) scale2): exact differences, so that scores of any size that
// equal the maximum have weight 1.  (One fused operation s * scale2 - base *
// scale2 would save an instruction, but its product is only rounded once:
// beyond 2^30 the difference it leaves is no longer small.)
__device__ __forceinline__ float weight2(float s, float base, float scale2) {
  return __builtin_amdgcn_exp2f((s - base) * scale2);
}
// The same times 2^up.
__device__ __forceinline__ float weight2(float s, float base, float scale2, float up) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(s - base, scale2, up));
}

// Weights are rounded to T for O = V^T P^T, because matrix products take 16-bit
// operands; float32 ones would go through products at a sixteenth of the rate.
// Their sum is taken of the unrounded weights: the output is off by half a step of
// the mean of |v| at most, and by none where the largest weight (exactly 1, or
// a power of two) outweighs the others.  (The sum of the rounded ones gives equal
// values as they are, but is off by up to twice that where values differ: numerator
// and denominator may be rounded apart.)
//
// Powers of two by which weights are raised before they are rounded to T, so that
// the largest stay below 2^16 (the largest of a row is 2^lag in many_kernel,
// whose references lag): float16 holds 11 bits down to 2^-14 and nothing below
// 2^-25, and a row's many small weights may be most of its sum.  Raised by 15, a
// weight of 2^-29 of the largest keeps its bits (by 8, one of 2^-22), and none is off
// by more than 2^-40 (2^-33) of it.  bfloat16 has float32's range.
template <class T>
constexpr float raised(float lag) {
  return __is_same(T, __bf16) ? 0.0f : 15.0f - lag;
}

// Where sequence i's rows start in the tensors, whatever q_start says.  Every
// way from a workgroup to its tile counts rows by it, as reject_rows does.
__device__ __forceinline__ int row_start(const Batch& b, int i) { return min(max(b.q_start[i], 0), b.n_tokens); }
__device__ __forceinline__ int rows_in(const Batch& b, int i) { return max(row_start(b, i + 1) - row_start(b, i), 0); }

// The row tile of a workgroup (rows count in 32 bits, divided by the group's
// size without the long way of 64): sequence s owns tiles
// floor(row_start(s) group / tile_rows) + s and up, or tile s alone where one
// holds any sequence's rows.
struct RowTile {
  int s;         // -1: none
  int row0;      // its first row within the sequence
  bool one;
};

__device__ __forceinline__ RowTile row_tile(const AttendArgs& a, int64_t tile, int tile_rows) {
  const Batch& b = a.b;
  const int64_t G = a.group;
  if (a.b.max_q * G <= tile_rows) return {(int)tile, 0, true};
  const int s = __builtin_amdgcn_readfirstlane(
      wave_count_le([&b, G, tile_rows](int i) { return row_start(b, i) * G / tile_rows + i; }, b.n_seqs, tile) - 1);
  const int64_t row0 = s < 0 ? 0 : (tile - (row_start(b, s) * G / tile_rows + s)) * tile_rows;
  if (row0 < 0 || row0 > kMostRows) return {-1, 0, false};
  return {s, (int)row0, false};
}

// Powers of two to a unit of many_kernel's references (a power of two itself: they
// stay exact), so large that a finite score's never overflows.
constexpr float kBaseUnit = 0x1p64f;

// A sequence, one of its row tiles and one of their runs.
struct Run {
  int s, tile, split;  // s -1: none
};

// Inclusive sums over the lanes.
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = (int)(threadIdx.x & 63);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// The `rank`-th run, sequence by sequence, of at most 64 x 64
// sequences: the workgroups with a run are then the first ones of the launch,
// which spreads them evenly over the chip (8 requests of 12 rows and 8 heads 18
// us, by sequence and run 21; 64 of 64 rows 41 us and 48).  Every tile is taken to
// have the runs of the last one; a sequence that is rejected or has no rows has
// one.  `one`: a tile holds any sequence's rows.
__device__ __forceinline__ Run nth_run(const AttendArgs& a, int rank, bool one) {
  const int lane = (int)(threadIdx.x & 63), n = a.b.n_seqs, per = (n + 63) / 64;
  auto runs = [&](int i) {
    const int q0 = a.b.q_start[i], q1 = a.b.q_start[i + 1], kvl = a.b.kv_len[i];
    return q0 == q1 || !accepted(a.b, q0, q1, kvl) ? 1 : (int)((uint32_t)(kvl + a.chunk - 1) / (uint32_t)a.chunk);
  };
  auto tiles = [&](int i) {
    return one ? 1 : max((int)((uint32_t)(rows_in(a.b, i) * a.group + a.tile_rows - 1) / (uint32_t)a.tile_rows), 1);
  };
  auto find = [&](int count) {  // the lane whose counts reach the rank, which becomes the one among its own
    const int upto = wave_scan(count);
    const int at = __popcll(__ballot(upto <= rank));
    if (at < 64) rank -= __builtin_amdgcn_readlane(upto - count, at);
    return at;
  };
  int mine = 0;
  for (int i = lane * per; i < min(lane * per + per, n); ++i) mine += runs(i) * tiles(i);
  int s = find(mine);
  if (s == 64) return {-1, 0, 0};
  if (per > 1) {
    const int i = s * per + lane, count = lane < per && i < n ? runs(i) * tiles(i) : 0;
    s = s * per + find(count);
  }
  const int t = __builtin_amdgcn_readfirstlane(tiles(s));
  return {s, rank % t, rank / t};  // tiles of a run side by side: they read the same places
}

// Where the rows of a tile end, of those that a sequence with n_rows rows has:
// one more than the last place that any of them sees.
__device__ __forceinline__ int tile_end(const AttendArgs& a, const Seq& sq, int row0) {
  const int n_rows = sq.n * a.group;
  return a.tree ? sq.kvl : sq.kvl - sq.n + (int)((uint32_t)(min(row0 + a.tile_rows, n_rows) - 1) / (uint32_t)a.group) + 1;
}

// The result of row `rr` of a sequence (as few_kernel and many_kernel count
// rows): o / l of a tile with one run, or the partial result of a run.
template <class T, int D>
struct RowOut {
  const AttendArgs& a;
  int split;  // -1: the only run
  int64_t token, head;
  __device__ __forceinline__ RowOut(const AttendArgs& a, const Seq& sq, int h, int split, int rr) : a(a), split(split) {
    const uint32_t t = (uint32_t)rr / (uint32_t)a.group;
    token = sq.q0 + (int)t;
    head = h * a.group + (rr - (int)t * a.group);
  }
  __device__ __forceinline__ T* row() const { return (T*)a.o.data + token * a.o.ts + head * a.o.hs; }
  __device__ __forceinline__ int64_t part() const {
    return (int64_t)split * a.b.n_tokens * a.hq + token * a.hq + head;
  }
  // elements d0 .. d0 + 3
  __device__ __forceinline__ void put4(int d0, f32x4 o, float inv) const {
    if (split < 0) {
      typename Half<T>::x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (T)(o[i] * inv);
      *(typename Half<T>::x4*)(row() + d0) = y;
    } else {
      *(f32x4*)(a.part_o + part() * D + d0) = o;
    }
  }
  // the base of the weights, in units, and their sum
  __device__ __forceinline__ void put_sum(float base, float l) const {
    if (split >= 0) a.part_ml[part()] = make_float2(base, l);
  }
};

// One row, place by place, by one wave: for runs in which a place that some
// row of the workgroup does not see holds a value that is not finite (weight 0
// times it would not be 0 in a matrix product), a page lies outside the cache,
// or scores are such that many_kernel's exponents do not serve.  Lanes take 64
// places each for the scores and D / 64 elements each for the sum; only what the
// row sees is used.  kScores: references in scores, as few_kernel's, not in
// kBaseUnit powers of two, as many_kernel's.
template <class T, int D, bool kScores>
__device__ void row_by_place(const AttendArgs& a, const Seq& sq, int s, int h, int split, int rr, int c0, int c1) {
  constexpr int E = D / 64;
  const int lane = (int)(threadIdx.x & 63), shift = a.c.shift, ps = 1 << shift;
  const RowOut<T, D> out(a, sq, h, split, rr);
  const int first = sq.kvl - sq.n, t = (int)(out.token - sq.q0);
  const uint64_t bits = a.tree ? a.tree[out.token] : 0;
  const int end = min(a.tree ? sq.kvl : first + t + 1, c1);
  const T* q = (const T*)a.q.data + out.token * a.q.ts + out.head * a.q.hs;
  const int32_t* table = a.b.table + (int64_t)s * a.b.table_stride;
  float m = kLowest, l = 0.0f, o[E] = {};
  for (int j0 = c0; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    const bool vis = j < end && (!a.tree || j < first || (bits >> (j - first) & 1));
    int pg = vis ? table[j >> shift] : 0;
    const bool bad = pg < 0 || pg >= a.c.n_pages;
    if (bad) pg = 0;
    float x = kLowest;
    if (vis) {
      const T* k = (const T*)a.c.k + ((((int64_t)pg * a.c.hkv + h) << shift) + (j & (ps - 1))) * D;
      x = 0.0f;
      for (int d = 0; d < D; ++d) x = __builtin_fmaf((float)k[d], (float)q[d], x);
      if (bad) x = __builtin_nanf("");
    }
    float mn = x;
    for (int i = 32; i; i >>= 1) mn = fmaxf(mn, __shfl_xor(mn, i));
    mn = fmaxf(mn, m);
    const float base = mn == kLowest ? 0.0f : mn;
    const float f = weight2(m, base, a.scale2), w = weight2(x, base, a.scale2, kScores ? raised<T>(0.0f) : 0.0f);
    m = mn;
    l = l * f + (vis ? w : 0.0f);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= f;
    const uint64_t all = __ballot(vis);
    for (int i = 0; i < 64 && j0 + i < end; ++i) {
      if (!(all >> i & 1)) continue;
      const float p = __shfl(w, i);  // (no matrix product: no rounding to T)
      const int pi = __shfl(pg, i), slot = (j0 + i) & (ps - 1);
      const T* v = (const T*)a.c.v + ((((int64_t)pi * a.c.hkv + h) << shift) + (slot & ~7)) * D + (slot & 7);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(p, (float)v[8 * (E * lane + e)], o[e]);
    }
  }
  for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (split < 0)
      out.row()[E * lane + e] = (T)(o[e] * inv);
    else
      a.part_o[out.part() * D + E * lane + e] = o[e];
  }
  if (lane == 0) out.put_sum(kScores ? m : m / kBaseUnit * a.scale2, l);
}

// Rows of a rejected sequence, as far as they lie in the tensors, from row
// `row0` of the sequence to `stop`: NaN.
template <class T, int D>
__device__ __forceinline__ void reject_rows(const AttendArgs& a, const Seq& sq, int s, int h, int64_t row0, int64_t stop) {
  const int q0 = row_start(a.b, s);
  stop = min(stop, (int64_t)rows_in(a.b, s) * a.group);
  for (int64_t i = row0 * D + threadIdx.x; i < stop * D; i += blockDim.x) {
    const int64_t rr = i / D;
    ((T*)a.o.data)[(q0 + rr / a.group) * a.o.ts + (h * a.group + rr % a.group) * a.o.hs + i % D] =
        (T)__builtin_nanf("");
  }
}

}  // namespace rt
