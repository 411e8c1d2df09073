// rt_paged_attention, kernels for few rows per sequence and KV head, and the
// join of split runs.
//
// Rows are (new token, query head of the KV head's group) pairs, 16 to a
// column tile of the matrix products.  Scores are formed transposed,
//   S^T = K Q^T (16 tokens x 16 rows, K and Q^T both 8 consecutive d a lane),
//   O^T = V^T P^T (16 d x 16 rows, V^T and P^T 8 consecutive tokens a lane),
// so that a lane's column is one row throughout: maximum, sum and rescaling
// are per lane (with two exchanges between the four lanes of a column), and
// with the tokens of two score tiles dealt as token 8 (r / 4) + 4 m + r % 4 for
// row r of tile m, the scores a lane gets are the weights it needs next: no
// exchange and no LDS between the products.
//
// A workgroup is four waves on one (sequence, row tile, KV head, run of
// `chunk` tokens); the waves take 32 tokens in turn, each with a running
// maximum and sum of its own, and join at the end.  Runs go to memory as float32
// and are joined by a second kernel.
//
// K and V are read once (a KV head's query heads share a tile), so HBM bounds
// large batches and the chain of dependent loads (lengths, pages, K, V, then the
// join's) small ones.  One token each of 3 requests with up to 131,072 cached, 8 KV
// heads of 128: 1.35 GB in 243 to 253 us, 5.4 TB/s (a large copy reaches 4.9);
// of 256 uneven requests with 2 KV heads: 394 MB in 99 us, 4.0 TB/s; of 64: 133
// MB in 33 us, 4.0 TB/s; one request of 700 tokens: 9.7 us.  Loading a step ahead
// (32 more tokens in registers) changes nothing: other waves fill the wait.
#include "serve_device.h"

namespace rt {
namespace {

// The last place a row sees, plus one, and its tree word.
struct RowSight {
  int end;        // places below this one are visible (tree: places before the new ones)
  uint64_t bits;  // tree word
};

// (NT = 2 in 256 registers, two workgroups a compute unit: 64 requests with 32
// rows each 36 us in place of 50)
template <class T, int D, int NT>
__global__ __launch_bounds__(256, NT) void few_kernel(AttendArgs a) {
  typedef typename Half<T>::x8 x8;
  constexpr int KS = D / 32, DT = D / 16, R = 16 * NT;
  extern __shared__ char lds[];
  float2* ml_s = (float2*)lds;                        // [4][R]
  f32x4* o_s = (f32x4*)(lds + 4 * R * sizeof(float2));  // [4][DT][64]
  int* page_s = (int*)((char*)o_s + 4 * DT * 64 * sizeof(f32x4));

  const int tid = (int)threadIdx.x, lane = tid & 63, col = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group;
  int h, s, split;
  if (gridDim.z > 1) {
    // Workgroups go to the eight dies by their number: shifted by run and head,
    // or a die would have all runs of a long sequence.
    h = (int)blockIdx.y, split = (int)blockIdx.z;
    s = (int)((blockIdx.x + (uint32_t)(split * a.c.hkv + h)) % gridDim.x);
  } else {
    const int rank = (int)(blockIdx.x / (uint32_t)a.c.hkv);
    h = (int)(blockIdx.x % (uint32_t)a.c.hkv);
    const Run r = a.n_splits > 1 ? nth_run(a, rank, true) : Run{rank, 0, 0};
    s = r.s, split = r.split;
  }
  if (s < 0) return;
  const Seq sq = load_seq(a.b, s);
  if (!sq.ok) {
    if (split == 0) reject_rows<T, D>(a, sq, s, h, 0, INT64_MAX);
    return;
  }
  const int n_rows = sq.n * G;
  const int c0 = split * a.chunk;
  if (n_rows == 0 || c0 >= sq.kvl) return;
  const int first = sq.kvl - sq.n;  // place of the first new token
  const int c1 = min(sq.kvl, c0 + a.chunk), run = sq.kvl <= a.chunk ? -1 : split;
  const int whole = a.tree ? first : first + 1;  // every row sees the places below

  bool bad = false;  // a page outside the cache
  uint32_t odd = 0;  // a value that is not finite at a place that some row may not see
  const int shift = a.c.shift, ps = 1 << shift, p0 = c0 >> shift;
  for (int i = tid; i < ((c1 - 1) >> shift) - p0 + 1; i += 256) {
    const int pg = a.b.table[(int64_t)s * a.b.table_stride + p0 + i];
    const bool in = pg >= 0 && pg < a.c.n_pages;
    page_s[i] = in ? pg : 0;
    bad = bad || !in;
  }

  // queries and what each row sees
  x8 qf[NT][KS];
  RowSight see[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rr = 16 * nt + col;
    const bool in = rr < n_rows;
    const int t = in ? (int)((uint32_t)rr / (uint32_t)G) : 0, g = in ? rr - t * G : 0;
    const T* src = (const T*)a.q.data + (int64_t)(sq.q0 + t) * a.q.ts + (h * G + g) * a.q.hs + 8 * lg;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[nt][ks] = in ? *(const x8*)(src + 32 * ks) : as_half8<T>(u32x4{0, 0, 0, 0});
    see[nt].bits = in && a.tree ? a.tree[sq.q0 + t] : 0;
    see[nt].end = !in ? 0 : a.tree ? first : first + t + 1;
  }
  __syncthreads();

  f32x4 o[NT][DT];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = kLowest;
    l[nt] = 0.0f;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[nt][j] = f32x4{0, 0, 0, 0};
  }

  const T* kbase = (const T*)a.c.k;
  const T* vbase = (const T*)a.c.v;
  const int krow = 8 * (col >> 2) + (col & 3);  // token of this lane's K rows, + 4 m
  for (int t0 = c0 + 32 * wave; t0 < c1; t0 += 128) {
    // K rows and V groups; places at or behind c1 read the last one instead
    x8 kf[2][KS], vf[DT];
#pragma unroll
    for (int mi = 0; mi < 2; ++mi) {
      const int tk = min(t0 + krow + 4 * mi, c1 - 1);
      const int pg = page_s[(tk >> shift) - p0];
      const T* src = kbase + ((((int64_t)pg * a.c.hkv + h) << shift) + (tk & (ps - 1))) * D + 8 * lg;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[mi][ks] = *(const x8*)(src + 32 * ks);
    }
    const int tv = min(t0 + 8 * lg, (c1 - 1) & ~7);
    const int vpg = page_s[(tv >> shift) - p0];
    {
      const T* src =
          vbase + ((((int64_t)vpg * a.c.hkv + h) << shift) + (tv & (ps - 1))) * D + 8 * col;
#pragma unroll
      for (int j = 0; j < DT; ++j) vf[j] = *(const x8*)(src + 128 * j);
    }
    f32x4 sc[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mi = 0; mi < 2; ++mi) {
        sc[nt][mi] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc[nt][mi] = Half<T>::mma16(kf[mi][ks], qf[nt][ks], sc[nt][mi]);
      }
    if (t0 + 32 > whole) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = t0 + 8 * lg + i;
          bool vis = j < see[nt].end;
          if (a.tree && j >= first && j < sq.kvl) vis = see[nt].bits >> (j - first) & 1;
          if (!vis) sc[nt][i >> 2][i & 3] = kLowest;
        }
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const u32x4 u = first_of8(__builtin_bit_cast(u32x4, vf[j]), c1 - (t0 + 8 * lg));
        odd |= not_finite8<T>(u);
        vf[j] = as_half8<T>(u);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float mx = kLowest;
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, sc[nt][i >> 2][i & 3]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m[nt], mx);
      const float base = mn == kLowest ? 0.0f : mn;
      if (__ballot(mn > m[nt])) {
        const float f = weight2(m[nt], base, a.scale2);
        l[nt] *= f;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[nt][j] *= f;
        m[nt] = mn;
      }
      x8 p;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = weight2(sc[nt][i >> 2][i & 3], base, a.scale2, raised<T>(0.0f));
        sum += e;
        p[i] = (T)e;
      }
      l[nt] += sum;
#pragma unroll
      for (int j = 0; j < DT; ++j) o[nt][j] = Half<T>::mma16(vf[j], p, o[nt][j]);
    }
  }
  if (__syncthreads_or(bad || odd)) {
    for (int rr = wave; rr < n_rows; rr += 4)
      row_by_place<T, D, true>(a, sq, s, h, run, rr, c0, c1);
    return;
  }

  // join the four waves
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += __shfl_xor(l[nt], 16);
    l[nt] += __shfl_xor(l[nt], 32);
    if (lg == 0) ml_s[wave * R + 16 * nt + col] = make_float2(m[nt], l[nt]);
  }
  __syncthreads();
  float lsum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float2 w[4];
    float mn = kLowest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = ml_s[i * R + 16 * nt + col];
      mn = fmaxf(mn, w[i].x);
    }
    const float base = mn == kLowest ? 0.0f : mn;
    lsum[nt] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) lsum[nt] += w[i].y * weight2(w[i].x, base, a.scale2);
    const float f = weight2(m[nt], base, a.scale2);
    m[nt] = mn;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[nt][j] *= f;
  }
  // sums over the waves: a row tile's elements dealt to all of them
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (nt > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < DT; ++j) o_s[(wave * DT + j) * 64 + lane] = o[nt][j];
    __syncthreads();
    const int rr = 16 * nt + col;
    if (rr >= n_rows) continue;
    const RowOut<T, D> out(a, sq, h, run, rr);
    const float inv = lsum[nt] == 0.0f ? 0.0f : 1.0f / lsum[nt];
#pragma unroll
    for (int jj = 0; jj < DT / 4; ++jj) {
      const int j = 4 * jj + wave;
      f32x4 x = o_s[j * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) x += o_s[(w * DT + j) * 64 + lane];
      out.put4(16 * j + 4 * lg, x, inv);
    }
    if (wave == 0 && lg == 0) out.put_sum(m[nt], lsum[nt]);
  }
}

// Join of the runs of the rows of tiles with more than one:
//   out = sum_i f_i O_i / sum_i f_i l_i,  f_i = 2^((base_i - max base) unit),
// in few_kernel's units (scores) as exact as the weights of one run.
// Many runs, a row to a workgroup.  A wave's lanes are 16-byte pieces of 256 / D
// runs; a row's runs are those that begin at or before its last place.
template <class T, int D>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
  constexpr int kPieces = D / 4, kRuns = 256 / kPieces;  // runs side by side
  __shared__ f32x4 acc_s[256];
  const int tid = (int)threadIdx.x, lane = tid & 63, h = (int)blockIdx.y;
  const RowTile rt = row_tile(a, blockIdx.x, a.tile_rows);
  if (rt.s < 0) return;
  const Seq sq = load_seq(a.b, rt.s);
  const int n_rows = sq.ok ? sq.n * a.group : 0;
  if (!sq.ok || rt.row0 >= n_rows || tile_end(a, sq, rt.row0) <= a.chunk) return;  // written already
  const int64_t step = (int64_t)a.b.n_tokens * a.hq;
  const int rr = rt.row0 + (int)blockIdx.z;
  if (rr >= n_rows) return;
  const int mine = tid / kPieces, piece = tid % kPieces;
  const RowOut<T, D> out(a, sq, h, 0, rr);
  const int end = a.tree ? sq.kvl : sq.kvl - sq.n + (int)(out.token - sq.q0) + 1;
  const int runs = (end + a.chunk - 1) / a.chunk;
  const int64_t at = out.part();
  f32x4 acc = {0, 0, 0, 0};
  float l = 0.0f, base = kLowest;
  for (int i0 = 0; i0 < runs; i0 += 64) {
    const float2 ml = i0 + lane < runs ? a.part_ml[(i0 + lane) * step + at] : make_float2(kLowest, 0.0f);
    const f32x4* src = (const f32x4*)a.part_o + ((i0 + mine) * step + at) * kPieces + piece;
    constexpr int kMost = 64 / kRuns < 8 ? 64 / kRuns : 8;
    const int n = min(64, runs - i0);
    float mx = ml.x;
    for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    mx = fmaxf(mx, base);
    const float to = mx == kLowest ? 0.0f : mx;
    const float keep = weight2(base, to, a.unit), f = weight2(ml.x, to, a.unit);
    base = mx;
    l = l * keep + f * ml.y;
    acc *= keep;
    for (int i = 0; i < n; i += kMost * kRuns) {
      f32x4 x[kMost];
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        const int at_run = i + j * kRuns;
        x[j] = at_run + mine < n ? src[at_run * step * kPieces] : f32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        const float fi = __shfl(f, i + j * kRuns + mine);
        const float w = i + j * kRuns + mine < n ? fi : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(w, x[j][e], acc[e]);
      }
    }
  }
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
#pragma unroll
  for (int o = kPieces; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
  acc_s[tid] = acc;
  __syncthreads();
  if (tid >= kPieces) return;
#pragma unroll
  for (int w = 1; w < 4; ++w) acc += acc_s[64 * w + lane];
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* dst = out.row() + 4 * piece;
#pragma unroll
  for (int e = 0; e < 4; ++e) dst[e] = (T)(acc[e] * inv);
}

// Fewer runs or more rows: kRows rows to a wave, whose loads go out together, 16
// runs at a time.  Bases and sums: 16 lanes a row, a run each.
template <class T, int D, int kRows>
__global__ __launch_bounds__(256) void join_few_kernel(AttendArgs a) {
  constexpr int kPieces = D / 4, kRuns = 64 / kPieces;
  const int tid = (int)threadIdx.x, lane = tid & 63, h = (int)blockIdx.y;
  const RowTile rt = row_tile(a, blockIdx.x, a.tile_rows);
  if (rt.s < 0) return;
  const Seq sq = load_seq(a.b, rt.s);
  const int n_rows = sq.ok ? sq.n * a.group : 0;
  if (!sq.ok || rt.row0 >= n_rows || tile_end(a, sq, rt.row0) <= a.chunk) return;  // written already
  const int64_t step = (int64_t)a.b.n_tokens * a.hq;
  const int r0 = rt.row0 + kRows * (4 * (int)blockIdx.z + (tid >> 6));
  if (r0 >= n_rows) return;
  const RowOut<T, D> mine(a, sq, h, 0, min(r0 + (kRows > 1 ? lane / 16 : 0), n_rows - 1));
  const int end = a.tree ? sq.kvl : sq.kvl - sq.n + (int)(mine.token - sq.q0) + 1;
  const int runs = (end + a.chunk - 1) / a.chunk, side = lane / kPieces, piece = lane % kPieces;
  int n[kRows], most = 0;
  int64_t at[kRows];
  f32x4 acc[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    n[r] = __builtin_amdgcn_readlane(runs, 16 * r);
    most = max(most, n[r]);
    at[r] = RowOut<T, D>(a, sq, h, 0, min(r0 + r, n_rows - 1)).part();
    acc[r] = f32x4{0, 0, 0, 0};
  }
  float l = 0.0f, base = kLowest;
  for (int i0 = 0; i0 < most; i0 += 16) {
    const int my_run = i0 + lane % 16;
    const float2 ml = my_run < runs ? a.part_ml[my_run * step + mine.part()] : make_float2(kLowest, 0.0f);
    float mx = fmaxf(ml.x, base);
    for (int o = 8; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    const float to = mx == kLowest ? 0.0f : mx;
    const float keep = weight2(base, to, a.unit), f = weight2(ml.x, to, a.unit);
    base = mx;
    l = l * keep + f * ml.y;
#pragma unroll
    for (int r = 0; r < kRows; ++r) acc[r] *= __shfl(keep, 16 * r);
    for (int i = i0; i < min(most, i0 + 16); i += 2 * kRuns) {
      f32x4 x[kRows][2];
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int run = i + j * kRuns + side;
          x[r][j] = run < n[r] ? ((const f32x4*)a.part_o)[(run * step + at[r]) * kPieces + piece] : f32x4{0, 0, 0, 0};
        }
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int run = i + j * kRuns + side;
          const float fr = __shfl(f, 16 * r + run - i0);
          const float w = run < n[r] ? fr : 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[r][e] = __builtin_fmaf(w, x[r][j][e], acc[r][e]);
        }
    }
  }
  for (int o = 8; o; o >>= 1) l += __shfl_xor(l, o);
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
#pragma unroll
    for (int o = kPieces; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[r][e] += __shfl_xor(acc[r][e], o);
    const float sum = __shfl(l, 16 * r);
    if (side != r % kRuns || r0 + r >= n_rows) continue;
    RowOut<T, D>(a, sq, h, -1, r0 + r).put4(4 * piece, acc[r], sum == 0.0f ? 0.0f : 1.0f / sum);
  }
}

template <class T, int D, int NT>
void launch_few(const AttendPlan& p, const AttendArgs& a, hipStream_t stream) {
  const int pages = (min((int64_t)p.chunk, (int64_t)a.b.max_kv) >> a.c.shift) + 2;
  const size_t lds = 4 * 16 * NT * sizeof(float2) + 4 * (D / 16) * 64 * sizeof(f32x4) + pages * sizeof(int);
  const uint32_t x = (uint32_t)p.groups_x(a.c.hkv, a.b.n_seqs);
  const dim3 grid = p.n_splits == 1 || p.runs_in_a_row(a.c.hkv, a.b.n_seqs) ? dim3(x) : dim3(x, a.c.hkv, p.n_splits);
  few_kernel<T, D, NT><<<grid, 256, lds, stream>>>(a);
}

template <class T, int D>
hipError_t launch(int dtype, const AttendPlan& p, const AttendArgs& a, hipStream_t stream) {
  if (p.tile_rows > 32)
    launch_attend_many(dtype, D, p, a, stream);
  else if (p.tile_rows == 16)
    launch_few<T, D, 1>(p, a, stream);
  else
    launch_few<T, D, 2>(p, a, stream);
  if (p.n_splits > 1) {
    // Many runs go with few rows: a row to a workgroup (43 runs of 96 rows 5 us,
    // a row to a wave 12).  Else a row to a wave, or four where there are many (3
    // runs of 48,992 rows of 64 19 us, a row to a wave 33; 17 trees of 21 tokens,
    // 5,712 rows, join and all 34 us, with four rows to a wave 36).
    const dim3 grid((uint32_t)p.tiles, a.c.hkv, p.tile_rows);
    if (p.n_splits > 16 && p.tiles * a.c.hkv * p.tile_rows <= 4096)
      join_kernel<T, D><<<grid, 256, 0, stream>>>(a);
    else if (p.tiles * a.c.hkv * p.tile_rows <= 16384)
      join_few_kernel<T, D, 1><<<dim3(grid.x, grid.y, grid.z / 4), 256, 0, stream>>>(a);
    else
      join_few_kernel<T, D, 4><<<dim3(grid.x, grid.y, grid.z / 16), 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

AttendPlan plan_attend(int head_dim, const Batch& b, int hkv, int hq) {
  AttendPlan p{};
  p.group = hq / hkv;
  const int64_t rows = (int64_t)b.max_q * p.group;
  // (64 requests with 32 rows each: 36 us in tiles of 32, 53 in those of 128;
  // with 64 rows each four column tiles a wave took 70, tiles of 128 take 57)
  p.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 128;
  p.out_rows = (int64_t)b.n_tokens * hq;
  p.tiles = rows <= p.tile_rows ? b.n_seqs : (int64_t)b.n_tokens * p.group / p.tile_rows + b.n_seqs;
  // Runs of at least 128 tokens, so many that sequences of max_kv tokens would
  // make 16 workgroups a compute unit, 8 in tiles of 32 rows and in those of 128
  // with heads of 64, 4 with heads of 128 (256 uneven requests of up to 8,000 tokens:
  // 99 us, with 8 105; 64 with 32 rows each: 34 us, with 16 44; 64 with 60 rows on
  // each of 8 heads of 64: 67 us, with 4 99; 17 trees of 21 tokens, heads of 128:
  // 32.5 us, with 8 31; 8 of 16 tokens on 8 heads of 128: 26 us, with 8 35).
  const int64_t per_unit = p.tile_rows == 16 ? 16 : p.tile_rows == 32 || head_dim == 64 ? 8 : 4;
  const int64_t want = per_unit * kComputeUnits, units = p.tiles * hkv;
  int64_t splits = units > 0 ? (want + units - 1) / units : 1;
  int64_t chunk = ((b.max_kv + splits - 1) / splits + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;  // (one request of 700 tokens: 9.5 us, from 256 on 10.9)
  if (chunk > 16384) chunk = 16384;
  p.chunk = (int32_t)chunk;
  p.n_splits = (int32_t)((b.max_kv + chunk - 1) / chunk);
  if (p.n_splits < 1) p.n_splits = 1;
  p.bytes = p.n_splits > 1 ? p.n_splits * p.out_rows * (head_dim + 2) * 4 : 0;
  return p;
}

hipError_t launch_attend(int dtype, int head_dim, const AttendPlan& p, AttendArgs a, hipStream_t stream) {
  a.unit = p.tile_rows > 32 ? kBaseUnit : a.scale2;
  if (dtype == 0)
    return head_dim == 64 ? launch<__bf16, 64>(0, p, a, stream) : launch<__bf16, 128>(0, p, a, stream);
  return head_dim == 64 ? launch<_Float16, 64>(1, p, a, stream) : launch<_Float16, 128>(1, p, a, stream);
}

}  // namespace rt
