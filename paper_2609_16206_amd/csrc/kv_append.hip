// rt_kv_append: rotation of queries and keys, and the write of keys and
// values into the pages of a cache.
//
//   (a, b) -> scale (a cos - b sin, b cos + a sin),  angle = position * inv_freq[j]
//
// The angle is taken in turns and float64, reduced to half a turn exactly, and
// only then rounded to float32 (error 2^-26 turns, beside float64's own of
// 2^-51 of the angle at far positions); the products are float32, and a value
// is rounded once, to the cache's type.
//
// A workgroup takes kRows rows.  One wave per row finds its sequence and
// place and the row's sines, once for all heads; then threads take 16 elements
// each of q and k (two 16-byte vectors, a pair's halves in one thread), and
// 8 x 8 blocks of v: eight tokens of one group of a page are transposed in
// registers into 16-byte stores, and the tokens of a group that is not whole
// are stored one by one (2 bytes at a stride of 16).
//
// Each input is read and each output written once.  18,606 rows of prompts with
// 16 query heads and 2 KV heads of 128: 191 MB in 42 us, 4.5 TB/s (a large copy
// reaches 4.9).  A decode batch is bound by its launch and four dependent loads:
// 3.7 us for one row, 5.8 us for 192 rows of 32 + 8 heads.
#include "serve_device.h"

namespace rt {
namespace {

struct RowPlace {
  int page;   // -1: do not write
  int slot;   // token of the page
  int run;    // rows of the 8-token group that starts here (0: not its first row)
  int state;  // 0 belongs to no sequence, 1 fine, 2 rejected
};

template <class T>
__device__ __forceinline__ void turn8(typename Half<T>::x8& a, typename Half<T>::x8& b, const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = (float)a[i], y = (float)b[i], c = cs[i].x, s = cs[i].y;
    a[i] = (T)__builtin_fmaf(x, c, -(y * s));
    b[i] = (T)__builtin_fmaf(y, c, x * s);
  }
}

template <class T>
__device__ __forceinline__ void turn_pairs8(typename Half<T>::x8& a, const float2* cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = (float)a[2 * i], y = (float)a[2 * i + 1], c = cs[i].x, s = cs[i].y;
    a[2 * i] = (T)__builtin_fmaf(x, c, -(y * s));
    a[2 * i + 1] = (T)__builtin_fmaf(y, c, x * s);
  }
}

template <class T, int D, int kRows>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  typedef typename Half<T>::x8 x8;
  __shared__ RowPlace place[kRows];
  __shared__ float2 cs[kRows][D / 2];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row0 = (int)blockIdx.x * kRows;
  const int ps = 1 << a.c.shift;

  if (wave < kRows && row0 + wave < a.b.n_tokens) {
    const int row = row0 + wave;
    const int s = seq_of_row(a.b, row);
    RowPlace p{-1, 0, 0, 0};
    if (s >= 0) {
      const Seq q = load_seq(a.b, s);
      p.state = 2;
      if (q.ok) {
        const int at = q.kvl - q.n + (row - q.q0);
        const int page = a.b.table[(int64_t)s * a.b.table_stride + (at >> a.c.shift)];
        if (page >= 0 && page < a.c.n_pages) {
          p.state = 1;
          p.page = page;
          p.slot = at & (ps - 1);
          if ((at & 7) == 0 || row == q.q0) p.run = min(8 - (at & 7), q.q0 + q.n - row);
        }
        if (lane < a.rot / 2) {
          const int pos = a.positions ? a.positions[row] : at;
          const double turns = (double)pos * (a.inv_freq[lane] * 0.15915494309189533577);
          const float f = (float)(turns - __builtin_rint(turns));
          float sn, cn;
          sincospif(2.0f * f, &sn, &cn);
          cs[wave][lane] = make_float2(cn * a.scale, sn * a.scale);
        }
      }
    }
    if (lane == 0) place[wave] = p;
  }
  __syncthreads();

  const int rows = min(kRows, a.b.n_tokens - row0);
  const int heads = (a.q.data ? a.hq : 0) + a.c.hkv;
  constexpr int kC = D / 16;
  for (int it = tid; it < rows * heads * kC; it += 256) {
    const int c = it % kC, h = it / kC % heads, r = it / (kC * heads);
    const RowPlace p = place[r];
    const bool is_k = h < a.c.hkv;
    if (p.state == 0 || (is_k && p.state == 2)) continue;
    const bool turned = c < a.rot / 16, halves = turned && !a.interleaved;
    const int e0 = halves ? 8 * c : 16 * c, e1 = halves ? a.rot / 2 + 8 * c : 16 * c + 8;
    const int64_t row = row0 + r;
    T* dst;
    const T* src;
    if (is_k) {
      src = (const T*)a.k.data + row * a.k.ts + h * a.k.hs;
      dst = (T*)a.c.k + ((((int64_t)p.page * a.c.hkv + h) << a.c.shift) + p.slot) * D;
    } else {
      src = (const T*)a.q.data + row * a.q.ts + (h - a.c.hkv) * a.q.hs;
      dst = (T*)a.qo.data + row * a.qo.ts + (h - a.c.hkv) * a.qo.hs;
    }
    x8 x = *(const x8*)(src + e0), y = *(const x8*)(src + e1);
    if (p.state == 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i] = (T)__builtin_nanf("");
    } else if (halves) {
      turn8<T>(x, y, &cs[r][8 * c]);
    } else if (turned) {
      turn_pairs8<T>(x, &cs[r][8 * c]);
      turn_pairs8<T>(y, &cs[r][8 * c + 4]);
    }
    *(x8*)(dst + e0) = x;
    *(x8*)(dst + e1) = y;
  }

  constexpr int kV = D / 8;
  for (int it = tid; it < rows * a.c.hkv * kV; it += 256) {
    const int c = it % kV, h = it / kV % a.c.hkv, r = it / (kV * a.c.hkv);
    const RowPlace p = place[r];
    if (p.run == 0) continue;
    const T* src = (const T*)a.v.data + (int64_t)(row0 + r) * a.v.ts + h * a.v.hs + 8 * c;
    T* dst = (T*)a.c.v + (((((int64_t)p.page * a.c.hkv + h) << a.c.shift) + (p.slot & ~7)) * D + 64 * c);
    if (p.run == 8) {
      x8 t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = *(const x8*)(src + i * a.v.ts);
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = t[i][d];
        *(x8*)(dst + 8 * d) = o;
      }
    } else {
      for (int i = 0; i < p.run; ++i) {
        const x8 x = *(const x8*)(src + i * a.v.ts);
#pragma unroll
        for (int d = 0; d < 8; ++d) dst[8 * d + (p.slot & 7) + i] = x[d];
      }
    }
  }
}

template <class T, int D>
hipError_t launch(const AppendArgs& a, hipStream_t stream) {
  // Four rows share a workgroup's start where there are many (18,606 rows of 16 + 2
  // heads 44 us, one a workgroup 49); few leave compute units idle that way (512
  // rows 6.1 us, one a workgroup 5.1; 2,000 rows 10.9 and 10.2, 4,000 rows 18.0 and 18.8).
  if (a.b.n_tokens >= 10 * kComputeUnits)
    append_kernel<T, D, kAppendRows><<<(a.b.n_tokens + kAppendRows - 1) / kAppendRows, 256, 0, stream>>>(a);
  else
    append_kernel<T, D, 1><<<a.b.n_tokens, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(int dtype, int head_dim, const AppendArgs& a, hipStream_t stream) {
  if (dtype == 0) return head_dim == 64 ? launch<__bf16, 64>(a, stream) : launch<__bf16, 128>(a, stream);
  return head_dim == 64 ? launch<_Float16, 64>(a, stream) : launch<_Float16, 128>(a, stream);
}

}  // namespace rt
