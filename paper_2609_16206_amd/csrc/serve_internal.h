// Declarations shared by the serving operators' kernels (kv_append.hip,
// attend_*.hip, sample.hip) and their entry points (serve_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rt {

// A cache, a batch over it and rows of heads, as the kernels read them (the
// public structs with the page size as a shift).
struct Pages {
  void* k;
  void* v;
  int64_t n_pages;
  int32_t hkv, shift;  // page size = 1 << shift tokens
};

struct Batch {
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* table;
  int64_t table_stride;
  int32_t n_seqs, n_tokens, max_q, max_kv;
};

struct Heads {
  char* data;
  int64_t ts, hs;  // strides in elements
};

constexpr int kAppendRows = 4;  // of a workgroup of an append of many rows

struct AppendArgs {
  Pages c;
  Batch b;
  Heads q, qo, k, v;
  const double* inv_freq;
  const int32_t* positions;
  int32_t hq, rot, interleaved;
  float scale;
};

// Rows of a call, over all heads, at most.
constexpr int64_t kMostRows = INT32_MAX - 4096;

// Workgroups of 256 threads in one dimension of a launch, at most: its work
// items are counted in 32 bits.
constexpr int64_t kMostGroups = (1 << 24) - 1;

// A launch of attention: rows of one sequence and KV head are (token, query
// head of the group) pairs, tile_rows of them to a workgroup; the cache is
// cut into n_splits runs of `chunk` tokens that separate workgroups take.
struct AttendPlan {
  int32_t group, tile_rows, chunk, n_splits;
  int64_t tiles;     // row tiles of all sequences
  int64_t out_rows;  // n_tokens * query heads
  int64_t bytes;     // partial results: per split and row head_dim floats, then per split and row (max, sum)

  // Launched in one dimension, for nth_run, unless sequences or runs are very many.
  bool runs_in_a_row(int32_t hkv, int32_t n_seqs) const {
    return n_seqs <= 1024 && tiles * hkv * n_splits <= 1 << 20;
  }
  // Workgroups in x: few rows in runs go by sequence, KV head and run, many by
  // tile and head, and run.
  int64_t groups_x(int32_t hkv, int32_t n_seqs) const {
    if (n_splits == 1 || runs_in_a_row(hkv, n_seqs)) return tiles * hkv * n_splits;
    return tile_rows > 32 ? tiles * hkv : tiles;
  }
};

struct AttendArgs {
  Pages c;
  Batch b;
  Heads q, o;
  const uint64_t* tree;
  int32_t hq, group, tile_rows, chunk, n_splits;
  float scale2;      // scale * log2(e)
  float* part_o;     // [n_splits][n_tokens * hq][head_dim]
  float2* part_ml;   // [n_splits][n_tokens * hq] reference of the weights, in units, and their sum
  float unit;        // powers of two to a unit: no finite score's reference leaves float32
};

struct SampleArgs {
  const void* logits;
  int64_t stride;
  int64_t n_rows;
  int32_t vocab;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const uint64_t* bits;
  int32_t* out;
  char* ws;
};

hipError_t launch_append(int dtype, int head_dim, const AppendArgs& a, hipStream_t stream);
AttendPlan plan_attend(int head_dim, const Batch& b, int hkv, int hq);
hipError_t launch_attend(int dtype, int head_dim, const AttendPlan& p, AttendArgs a, hipStream_t stream);
void launch_attend_many(int dtype, int head_dim, const AttendPlan& p, const AttendArgs& a, hipStream_t stream);
int64_t sample_workspace(int64_t n_rows, int32_t vocab);
hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t stream);

}  // namespace rt
