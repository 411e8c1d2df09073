// Entry points of the serving operators (include/rt_router.h): argument
// checks and launches.  Nothing is allocated here and no array is read.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "rt_error.h"
#include "serve_internal.h"

namespace {

// rt::fail and rt::hip_fail for "fn: name what"; without memory for the message
// the status alone goes back.  Nothing else here allocates or throws.
rt_status bad(rt_status s, const char* fn, const char* what, const char* name = "") noexcept {
  try {
    return rt::fail(s, std::string(fn) + ": " + name + what);
  } catch (...) {
    return s;
  }
}
rt_status launched(hipError_t e, const char* what) noexcept {
  if (e == hipSuccess) return RT_OK;
  try {
    return rt::hip_fail(e, what);
  } catch (...) {
    return RT_EDEVICE;
  }
}

constexpr int64_t kMaxInt = INT32_MAX;
constexpr int32_t kMaxKv = 1 << 28;  // splits of 16,384 tokens stay within a launch's grid
constexpr int32_t kMaxVocab = 262144;

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

rt_status check_cache(const char* fn, const rt_kv_cache* c) {
  if (!c) return bad(RT_EINVAL, fn, "null cache");
  if (c->dtype != RT_BF16 && c->dtype != RT_FP16) return bad(RT_EINVAL, fn, "cache dtype must be RT_BF16 or RT_FP16");
  if (c->n_kv_heads < 1) return bad(RT_EINVAL, fn, "n_kv_heads must be >= 1");
  if (c->n_kv_heads > 1024) return bad(RT_ERANGE, fn, "n_kv_heads > 1024");
  if (c->head_dim < 1) return bad(RT_EINVAL, fn, "head_dim must be >= 1");
  if (c->head_dim != 64 && c->head_dim != 128) return bad(RT_EUNSUPPORTED, fn, "head_dim must be 64 or 128");
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return bad(RT_EINVAL, fn, "page_size must be a power of two in [16, 1024]");
  if (c->n_pages < 1 || c->n_pages > kMaxInt) return bad(RT_EINVAL, fn, "n_pages must be in [1, 2^31)");
  return RT_OK;
}

rt_status check_sizes(const char* fn, const rt_kv_cache* c, const rt_kv_batch* b) {
  if (!b) return bad(RT_EINVAL, fn, "null batch");
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_q < 0 || b->max_kv < 0) return bad(RT_EINVAL, fn, "negative size");
  if (b->n_seqs >= kMaxInt || b->n_tokens >= kMaxInt) return bad(RT_ERANGE, fn, "n_seqs and n_tokens must be < 2^31 - 1");
  if (b->max_kv > kMaxKv) return bad(RT_ERANGE, fn, "max_kv > 2^28");
  if (b->table_stride < ((int64_t)b->max_kv + c->page_size - 1) / c->page_size)
    return bad(RT_EINVAL, fn, "table_stride does not hold max_kv tokens");
  if (b->n_seqs > 0 && b->table_stride > INT64_MAX / b->n_seqs) return bad(RT_ERANGE, fn, "size overflow");
  return RT_OK;
}

rt_status check_arrays(const char* fn, const rt_kv_cache* c, const rt_kv_batch* b) {
  if (!c->k || !c->v || !b->q_start || !b->kv_len || !b->page_table) return bad(RT_EINVAL, fn, "null array");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return bad(RT_EINVAL, fn, "k and v must be 16-byte aligned");
  return RT_OK;
}

// `rows`: tokens; heads overlap nothing in an output.
rt_status check_heads(const char* fn, const char* name, const rt_heads* h, int32_t n_heads, int32_t head_dim,
                      int64_t rows, bool output) {
  if (!h || !h->data) return bad(RT_EINVAL, fn, " is null", name);
  if (!aligned(h->data, 16)) return bad(RT_EINVAL, fn, " must be 16-byte aligned", name);
  if (h->token_stride < 0 || h->head_stride < 0 || h->token_stride % 8 || h->head_stride % 8)
    return bad(RT_EINVAL, fn, ": strides must be >= 0 and multiples of 8", name);
  if ((n_heads > 1 && h->head_stride > (INT64_MAX >> 4) / n_heads) ||
      (rows > 1 && h->token_stride > (INT64_MAX >> 4) / rows))
    return bad(RT_ERANGE, fn, ": size overflow", name);
  if (output) {
    // heads side by side within a token, or tokens side by side within a head
    const bool hs_ok = n_heads == 1 || h->head_stride >= head_dim, ts_ok = rows <= 1 || h->token_stride >= head_dim;
    const bool heads_in = rows <= 1 || h->token_stride >= (n_heads - 1) * h->head_stride + head_dim;
    const bool tokens_in = n_heads == 1 || h->head_stride >= (rows - 1) * h->token_stride + head_dim;
    if (!hs_ok || !ts_ok || !(heads_in || tokens_in)) return bad(RT_EINVAL, fn, ": rows overlap", name);
  }
  return RT_OK;
}

rt::Pages pages(const rt_kv_cache& c) {
  rt::Pages p;
  p.k = c.k;
  p.v = c.v;
  p.n_pages = c.n_pages;
  p.hkv = c.n_kv_heads;
  p.shift = 0;
  while ((1 << p.shift) < c.page_size) ++p.shift;
  return p;
}

rt::Batch batch_of(const rt_kv_batch& b) {
  rt::Batch r;
  r.q_start = b.q_start;
  r.kv_len = b.kv_len;
  r.table = b.page_table;
  r.table_stride = b.table_stride;
  r.n_seqs = (int32_t)b.n_seqs;
  r.n_tokens = (int32_t)b.n_tokens;
  r.max_q = (int32_t)std::min<int64_t>(b.max_q, b.n_tokens);
  r.max_kv = b.max_kv;
  return r;
}

rt::Heads heads_of(const rt_heads* h) {
  rt::Heads r{nullptr, 0, 0};
  if (h) r = {(char*)h->data, h->token_stride, h->head_stride};
  return r;
}

rt_status check_q_heads(const char* fn, int32_t hq, int32_t hkv) {
  if (hq < 1 || hq % hkv != 0) return bad(RT_EINVAL, fn, "n_q_heads must be a multiple of n_kv_heads");
  if (hq / hkv > 64) return bad(RT_ERANGE, fn, "more than 64 query heads per KV head");
  return RT_OK;
}

// The plan of a call whose sizes have been checked, or RT_ERANGE.
rt_status plan(const char* fn, const rt_kv_cache& c, const rt_kv_batch& b, int32_t hq, rt::AttendPlan* p) {
  *p = rt::plan_attend(c.head_dim, batch_of(b), c.n_kv_heads, hq);
  if (p->groups_x(c.n_kv_heads, (int32_t)b.n_seqs) > rt::kMostGroups || p->out_rows > rt::kMostRows)
    return bad(RT_ERANGE, fn, "too many sequences or rows");
  return RT_OK;
}

}  // namespace

extern "C" {

rt_status rt_kv_append(const rt_kv_cache* cache, const rt_kv_batch* batch, const rt_rope* rope,
                       const int32_t* positions, int32_t n_q_heads, const rt_heads* q, const rt_heads* q_out,
                       const rt_heads* k, const rt_heads* v, void* hip_stream) {
  const char* fn = "rt_kv_append";
  rt_status st;
  if ((st = check_cache(fn, cache)) != RT_OK || (st = check_sizes(fn, cache, batch)) != RT_OK) return st;
  if ((batch->n_tokens + rt::kAppendRows - 1) / rt::kAppendRows > rt::kMostGroups)
    return bad(RT_ERANGE, fn, "n_tokens must be below 2^26 - 3");
  if (q && (n_q_heads < 1 || n_q_heads > 65536)) return bad(RT_EINVAL, "rt_kv_append", "n_q_heads must be in [1, 65536]");
  if (rope) {
    if (rope->rot_dim < 16 || rope->rot_dim > cache->head_dim || rope->rot_dim % 16 != 0)
      return bad(RT_EINVAL, "rt_kv_append", "rot_dim must be a multiple of 16 in [16, head_dim]");
    if (rope->interleaved != 0 && rope->interleaved != 1)
      return bad(RT_EINVAL, "rt_kv_append", "interleaved must be 0 or 1");
    if (!std::isfinite(rope->scale)) return bad(RT_EINVAL, "rt_kv_append", "the rotation's scale must be finite");
    if (!rope->inv_freq) return bad(RT_EINVAL, "rt_kv_append", "null inv_freq");
  }
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return RT_OK;
  if ((st = check_arrays(fn, cache, batch)) != RT_OK) return st;
  const int32_t d = cache->head_dim;
  const int64_t rows = batch->n_tokens;
  if ((st = check_heads(fn, "k", k, cache->n_kv_heads, d, rows, false)) != RT_OK ||
      (st = check_heads(fn, "v", v, cache->n_kv_heads, d, rows, false)) != RT_OK)
    return st;
  if (q && ((st = check_heads(fn, "q", q, n_q_heads, d, rows, false)) != RT_OK ||
            (st = check_heads(fn, "q_out", q_out, n_q_heads, d, rows, true)) != RT_OK))
    return st;
  if (q && q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))
    return bad(RT_EINVAL, "rt_kv_append", "q_out in the place of q must have its strides");
  rt::AppendArgs a;
  a.c = pages(*cache);
  a.b = batch_of(*batch);
  a.q = heads_of(q);
  a.qo = heads_of(q_out);
  a.k = heads_of(k);
  a.v = heads_of(v);
  a.inv_freq = rope ? rope->inv_freq : nullptr;
  a.positions = positions;
  a.hq = q ? n_q_heads : 0;
  a.rot = rope ? rope->rot_dim : 0;
  a.interleaved = rope ? rope->interleaved : 0;
  a.scale = rope ? rope->scale : 1.0f;
  const hipError_t e = rt::launch_append(cache->dtype, d, a, (hipStream_t)hip_stream);
  return launched(e, "launch(kv_append)");
}

rt_status rt_paged_attention_workspace(const rt_kv_cache* cache, const rt_kv_batch* batch, int32_t n_q_heads,
                                       int64_t* bytes) {
  const char* fn = "rt_paged_attention_workspace";
  rt_status st;
  if (!bytes) return bad(RT_EINVAL, "rt_paged_attention_workspace", "null pointer");
  if ((st = check_cache(fn, cache)) != RT_OK || (st = check_sizes(fn, cache, batch)) != RT_OK ||
      (st = check_q_heads(fn, n_q_heads, cache->n_kv_heads)) != RT_OK)
    return st;
  rt::AttendPlan p;
  if ((st = plan(fn, *cache, *batch, n_q_heads, &p)) != RT_OK) return st;
  *bytes = p.bytes;
  return RT_OK;
}

rt_status rt_paged_attention(const rt_kv_cache* cache, const rt_kv_batch* batch, int32_t n_q_heads, float scale,
                             const rt_heads* q, const uint64_t* tree_mask, const rt_heads* out, void* workspace,
                             int64_t workspace_bytes, void* hip_stream) {
  const char* fn = "rt_paged_attention";
  rt_status st;
  if ((st = check_cache(fn, cache)) != RT_OK || (st = check_sizes(fn, cache, batch)) != RT_OK ||
      (st = check_q_heads(fn, n_q_heads, cache->n_kv_heads)) != RT_OK)
    return st;
  if (!std::isfinite(scale) || scale <= 0.0f) return bad(RT_EINVAL, "rt_paged_attention", "scale must be finite and > 0");
  if (scale > 0x1p127f) return bad(RT_ERANGE, "rt_paged_attention", "scale > 2^127");  // (times log2(e): still a float)
  if (tree_mask && batch->max_q > 64) return bad(RT_ERANGE, "rt_paged_attention", "a tree has at most 64 new tokens");
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return RT_OK;
  if ((st = check_arrays(fn, cache, batch)) != RT_OK) return st;
  if ((st = check_heads(fn, "q", q, n_q_heads, cache->head_dim, batch->n_tokens, false)) != RT_OK ||
      (st = check_heads(fn, "out", out, n_q_heads, cache->head_dim, batch->n_tokens, true)) != RT_OK)
    return st;
  rt::AttendPlan p;
  if ((st = plan(fn, *cache, *batch, n_q_heads, &p)) != RT_OK) return st;
  if (p.bytes > 0) {
    if (!workspace || workspace_bytes < p.bytes)
      return bad(RT_EINVAL, "rt_paged_attention", "workspace smaller than rt_paged_attention_workspace says");
    if (!aligned(workspace, 16)) return bad(RT_EINVAL, "rt_paged_attention", "workspace must be 16-byte aligned");
  }
  rt::AttendArgs a;
  a.c = pages(*cache);
  a.b = batch_of(*batch);
  a.q = heads_of(q);
  a.o = heads_of(out);
  a.tree = tree_mask;
  a.hq = n_q_heads;
  a.group = p.group;
  a.tile_rows = p.tile_rows;
  a.chunk = p.chunk;
  a.n_splits = p.n_splits;
  a.scale2 = scale * 1.44269504088896340736f;
  a.part_o = (float*)workspace;
  a.part_ml = p.bytes > 0 ? (float2*)((float*)workspace + p.n_splits * p.out_rows * cache->head_dim) : nullptr;
  const hipError_t e = rt::launch_attend(cache->dtype, cache->head_dim, p, a, (hipStream_t)hip_stream);
  return launched(e, "launch(paged_attention)");
}

rt_status rt_sample_workspace(int64_t n_rows, int32_t vocab, int64_t* bytes) {
  if (!bytes) return bad(RT_EINVAL, "rt_sample_workspace", "null pointer");
  if (n_rows < 0 || vocab < 1) return bad(RT_EINVAL, "rt_sample_workspace", "n_rows must be >= 0 and vocab >= 1");
  if (n_rows > kMaxInt || vocab > kMaxVocab)
    return bad(RT_ERANGE, "rt_sample_workspace", "n_rows must be < 2^31 and vocab <= 262,144");
  *bytes = rt::sample_workspace(n_rows, vocab);
  return RT_OK;
}

rt_status rt_sample_tokens(int32_t dtype, int64_t n_rows, int32_t vocab, const void* logits, int64_t row_stride,
                           const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                           const uint64_t* random_bits, int32_t* out, void* workspace, int64_t workspace_bytes,
                           void* hip_stream) {
  if (dtype != RT_BF16 && dtype != RT_FP16 && dtype != RT_FP32) return bad(RT_EINVAL, "rt_sample_tokens", "unknown dtype");
  if (n_rows < 0 || vocab < 1) return bad(RT_EINVAL, "rt_sample_tokens", "n_rows must be >= 0 and vocab >= 1");
  if (n_rows > kMaxInt || vocab > kMaxVocab)
    return bad(RT_ERANGE, "rt_sample_tokens", "n_rows must be < 2^31 and vocab <= 262,144");
  if (row_stride < vocab) return bad(RT_EINVAL, "rt_sample_tokens", "row_stride must be >= vocab");
  if (n_rows == 0) return RT_OK;
  if (row_stride > (INT64_MAX >> 3) / n_rows) return bad(RT_ERANGE, "rt_sample_tokens", "size overflow");
  if (!logits || !random_bits || !out) return bad(RT_EINVAL, "rt_sample_tokens", "null array");
  if (!aligned(logits, dtype == RT_FP32 ? 4 : 2)) return bad(RT_EINVAL, "rt_sample_tokens", "logits not aligned to their type");
  const int64_t need = rt::sample_workspace(n_rows, vocab);
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return bad(RT_EINVAL, "rt_sample_tokens", "workspace smaller than rt_sample_workspace says");
    if (!aligned(workspace, 16)) return bad(RT_EINVAL, "rt_sample_tokens", "workspace must be 16-byte aligned");
  }
  rt::SampleArgs a;
  a.logits = logits;
  a.stride = row_stride;
  a.n_rows = n_rows;
  a.vocab = vocab;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.bits = random_bits;
  a.out = out;
  a.ws = (char*)workspace;
  const hipError_t e = rt::launch_sample(dtype, a, (hipStream_t)hip_stream);
  return launched(e, "launch(sample_tokens)");
}

}  // extern "C"
