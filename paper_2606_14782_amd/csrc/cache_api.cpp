// Host side of the cache declared in include/bacon.h: argument checks,
// the layout of its memory and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/bacon.h"
#include "cache.h"
#include "error.h"

using namespace bacon;

struct bacon_cache {
  bacon_cache_shape shape;
  char *mem;
  bacon_cache_offsets off;
  uint64_t cleared = 0;    // sequences that bacon_cache_clear has emptied
};

namespace {

#define TRY(x)                     \
  do {                             \
    bacon_status _s = (x);         \
    if (_s != BACON_OK) return _s; \
  } while (0)

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

bacon_status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return BACON_OK;
  return fail(BACON_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bacon_status check_shape(const bacon_cache_shape *s) {
  if (!s) return fail(BACON_ERR_INVALID, "shape is NULL");
  if (s->num_layers < 1) return fail(BACON_ERR_INVALID, "num_layers must be >= 1");
  if (s->num_q_heads < 1 || s->num_kv_heads < 1) return fail(BACON_ERR_INVALID, "head counts must be >= 1");
  if (s->num_q_heads % s->num_kv_heads)
    return fail(BACON_ERR_INVALID, "num_q_heads (%d) is not a multiple of num_kv_heads (%d)", s->num_q_heads,
                s->num_kv_heads);
  if (s->window < 1) return fail(BACON_ERR_INVALID, "window must be >= 1");
  if (s->max_batch < 1) return fail(BACON_ERR_INVALID, "max_batch must be >= 1");
  if (s->max_blocks < 1) return fail(BACON_ERR_INVALID, "max_blocks must be >= 1");
  if (s->num_blocks < 1) return fail(BACON_ERR_INVALID, "num_blocks must be >= 1");
  if (s->dtype != BACON_FP32 && s->dtype != BACON_BF16)
    return fail(BACON_ERR_UNSUPPORTED, "dtype %d is not supported", (int)s->dtype);
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail(BACON_ERR_UNSUPPORTED, "head_dim %d is not supported (64 or 128)", s->head_dim);
  if (s->block_tokens != 16 && s->block_tokens != 32 && s->block_tokens != 64)
    return fail(BACON_ERR_UNSUPPORTED, "block_tokens %d is not supported (16, 32 or 64)", s->block_tokens);
  if (s->max_batch > kCacheMaxBatch)
    return fail(BACON_ERR_UNSUPPORTED, "max_batch %d exceeds %d", s->max_batch, kCacheMaxBatch);
  if (s->num_q_heads / s->num_kv_heads > kCacheMaxQRows)
    return fail(BACON_ERR_UNSUPPORTED, "%d query heads per KV head exceed %d", s->num_q_heads / s->num_kv_heads,
                kCacheMaxQRows);
  if (s->num_kv_heads > kCacheMaxHeads)
    return fail(BACON_ERR_UNSUPPORTED, "%d KV heads exceed %d", s->num_kv_heads, kCacheMaxHeads);
  if (s->format != BACON_CACHE_E4M3 && s->format != BACON_CACHE_E2M1)
    return fail(BACON_ERR_UNSUPPORTED, "format %d is not supported", s->format);
  if (s->num_blocks > 0x7FFFFFFF) return fail(BACON_ERR_UNSUPPORTED, "num_blocks too large");
  if ((int64_t)s->max_blocks * s->block_tokens > (1 << 30))
    return fail(BACON_ERR_UNSUPPORTED, "a pair's %d blocks of %d tokens exceed 2^30 tokens", s->max_blocks,
                s->block_tokens);
  if ((double)s->num_layers * s->max_batch * s->num_kv_heads > (double)(1 << 24))
    return fail(BACON_ERR_UNSUPPORTED, "more than 2^24 (layer, sequence, KV head) pairs");
  return BACON_OK;
}

int64_t pairs_of(const bacon_cache_shape *s) {
  return (int64_t)s->num_layers * s->max_batch * s->num_kv_heads;
}

// Bytes of a block's codes and of its scales.
int64_t block_bytes(const bacon_cache_shape *s) {
  return 2LL * s->block_tokens * s->head_dim / (s->format == BACON_CACHE_E2M1 ? 2 : 1);
}
int64_t scale_bytes(const bacon_cache_shape *s) {
  return s->format == BACON_CACHE_E2M1 ? 2LL * s->block_tokens * s->head_dim / 32 : 8;
}

bacon_cache_offsets layout_of(const bacon_cache_shape *s) {
  bacon_cache_offsets o{};
  const size_t pairs = (size_t)pairs_of(s);
  size_t at = 0;
  o.errors = at; at += 256;
  o.lens = at;   at += align256(pairs * 4);
  o.starts = at; at += align256(pairs * 4);
  o.table = at;  at += align256(pairs * s->max_blocks * 4);
  o.scales = at; at += align256((size_t)(s->num_blocks * scale_bytes(s)));
  o.codes = at;  at += align256((size_t)(s->num_blocks * block_bytes(s)));
  o.total = at;
  return o;
}

CacheDev device_of(const bacon_cache *c) {
  const bacon_cache_shape &s = c->shape;
  CacheDev d{};
  d.L = s.num_layers;
  d.B = s.max_batch;
  d.Hq = s.num_q_heads;
  d.Hkv = s.num_kv_heads;
  d.W = s.window;
  d.bt_log = s.block_tokens == 16 ? 4 : s.block_tokens == 32 ? 5 : 6;
  d.max_blocks = s.max_blocks;
  d.num_blocks = (int)s.num_blocks;
  d.format = s.format;
  d.lens = reinterpret_cast<int32_t *>(c->mem + c->off.lens);
  d.starts = reinterpret_cast<int32_t *>(c->mem + c->off.starts);
  d.table = reinterpret_cast<int32_t *>(c->mem + c->off.table);
  d.scales = reinterpret_cast<float *>(c->mem + c->off.scales);
  d.scales4 = reinterpret_cast<uint8_t *>(c->mem + c->off.scales);
  d.codes = reinterpret_cast<uint8_t *>(c->mem + c->off.codes);
  d.err = reinterpret_cast<unsigned *>(c->mem + c->off.errors);
  return d;
}

bacon_status check_ptr(const void *p, const char *name, size_t align) {
  if (!p) return fail(BACON_ERR_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(BACON_ERR_INVALID, "%s is not %zu-byte aligned", name, align);
  return BACON_OK;
}

bacon_status check_seqs(const bacon_cache *c, int first, int n) {
  if (!c) return fail(BACON_ERR_INVALID, "cache is NULL");
  if (first < 0 || n < 1 || n > c->shape.max_batch - first)
    return fail(BACON_ERR_INVALID, "sequences %d .. %lld are not within the cache's %d", first,
                (long long)first + n - 1, c->shape.max_batch);
  return BACON_OK;
}

uint64_t seq_mask(int first, int n) { return (n == 64 ? ~0ull : ((1ull << n) - 1)) << first; }

// The last check of a call: its sequences have all been cleared before.
bacon_status check_cleared(const bacon_cache *c, int first, int n) {
  const uint64_t m = seq_mask(first, n);
  if ((c->cleared & m) != m)
    return fail(BACON_ERR_ORDER, "sequences %d .. %d have not been cleared (call bacon_cache_clear)", first,
                first + n - 1);
  return BACON_OK;
}

bacon_status check_layers(const bacon_cache *c, int first, int n) {
  if (first < 0 || n < 1 || n > c->shape.num_layers - first)
    return fail(BACON_ERR_INVALID, "layers %d .. %lld are not within the cache's %d", first,
                (long long)first + n - 1, c->shape.num_layers);
  return BACON_OK;
}

// A prompt's sequences; budgets may be absent where the call does not read them.
bacon_status check_batch(const bacon_cache *c, const bacon_batch *bt, int first, bool budgets, CacheSeqs *out) {
  if (!bt) return fail(BACON_ERR_INVALID, "batch is NULL");
  TRY(check_seqs(c, first, bt->batch));
  if (!bt->cu_seqlens) return fail(BACON_ERR_INVALID, "batch arrays are NULL");
  if (bt->cu_seqlens[0] != 0) return fail(BACON_ERR_INVALID, "cu_seqlens[0] must be 0");
  if (budgets && bt->head_budgets)
    return fail(BACON_ERR_INVALID, "head-wise budgets are given on the device (d_budgets), not in the batch");
  if (budgets && !bt->budgets) return fail(BACON_ERR_INVALID, "batch budgets are NULL");
  *out = CacheSeqs{};
  out->batch = bt->batch;
  for (int b = 0; b < bt->batch; ++b) {
    const int64_t n = (int64_t)bt->cu_seqlens[b + 1] - bt->cu_seqlens[b];
    if (n < c->shape.window)
      return fail(BACON_ERR_INVALID, "sequence %d has %lld tokens, fewer than the window %d", b, (long long)n,
                  c->shape.window);
    out->cu[b + 1] = bt->cu_seqlens[b + 1];
    if (!budgets) continue;
    if (bt->budgets[b] < 1) return fail(BACON_ERR_INVALID, "budget of sequence %d must be >= 1", b);
    out->budget[b] = bt->budgets[b];
  }
  return BACON_OK;
}

int capacity(const bacon_cache *c) { return c->shape.max_blocks * c->shape.block_tokens; }

int elem_size(const bacon_cache *c) { return c->shape.dtype == BACON_BF16 ? 2 : 4; }

// Rows of `heads` x d elements, `stride` elements apart.
bacon_status check_rows(const bacon_cache *c, const void *p, int64_t stride, int heads, const char *name) {
  TRY(check_ptr(p, name, 16));
  const int64_t row = (int64_t)heads * c->shape.head_dim;
  if (stride < row)
    return fail(BACON_ERR_INVALID, "%s rows of %lld elements are %lld elements apart", name, (long long)row,
                (long long)stride);
  if (stride * elem_size(c) % 16)
    return fail(BACON_ERR_INVALID, "the distance of %s rows (%lld elements) is not a multiple of 16 bytes", name,
                (long long)stride);
  return BACON_OK;
}

bacon_status check_tokens(int tokens, const int32_t *d_counts) {
  if (tokens < 1) return fail(BACON_ERR_INVALID, "tokens must be >= 1");
  if (tokens > kCacheMaxTokens)
    return fail(BACON_ERR_UNSUPPORTED, "%d new tokens exceed %d", tokens, kCacheMaxTokens);
  if (d_counts) TRY(check_ptr(d_counts, "counts", 4));
  return BACON_OK;
}

bacon_status check_append(const bacon_cache *c, int layer, int first, int n, int tokens, const int32_t *d_counts,
                          const void *k, int64_t k_stride, const void *v, int64_t v_stride) {
  TRY(check_seqs(c, first, n));
  TRY(check_layers(c, layer, 1));
  TRY(check_tokens(tokens, d_counts));
  TRY(check_rows(c, k, k_stride, c->shape.num_kv_heads, "k"));
  return check_rows(c, v, v_stride, c->shape.num_kv_heads, "v");
}

bacon_status check_attend(const bacon_cache *c, int layer, int first, int n, int tokens, const int32_t *d_counts,
                          const void *q, int64_t q_stride, int max_tokens, const void *out, const float *lse,
                          const void *work, size_t work_bytes) {
  TRY(check_seqs(c, first, n));
  TRY(check_layers(c, layer, 1));
  TRY(check_tokens(tokens, d_counts));
  const int rows = c->shape.num_q_heads / c->shape.num_kv_heads * tokens;
  if (rows > kCacheMaxQRows)
    return fail(BACON_ERR_UNSUPPORTED, "%d query rows per KV head exceed %d", rows, kCacheMaxQRows);
  if (max_tokens < 0) return fail(BACON_ERR_INVALID, "max_tokens must be >= 0");
  TRY(check_rows(c, q, q_stride, c->shape.num_q_heads, "q"));
  TRY(check_ptr(out, "out", 16));
  if (lse) TRY(check_ptr(lse, "lse", 4));
  const size_t need = bacon_cache_work_bytes(c, n, tokens, max_tokens);
  if (need) {
    TRY(check_ptr(work, "work", 256));
    if (work_bytes < need)
      return fail(BACON_ERR_WORKSPACE, "the call needs %zu bytes of work, %zu given", need, work_bytes);
  }
  return check_cleared(c, first, n);
}

CachePlan plan_of(const bacon_cache *c, int num_seqs, int tokens, int max_tokens) {
  const int most = max_tokens ? std::min(max_tokens, capacity(c)) : capacity(c);
  return cache_plan(num_seqs * c->shape.num_kv_heads, c->shape.num_q_heads / c->shape.num_kv_heads * tokens,
                    c->shape.head_dim, most);
}

// The query side of an attend.
void set_query(CacheStepArgs *a, const bacon_cache *c, const void *q, int64_t q_stride, int max_tokens, void *out,
               float *lse, void *work) {
  const CachePlan p = plan_of(c, a->num_seqs, a->tokens, max_tokens);
  a->q = q;
  a->q_stride = q_stride;
  a->out = out;
  a->lse = lse;
  a->splits = p.splits;
  a->chunk = p.chunk;
  a->part_ml = static_cast<float2 *>(work);
  a->part_o = reinterpret_cast<float *>(static_cast<char *>(work) + p.ml_bytes);
}

CacheStepArgs step_args(const bacon_cache *c, int layer, int first, int n, int tokens, const int32_t *d_counts) {
  CacheStepArgs a{};
  a.c = device_of(c);
  a.layer = layer;
  a.first_seq = first;
  a.num_seqs = n;
  a.tokens = tokens;
  a.counts = d_counts;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)c->shape.head_dim));
  return a;
}

}  // namespace

extern "C" {

bacon_status bacon_cache_layout(const bacon_cache_shape *shape, bacon_cache_offsets *out) {
  TRY(check_shape(shape));
  if (!out) return fail(BACON_ERR_INVALID, "offsets are NULL");
  *out = layout_of(shape);
  return BACON_OK;
}

bacon_status bacon_cache_init(bacon_cache **cache, const bacon_cache_shape *shape, void *d_mem, size_t bytes) {
  if (!cache) return fail(BACON_ERR_INVALID, "cache is NULL");
  *cache = nullptr;
  TRY(check_shape(shape));
  if (!d_mem) return fail(BACON_ERR_INVALID, "memory is NULL");
  if (reinterpret_cast<uintptr_t>(d_mem) % 256)
    return fail(BACON_ERR_WORKSPACE, "memory is not 256-byte aligned");
  const bacon_cache_offsets off = layout_of(shape);
  if (bytes < off.total)
    return fail(BACON_ERR_WORKSPACE, "the cache needs %zu bytes, %zu given", off.total, bytes);
  bacon_cache *c = new (std::nothrow) bacon_cache;
  if (!c) return fail(BACON_ERR_INVALID, "out of host memory");
  c->shape = *shape;
  c->mem = static_cast<char *>(d_mem);
  c->off = off;
  *cache = c;
  return BACON_OK;
}

bacon_status bacon_cache_free(bacon_cache *cache) {
  if (!cache) return fail(BACON_ERR_INVALID, "cache is NULL");
  delete cache;
  return BACON_OK;
}

bacon_status bacon_cache_clear(bacon_cache *c, int32_t first_seq, int32_t num_seqs, void *stream) {
  TRY(check_seqs(c, first_seq, num_seqs));
  const bool errors = c->cleared == 0 || num_seqs == c->shape.max_batch;
  TRY(launched(launch_cache_clear(device_of(c), first_seq, num_seqs, errors, static_cast<hipStream_t>(stream)),
               "cache_clear"));
  c->cleared |= seq_mask(first_seq, num_seqs);
  return BACON_OK;
}

bacon_status bacon_cache_tables(bacon_cache *c, const bacon_batch *bt, int32_t first_seq, const int32_t *d_budgets,
                                int32_t budgets_batch, int32_t reserve, const int32_t *d_free, int64_t num_free,
                                int64_t *d_used, void *stream) {
  if (!c) return fail(BACON_ERR_INVALID, "cache is NULL");
  CacheTablesArgs a{};
  TRY(check_batch(c, bt, first_seq, !d_budgets, &a.s));
  if (d_budgets) {
    TRY(check_ptr(d_budgets, "budgets", 4));
    if (budgets_batch < bt->batch)
      return fail(BACON_ERR_INVALID, "budgets of %d sequences for a batch of %d", budgets_batch, bt->batch);
  }
  if (reserve < 0 || reserve > capacity(c))
    return fail(BACON_ERR_INVALID, "reserve %d outside [0, %d]", reserve, capacity(c));
  if (d_free) {
    TRY(check_ptr(d_free, "free", 4));
    if (num_free < 0) return fail(BACON_ERR_INVALID, "num_free must be >= 0");
  }
  if (d_used) TRY(check_ptr(d_used, "used", 8));
  TRY(check_cleared(c, first_seq, bt->batch));
  a.c = device_of(c);
  a.first_seq = first_seq;
  a.budgets = d_budgets;
  a.budgets_batch = budgets_batch;
  a.reserve = reserve;
  a.free_ids = d_free;
  a.num_free = d_free ? num_free : c->shape.num_blocks;
  a.used = d_used;
  return launched(launch_cache_tables(a, static_cast<hipStream_t>(stream)), "cache_tables");
}

bacon_status bacon_cache_store(bacon_cache *c, const bacon_batch *bt, int32_t first_seq, int32_t first_layer,
                               int32_t num_layers, const void *const *d_k, const void *const *d_v,
                               const int32_t *const *d_idx, int64_t idx_count, void *stream) {
  if (!c) return fail(BACON_ERR_INVALID, "cache is NULL");
  CacheStoreArgs a{};
  TRY(check_batch(c, bt, first_seq, false, &a.s));
  TRY(check_layers(c, first_layer, num_layers));
  if (!d_k || !d_v) return fail(BACON_ERR_INVALID, "pointer arrays are NULL");
  if (d_idx && idx_count < 0) return fail(BACON_ERR_INVALID, "idx_count must be >= 0");
  for (int l = 0; l < num_layers; ++l) {
    TRY(check_ptr(d_k[l], "k", 16));
    TRY(check_ptr(d_v[l], "v", 16));
    if (d_idx) TRY(check_ptr(d_idx[l], "idx", 4));
  }
  TRY(check_cleared(c, first_seq, bt->batch));
  int most = 1;
  for (int b = 0; b < bt->batch; ++b) most = std::max(most, bt->cu_seqlens[b + 1] - bt->cu_seqlens[b]);
  most = std::min(most, capacity(c));
  a.c = device_of(c);
  a.idx_count = idx_count;
  a.first_seq = first_seq;
  for (int l = 0; l < num_layers; l += kCacheLayersPerLaunch) {
    a.first_layer = first_layer + l;
    a.layers = std::min(num_layers - l, kCacheLayersPerLaunch);
    for (int i = 0; i < a.layers; ++i) {
      a.k[i] = d_k[l + i];
      a.v[i] = d_v[l + i];
      a.idx[i] = d_idx ? d_idx[l + i] : nullptr;
    }
    TRY(launched(launch_cache_store(a, c->shape.dtype == BACON_BF16, c->shape.head_dim, most,
                                    static_cast<hipStream_t>(stream)),
                 "cache_store"));
  }
  return BACON_OK;
}

bacon_status bacon_cache_load(bacon_cache *c, int32_t first_layer, int32_t num_layers, int32_t first_seq,
                              int32_t num_seqs, int32_t first_token, int32_t count, void *d_k_out, void *d_v_out,
                              void *stream) {
  TRY(check_seqs(c, first_seq, num_seqs));
  TRY(check_layers(c, first_layer, num_layers));
  if (count < 1 || count > (1 << 30)) return fail(BACON_ERR_INVALID, "count %d outside [1, 2^30]", count);
  if (first_token < -(1 << 30) || first_token > (1 << 30))
    return fail(BACON_ERR_INVALID, "first_token %d outside [-2^30, 2^30]", first_token);
  TRY(check_ptr(d_k_out, "k_out", 16));
  TRY(check_ptr(d_v_out, "v_out", 16));
  const int64_t pairs = (int64_t)num_layers * num_seqs * c->shape.num_kv_heads;
  if (cache_load_groups(pairs, count, c->shape.head_dim) > kCacheMaxGroups)
    return fail(BACON_ERR_UNSUPPORTED, "a load of %d rows of %d layers and %d sequences is too large", count,
                num_layers, num_seqs);
  TRY(check_cleared(c, first_seq, num_seqs));
  CacheLoadArgs a{};
  a.c = device_of(c);
  a.first_layer = first_layer;
  a.layers = num_layers;
  a.first_seq = first_seq;
  a.num_seqs = num_seqs;
  a.first_token = first_token;
  a.count = count;
  a.k = d_k_out;
  a.v = d_v_out;
  return launched(launch_cache_load(a, c->shape.dtype == BACON_BF16, c->shape.head_dim,
                                    static_cast<hipStream_t>(stream)),
                  "cache_load");
}

bacon_status bacon_cache_append(bacon_cache *c, int32_t layer, int32_t first_seq, int32_t num_seqs, int32_t tokens,
                                const int32_t *d_counts, const void *d_k, int64_t k_stride, const void *d_v,
                                int64_t v_stride, void *stream) {
  TRY(check_append(c, layer, first_seq, num_seqs, tokens, d_counts, d_k, k_stride, d_v, v_stride));
  TRY(check_cleared(c, first_seq, num_seqs));
  CacheStepArgs a = step_args(c, layer, first_seq, num_seqs, tokens, d_counts);
  a.k = d_k;
  a.v = d_v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  return launched(launch_cache_append(a, c->shape.dtype == BACON_BF16, c->shape.head_dim,
                                      static_cast<hipStream_t>(stream)),
                  "cache_append");
}

size_t bacon_cache_work_bytes(const bacon_cache *c, int32_t num_seqs, int32_t tokens, int32_t max_tokens) {
  if (!c || num_seqs < 1 || num_seqs > c->shape.max_batch || tokens < 1 || tokens > kCacheMaxTokens ||
      max_tokens < 0 || c->shape.num_q_heads / c->shape.num_kv_heads * tokens > kCacheMaxQRows)
    return 0;
  return plan_of(c, num_seqs, tokens, max_tokens).bytes;
}

bacon_status bacon_cache_attend(bacon_cache *c, int32_t layer, int32_t first_seq, int32_t num_seqs, int32_t tokens,
                                const int32_t *d_counts, const void *d_q, int64_t q_stride, int32_t max_tokens,
                                void *d_out, float *d_lse, void *d_work, size_t work_bytes, void *stream) {
  TRY(check_attend(c, layer, first_seq, num_seqs, tokens, d_counts, d_q, q_stride, max_tokens, d_out, d_lse, d_work,
                   work_bytes));
  CacheStepArgs a = step_args(c, layer, first_seq, num_seqs, tokens, d_counts);
  set_query(&a, c, d_q, q_stride, max_tokens, d_out, d_lse, d_work);
  return launched(launch_cache_attend(a, c->shape.dtype == BACON_BF16, c->shape.head_dim,
                                      static_cast<hipStream_t>(stream)),
                  "cache_attend");
}

bacon_status bacon_cache_step(bacon_cache *c, int32_t layer, int32_t first_seq, int32_t num_seqs, int32_t tokens,
                              const int32_t *d_counts, const void *d_q, int64_t q_stride, const void *d_k,
                              int64_t k_stride, const void *d_v, int64_t v_stride, int32_t max_tokens, void *d_out,
                              float *d_lse, void *d_work, size_t work_bytes, void *stream) {
  TRY(check_append(c, layer, first_seq, num_seqs, tokens, d_counts, d_k, k_stride, d_v, v_stride));
  TRY(check_attend(c, layer, first_seq, num_seqs, tokens, d_counts, d_q, q_stride, max_tokens, d_out, d_lse, d_work,
                   work_bytes));
  CacheStepArgs s = step_args(c, layer, first_seq, num_seqs, tokens, d_counts);
  s.k = d_k;
  s.v = d_v;
  s.k_stride = k_stride;
  s.v_stride = v_stride;
  set_query(&s, c, d_q, q_stride, max_tokens, d_out, d_lse, d_work);
  if (!cache_appends(c->shape.num_q_heads / c->shape.num_kv_heads * tokens)) {
    TRY(launched(launch_cache_append(s, c->shape.dtype == BACON_BF16, c->shape.head_dim,
                                     static_cast<hipStream_t>(stream)),
                 "cache_append"));
    s.k = s.v = nullptr;
  }
  return launched(launch_cache_attend(s, c->shape.dtype == BACON_BF16, c->shape.head_dim,
                                      static_cast<hipStream_t>(stream)),
                  "cache_step");
}

bacon_status bacon_cache_advance(bacon_cache *c, int32_t first_layer, int32_t num_layers, int32_t first_seq,
                                 int32_t num_seqs, int32_t delta, const int32_t *d_delta, void *stream) {
  TRY(check_seqs(c, first_seq, num_seqs));
  TRY(check_layers(c, first_layer, num_layers));
  if (d_delta) TRY(check_ptr(d_delta, "delta", 4));
  TRY(check_cleared(c, first_seq, num_seqs));
  CacheMoveArgs a{};
  a.c = device_of(c);
  a.first_layer = first_layer;
  a.layers = num_layers;
  a.first_seq = first_seq;
  a.num_seqs = num_seqs;
  a.delta = delta;
  a.deltas = d_delta;
  return launched(launch_cache_advance(a, static_cast<hipStream_t>(stream)), "cache_advance");
}

int32_t bacon_cache_errors(bacon_cache *c) {
  if (!c) return -1;
  unsigned v = 0;
  if (hipDeviceSynchronize() != hipSuccess ||
      hipMemcpy(&v, c->mem + c->off.errors, sizeof v, hipMemcpyDeviceToHost) != hipSuccess)
    return -1;
  return (int32_t)v;
}

}  // extern "C"
