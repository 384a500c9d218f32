// Host side of the prompt's attention declared in include/bacon.h: argument
// checks, the division of the work and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/bacon.h"
#include "error.h"
#include "prompt.h"

using namespace bacon;

namespace {

#define TRY(x)                     \
  do {                             \
    bacon_status _s = (x);         \
    if (_s != BACON_OK) return _s; \
  } while (0)

constexpr int kMaxGroup = 1024;            // query heads of a KV head
constexpr int64_t kMaxTokens = 1 << 30;
constexpr int64_t kMaxStride = 1 << 26;    // bytes between rows of K or V: 64 of them within 2^32
constexpr int kMaxUnits = (1 << 24) - 1;   // workgroups of 256 threads: a launch holds fewer than 2^32

bacon_status check_shape(const bacon_shape *s) {
  if (!s) return fail(BACON_ERR_INVALID, "shape is NULL");
  if (s->num_q_heads < 1 || s->num_kv_heads < 1) return fail(BACON_ERR_INVALID, "head counts must be >= 1");
  if (s->num_q_heads % s->num_kv_heads)
    return fail(BACON_ERR_INVALID, "num_q_heads (%d) is not a multiple of num_kv_heads (%d)", s->num_q_heads,
                s->num_kv_heads);
  if (s->window < 1) return fail(BACON_ERR_INVALID, "window must be >= 1");
  if (s->max_batch < 1) return fail(BACON_ERR_INVALID, "max_batch must be >= 1");
  if (s->max_total_tokens < 1) return fail(BACON_ERR_INVALID, "max_total_tokens must be >= 1");
  if (s->dtype != BACON_FP32 && s->dtype != BACON_BF16)
    return fail(BACON_ERR_UNSUPPORTED, "dtype %d is not supported", (int)s->dtype);
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail(BACON_ERR_UNSUPPORTED, "head_dim %d is not supported (64 or 128)", s->head_dim);
  if (s->max_batch > kPromptMaxBatch)
    return fail(BACON_ERR_UNSUPPORTED, "max_batch %d exceeds %d", s->max_batch, kPromptMaxBatch);
  if (s->num_q_heads / s->num_kv_heads > kMaxGroup)
    return fail(BACON_ERR_UNSUPPORTED, "%d query heads per KV head exceed %d", s->num_q_heads / s->num_kv_heads,
                kMaxGroup);
  if (s->max_total_tokens > kMaxTokens) return fail(BACON_ERR_UNSUPPORTED, "max_total_tokens too large");
  return BACON_OK;
}

bacon_status check_cu(const bacon_shape *s, const int32_t *cu, int batch, const char *name, int64_t most) {
  if (cu[0] != 0) return fail(BACON_ERR_INVALID, "%s[0] must be 0", name);
  for (int b = 0; b < batch; ++b)
    if (cu[b + 1] < cu[b]) return fail(BACON_ERR_INVALID, "%s falls at sequence %d", name, b);
  if (cu[batch] > most)
    return fail(BACON_ERR_INVALID, "%s: %d tokens exceed %lld", name, cu[batch], (long long)most);
  return BACON_OK;
}

// The batch's sequences that have queries, divided.  window_ends: tokens of each prompt
// at its end, whose last W the window is of (NULL: its keys).
bacon_status check_batch(const bacon_shape *s, const bacon_batch *bt, const int32_t *cu_queries,
                         const int32_t *window_ends, PromptArgs *a, PromptPlan *plan) {
  TRY(check_shape(s));
  if (!bt) return fail(BACON_ERR_INVALID, "batch is NULL");
  if (bt->batch < 1 || bt->batch > s->max_batch)
    return fail(BACON_ERR_INVALID, "batch %d outside [1, %d]", bt->batch, s->max_batch);
  if (!bt->cu_seqlens) return fail(BACON_ERR_INVALID, "batch arrays are NULL");
  TRY(check_cu(s, bt->cu_seqlens, bt->batch, "cu_seqlens", s->max_total_tokens));
  const int32_t *cuq = cu_queries ? cu_queries : bt->cu_seqlens;
  TRY(check_cu(s, cuq, bt->batch, "cu_queries", kMaxTokens));
  a->Hq = s->num_q_heads;
  a->Hkv = s->num_kv_heads;
  a->G = s->num_q_heads / s->num_kv_heads;
  a->W = s->window;
  a->group_magic = a->G == 1 ? 0 : (unsigned)((0x100000000ull + a->G - 1) / a->G);
  a->scale = (float)(1.0 / std::sqrt((double)s->head_dim));
  for (int b = 0; b < bt->batch; ++b) {
    const int queries = cuq[b + 1] - cuq[b], keys = bt->cu_seqlens[b + 1] - bt->cu_seqlens[b];
    if (window_ends && window_ends[b] < keys)
      return fail(BACON_ERR_INVALID, "sequence %d has %d keys, its window ends at token %d", b, keys, window_ends[b]);
    if (queries == 0) continue;
    if ((int64_t)queries * a->G > kMaxTokens)
      return fail(BACON_ERR_UNSUPPORTED, "%d queries of %d heads per KV head are too many", queries, a->G);
    PromptSeq &q = a->s[a->seqs++];
    q.k0 = bt->cu_seqlens[b];
    q.keys = keys;
    q.q0 = cuq[b];
    q.queries = queries;
    q.index = b;
    // (queries are at most 2^30: none of them has an entry where this is below)
    const int64_t to_come = window_ends ? (int64_t)window_ends[b] - keys : 0;
    q.window0 = (int)std::max<int64_t>((int64_t)a->W - queries - to_come, -kMaxTokens);
  }
  *plan = prompt_plan(a, s->head_dim, s->dtype == BACON_BF16);
  if (a->units > kMaxUnits) return fail(BACON_ERR_UNSUPPORTED, "the batch's queries are too many for one call");
  return BACON_OK;
}

bacon_status check_ptr(const void *p, const char *name, size_t align) {
  if (!p) return fail(BACON_ERR_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(BACON_ERR_INVALID, "%s is not %zu-byte aligned", name, align);
  return BACON_OK;
}

bacon_status check_rows(const bacon_shape *s, const void *p, int64_t stride, int heads, const char *name) {
  TRY(check_ptr(p, name, 16));
  const int64_t row = (int64_t)heads * s->head_dim;
  if (stride < row)
    return fail(BACON_ERR_INVALID, "%s rows of %lld elements are %lld elements apart", name, (long long)row,
                (long long)stride);
  if (stride % (s->dtype == BACON_BF16 ? 8 : 4))
    return fail(BACON_ERR_INVALID, "the distance of %s rows (%lld elements) is not a multiple of 16 bytes", name,
                (long long)stride);
  return BACON_OK;
}

// K's and V's tiles are found from their first rows in 32 bits.
bacon_status check_tile(const bacon_shape *s, int64_t stride, const char *name) {
  if (stride * (s->dtype == BACON_BF16 ? 2 : 4) >= kMaxStride)
    return fail(BACON_ERR_UNSUPPORTED, "%s rows of %lld elements' distance are too far apart", name, (long long)stride);
  return BACON_OK;
}

}  // namespace

extern "C" {

size_t bacon_prompt_work_bytes(const bacon_shape *shape, const bacon_batch *batch, const int32_t *cu_queries) {
  PromptArgs a{};
  PromptPlan p{};
  return check_batch(shape, batch, cu_queries, nullptr, &a, &p) == BACON_OK ? p.bytes : 0;
}

bacon_status bacon_prompt_attend_chunk(const bacon_shape *shape, const bacon_batch *batch, const int32_t *cu_queries,
                                       const int32_t *window_ends, const void *d_q, int64_t q_stride, const void *d_k,
                                       int64_t k_stride, const void *d_v, int64_t v_stride, void *d_out, float *d_lse,
                                       float *d_window_lse, void *d_work, size_t work_bytes, void *stream) {
  PromptArgs a{};
  PromptPlan p{};
  TRY(check_batch(shape, batch, cu_queries, window_ends, &a, &p));
  if (a.seqs == 0) return BACON_OK;
  TRY(check_rows(shape, d_q, q_stride, a.Hq, "q"));
  TRY(check_ptr(d_out, "out", 16));
  if (d_lse) TRY(check_ptr(d_lse, "lse", 4));
  if (d_window_lse) TRY(check_ptr(d_window_lse, "window_lse", 4));
  if (batch->cu_seqlens[batch->batch]) {       // (queries of no keys at all need none)
    TRY(check_rows(shape, d_k, k_stride, a.Hkv, "k"));
    TRY(check_rows(shape, d_v, v_stride, a.Hkv, "v"));
    TRY(check_tile(shape, k_stride, "k"));
    TRY(check_tile(shape, v_stride, "v"));
  }
  if (p.bytes) {
    TRY(check_ptr(d_work, "work", 256));
    if (work_bytes < p.bytes)
      return fail(BACON_ERR_WORKSPACE, "the call needs %zu bytes of work, %zu given", p.bytes, work_bytes);
  }
  a.q = d_q;
  a.k = d_k;
  a.v = d_v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.out = d_out;
  a.lse = d_lse;
  a.window = d_window_lse;
  a.part_ml = static_cast<float2 *>(d_work);
  a.part_o = reinterpret_cast<float *>(static_cast<char *>(d_work) + p.ml_bytes);
  const hipError_t e = launch_prompt(a, shape->dtype == BACON_BF16, shape->head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? BACON_OK : fail(BACON_ERR_HIP, "prompt_attend: %s", hipGetErrorString(e));
}

bacon_status bacon_prompt_attend(const bacon_shape *shape, const bacon_batch *batch, const int32_t *cu_queries,
                                 const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride,
                                 const void *d_v, int64_t v_stride, void *d_out, float *d_lse, float *d_window_lse,
                                 void *d_work, size_t work_bytes, void *stream) {
  return bacon_prompt_attend_chunk(shape, batch, cu_queries, nullptr, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_out,
                                   d_lse, d_window_lse, d_work, work_bytes, stream);
}

}  // extern "C"
