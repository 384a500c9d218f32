// gfx950 kernels of the cache in e2m1: the kept rows quantised into blocks and
// read back, and new tokens' rows.  include/bacon.h states the layouts and the
// numbers; clearing, tables and lengths are the same for every format.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_dev.h"
#include "cache_rows.h"

namespace bacon {
namespace {

// ------------------------------------------------------------------- store
// A thread holds 4 rows of 8 dimensions of K and of V, four neighbouring lanes
// a scale's 32 dimensions of them.  Lane bits 4 and 5 choose the rows of a group
// of 16, so that V's transpose ends in exchanges of 16-lane rows and 16-byte
// stores.  Bytes bound it; nothing is read twice or passes between waves.

// Magnitude bits (as a float's) of the largest of eight elements.
template <bool BF16>
__device__ __forceinline__ unsigned row_top(const Raw8<BF16> &r) {
  if constexpr (BF16) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r.w[j] & 0x7FFF7FFFu));
    return (unsigned)(m[0] > m[1] ? m[0] : m[1]) << 16;
  } else {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(max(m, r.w[j] & 0x7FFFFFFFu), r.x[j] & 0x7FFFFFFFu);
    return m;
  }
}

// The largest of four neighbouring lanes.
__device__ __forceinline__ unsigned quad_max(unsigned m) {
  m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));    // lanes 1 0 3 2
  return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true)); // lanes 2 3 0 1
}

template <bool BF16>
__device__ __forceinline__ unsigned raw_codes4(const Raw8<BF16> &r, float scale) {
  unsigned w = 0;
  if constexpr (BF16) {
    const unsigned x0 = r.w[0], x1 = r.w[1], x2 = r.w[2], x3 = r.w[3];
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), scale, 3);
  } else {
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned a = r.w[j], b = r.x[j];
      x[j] = __uint_as_float(a);
      x[4 + j] = __uint_as_float(b);
    }
    return codes4(x, scale);
  }
}

template <bool BF16, int D, bool STREAM>
__device__ __forceinline__ void store_rows4(const CacheStoreArgs &a) {
  constexpr int WG = 128 / D;                                // groups of 16 rows of a wave: 1 or 2
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63;
  const int h = blockIdx.y, b = blockIdx.z % a.s.batch, l = blockIdx.z / a.s.batch;
  const int64_t pair = pair_of(c, a.first_layer + l, a.first_seq + b, h);
  const int len = pair_len(c, pair), cand = a.s.cu[b + 1] - a.s.cu[b] - c.W, kept = len - c.W;
  const int32_t *idx = a.idx[l];
  const int64_t start = c.starts[pair];
  const int group = (t >> 6) * WG + (WG == 2 ? lane >> 3 & 1 : 0);   // of the workgroup's
  const int col = lane % (D / 8) * 8, q = lane >> 4, step = gridDim.x * 64 * WG;
  const int64_t row_elems = (int64_t)c.Hkv * D, first = (int64_t)a.s.cu[b] * row_elems + h * D + col;
  for (int base = blockIdx.x * 64 * WG; base < len; base += step) {
    const int i0 = base + group * 16 + 4 * q, blk = i0 >> c.bt_log;
    Raw8<BF16> v[2][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = i0 + r;
      int at = -1;
      if (i >= kept && i < len)
        at = cand + (i - kept);
      else if (i < kept)
        at = !idx ? i : start >= 0 && start + i < a.idx_count ? idx[start + i] : -1;
      const bool ok = (unsigned)at < (unsigned)(i < kept ? cand : cand + c.W);
      if (i < len && !ok && col == 0) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_INDEX);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        v[kv][r] = Raw8<BF16>{};
        if (ok) v[kv][r] = raw8<BF16, STREAM>(kv ? a.v[l] : a.k[l], first + at * row_elems);
      }
    }
    const bool any = blk << c.bt_log < len;
    const int id = any ? block_id(c, pair, blk) : -1;
    if (any && id < 0 && col == 0 && q == 0) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
    unsigned w[2][4], scales[2] = {0, 0};
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const unsigned byte = scale4_byte(__uint_as_float(quad_max(row_top<BF16>(v[kv][r]))));
        scales[kv] |= byte << (8 * r);
        w[kv][r] = raw_codes4<BF16>(v[kv][r], __uint_as_float(byte << 23));
      }
    unsigned x[4];                                           // byte column j: the four rows' bytes
    transpose4(w[1][0], w[1][1], w[1][2], w[1][3], x);
    transpose_rows(x[0], x[1], x[2], x[3]);                  // byte column q: the group's 16 rows
    if (id < 0) continue;
    const int row = i0 & ((1 << c.bt_log) - 1);              // of the block: this thread's four rows from here on
    if (lane % 4 == 0)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        *reinterpret_cast<unsigned *>(block_scales4<D>(c, id, kv, row >> 4, col / 32) + (row & 15)) = scales[kv];
    uint8_t *kd = block_codes<D / 2>(c, id, 0) + row * (D / 2) + col / 2;
#pragma unroll
    for (int r = 0; r < 4; ++r) *reinterpret_cast<unsigned *>(kd + r * (D / 2)) = w[0][r];
    *reinterpret_cast<u32x4 *>(block_codes<D / 2>(c, id, 1) + v_at<D / 2>(row & ~15, col / 2 + q)) =
        u32x4{x[0], x[1], x[2], x[3]};
  }
}

// The kept positions of an idx, or rows in order.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache4_store(CacheStoreArgs a) {
  store_rows4<BF16, D, false>(a);
}
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache4_store_whole(CacheStoreArgs a) {
  store_rows4<BF16, D, true>(a);
}

// -------------------------------------------------------------------- load
// The store's division the other way.
template <bool BF16>
__device__ __forceinline__ void store_values4(void *p, int64_t i, unsigned w, float scale) {
  if constexpr (BF16) {                // values held are bf16 exactly
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    const u32x4 x = {__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, c),
                     __builtin_bit_cast(unsigned, d)};
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(p) + i));
  } else {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(p) + i);
    __builtin_nontemporal_store(f32x4{a[0], a[1], b[0], b[1]}, q);
    __builtin_nontemporal_store(f32x4{c[0], c[1], d[0], d[1]}, q + 1);
  }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache4_load(CacheLoadArgs a, unsigned per_pair) {
  constexpr int WG = 128 / D;                                // groups of 16 rows of a wave: 1 or 2
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63;
  const int part = (int)(blockIdx.x % per_pair);
  unsigned u = blockIdx.x / per_pair;
  const int64_t out_pair = u;
  const int h = (int)(u % c.Hkv);
  u /= c.Hkv;
  const int64_t pair = pair_of(c, a.first_layer + (int)(u / a.num_seqs), a.first_seq + (int)(u % a.num_seqs), h);
  const int len = pair_len(c, pair), col = lane % (D / 8) * 8, q = lane >> 4;
  const int64_t start = (int64_t)a.first_token + (a.first_token < 0 ? len : 0);   // the pair's row of output row 0
  const int64_t group = (start >> 4) + (int64_t)part * 4 * WG + (t >> 6) * WG + (WG == 2 ? lane >> 3 & 1 : 0);
  const int64_t base = group * 16, pos0 = base + 4 * q;      // this thread's four rows
  unsigned kw[4] = {0, 0, 0, 0}, ks = 0, vs = 0;
  u32x4 v = {0, 0, 0, 0};
  if (base >= 0 && base < len && base < start + a.count) {
    const int id = block_id(c, pair, (int)(base >> c.bt_log)), at = (int)base & ((1 << c.bt_log) - 1);
    if (id >= 0) {
      const uint8_t *k = block_codes<D / 2>(c, id, 0) + (at + 4 * q) * (D / 2) + col / 2;
#pragma unroll
      for (int r = 0; r < 4; ++r) kw[r] = *reinterpret_cast<const unsigned *>(k + r * (D / 2));
      v = *reinterpret_cast<const u32x4 *>(block_codes<D / 2>(c, id, 1) + v_at<D / 2>(at, col / 2 + q));
      ks = *reinterpret_cast<const unsigned *>(block_scales4<D>(c, id, 0, at >> 4, col / 32) + 4 * q);
      vs = *reinterpret_cast<const unsigned *>(block_scales4<D>(c, id, 1, at >> 4, col / 32) + 4 * q);
    } else if (col == 0 && q == 0) {
      atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
    }
  }
  unsigned x[4] = {v[0], v[1], v[2], v[3]}, w[4];
  transpose_rows(x[0], x[1], x[2], x[3]);                    // byte column j: this thread's four rows' bytes
  transpose4(x[0], x[1], x[2], x[3], w);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t pos = pos0 + r, o = pos - start;
    if (o < 0 || o >= a.count) continue;
    const bool row = pos >= 0 && pos < len;                  // others hold any bytes
    const int64_t out = (out_pair * a.count + o) * D + col;
    store_values4<BF16>(a.k, out, row ? kw[r] : 0, row ? scale4(ks, r) : 1.f);
    store_values4<BF16>(a.v, out, row ? w[r] : 0, row ? scale4(vs, r) : 1.f);
  }
}

// ------------------------------------------------------------------ append
// One wave per pair, one touched block after the other.
template <bool BF16, int D>
__global__ __launch_bounds__(64) void k_cache4_append(CacheStepArgs a) {
  const CacheDev &c = a.c;
  const int h = blockIdx.x % c.Hkv, b = blockIdx.x / c.Hkv;
  const int64_t pair = pair_of(c, a.layer, a.first_seq + b, h);
  const NewRows n = new_rows(a, pair, b, h, pair_len(c, pair), call_count(a, b));
  if (n.count == 0) return;
  if (!n.room) {
    if (threadIdx.x == 0) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
    return;
  }
  for (int i = n.b0; i <= n.b1; ++i) append_block4<BF16, D>(a, pair, n, i);
  if (threadIdx.x == 0) c.lens[pair] = n.len + n.count;
}

}  // namespace

#define CACHE4_LAUNCH(kernel, grid, threads, s, ...)                                       \
  do {                                                                                     \
    if (bf16 && head_dim == 128)                                                           \
      hipLaunchKernelGGL((kernel<true, 128>), grid, dim3(threads), 0, s, __VA_ARGS__);     \
    else if (bf16)                                                                         \
      hipLaunchKernelGGL((kernel<true, 64>), grid, dim3(threads), 0, s, __VA_ARGS__);      \
    else if (head_dim == 128)                                                              \
      hipLaunchKernelGGL((kernel<false, 128>), grid, dim3(threads), 0, s, __VA_ARGS__);    \
    else                                                                                   \
      hipLaunchKernelGGL((kernel<false, 64>), grid, dim3(threads), 0, s, __VA_ARGS__);     \
  } while (0)

hipError_t launch_cache4_store(const CacheStoreArgs &a, bool bf16, int head_dim, dim3 grid, hipStream_t s) {
  if (a.idx[0])
    CACHE4_LAUNCH(k_cache4_store, grid, 256, s, a);
  else
    CACHE4_LAUNCH(k_cache4_store_whole, grid, 256, s, a);
  return hipGetLastError();
}

hipError_t launch_cache4_load(const CacheLoadArgs &a, bool bf16, int head_dim, dim3 grid, unsigned per_pair,
                              hipStream_t s) {
  CACHE4_LAUNCH(k_cache4_load, grid, 256, s, a, per_pair);
  return hipGetLastError();
}

hipError_t launch_cache4_append(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s) {
  CACHE4_LAUNCH(k_cache4_append, dim3((unsigned)(a.num_seqs * a.c.Hkv)), 64, s, a);
  return hipGetLastError();
}

}  // namespace bacon
