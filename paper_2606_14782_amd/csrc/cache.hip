// gfx950 kernels of the cache: block tables from the budgets, the kept
// rows quantised into blocks and read back, and new tokens' rows.
// include/bacon.h states the layouts and the numbers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_dev.h"
#include "cache_rows.h"

namespace bacon {
namespace {

// ------------------------------------------------------------------- clear

__global__ __launch_bounds__(256) void k_cache_clear(CacheDev c, int first_seq, int num_seqs, bool errors) {
  const int64_t per = (int64_t)num_seqs * c.Hkv;             // pairs of a layer, consecutive
  const int64_t pairs = per * c.L, step = (int64_t)gridDim.x * 256;
  const int64_t t0 = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = t0; i < pairs; i += step) {
    const int64_t pair = (i / per * c.B + first_seq) * c.Hkv + i % per;
    c.lens[pair] = 0;
    c.starts[pair] = 0;
  }
  const int64_t row = per * c.max_blocks, n = row * c.L;     // table entries of a layer, consecutive
  for (int64_t i = t0; i < n; i += step)
    c.table[(i / row * c.B + first_seq) * c.Hkv * c.max_blocks + i % row] = -1;
  if (errors && t0 == 0) *c.err = 0;
}

// ------------------------------------------------------------------ tables
// Pairs in (layer, sequence, head) order.  A workgroup owns a few of them and
// sums the needs of all pairs before its own itself: one launch, nothing
// passed between workgroups.  Large workgroups keep that small: of the 16384
// pairs of 32 layers, 64 sequences and 8 heads, 256 workgroups read half on
// average; 1024 of 256 threads spent 14 of 22 us there.
constexpr int kTabPairs = 64;          // most pairs of a workgroup
constexpr int kTabThreads = 1024;

// i / d for i d < 2^32 and d > 1, with magic = 2^32 / d rounded up.
__device__ __forceinline__ unsigned quotient(unsigned i, unsigned magic) { return __umulhi(i, magic); }

// Steps of kTabThreads through rows of `len` entries, without a division a step.
struct Walk {
  int row, at, len, rows, rest;
  __device__ __forceinline__ Walk(int t, int n)
      : row(t / n), at(t % n), len(n), rows(kTabThreads / n), rest(kTabThreads % n) {}
  __device__ __forceinline__ void next() {
    row += rows;
    at += rest;
    if (at >= len) {
      at -= len;
      ++row;
    }
  }
};

struct PairNeed {
  int K, rows, need;
};

// Pair r of layer l of the batch.
__device__ __forceinline__ PairNeed pair_need(const CacheTablesArgs &a, const int *cand, const int *budget, int l,
                                              int r) {
  const int b = a.c.Hkv == 1 ? r : (int)quotient(r, a.head_magic);
  PairNeed n;
  n.K = a.budgets ? a.budgets[(int64_t)l * a.budgets_batch * a.c.Hkv + r] : budget[b];
  n.K = n.K < 0 ? 0 : n.K;
  n.rows = min(n.K, cand[b]) + a.c.W;
  n.need = (int)(((unsigned)n.rows + (unsigned)a.reserve + (1u << a.c.bt_log) - 1u) >> a.c.bt_log);
  return n;
}

__global__ __launch_bounds__(kTabThreads) void k_cache_tables(CacheTablesArgs a, int own) {
  __shared__ int64_t s_sum[kTabThreads / 64], s_k[kTabThreads / 64], s_first[kTabPairs], s_row[kTabPairs];
  __shared__ int s_need[kTabPairs], s_cand[kCacheMaxBatch], s_budget[kCacheMaxBatch];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63, per = a.s.batch * c.Hkv;
  const int pairs = per * c.L, p0 = blockIdx.x * own;
  const int l0 = p0 / per;                                   // p0's layer
  if (t < a.s.batch) {
    s_cand[t] = a.s.cu[t + 1] - a.s.cu[t] - c.W;
    s_budget[t] = a.s.budget[t];
  }
  __syncthreads();
  int64_t sum = 0, ksum = 0;                                 // needs before p0; budgets before p0 in its layer
  Walk w(t, per);
  for (int p = t; p < p0; p += kTabThreads * 8) {
    PairNeed x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i, w.next()) {
      x[i] = PairNeed{0, 0, 0};
      if (p + kTabThreads * i < p0) x[i] = pair_need(a, s_cand, s_budget, w.row, w.at);
      if (w.row != l0) x[i].K = 0;
    }
    unsigned some = 0;                                       // eight needs below 2^28 each
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      some += x[i].need;
      ksum += x[i].K;
    }
    sum += some;
  }
  for (int m = 32; m; m >>= 1) {
    sum += __shfl_xor(sum, m);
    ksum += __shfl_xor(ksum, m);
  }
  if (lane == 0) {
    s_sum[t >> 6] = sum;
    s_k[t >> 6] = ksum;
  }
  __syncthreads();
  const int mine = min(own, pairs - p0);
  if (t < 64) {
    sum = ksum = 0;
    for (int i = 0; i < kTabThreads / 64; ++i) {
      sum += s_sum[i];
      ksum += s_k[i];
    }
    const int p = p0 + lane, l = p / per;
    PairNeed n{0, 0, 0};
    if (lane < mine) n = pair_need(a, s_cand, s_budget, l, p - l * per);
    int64_t need_in = n.need, k_in = n.K;                    // inclusive scans over the lanes
    for (int m = 1; m < kTabPairs; m <<= 1) {
      const int64_t x = __shfl_up(need_in, m), y = __shfl_up(k_in, m);
      if (lane >= m) {
        need_in += x;
        k_in += y;
      }
    }
    const int64_t first = sum + need_in - n.need;
    const int from = max(0, l * per - p0);                   // lane of the layer's first pair, if it is here
    const int64_t start = k_in - n.K - __shfl(k_in - n.K, from & 63) + (l == l0 ? ksum : 0);
    if (lane < mine) {
      const bool fits = first + n.need <= a.num_free && n.need <= c.max_blocks;
      if (!fits) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
      const int64_t pair = ((int64_t)l * c.B + a.first_seq) * c.Hkv + (p - l * per);
      s_first[lane] = first;
      s_need[lane] = fits ? n.need : 0;
      s_row[lane] = pair * c.max_blocks;
      c.lens[pair] = fits ? n.rows : 0;
      c.starts[pair] = start > 0x7FFFFFFF ? -1 : (int)start;   // -1: the store finds no entry there
      if (a.used && p == pairs - 1) *a.used = first + n.need;
    }
  }
  __syncthreads();
  // the table rows: whole waves to a pair, four entries of a thread on their way at a time
  const int wide = a.row_threads;
  for (int q = t / wide; q < mine; q += kTabThreads / wide) {
    const int need = __builtin_amdgcn_readfirstlane(s_need[q]);
    const int64_t first = s_first[q];
    const int32_t *ids = a.free_ids ? a.free_ids + first : nullptr;
    int32_t *row = c.table + s_row[q];
    for (int i0 = t & (wide - 1); i0 < c.max_blocks; i0 += 4 * wide) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * wide;
        id[u] = -1;
        if (i < need) id[u] = ids ? ids[i] : (int)(first + i);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * wide;
        if (i >= c.max_blocks) break;
        if (i < need && (unsigned)id[u] >= (unsigned)c.num_blocks) {
          atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
          id[u] = -1;
        }
        row[i] = id[u];
      }
    }
  }
}

// ------------------------------------------------------------------- store
// A thread holds 4 rows of 8 dimensions of K and of V: lane bits 4 and 5
// choose the rows of a group of 16, so that V's transpose ends in exchanges of
// 16-lane rows and 16-byte stores.  A workgroup takes 4 groups (d 128) or 8.
// Eight codes of a row: the conversion divides by the scale, a power of two,
// and rounds to nearest even.
template <bool BF16>
__device__ __forceinline__ u32x2 raw_codes(const Raw8<BF16> &r, float scale) {
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s16x2 c = {0, 0};
    if constexpr (BF16) {
      const unsigned lo = r.w[2 * i], hi = r.w[2 * i + 1];
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, lo), scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, hi), scale, true);
    } else {
      const u32x4 w = i ? r.x : r.w;
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, true);
    }
    out[i] = __builtin_bit_cast(unsigned, c);
  }
  return out;
}

template <bool BF16, int D, bool STREAM>
__device__ __forceinline__ void store_rows(const CacheStoreArgs &a) {
  constexpr int WG = 128 / D;                                // groups of 16 rows of a wave: 1 or 2
  __shared__ float red[2][4 * WG];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63, gl = c.bt_log - 4;
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
    float top[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      top[kv] = raw_top<BF16>(v[kv]);
#pragma unroll
      for (int m = 1; m < 64; m <<= 1)
        if (WG == 1 || m != 8) top[kv] = fmaxf(top[kv], __shfl_xor(top[kv], m));
    }
    if (gl) {                                                // a block of two or four groups
      __syncthreads();
      if (col == 0 && q == 0) {
        red[0][group] = top[0];
        red[1][group] = top[1];
      }
      __syncthreads();
      for (int i = 0; i < 1 << gl; ++i)
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) top[kv] = fmaxf(top[kv], red[kv][(group >> gl << gl) + i]);
    }
    if (id < 0) continue;
    const int row = (i0 & ((1 << c.bt_log) - 1));            // of the block: this thread's four rows from here on
    const float ks = block_scale(top[0]), vs = block_scale(top[1]);
    if (row == 0 && col == 0) *reinterpret_cast<float2 *>(c.scales + (int64_t)id * 2) = make_float2(ks, vs);
    uint8_t *kd = block_codes<D>(c, id, 0) + row * D + col;
    u32x2 w[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      *reinterpret_cast<u32x2 *>(kd + r * D) = raw_codes<BF16>(v[0][r], ks);
      w[r] = raw_codes<BF16>(v[1][r], vs);
    }
    unsigned x[8];                                           // dimension j: the four rows' bytes
    transpose4(w[0][0], w[1][0], w[2][0], w[3][0], *reinterpret_cast<unsigned(*)[4]>(x));
    transpose4(w[0][1], w[1][1], w[2][1], w[3][1], *reinterpret_cast<unsigned(*)[4]>(x + 4));
    transpose_rows(x[0], x[2], x[4], x[6]);                  // dimension 2 q: the group's 16 rows
    transpose_rows(x[1], x[3], x[5], x[7]);
    uint8_t *vd = block_codes<D>(c, id, 1) + v_at<D>(row & ~15, col + 2 * q);
    *reinterpret_cast<u32x4 *>(vd) = u32x4{x[0], x[2], x[4], x[6]};
    *reinterpret_cast<u32x4 *>(vd + 16) = u32x4{x[1], x[3], x[5], x[7]};
  }
}

// The kept positions of an idx, or rows in order.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_store(CacheStoreArgs a) {
  store_rows<BF16, D, false>(a);
}
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_store_whole(CacheStoreArgs a) {
  store_rows<BF16, D, true>(a);
}

// -------------------------------------------------------------------- load
// The store's division the other way: 16-byte reads of two dimensions' 16
// rows, exchanged between 16-lane rows, then bytes transposed so that a conversion gives
// neighbouring dimensions of a row.  The rows are written past the caches: a
// ragged batch kept whole (220 MB of codes, 918 MB out) takes 177 us, through them 234.
template <bool BF16>
__device__ __forceinline__ void store_codes8(void *p, int64_t i, unsigned lo, unsigned hi, float scale) {
  if constexpr (BF16) {                // values held are bf16 exactly
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    const u32x4 w = {__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, c),
                     __builtin_bit_cast(unsigned, d)};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(p) + i));
  } else {
    float x[4], y[4];
    unpack4(lo, x);
    unpack4(hi, y);
    f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(p) + i);
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]} * scale, q);
    __builtin_nontemporal_store(f32x4{y[0], y[1], y[2], y[3]} * scale, q + 1);
  }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_load(CacheLoadArgs a, unsigned per_pair) {
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
  u32x2 kw[4] = {};
  u32x4 v0 = {0, 0, 0, 0}, v1 = {0, 0, 0, 0};
  float2 scale = {0.f, 0.f};
  if (base >= 0 && base < len && base < start + a.count) {
    const int id = block_id(c, pair, (int)(base >> c.bt_log)), at = (int)base & ((1 << c.bt_log) - 1);
    if (id >= 0) {
      const uint8_t *k = block_codes<D>(c, id, 0) + (at + 4 * q) * D + col;
      const uint8_t *v = block_codes<D>(c, id, 1) + v_at<D>(at, col + 2 * q);
#pragma unroll
      for (int r = 0; r < 4; ++r) kw[r] = *reinterpret_cast<const u32x2 *>(k + r * D);
      v0 = *reinterpret_cast<const u32x4 *>(v);
      v1 = *reinterpret_cast<const u32x4 *>(v + 16);
      scale = *reinterpret_cast<const float2 *>(c.scales + (int64_t)id * 2);
    } else if (col == 0 && q == 0) {
      atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
    }
  }
  unsigned x[8] = {v0[0], v1[0], v0[1], v1[1], v0[2], v1[2], v0[3], v1[3]}, w[8];
  transpose_rows(x[0], x[2], x[4], x[6]);                    // dimension j: this thread's four rows' bytes
  transpose_rows(x[1], x[3], x[5], x[7]);
  transpose4(x[0], x[1], x[2], x[3], *reinterpret_cast<unsigned(*)[4]>(w));
  transpose4(x[4], x[5], x[6], x[7], *reinterpret_cast<unsigned(*)[4]>(w + 4));
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t pos = pos0 + r, o = pos - start;
    if (o < 0 || o >= a.count) continue;
    const bool row = pos >= 0 && pos < len;                  // others hold any bytes
    const int64_t out = (out_pair * a.count + o) * D + col;
    store_codes8<BF16>(a.k, out, row ? kw[r][0] : 0, row ? kw[r][1] : 0, row ? scale.x : 1.f);
    store_codes8<BF16>(a.v, out, row ? w[r] : 0, row ? w[4 + r] : 0, row ? scale.y : 1.f);
  }
}

// ------------------------------------------------------------------ append
// One wave per pair, one touched block after the other.
template <bool BF16, int D>
__global__ __launch_bounds__(64) void k_cache_append(CacheStepArgs a) {
  const CacheDev &c = a.c;
  const int h = blockIdx.x % c.Hkv, b = blockIdx.x / c.Hkv;
  const int64_t pair = pair_of(c, a.layer, a.first_seq + b, h);
  const NewRows n = new_rows(a, pair, b, h, pair_len(c, pair), call_count(a, b));
  if (n.count == 0) return;
  if (!n.room) {
    if (threadIdx.x == 0) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
    return;
  }
  for (int i = n.b0; i <= n.b1; ++i) append_block<BF16, D>(a, pair, n, i);
  if (threadIdx.x == 0) c.lens[pair] = n.len + n.count;
}

// ----------------------------------------------------------------- advance

__global__ __launch_bounds__(256) void k_cache_advance(CacheMoveArgs a) {
  const CacheDev &c = a.c;
  const int per = a.num_seqs * c.Hkv;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)per * a.layers) return;
  const int l = (int)(i / per), r = (int)(i - (int64_t)l * per);
  const int64_t pair = pair_of(c, a.first_layer + l, a.first_seq, 0) + r;
  const int64_t n = (int64_t)pair_len(c, pair) + (a.deltas ? a.deltas[r / c.Hkv] : a.delta);
  const int cap = c.max_blocks << c.bt_log;
  c.lens[pair] = (int)(n < 0 ? 0 : n > cap ? cap : n);
}

int blocks_for(int64_t n, int per, int most) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, (n + per - 1) / per));
}

// The instance for a dtype and head size.
#define CACHE_LAUNCH(kernel, grid, threads, s, ...)                                        \
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

}  // namespace

hipError_t launch_cache_clear(const CacheDev &c, int first_seq, int num_seqs, bool errors, hipStream_t s) {
  const int64_t n = (int64_t)c.L * num_seqs * c.Hkv * c.max_blocks;
  hipLaunchKernelGGL(k_cache_clear, dim3(blocks_for(n, 1024, 4096)), dim3(256), 0, s, c, first_seq, num_seqs, errors);
  return hipGetLastError();
}

hipError_t launch_cache_tables(CacheTablesArgs a, hipStream_t s) {
  const int pairs = a.c.L * a.s.batch * a.c.Hkv;
  const int own = std::max(1, std::min(kTabPairs, pairs / 256));
  a.row_threads = 64;
  while (a.row_threads < kTabThreads && a.row_threads * own < kTabThreads) a.row_threads *= 2;
  a.head_magic = (unsigned)((0x100000000ull + a.c.Hkv - 1) / a.c.Hkv);
  hipLaunchKernelGGL(k_cache_tables, dim3((unsigned)((pairs + own - 1) / own)), dim3(kTabThreads), 0, s, a, own);
  return hipGetLastError();
}

hipError_t launch_cache_store(const CacheStoreArgs &a, bool bf16, int head_dim, int most_rows, hipStream_t s) {
  const int64_t pairs = (int64_t)a.layers * a.s.batch * a.c.Hkv;
  const int rows = 64 * (128 / head_dim), parts = (most_rows + rows - 1) / rows;
  // (lengths known to the device alone may be far below most_rows: a bounded
  // number of workgroups, each of several parts)
  const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>(parts, (1 << 18) / pairs)), a.c.Hkv,
                  a.layers * a.s.batch);
  if (a.c.format == BACON_CACHE_E2M1) return launch_cache4_store(a, bf16, head_dim, grid, s);
  // Whole rows in order are streamed (a ragged batch kept whole: 133 -> 113 us);
  // gathered rows of a prompt just written may still be in the caches (32
  // layers' kept rows that are: 12.6 us, streamed 15.7).
  if (a.idx[0])
    CACHE_LAUNCH(k_cache_store, grid, 256, s, a);
  else
    CACHE_LAUNCH(k_cache_store_whole, grid, 256, s, a);
  return hipGetLastError();
}

static int64_t load_groups_of_pair(int count, int head_dim) {
  const int rows = 16 * 256 / (head_dim / 2);                // a workgroup's; the first lies anywhere in a group of 16
  return (((int64_t)count + 15) / 16 * 16 + 16 + rows - 1) / rows;
}

int64_t cache_load_groups(int64_t pairs, int count, int head_dim) {
  return pairs * load_groups_of_pair(count, head_dim);
}

hipError_t launch_cache_load(const CacheLoadArgs &a, bool bf16, int head_dim, hipStream_t s) {
  const int64_t pairs = (int64_t)a.layers * a.num_seqs * a.c.Hkv;
  const dim3 grid((unsigned)cache_load_groups(pairs, a.count, head_dim));
  if (a.c.format == BACON_CACHE_E2M1)
    return launch_cache4_load(a, bf16, head_dim, grid, (unsigned)load_groups_of_pair(a.count, head_dim), s);
  CACHE_LAUNCH(k_cache_load, grid, 256, s, a, (unsigned)load_groups_of_pair(a.count, head_dim));
  return hipGetLastError();
}

hipError_t launch_cache_append(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s) {
  if (a.c.format == BACON_CACHE_E2M1) return launch_cache4_append(a, bf16, head_dim, s);
  const dim3 grid((unsigned)(a.num_seqs * a.c.Hkv));
  CACHE_LAUNCH(k_cache_append, grid, 64, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_advance(const CacheMoveArgs &a, hipStream_t s) {
  const int64_t n = (int64_t)a.layers * a.num_seqs * a.c.Hkv;
  hipLaunchKernelGGL(k_cache_advance, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace bacon
