// gfx950 kernels of the 8-bit cache: block tables from the budgets, the kept
// rows quantised into blocks and read back, new tokens' rows, and attention
// over a layer's cache.  include/bacon.h states the layouts and the numbers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <math.h>
#include <stdint.h>

#include "../../include/bacon.h"
#include "cache.h"

namespace bacon {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kTop = 448.f;          // largest e4m3 value
constexpr float kLn2f = 0.69314718055994531f;

__device__ __forceinline__ float bf16_float(unsigned bits) { return __uint_as_float(bits << 16); }

// bfloat16 bits of x, rounded to nearest, ties to even (x finite).
__device__ __forceinline__ unsigned float_bf16(float x) {
  const unsigned u = __float_as_uint(x);
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// 2^e as a float, -126 <= e <= 127.
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// The scale of a block whose largest magnitude is a: 2^e, e the smallest
// integer with a <= 448 2^e = 1.75 2^(e+8), within the bounds.
__device__ __forceinline__ float block_scale(float a) {
  const unsigned u = __float_as_uint(a);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = e < kCacheLow ? kCacheLow : e > kCacheHigh ? kCacheHigh : e;
  return two_to(e);
}

// Four values, already divided by their scale, as e4m3 bytes.
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (unsigned)r;
}

__device__ __forceinline__ void unpack4(unsigned w, float (&x)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

__device__ __forceinline__ int64_t pair_of(const CacheDev &c, int layer, int seq, int h) {
  return ((int64_t)layer * c.B + seq) * c.Hkv + h;
}

// A pair's length, held to its table.
__device__ __forceinline__ int pair_len(const CacheDev &c, int64_t pair) {
  const int n = c.lens[pair], cap = c.max_blocks << c.bt_log;
  return n < 0 ? 0 : n > cap ? cap : n;
}

// Id of the pair's block i, or -1 where the table holds none of the pool's.
__device__ __forceinline__ int block_id(const CacheDev &c, int64_t pair, int i) {
  const int id = i < c.max_blocks ? c.table[pair * c.max_blocks + i] : -1;
  return (unsigned)id < (unsigned)c.num_blocks ? id : -1;
}

template <int D>
__device__ __forceinline__ uint8_t *block_codes(const CacheDev &c, int id, int kv) {
  return c.codes + (((int64_t)id * 2 + kv) << c.bt_log) * D;
}

__device__ __forceinline__ float wave_max(float v) {
  for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}
__device__ __forceinline__ float wave_add(float v) {
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// The largest v of a 256-thread workgroup; red holds 4 floats, free again
// after the next barrier.
__device__ __forceinline__ float block_max(float v, float *red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

template <bool BF16>
__device__ __forceinline__ float load_elem(const void *p, int64_t i) {
  if constexpr (BF16) return bf16_float(static_cast<const uint16_t *>(p)[i]);
  return static_cast<const float *>(p)[i];
}
template <bool BF16>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float x) {
  if constexpr (BF16)
    static_cast<uint16_t *>(p)[i] = (uint16_t)float_bf16(x);
  else
    static_cast<float *>(p)[i] = x;
}

// Eight consecutive elements as floats (i a multiple of 8).
template <bool BF16>
__device__ __forceinline__ void load8(const void *p, int64_t i, float (&x)[8]) {
  if constexpr (BF16) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_float(w[j] & 0xFFFFu);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  } else {
    const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
    const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

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
// Pairs in (layer, sequence, head) order; a workgroup owns kTabPairs of them and sums
// the needs of all pairs before its own itself, which spares a second launch.
constexpr int kTabPairs = 32;

struct PairNeed {
  int K, rows, need;
};

__device__ __forceinline__ PairNeed pair_need(const CacheTablesArgs &a, int64_t p) {
  const int per = a.s.batch * a.c.Hkv;
  const int l = (int)(p / per), r = (int)(p - (int64_t)l * per), b = r / a.c.Hkv, h = r - b * a.c.Hkv;
  int K = a.budgets ? a.budgets[((int64_t)l * a.budgets_batch + b) * a.c.Hkv + h] : a.s.budget[b];
  K = K < 0 ? 0 : K;
  const int cand = a.s.cu[b + 1] - a.s.cu[b] - a.c.W;
  PairNeed n;
  n.K = K;
  n.rows = (K < cand ? K : cand) + a.c.W;
  n.need = (int)(((int64_t)n.rows + a.reserve + (1 << a.c.bt_log) - 1) >> a.c.bt_log);
  return n;
}

__global__ __launch_bounds__(256) void k_cache_tables(CacheTablesArgs a) {
  __shared__ int64_t s_sum[4], s_k[4], s_first[kTabPairs];
  __shared__ int s_need[kTabPairs];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63, per = a.s.batch * c.Hkv;
  const int64_t pairs = (int64_t)per * c.L, p0 = (int64_t)blockIdx.x * kTabPairs;
  const int64_t layer0 = p0 / per * per;                     // first pair of p0's layer
  int64_t sum = 0, ksum = 0;
  for (int64_t p = t; p < p0; p += 256) {
    const PairNeed n = pair_need(a, p);
    sum += n.need;
    if (p >= layer0) ksum += n.K;
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
  sum = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
  ksum = s_k[0] + s_k[1] + s_k[2] + s_k[3];
  if (t < 64) {
    const int64_t p = p0 + lane;
    const bool mine = lane < kTabPairs && p < pairs;
    PairNeed n{0, 0, 0};
    if (mine) n = pair_need(a, p);
    int64_t need_in = n.need, k_in = n.K;                    // inclusive scans over the lanes
    for (int m = 1; m < kTabPairs; m <<= 1) {
      const int64_t x = __shfl_up(need_in, m), y = __shfl_up(k_in, m);
      if (lane >= m) {
        need_in += x;
        k_in += y;
      }
    }
    const int64_t first = sum + need_in - n.need;
    const int64_t layer = p / per * per;                     // first pair of this pair's layer
    const int from = layer > p0 ? (int)(layer - p0) : 0;     // its lane, if it lies in this workgroup
    const int64_t before = __shfl(k_in - n.K, from);
    const int64_t start = k_in - n.K - before + (layer > p0 ? 0 : ksum);
    if (mine) {
      const bool fits = first + n.need <= a.num_free && n.need <= c.max_blocks;
      if (!fits) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
      s_first[lane] = first;
      s_need[lane] = fits ? n.need : 0;
      const int l = (int)(p / per);
      const int64_t pair = ((int64_t)l * c.B + a.first_seq) * c.Hkv + (p - layer);
      c.lens[pair] = fits ? n.rows : 0;
      c.starts[pair] = (int)start;
      if (a.used && p == pairs - 1) *a.used = first + n.need;
    }
  }
  __syncthreads();
  const int mine = (int)(pairs - p0 < kTabPairs ? pairs - p0 : kTabPairs);
  for (int q = 0; q < mine; ++q) {
    const int64_t p = p0 + q;
    const int64_t pair = (p / per * c.B + a.first_seq) * c.Hkv + p % per;
    for (int i = t; i < c.max_blocks; i += 256) {
      int id = -1;
      if (i < s_need[q]) {
        const int64_t at = s_first[q] + i;
        id = a.free_ids ? a.free_ids[at] : (int)at;
        if ((unsigned)id >= (unsigned)c.num_blocks) {
          atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
          id = -1;
        }
      }
      c.table[pair * c.max_blocks + i] = id;
    }
  }
}

// ------------------------------------------------------------------- store
// A workgroup takes K or V of one block at a time: its rows into registers
// (8 elements a thread and pass), the largest magnitude, the codes out.  V's
// codes are transposed through LDS.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_store(CacheStoreArgs a, int per_pair) {
  constexpr int TR = D / 8, RP = 256 / TR;                   // threads of a row, rows of a pass
  constexpr int PASSES = 64 / RP;                            // of the largest block
  __shared__ float red[4];
  __shared__ alignas(16) uint8_t tile[64 * D];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, bt = 1 << c.bt_log;
  const int x = blockIdx.x % per_pair, kv = blockIdx.y;
  int64_t u = blockIdx.x / per_pair;
  const int h = (int)(u % c.Hkv);
  u /= c.Hkv;
  const int b = (int)(u % a.s.batch), l = (int)(u / a.s.batch);
  const int64_t pair = pair_of(c, a.first_layer + l, a.first_seq + b, h);
  const int len = pair_len(c, pair), cand = a.s.cu[b + 1] - a.s.cu[b] - c.W, kept = len - c.W;
  const void *src = kv ? a.v[l] : a.k[l];
  const int32_t *idx = a.idx[l] ? a.idx[l] + c.starts[pair] : nullptr;
  for (int blk = x; (blk << c.bt_log) < len; blk += per_pair) {
    const int id = block_id(c, pair, blk);
    if (id < 0) {
      if (t == 0) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
      continue;
    }
    float v[PASSES][8];
    float top = 0.f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * RP + t / TR, i = (blk << c.bt_log) + r;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[p][j] = 0.f;
      if (r < bt && i < len) {
        int at = i < kept ? (idx ? idx[i] : i) : cand + (i - kept);
        const bool ok = (unsigned)at < (unsigned)(i < kept ? cand : cand + c.W);
        if (!ok) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_INDEX);
        if (ok) load8<BF16>(src, ((int64_t)(a.s.cu[b] + at) * c.Hkv + h) * D + (t % TR) * 8, v[p]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[p][j]));
    }
    __syncthreads();                                         // red and tile are free
    const float scale = block_scale(block_max(top, red)), inv = 1.f / scale;
    uint8_t *dst = block_codes<D>(c, id, kv);
    if (t == 0) c.scales[(int64_t)id * 2 + kv] = scale;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * RP + t / TR;
      if (r >= bt) continue;
      u32x2 w;
      w[0] = pack4(v[p][0] * inv, v[p][1] * inv, v[p][2] * inv, v[p][3] * inv);
      w[1] = pack4(v[p][4] * inv, v[p][5] * inv, v[p][6] * inv, v[p][7] * inv);
      if (kv == 0) {
        *reinterpret_cast<u32x2 *>(dst + r * D + (t % TR) * 8) = w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[((t % TR) * 8 + j) * bt + r] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
      }
    }
    if (kv == 1) {
      __syncthreads();
      for (int i = t * 16; i < bt * D; i += 256 * 16)
        *reinterpret_cast<u32x4 *>(dst + i) = *reinterpret_cast<const u32x4 *>(tile + i);
    }
  }
}

// -------------------------------------------------------------------- load

template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_load(CacheLoadArgs a, int64_t rows) {
  const CacheDev &c = a.c;
  const int64_t step = (int64_t)gridDim.x * 256, n = rows * D;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const int dim = (int)(i % D);
    int64_t u = i / D;
    const int r = (int)(u % a.count);
    u /= a.count;
    const int h = (int)(u % c.Hkv);
    u /= c.Hkv;
    const int64_t pair = pair_of(c, a.first_layer + (int)(u / a.num_seqs), a.first_seq + (int)(u % a.num_seqs), h);
    const int len = pair_len(c, pair);
    const int64_t pos = (int64_t)a.first_token + r + (a.first_token < 0 ? len : 0);
    float k = 0.f, v = 0.f;
    if (pos >= 0 && pos < len) {
      const int id = block_id(c, pair, (int)(pos >> c.bt_log)), at = (int)pos & ((1 << c.bt_log) - 1);
      if (id >= 0) {
        const unsigned kc = block_codes<D>(c, id, 0)[at * D + dim], vc = block_codes<D>(c, id, 1)[(dim << c.bt_log) + at];
        k = __builtin_amdgcn_cvt_f32_fp8((int)kc, 0) * c.scales[(int64_t)id * 2];
        v = __builtin_amdgcn_cvt_f32_fp8((int)vc, 0) * c.scales[(int64_t)id * 2 + 1];
      } else if (dim == 0) {
        atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
      }
    }
    store_elem<BF16>(a.k, i, k);
    store_elem<BF16>(a.v, i, v);
  }
}

// ------------------------------------------------------------------ append
// One workgroup per pair, K then V, one touched block after the other.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_append(CacheStepArgs a) {
  __shared__ float red[4];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, bt = 1 << c.bt_log, h = blockIdx.x % c.Hkv, b = blockIdx.x / c.Hkv;
  const int64_t pair = pair_of(c, a.layer, a.first_seq + b, h);
  const int len = pair_len(c, pair);
  int count = a.tokens;
  if (a.counts) count = min(max(a.counts[b], 0), a.tokens);
  if (count == 0) return;
  const int b0 = len >> c.bt_log, b1 = (len + count - 1) >> c.bt_log;
  for (int i = b0; i <= b1; ++i)
    if (block_id(c, pair, i) < 0) {
      if (t == 0) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
      return;
    }
  for (int kv = 0; kv < 2; ++kv) {
    const void *src = kv ? a.v : a.k;
    const int64_t stride = kv ? a.v_stride : a.k_stride;
    for (int i = b0; i <= b1; ++i) {
      const int id = block_id(c, pair, i), base = i << c.bt_log;
      const int from = max(len, base), m = min(len + count, base + bt) - from, old = from - base;
      const int64_t row0 = (int64_t)b * a.tokens + (from - len);
      uint8_t *dst = block_codes<D>(c, id, kv);
      float top = 0.f;
      for (int e = t; e < m * D; e += 256)
        top = fmaxf(top, fabsf(load_elem<BF16>(src, (row0 + e / D) * stride + h * D + e % D)));
      const float was = c.scales[(int64_t)id * 2 + kv];
      __syncthreads();
      float scale = block_scale(block_max(top, red));
      if (old && scale < was) scale = was;
      if (old && scale > was) {
        const float f = was / scale;                         // a power of two: the product is exact
        for (int e = t; e < bt * D / 4; e += 256) {
          float x[4];
          unsigned *w = reinterpret_cast<unsigned *>(dst) + e;
          unpack4(*w, x);
          *w = pack4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
        }
      }
      __syncthreads();                                       // the old codes are in place, the scale was read
      if (t == 0) c.scales[(int64_t)id * 2 + kv] = scale;
      const float inv = 1.f / scale;
      for (int e = t; e < m * D; e += 256) {
        const int r = e / D, dim = e % D;
        const float x = load_elem<BF16>(src, (row0 + r) * stride + h * D + dim) * inv;
        const unsigned w = pack4(x, 0.f, 0.f, 0.f);
        dst[kv ? (dim << c.bt_log) + old + r : (old + r) * D + dim] = (uint8_t)w;
      }
    }
  }
  if (t == 0) c.lens[pair] = len + count;
}

// ------------------------------------------------------------------ attend
// One workgroup per query row: logits of 256 rows at a time, the running
// maximum and sum of the softmax, a thread per dimension for the output.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_attend(CacheStepArgs a) {
  constexpr int PARTS = 256 / D;
  __shared__ float red[4], q[D], p[256], part[256];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, G = c.Hq / c.Hkv, bt = 1 << c.bt_log;
  const int hq = blockIdx.x % c.Hq, j = blockIdx.x / c.Hq % a.tokens, b = blockIdx.x / c.Hq / a.tokens;
  const int64_t pair = pair_of(c, a.layer, a.first_seq + b, hq / G), row = (int64_t)b * a.tokens + j;
  int count = a.tokens;
  if (a.counts) count = min(max(a.counts[b], 0), a.tokens);
  const int end = j < count ? pair_len(c, pair) - (count - 1 - j) : 0;
  if (t < D) q[t] = load_elem<BF16>(a.q, row * a.q_stride + hq * D + t) * a.scale_log2;
  __syncthreads();
  float top = -1e30f, sum = 0.f, acc = 0.f;
  for (int base = 0; base < end; base += 256) {
    const int pos = base + t;
    const int id = pos < end ? block_id(c, pair, pos >> c.bt_log) : -1;
    if (pos < end && id < 0) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
    float s = -INFINITY;
    if (id >= 0) {
      const unsigned *w = reinterpret_cast<const unsigned *>(block_codes<D>(c, id, 0) + (pos & (bt - 1)) * D);
      s = 0.f;
      for (int i = 0; i < D / 4; ++i) {
        float x[4];
        unpack4(w[i], x);
        for (int e = 0; e < 4; ++e) s = fmaf(x[e], q[4 * i + e], s);
      }
      s *= c.scales[(int64_t)id * 2];
    }
    const float most = fmaxf(top, block_max(s, red)), f = exp2f(top - most);
    top = most;
    p[t] = exp2f(s - top);
    sum = sum * f + p[t];
    acc *= f;
    __syncthreads();
    const int dim = t % D;
    for (int i = t / D; i < 256 && base + i < end; i += PARTS) {
      const int at = base + i, vid = block_id(c, pair, at >> c.bt_log);
      if (vid < 0) continue;
      const unsigned code = block_codes<D>(c, vid, 1)[(dim << c.bt_log) + (at & (bt - 1))];
      acc = fmaf(p[i] * c.scales[(int64_t)vid * 2 + 1], __builtin_amdgcn_cvt_f32_fp8((int)code, 0), acc);
    }
    __syncthreads();
  }
  part[t] = acc;
  sum = wave_add(sum);
  if ((t & 63) == 0) red[t >> 6] = sum;
  __syncthreads();
  sum = red[0] + red[1] + red[2] + red[3];
  if (t < D) {
    for (int i = 1; i < PARTS; ++i) acc += part[i * D + t];
    store_elem<BF16>(a.out, (row * c.Hq + hq) * D + t, sum > 0.f ? acc / sum : 0.f);
  }
  if (t == 0 && a.lse) a.lse[row * c.Hq + hq] = sum > 0.f ? (top + log2f(sum)) * kLn2f : -INFINITY;
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

int blocks_for(int64_t n, int per, int most) { return (int)std::max<int64_t>(1, std::min<int64_t>(most, (n + per - 1) / per)); }

// The instance for a dtype and head size.
#define CACHE_LAUNCH(kernel, grid, s, ...)                                             \
  do {                                                                                 \
    if (bf16 && head_dim == 128)                                                       \
      hipLaunchKernelGGL((kernel<true, 128>), grid, dim3(256), 0, s, __VA_ARGS__);     \
    else if (bf16)                                                                     \
      hipLaunchKernelGGL((kernel<true, 64>), grid, dim3(256), 0, s, __VA_ARGS__);      \
    else if (head_dim == 128)                                                          \
      hipLaunchKernelGGL((kernel<false, 128>), grid, dim3(256), 0, s, __VA_ARGS__);    \
    else                                                                               \
      hipLaunchKernelGGL((kernel<false, 64>), grid, dim3(256), 0, s, __VA_ARGS__);     \
  } while (0)

}  // namespace

hipError_t launch_cache_clear(const CacheDev &c, int first_seq, int num_seqs, bool errors, hipStream_t s) {
  const int64_t n = (int64_t)c.L * num_seqs * c.Hkv * c.max_blocks;
  hipLaunchKernelGGL(k_cache_clear, dim3(blocks_for(n, 1024, 4096)), dim3(256), 0, s, c, first_seq, num_seqs, errors);
  return hipGetLastError();
}

hipError_t launch_cache_tables(const CacheTablesArgs &a, hipStream_t s) {
  const int64_t pairs = (int64_t)a.c.L * a.s.batch * a.c.Hkv;
  hipLaunchKernelGGL(k_cache_tables, dim3((unsigned)((pairs + kTabPairs - 1) / kTabPairs)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_store(const CacheStoreArgs &a, bool bf16, int head_dim, int most_rows, hipStream_t s) {
  const int64_t pairs = (int64_t)a.layers * a.s.batch * a.c.Hkv;
  const int blocks = (most_rows + (1 << a.c.bt_log) - 1) >> a.c.bt_log;
  const int per_pair = (int)std::max<int64_t>(1, std::min<int64_t>(blocks, 8192 / std::min<int64_t>(pairs, 8192)));
  const dim3 grid((unsigned)(pairs * per_pair), 2);
  CACHE_LAUNCH(k_cache_store, grid, s, a, per_pair);
  return hipGetLastError();
}

hipError_t launch_cache_load(const CacheLoadArgs &a, bool bf16, int head_dim, hipStream_t s) {
  const int64_t rows = (int64_t)a.layers * a.num_seqs * a.c.Hkv * a.count;
  const dim3 grid(blocks_for(rows * head_dim, 256, 1 << 20));
  CACHE_LAUNCH(k_cache_load, grid, s, a, rows);
  return hipGetLastError();
}

hipError_t launch_cache_append(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)(a.num_seqs * a.c.Hkv));
  CACHE_LAUNCH(k_cache_append, grid, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_attend(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)(a.num_seqs * a.tokens * a.c.Hq));
  CACHE_LAUNCH(k_cache_attend, grid, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_advance(const CacheMoveArgs &a, hipStream_t s) {
  const int64_t n = (int64_t)a.layers * a.num_seqs * a.c.Hkv;
  hipLaunchKernelGGL(k_cache_advance, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace bacon
