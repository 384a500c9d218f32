// Device helpers shared by the kernels of the 8-bit cache.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/bacon.h"
#include "cache.h"

namespace bacon {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLn2f = 0.69314718055994531f;

__device__ __forceinline__ float bf16_float(unsigned bits) { return __uint_as_float(bits << 16); }

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

// Byte of V's code (row r of its block, dimension dim): groups of 16 rows,
// each transposed, so that one lane's 16-byte load holds 16 rows of a dimension
// and the lanes of a wave read whole lines whatever the block's size.
template <int D>
__device__ __forceinline__ int v_at(int r, int dim) {
  return ((r >> 4) * D + dim) * 16 + (r & 15);
}

__device__ __forceinline__ float wave_max(float v) {
  for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
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

// New tokens of a pair in a call: sequence b of the call, `count` rows from
// row `len` of the pair on, in blocks b0 .. b1 of its table.
struct NewRows {
  int b, h, len, count, b0, b1;
  bool room;               // every block of them is one of the pool's
};

__device__ __forceinline__ int call_count(const CacheStepArgs &a, int b) {
  return a.counts ? min(max(a.counts[b], 0), a.tokens) : a.tokens;
}

__device__ __forceinline__ NewRows new_rows(const CacheStepArgs &a, int64_t pair, int b, int h, int len, int count) {
  NewRows n{b, h, len, count, len >> a.c.bt_log, (len + count - 1) >> a.c.bt_log, true};
  for (int i = n.b0; i <= n.b1; ++i) n.room &= block_id(a.c, pair, i) >= 0;
  return n;
}

// One wave puts the new rows of the pair's block i in place: 8 elements a
// lane, D / 8 lanes a row.  The scale is the larger of the one that the block's
// old rows have and the one that the new rows need; old codes are rounded again
// where it grew (in whole words, before the new codes are written).  A chain
// of reads bounds it (id, scale and new rows, store): a step over 288
// rows takes 8.2 us with it, 6.9 without.
template <bool BF16, int D>
__device__ void append_block(const CacheStepArgs &a, int64_t pair, const NewRows &n, int i) {
  constexpr int TR = D / 8, RP = 64 / TR;
  const CacheDev &c = a.c;
  const int lane = threadIdx.x & 63, bt = 1 << c.bt_log, base = i << c.bt_log;
  const int id = block_id(c, pair, i);
  const int from = max(n.len, base), old = from - base, m = min(n.len + n.count, base + bt) - from;
  const int64_t row0 = (int64_t)n.b * a.tokens + (from - n.len);
  float was[2], x[2][8], top[2] = {0.f, 0.f};
  const int col = n.h * D + lane % TR * 8;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) was[kv] = c.scales[(int64_t)id * 2 + kv];
  for (int r = lane / TR; r < m; r += RP)
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      load8<BF16>(kv ? a.v : a.k, (row0 + r) * (kv ? a.v_stride : a.k_stride) + col, x[kv]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top[kv] = fmaxf(top[kv], fabsf(x[kv][e]));
    }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint8_t *dst = block_codes<D>(c, id, kv);
    float scale = block_scale(wave_max(top[kv]));
    if (old && scale < was[kv]) scale = was[kv];
    if (old && scale > was[kv]) {
      const float f = was[kv] / scale;                       // a power of two: the product is exact
      for (int e = lane; e < bt * D / 16; e += 64) {
        u32x4 *p = reinterpret_cast<u32x4 *>(dst) + e;
        u32x4 w = *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float y[4];
          unpack4(w[j], y);
          w[j] = pack4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
        }
        *p = w;
      }
      __threadfence_block();
    }
    if (lane == 0) c.scales[(int64_t)id * 2 + kv] = scale;
    const float inv = 1.f / scale;
    for (int r = lane / TR; r < m; r += RP) {
      if (m > RP) load8<BF16>(kv ? a.v : a.k, (row0 + r) * (kv ? a.v_stride : a.k_stride) + col, x[kv]);
      u32x2 w;
      w[0] = pack4(x[kv][0] * inv, x[kv][1] * inv, x[kv][2] * inv, x[kv][3] * inv);
      w[1] = pack4(x[kv][4] * inv, x[kv][5] * inv, x[kv][6] * inv, x[kv][7] * inv);
      if (kv == 0) {
        *reinterpret_cast<u32x2 *>(dst + (old + r) * D + lane % TR * 8) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[v_at<D>(old + r, lane % TR * 8 + e)] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
      }
    }
  }
}

}  // namespace
}  // namespace bacon
