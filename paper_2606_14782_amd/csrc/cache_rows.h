// Rows as the cache's stores and loads hold them: raw 8-element runs, and
// transposes of bytes and of 16-lane rows.
#pragma once

#include "cache_dev.h"

namespace bacon {
namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <bool BF16>
struct Raw8;                           // eight elements of a row as they lie in memory
template <>
struct Raw8<true> {
  u32x4 w;
};
template <>
struct Raw8<false> {
  u32x4 w, x;
};

// STREAM: past the caches, for rows read once in order.
template <bool STREAM>
__device__ __forceinline__ u32x4 load16(const u32x4 *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}

template <bool BF16, bool STREAM>
__device__ __forceinline__ Raw8<BF16> raw8(const void *p, int64_t i) {
  Raw8<BF16> r;
  if constexpr (BF16) {
    r.w = load16<STREAM>(reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + i));
  } else {
    const u32x4 *q = reinterpret_cast<const u32x4 *>(static_cast<const float *>(p) + i);
    r.w = load16<STREAM>(q);
    r.x = load16<STREAM>(q + 1);
  }
  return r;
}

// The largest magnitude of four rows (bf16 magnitudes compare as integers).
template <bool BF16>
__device__ __forceinline__ float raw_top(const Raw8<BF16> (&r)[4]) {
  if constexpr (BF16) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r[i].w[j] & 0x7FFF7FFFu));
    return bf16_float(m[0] > m[1] ? m[0] : m[1]);
  } else {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) m = max(max(m, r[i].w[j] & 0x7FFFFFFFu), r[i].x[j] & 0x7FFFFFFFu);
    return __uint_as_float(m);
  }
}

// Bytes j of a, b, c, d as word j.
__device__ __forceinline__ void transpose4(unsigned a, unsigned b, unsigned c, unsigned d, unsigned (&w)[4]) {
  const unsigned ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602);
  const unsigned cd0 = __builtin_amdgcn_perm(d, c, 0x05010400), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602);
  w[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100);
  w[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302);
  w[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100);
  w[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302);
}

// Four registers of four 16-lane rows, transposed: register i of row q becomes
// register q of row i.
__device__ __forceinline__ void transpose_rows(unsigned &a, unsigned &b, unsigned &c, unsigned &d) {
  const auto ac = __builtin_amdgcn_permlane32_swap(a, c, false, false);
  const auto bd = __builtin_amdgcn_permlane32_swap(b, d, false, false);
  const auto ab = __builtin_amdgcn_permlane16_swap(ac[0], bd[0], false, false);
  const auto cd = __builtin_amdgcn_permlane16_swap(ac[1], bd[1], false, false);
  a = ab[0];
  b = ab[1];
  c = cd[0];
  d = cd[1];
}

}  // namespace
}  // namespace bacon
