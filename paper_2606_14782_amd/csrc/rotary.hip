// Rotary positions of queries and keys on gfx950; include/bacon.h states the
// formulas.
//
// Bytes bound it: each value is read once and written once.  A wave takes one
// token: its lanes form the angle of one pair each, in turns and in 64 bits
// (p f is exact to 2^-53 of itself, so a position of 2^20 keeps 2^-33 of a turn),
// and leave cos and sin in LDS for every head of the token.  A lane then holds 16
// elements of a head in two runs of 8, which its neighbours' go on.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "rotary.h"

namespace bacon {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Which elements a lane holds: four pairs of neighbours in each run, or of halves a
// run and its partners' run, or, where r / 2 is no multiple of 8, any, exchanged
// through LDS.
enum RotaryKind { kPairs, kHalves, kHalvesAny };

template <bool BF16>
__device__ __forceinline__ void load8(const void *p, int64_t i, float *x) {
  if constexpr (BF16) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  } else {
    const f32x4 *q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + i);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void store8(void *p, int64_t i, const float *x) {
  if constexpr (BF16) {
    bf16x8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (__bf16)x[j];
    // (past the caches: 8K tokens of 40 heads 32 us -> 30, 32K 123 -> 116; floats,
    // whose 16-byte stores leave gaps that the next one fills, 12 us -> 17)
    __builtin_nontemporal_store(w, reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(p) + i));
  } else {
    f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(p) + i);
    q[0] = f32x4{x[0], x[1], x[2], x[3]};
    q[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// cos and sin of t turns, |t| <= 1/2 after the whole turns are taken off: the
// nearest quarter turn is taken off too (exactly, in 64 bits), which leaves
// |x| <= pi/4, where the Taylor series to x^9 and x^10 end below 2e-9.
__device__ __forceinline__ float2 turn(double t, float magnitude) {
  const double quarters = rint(4.0 * t);
  const float x = (float)((t - 0.25 * quarters) * 6.283185307179586), z = x * x;
  const int n = (int)(long long)quarters & 3;
  const float s = x * (1.f + z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880)))));
  const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
  float cs = n & 1 ? s : c, sn = n & 1 ? c : s;
  cs = n == 1 || n == 2 ? -cs : cs;
  sn = n & 2 ? -sn : sn;
  return make_float2(cs * magnitude, sn * magnitude);
}

// LDS traffic of one wave: in order, and the compiler keeps it so.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <bool BF16, int D, int KIND>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a) {
  constexpr int LH = D / 16, HW = 64 / LH;                   // lanes of a head, heads of a wave
  constexpr int PITCH = D + 4;
  __shared__ __align__(16) float2 table[4][kRotaryMaxPairs];
  __shared__ float staged[KIND == kHalvesAny ? 4 : 1][KIND == kHalvesAny ? HW * PITCH : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LH, pairs = a.pairs;
  const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
  const int64_t token = unit / a.parts;
  const int part = (int)(unit - token * a.parts);
  if (token >= a.tokens) return;
  const int heads = a.q.heads + a.k.heads;
  // this lane's two runs of 8 dimensions
  const bool turned = KIND != kHalves || j < pairs / 8;
  int d0 = 8 * j, d1 = D / 2 + 8 * j;
  if (KIND == kHalves && turned) {
    d1 = pairs + 8 * j;
  } else if (KIND == kHalves) {
    d0 = 2 * pairs + 8 * (j - pairs / 8);
    d1 = d0 + D / 2 - pairs;
  }
  {                                                          // one pair a lane
    const int i = min(lane, pairs - 1);
    const int row = i < a.row1 ? 0 : i < a.row2 ? 1 : 2;
    const double t = (double)a.pos[row * a.tokens + token] * a.turns[i];
    table[wave][lane] = turn(t - rint(t), a.magnitude);
  }
  wave_sync();
  float c[8], s[8];
  if (KIND != kHalvesAny && turned) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 v = table[wave][KIND == kHalves ? 8 * j + e : (e < 4 ? 0 : D / 4 - 4) + 4 * j + e];
      c[e] = v.x;
      s[e] = v.y;
    }
  }
  const int last = min(heads, (part + 1) * a.per_wave * HW);
  for (int h = part * a.per_wave * HW + lane / LH; h - lane / LH < last; h += HW) {
    const bool here = h < last, is_q = h < a.q.heads;
    const RotarySide &side = is_q ? a.q : a.k;
    const int64_t at = (int64_t)(is_q ? h : h - a.q.heads) * D;
    float x[16];
    if (here) {
      load8<BF16>(side.x, token * side.x_stride + at + d0, x);
      load8<BF16>(side.x, token * side.x_stride + at + d1, x + 8);
      if (side.norm) {
        float w[16], sum = 0.f;
        load8<BF16>(side.norm, d0, w);
        load8<BF16>(side.norm, d1, w + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += x[e] * x[e];
#pragma unroll
        for (int m = 1; m < LH; m <<= 1) sum += __shfl_xor(sum, m);
        float f = 1.f / sqrtf(sum * (1.f / D) + a.eps);
        // Squares past 2^128 (the largest value is then 2^60 or more), or a sum below 2^-80,
        // of which squares under 2^-126 may be a part: the same of values times a power of
        // two, which brings the largest to 2^-12 .. 2^56, or below 2^60.  (The lanes of a
        // head hold the same sum.)
        if (__builtin_expect(!(sum < INFINITY) || sum + a.eps < 0x1p-80f, 0)) {
          const bool large = !(sum < INFINITY);
          const float by = large ? kNormLarge : kNormSmall;
          sum = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            x[e] *= by;
            sum += x[e] * x[e];
          }
#pragma unroll
          for (int m = 1; m < LH; m <<= 1) sum += __shfl_xor(sum, m);
          f = 1.f / sqrtf(sum * (1.f / D) + (large ? a.eps_large : a.eps_small));
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * f * w[e];
      }
    }
    float y[16];
    if constexpr (KIND == kHalvesAny) {
      float *row = staged[wave] + lane / LH * PITCH;
      wave_sync();                                           // the head before has been read
#pragma unroll
      for (int e = 0; e < 16; ++e) row[(e < 8 ? d0 : d1 - 8) + e] = here ? x[e] : 0.f;
      wave_sync();
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int d = (e < 8 ? d0 : d1 - 8) + e, i = d < pairs ? d : d - pairs;
        if (d < 2 * pairs) {
          const float2 v = table[wave][i];
          y[e] = d < pairs ? x[e] * v.x - row[d + pairs] * v.y : x[e] * v.x + row[i] * v.y;
        } else {
          y[e] = x[e];
        }
      }
    } else if constexpr (KIND == kPairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool on = (e < 4 ? 0 : D / 4 - 4) + 4 * j + e < pairs;
        const float p = x[2 * e], q = x[2 * e + 1];
        y[2 * e] = on ? p * c[e] - q * s[e] : p;
        y[2 * e + 1] = on ? q * c[e] + p * s[e] : q;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = turned ? x[e] * c[e] - x[8 + e] * s[e] : x[e];
        y[8 + e] = turned ? x[8 + e] * c[e] + x[e] * s[e] : x[8 + e];
      }
    }
    if (here) {
      store8<BF16>(side.y, token * side.y_stride + at + d0, y);
      store8<BF16>(side.y, token * side.y_stride + at + d1, y + 8);
    }
  }
}

template <bool BF16, int D>
void launch(const RotateArgs &a, bool half, dim3 grid, hipStream_t s) {
  if (!half)
    hipLaunchKernelGGL((k_rotate<BF16, D, kPairs>), grid, dim3(256), 0, s, a);
  else if (a.pairs % 8 == 0)
    hipLaunchKernelGGL((k_rotate<BF16, D, kHalves>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_rotate<BF16, D, kHalvesAny>), grid, dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_rotate(RotateArgs a, bool bf16, int head_dim, bool half, hipStream_t s) {
  // A token's heads over several waves up to 65536 of them, so that more loads are
  // on their way: 32K tokens of 40 heads in two waves each 116 us, in one 126; 300 in
  // five 4.0, in one 5.7.
  const int per = 64 / (head_dim / 16), groups = (a.q.heads + a.k.heads + per - 1) / per;
  a.parts = (int)std::min<int64_t>(groups, std::max<int64_t>(1, 65536 / a.tokens));
  a.per_wave = (groups + a.parts - 1) / a.parts;
  a.parts = (groups + a.per_wave - 1) / a.per_wave;
  const dim3 grid((unsigned)((a.tokens * a.parts + 3) / 4));
  if (bf16)
    head_dim == 128 ? launch<true, 128>(a, half, grid, s) : launch<true, 64>(a, half, grid, s);
  else
    head_dim == 128 ? launch<false, 128>(a, half, grid, s) : launch<false, 64>(a, half, grid, s);
  return hipGetLastError();
}

}  // namespace bacon
