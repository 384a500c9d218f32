// Attention over the 8-bit cache on gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "allow_lds.h"
#include "cache_dev.h"

namespace bacon {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A wave takes tiles of 64 rows.  Both products are 16x16x32 bf16 MFMAs with
// the rows of K, then the dimensions of V, along M and 16 query rows along N:
//
//   S^T = K Q^T    lane (n = lane & 15, g = lane >> 4) holds, of query n, the
//                  logits of four rows of each of the four steps t
//   O^T = V^T P^T  lane (n, g) gives 8 rows' weights of query n to a step
//
// Row 16 g + 4 t + i of the tile is M index 4 g + i of step t, so a lane's 16
// weights belong to rows 16 g .. 16 g + 15, which are what it gives to the
// second product, without an exchange between lanes, and V's 16-byte groups
// are read in that order.  The codes become bf16 in registers, exactly, the
// block's scale applied by the conversion.
template <int D>
struct KTile {
  u32x4 w[4][D / 64];
  float scale;
};
template <int D>
struct VTile {
  u32x4 w[D / 16];
  float scale;
};

// Block ids of a tile: of the rows this lane loads K of (group (lane & 15) >> 2)
// and of those it loads V of (group lane >> 4); -1 where there is none.
struct TileIds {
  int k, v;
};

// The entries for a tile's rows, whatever the pair's length (bounded by the table).
__device__ __forceinline__ TileIds any_ids(const CacheDev &c, const int32_t *row, int base) {
  const int lane = threadIdx.x & 63, last = c.max_blocks - 1;
  return TileIds{row[min((base + 16 * ((lane & 15) >> 2)) >> c.bt_log, last)],
                 row[min((base + 16 * (lane >> 4)) >> c.bt_log, last)]};
}

__device__ __forceinline__ TileIds bound_ids(TileIds t, int base, int to) {
  const int lane = threadIdx.x & 63;
  return TileIds{base + 16 * ((lane & 15) >> 2) < to ? t.k : -1, base + 16 * (lane >> 4) < to ? t.v : -1};
}

// (An absent block's rows are masked: any address of the pool will do.)
template <int D>
__device__ __forceinline__ void load_k(const CacheDev &c, int id, int base, KTile<D> &x) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int i = (unsigned)id < (unsigned)c.num_blocks ? id : 0;
  const int r = ((base + 16 * (m >> 2)) & ((1 << c.bt_log) - 1)) + (m & 3);
  const uint8_t *p = block_codes<D>(c, i, 0) + r * D + 16 * g;
  x.scale = c.scales[(int64_t)i * 2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) x.w[t][j] = *reinterpret_cast<const u32x4 *>(p + 4 * t * D + 64 * j);
}

template <int D>
__device__ __forceinline__ void load_v(const CacheDev &c, int id, int base, VTile<D> &x) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int i = (unsigned)id < (unsigned)c.num_blocks ? id : 0;
  const uint8_t *p = block_codes<D>(c, i, 1) + ((base + 16 * g) & ((1 << c.bt_log) - 1)) * D + 16 * m;
  x.scale = c.scales[(int64_t)i * 2 + 1];
#pragma unroll
  for (int e = 0; e < D / 16; ++e) x.w[e] = *reinterpret_cast<const u32x4 *>(p + 256 * e);
}

// Eight codes as bf16 values times the scale (exact).
__device__ __forceinline__ bf16x8 dequant(unsigned lo, unsigned hi, float scale) {
  bf16x8 r;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1];
  r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}

// Eight floats as NP bf16 parts whose sum they are, to 8 bits more a part: all
// but the last are cut off (a mask, and the rest is exact), the last is rounded.
template <int NP>
__device__ __forceinline__ void split8(float (&x)[8], bf16x8 (&part)[NP]) {
#pragma unroll
  for (int p = 0; p + 1 < NP; ++p) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302);
    part[p] = __builtin_bit_cast(bf16x8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xFFFF0000u);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[NP - 1][i] = (__bf16)x[i];
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Barrier for LDS traffic alone: the global loads in flight stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ float xor16_32_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// Most waves of a workgroup: 8 fill a compute unit at 256 registers a lane;
// 32 fp32 queries of 128 dimensions need more and take 4.
constexpr int max_waves(bool bf16, int d, int nt) { return nt == 2 && !bf16 && d == 128 ? 4 : 8; }

// Maximum of no logits: below every finite one, since a sum of products in 32
// bits is scaled by log2(e) / sqrt(d) < 1/5.
constexpr float kFloor = -3.402823466e38f;

// A query's maximum over no row at all, in what waves, parts and groups hand on:
// what tells "sees no row" from logits that fell below all floats.
constexpr float kNoRow = -INFINITY;

// a - b of two values rounded before (a product and a subtraction joined into
// one rounding would not give 0 for equal ones).
__device__ __forceinline__ float minus(float a, float b) {
#pragma clang fp contract(off)
  return a - b;
}

template <int D>
constexpr int o_pitch() { return D + 4; }

// Token of query row r < 64 of a pair (r / G).
__device__ __forceinline__ int token_of(const CacheStepArgs &a, int r) {
  return (int)((unsigned)r * a.group_magic >> 16);
}

// Eight elements of a query as they lie in memory, and as floats.
template <bool BF16>
struct QRaw {
  u32x4 w[BF16 ? 1 : 2];
};

template <bool BF16>
__device__ __forceinline__ QRaw<BF16> load_raw(const void *p, int64_t i) {
  const u32x4 *q = reinterpret_cast<const u32x4 *>(static_cast<const char *>(p) + i * (BF16 ? 2 : 4));
  QRaw<BF16> r;
  r.w[0] = q[0];
  if constexpr (!BF16) r.w[1] = q[1];
  return r;
}

template <bool BF16>
__device__ __forceinline__ void raw_floats(const QRaw<BF16> &r, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned w = r.w[0][j];
    if constexpr (BF16) {
      x[2 * j] = bf16_float(w & 0xFFFFu);
      x[2 * j + 1] = __uint_as_float(w & 0xFFFF0000u);
    } else {
      x[j] = __uint_as_float(w);
      x[4 + j] = __uint_as_float(r.w[1][j]);
    }
  }
}

// Four dimensions of a query's output from their weighted sums (zeros where it
// sees no row), its normaliser and its maximum.  A query that sees rows has a
// normaliser of 1 at least, unless its logits are no numbers (one NaN or
// +infinity, or all -infinity): then all of it is NaN.
template <bool BF16, int D>
__device__ __forceinline__ void store_out(const CacheStepArgs &a, int64_t at, int dim, f32x4 acc, float l, float top) {
  const bool none = top == kNoRow;
  l = none ? 1.f : l > 0.f ? l : __builtin_nanf("");
  acc *= 1.f / l;
  if constexpr (BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.out) + at * D + dim) = __builtin_convertvector(acc, bf16x4);
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at * D + dim) = acc;
  }
  if (dim == 0 && a.lse) a.lse[at] = none ? -INFINITY : (top + __log2f(l)) * kLn2f;
}

template <bool BF16, int D, int NT>
__global__ __launch_bounds__(64 * max_waves(BF16, D, NT)) void k_cache_attend(CacheStepArgs a) {
  constexpr int QP = BF16 ? 1 : 3;     // parts of a query: bf16 is one; fp32 needs three for its 24 bits
  constexpr int PP = BF16 ? 2 : 3;     // parts of a weight: one would add 2^-8 to a bf16 output's own 2^-8, two 2^-16
  constexpr int KS = D / 32;
  extern __shared__ __align__(16) char lds[];
  bf16x8 *q_lds = reinterpret_cast<bf16x8 *>(lds);           // [NT][KS][QP][64]
  const CacheDev &c = a.c;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), waves = blockDim.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  // One workgroup a unit (pair and part): a grid of parts, heads and sequences.
  // The workgroups of a unit's further query rows follow the first's eight
  // apart: on the same die (workgroups go to the eight in turn), whose L2 then
  // still holds the codes (it took 512 pairs of 64 query rows over 1K rows from
  // 66 us to 58; they take 44 now).
  int split = blockIdx.x, h = blockIdx.y, b = blockIdx.z, row0 = 0;
  if (a.groups > 1) {
    const int eights = blockIdx.x >> 3, unit = eights / a.groups * 8 + (blockIdx.x & 7);
    if (unit >= a.num_seqs * c.Hkv * a.splits) return;
    row0 = eights % a.groups * NT * 16;
    split = unit % a.splits;
    const int pair = unit / a.splits;
    b = pair / c.Hkv;
    h = pair - b * c.Hkv;
  }
  const int G = a.G, R = a.R, bh = b * c.Hkv + h;
  // Queries: lane (n, g) holds 8 dimensions of query n for each step of 32.
  // A wave's are asked for first of all, and formed while codes are on their way.
  constexpr int QI = (NT * KS + 3) / 4;
  QRaw<BF16> q_raw[QI];
#pragma unroll
  for (int u = 0; u < QI; ++u) {
    const int i = wave + u * waves, nt = i / KS, s = i - nt * KS, r = row0 + nt * 16 + m;
    const int j = token_of(a, r), dim = 64 * (s >> 1) + 16 * g + 8 * (s & 1);
    q_raw[u] = QRaw<BF16>{};
    if (i < NT * KS && r < R)
      q_raw[u] = load_raw<BF16>(a.q, ((int64_t)b * a.tokens + j) * a.q_stride + (h * G + r - j * G) * D + dim);
  }
  const int64_t pair = pair_of(c, a.layer, a.first_seq + b, h);
  const int32_t *row = c.table + pair * c.max_blocks;
  // The first two tiles' ids are asked for before the length is known (and
  // before any codes: a wait for an id is then no wait for codes).
  const int step = 64 * waves;
  const int guess = (int)min((int64_t)split * a.chunk + 64 * wave, (int64_t)1 << 30);
  TileIds id0 = any_ids(c, row, guess), id1 = any_ids(c, row, guess + step);
  // (scalar, so that the loops below end for a whole wave at once)
  const int len = __builtin_amdgcn_readfirstlane(pair_len(c, pair));
  const int count = __builtin_amdgcn_readfirstlane(call_count(a, b));
  const bool append = a.k && count > 0;
  NewRows fresh{};
  if (append) {
    fresh = new_rows(a, pair, b, h, len, count);
    fresh.room = __builtin_amdgcn_readfirstlane((int)fresh.room);
    if (!fresh.room && split == 0 && t == 0) atomicOr(c.err, (unsigned)BACON_CACHE_NO_BLOCKS);
  }
  const bool grow = append && fresh.room;
  const int total = __builtin_amdgcn_readfirstlane(grow ? len + count : len);
  // this workgroup's rows
  const int chunk = max(a.chunk, ((total + a.splits - 1) / a.splits + 63) & ~63);
  const int from = split * chunk, to = min(total, from + chunk);
  const int first_end = total - max(count - 1, 0);           // of the first query: below it nothing is masked

  // the first tile's codes, asked for before the queries are formed
  int base = from + 64 * wave;
  KTile<D> kt;
  VTile<D> vt;
  if (base != guess) {
    id0 = any_ids(c, row, base);
    id1 = any_ids(c, row, base + step);
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt 0: else the loop waits for ids after codes
  }
  TileIds ids = bound_ids(id0, base, to);
  const bool late = grow && base + 64 > fresh.b0 << c.bt_log;
  if (base < to && !late) {
    load_k<D>(c, ids.k, base, kt);
    load_v<D>(c, ids.v, base, vt);
  }
  // (taken to be waited for here: nothing in the loop then waits for them)
  asm volatile("" : "+v"(id1.k), "+v"(id1.v));
#pragma unroll
  for (int u = 0; u < QI; ++u) {
    const int i = wave + u * waves;
    if (i >= NT * KS) continue;
    float x[8];
    raw_floats<BF16>(q_raw[u], x);
    bf16x8 part[QP];
    split8<QP>(x, part);
#pragma unroll
    for (int p = 0; p < QP; ++p) q_lds[(i * QP + p) * 64 + lane] = part[p];
  }
  int end[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row0 + nt * 16 + m, j = token_of(a, r);
    end[nt] = r < R && j < count ? max(0, total - (count - 1 - j)) : 0;
  }
  lds_barrier();
  // The new rows: the wave that owns a tile puts those of its blocks in place
  // before it reads them (no block passes the border of a tile, so no other wave
  // does).  After the barrier: the other waves go on.
  if (grow) {
    for (int i = fresh.b0; i <= fresh.b1; ++i) {
      const int at = (i << c.bt_log & ~63) - from;
      if (at >= 0 && at < to - from && (at >> 6) % waves == wave) append_block<BF16, D>(a, pair, fresh, i);
    }
    // (a wave's loads follow its stores through the unit's L1 in order: the
    // fence keeps the compiler to that and waits for nothing)
    __threadfence_block();
  }
  if (base < to && late) {
    load_k<D>(c, ids.k, base, kt);
    load_v<D>(c, ids.v, base, vt);
  }

  f32x4 o[NT][D / 16];
  float mx[NT], sum[NT];
  int seen[NT];                        // whether this lane's rows held one that the query sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    mx[nt] = kFloor;
    seen[nt] = 0;
    sum[nt] = 0.f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[nt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // A tile's K gives way to the next tile's as soon as the logits are formed,
  // its V once the outputs have it: each is in flight while the other half of
  // the work is done, in one set of registers.  No load hangs on a condition,
  // since the compiler would wait for all of them where the paths meet: past
  // the end they read block 0.
  for (; base < to; base += step) {
    const bool here = (unsigned)ids.v < (unsigned)c.num_blocks;
    const bool masked = base + 64 > first_end || !__all(here);
    f32x4 s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[nt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      bf16x8 kk[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        kk[i] = dequant(kt.w[i][k >> 1][2 * (k & 1)], kt.w[i][k >> 1][2 * (k & 1) + 1], kt.scale);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          const bf16x8 qq = q_lds[((nt * KS + k) * QP + p) * 64 + lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][i] = mfma(kk[i], qq, s[nt][i]);
        }
    }
    const TileIds next = bound_ids(id1, base + step, to);
    id1 = any_ids(c, row, base + 2 * step);
    load_k<D>(c, next.k, base + step, kt);
    bf16x8 w[NT][2][PP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (masked) {
        const int n = here ? end[nt] - (base + 16 * g) : 0;
        seen[nt] |= n > 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * i + e >= n) s[nt][i][e] = -INFINITY;
      } else {
        seen[nt] = 1;
      }
      // In units of log2, rounded before the maximum is taken from them: the
      // largest logit's weight is then 1 whatever its size (a fused product and
      // difference is off by up to 2^-24 of the logit, which past 2^31 leaves no
      // weight or an infinite one).
#pragma unroll
      for (int i = 0; i < 4; ++i) s[nt][i] *= a.scale_log2;
      float top = s[nt][0][0];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, s[nt][i][e]);
      top = fmaxf(mx[nt], xor16_32_max(top));
      if (__any(top > mx[nt])) {
        const float f = __builtin_amdgcn_exp2f(mx[nt] - top);
        mx[nt] = top;
        sum[nt] *= f;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[nt][e] *= f;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float x8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x8[e] = __builtin_amdgcn_exp2f(minus(s[nt][2 * u + (e >> 2)][e & 3], mx[nt]));
          sum[nt] += x8[e];
        }
        split8<PP>(x8, w[nt][u]);
      }
    }
    if (masked) {
      // rows that hold nothing: their codes may be any bytes
      const int n = here ? total - (base + 16 * g) : 0;
      if (!here && base + 16 * g < total) atomicOr(c.err, (unsigned)BACON_CACHE_BAD_BLOCK);
      if (n <= 0) vt.scale = 1.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int left = n - 4 * i;
        const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) vt.w[e][i] &= keep;
      }
    }
#pragma unroll
    for (int e = 0; e < D / 16; ++e)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 vv = dequant(vt.w[e][2 * u], vt.w[e][2 * u + 1], vt.scale);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int p = 0; p < PP; ++p) o[nt][e] = mfma(vv, w[nt][u][p], o[nt][e]);
      }
    ids = next;
    load_v<D>(c, ids.v, base + step, vt);
  }

  // Join the waves through LDS, all query rows at once.
  float *ml = reinterpret_cast<float *>(lds);                // [waves][NT * 16][2]
  float *oo = ml + waves * NT * 32;                          // [waves][NT * 16][o_pitch]
  constexpr int P = o_pitch<D>();
  lds_barrier();                                             // the queries are done with
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float l = sum[nt] + __shfl_xor(sum[nt], 16);
    l += __shfl_xor(l, 32);
    const bool any = (__ballot(seen[nt]) >> m & 0x0001000100010001ull) != 0;
    const int n = nt * 16 + m, at = wave * NT * 16 + n;
    if (row0 + n >= R) continue;
    if (g == 0) *reinterpret_cast<float2 *>(ml + at * 2) = make_float2(any ? mx[nt] : kNoRow, l);
#pragma unroll
    for (int e = 0; e < D / 16; ++e) *reinterpret_cast<f32x4 *>(oo + at * P + 16 * e + 4 * g) = o[nt][e];
  }
  lds_barrier();
  // every wave has read the old length
  if (grow && a.splits == 1 && t == 0) c.lens[pair] = total;
  const auto join = [&](auto count_waves) {
    constexpr int WAVES = decltype(count_waves)::value;
    for (int i = t; i < min(NT * 16, R - row0) * (D / 4); i += 64 * WAVES) {
      const int n = i / (D / 4), dim = i % (D / 4) * 4, r = row0 + n;
      float2 part[WAVES];
      f32x4 x[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        part[w] = *reinterpret_cast<const float2 *>(ml + (w * NT * 16 + n) * 2);
        x[w] = *reinterpret_cast<const f32x4 *>(oo + (w * NT * 16 + n) * P + dim);
      }
      float top = kNoRow, l = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part[w].x);
      const float most = fmaxf(top, kFloor);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(part[w].x - most);
        l += f * part[w].y;
        acc += f * x[w];
      }
      const int j = token_of(a, r);
      if (j >= count) {                                      // padding sees no row, whatever its query is
        top = kNoRow;
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      if (a.splits > 1) {
        const int64_t at = ((int64_t)bh * a.splits + split) * R + r;
        if (dim == 0) a.part_ml[at] = make_float2(top, l);
        *reinterpret_cast<f32x4 *>(a.part_o + at * D + dim) = acc;   // zeros where no row is seen
      } else {
        store_out<BF16, D>(a, ((int64_t)b * a.tokens + j) * c.Hq + h * G + (r - j * G), dim, acc, l, top);
      }
    }
  };
  if (waves == 4)
    join(std::integral_constant<int, 4>{});
  else
    join(std::integral_constant<int, 8>{});
}

// Joins the parts of one query row: D / 4 threads a part, each group of them
// every SP-th part with a running maximum, then the groups through LDS.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_cache_join(CacheStepArgs a) {
  constexpr int TR = D / 4, SP = 256 / TR;
  __shared__ f32x4 acc_lds[SP][TR];
  __shared__ float2 ml_lds[SP];
  const CacheDev &c = a.c;
  const int t = threadIdx.x, G = a.G, R = a.R, dim = t % TR, group = t / TR;
  const int r = blockIdx.x, h = blockIdx.y, b = blockIdx.z, bh = b * c.Hkv + h, j = token_of(a, r);
  const float2 *ml = a.part_ml + (int64_t)bh * a.splits * R + r;
  const f32x4 *o = reinterpret_cast<const f32x4 *>(a.part_o) + ((int64_t)bh * a.splits * R + r) * TR + dim;
  float top = kNoRow, most = kFloor, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i = group; i < a.splits; i += 4 * SP) {
    float2 x[4];
    f32x4 y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t at = (int64_t)min(i + u * SP, a.splits - 1) * R;
      x[u] = ml[at];
      y[u] = o[at * TR];
      if (i + u * SP >= a.splits) x[u] = make_float2(kNoRow, 0.f);   // (the last part's sums, times 0)
    }
    top = fmaxf(fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x)), top);
    const float m = fmaxf(top, kFloor), f = __builtin_amdgcn_exp2f(most - m);
    l *= f;
    acc *= f;
    most = m;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float g = __builtin_amdgcn_exp2f(x[u].x - m);
      l += g * x[u].y;
      acc += g * y[u];
    }
  }
  acc_lds[group][dim] = acc;
  if (dim == 0) ml_lds[group] = make_float2(top, l);
  // the new length, once every part was formed with the old one
  if (a.k && r == 0 && t == 255) {
    const int64_t pair = pair_of(c, a.layer, a.first_seq + b, h);
    const NewRows n = new_rows(a, pair, b, h, pair_len(c, pair), call_count(a, b));
    if (n.count > 0 && n.room) c.lens[pair] = n.len + n.count;
  }
  lds_barrier();
  if (t >= TR) return;
  float2 x[SP];
  f32x4 y[SP];
#pragma unroll
  for (int i = 0; i < SP; ++i) {
    x[i] = ml_lds[i];
    y[i] = acc_lds[i][dim];
  }
  top = x[0].x;
#pragma unroll
  for (int i = 1; i < SP; ++i) top = fmaxf(top, x[i].x);
  most = fmaxf(top, kFloor);
  l = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < SP; ++i) {
    const float g = __builtin_amdgcn_exp2f(x[i].x - most);
    l += g * x[i].y;
    acc += g * y[i];
  }
  store_out<BF16, D>(a, ((int64_t)b * a.tokens + j) * c.Hq + h * G + (r - j * G), t * 4, acc, l, top);
}

template <bool BF16, int D, int NT>
constexpr int attend_lds(int waves) {
  const int q = NT * (D / 32) * (BF16 ? 1 : 3) * 1024, o = waves * NT * (128 + 64 * o_pitch<D>());
  return q > o ? q : o;
}

template <bool BF16, int D, int NT>
hipError_t attend(const CacheStepArgs &a, hipStream_t s) {
  const int units = a.num_seqs * a.c.Hkv * a.splits;
  // Four waves, also where some have no tile (they share the queries and the
  // join: one sequence over 1K rows in parts of 64 takes 7.3 us with four and
  // with one).  Eight for a step of 17 to 32 query rows over parts of more than
  // 256, whose appending wave is late, as long as every workgroup has a compute
  // unit of its own: 64 sequences of four drafted tokens, 256 pairs, take 18.5 us
  // with eight and 19.2 with four; but 512 pairs of 700 rows 33.5 and 25.8 (a
  // unit holds two workgroups of four waves), one of 400 rows 13.6 and 13.3.  Attends
  // gain nothing (four sequences over 8K rows, 28 query rows, 15.7 and 14.6, eight
  // over 16K 47.9 and 48.9; one query row, 64 over 300 to 993 rows, 22.8 and 17.2).
  const bool late = a.k && NT == 2 && a.chunk > 256 && units <= 256;
  const int waves = late && max_waves(BF16, D, NT) == 8 ? 8 : 4;
  if (hipError_t e = allow_lds<k_cache_attend<BF16, D, NT>>(attend_lds<BF16, D, NT>(waves))) return e;
  const dim3 grid = a.groups == 1 ? dim3(a.splits, a.c.Hkv, a.num_seqs) : dim3((units + 7) / 8 * 8 * a.groups);
  hipLaunchKernelGGL((k_cache_attend<BF16, D, NT>), grid, dim3(64 * waves), (attend_lds<BF16, D, NT>(waves)), s,
                     a);
  if (a.splits > 1) hipLaunchKernelGGL((k_cache_join<BF16, D>), dim3(a.R, a.c.Hkv, a.num_seqs), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

CachePlan cache_plan(int pairs, int q_rows, int head_dim, int max_tokens) {
  CachePlan p{};
  // About 256 workgroups, one a compute unit: one sequence over 32K rows (8
  // pairs) takes 17 us divided into 256, 19 into 128 and 18 into 512.  A pair of
  // up to 768 rows stays whole (over 512 rows 6.7 us, in parts 7.2; over 768
  // 7.7 and 7.3, but the second launch costs the host 3 more); longer ones may
  // go down to a tile a part (over 1K rows 7.3 us, in parts of 256 8.1, whole
  // 8.9), with more than 16 query rows, whose workgroups are more already, to
  // 256 rows (three over 2K rows, 56 query rows: 18.0 us, in parts of 128 21.8).
  const int64_t want = (256 + pairs - 1) / pairs;
  const int64_t by_rows = max_tokens <= 768 ? 1 : max_tokens / (q_rows > 16 ? 256 : 64);
  p.splits = (int)std::min(want, by_rows);
  p.chunk = (int)((((int64_t)max_tokens + p.splits - 1) / p.splits + 63) / 64 * 64);
  if (p.splits > 1) {
    const size_t parts = (size_t)pairs * p.splits * q_rows;
    p.ml_bytes = (parts * sizeof(float2) + 255) / 256 * 256;
    p.bytes = p.ml_bytes + parts * head_dim * sizeof(float);
  }
  return p;
}

bool cache_appends(int q_rows) { return q_rows <= 32; }

hipError_t launch_cache_attend(CacheStepArgs a, bool bf16, int head_dim, hipStream_t s) {
  const int G = a.c.Hq / a.c.Hkv, R = G * a.tokens;
  a.G = G;
  a.R = R;
  a.group_magic = (65536 + G - 1) / G;
  // 16 query rows a workgroup or 32: 32 share the codes' conversion, 16 are
  // sooner done with a tile.  Attends in bf16, us with 16 and with 32: three
  // sequences up to 70K rows (28/4 heads, five tokens) 55.8 and 49.6, four over 4K
  // (64/8, eight tokens) 25.3 and 20.4, eight over 16K (32 query rows) 56.1 and
  // 48.9; but 64 over 300 to 993 rows (28 query rows) 15.4 and 16.1, one over 64 rows
  // 5.5 and 7.0.  fp32, whose parts fill the registers: five tokens of four
  // sequences 13.1 and 14.8.  A step of 17 to 32 query rows keeps them in the one
  // workgroup that appends: two would not see each other's rows.
  const bool shared = bf16 && a.chunk > 256 && (R > 32 || a.chunk > 1024);
  const bool one = R <= 16 || !(a.k || shared);
  a.groups = (R + (one ? 15 : 31)) / (one ? 16 : 32);
#define ATTEND(nt)                                                                                \
  return bf16 ? (head_dim == 128 ? attend<true, 128, nt>(a, s) : attend<true, 64, nt>(a, s))      \
              : (head_dim == 128 ? attend<false, 128, nt>(a, s) : attend<false, 64, nt>(a, s))
  if (one) ATTEND(1);
  ATTEND(2);
#undef ATTEND
}

}  // namespace bacon
