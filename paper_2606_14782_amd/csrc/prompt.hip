// The prompt's attention on gfx950; include/bacon.h states the formulas.
//
// A workgroup takes 128 query rows of one KV head: row r of a sequence is query
// r / G of head h G + r % G, so the G heads that share K and V share its tiles.
// Each of its four waves holds 32 of them and sees every tile of keys, which
// come through LDS, read directly from memory into one of two buffers while the
// other is computed on; or two sets of four waves take the tiles in turn and are
// joined at the end.  Both products have the query rows along N:
//
//   S^T = K Q^T    lane (n = lane & 31, g = lane >> 5) holds, of row n, the logits
//                  of keys 8 t + 4 g + i (t < 4, i < 4) of every 32
//   O^T = V^T P^T  takes them from there: a lane's own weights are its share of
//                  the keys, so nothing passes between lanes but the row's
//                  maximum, once a tile, and its sum, once at the end
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "prompt.h"

namespace bacon {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

#define LDS __attribute__((address_space(3)))

constexpr int kWaves = 4;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
// The maximum before any logit: below every finite one times log2(e) / sqrt(d).
constexpr float kFloor = -3.402823466e38f;
// A row's maximum over no key at all, in what parts hand on.
constexpr float kNoKey = -INFINITY;
// How far (in powers of two) weights may grow past 1 before the maximum they are
// taken from moves: sums in 32 bits are as exact, and most tiles then move none.
constexpr float kSlack = 8.f;

// A unit of work: 128 query rows of a KV head of a sequence, over keys from .. to.
struct Unit {
  PromptSeq s;
  int h, tile, split, row0, rows;      // row0: the first query row, rows: the sequence's
  int from, to;
};

__device__ __forceinline__ int division(int i, unsigned magic) {     // i / G for small i
  return magic ? (int)__umulhi((unsigned)i, magic) : i;
}

// The last sequence whose first unit (or joined tile) is not past i: the lanes look
// at one each, in one round trip to the arguments (16 prompts of 100 tokens 17.1 us
// -> 15.9).
template <int PromptSeq::*FIRST>
__device__ __forceinline__ int seq_of(const PromptArgs &a, int i) {
  if (a.seqs == 1) return 0;
  const int lane = threadIdx.x & 63;
  const bool at = lane < a.seqs && i >= a.s[lane].*FIRST;
  return __popcll(__ballot(at)) - 1;
}

// The keys that query i of a sequence sees.
__device__ __forceinline__ int keys_seen(const PromptSeq &s, int i) {
  return min(max(s.keys - s.queries + i + 1, 0), s.keys);
}

// The longest rows come first, the heads next to each other (and so on dies of
// their own, whose L2 then serves one head's keys to all its workgroups).
__device__ __forceinline__ Unit unit_of(const PromptArgs &a, int i) {
  Unit u;
  u.s = a.s[seq_of<&PromptSeq::unit0>(a, i)];
  const int local = i - u.s.unit0, rest = local / a.Hkv;
  u.h = local - rest * a.Hkv;
  const int from_last = rest / u.s.splits;
  u.split = rest - from_last * u.s.splits;
  u.tile = u.s.tiles - 1 - from_last;
  u.row0 = u.tile * kPromptRows;
  u.rows = u.s.queries * a.G;
  const int most = keys_seen(u.s, (min(u.row0 + kPromptRows, u.rows) - 1) / a.G);
  const int chunk = ((u.s.keys + u.s.splits - 1) / u.s.splits + 63) & ~63;
  u.from = u.split * chunk;
  u.to = min(most, u.from + chunk);
  return u;
}

// (NaN where one of them is: such a row gives NaN whatever its maximum.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The value of the lane 32 away.
__device__ __forceinline__ float other_half(float x) {
  const unsigned u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// (A product and a difference joined into one rounding would leave an
// unbounded rest of a huge logit.)
__device__ __forceinline__ float minus(float a, float b) {
#pragma clang fp contract(off)
  return a - b;
}

// One query row of a lane.
struct Row {
  int query, head, end;      // end: keys seen (0 past the rows)
  bool valid;
};

__device__ __forceinline__ Row row_of(const PromptArgs &a, const Unit &u, int r) {
  const int first = u.row0 / a.G, rem = u.row0 - first * a.G;
  const int q = division(rem + r, a.group_magic);
  Row x;
  x.valid = u.row0 + r < u.rows;
  x.query = first + q;
  x.head = u.h * a.G + rem + r - q * a.G;
  x.end = x.valid ? keys_seen(u.s, x.query) : 0;
  return x;
}

// What a row's weights are taken from: 2^(logit log2(e) - at), `at` the maximum so
// far in units of log2, rounded once.  A weight is then one product, subtracted in
// the same rounding, since an error of `at` is every weight's alike; where `at` is
// so large that the product's rest would count (`far`), the product is rounded first.
struct Weighed {
  float at = kFloor, sum = 0.f;
  bool far = false;          // one of the wave's rows is
};

__device__ __forceinline__ bool is_far(float at) { return __builtin_fabsf(at) > 0x1p20f && at != kFloor; }

// What a lane hands on of its row: four runs of four dimensions of every 32.
template <bool BF16, int D>
__device__ __forceinline__ void finish(const PromptArgs &a, const Unit &u, const Row &row, int r, const f32x16 (&o)[D / 32],
                                       const Weighed &w) {
  const int g = (threadIdx.x & 63) >> 5;
  const float sum = w.sum + other_half(w.sum);
  if (!row.valid) return;
  const bool none = min(row.end, u.to) <= u.from;
  if (u.s.splits > 1) {
    const int64_t at = (int64_t)blockIdx.x * kPromptRows + r;
    if (g == 0) a.part_ml[at] = make_float2(none ? kNoKey : w.at, none ? 0.f : sum);
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4 x = {o[e][4 * t], o[e][4 * t + 1], o[e][4 * t + 2], o[e][4 * t + 3]};
        if (none) x = f32x4{0.f, 0.f, 0.f, 0.f};
        *reinterpret_cast<f32x4 *>(a.part_o + at * D + 32 * e + 8 * t + 4 * g) = x;
      }
    return;
  }
  const float l = none ? 1.f : sum > 0.f ? sum : __builtin_nanf(""), inv = 1.f / l;
  const int64_t token = u.s.q0 + row.query;
  const int64_t at = (token * a.Hq + row.head) * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 x = {o[e][4 * t], o[e][4 * t + 1], o[e][4 * t + 2], o[e][4 * t + 3]};
      x = none ? f32x4{0.f, 0.f, 0.f, 0.f} : x * inv;
      const int64_t i = at + 32 * e + 8 * t + 4 * g;
      if constexpr (BF16)
        *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.out) + i) = __builtin_convertvector(x, bf16x4);
      else
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + i) = x;
    }
  if (g == 0) {
    const float lse = none ? -INFINITY : (w.at + __log2f(l)) * kLn2;
    if (a.lse) a.lse[token * a.Hq + row.head] = lse;
    const int at_window = u.s.window0 + row.query;
    if (a.window && at_window >= 0) a.window[((int64_t)u.s.index * a.Hq + row.head) * a.W + at_window] = lse;
  }
}

// A tile's logits become weights.  A row's maximum moves where they pass it by more
// than kSlack, each row's by itself: its results depend on no other.
template <int N, int E>
__device__ __forceinline__ void weigh(f32x16 (&s)[N], f32x16 (&o)[E], Weighed &w, float scale_log2) {
  float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = i ? 0 : 3; e + 1 < 16; e += 2) top = max3(top, s[i][e], s[i][e + 1]);
  top = __builtin_elementwise_maximum(top, s[0][15]);
  top = __builtin_elementwise_maximum(top, other_half(top)) * scale_log2;
  const bool moves = top > w.at + kSlack;
  if (__any(moves)) {
    const float next = moves ? top : w.at, f = __builtin_amdgcn_exp2f(minus(w.at, next));
    w.at = next;
    w.far = __any(is_far(next));
    w.sum *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= f;
  }
  if (__builtin_expect(w.far, 0)) {
    const bool far = is_far(w.at);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = far ? minus(s[i][e] * scale_log2, w.at) : __builtin_fmaf(s[i][e], scale_log2, -w.at);
        s[i][e] = __builtin_amdgcn_exp2f(x);
      }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], scale_log2, -w.at));
  }
  float part[4] = {0.f, 0.f, 0.f, 0.f};                      // (chains of their own)
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) part[e & 3] += s[i][e];
  w.sum += (part[0] + part[1]) + (part[2] + part[3]);
}

// Keys base + 32 i + 8 (e / 4) + 4 g + e % 4 from `end` on are not seen.
template <int N>
__device__ __forceinline__ void mask(f32x16 (&s)[N], int left) {
  left -= 4 * ((threadIdx.x & 63) >> 5);
  asm volatile("" : "+v"(left));                             // (else 32 registers hold the keys' numbers)
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (32 * i + 8 * (e >> 2) + (e & 3) >= left) s[i][e] = -INFINITY;
}

// Rows of a tile as 16-byte pieces in LDS, piece c of row r at place c ^ f(r):
// a read of the same piece of 16 or 32 rows then meets every bank once.
template <int PIECES>
__device__ __forceinline__ int k_place(int row) { return PIECES == 16 ? row & 15 : row >> 1 & 7; }
template <int PIECES>
__device__ __forceinline__ int v_place(int row) {
  return PIECES == 16 ? (row & 3) << 2 : (row >> 1 & 1) << 2;
}

// What this wave asked for is there, and every other wave's: its reads of the
// other buffer are done too.
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0070);                        // vmcnt 0, lgkmcnt 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The same for LDS traffic alone: loads into registers stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// This wave's share of a tile's ROWS rows of K or V, in 16-byte pieces: where
// each piece lies from the tile's first row on.
template <int ROWS, int PIECES>
struct Share {
  static constexpr int kEach = ROWS * PIECES / 64 / kWaves;
  unsigned at[kEach];

  template <class Place>
  __device__ __forceinline__ void find(unsigned stride_bytes, int rows, int wave, Place place) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = ((wave * kEach + i) * 64 + lane) / PIECES, c = (lane & (PIECES - 1)) ^ place(row);
      at[i] = (unsigned)min(row, rows - 1) * stride_bytes + c * 16;   // (rows past the last stand for it: they are masked)
    }
  }

  // Asks for it, directly into LDS (a wave's 64 pieces one after the other).  The
  // compiler does not see these: it would wait for them before it reads the other
  // buffer.  tile_barrier waits.  (m0 is the compiler's to set where an instruction of its
  // own reads it: it has to know that this does.  It warns of any such register.)
  __device__ __forceinline__ void ask(const char *tile, unsigned to, int wave) const {
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :: "s"(to + (wave * kEach + i) * 1024), "v"(at[i]), "s"(tile) : "m0", "memory");
#pragma clang diagnostic pop
  }
};

// V of a tile, 16 keys of step j for the dimensions 32 e .. of a lane.
template <int ROW>
__device__ __forceinline__ bf16x8 v_piece(const char *vt, int v_at, int j, int e) {
  const char *at = vt + (v_at ^ (e << 6)) + j * 16 * ROW;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4 *)at);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4 *)(at + 8 * ROW));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Halves of a word with those that are infinite or NaN as 0.
__device__ __forceinline__ unsigned finite_halves(unsigned w) {
  const unsigned x = ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;      // top bits of those that are not
  return w & ~((x << 1) - (x >> 15));
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// The outputs of a lane's row that a key from `from` on, which the row sees, holds
// such a value for are NaN.  (Rare, and slow.)
template <bool BF16, int D>
__device__ __forceinline__ void spoil(const char *v, int64_t stride_bytes, int from, int end, f32x16 (&o)[D / 32]) {
  const int g = (threadIdx.x & 63) >> 5;
  for (int key = from; key < end; ++key) {
    const char *p = v + key * stride_bytes;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int dim = 32 * e + 8 * t + 4 * g + i;
          const float x = BF16 ? __uint_as_float((unsigned)reinterpret_cast<const uint16_t *>(p)[dim] << 16)
                               : reinterpret_cast<const float *>(p)[dim];
          if (!finite(x)) o[e][4 * t + i] = __builtin_nanf("");
        }
  }
}

// A unit's outputs; false where one came out that is not finite, and nothing is
// handed on.  That may be by a masked key's value (0 times it): CAREFUL counts such
// values as 0 in tiles that mask keys, and finds what sees them.  (Looking for them
// at once took 1.5 us of a masked tile's 3.)  SETS of four waves take tiles in turn,
// each through two buffers of its own.
template <int D, int SETS, bool CAREFUL>
__device__ __forceinline__ bool attend_unit(const PromptArgs &a, int unit, int t, char *lds) {
  constexpr int KEYS = 64, PIECES = D / 8, TILE = KEYS * D * 2, ROW = D * 2;
  const Unit u = unit_of(a, unit);
  const int lane = t & 63, set = SETS == 1 ? 0 : __builtin_amdgcn_readfirstlane(t >> 8);
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6 & 3);
  const int n = lane & 31, g = lane >> 5;
  const Row row = row_of(a, u, wave * 32 + n);
  const char *k = static_cast<const char *>(a.k) + ((int64_t)u.s.k0 * a.k_stride + u.h * D) * 2;
  const char *v = static_cast<const char *>(a.v) + ((int64_t)u.s.k0 * a.v_stride + u.h * D) * 2;
  char *own = lds + set * 4 * TILE;                          // this set's two buffers
  const unsigned lds_at = (unsigned)(uintptr_t)(LDS char *)own;
  Share<KEYS, PIECES> ks, vs;
  ks.find(a.k_stride * 2, KEYS, wave, k_place<PIECES>);
  vs.find(a.v_stride * 2, KEYS, wave, v_place<PIECES>);
  const auto ask = [&](int base, int buffer) {
    const unsigned to = lds_at + buffer * 2 * TILE;
    if (u.s.keys - base < KEYS) {
      ks.find(a.k_stride * 2, u.s.keys - base, wave, k_place<PIECES>);
      vs.find(a.v_stride * 2, u.s.keys - base, wave, v_place<PIECES>);
    }
    ks.ask(k + base * a.k_stride * 2, to, wave);
    vs.ask(v + base * a.v_stride * 2, to + TILE, wave);
  };
  bf16x8 q[D / 16];
  if (u.from + set * KEYS < u.to) ask(u.from + set * KEYS, 0);
  {
    const char *p = static_cast<const char *>(a.q) +
                    (((int64_t)u.s.q0 + row.query) * a.q_stride + (int64_t)row.head * D) * 2 + g * 16;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      u32x4 w = {0, 0, 0, 0};
      if (row.valid) w = *reinterpret_cast<const u32x4 *>(p + 32 * i);
      q[i] = __builtin_bit_cast(bf16x8, w);
    }
  }
  // below this key nothing of the wave's is masked
  const int clear = __builtin_amdgcn_readfirstlane(row.valid ? row.end : u.s.keys);
  const int far = __builtin_amdgcn_readfirstlane(
      min(u.to, u.row0 + wave * 32 >= u.rows ? 0
                                             : keys_seen(u.s, (min(u.row0 + wave * 32 + 32, u.rows) - 1) / a.G)));
  const float scale_log2 = a.scale * kLog2e;
  // this lane's places in a tile: K rows n (+ 32), V rows 4 g + n / 4 % 4 (+ 8 ..)
  const int k_at = n * ROW + ((g ^ k_place<PIECES>(n)) << 4);
  const int key = 4 * g + ((lane & 15) >> 2);
  const int v_at = key * ROW + (((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ v_place<PIECES>(key)) << 4) + (lane & 1) * 8;
  f32x16 o[D / 32];
  Weighed w;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] = 0.f;
  int buffer = 0;
  for (int step = u.from; step < u.to; step += SETS * KEYS, buffer ^= 1) {
    const int base = step + set * KEYS;
    tile_barrier();
    if (base + SETS * KEYS < u.to) ask(base + SETS * KEYS, buffer ^ 1);
    if (base >= far) continue;
    const char *kt = own + buffer * 2 * TILE, *vt = kt + TILE;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const bf16x8 x = *reinterpret_cast<const bf16x8 *>(kt + (k_at ^ (c << 5)) + i * 32 * ROW);
        s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[c], s[i], 0, 0, 0);
      }
    }
    const bool masked = base + KEYS > clear;
    if (masked) mask(s, row.end - base);
    weigh(s, o, w, scale_log2);
    const auto product = [&](auto value) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {                        // 16 keys a step
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[j >> 1][8 * (j & 1) + e];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(j, e), p, o[e], 0, 0, 0);
      }
    };
    if (CAREFUL && masked)
      product([&](int j, int e) {
        u32x4 y = __builtin_bit_cast(u32x4, v_piece<ROW>(vt, v_at, j, e));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = finite_halves(y[i]);
        return __builtin_bit_cast(bf16x8, y);
      });
    else
      product([&](int j, int e) { return v_piece<ROW>(vt, v_at, j, e); });
  }
  // (the buffer that nothing reads or fills now, and the one read last)
  int *stop = reinterpret_cast<int *>(lds + buffer * 2 * TILE);
  if constexpr (!CAREFUL) {
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 2) most = max3(most, __builtin_fabsf(o[e][i]), __builtin_fabsf(o[e][i + 1]));
    const int at = set * 4 + wave;
    if (lane == 0) stop[at] = 0;
    if (row.valid && !finite(most)) stop[at] = 1;
    tile_barrier();
    int any = 0;
#pragma unroll
    for (int i = 0; i < 4 * SETS; ++i) any |= stop[i];
    if (any) return false;
  }
  if constexpr (SETS == 2) {
    if (CAREFUL) tile_barrier();
    // the second set's rows, each lane's for the same lane of the first
    f32x4 *to = reinterpret_cast<f32x4 *>(lds + 4 * TILE) + wave * (D / 8) * 64 + lane;
    float2 *ml = reinterpret_cast<float2 *>(lds + (buffer ^ 1) * 2 * TILE) + wave * 64 + lane;
    if (set == 1) {
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          to[(e * 4 + i) * 64] = f32x4{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]};
      *ml = make_float2(w.at, w.sum);
    }
    tile_barrier();
    if (set == 1) return true;
    const float2 x = *ml;
    const float at = fmaxf(w.at, x.x), f = __builtin_amdgcn_exp2f(minus(w.at, at)), h = __builtin_amdgcn_exp2f(minus(x.x, at));
    w.at = at;
    w.sum = w.sum * f + x.y * h;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 y = to[(e * 4 + i) * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[e][4 * i + j] = o[e][4 * i + j] * f + y[j] * h;
      }
  }
  if constexpr (CAREFUL) spoil<true, D>(v, a.v_stride * 2, max(u.from, clear & ~(KEYS - 1)), min(row.end, u.to), o);
  finish<true, D>(a, u, row, wave * 32 + n, o, w);
  return true;
}

template <int D, int SETS>
__global__ __launch_bounds__(256 * SETS, 2) void k_prompt_bf16(PromptArgs a) {
  __shared__ __align__(16) char lds[SETS * 4 * 64 * D * 2];  // K, V of two tiles a set
  if (attend_unit<D, SETS, false>(a, blockIdx.x, threadIdx.x, lds)) return;
  tile_barrier();                                            // every wave has seen that
  int unit = blockIdx.x, t = threadIdx.x;                    // (as if others: else the first time keeps what the
  asm volatile("" : "+s"(unit), "+v"(t));                    // second needs)
  attend_unit<D, SETS, true>(a, unit, t, lds);
}

// Eight floats as three bf16 parts whose sum they are: two cut off (a mask, and the
// rest is exact), the last one rounded.
__device__ __forceinline__ void split8(float (&x)[8], bf16x8 (&part)[3]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302);
    part[p] = __builtin_bit_cast(bf16x8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xFFFF0000u);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[2][i] = (__bf16)x[i];
}

// acc + a b of values in three parts: the six products that 24 bits of the whole
// can tell, the smallest first.
__device__ __forceinline__ f32x16 product(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16 acc) {
#pragma unroll
  for (int sum = 2; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i <= sum; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[sum - i], acc, 0, 0, 0);
  return acc;
}

// In full precision: the same products of values in three bf16 parts, six of
// them for one, which takes three eighths of the time of the matrix
// instructions for floats.  The workgroup splits a tile of 32 keys into LDS, each
// thread its share, read into registers while the tile before was computed on.
// In tiles that mask keys V's values that are not finite count as 0 and are noted:
// spoil finds who sees them.
template <int D>
__global__ __launch_bounds__(256, 2) void k_prompt_fp32(PromptArgs a) {
  constexpr int KEYS = 32, PIECES = D / 8, ROW = D * 2, PART = KEYS * ROW, EACH = KEYS * PIECES / 256;
  __shared__ __align__(16) char lds[6 * PART];               // K's parts, V's
  __shared__ int noted;
  const Unit u = unit_of(a, blockIdx.x);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int n = lane & 31, g = lane >> 5;
  const Row row = row_of(a, u, wave * 32 + n);
  const char *k = static_cast<const char *>(a.k) + ((int64_t)u.s.k0 * a.k_stride + u.h * D) * 4;
  const char *v = static_cast<const char *>(a.v) + ((int64_t)u.s.k0 * a.v_stride + u.h * D) * 4;
  f32x4 kr[EACH][2], vr[EACH][2];
  const auto ask = [&](int base) {                           // (rows past the last stand for it: they are masked)
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int at = i * 256 + t;
      const int64_t r = min(base + at / PIECES, u.s.keys - 1);
      const f32x4 *x = reinterpret_cast<const f32x4 *>(k + r * a.k_stride * 4) + at % PIECES * 2;
      const f32x4 *y = reinterpret_cast<const f32x4 *>(v + r * a.v_stride * 4) + at % PIECES * 2;
      kr[i][0] = x[0];
      kr[i][1] = x[1];
      vr[i][0] = y[0];
      vr[i][1] = y[1];
    }
  };
  if (u.from < u.to) ask(u.from);
  if (t == 0) noted = 0;
  bf16x8 q[D / 16][3];
  {
    const float *p = static_cast<const float *>(a.q) + ((int64_t)u.s.q0 + row.query) * a.q_stride + (int64_t)row.head * D + 8 * g;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
        if (row.valid) w = *reinterpret_cast<const f32x4 *>(p + 16 * i + 4 * e);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * e + j] = w[j];
      }
      split8(x, q[i]);
    }
  }
  const int clear = __builtin_amdgcn_readfirstlane(row.valid ? row.end : u.s.keys);
  const int far = __builtin_amdgcn_readfirstlane(
      min(u.to, u.row0 + wave * 32 >= u.rows ? 0
                                             : keys_seen(u.s, (min(u.row0 + wave * 32 + 32, u.rows) - 1) / a.G)));
  const int all_clear = keys_seen(u.s, u.row0 / a.G);        // below this key none of the workgroup's waves masks one
  const float scale_log2 = a.scale * kLog2e;
  f32x16 o[D / 32];
  Weighed w;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] = 0.f;
  const int k_at = n * ROW + ((g ^ k_place<PIECES>(n)) << 4);
  const int key = 4 * g + ((lane & 15) >> 2);
  const int v_at = key * ROW + (((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ v_place<PIECES>(key)) << 4) + (lane & 1) * 8;
  for (int base = u.from; base < u.to; base += KEYS) {
    lds_barrier();                                           // the tile before has been read
    bool bad = false;
    if (base + KEYS > all_clear)
#pragma unroll
      for (int i = 0; i < EACH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!finite(vr[i][e >> 2][e & 3])) {
            vr[i][e >> 2][e & 3] = 0.f;
            bad = true;
          }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int at = i * 256 + t, r = at / PIECES, c = at % PIECES;
      float x[8], y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = kr[i][e >> 2][e & 3];
        y[e] = vr[i][e >> 2][e & 3];
      }
      bf16x8 xp[3], yp[3];
      split8(x, xp);
      split8(y, yp);
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        *reinterpret_cast<bf16x8 *>(lds + p * PART + r * ROW + ((c ^ k_place<PIECES>(r)) << 4)) = xp[p];
        *reinterpret_cast<bf16x8 *>(lds + (3 + p) * PART + r * ROW + ((c ^ v_place<PIECES>(r)) << 4)) = yp[p];
      }
    }
    if (bad) noted = 1;
    ask(base + KEYS);
    lds_barrier();
    if (base >= far) continue;
    f32x16 s[1];
#pragma unroll
    for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      bf16x8 x[3];
#pragma unroll
      for (int p = 0; p < 3; ++p) x[p] = *reinterpret_cast<const bf16x8 *>(lds + p * PART + (k_at ^ (c << 5)));
      s[0] = product(x, q[c], s[0]);
    }
    if (base + KEYS > clear) mask(s, row.end - base);
    weigh(s, o, w, scale_log2);
#pragma unroll
    for (int j = 0; j < 2; ++j) {                            // 16 keys a step
      float x[8];
      bf16x8 p[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[0][8 * j + e];
      split8(x, p);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        bf16x8 y[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) y[i] = v_piece<ROW>(lds + (3 + i) * PART, v_at, j, e);
        o[e] = product(y, p, o[e]);
      }
    }
  }
  lds_barrier();
  if (noted) spoil<false, D>(v, a.v_stride * 4, max(u.from, all_clear & ~(KEYS - 1)), min(row.end, u.to), o);
  finish<false, D>(a, u, row, wave * 32 + n, o, w);
}

// Joins the parts of query rows: D / 4 threads a row, one row each.  Bytes bound
// it; the parts of a row are asked for four at a time.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void k_prompt_join(PromptArgs a) {
  constexpr int TR = D / 4, ROWS = 256 / TR;
  constexpr int GROUPS = kPromptRows / ROWS;
  const int group = blockIdx.x % GROUPS;
  const int i = blockIdx.x / GROUPS;                         // a tile of a KV head, of sequences that have parts
  const PromptSeq &s = a.s[seq_of<&PromptSeq::join0>(a, i)];
  const int tile = (i - s.join0) / a.Hkv, h = (i - s.join0) - tile * a.Hkv;
  const int first_unit = s.unit0 + tile * s.splits * a.Hkv + h;      // (tiles from the last one on, as in unit_of)
  const Unit u = unit_of(a, first_unit);
  const int r = group * ROWS + threadIdx.x / TR, dim = threadIdx.x % TR * 4;
  const Row row = row_of(a, u, r);
  if (!row.valid) return;
  const float2 *ml = a.part_ml + (int64_t)first_unit * kPromptRows + r;
  const float *po = a.part_o + ((int64_t)first_unit * kPromptRows + r) * D + dim;
  const int64_t step = (int64_t)a.Hkv * kPromptRows;
  float l = 0.f, most = kFloor;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < s.splits; p += 4) {
    float2 x[4];
    f32x4 y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = min(p + j, s.splits - 1) * step;
      x[j] = ml[at];
      y[j] = *reinterpret_cast<const f32x4 *>(po + at * D);
    }
    float m = most;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (p + j >= s.splits) x[j] = make_float2(kNoKey, 0.f);
      m = fmaxf(m, x[j].x);
    }
    const float f = __builtin_amdgcn_exp2f(minus(most, m));
    l *= f;
    acc *= f;
    most = m;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (x[j].x == kNoKey) continue;
      const float w = __builtin_amdgcn_exp2f(minus(x[j].x, m));
      l += x[j].y * w;
      acc += y[j] * w;
    }
  }
  const bool none = row.end <= 0;
  const float sum = none ? 1.f : l > 0.f ? l : __builtin_nanf(""), inv = 1.f / sum;
  acc = none ? f32x4{0.f, 0.f, 0.f, 0.f} : acc * inv;
  const int64_t token = u.s.q0 + row.query, at = (token * a.Hq + row.head) * D + dim;
  if constexpr (BF16)
    *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.out) + at) = __builtin_convertvector(acc, bf16x4);
  else
    *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at) = acc;
  if (dim == 0) {
    const float lse = none ? -INFINITY : (most + __log2f(sum)) * kLn2;
    if (a.lse) a.lse[token * a.Hq + row.head] = lse;
    const int place = u.s.window0 + row.query;
    if (a.window && place >= 0) a.window[((int64_t)u.s.index * a.Hq + row.head) * a.W + place] = lse;
  }
}

}  // namespace

// Microseconds of a step (a tile of keys) of a workgroup that has a compute unit to
// itself, of one of two that share it, and of the whole GPU for 256 steps.
struct StepTimes {
  double alone, shared, all;
};

static StepTimes step_times(int head_dim, bool bf16) {
  if (bf16) return head_dim == 128 ? StepTimes{1.17, 2.0, 1.0} : StepTimes{0.7, 0.95, 0.95};
  return head_dim == 128 ? StepTimes{3.2, 5.1, 2.35} : StepTimes{1.4, 1.9, 1.0};
}

// A batch takes what its longest workgroup does, or what all of them do together; a
// workgroup costs seven steps besides its own, and parts, alike in length, end in
// rounds of 512 (us, forecast and measured: 1K tokens of 28 heads 27 and 28; 512
// queries over 8K keys 158 and 156, in four parts 78 and 75, in five 105 and 90, in
// eight 92 and 83).
constexpr double kUnitSteps = 7;

static double forecast(const PromptArgs *a, const StepTimes &t, int keys_a_step, int chunk) {
  double steps = 0, units = 0, longest = 0;
  for (int i = 0; i < a->seqs; ++i) {
    const PromptSeq &s = a->s[i];
    const double seen = 0.5 * (std::max(0, s.keys - s.queries) + s.keys), n = (double)s.tiles * a->Hkv;
    steps += n * seen / keys_a_step;
    units += n * (chunk ? std::max(1.0, std::min(seen / chunk + 0.5, std::ceil((double)s.keys / chunk))) : 1.0);
    longest = std::max(longest, (double)(chunk ? std::min(s.keys, chunk) : s.keys) / keys_a_step);
  }
  double last = (longest + kUnitSteps) * t.alone;
  if (chunk) {
    const double full = std::floor(units / 512), rest = units - 512 * full;
    last = (longest + kUnitSteps) * (full * t.shared + (rest > 256 ? t.shared : rest > 0 ? t.alone : 0));
  } else if (units > 256) {
    last += (steps / units + kUnitSteps) * (t.shared - t.alone);      // beside one of mean length
  }
  return std::max(last, (steps + kUnitSteps * units) / 256 * t.all);
}

// The same with two sets of waves a workgroup and one part: a tile of a set costs half,
// a workgroup's join three steps more, and a compute unit holds one.  It pays where
// the longest rows are what the call waits for (us, one set and two: 1K tokens of 28
// heads 28.8 and 26.3, 2K of 16 47.6 and 41.5, of 28 52.9 and 48.1, of 32 53.7 and
// 52.1; not 256 tokens of 32, 12.7 and 13.9, nor four prompts of 4K, 572 and 657).
static bool two_sets(const PromptArgs *a, int head_dim, double *time) {
  double steps = 0, units = 0, longest = 0;
  for (int i = 0; i < a->seqs; ++i) {
    const PromptSeq &s = a->s[i];
    const double n = (double)s.tiles * a->Hkv;
    steps += n * 0.5 * (std::max(0, s.keys - s.queries) + s.keys) / 64;
    units += n;
    longest = std::max(longest, s.keys / 64.0);
  }
  if (!(units <= 256 ? longest >= 12 : units <= 512 && longest >= 20 && steps <= 0.6 * longest * units)) return false;
  *time = std::max(longest + 10, (steps + 10 * units) / 256) * (head_dim == 128 ? 1.0 : 0.61);
  return true;
}

PromptPlan prompt_plan(PromptArgs *a, int head_dim, bool bf16) {
  PromptPlan p{};
  int longest = 0;
  int64_t rows = 0, tiles = 0;
  for (int i = 0; i < a->seqs; ++i) {
    PromptSeq &s = a->s[i];
    const int64_t r = (int64_t)s.queries * a->G;
    s.tiles = (int)((r + kPromptRows - 1) / kPromptRows);
    longest = std::max(longest, s.keys);
    rows += r * a->Hkv;
    tiles += (int64_t)s.tiles * a->Hkv;
  }
  // The parts that the longest keys are divided into: as many as make the forecast
  // least, with the joining launch's time: 5 us and what its parts' bytes take
  // (512 parts of 128 rows of 128 dimensions 7.6 us, 1024 12.4).
  const StepTimes times = step_times(head_dim, bf16);
  const int keys_a_step = bf16 ? 64 : 32;
  double best = forecast(a, times, keys_a_step, 0);
  a->sets = bf16 && two_sets(a, head_dim, &best) ? 2 : 1;
  int chunk = 0;
  // (2^20 tiles fill the GPU; their join, of 4096 threads each, would pass a launch's 2^32.)
  for (int parts = 2; parts <= 64 && longest > 64 && tiles < 1 << 20; parts += std::max(1, parts / 4)) {
    const int c = ((longest + parts - 1) / parts + 63) / 64 * 64;
    const double time = forecast(a, times, keys_a_step, c) + 5 + 0.15 * parts + 7e-5 * head_dim / 128 * rows * parts;
    if (time < best) {
      best = time;
      chunk = c;
      a->sets = 1;
    }
    if (c == 64) break;
  }
  int64_t units = 0, joined = 0;
  std::sort(a->s, a->s + a->seqs, [](const PromptSeq &x, const PromptSeq &y) {
    return x.keys != y.keys ? x.keys > y.keys : x.index < y.index;
  });
  for (int i = 0; i < a->seqs; ++i) {
    PromptSeq &s = a->s[i];
    s.splits = chunk ? std::max(1, (s.keys + chunk - 1) / chunk) : 1;
    s.unit0 = (int)std::min<int64_t>(units, 0x7FFFFFFF);
    s.join0 = (int)std::min<int64_t>(joined, 0x7FFFFFFF);
    units += (int64_t)s.tiles * s.splits * a->Hkv;
    if (s.splits > 1) joined += (int64_t)s.tiles * a->Hkv;   // (the longest come first: those behind have one part)
  }
  a->units = (int)std::min<int64_t>(units, 0x7FFFFFFF);
  a->joined = (int)std::min<int64_t>(joined, 0x7FFFFFFF);
  if (joined) {
    const size_t part_rows = (size_t)units * kPromptRows;
    p.ml_bytes = part_rows * sizeof(float2);
    p.bytes = p.ml_bytes + part_rows * head_dim * sizeof(float);
  }
  return p;
}

template <int D>
static void launch(const PromptArgs &a, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)a.units);
  if (bf16 && a.sets == 2)
    hipLaunchKernelGGL((k_prompt_bf16<D, 2>), grid, dim3(512), 0, s, a);
  else if (bf16)
    hipLaunchKernelGGL((k_prompt_bf16<D, 1>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_prompt_fp32<D>), grid, dim3(256), 0, s, a);
  if (!a.joined) return;
  const dim3 join((unsigned)a.joined * (kPromptRows * D / 4 / 256));
  if (bf16)
    hipLaunchKernelGGL((k_prompt_join<true, D>), join, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_prompt_join<false, D>), join, dim3(256), 0, s, a);
}

hipError_t launch_prompt(const PromptArgs &a, bool bf16, int head_dim, hipStream_t s) {
  head_dim == 128 ? launch<128>(a, bf16, s) : launch<64>(a, bf16, s);
  return hipGetLastError();
}

}  // namespace bacon
