// gfx950 kernels of the 8-bit cache: block tables from the budgets, the kept
// rows quantised into blocks and read back, and new tokens' rows.
// include/bacon.h states the layouts and the numbers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_dev.h"

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
        for (int j = 0; j < 8; ++j) tile[v_at<D>(r, (t % TR) * 8 + j)] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
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
        const unsigned kc = block_codes<D>(c, id, 0)[at * D + dim], vc = block_codes<D>(c, id, 1)[v_at<D>(at, dim)];
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

int blocks_for(int64_t n, int per, int most) { return (int)std::max<int64_t>(1, std::min<int64_t>(most, (n + per - 1) / per)); }

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
  CACHE_LAUNCH(k_cache_store, grid, 256, s, a, per_pair);
  return hipGetLastError();
}

hipError_t launch_cache_load(const CacheLoadArgs &a, bool bf16, int head_dim, hipStream_t s) {
  const int64_t rows = (int64_t)a.layers * a.num_seqs * a.c.Hkv * a.count;
  const dim3 grid(blocks_for(rows * head_dim, 256, 1 << 20));
  CACHE_LAUNCH(k_cache_load, grid, 256, s, a, rows);
  return hipGetLastError();
}

hipError_t launch_cache_append(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s) {
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
