// Declarations shared by the kernels of the 8-bit cache and its host API.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bacon {

constexpr int kCacheLow = -100, kCacheHigh = 120;   // exponents a block's scale may take
constexpr int kCacheMaxBatch = 64;
constexpr int kCacheMaxHeads = 1024;               // KV heads
constexpr int kCacheMaxTokens = 64;                 // new tokens of one call
constexpr int kCacheMaxQRows = 64;                  // G * tokens of one attend
constexpr int kCacheLayersPerLaunch = 64;           // layers' pointers in one launch's arguments

// A cache in device memory (include/bacon.h states the layouts).
struct CacheDev {
  int L, B, Hq, Hkv, W;
  int bt_log;              // log2 of the tokens of a block
  int max_blocks;
  int num_blocks;
  int32_t *lens, *starts, *table;
  float *scales;
  uint8_t *codes;
  unsigned *err;
};

// The sequences of a prompt: tokens before each and its budget.
struct CacheSeqs {
  int batch;
  int cu[kCacheMaxBatch + 1];
  int budget[kCacheMaxBatch];
};

struct CacheTablesArgs {
  CacheDev c;
  CacheSeqs s;
  int first_seq;
  const int32_t *budgets;  // optional [L, budgets_batch, Hkv]
  int budgets_batch;
  int reserve;
  const int32_t *free_ids; // optional [num_free]
  int64_t num_free;
  int64_t *used;           // optional
  unsigned head_magic;     // 2^32 / Hkv, rounded up (set by the launch)
  int row_threads;         // threads of a table row, 64 to 1024 (set by the launch)
};

struct CacheStoreArgs {
  CacheDev c;
  CacheSeqs s;
  int first_seq, first_layer, layers;
  const void *k[kCacheLayersPerLaunch], *v[kCacheLayersPerLaunch];
  const int32_t *idx[kCacheLayersPerLaunch];   // NULL: entries 0, 1, 2, ...
  int64_t idx_count;       // entries of each
};

struct CacheLoadArgs {
  CacheDev c;
  int first_seq, num_seqs, first_layer, layers;
  int first_token, count;
  void *k, *v;
};

struct CacheStepArgs {
  CacheDev c;
  int layer, first_seq, num_seqs, tokens;
  const int32_t *counts;   // optional [num_seqs]
  // append
  const void *k, *v;
  int64_t k_stride, v_stride;   // elements between tokens
  // attend
  const void *q;
  int64_t q_stride;
  void *out;
  float *lse;              // optional
  float scale_log2;        // log2(e) / sqrt(d)
  int G, R;                // query heads of a KV head, query rows of a pair (set by the launch, as the next two)
  unsigned group_magic;    // 2^16 / G, rounded up
  int groups;              // workgroups that a unit's query rows take
  // Division of a pair's rows: `splits` workgroups of `chunk` rows (more where
  // the pair is longer); with several, each leaves its part in work.
  int splits, chunk;
  float2 *part_ml;         // [pairs, splits, R] maximum (log2 units) and sum
  float *part_o;           // [pairs, splits, R, d] sums weighted by 2^(logit - maximum)
};

// How an attend of q_rows query rows per pair is divided.
struct CachePlan {
  int splits, chunk;
  size_t ml_bytes, bytes;  // of the work buffer: part_ml, then part_o
};
CachePlan cache_plan(int pairs, int q_rows, int head_dim, int max_tokens);

struct CacheMoveArgs {
  CacheDev c;
  int first_seq, num_seqs, first_layer, layers, delta;
  const int32_t *deltas;   // optional [num_seqs]
};

hipError_t launch_cache_clear(const CacheDev &c, int first_seq, int num_seqs, bool errors, hipStream_t s);
hipError_t launch_cache_tables(CacheTablesArgs a, hipStream_t s);
// most_rows: upper bound of a pair's rows.
hipError_t launch_cache_store(const CacheStoreArgs &a, bool bf16, int head_dim, int most_rows, hipStream_t s);
// Workgroups of 256 threads that a load takes; a launch holds fewer than 2^32 threads.
int64_t cache_load_groups(int64_t pairs, int count, int head_dim);
constexpr int64_t kCacheMaxGroups = (1 << 24) - 1;
hipError_t launch_cache_load(const CacheLoadArgs &a, bool bf16, int head_dim, hipStream_t s);
hipError_t launch_cache_append(const CacheStepArgs &a, bool bf16, int head_dim, hipStream_t s);
// Whether an attend of q_rows query rows per pair also appends a's new rows
// (a.k not NULL); otherwise one workgroup would read rows that another writes.
bool cache_appends(int q_rows);
hipError_t launch_cache_attend(CacheStepArgs a, bool bf16, int head_dim, hipStream_t s);
hipError_t launch_cache_advance(const CacheMoveArgs &a, hipStream_t s);

}  // namespace bacon
