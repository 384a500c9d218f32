// Declarations shared by the kernels of the prompt's attention and its host API.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bacon {

constexpr int kPromptMaxBatch = 64;

// A sequence: its first row of K, keys, first row of Q, queries, and the units
// (a tile of query rows of one KV head, or a part of its keys) before it.
struct PromptSeq {
  int k0, keys, q0, queries;
  int unit0, tiles, splits, index;
  int join0;               // tiles of KV heads before it that are joined
  int window0;             // its first query's entry of the window (below 0: that query has none)
};

struct PromptArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;   // elements between tokens
  void *out;
  float *lse, *window;     // optional
  int Hq, Hkv, G, W;
  unsigned group_magic;    // 2^32 / G, rounded up (0 where G is 1)
  float scale;             // 1 / sqrt(d)
  int seqs, units;
  int sets;                // of four waves a workgroup (bf16), which take a unit's keys in turn
  int joined;              // tiles of KV heads whose parts are joined
  float2 *part_ml;         // [unit rows] maximum and sum of every part
  float *part_o;           // [unit rows, d]
  PromptSeq s[kPromptMaxBatch];
};

// Query rows (queries x G heads of a KV head) of a workgroup.
constexpr int kPromptRows = 128;

struct PromptPlan {
  size_t ml_bytes, bytes;  // of the work buffer
};

// Divides the sequences that a holds (k0, keys, q0, queries, index) into units.
PromptPlan prompt_plan(PromptArgs *a, int head_dim, bool bf16);
hipError_t launch_prompt(const PromptArgs &a, bool bf16, int head_dim, hipStream_t s);

}  // namespace bacon
