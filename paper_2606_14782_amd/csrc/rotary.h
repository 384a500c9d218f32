// Declarations shared by the rotary positions' kernel and its host API.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bacon {

constexpr int kRotaryMaxHeads = 4096;
constexpr int kRotaryMaxPairs = 64;
// What a head's values are multiplied by where their squares pass a float's range, or
// come so low that they lose bits.
constexpr float kNormLarge = 0x1p-72f, kNormSmall = 0x1p100f;
constexpr int kRotaryMaxTokens = 1 << 25;     // of a call: a launch holds fewer than 2^32 threads

// Heads of one side (q or k): [tokens, heads, d], tokens `stride` elements apart.
struct RotarySide {
  const void *x;
  void *y;
  const void *norm;        // optional [d]
  int64_t x_stride, y_stride;
  int heads;               // 0: not given
};

struct RotateArgs {
  RotarySide q, k;
  int64_t tokens;
  const int32_t *pos;      // [tokens] or [3, tokens]
  int pairs;               // rotary_dim / 2
  int row1, row2;          // pairs from row1 on turn by the second row, from row2 on by the third
  float magnitude, eps;
  float eps_large, eps_small;      // eps beside the squares of values times kNormLarge, kNormSmall
  int per_wave;            // head groups a wave takes of its token (set by the launch, as the next)
  int parts;               // waves of a token
  double turns[kRotaryMaxPairs];   // of a pair, a position
};

hipError_t launch_rotate(RotateArgs a, bool bf16, int head_dim, bool half, hipStream_t s);

}  // namespace bacon
