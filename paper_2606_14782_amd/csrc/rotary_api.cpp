// Host side of the rotary positions declared in include/bacon.h: argument
// checks, frequencies and the launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/bacon.h"
#include "error.h"
#include "rotary.h"

using namespace bacon;

namespace {

#define TRY(x)                     \
  do {                             \
    bacon_status _s = (x);         \
    if (_s != BACON_OK) return _s; \
  } while (0)

constexpr double kTwoPi = 6.283185307179586;
constexpr double kMostFrequency = 1e6;

bacon_status check_rotary(const bacon_rotary *r) {
  if (!r) return fail(BACON_ERR_INVALID, "rotary is NULL");
  if (r->num_q_heads < 1 || r->num_kv_heads < 1) return fail(BACON_ERR_INVALID, "head counts must be >= 1");
  if (r->num_q_heads > kRotaryMaxHeads || r->num_kv_heads > kRotaryMaxHeads)
    return fail(BACON_ERR_UNSUPPORTED, "%d and %d heads exceed %d", r->num_q_heads, r->num_kv_heads, kRotaryMaxHeads);
  if (r->dtype != BACON_FP32 && r->dtype != BACON_BF16)
    return fail(BACON_ERR_UNSUPPORTED, "dtype %d is not supported", (int)r->dtype);
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(BACON_ERR_UNSUPPORTED, "head_dim %d is not supported (64 or 128)", r->head_dim);
  if (r->rotary_dim < 2 || r->rotary_dim > r->head_dim || r->rotary_dim % 2)
    return fail(BACON_ERR_INVALID, "rotary_dim %d is not even and in [2, %d]", r->rotary_dim, r->head_dim);
  if (r->layout != BACON_ROTARY_HALF && r->layout != BACON_ROTARY_PAIRS)
    return fail(BACON_ERR_INVALID, "layout %d is none", r->layout);
  int64_t sum = 0;
  for (int i = 0; i < 3; ++i) {
    if (r->sections[i] < 0) return fail(BACON_ERR_INVALID, "sections must be >= 0");
    sum += r->sections[i];
  }
  if (sum && sum != r->rotary_dim / 2)
    return fail(BACON_ERR_INVALID, "sections hold %lld pairs of %d", (long long)sum, r->rotary_dim / 2);
  if (!(r->norm_eps >= 0) || !(r->norm_eps <= 3e38)) return fail(BACON_ERR_INVALID, "norm_eps must be >= 0 and finite");
  if (!(r->magnitude >= 0) || !(r->magnitude <= 3e38))
    return fail(BACON_ERR_INVALID, "magnitude must be >= 0 and finite");
  if (r->scaling < BACON_ROTARY_PLAIN || r->scaling > BACON_ROTARY_GIVEN)
    return fail(BACON_ERR_INVALID, "scaling %d is none", r->scaling);
  if (r->scaling == BACON_ROTARY_GIVEN) {
    if (!r->frequencies) return fail(BACON_ERR_INVALID, "frequencies are NULL");
    for (int i = 0; i < r->rotary_dim / 2; ++i)
      if (!(std::fabs(r->frequencies[i]) <= kMostFrequency))
        return fail(BACON_ERR_INVALID, "frequency %d is not within +-%g", i, kMostFrequency);
    return BACON_OK;
  }
  if (!(r->base > 1) || !std::isfinite(r->base)) return fail(BACON_ERR_INVALID, "base must be > 1 and finite");
  if (!(r->factor >= 1) || !std::isfinite(r->factor)) return fail(BACON_ERR_INVALID, "factor must be >= 1 and finite");
  if (r->scaling == BACON_ROTARY_PLAIN && r->factor != 1)
    return fail(BACON_ERR_INVALID, "a factor needs a scaling that uses it");
  if (r->scaling == BACON_ROTARY_NTK && r->rotary_dim <= 2)
    return fail(BACON_ERR_INVALID, "NTK scaling needs a rotary_dim > 2");
  if (r->scaling == BACON_ROTARY_YARN) {
    if (r->trained_tokens < 1) return fail(BACON_ERR_INVALID, "trained_tokens must be >= 1");
    if (!(r->beta_slow > 0) || !(r->beta_fast > r->beta_slow) || !std::isfinite(r->beta_fast))
      return fail(BACON_ERR_INVALID, "betas must be finite with beta_fast > beta_slow > 0");
  }
  return BACON_OK;
}

// The frequencies (radians a token) of a checked rotary, and its magnitude.
double frequencies_of(const bacon_rotary *r, double *f) {
  const int dim = r->rotary_dim;
  double m = 1;
  const double base =
      r->scaling == BACON_ROTARY_NTK ? r->base * std::pow(r->factor, (double)dim / (dim - 2)) : r->base;
  for (int i = 0; i < dim / 2; ++i) {
    if (r->scaling == BACON_ROTARY_GIVEN) {
      f[i] = r->frequencies[i];
      continue;
    }
    const double w = std::pow(base, -2.0 * i / dim);
    f[i] = r->scaling == BACON_ROTARY_LINEAR ? w / r->factor : w;
    if (r->scaling == BACON_ROTARY_YARN) {
      const double n = r->trained_tokens * w / kTwoPi;
      const double g = std::min(1.0, std::max(0.0, (n - r->beta_slow) / (r->beta_fast - r->beta_slow)));
      f[i] = (1 - g) * w / r->factor + g * w;
    }
  }
  if (r->scaling == BACON_ROTARY_YARN) m = 0.1 * std::log(r->factor) + 1;
  return r->magnitude > 0 ? r->magnitude : m;
}

bacon_status check_ptr(const void *p, const char *name, size_t align) {
  if (!p) return fail(BACON_ERR_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(BACON_ERR_INVALID, "%s is not %zu-byte aligned", name, align);
  return BACON_OK;
}

bacon_status check_rows(const bacon_rotary *r, const void *p, int64_t stride, int heads, const char *name) {
  TRY(check_ptr(p, name, 16));
  const int64_t row = (int64_t)heads * r->head_dim;
  if (stride < row)
    return fail(BACON_ERR_INVALID, "%s tokens of %lld elements are %lld elements apart", name, (long long)row,
                (long long)stride);
  if (stride % (r->dtype == BACON_BF16 ? 8 : 4))
    return fail(BACON_ERR_INVALID, "the distance of %s tokens (%lld elements) is not a multiple of 16 bytes", name,
                (long long)stride);
  return BACON_OK;
}

bacon_status check_side(const bacon_rotary *r, const RotarySide &s, int heads, const char *in, const char *out,
                        const char *norm) {
  if (!s.x) {
    if (s.y) return fail(BACON_ERR_INVALID, "%s is NULL, %s is not", in, out);
    return BACON_OK;
  }
  TRY(check_rows(r, s.x, s.x_stride, heads, in));
  TRY(check_rows(r, s.y, s.y_stride, heads, out));
  if (s.x == s.y && s.x_stride != s.y_stride)
    return fail(BACON_ERR_INVALID, "%s is %s with tokens another distance apart", out, in);
  if (s.norm) TRY(check_ptr(s.norm, norm, 16));
  return BACON_OK;
}

}  // namespace

extern "C" {

void bacon_default_rotary(bacon_rotary *r) {
  if (!r) return;
  *r = bacon_rotary{};
  r->num_q_heads = r->num_kv_heads = 1;
  r->head_dim = r->rotary_dim = 128;
  r->base = 10000;
  r->factor = 1;
  r->beta_fast = 32;
  r->beta_slow = 1;
  r->norm_eps = 1e-6;
  r->dtype = BACON_BF16;
}

bacon_status bacon_rotary_frequencies(const bacon_rotary *r, double *frequencies, double *magnitude) {
  TRY(check_rotary(r));
  if (!frequencies || !magnitude) return fail(BACON_ERR_INVALID, "outputs are NULL");
  *magnitude = frequencies_of(r, frequencies);
  return BACON_OK;
}

bacon_status bacon_rotate(const bacon_rotary *r, int64_t tokens, const int32_t *d_positions, const void *d_q,
                          int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_q_norm,
                          const void *d_k_norm, void *d_q_out, int64_t q_out_stride, void *d_k_out,
                          int64_t k_out_stride, void *stream) {
  TRY(check_rotary(r));
  if (tokens < 0) return fail(BACON_ERR_INVALID, "%lld tokens", (long long)tokens);
  if (tokens > kRotaryMaxTokens)
    return fail(BACON_ERR_UNSUPPORTED, "%lld tokens exceed %d", (long long)tokens, kRotaryMaxTokens);
  RotateArgs a{};
  a.q = RotarySide{d_q, d_q_out, d_q_norm, q_stride, q_out_stride, d_q ? r->num_q_heads : 0};
  a.k = RotarySide{d_k, d_k_out, d_k_norm, k_stride, k_out_stride, d_k ? r->num_kv_heads : 0};
  if (tokens == 0) return BACON_OK;
  if (!d_q && !d_k) return fail(BACON_ERR_INVALID, "q and k are NULL");
  TRY(check_ptr(d_positions, "positions", 4));
  TRY(check_side(r, a.q, r->num_q_heads, "q", "q_out", "q_norm"));
  TRY(check_side(r, a.k, r->num_kv_heads, "k", "k_out", "k_norm"));
  double f[kRotaryMaxPairs];
  a.tokens = tokens;
  a.pos = d_positions;
  a.pairs = r->rotary_dim / 2;
  const bool rows = r->sections[0] || r->sections[1] || r->sections[2];
  a.row1 = rows ? r->sections[0] : a.pairs;
  a.row2 = rows ? r->sections[0] + r->sections[1] : a.pairs;
  a.magnitude = (float)frequencies_of(r, f);
  a.eps = (float)r->norm_eps;
  a.eps_large = (float)(r->norm_eps * kNormLarge * kNormLarge);
  a.eps_small = (float)std::min(r->norm_eps * kNormSmall * kNormSmall, 3e38);
  for (int i = 0; i < a.pairs; ++i) a.turns[i] = f[i] / kTwoPi;
  const hipError_t e = launch_rotate(a, r->dtype == BACON_BF16, r->head_dim, r->layout == BACON_ROTARY_HALF,
                                     static_cast<hipStream_t>(stream));
  return e == hipSuccess ? BACON_OK : fail(BACON_ERR_HIP, "rotate: %s", hipGetErrorString(e));
}

}  // extern "C"
