// Checks and numbers that every entry point derives from its lazy_attn_params_t (host code, no HIP).
#pragma once

#include <math.h>
#include <stdint.h>

#include "lazy_attn.h"

namespace lazy {

constexpr int kNumCUs = 256;  // MI355X compute units

// Workgroups of one launch dimension: with 256 threads each, a launch holds fewer than 2^32.
constexpr int64_t kMaxGroups = ((int64_t)1 << 24) - 1;
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_params(const lazy_attn_params_t* p) {
  if (!p) return LAZY_EINVAL;
  if (p->num_q_heads <= 0 || p->num_kv_heads <= 0 || p->num_q_heads % p->num_kv_heads != 0) return LAZY_EINVAL;
  if (p->causal != 0 && p->causal != 1) return LAZY_EINVAL;
  if (!isfinite(p->softmax_scale) || p->softmax_scale < 0.f) return LAZY_EINVAL;
  if (p->rope_style != LAZY_ALIBI && !p->inv_freq && !(isfinite(p->rope_base) && p->rope_base > 0.f)) return LAZY_EINVAL;
  if (p->num_splits < 0) return LAZY_EINVAL;
  if (p->key_positions != LAZY_KEYS_NOPE && p->key_positions != LAZY_KEYS_LOCAL) return LAZY_EINVAL;
  if (p->rope_style != LAZY_ROPE_HALF && p->rope_style != LAZY_ROPE_INTERLEAVED && p->rope_style != LAZY_ALIBI)
    return LAZY_EINVAL;
  if (p->rope_style == LAZY_ALIBI && p->key_positions != LAZY_KEYS_NOPE) return LAZY_EINVAL;
  if (p->q_prerotated != 0 && p->q_prerotated != 1) return LAZY_EINVAL;
  if (p->cache_hint != LAZY_CACHE_DEFAULT && p->cache_hint != LAZY_CACHE_STREAM) return LAZY_EINVAL;
  if (p->head_dim != 64 && p->head_dim != 128) return LAZY_EUNSUPPORTED;
  return LAZY_OK;
}

inline float scale_log2(const lazy_attn_params_t* p) {
  const float s = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  return s * 1.4426950408889634f;
}

inline double rope_log2_base(const lazy_attn_params_t* p) {
  return p->inv_freq || p->rope_style == LAZY_ALIBI ? 0.0 : log2((double)p->rope_base);
}

// Rotations per position of every pair, in revolutions (not used with a table of the caller's, or with ALiBi).
inline void rope_revolutions(const lazy_attn_params_t* p, double (&rev)[64]) {
  const double l = rope_log2_base(p);
  for (int t = 0; t < 64; ++t)
    rev[t] = t < p->head_dim / 2 ? exp2(-2.0 * t / p->head_dim * l) * 0.15915494309189533577 : 0.0;
}

}  // namespace lazy
