// C entry points of the eviction by accumulated attention weight: argument checks, launch sizes and dispatch.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "lazy_attn_internal.h"
#include "lazy_attn_params.h"

namespace {

using lazy::ceil_div, lazy::check_params, lazy::kMaxGroups, lazy::kNumCUs;

constexpr int kTileKeys = 64, kAngleRows = 32;
constexpr int64_t kSortBytes = 512 << 10;

int status(hipError_t e) { return e == hipSuccess ? LAZY_OK : LAZY_EHIP; }

struct PromptSizes {
  int splits, row_splits;
  size_t q, nlse, angles, part, bytes;
};

// A workgroup takes two 64-key tiles at a time; its rows are divided where the tiles alone do not fill the chip.
PromptSizes prompt_sizes(const lazy_attn_params_t* p, int32_t batch, int32_t total_q, int32_t max_q_len,
                         int32_t max_kv_len, int32_t num_keys) {
  PromptSizes z = {};
  const int64_t rows = (int64_t)total_q * p->num_q_heads, tiles = std::max<int64_t>(1, ceil_div(max_kv_len, kTileKeys));
  z.splits = (int)std::min<int64_t>(ceil_div(tiles, 4), 1 << 20);  // two rounds each
  const int64_t steps = ceil_div((int64_t)max_q_len * (p->num_q_heads / p->num_kv_heads), 32);
  const int64_t groups = (int64_t)z.splits * p->num_kv_heads * std::max(batch, 1);
  z.row_splits = (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(2 * kNumCUs, groups), steps / 4, 16}));
  const auto put = [&z](size_t bytes) {
    const size_t here = z.bytes;
    z.bytes += (bytes + 255) & ~(size_t)255;
    return here;
  };
  z.q = put((size_t)rows * p->head_dim * sizeof(uint16_t) * (p->rope_style == LAZY_ALIBI ? 1 : 2));
  z.nlse = put((size_t)rows * sizeof(float));
  const bool block_angles = p->key_positions == LAZY_KEYS_NOPE && p->rope_style != LAZY_ALIBI;
  z.angles = put((block_angles ? (size_t)kAngleRows : 0) * p->head_dim * sizeof(float));
  z.part = put((size_t)z.row_splits * p->num_kv_heads * (size_t)num_keys * sizeof(float));
  return z;
}

void fill(lazy::WeightArgs& a, const lazy_attn_params_t* p) {
  a.inv_freq = p->inv_freq;
  a.hq = p->num_q_heads;
  a.hkv = p->num_kv_heads;
  a.group = a.hq / a.hkv;
  a.group_magic = a.group == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
  a.causal = p->causal;
  a.rotate_q = !p->q_prerotated && p->rope_style != LAZY_ALIBI;
  a.rotate_k = p->rope_style != LAZY_ALIBI;
  lazy::rope_revolutions(p, a.rev);
  a.scale_log2 = lazy::scale_log2(p);
}

}  // namespace

extern "C" {

size_t lazy_attn_prefill_key_weights_workspace_size(const lazy_attn_params_t* params, int32_t batch, int32_t total_q,
                                                    int32_t max_q_len, int32_t max_kv_len, int32_t num_keys) {
  if (check_params(params) != LAZY_OK || batch <= 0 || total_q < 0 || max_q_len < 0 || max_kv_len <= 0 || num_keys <= 0)
    return 0;
  return prompt_sizes(params, batch, total_q, max_q_len, max_kv_len, num_keys).bytes;
}

int lazy_attn_prefill_key_weights(const lazy_attn_params_t* p, const void* q, const int32_t* q_start,
                                  const int32_t* q_pos0, const void* k_pool, const lazy_chunk_t* chunks,
                                  const int32_t* chunk_start, const int32_t* key_start, int32_t batch, int32_t total_q,
                                  int32_t max_q_len, int32_t max_kv_len, int32_t num_keys, const float* lse,
                                  const float* weights_in, float decay, float* weights, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  const int e = check_params(p);
  if (e != LAZY_OK) return e;
  if (batch < 0 || total_q < 0 || max_q_len < 0 || max_kv_len < 0 || num_keys < 0 || !std::isfinite(decay))
    return LAZY_EINVAL;
  if (batch == 0 || max_kv_len == 0 || num_keys == 0) return LAZY_OK;
  if (total_q > 0 && (max_q_len == 0 || !q || !lse)) return LAZY_EINVAL;
  if (!q_start || !q_pos0 || !k_pool || !chunks || !chunk_start || !key_start || !weights) return LAZY_EINVAL;
  const int64_t g = p->num_q_heads / p->num_kv_heads;
  if ((int64_t)total_q * g * g >= (int64_t)1 << 32 || (int64_t)total_q * g >= INT32_MAX) return LAZY_EUNSUPPORTED;
  if (batch > 65535 || p->num_kv_heads > 65535 || total_q > kMaxGroups) return LAZY_EUNSUPPORTED;
  const PromptSizes z = prompt_sizes(p, batch, total_q, max_q_len, max_kv_len, num_keys);
  if (!workspace || workspace_bytes < z.bytes || ((uintptr_t)workspace & 15u)) return LAZY_EWORKSPACE;
  char* ws = static_cast<char*>(workspace);
  lazy::WeightArgs a = {};
  fill(a, p);
  a.q = static_cast<const uint16_t*>(q);
  a.q_start = q_start;
  a.q_pos0 = q_pos0;
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.chunks = chunks;
  a.chunk_start = chunk_start;
  a.key_start = key_start;
  a.lse = lse;
  a.weights_in = weights_in;
  a.weights = weights;
  a.ws_q = reinterpret_cast<uint16_t*>(ws + z.q);
  a.ws_nlse = reinterpret_cast<float*>(ws + z.nlse);
  a.ws_angles = reinterpret_cast<float*>(ws + z.angles);
  a.ws_part = reinterpret_cast<float*>(ws + z.part);
  a.rows = (int64_t)total_q * g;
  a.total_q = total_q;
  a.batch = batch;
  a.splits = z.splits;
  a.row_splits = z.row_splits;
  a.num_keys = num_keys;
  a.decay = decay;
  return status(lazy::launch_prefill_weights(a, p->head_dim, p->key_positions == LAZY_KEYS_LOCAL,
                                             p->rope_style == LAZY_ROPE_INTERLEAVED, p->rope_style == LAZY_ALIBI,
                                             max_kv_len, static_cast<hipStream_t>(stream)));
}

size_t lazy_attn_decode_key_weights_workspace_size(const lazy_attn_params_t*, int32_t, int32_t) { return 0; }

int lazy_attn_decode_key_weights(const lazy_attn_params_t* p, const void* q, const int32_t* q_pos, const void* k_pool,
                                 const lazy_chunk_t* chunks, const int32_t* chunk_start, const int32_t* key_start,
                                 int32_t batch, int32_t max_kv_len, const float* lse, const float* weights_in,
                                 float decay, float* weights, void*, size_t, void* stream) {
  const int e = check_params(p);
  if (e != LAZY_OK) return e;
  if (batch < 0 || max_kv_len < 0 || !std::isfinite(decay)) return LAZY_EINVAL;
  if (batch == 0 || max_kv_len == 0) return LAZY_OK;
  if (!q || !q_pos || !k_pool || !chunks || !chunk_start || !key_start || !lse || !weights) return LAZY_EINVAL;
  if (batch > 65535) return LAZY_EUNSUPPORTED;
  lazy::WeightArgs a = {};
  fill(a, p);
  a.q = static_cast<const uint16_t*>(q);
  a.q_pos0 = q_pos;
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.chunks = chunks;
  a.chunk_start = chunk_start;
  a.key_start = key_start;
  a.lse = lse;
  a.weights_in = weights_in;
  a.weights = weights;
  a.total_q = batch;
  a.batch = batch;
  // Three workgroups a CU, at least one tile each; where there are fewer tiles than that, four workgroups a tile.
  const int64_t tiles = ceil_div(max_kv_len, kTileKeys);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(3 * kNumCUs, batch), tiles));
  a.head_split = p->num_kv_heads > 1 && tiles * batch <= kNumCUs;
  // Storage order: where a workgroup reads enough for the caches to matter (sorting takes it 1-2 us).
  a.sort_records = batch > 1 && !a.head_split &&
                   (int64_t)max_kv_len / a.splits * p->num_kv_heads * p->head_dim * 2 >= kSortBytes;
  a.decay = decay;
  return status(lazy::launch_decode_weights(a, p->head_dim, p->key_positions == LAZY_KEYS_LOCAL,
                                            p->rope_style == LAZY_ROPE_INTERLEAVED, p->rope_style == LAZY_ALIBI,
                                            static_cast<hipStream_t>(stream)));
}

size_t lazy_cache_select_workspace_size(int32_t batch, int32_t max_kv_len) {
  return batch <= 0 || max_kv_len <= 0 ? 0 : lazy::select_workspace(batch, max_kv_len);
}

int lazy_cache_select(const float* weights, const int32_t* key_start, const int32_t* key_count,
                      const int32_t* kept_start, int32_t batch, int32_t max_kv_len, int32_t sink, int32_t recent,
                      int32_t* kept, void* workspace, size_t workspace_bytes, void* stream) {
  if (batch < 0 || max_kv_len < 0 || sink < 0 || recent < 0) return LAZY_EINVAL;
  if (batch == 0) return LAZY_OK;
  if (!key_start || !kept_start || !kept || (max_kv_len > 0 && !weights)) return LAZY_EINVAL;
  if (batch > 65535) return LAZY_EUNSUPPORTED;
  const size_t need = lazy::select_workspace(batch, max_kv_len);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15u))) return LAZY_EWORKSPACE;
  return status(lazy::launch_select(weights, key_start, key_count, kept_start, batch, max_kv_len, sink, recent, kept,
                                    workspace, static_cast<hipStream_t>(stream)));
}

int lazy_cache_compact(const lazy_attn_params_t* p, const void* k_pool, const void* v_pool, const lazy_chunk_t* chunks,
                       const int32_t* chunk_start, int32_t batch, const int32_t* kept, const int32_t* kept_start,
                       int32_t max_kept, const lazy_chunk_t* dst, int32_t rotate, void* k_out, void* v_out,
                       const int32_t* key_start, const float* weights, float* weights_out, void* stream) {
  const int e = check_params(p);
  if (e != LAZY_OK) return e;
  if (batch < 0 || max_kept < 0 || (rotate != 0 && rotate != 1)) return LAZY_EINVAL;
  if (rotate && p->rope_style == LAZY_ALIBI) return LAZY_EUNSUPPORTED;
  const int some = (key_start != nullptr) + (weights != nullptr) + (weights_out != nullptr);
  if (some != 0 && some != 3) return LAZY_EINVAL;
  if (some == 3 && weights_out == weights) return LAZY_EINVAL;  // other workgroups still read what one writes
  if (batch == 0 || max_kept == 0) return LAZY_OK;
  if (!k_pool || !v_pool || !chunks || !chunk_start || !kept || !kept_start || !dst || !k_out || !v_out)
    return LAZY_EINVAL;
  if (batch > 65535 || p->num_kv_heads > 65535 || max_kept > kMaxGroups) return LAZY_EUNSUPPORTED;
  lazy::CompactArgs a = {};
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.v_pool = static_cast<const uint16_t*>(v_pool);
  a.chunks = chunks;
  a.chunk_start = chunk_start;
  a.kept = kept;
  a.kept_start = kept_start;
  a.dst = dst;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.key_start = key_start;
  a.weights = weights;
  a.weights_out = weights_out;
  a.inv_freq = p->inv_freq;
  a.hkv = p->num_kv_heads;
  lazy::rope_revolutions(p, a.rev);
  const bool local = p->key_positions == LAZY_KEYS_LOCAL;
  return status(lazy::launch_compact(a, p->head_dim, batch, max_kept, rotate ? 1 : local ? 2 : 0, local,
                                     p->rope_style == LAZY_ROPE_INTERLEAVED, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
