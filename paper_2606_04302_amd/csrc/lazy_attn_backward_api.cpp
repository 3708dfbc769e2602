// C entry point of the backward pass: argument checks and dispatch.
#include <hip/hip_runtime_api.h>

#include "lazy_attn_internal.h"
#include "lazy_attn_params.h"

extern "C" int lazy_attn_prefill_backward(const lazy_attn_params_t* p, const void* q, const int32_t* q_start,
                                          const int32_t* q_pos0, const void* k_pool, const void* v_pool,
                                          const lazy_chunk_t* chunks, const int32_t* chunk_start, int32_t batch,
                                          int32_t total_q, const void* out, const float* lse, const void* dout,
                                          const float* dlse, const void* plan, const lazy_backward_info_t* info,
                                          void* dq, void* dk_pool, void* dv_pool, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  const int e = lazy::check_params(p);
  if (e != LAZY_OK) return e;
  if (!info || batch < 0 || total_q < 0) return LAZY_EINVAL;
  if (info->batch != batch || info->total_q != total_q || info->num_q_heads != p->num_q_heads ||
      info->num_kv_heads != p->num_kv_heads || info->head_dim != p->head_dim || info->causal != p->causal ||
      info->key_positions != p->key_positions)
    return LAZY_EINVAL;
  const lazy::GradPlanLayout at(*info);
  if (info->plan_bytes != (int64_t)at.bytes) return LAZY_EINVAL;
  if (at.bytes == 0) return LAZY_OK;  // no query and no key
  if (!q_start || !q_pos0 || !chunk_start || !plan || ((uintptr_t)plan & 15u)) return LAZY_EINVAL;
  if (total_q > 0 && (!q || !out || !lse || !dout || !dq)) return LAZY_EINVAL;
  if (info->num_tiles > 0 && (!k_pool || !v_pool || !chunks || !dk_pool || !dv_pool)) return LAZY_EINVAL;
  const lazy::GradWorkLayout ws(p->num_q_heads, p->num_kv_heads, p->head_dim, lazy::query_parts(p), *info);
  if (ws.bytes > 0 && (!workspace || workspace_bytes < ws.bytes || ((uintptr_t)workspace & 15u)))
    return LAZY_EWORKSPACE;
  // The keys and values are read again after the first gradients are written.
  if (info->num_tiles > 0 && (dk_pool == k_pool || dk_pool == v_pool || dv_pool == k_pool || dv_pool == v_pool))
    return LAZY_EINVAL;

  const char* base = static_cast<const char*>(plan);
  char* work = static_cast<char*>(workspace);
  lazy::GradArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.q_start = q_start;
  a.q_pos0 = q_pos0;
  a.k_pool = static_cast<const uint16_t*>(k_pool);
  a.v_pool = static_cast<const uint16_t*>(v_pool);
  a.chunks = chunks;
  a.chunk_start = chunk_start;
  a.out = static_cast<const uint16_t*>(out);
  a.lse = lse;
  a.dout = static_cast<const uint16_t*>(dout);
  a.dlse = dlse;
  a.blocks = reinterpret_cast<const lazy::GradBlock*>(base + at.blocks);
  a.row_items = reinterpret_cast<const lazy::GradRowItem*>(base + at.rows);
  a.segs = reinterpret_cast<const lazy::GradSeg*>(base + at.segs);
  a.tiles = reinterpret_cast<const lazy::GradTile*>(base + at.tiles);
  a.merges = reinterpret_cast<const lazy::GradMerge*>(base + at.merges);
  a.dq = static_cast<uint16_t*>(dq);
  a.dk_pool = static_cast<uint16_t*>(dk_pool);
  a.dv_pool = static_cast<uint16_t*>(dv_pool);
  a.ws_q = reinterpret_cast<uint16_t*>(work + ws.q);
  a.ws_do = reinterpret_cast<uint16_t*>(work + ws.dout);
  a.ws_info = reinterpret_cast<float*>(work + ws.info);
  a.ws_dq = reinterpret_cast<float*>(work + ws.dq);
  a.ws_parts = reinterpret_cast<float*>(work + ws.parts);
  a.inv_freq = p->inv_freq;
  a.hq = p->num_q_heads;
  a.hkv = p->num_kv_heads;
  a.group = a.hq / a.hkv;
  a.rows = (int64_t)total_q * a.group;
  a.group_magic = a.group == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
  a.causal = p->causal;
  a.rotate_q = !p->q_prerotated && p->rope_style != LAZY_ALIBI;
  a.parts = lazy::query_parts(p);
  a.lse_scale = p->rope_style == LAZY_ALIBI ? 1.f : 1.4426950408889634f;
  lazy::rope_revolutions(p, a.rev);
  a.scale_log2 = lazy::scale_log2(p);
  const hipError_t err =
      lazy::launch_backward(a, p->head_dim, p->key_positions == LAZY_KEYS_LOCAL,
                            p->rope_style == LAZY_ROPE_INTERLEAVED, p->rope_style == LAZY_ALIBI, *info,
                            static_cast<hipStream_t>(stream));
  return err == hipSuccess ? LAZY_OK : LAZY_EHIP;
}
