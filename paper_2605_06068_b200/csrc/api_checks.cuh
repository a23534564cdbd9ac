// Argument checks shared by the entry points over the paged key/value cache.
#pragma once

#include <cstdint>

#include "common.cuh"

namespace pda {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Checks the cache descriptor; on success fills `g`.
inline int check_desc(const pda_cache_desc* d, CacheGeom* g) {
  if (d == nullptr) return PDA_ERR_INVALID_ARG;
  if (d->num_pages < 0 || d->num_kv_heads <= 0 || d->head_dim <= 0 || d->page_size <= 0)
    return PDA_ERR_INVALID_ARG;
  if (d->dtype != PDA_BF16 && d->dtype != PDA_FP8_E4M3) return PDA_ERR_UNSUPPORTED;
  if (d->page_size != kPageSize) return PDA_ERR_UNSUPPORTED;
  if (d->head_dim % 32 != 0 || d->head_dim > 256) return PDA_ERR_UNSUPPORTED;
  if (d->page_stride <= 0 || d->head_stride <= 0 || d->slot_stride < d->head_dim)
    return PDA_ERR_INVALID_ARG;
  const int64_t eb = d->dtype == PDA_BF16 ? 2 : 1;
  if ((d->page_stride * eb) % 16 || (d->head_stride * eb) % 16 || (d->slot_stride * eb) % 16)
    return PDA_ERR_MISALIGNED;
  g->page_stride = d->page_stride;
  g->head_stride = d->head_stride;
  g->slot_stride = d->slot_stride;
  g->num_pages = d->num_pages;
  g->num_kv_heads = d->num_kv_heads;
  g->head_dim = d->head_dim;
  g->dtype = d->dtype;
  return PDA_OK;
}

inline int check_attention(const void* q, const void* k_cache, const void* v_cache,
                    const pda_cache_desc* desc, const float* k_scale, const float* v_scale,
                    const int32_t* block_table, int32_t block_table_stride,
                    const int32_t* seq_lens, int32_t batch, int32_t num_q_heads,
                    int32_t chunk_tokens, void* out, float* part_o, float* part_lse,
                    int32_t max_chunks, AttnParams* p) {
  CacheGeom g;
  if (int rc = check_desc(desc, &g)) return rc;
  if (batch < 0 || num_q_heads <= 0 || block_table_stride < 0 || chunk_tokens < 0)
    return PDA_ERR_INVALID_ARG;
  if (num_q_heads % g.num_kv_heads != 0) return PDA_ERR_INVALID_ARG;
  if (chunk_tokens % kPageSize != 0) return PDA_ERR_INVALID_ARG;
  if (batch > 65535 || num_q_heads > 65535) return PDA_ERR_TOO_LARGE;
  if (batch > 0) {
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens) return PDA_ERR_INVALID_ARG;
    if (block_table_stride == 0) return PDA_ERR_INVALID_ARG;
    if (g.dtype == PDA_FP8_E4M3 && (!k_scale || !v_scale)) return PDA_ERR_INVALID_ARG;
    if (chunk_tokens == 0) {
      if (!out) return PDA_ERR_INVALID_ARG;
    } else {
      if (!part_o || !part_lse || max_chunks <= 0) return PDA_ERR_INVALID_ARG;
    }
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) ||
        (chunk_tokens == 0 && !aligned16(out)) || (chunk_tokens > 0 && !aligned16(part_o)))
      return PDA_ERR_MISALIGNED;
  }
  p->q = static_cast<const __nv_bfloat16*>(q);
  p->k_cache = k_cache;
  p->v_cache = v_cache;
  p->k_scale = k_scale;
  p->v_scale = v_scale;
  p->block_table = block_table;
  p->seq_lens = seq_lens;
  p->out = static_cast<__nv_bfloat16*>(out);
  p->part_o = part_o;
  p->part_lse = part_lse;
  p->status = nullptr;
  p->geom = g;
  p->block_table_stride = block_table_stride;
  p->batch = batch;
  p->num_q_heads = num_q_heads;
  p->group = num_q_heads / g.num_kv_heads;
  p->chunk_tokens = chunk_tokens;
  p->max_chunks = max_chunks;
  p->scale = 0.f;
  p->window = 0;
  p->first_token = 0;
  p->chunk_slot0 = 0;
  return PDA_OK;
}

}  // namespace pda
