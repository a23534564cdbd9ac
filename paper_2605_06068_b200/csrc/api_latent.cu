// C ABI of the step tables and the latent attention: argument validation on the host, then dispatch.
#include <cmath>
#include <cstdint>

#include "latent.cuh"

namespace {

using pda::LatentGeom;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// Element strides of bf16 rows that are read 16 bytes at a time.
inline int check_stride(int64_t s) { return s < 0 ? PDA_ERR_INVALID_ARG : s % 8 ? PDA_ERR_MISALIGNED : PDA_OK; }

int check_latent_desc(const pda_latent_desc* d, LatentGeom* g) {
  if (!d || d->num_pages < 0 || d->page_size <= 0 || d->latent_dim <= 0 || d->rope_dim < 0) return PDA_ERR_INVALID_ARG;
  if (d->dtype != PDA_BF16 || d->page_size > 1024 || d->latent_dim % 8 || d->latent_dim > 1024 || d->rope_dim % 8 ||
      d->rope_dim > 256)
    return PDA_ERR_UNSUPPORTED;
  if (d->slot_stride < d->latent_dim + d->rope_dim || d->page_stride <= 0) return PDA_ERR_INVALID_ARG;
  if (d->slot_stride % 8 || d->page_stride % 8) return PDA_ERR_MISALIGNED;
  *g = LatentGeom{d->page_stride, d->slot_stride, d->num_pages, d->page_size, d->latent_dim, d->rope_dim};
  return PDA_OK;
}

}  // namespace

extern "C" {

int paged_build_tables(const int32_t* seq_lens, const int32_t* new_lens, int32_t batch, int32_t page_size,
                       const int32_t* free_pages, int32_t free_capacity, const int32_t* free_count,
                       int32_t* free_count_out, int32_t* block_table, int32_t block_table_stride, int32_t* cu_new,
                       int32_t* slot_map, int32_t* positions, int32_t capacity, int32_t* status, pda_stream_t stream) {
  if (batch < 0 || page_size <= 0 || free_capacity < 0 || block_table_stride < 0 || capacity < 0) return PDA_ERR_INVALID_ARG;
  if (page_size > 1024) return PDA_ERR_UNSUPPORTED;
  if (!free_count || !free_count_out || !cu_new || (free_capacity > 0 && !free_pages) || (capacity > 0 && !slot_map))
    return PDA_ERR_INVALID_ARG;
  if (batch > 0 && (!seq_lens || !new_lens || (block_table_stride > 0 && !block_table))) return PDA_ERR_INVALID_ARG;
  const void* ptrs[] = {seq_lens, new_lens, free_pages, free_count, free_count_out, block_table, cu_new, slot_map, positions, status};
  for (const void* p : ptrs)
    if (!aligned4(p)) return PDA_ERR_MISALIGNED;
  pda::TablesParams p{seq_lens, new_lens, free_pages, free_count, free_count_out, block_table, cu_new, slot_map, positions,
                      status, batch, page_size, free_capacity, block_table_stride, capacity};
  return static_cast<int>(pda::launch_build_tables(p, static_cast<cudaStream_t>(stream)));
}

int latent_append(const void* c_new, int64_t c_stride, const void* rope_new, int64_t rope_stride, void* cache,
                  const pda_latent_desc* desc, const void* norm_weight, float eps, const int32_t* slot_map,
                  int32_t n_tokens, int32_t* status, pda_stream_t stream) {
  LatentGeom g;
  if (int rc = check_latent_desc(desc, &g)) return rc;
  if (n_tokens < 0 || !(eps >= 0.f) || std::isinf(eps)) return PDA_ERR_INVALID_ARG;
  if (n_tokens == 0) return PDA_OK;
  if (!c_new || !cache || !slot_map || (g.rope_dim > 0 && !rope_new)) return PDA_ERR_INVALID_ARG;
  if (int rc = check_stride(c_stride)) return rc;
  if (g.rope_dim > 0)
    if (int rc = check_stride(rope_stride)) return rc;
  if (!aligned16(c_new) || !aligned16(rope_new) || !aligned16(cache) || !aligned16(norm_weight) || !aligned4(slot_map) ||
      !aligned4(status))
    return PDA_ERR_MISALIGNED;
  pda::LatentAppendParams p{static_cast<const __nv_bfloat16*>(c_new), static_cast<const __nv_bfloat16*>(rope_new), c_stride,
                            rope_stride, static_cast<__nv_bfloat16*>(cache),
                            static_cast<const __nv_bfloat16*>(norm_weight), slot_map, status, g, n_tokens, eps};
  return static_cast<int>(pda::launch_latent_append(p, static_cast<cudaStream_t>(stream)));
}

int64_t pda_latent_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t n_query_tokens, int32_t latent_dim) {
  if (batch < 0 || num_q_heads <= 0 || n_query_tokens <= 0 || latent_dim <= 0 || latent_dim > 1024) return PDA_ERR_INVALID_ARG;
  return pda::latent_workspace_bytes(num_q_heads, n_query_tokens, latent_dim);
}

int paged_latent_attention(const void* q_latent, int64_t ql_token_stride, int64_t ql_head_stride, const void* q_rope,
                           int64_t qr_token_stride, int64_t qr_head_stride, const void* cache, const pda_latent_desc* desc,
                           const int32_t* block_table, int32_t block_table_stride, const int32_t* seq_lens, int32_t batch,
                           int32_t num_q_heads, int32_t n_query_tokens, float scale, void* out, int64_t out_token_stride,
                           int64_t out_head_stride, void* workspace, int64_t workspace_bytes, uint32_t flags,
                           int32_t* status, pda_stream_t stream) {
  LatentGeom g;
  if (int rc = check_latent_desc(desc, &g)) return rc;
  if (batch < 0 || num_q_heads <= 0 || block_table_stride < 0 || n_query_tokens <= 0 || n_query_tokens > 4096)
    return PDA_ERR_INVALID_ARG;
  if (flags & ~PDA_FLAG_FORCE_GENERIC) return PDA_ERR_INVALID_ARG;
  if (num_q_heads > 65535 || static_cast<int64_t>(batch) * n_query_tokens > 65535) return PDA_ERR_TOO_LARGE;
  if (batch == 0) return PDA_OK;
  if (!q_latent || (g.rope_dim > 0 && !q_rope) || !block_table || !seq_lens || !out || !workspace || block_table_stride == 0)
    return PDA_ERR_INVALID_ARG;
  if (!cache && g.num_pages > 0) return PDA_ERR_INVALID_ARG;
  const int64_t strides[] = {ql_token_stride, ql_head_stride, out_token_stride, out_head_stride,
                             g.rope_dim ? qr_token_stride : 0, g.rope_dim ? qr_head_stride : 0};
  for (int64_t s : strides)
    if (int rc = check_stride(s)) return rc;
  if (!aligned16(q_latent) || !aligned16(q_rope) || !aligned16(cache) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u) || !aligned4(block_table) || !aligned4(seq_lens) || !aligned4(status))
    return PDA_ERR_MISALIGNED;
  if (workspace_bytes < pda::latent_workspace_bytes(num_q_heads, n_query_tokens, g.latent_dim)) return PDA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(batch) * n_query_tokens * num_q_heads > INT32_MAX) return PDA_ERR_TOO_LARGE;
  pda::LatentParams p{static_cast<const __nv_bfloat16*>(q_latent), static_cast<const __nv_bfloat16*>(q_rope),
                      static_cast<__nv_bfloat16*>(out), static_cast<const __nv_bfloat16*>(cache), block_table, seq_lens,
                      status, ql_token_stride, ql_head_stride, qr_token_stride, qr_head_stride, out_token_stride,
                      out_head_stride, g, block_table_stride, batch, num_q_heads, n_query_tokens, scale, workspace};
  if (!(flags & PDA_FLAG_FORCE_GENERIC) && pda::latent_tc_supports(p))
    return static_cast<int>(pda::launch_latent_tc(p, static_cast<cudaStream_t>(stream)));
  return static_cast<int>(pda::launch_latent_generic(p, static_cast<cudaStream_t>(stream)));
}

int latent_prefill_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k_nope,
                             int64_t kn_token_stride, int64_t kn_head_stride, const void* k_rope, int64_t kr_token_stride,
                             const void* v, int64_t v_token_stride, int64_t v_head_stride, const int32_t* cu_q,
                             const int32_t* cu_k, int32_t batch, int32_t num_heads, int32_t nope_dim, int32_t rope_dim,
                             int32_t v_dim, int32_t max_q, int32_t total_q, int32_t total_k, float scale, void* out,
                             int64_t out_token_stride, int64_t out_head_stride, uint32_t flags, int32_t* status,
                             pda_stream_t stream) {
  if (batch < 0 || num_heads <= 0 || nope_dim <= 0 || rope_dim < 0 || v_dim <= 0 || max_q < 0 || total_q < 0 || total_k < 0)
    return PDA_ERR_INVALID_ARG;
  if (flags & ~PDA_FLAG_FORCE_GENERIC) return PDA_ERR_INVALID_ARG;
  if (max_q > total_q) max_q = total_q;  // (no sequence has more)
  if (nope_dim % 8 || nope_dim > 512 || rope_dim % 8 || rope_dim > 256 || v_dim % 8 || v_dim > 512) return PDA_ERR_UNSUPPORTED;
  if (batch > 65535 || num_heads > 65535 || static_cast<int64_t>(max_q) * num_heads > INT32_MAX) return PDA_ERR_TOO_LARGE;
  if (batch == 0 || max_q == 0 || total_q == 0) return PDA_OK;
  if (!q || !out || !cu_q || !cu_k || (total_k > 0 && (!k_nope || !v || (rope_dim > 0 && !k_rope)))) return PDA_ERR_INVALID_ARG;
  const int64_t strides[] = {q_token_stride, q_head_stride, kn_token_stride, kn_head_stride, rope_dim ? kr_token_stride : 0,
                             v_token_stride, v_head_stride, out_token_stride, out_head_stride};
  for (int64_t s : strides)
    if (int rc = check_stride(s)) return rc;
  if (!aligned16(q) || !aligned16(k_nope) || !aligned16(k_rope) || !aligned16(v) || !aligned16(out) || !aligned4(cu_q) ||
      !aligned4(cu_k) || !aligned4(status))
    return PDA_ERR_MISALIGNED;
  pda::LatentPrefillParams p{static_cast<const __nv_bfloat16*>(q), static_cast<const __nv_bfloat16*>(k_nope),
                             static_cast<const __nv_bfloat16*>(k_rope), static_cast<const __nv_bfloat16*>(v),
                             static_cast<__nv_bfloat16*>(out), cu_q, cu_k, status, q_token_stride, q_head_stride,
                             kn_token_stride, kn_head_stride, kr_token_stride, v_token_stride, v_head_stride,
                             out_token_stride, out_head_stride, batch, num_heads, nope_dim, rope_dim, v_dim, max_q, total_q,
                             total_k, scale};
  if (!(flags & PDA_FLAG_FORCE_GENERIC) && pda::latent_prefill_tc_supports(p))
    return static_cast<int>(pda::launch_latent_prefill_tc(p, static_cast<cudaStream_t>(stream)));
  return static_cast<int>(pda::launch_latent_prefill_generic(p, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
