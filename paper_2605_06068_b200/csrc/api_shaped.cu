// C ABI of the rotating cache append and of attention with shaped scores: argument validation on the host, then dispatch.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "api_checks.cuh"
#include "shaped.cuh"

namespace {

using pda::aligned16;
using pda::CacheGeom;

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// Element strides of bf16 rows that are read 16 bytes at a time.
inline int check_stride(int64_t s) { return s < 0 ? PDA_ERR_INVALID_ARG : s % 8 ? PDA_ERR_MISALIGNED : PDA_OK; }

int check_score(const pda_score_desc* d, pda::ScoreParams* s) {
  if (!d || !std::isfinite(d->scale) || !std::isfinite(d->softcap) || d->softcap < 0.f || d->window < 0) return PDA_ERR_INVALID_ARG;
  if (!aligned4(d->slopes)) return PDA_ERR_MISALIGNED;
  const double log2e = 1.4426950408889634;
  s->mul = static_cast<float>(log2e * d->scale);
  s->cap = static_cast<float>(log2e * d->softcap);
  s->rate = 0.f;
  if (!std::isfinite(s->mul) || !std::isfinite(s->cap)) return PDA_ERR_INVALID_ARG;
  if (d->softcap > 0.f) {
    if (!std::isfinite(static_cast<float>(2.0 * log2e * d->scale / d->softcap))) return PDA_ERR_INVALID_ARG;
    s->rate = static_cast<float>(std::min(2.0 / d->softcap, static_cast<double>(FLT_MAX)));
  }
  s->slopes = d->slopes;
  s->window = d->window;
  return PDA_OK;
}

}  // namespace

extern "C" {

int rope_kv_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                   int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
                   const int32_t* positions, int64_t positions_stride, int32_t num_axes, const uint8_t* freq_axis,
                   const float* cos_sin, int32_t table_len, int32_t rot_dim, int32_t interleaved, const void* q_norm,
                   const void* k_norm, float eps, const int32_t* slot_map, int32_t n_tokens, int32_t num_q_heads, void* q_out,
                   int64_t qo_token_stride, int64_t qo_head_stride, void* k_cache, void* v_cache, const pda_cache_desc* desc,
                   float* k_scale, float* v_scale, int32_t* status, pda_stream_t stream) {
  CacheGeom g;
  if (int rc = pda::check_desc(desc, &g)) return rc;
  if (n_tokens < 0 || num_q_heads <= 0 || rot_dim < 0 || rot_dim > g.head_dim || table_len < 0 || num_axes < 1 || !(eps >= 0.f) ||
      std::isinf(eps))
    return PDA_ERR_INVALID_ARG;
  if (rot_dim % 16 || num_axes > 4) return PDA_ERR_UNSUPPORTED;
  const bool fp8 = g.dtype == PDA_FP8_E4M3;
  const int64_t heads = static_cast<int64_t>(num_q_heads) + 2ll * g.num_kv_heads;
  if (heads > 65535 || heads * n_tokens > INT32_MAX) return PDA_ERR_TOO_LARGE;
  if (n_tokens == 0) return PDA_OK;
  if (!q || !k || !v || !q_out || !slot_map || (g.num_pages > 0 && (!k_cache || !v_cache)) || (fp8 && (!k_scale || !v_scale)))
    return PDA_ERR_INVALID_ARG;
  if (rot_dim > 0 && (!positions || !cos_sin)) return PDA_ERR_INVALID_ARG;
  if (num_axes > 1 && rot_dim > 0 && positions_stride < n_tokens) return PDA_ERR_INVALID_ARG;
  const int64_t strides[] = {q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride, qo_token_stride, qo_head_stride};
  for (int64_t s : strides)
    if (int rc = check_stride(s)) return rc;
  // (rows of a token are found by 32-bit strides)
  if (q_head_stride > INT32_MAX || k_head_stride > INT32_MAX || v_head_stride > INT32_MAX || qo_head_stride > INT32_MAX || g.head_stride > INT32_MAX)
    return PDA_ERR_TOO_LARGE;
  const void* rows[] = {q, k, v, q_out, k_cache, v_cache, q_norm, k_norm, rot_dim > 0 ? cos_sin : nullptr};
  for (const void* r : rows)
    if (!aligned16(r)) return PDA_ERR_MISALIGNED;
  if (!aligned4(positions) || !aligned4(slot_map) || !aligned4(k_scale) || !aligned4(v_scale) || !aligned4(status)) return PDA_ERR_MISALIGNED;
  pda::RopeAppendParams p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.positions = positions;
  p.cos_sin = cos_sin;
  p.q_norm = static_cast<const __nv_bfloat16*>(q_norm);
  p.k_norm = static_cast<const __nv_bfloat16*>(k_norm);
  p.slot_map = slot_map;
  p.status = status;
  p.q_token_stride = q_token_stride;
  p.q_head_stride = q_head_stride;
  p.k_token_stride = k_token_stride;
  p.k_head_stride = k_head_stride;
  p.v_token_stride = v_token_stride;
  p.v_head_stride = v_head_stride;
  p.qo_token_stride = qo_token_stride;
  p.qo_head_stride = qo_head_stride;
  p.positions_stride = positions_stride;
  p.geom = g;
  p.eps = eps;
  p.inv_dim = 1.f / static_cast<float>(g.head_dim);
  p.n_tokens = n_tokens;
  p.num_q_heads = num_q_heads;
  p.table_len = table_len;
  p.rot_dim = rot_dim;
  p.axes_used = 0;
  for (int f = 0; f < rot_dim / 2; ++f) {
    const int a = freq_axis ? freq_axis[f] : 0;
    if (a >= num_axes) return PDA_ERR_INVALID_ARG;
    p.freq_axis[f] = static_cast<uint8_t>(a);
    p.axes_used |= 1 << a;
  }
  return static_cast<int>(pda::launch_rope_append(p, interleaved != 0, static_cast<cudaStream_t>(stream)));
}

int64_t pda_prefill_workspace_bytes(int32_t num_q_heads, int32_t head_dim) {
  if (num_q_heads <= 0 || head_dim <= 0 || head_dim % 32 || head_dim > 256) return PDA_ERR_INVALID_ARG;
  return pda::prefill_workspace_bytes(head_dim);
}

int paged_prefill_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k_cache, const void* v_cache,
                            const pda_cache_desc* desc, const float* k_scale, const float* v_scale, const int32_t* block_table,
                            int32_t block_table_stride, const int32_t* seq_lens, const int32_t* cu_q, int32_t batch,
                            int32_t num_q_heads, int32_t max_q, int32_t total_q, const pda_score_desc* score,
                            const int32_t* prefix_lens, const int32_t* first_keys, void* out, int64_t out_token_stride,
                            int64_t out_head_stride, void* workspace, int64_t workspace_bytes, uint32_t flags, int32_t* status,
                            pda_stream_t stream) {
  CacheGeom g;
  if (int rc = pda::check_desc(desc, &g)) return rc;
  pda::PrefillParams p{};
  if (int rc = check_score(score, &p.score)) return rc;
  if (batch < 0 || num_q_heads <= 0 || block_table_stride < 0 || max_q < 0 || total_q < 0 || num_q_heads % g.num_kv_heads)
    return PDA_ERR_INVALID_ARG;
  if (flags & ~PDA_FLAG_FORCE_GENERIC) return PDA_ERR_INVALID_ARG;
  if (max_q > total_q) max_q = total_q;  // (no sequence has more)
  if (batch > 65535 || num_q_heads > 65535 || static_cast<int64_t>(max_q) * num_q_heads > INT32_MAX) return PDA_ERR_TOO_LARGE;
  if (batch == 0 || max_q == 0) return PDA_OK;
  if (!q || !out || !seq_lens || !cu_q || !block_table || block_table_stride == 0) return PDA_ERR_INVALID_ARG;
  if (g.num_pages > 0 && (!k_cache || !v_cache)) return PDA_ERR_INVALID_ARG;
  if (g.dtype == PDA_FP8_E4M3 && g.num_pages > 0 && (!k_scale || !v_scale)) return PDA_ERR_INVALID_ARG;
  const int64_t strides[] = {q_token_stride, q_head_stride, out_token_stride, out_head_stride};
  for (int64_t s : strides)
    if (int rc = check_stride(s)) return rc;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return PDA_ERR_MISALIGNED;
  const void* words[] = {k_scale, v_scale, block_table, seq_lens, cu_q, prefix_lens, first_keys, status};
  for (const void* w : words)
    if (!aligned4(w)) return PDA_ERR_MISALIGNED;
  if (workspace && workspace_bytes < pda::prefill_workspace_bytes(g.head_dim)) return PDA_ERR_INVALID_ARG;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.cu_q = cu_q;
  p.prefix_lens = prefix_lens;
  p.first_keys = first_keys;
  p.status = status;
  p.workspace = workspace;
  p.q_token_stride = q_token_stride;
  p.q_head_stride = q_head_stride;
  p.out_token_stride = out_token_stride;
  p.out_head_stride = out_head_stride;
  p.geom = g;
  p.block_table_stride = block_table_stride;
  p.batch = batch;
  p.num_q_heads = num_q_heads;
  p.group = num_q_heads / g.num_kv_heads;
  p.max_q = max_q;
  p.total_q = total_q;
  if (!(flags & PDA_FLAG_FORCE_GENERIC) && pda::prefill_tc_supports(p))
    return static_cast<int>(pda::launch_prefill_tc(p, static_cast<cudaStream_t>(stream)));
  return static_cast<int>(pda::launch_prefill_generic(p, static_cast<cudaStream_t>(stream)));
}

int paged_biased_decode_attention(const void* q, const void* k_cache, const void* v_cache, const pda_cache_desc* desc,
                                  const float* k_scale, const float* v_scale, const int32_t* block_table,
                                  int32_t block_table_stride, const int32_t* seq_lens, int32_t batch, int32_t num_q_heads,
                                  const pda_score_desc* score, const int32_t* first_keys, int32_t chunk_tokens, void* out,
                                  float* part_o, float* part_lse, int32_t max_chunks, int32_t* workspace, uint32_t flags,
                                  int32_t* status, pda_stream_t stream) {
  pda::ScoreParams sc;
  if (int rc = check_score(score, &sc)) return rc;
  if (flags & ~PDA_FLAG_FORCE_GENERIC) return PDA_ERR_INVALID_ARG;
  pda::AttnParams a;
  if (int rc = pda::check_attention(q, k_cache, v_cache, desc, k_scale, v_scale, block_table, block_table_stride, seq_lens, batch,
                                    num_q_heads, chunk_tokens, out, part_o, part_lse, max_chunks, &a))
    return rc;
  if (batch == 0) return PDA_OK;
  if (!out) return PDA_ERR_INVALID_ARG;
  if (!aligned16(out)) return PDA_ERR_MISALIGNED;
  const void* words[] = {k_scale, v_scale, block_table, seq_lens, first_keys, part_lse, workspace, status};
  for (const void* w : words)
    if (!aligned4(w)) return PDA_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!(flags & PDA_FLAG_FORCE_GENERIC) && pda::biased_decode_tma_supports(a)) {
    a.status = status;
    a.window = sc.window;
    const bool merge_here = chunk_tokens > 0 && workspace == nullptr;
    pda::StepParams sp{a, nullptr, nullptr, nullptr, nullptr, workspace, merge_here ? 0 : 1};
    if (cudaError_t e = pda::launch_biased_decode_tma(sp, sc, first_keys, s)) return static_cast<int>(e);
    if (!merge_here) return PDA_OK;
    return static_cast<int>(pda::launch_reduce(part_o, part_lse, seq_lens, batch, num_q_heads, a.geom.head_dim, chunk_tokens,
                                               max_chunks, 0, 0, 1, static_cast<__nv_bfloat16*>(out), s));
  }
  pda::PrefillParams p{};
  p.q = a.q;
  p.out = a.out;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.first_keys = first_keys;
  p.status = status;
  p.q_token_stride = p.out_token_stride = static_cast<int64_t>(num_q_heads) * a.geom.head_dim;
  p.q_head_stride = p.out_head_stride = a.geom.head_dim;
  p.geom = a.geom;
  p.score = sc;
  p.block_table_stride = block_table_stride;
  p.batch = batch;
  p.num_q_heads = num_q_heads;
  p.group = a.group;
  p.max_q = 1;
  p.total_q = batch;
  return static_cast<int>(pda::launch_prefill_generic(p, s));
}

}  // extern "C"
