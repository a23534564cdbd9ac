// Shared declarations of the latent-attention operators and the step tables.
#pragma once

#include "common.cuh"

namespace pda {

// Geometry of a latent cache: row (page, slot) = [latent_dim | rope_dim] elements.
struct LatentGeom {
  int64_t page_stride, slot_stride;  // elements
  int32_t num_pages, page_size, latent_dim, rope_dim;
};

struct TablesParams {
  const int32_t* seq_lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* block_table;
  int32_t* cu_new;
  int32_t* slot_map;
  int32_t* positions;  // may be nullptr
  int32_t* status;
  int32_t batch, page_size, free_capacity, block_table_stride, capacity;
};

struct LatentAppendParams {
  const __nv_bfloat16* c_new;
  const __nv_bfloat16* rope_new;
  int64_t c_stride, rope_stride;  // elements between tokens
  __nv_bfloat16* cache;
  const __nv_bfloat16* norm_weight;  // nullptr: rows are copied as they are
  const int32_t* slot_map;
  int32_t* status;
  LatentGeom geom;
  int32_t n_tokens;
  float eps;
};

// Absorbed attention over the paged latent cache. Row r = t * num_q_heads + h of a sequence is query token
// t of its n_q, head h; token index b * n_q + t.
struct LatentParams {
  const __nv_bfloat16* q_latent;
  const __nv_bfloat16* q_rope;
  __nv_bfloat16* out;
  const __nv_bfloat16* cache;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* status;
  int64_t ql_token_stride, ql_head_stride, qr_token_stride, qr_head_stride, out_token_stride, out_head_stride;
  LatentGeom geom;
  int32_t block_table_stride, batch, num_q_heads, n_q;
  float scale;
  void* workspace;
};

// Expanded attention over packed ragged sequences.
struct LatentPrefillParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k_nope;
  const __nv_bfloat16* k_rope;
  const __nv_bfloat16* v;
  __nv_bfloat16* out;
  const int32_t* cu_q;
  const int32_t* cu_k;
  int32_t* status;
  int64_t q_token_stride, q_head_stride, kn_token_stride, kn_head_stride, kr_token_stride, v_token_stride,
      v_head_stride, out_token_stride, out_head_stride;
  int32_t batch, num_heads, nope_dim, rope_dim, v_dim, max_q, total_q, total_k;
  float scale;
};

// What sequence b asks for. A sequence whose ranges do not fit the arrays, or that has more than max_q
// query tokens, is reported and gets no keys; of its rows, those that lie in the array (up to max_q) are
// zeroed.
struct PrefillSpan {
  int32_t q0, nq, nq_all, k0, nk;
};
__device__ __forceinline__ PrefillSpan prefill_span(const LatentPrefillParams& p, int b) {
  const int q0 = p.cu_q[b], q1 = p.cu_q[b + 1], k0 = p.cu_k[b], k1 = p.cu_k[b + 1];
  if (q0 >= 0 && q1 >= q0 && q1 <= p.total_q && k0 >= 0 && k1 >= k0 && k1 <= p.total_k && q1 - q0 <= p.max_q)
    return {q0, q1 - q0, q1 - q0, k0, k1 - k0};
  report(p.status, PDA_DEV_BAD_SEQ_LEN);
  if (q0 < 0 || q1 <= q0 || q0 >= p.total_q) return {0, 0, 0, 0, 0};
  const int n = min(min(q1, p.total_q) - q0, p.max_q);
  return {q0, n, n, 0, 0};
}

// ---- workspace of paged_latent_attention: partial results of sequences that several CTAs share ----
constexpr int kLatMaxCtas = 148;   // one CTA per SM; a device with more SMs uses this many
constexpr int kLatMaxRows = 64;    // query rows per CTA
// Rows are padded to the tile a launch uses: 16, 32 or 64.
__host__ __device__ constexpr int latent_tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : kLatMaxRows; }
struct LatentWorkspace {           // byte offsets
  int64_t part_o, part_w, records, bytes;
};
__host__ __device__ inline LatentWorkspace latent_workspace_layout(int num_q_heads, int n_q, int latent_dim) {
  const int64_t rows = 2ll * kLatMaxCtas * latent_tile_rows(static_cast<int64_t>(num_q_heads) * n_q);
  LatentWorkspace w;
  w.part_o = 0;
  w.part_w = rows * latent_dim * 4;  // float2: reference and sum of the weights
  w.records = (w.part_w + rows * 8 + 255) / 256 * 256;
  w.bytes = w.records + (kLatMaxCtas * 16 + 255) / 256 * 256;
  return w;
}
inline int64_t latent_workspace_bytes(int num_q_heads, int n_q, int latent_dim) {
  return latent_workspace_layout(num_q_heads, n_q, latent_dim).bytes;
}

cudaError_t launch_build_tables(const TablesParams& p, cudaStream_t stream);
cudaError_t launch_latent_append(const LatentAppendParams& p, cudaStream_t stream);
cudaError_t launch_latent_generic(const LatentParams& p, cudaStream_t stream);
bool latent_tc_supports(const LatentParams& p);  // tcgen05 kernel
cudaError_t launch_latent_tc(const LatentParams& p, cudaStream_t stream);
cudaError_t launch_latent_prefill_generic(const LatentPrefillParams& p, cudaStream_t stream);
bool latent_prefill_tc_supports(const LatentPrefillParams& p);  // tcgen05 kernel
cudaError_t launch_latent_prefill_tc(const LatentPrefillParams& p, cudaStream_t stream);

}  // namespace pda
