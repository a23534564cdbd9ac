// Shared declarations of the rotating cache append and of attention with shaped scores over the paged cache.
#pragma once

#include "common.cuh"
#include "tma_ptx.cuh"

namespace pda {

// Scores are carried in the base-2 exponent: z = log2(e) * score. A cap C = log2(e) * softcap makes it C tanh(z / C).
struct ScoreParams {
  float mul;            // log2(e) * scale: multiplies q.k and gives z, before any cap
  float cap;            // C, 0: no cap
  float rate;           // 2 log2(e) / C, the largest 32-bit number if that is beyond it
  const float* slopes;  // nullptr: no bias
  int32_t window;       // 0: none
};
constexpr float kLog2e = 1.4426950408889634f;

// tanh(x) / x for |x| <= 3/4 in powers of x^2, the polynomial of this degree whose largest relative error is least (2.9e-8, by
// linear programming over 4000 points).
constexpr float kTanhReach = 0.75f;
#define PDA_TANH_COEFFICIENTS \
  {0.9999999710136436f, -0.3333295887857063f, 0.13325406008671778f, -0.05334442977807218f, 0.019582907537387773f, -0.004716256828599296f}

__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Polynomials and other forms of the cap whose error is relative to C are for C up to this one (a cap of 128): 5.3e-6 C is 2^-10 of an
// exponent here, a quarter of a weight's rounding to bf16.
constexpr float kAbsoluteCap = 184.f;

// The cap on a score z: C - 2 C / (2^y + 1), y = 2 log2(e) z / C, whose error is a few 2^-23 C. Above kAbsoluteCap scores may be far below
// the cap (which may be 10^8 times as large): there by the polynomial, whose error goes with the score, and only scores of 0.63 C and
// more the first way. NaN stays, infinities give +-C. (All by the polynomial, decoding 64 sequences of 512..4096: 105 us instead of 103.)
__device__ __forceinline__ float cap_score(float z, float cap, float rate) {
  constexpr float c[6] = PDA_TANH_COEFFICIENTS;
  const float y = z * rate;
  if (cap > kAbsoluteCap) {
    const float x = y * (0.5f / kLog2e);
    if (fabsf(x) <= kTanhReach) {
      const float t = x * x;
      float r = fmaf(t, c[5], c[4]);
#pragma unroll
      for (int i = 3; i >= 0; --i) r = fmaf(t, r, c[i]);
      return z * r;
    }
  }
  return fmaf(-cap, 2.f * rcp_approx(ex2(y) + 1.f), cap);  // (2 C may be beyond 32 bits)
}

// Packed ragged queries (cu_q) or one query per sequence (cu_q == nullptr) over the paged cache.
struct PrefillParams {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* cu_q;
  const int32_t* prefix_lens;  // may be nullptr
  const int32_t* first_keys;   // may be nullptr
  int32_t* status;
  void* workspace;             // may be nullptr
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
  CacheGeom geom;
  ScoreParams score;
  int32_t block_table_stride, batch, num_q_heads, group, max_q, total_q;
};

// What sequence b asks for: its query tokens q0 .. q0 + nq - 1 are the last of its L tokens. A sequence whose ranges do
// not fit is reported and has no keys; of its rows, those that lie in the array (up to max_q) are zeroed.
constexpr int32_t kMaxTokens = 1 << 30;  // of a sequence with packed queries: keys are counted in 32 bits from anywhere
struct SeqSpan {
  int32_t q0, nq, L;
};
__device__ __forceinline__ SeqSpan seq_span(const PrefillParams& p, int b) {
  const int L = max(p.seq_lens[b], 0);
  const bool fits = static_cast<int64_t>(L) <= static_cast<int64_t>(p.block_table_stride) * kPageSize && (L <= kMaxTokens || p.cu_q == nullptr);
  if (p.cu_q == nullptr) {
    if (!fits) report(p.status, PDA_DEV_BAD_SEQ_LEN);
    return {b, 1, fits ? L : 0};
  }
  const int q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
  if (q0 >= 0 && q1 >= q0 && q1 <= p.total_q && q1 - q0 <= p.max_q) {
    if (!fits && q1 > q0) report(p.status, PDA_DEV_BAD_SEQ_LEN);
    return {q0, q1 - q0, fits ? L : 0};
  }
  report(p.status, PDA_DEV_BAD_SEQ_LEN);
  if (q0 < 0 || q1 <= q0 || q0 >= p.total_q) return {0, 0, 0};
  return {q0, min(min(q1, p.total_q) - q0, p.max_q), 0};
}
// Keys lo <= j < hi that the token at position pos of a sequence of L tokens sees; first and prefix: its first_keys and
// prefix_lens entries (0 without). Nothing for pos < 0.
__device__ __forceinline__ void visible_keys(int pos, int L, int window, int first, int prefix, int& lo, int& hi) {
  hi = pos < 0 ? 0 : max(pos + 1, min(prefix, L));
  lo = max(max(first, 0), window > 0 ? pos - window + 1 : 0);
}

struct RopeAppendParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  __nv_bfloat16* q_out;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  const int32_t* positions;
  const float* cos_sin;
  const __nv_bfloat16* q_norm;  // nullptr: no norm
  const __nv_bfloat16* k_norm;
  const int32_t* slot_map;
  int32_t* status;
  int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride, qo_token_stride,
      qo_head_stride, positions_stride;
  CacheGeom geom;
  float eps, inv_dim;  // 1 / head_dim
  int32_t n_tokens, num_q_heads, table_len, rot_dim, axes_used;  // axes_used: bit a for axis a
  alignas(4) uint8_t freq_axis[128];
};

cudaError_t launch_rope_append(const RopeAppendParams& p, bool interleaved, cudaStream_t stream);
cudaError_t launch_prefill_generic(const PrefillParams& p, cudaStream_t stream);
bool prefill_tc_supports(const PrefillParams& p);  // tcgen05 kernel
cudaError_t launch_prefill_tc(const PrefillParams& p, cudaStream_t stream);
int64_t prefill_workspace_bytes(int head_dim);
// Decode attention with shaped scores on the TMA kernel (attention_tma.cu); first_keys may be nullptr.
bool biased_decode_tma_supports(const AttnParams& p);
cudaError_t launch_biased_decode_tma(const StepParams& sp, const ScoreParams& score, const int32_t* first_keys, cudaStream_t stream);

}  // namespace pda
