// Attention with shaped scores on CUDA cores: any group size, any head_dim that is a multiple of 32 up to 256, any
// strides, bf16 or e4m3. One warp per (query token, query head); prompts and single tokens alike. It is the simple path for
// shapes outside the tensor-core kernels and the in-library cross-check for them.
//
// Per tile of 32 keys: lane j scores key j (32-bit sum over head_dim, 16-byte loads), the warp takes maximum and sum by
// shuffles, then each lane accumulates its own head_dim / 32 output columns over the tile's keys.
#include <cfloat>

#include "shaped.cuh"

namespace pda {

namespace {

constexpr int kMaxDPerLane = 8;  // head_dim <= 256

template <bool kFp8>
__device__ __forceinline__ float value_at(const void* base, int64_t idx) {
  if (kFp8) return e4m3_to_float(static_cast<const uint8_t*>(base)[idx]);
  return bf16_bits_to_float(static_cast<const uint16_t*>(base)[idx]);
}

template <bool kFp8>
__global__ void __launch_bounds__(32) prefill_generic_kernel(const __grid_constant__ PrefillParams p) {
  const int lane = threadIdx.x, t = blockIdx.x, h = blockIdx.y;
  const int D = p.geom.head_dim, g = h / p.group;
  // the token's sequence: the last one that starts at or before it
  int b = t;
  if (p.cu_q != nullptr) {
    int lo = 0, hi = p.batch;  // cu_q[lo] <= t < cu_q[hi], where there is such a sequence
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.cu_q[mid] <= t) lo = mid; else hi = mid;
    }
    b = lo;
  }
  const SeqSpan sp = seq_span(p, b);
  if (t < sp.q0 || t - sp.q0 >= sp.nq) return;
  const int L = sp.L, pos = L - sp.nq + (t - sp.q0);
  int k_lo, k_hi;
  visible_keys(pos, L, p.score.window, p.first_keys != nullptr ? p.first_keys[t] : 0, p.prefix_lens != nullptr ? p.prefix_lens[b] : 0,
               k_lo, k_hi);

  __shared__ float q_s[256];
  const __nv_bfloat16* q = p.q + t * p.q_token_stride + h * p.q_head_stride;
  for (int d = lane; d < D; d += 32) q_s[d] = __bfloat162float(q[d]);
  __syncwarp();

  const float slope = p.score.slopes != nullptr ? p.score.slopes[h] * kLog2e : 0.f;
  float m = -FLT_MAX, l = 0.f;
  float acc[kMaxDPerLane];
#pragma unroll
  for (int i = 0; i < kMaxDPerLane; ++i) acc[i] = 0.f;
  bool bad_page = false;
  const int32_t* table = p.block_table + static_cast<int64_t>(b) * p.block_table_stride;

  for (int64_t base = k_lo; base < k_hi; base += 32) {
    const int j = static_cast<int>(min(base + lane, static_cast<int64_t>(k_hi)));
    const bool valid = j < k_hi;
    int page = 0;
    if (valid) {
      page = table[j / kPageSize];
      bad_page = page < 0 || page >= p.geom.num_pages;
    }
    if (__any_sync(0xffffffffu, bad_page)) {
      bad_page = true;
      break;
    }
    const int64_t row = page * p.geom.page_stride + g * p.geom.head_stride + (j % kPageSize) * p.geom.slot_stride;
    float z = -INFINITY;
    if (valid) {
      float dot = 0.f;
      constexpr int kVec = kFp8 ? 16 : 8;
      const uint4* k = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.k_cache) + row * (kFp8 ? 1 : 2));
      for (int c = 0; c < D / kVec; ++c) {
        const uint4 u = k[c];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (kFp8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) dot = fmaf(q_s[16 * c + 4 * e + i], e4m3_to_float(static_cast<uint8_t>(w[e] >> (8 * i))), dot);
          } else {
            dot = fmaf(q_s[8 * c + 2 * e], __uint_as_float(w[e] << 16), dot);
            dot = fmaf(q_s[8 * c + 2 * e + 1], __uint_as_float(w[e] & 0xffff0000u), dot);
          }
        }
      }
      if (kFp8) dot *= p.k_scale[static_cast<int64_t>(page) * p.geom.num_kv_heads + g];
      z = dot * p.score.mul;
      if (p.score.cap > 0.f) z = cap_score(z, p.score.cap, p.score.rate);
      z = fmaf(-slope, static_cast<float>(abs(pos - j)), z);
    }
    float top = z;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float m_new = fmaxf(m, top);
    const float alpha = exp2f(m - m_new);
    float w = exp2f(z - m_new);  // (zero for keys behind the last)
    float sum = w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l = l * alpha + sum;
    m = m_new;
    if (kFp8 && valid) w *= p.v_scale[static_cast<int64_t>(page) * p.geom.num_kv_heads + g];
#pragma unroll
    for (int i = 0; i < kMaxDPerLane; ++i) acc[i] *= alpha;
    const int n = static_cast<int>(min(static_cast<int64_t>(32), k_hi - base));
    for (int k = 0; k < n; ++k) {
      const float wk = __shfl_sync(0xffffffffu, w, k);
      const int64_t rk = __shfl_sync(0xffffffffu, row, k);
#pragma unroll
      for (int i = 0; i < kMaxDPerLane; ++i) {
        const int d = lane + 32 * i;
        if (d < D) acc[i] = fmaf(wk, value_at<kFp8>(p.v_cache, rk + d), acc[i]);
      }
    }
  }
  if (bad_page && lane == 0) report(p.status, PDA_DEV_BAD_PAGE);
  const float inv = l == 0.f || bad_page ? 0.f : 1.f / l;
  __nv_bfloat16* out = p.out + t * p.out_token_stride + h * p.out_head_stride;
#pragma unroll
  for (int i = 0; i < kMaxDPerLane; ++i) {
    const int d = lane + 32 * i;
    if (d < D) out[d] = __float2bfloat16_rn(bad_page ? 0.f : acc[i] * inv);
  }
}

}  // namespace

cudaError_t launch_prefill_generic(const PrefillParams& p, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.cu_q != nullptr ? p.total_q : p.batch), static_cast<unsigned>(p.num_q_heads));
  if (p.geom.dtype == PDA_FP8_E4M3) prefill_generic_kernel<true><<<grid, 32, 0, stream>>>(p);
  else prefill_generic_kernel<false><<<grid, 32, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace pda
