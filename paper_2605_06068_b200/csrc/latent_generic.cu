// The plain kernels of the two latent-attention forms, for shapes outside the tensor-core kernels: one CTA
// per query row, scores by a warp per token, the running maximum and sum of the softmax over blocks of
// tokens, everything in 32 bits. Bound by reading every key and value once per query row: 2048-token prompt, 16 heads, dims
// 64/32/64 13.3 ms; 64 x 2304 cached tokens, 16 heads, 512 + 64, pages of 8 2.2 ms.
#include <cfloat>

#include "latent.cuh"

namespace pda {

namespace {

constexpr int kGenThreads = 128;
constexpr int kGenBlock = 64;     // tokens per softmax step
constexpr int kGenMaxDims = 8;    // output elements per thread: up to 1024

__device__ __forceinline__ float block_reduce(float x, bool is_max, float* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, x, o);
    x = is_max ? fmaxf(x, y) : x + y;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sh[0];
  for (int w = 1; w < kGenThreads / 32; ++w) x = is_max ? fmaxf(x, sh[w]) : x + sh[w];
  return x;
}

// Attention of one query row over tokens [0, n): key_a(j) has da elements, key_b(j) db more, val(j) dv.
// q_sh holds da + db floats. Writes dv bf16 to out.
template <class KeyA, class KeyB, class Val>
__device__ __forceinline__ void attend_row(const float* q_sh, int da, int db, int dv, int n, float scale, KeyA key_a,
                                           KeyB key_b, Val val, __nv_bfloat16* out, float* p_sh, float* red_sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float acc[kGenMaxDims];
#pragma unroll
  for (int e = 0; e < kGenMaxDims; ++e) acc[e] = 0.f;
  // (the maximum starts at the lowest finite number, so that scores of -inf get a weight of 0 and not inf - inf)
  float m = -FLT_MAX, l = 0.f;
  for (int j0 = 0, nb; j0 < n; j0 += nb) {  // (n goes up to 2^31 - 1, and j0 no further)
    nb = min(kGenBlock, n - j0);
    __syncthreads();
    for (int j = warp; j < nb; j += kGenThreads / 32) {
      const __nv_bfloat16* ka = key_a(j0 + j);
      const __nv_bfloat16* kb = key_b(j0 + j);
      float s = 0.f;
      for (int d = lane; d < da; d += 32) s = fmaf(q_sh[d], __bfloat162float(ka[d]), s);
      for (int d = lane; d < db; d += 32) s = fmaf(q_sh[da + d], __bfloat162float(kb[d]), s);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) p_sh[j] = s * scale;
    }
    __syncthreads();
    const float bm = block_reduce(tid < nb ? p_sh[tid] : -INFINITY, true, red_sh);
    const float m_new = fmaxf(m, bm);
    const float keep = expf(m - m_new);
    const float w = tid < nb ? expf(p_sh[tid] - m_new) : 0.f;
    l = l * keep + block_reduce(w, false, red_sh);
    if (tid < nb) p_sh[tid] = w;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kGenMaxDims; ++e) acc[e] *= keep;
    for (int j = 0; j < nb; ++j) {
      const __nv_bfloat16* v = val(j0 + j);
      const float wj = p_sh[j];
#pragma unroll
      for (int e = 0; e < kGenMaxDims; ++e)
        if (tid + e * kGenThreads < dv) acc[e] = fmaf(wj, __bfloat162float(v[tid + e * kGenThreads]), acc[e]);
    }
    m = m_new;
  }
  const float inv = n > 0 ? 1.f / l : 0.f;  // (all scores -inf: 0 * inf, a NaN)
#pragma unroll
  for (int e = 0; e < kGenMaxDims; ++e)
    if (tid + e * kGenThreads < dv) out[tid + e * kGenThreads] = __float2bfloat16(n > 0 ? acc[e] * inv : 0.f);
}

__global__ void __launch_bounds__(kGenThreads) latent_generic_kernel(LatentParams p) {
  extern __shared__ float q_sh[];
  __shared__ float p_sh[kGenBlock], red_sh[kGenThreads / 32];
  const int64_t unit = blockIdx.x;
  const int h = static_cast<int>(unit % p.num_q_heads);
  const int64_t token = unit / p.num_q_heads;
  const int b = static_cast<int>(token / p.n_q), t = static_cast<int>(token % p.n_q);
  const LatentGeom g = p.geom;
  int L = max(p.seq_lens[b], 0);
  const int32_t* table = p.block_table + static_cast<int64_t>(b) * p.block_table_stride;
  if (L > static_cast<int64_t>(p.block_table_stride) * g.page_size) {
    if (threadIdx.x == 0) report(p.status, PDA_DEV_BAD_SEQ_LEN);
    L = 0;
  }
  int bad = 0;  // a bad page anywhere in the sequence zeroes all its rows
  for (int i = threadIdx.x; i < static_cast<int>((static_cast<int64_t>(L) + g.page_size - 1) / g.page_size); i += kGenThreads)
    bad |= table[i] < 0 || table[i] >= g.num_pages;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(p.status, PDA_DEV_BAD_PAGE);
    L = 0;
  }
  const int n = max(L - p.n_q + t + 1, 0) * (L > 0);
  for (int d = threadIdx.x; d < g.latent_dim + g.rope_dim; d += kGenThreads)
    q_sh[d] = __bfloat162float(d < g.latent_dim ? p.q_latent[token * p.ql_token_stride + h * p.ql_head_stride + d]
                                                : p.q_rope[token * p.qr_token_stride + h * p.qr_head_stride + d - g.latent_dim]);
  auto row = [&](int j) {
    const int page = table[j / g.page_size];
    return p.cache + page * g.page_stride + static_cast<int64_t>(j % g.page_size) * g.slot_stride;
  };
  auto rope = [&](int j) { return row(j) + g.latent_dim; };
  attend_row(q_sh, g.latent_dim, g.rope_dim, g.latent_dim, n, p.scale, row, rope, row,
             p.out + token * p.out_token_stride + h * p.out_head_stride, p_sh, red_sh);
}

__global__ void __launch_bounds__(kGenThreads) latent_prefill_generic_kernel(LatentPrefillParams p) {
  extern __shared__ float q_sh[];
  __shared__ float p_sh[kGenBlock], red_sh[kGenThreads / 32];
  // (every sequence's ranges are looked at, those without rows among them)
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * kGenThreads + threadIdx.x; b < p.batch;
       b += static_cast<int64_t>(gridDim.x) * kGenThreads)
    prefill_span(p, static_cast<int>(b));
  const int64_t units = static_cast<int64_t>(p.total_q) * p.num_heads;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t token = unit / p.num_heads;
    const int h = static_cast<int>(unit % p.num_heads);
    int b = 0;  // the last sequence that does not start behind the token
    for (int hi = p.batch; hi - b > 1;) {
      const int mid = (b + hi) >> 1;
      if (p.cu_q[mid] <= token) b = mid; else hi = mid;
    }
    const PrefillSpan sp = prefill_span(p, b);
    if (token < sp.q0 || token - sp.q0 >= sp.nq) continue;
    const int i = static_cast<int>(token - sp.q0);
    __syncthreads();  // (q_sh may still be read for the last row)
    const int n = max(sp.nk - sp.nq_all + i + 1, 0) * (sp.nk > 0);
    for (int d = threadIdx.x; d < p.nope_dim + p.rope_dim; d += kGenThreads)
      q_sh[d] = __bfloat162float(p.q[token * p.q_token_stride + h * p.q_head_stride + d]);
    const int64_t k0 = sp.k0;
    auto kn = [&](int j) { return p.k_nope + (k0 + j) * p.kn_token_stride + h * p.kn_head_stride; };
    auto kr = [&](int j) { return p.k_rope + (k0 + j) * p.kr_token_stride; };
    auto v = [&](int j) { return p.v + (k0 + j) * p.v_token_stride + h * p.v_head_stride; };
    attend_row(q_sh, p.nope_dim, p.rope_dim, p.v_dim, n, p.scale, kn, kr, v,
               p.out + token * p.out_token_stride + h * p.out_head_stride, p_sh, red_sh);
  }
}

}  // namespace

cudaError_t launch_latent_generic(const LatentParams& p, cudaStream_t stream) {
  const int64_t units = static_cast<int64_t>(p.batch) * p.n_q * p.num_q_heads;
  if (units > INT32_MAX) return cudaErrorInvalidValue;
  latent_generic_kernel<<<static_cast<unsigned>(units), kGenThreads, (p.geom.latent_dim + p.geom.rope_dim) * 4, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_latent_prefill_generic(const LatentPrefillParams& p, cudaStream_t stream) {
  const int64_t units = static_cast<int64_t>(p.total_q) * p.num_heads;
  const unsigned ctas = static_cast<unsigned>(units < INT32_MAX ? units : INT32_MAX);
  latent_prefill_generic_kernel<<<ctas, kGenThreads, (p.nope_dim + p.rope_dim) * 4, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace pda
