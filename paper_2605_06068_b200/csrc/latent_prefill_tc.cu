// Expanded attention (keys [k_nope per head | k_rope shared], values per head; packed ragged sequences,
// causal from the end) on tcgen05 + TMEM, dims 128 + 64 and 128.
//
// A CTA takes 256 query rows of one head as two halves of 128 (TMEM lane = row) and walks over the keys
// 128 at a time:
//   S[w] = Q[w] . K^T    12 MMAs M128 N128 K16, Q and K in shared memory (2 lines of k_nope, 1 of k_rope:
//                        the shared part is copied from its one array, never concatenated in memory)
//   O[w] += P[w] . V     2 x 8 MMAs M128 N64 K16, P (bf16) in tensor memory over the S it came from
// S[0], S[1], O[0], O[1] fill the 512 columns. The tensor core alternates between the halves (PV of one,
// the next S of the same, then the other's), so that one half's softmax runs under the other's products:
// 1300 clocks of products per half and tile against 1024 of exponentials. That is the bound: 2 x 320 x
// 128 x 256 operations per 2600 clocks.
// K and V lines (128 keys x 128 bytes = 16 KB) go through a ring of 8 in the order in which they are used
// and freed: 3 of K(j), 2 of V(j), ...
// The softmax takes weights relative to a reference per row that is raised (and O rescaled in tensor memory)
// only when the row's maximum passes it by more than 2^8; row sums are kept by the row's thread, of the
// 32-bit weights; the rounding of the weights to bf16 is 2^-8 of each.
// Blocks at the end of the longest prompts have the most keys and start first.
// Warps: 0-3, 4-7 softmax of the halves, 8 TMA producer, 9 MMA issue + TMEM. All waits are bounded.
#include "latent.cuh"
#include "latent_ptx.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_ptx.cuh"

namespace pda {

namespace {

constexpr int kFRows = 256, kFKeys = 128;
constexpr int kFLine = kFKeys * 128;         // 16 KB: one 128-byte line of 128 rows
constexpr int kFQLines = 3, kFKLines = 3, kFVLines = 2, kFUnits = kFKLines + kFVLines;
constexpr int kFSlots = 8;
constexpr int kFThreads = 384, kFProducer = 8, kFMma = 9;
constexpr int kFSmemBytes = 2 * kFQLines * kFLine + kFSlots * kFLine + 512 + 1024;
static_assert(kFSmemBytes <= 232448, "shared memory");
// 384 threads start with 168 registers; the control warps keep 72 and the softmax warps take 208
constexpr uint32_t kFRegsSoftmax = 208, kFRegsControl = 72;
constexpr uint32_t kFTmemCols = 512, kFTmemO = 256;  // S[w] at 128 w, P[w] over its first 64 columns, O[w] at 256 + 128 w
constexpr float kFNoMax = -1e30f;
constexpr float kFRescale = 8.f;

struct FMaps {
  CUtensorMap q, k_nope, k_rope, v;
};

__global__ void __launch_bounds__(kFThreads, 1)
latent_prefill_tc_kernel(const __grid_constant__ FMaps maps, const __grid_constant__ LatentPrefillParams p, int q_blocks) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (2 * kFQLines + kFSlots) * kFLine);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 32);
  int* cta_err = reinterpret_cast<int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // late blocks first (all heads and sequences of a block index together)
  const int per_block = p.num_heads * p.batch;
  const int qb = q_blocks - 1 - static_cast<int>(blockIdx.x / per_block);
  const int b = static_cast<int>(blockIdx.x % per_block) / p.num_heads, h = static_cast<int>(blockIdx.x % per_block) % p.num_heads;
  const PrefillSpan sp = prefill_span(p, b);
  const int row0 = qb * kFRows;
  if (row0 >= sp.nq) return;
  // keys that the last row of half w can see, in tiles
  int n_tiles[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int first = row0 + 128 * w, last = min(first + 127, sp.nq - 1);
    const int see = first >= sp.nq ? 0 : min(max(sp.nk - sp.nq_all + last + 1, 0), sp.nk);
    n_tiles[w] = (see + kFKeys - 1) / kFKeys;
  }
  const int n_max = max(n_tiles[0], n_tiles[1]);
  // (a CTA of this launch has met an expired wait: nothing more is attended)
  const bool dead = p.status != nullptr && *reinterpret_cast<volatile int32_t*>(p.status) == PDA_DEV_TIMEOUT;

  const uint32_t q_sm = smem_u32(smem), ring = q_sm + 2 * kFQLines * kFLine;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kFSlots, bar_q = empty0 + 8 * kFSlots;  // Q half w
  const uint32_t bar_s = bar_q + 16, bar_p = bar_s + 16, bar_pv = bar_p + 16, bar_drain = bar_pv + 16;
  if (tid == 0) {
    for (int i = 0; i < 2 * kFSlots; ++i) mbar_init(full0 + 8 * i, 1);
    for (int w = 0; w < 2; ++w) {
      mbar_init(bar_q + 8 * w, 1);
      mbar_init(bar_s + 8 * w, 1);
      mbar_init(bar_p + 8 * w, 4);
      mbar_init(bar_pv + 8 * w, 1);
    }
    mbar_init(bar_drain, 1);
    *cta_err = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == kFMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kFTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  const bool skip = __syncthreads_or(dead) || n_max == 0;
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;

  if (warp >= 8) {
    reg_alloc_dec<kFRegsControl>();
    if (warp == kFProducer && !skip) {
      // ================= TMA producer =================
      const uint32_t leader = elect_one();
      const uint32_t u_q = uniform(q_sm), u_ring = uniform(ring), u_h = uniform(h);
      const int token0 = uniform(sp.q0 + row0), key0 = uniform(sp.k0);
      int armed = 0;
      auto load_q = [&](int w) {
        mbar_expect_tx_if(leader, bar_q + 8 * w, kFQLines * kFLine);
#pragma unroll
        for (int ln = 0; ln < kFQLines; ++ln)
          tma_load_4d_if(leader, u_q + (w * kFQLines + ln) * kFLine, &maps.q, bar_q + 8 * w, ln, u_h, token0 + 128 * w);
      };
      if (n_tiles[0] > 0) load_q(0);
      int slot = 0;
      uint32_t round = 0;
      for (int j = 0; ok && j < n_max; ++j) {
#pragma unroll
        for (int u = 0; u < kFUnits; ++u) {
          if (round > 0) ok = mbar_wait_bounded(empty0 + 8 * slot, (round - 1) & 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint32_t bar = uniform(full0 + 8 * slot), dst = uniform(u_ring + slot * kFLine);
          const int key = key0 + j * kFKeys;
          mbar_expect_tx_if(leader, bar, kFLine);
          if (u < 2) tma_load_4d_if(leader, dst, &maps.k_nope, bar, u, u_h, key);
          else if (u == 2) tma_load_4d_if(leader, dst, &maps.k_rope, bar, 0, 0, key);
          else tma_load_4d_if(leader, dst, &maps.v, bar, u - 3, u_h, key);
          ++armed;
          if (++slot == kFSlots) { slot = 0; ++round; }
          if (j == 0 && u == 2 && n_tiles[1] > 0) load_q(1);
        }
      }
      if (!ok) {  // copies in flight end before the CTA does
        if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
        for (int u = max(armed - kFSlots, 0); u < armed; ++u) mbar_wait_bounded(full0 + 8 * (u % kFSlots), (u / kFSlots) & 1, 1u << 12);
        for (int w = 0; w < 2; ++w)
          if (n_tiles[w] > 0 && (w == 0 || armed > 2)) mbar_wait_bounded(bar_q + 8 * w, 0, 1u << 12);
      }
    } else if (warp == kFMma && !skip) {
      // ================= products =================
      constexpr uint32_t idesc_s = latent_idesc(128, kFKeys, false, false), idesc_o = latent_idesc(128, 64, false, true);
      const uint32_t leader = elect_one();
      const uint32_t u_q = uniform(q_sm), u_ring = uniform(ring), u_tmem = uniform(tmem);
      auto wait_unit = [&](int u) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(full0 + 8 * (u % kFSlots), (u / kFSlots) & 1));
      };
      auto s_product = [&](int w, int j) {
#pragma unroll
        for (int ln = 0; ln < kFKLines; ++ln) {
          const int u = j * kFUnits + ln;
          wait_unit(u);
          if (!ok) return;
          tc_fence_after();
          const uint64_t ad = tc_desc(uniform(u_q + (w * kFQLines + ln) * kFLine), 16, 1024);
          const uint64_t bd = tc_desc(uniform(u_ring + (u % kFSlots) * kFLine), 16, 1024);
          const uint32_t d = uniform(u_tmem + 128 * w);
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) mma_ss_if(leader, d, ad + 2 * ks, bd + 2 * ks, idesc_s, (ln > 0 || ks > 0) ? 1u : 0u);
        }
        tc_commit_if(leader, uniform(bar_s + 8 * w));
      };
      auto o_product = [&](int w, int j) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_p + 8 * w, j & 1));
        const uint32_t acc = uniform(j > 0 ? 1u : 0u);
#pragma unroll
        for (int ln = 0; ln < kFVLines; ++ln) {
          const int u = j * kFUnits + kFKLines + ln;
          wait_unit(u);
          if (!ok) return;
          tc_fence_after();
          const uint64_t bd = tc_desc(uniform(u_ring + (u % kFSlots) * kFLine), 16, 1024);
          const uint32_t pa = uniform(u_tmem + 128 * w), d = uniform(u_tmem + kFTmemO + 128 * w + 64 * ln);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) tc_mma_ts_if<false>(leader, d, pa + 8 * ks, bd + 128 * ks, idesc_o, ks > 0 ? 1u : acc);
        }
        tc_commit_if(leader, uniform(bar_pv + 8 * w));
      };
      auto release = [&](int j, int first, int n) {
        for (int k = 0; k < n; ++k) tc_commit_if(leader, uniform(empty0 + 8 * ((j * kFUnits + first + k) % kFSlots)));
      };
      for (int w = 0; w < 2; ++w) {
        if (n_tiles[w] == 0) continue;
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar_q + 8 * w, 0));
        if (ok) s_product(w, 0);
      }
      if (ok) release(0, 0, kFKLines);
      for (int j = 0; ok && j < n_max; ++j) {
        for (int w = 0; ok && w < 2; ++w) {
          // S(j + 1) takes the place of P(j): the tensor core works its products off in order
          if (j < n_tiles[w]) o_product(w, j);
          if (!ok) break;
          if (w == 1) release(j, kFKLines, kFVLines);
          if (j + 1 < n_tiles[w]) s_product(w, j + 1);
        }
        if (ok && j + 1 < n_max) release(j + 1, 0, kFKLines);
      }
      if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
      tc_commit_if(leader, bar_drain);
      __syncwarp();
      if (!mbar_wait_bounded(bar_drain, 0, 1u << 12) && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    }
  } else {
    reg_alloc_inc<kFRegsSoftmax>();
    // ================= softmax and output: thread = row =================
    const int w = warp >> 2, t = tid & 127;
    const int row = row0 + 128 * w + t;                       // query token of the sequence
    const int lim = min(sp.nk, sp.nk - sp.nq_all + row + 1);  // keys it sees
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t my_s = tmem + 128 * w + lane_base, my_o = tmem + kFTmemO + 128 * w + lane_base;
    const float scale_log2 = p.scale * 1.4426950408889634f;
    const uint64_t scale2 = f32x2(__float_as_uint(scale_log2), __float_as_uint(scale_log2));
    const int n = skip ? 0 : n_tiles[w];
    float m_ref = kFNoMax, l = 0.f;
    for (int j = 0; j < n; ++j) {
      if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_s + 8 * w, j & 1));
      if (!ok) break;
      tc_fence_after();
      uint32_t sv[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(my_s + 32 * c, sv[c]);
      tmem_wait_ld();
      const int vis = lim - j * kFKeys;  // visible columns of this row
      if (__any_sync(0xffffffffu, vis < kFKeys)) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (c * 32 + e >= vis) sv[c][e] = 0xff800000u;  // -inf
        const int valid = sp.nk - j * kFKeys;
        if (valid < kFKeys && (w == 0 || j >= n_tiles[0])) {
          // keys behind the sequence's end have weight 0, but their values may be anything: cleared (the halves
          // share V; the other half's product with it is issued after this one's)
          for (int ln = 0; ln < kFVLines; ++ln) {
            const int u = j * kFUnits + kFKLines + ln;
            if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(full0 + 8 * (u % kFSlots), (u / kFSlots) & 1));
            if (!ok) break;
            for (int k = t; k < (kFKeys - valid) * 8; k += 128)
              asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(ring + (u % kFSlots) * kFLine + valid * 128 + k * 16), "r"(0));
          }
          fence_proxy_async();
          if (!ok) break;
        }
      }
      float mx[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        mx[c] = fmaxf(__uint_as_float(sv[c][0]), __uint_as_float(sv[c][1]));
#pragma unroll
        for (int e = 2; e < 32; e += 2) mx[c] = max3(mx[c], __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
      }
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2;
      if (__any_sync(0xffffffffu, top > m_ref + kFRescale)) {
        const float m_new = fmaxf(m_ref, top), a = ex2(m_ref - m_new);
        m_ref = m_new;
        l *= a;
        if (j > 0) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 8 * w, (j - 1) & 1));
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t ov[32];
            tmem_ld32(my_o + 32 * c, ov);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * a);
            tmem_st32(my_o + 32 * c, ov);
          }
        }
      }
      const uint64_t ref2 = f32x2(__float_as_uint(-m_ref), __float_as_uint(-m_ref));
      uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float x0, x1;
          f32x2_split(fma_f32x2(f32x2(sv[c][e], sv[c][e + 1]), scale2, ref2), x0, x1);
          const float w0 = ex2(x0), w1 = ex2(x1);
          sum2[(e >> 1) & 1] = add_f32x2(sum2[(e >> 1) & 1], f32x2(__float_as_uint(w0), __float_as_uint(w1)));
          pk[e >> 1] = pack2<false>(w0, w1);
        }
        tmem_st16(my_s + 16 * c, pk);
      }
      float s0, s1;
      f32x2_split(add_f32x2(sum2[0], sum2[1]), s0, s1);
      l += s0 + s1;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_tc(bar_p + 8 * w);
    }
    // ---- output
    if (n > 0) {
      if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 8 * w, (n - 1) & 1));
      if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
      tc_fence_after();
    }
    if (row0 + 128 * w + (warp & 3) * 32 < sp.nq) {  // (warp-uniform)
      const float inv = n == 0 || !ok || l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* out = p.out + (static_cast<int64_t>(sp.q0) + row) * p.out_token_stride + h * p.out_head_stride;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t ov[32];
        tmem_ld32(my_o + 32 * c, ov);
        tmem_wait_ld();
        if (row < sp.nq) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              o[k] = inv == 0.f ? 0u : pack2<false>(__uint_as_float(ov[e + 2 * k]) * inv, __uint_as_float(ov[e + 2 * k + 1]) * inv);
            *reinterpret_cast<uint4*>(out + 32 * c + e) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
      }
    }
  }

  // ---- teardown
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && *cta_err) report(p.status, *cta_err);
  if (warp == kFMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kFTmemCols) : "memory");
  }
}

// [tokens][heads][lines][64]: a copy takes one line of 128 tokens of one head
bool encode_rows(EncodeFn enc, CUtensorMap* map, const void* base, int64_t dim, int64_t heads, int64_t tokens, int64_t head_stride,
                 int64_t token_stride) {
  const cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(dim / 64), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
  // (a dimension of extent 1 is never stepped over)
  const cuuint64_t strides[3] = {128, heads == 1 ? 128 : static_cast<cuuint64_t>(head_stride) * 2,
                                 tokens == 1 ? 128 : static_cast<cuuint64_t>(token_stride) * 2};
  const cuuint32_t box[4] = {64, 1, 1, kFKeys};
  const cuuint32_t step[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool latent_prefill_tc_supports(const LatentPrefillParams& p) {
  if (p.nope_dim != 128 || p.rope_dim != 64 || p.v_dim != 128 || p.total_k < 1) return false;
  if (!(p.scale > 0.f) || !(p.scale < INFINITY)) return false;  // (the row maximum is taken before scaling)
  const auto fits = [](int64_t stride, int64_t extent) { return extent == 1 || (stride > 0 && stride < (1ll << 38)); };
  if (!fits(p.q_token_stride, p.total_q) || !fits(p.q_head_stride, p.num_heads) || !fits(p.kn_token_stride, p.total_k) ||
      !fits(p.kn_head_stride, p.num_heads) || !fits(p.kr_token_stride, p.total_k) || !fits(p.v_token_stride, p.total_k) ||
      !fits(p.v_head_stride, p.num_heads))
    return false;
  // (row and key numbers are counted in 32 bits, up to one block behind the last)
  if (p.total_q > INT32_MAX - 512 || p.total_k > INT32_MAX - 512) return false;
  return static_cast<int64_t>((p.max_q + kFRows - 1) / kFRows) * p.num_heads * p.batch <= INT32_MAX;
}

cudaError_t launch_latent_prefill_tc(const LatentPrefillParams& p, cudaStream_t stream) {
  EncodeFn enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  FMaps maps{};
  if (!encode_rows(enc, &maps.q, p.q, 192, p.num_heads, p.total_q, p.q_head_stride, p.q_token_stride) ||
      !encode_rows(enc, &maps.k_nope, p.k_nope, 128, p.num_heads, p.total_k, p.kn_head_stride, p.kn_token_stride) ||
      !encode_rows(enc, &maps.k_rope, p.k_rope, 64, 1, p.total_k, 0, p.kr_token_stride) ||
      !encode_rows(enc, &maps.v, p.v, 128, p.num_heads, p.total_k, p.v_head_stride, p.v_token_stride))
    return cudaErrorNotSupported;
  cudaError_t e = cudaFuncSetAttribute(latent_prefill_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFSmemBytes);
  if (e != cudaSuccess) return e;
  const int q_blocks = (p.max_q + kFRows - 1) / kFRows;
  latent_prefill_tc_kernel<<<q_blocks * p.num_heads * p.batch, kFThreads, kFSmemBytes, stream>>>(maps, p, q_blocks);
  return cudaGetLastError();
}

}  // namespace pda
