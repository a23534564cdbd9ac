// Expanded attention (keys [k_nope per head | k_rope shared], values per head; packed ragged sequences,
// causal from the end) on tcgen05 + TMEM, dims 128 + 64 and 128.
//
// A pair of CTAs (a cluster of two SMs, tcgen05 cta_group::2) takes 512 query rows of one head as two halves
// of 256, 128 rows of each in either CTA (TMEM lane = row), and walks over the keys 128 at a time:
//   S[w] = Q[w] . K^T    12 MMAs M256 N128 K16; of K each CTA holds 64 keys (2 lines of k_nope, 1 of k_rope:
//                        the shared part is copied from its one array, never concatenated in memory)
//   O[w] += P[w] . V     8 MMAs M256 N128 K16; P (bf16) in tensor memory over the S it came from, of V each
//                        CTA holds 64 of the 128 dims
// Every MMA reads both CTAs' shares of B, so a CTA copies 40 KB a tile for 256 rows instead of 80: Q takes
// 96 KB, and with 80 KB a tile the ring was so short (1.6 tiles) that products waited for copies; with
// the pair it holds three tiles, and half the bytes come from L2.
// S[0], S[1], O[0], O[1] fill the 512 columns, P lies over the S it comes from, and a thread's softmax takes 64 keys at
// a time. Two forms of the kernel (the launch chooses, with figures there):
//   S at once     S of the next tile follows the second 64 keys' P . V; the halves take turns, one's softmax under the
//                 other's products: 1300 clocks of products per half and tile against 1024 of exponentials.
//   S in two runs 64 keys each (32 of either CTA's), each taken again as soon as its own P . V is through, so a half has
//                 scores of the next tile before its softmax is done with this one, and nobody takes turns: 10 % more
//                 clocks of products, which read A for 64 columns only.
// Of the exponentials every kFPolyOf-th pair is taken by a polynomial on the FMA units.
// The softmax takes weights relative to a reference per row that is raised (and O rescaled in tensor memory)
// only when the row's maximum passes it by more than 2^8; row sums are kept by the row's thread, of the
// 32-bit weights; the rounding of the weights to bf16 is 2^-8 of each.
// Each pair of CTAs works through several row blocks, those with the most keys first and dealt to and fro; the
// producer runs on into the next block's Q, K and V while the last one's output is written.
// A block of at most 256 rows would leave the second half idle. It gets the same rows of the next head instead (64
// prompts of 200 tokens with 16 heads: 102 us one head at a time, 83 two), or, where there is a pair of CTAs for each block and head
// already, the later part of the same head's keys (4 chunks of 24 tokens behind 2000..4000, 16 heads: 66 us with one
// half, 79 with two heads, 49 with half of the keys each).
// Measured (B200): a prompt of 8192 tokens with 32 heads 0.62 ms, 1.1 PFLOP/s; the clock is held near 1.6 GHz by the
// power cap. 24 prompts of 1..700 tokens with 16 heads: 76 us, of which a block of 200 rows and its two tiles a half
// take 7 us: copies of 256 KB a CTA (4000 to 5000 clocks from asking to use), two softmaxes and the output in a row.
// Warps of each CTA: 0-3, 4-7 softmax of the halves, 8 TMA producer, 9 and 10 MMA issue of the halves (in the
// pair's first CTA; 9: TMEM), 11 hands V tiles on, clearing what lies behind the sequence's end. All waits are
// bounded.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "latent.cuh"
#include "latent_ptx.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_ptx.cuh"

namespace pda {

namespace {

constexpr int kFRows = 512, kFHalf = 256, kFKeys = 128;  // query rows of a pair of CTAs, of a half; keys per tile
constexpr int kFQLines = 3;
constexpr int kFQLine = 128 * 128;                        // one 128-byte line of the CTA's 128 rows of a half
constexpr int kFKLine = 64 * 128, kFKBytes = 3 * kFKLine;  // of its 64 keys
constexpr int kFVBytes = kFKeys * 128;                    // its line (64 dims) of all keys
constexpr int kFStages = 3;                               // tiles
constexpr int kFSoftWarps = 8, kFThreads = (kFSoftWarps + 4) * 32, kFProducer = 8, kFMma = 9, kFRelay = 11;  // (9, 10: one per half)
constexpr int kFBookBytes = 5 * 1024;  // barriers, units, the list of row blocks, the second half's sums
constexpr int kFSmemBytes = 2 * kFQLines * kFQLine + kFStages * (kFKBytes + kFVBytes) + kFBookBytes + 1024;
static_assert(kFSmemBytes <= 232448, "shared memory");
// 384 threads start with 168 registers (64512 in all); the control warps keep 104 and the softmax warps take 200
constexpr uint32_t kFRegsSoftmax = 200, kFRegsControl = 104;
static_assert(kFSoftWarps * 32 * kFRegsSoftmax + 128 * kFRegsControl <= kFThreads * 168, "registers");
constexpr uint32_t kFTmemCols = 512, kFTmemO = 256;  // S[w] at 128 w, P[w] over its first 64 columns, O[w] at 256 + 128 w
constexpr int kFUnitSlots = 4;                            // units the producer may be ahead
constexpr int kFMaxList = 128;                            // row blocks that are sorted by their work
constexpr float kFNoMax = -FLT_MAX;  // reference of a row that has seen no finite score yet: the lowest it can be
constexpr float kFRescale = 8.f;
constexpr int kFPolyOf = 4;  // every fourth pair of exponentials by polynomial

__device__ __forceinline__ float max3_nan(float a, float b, float c) {  // NaN if any is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^x for two x <= 2^7 on the FMA units, so that the exponentials are not bound by the special-function unit
// alone: x = n + f with n the nearest integer (by adding 1.5 * 2^23, whose low bits then hold n), 2^f by the
// polynomial of degree 3 whose largest relative error over [-1/2, 1/2] is least (7.5e-5, found by Remez
// exchange; a weight's rounding to bf16 is 3.9e-3), n added to the exponent. x below -126 gives 2^-126, and so
// does a NaN: that is looked for in the scores' maximum.
__device__ __forceinline__ void exp2_pair(uint64_t x, float& w0, float& w1) {
  auto both = [](float v) { return f32x2(__float_as_uint(v), __float_as_uint(v)); };
  float x0, x1;
  f32x2_split(x, x0, x1);
  x = f32x2(__float_as_uint(fmaxf(x0, -126.f)), __float_as_uint(fmaxf(x1, -126.f)));
  const uint64_t t = add_f32x2(x, both(12582912.f));
  const uint64_t f = add_f32x2(x, fma_f32x2(t, both(-1.f), both(12582912.f)));
  uint64_t y = fma_f32x2(f, both(0.0551716691f), both(0.242611122f));
  y = fma_f32x2(y, f, both(0.693260985f));
  y = fma_f32x2(y, f, both(0.999928074f));
  float t0, t1;
  f32x2_split(t, t0, t1);
  f32x2_split(y, w0, w1);
  w0 = __uint_as_float(__float_as_uint(w0) + (__float_as_uint(t0) << 23));
  w1 = __uint_as_float(__float_as_uint(w1) + (__float_as_uint(t1) << 23));
}

// A row's weights are 2^(c s - c r), s its scores and r its reference as they come from the product, by one fused
// multiply-add with c r rounded: off by half a step of c r, the same for all of the row, so it cancels in the quotient. c is
// scale * log2(e) as long as |c r| < 2^28, where that is at most 2^8. Beyond, scores that differ at all differ by 16 and
// more there, so that only the largest one weighs anything in 32 bits, and by any c that is large enough: then c is a
// power of two with 2^31 <= |c r| < 2^32, c r is exact, and other scores are 2^7 and more away.
__device__ __forceinline__ float score_factor(float r, float scale_log2) {
  if (fabsf(r * scale_log2) < 268435456.f) return scale_log2;
  const uint32_t exponent = (__float_as_uint(r) >> 23) & 255u;
  return __uint_as_float(min(127u + 31u + 127u - min(exponent, 254u), 254u) << 23);
}
// What weights and sums taken at reference `from` are multiplied by to be those at a reference `to` >= from whose factor is c
// (each product rounded by itself, as the weights have it). Where either reference is far, the two are equal or the products
// are 16 or more apart, with any factor: then next to `to` what was taken at `from` is as good as nothing.
__device__ __forceinline__ float rescale(float from, float to, float c) { return ex2(__fmul_rn(from, c) - __fmul_rn(to, c)); }

// One row block of one head, as the producer hands it to the other warps of its CTA. row0 < 0: no more.
// dual: the block has at most kFHalf rows and both halves take the same ones, with tiles of their own by turns (first
// half's, second half's, ...; as many for both): kTwoHeads: the second half's are the next head's; kSplitKeys: the
// second half's are the later n1 tiles of the same head, and the first half's warps merge the two results.
enum : int { kOneHead = 0, kTwoHeads = 1, kSplitKeys = 2 };
struct FUnit {
  int row0, h, q0, nq, k0, nk, n0, n1, dual;
  __device__ int first_row(int w) const { return row0 + (dual ? 0 : kFHalf * w); }
  __device__ int head(int w) const { return h + (dual == kTwoHeads ? w : 0); }
  __device__ int tiles() const { return dual ? n0 + n1 : max(n0, n1); }
  // The pair's i-th tile: whose half's (where that matters), and which 128 keys.
  __device__ int half_of(int i) const { return i & 1; }
  __device__ int keys_of(int i) const { return dual ? key_tile(i & 1, i >> 1) : i; }
  __device__ int key_tile(int w, int j) const { return dual == kSplitKeys && w ? n0 + j : j; }
};
constexpr uint32_t kFSmallBlock = 1u << 30;  // (in a list entry) at most kFHalf rows
__device__ __forceinline__ int units_of(uint32_t entry, int num_heads, bool by_two) {
  return by_two && (entry & kFSmallBlock) ? (num_heads + 1) / 2 : num_heads;
}
struct FPlan {
  int q_blocks;  // blocks of max_q
  int listed;    // the row blocks of all sequences are few enough to be listed and sorted in shared memory
  int64_t slots;  // > 0: row blocks are looked for at this many places (below), not at each of q_blocks of each sequence
};

struct FMaps {
  CUtensorMap q, k_nope, k_rope, v;
};

// ---- the pair: instructions of cta_group::2 and barriers in the other CTA ----
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {  // bar: an address of in_cta
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The same where nothing has been written, or only tensor memory, which the tcgen05 fences order.
__device__ __forceinline__ void arrive_cluster_tc(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_spin_cluster(uint32_t bar, uint32_t parity) {  // for arrivals from either CTA
  for (uint32_t i = 0; i < kTestSpinLimit; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A copy into this CTA whose bytes count for a barrier of either CTA of the pair.
__device__ __forceinline__ void tma_load_4d_pair_if(uint32_t leader, uint32_t dst, const CUtensorMap* map, uint32_t bar, int c1, int c2,
                                                    int c3) {
  asm volatile(
      "{\n\t.reg .pred pe;\n\tsetp.ne.b32 pe, %6, 0;\n\t"
      "@pe cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {0, %3, %4, %5}], [%2];\n\t}"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c1), "r"(c2), "r"(c3), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma2_ss_if(uint32_t leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred pe, pa;\n\tsetp.ne.b32 pe, %5, 0;\n\tsetp.ne.b32 pa, %4, 0;\n\t"
      "@pe tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, pa;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma2_ts_if(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred pe, pa;\n\tsetp.ne.b32 pe, %5, 0;\n\tsetp.ne.b32 pa, %4, 0;\n\t"
      "@pe tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, pa;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// Arrival at the barrier at this offset in both CTAs once this thread's products so far are through.
__device__ __forceinline__ void commit2_if(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred pe;\n\t.reg .b16 m;\n\tsetp.ne.b32 pe, %1, 0;\n\tmov.b16 m, 3;\n\t"
      "@pe tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}"
      ::"r"(bar), "r"(leader) : "memory");
}

template <bool kRuns>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFThreads, 1)
latent_prefill_tc_kernel(const __grid_constant__ FMaps maps, const __grid_constant__ LatentPrefillParams p,
                         const __grid_constant__ FPlan plan) {
  constexpr uint32_t kRunP = kRuns ? 64 : 32;  // columns from the first run's weights to the second's
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 2 * kFQLines * kFQLine + kFStages * (kFKBytes + kFVBytes));
  FUnit* units = reinterpret_cast<FUnit*>(bars + 68);               // [kFUnitSlots]
  uint32_t* list = reinterpret_cast<uint32_t*>(units + kFUnitSlots);  // [kFMaxList] sequence and block, most work first
  uint32_t* work = list + kFMaxList;                                // [kFMaxList] keys, then units of the entries before
  uint32_t* scan = work + kFMaxList;                                // [5] sequences' blocks, by warp; their sum
  uint32_t* tmem_slot = scan + 6;
  int* cta_err = reinterpret_cast<int*>(tmem_slot + 1);
  float* merge_sh = reinterpret_cast<float*>(cta_err + 1);          // [128][2]
  int4* spans = reinterpret_cast<int4*>(reinterpret_cast<uint8_t*>(bars) + kFBookBytes - kFMaxList * 16);  // listed sequences' q0, nq, k0, nk
  static_assert(68 * 8 + kFUnitSlots * sizeof(FUnit) + 2 * kFMaxList * 4 + 8 * 4 + 1024 + kFMaxList * 16 <= kFBookBytes, "shared memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x & 1;  // in the pair
  const int pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  bool ok = true;

  const uint32_t q_sm = smem_u32(smem), k_sm = q_sm + 2 * kFQLines * kFQLine, v_sm = k_sm + kFStages * kFKBytes;
  // Barriers, at the same place in both CTAs. Of the pair's first CTA: full_k (both CTAs' copies), v_ready, bar_q,
  // bar_p, bar_turn, bar_ofree. In each: empty_k, empty_v (both halves' products), full_v (its own copy), bar_s,
  // bar_pv, bar_qfree, the unit slots'. bar_s, bar_p and bar_pv: [half w][run of
  // 64 keys] (bar_s with S at once: the first only).
  const uint32_t full_k = smem_u32(bars), empty_k = full_k + 24 * kFStages, full_v = empty_k + 8 * kFStages,
                 empty_v = full_v + 8 * kFStages, v_ready = empty_v + 8 * kFStages, bar_q = v_ready + 24 * kFStages;
  const uint32_t bar_s = bar_q + 16, bar_p = bar_s + 32, bar_pv = bar_p + 32, bar_turn = bar_pv + 32, bar_qfree = bar_turn + 16,
                 bar_ofree = bar_qfree + 16, unit_full = bar_ofree + 16, unit_empty = unit_full + 8 * kFUnitSlots,
                 bar_drain = unit_empty + 8 * kFUnitSlots, bar_never = bar_drain + 8, bar_merge = bar_never + 8;
  if (tid == 0) {
    for (int i = 0; i < kFStages; ++i) {
      for (int set = 0; set < 3; ++set) {
        mbar_init(full_k + 8 * (kFStages * set + i), 1);
        mbar_init(v_ready + 8 * (kFStages * set + i), 2);
      }
      mbar_init(empty_k + 8 * i, 2);
      mbar_init(full_v + 8 * i, 1);
      mbar_init(empty_v + 8 * i, 2);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(bar_q + 8 * w, 1);
      for (int k = 0; k < 2; ++k) {
        mbar_init(bar_s + 16 * w + 8 * k, 1);
        mbar_init(bar_p + 16 * w + 8 * k, 8);  // four warps of each CTA
        mbar_init(bar_pv + 16 * w + 8 * k, 1);
      }
      mbar_init(bar_turn + 8 * w, 1);
      mbar_init(bar_qfree + 8 * w, 1);
      mbar_init(bar_ofree + 8 * w, 8);
    }
    for (int i = 0; i < kFUnitSlots; ++i) {
      mbar_init(unit_full + 8 * i, 1);
      mbar_init(unit_empty + 8 * i, kFSoftWarps + 1 + (rank == 0 ? 2 : 0));  // softmax, relay, product warps
    }
    mbar_init(bar_drain, 2);
    mbar_init(bar_never, 1);
    for (int i = 0; i < 4; ++i) mbar_init(bar_merge + 8 * i, 1);
    *cta_err = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == kFProducer && elect_one()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k_nope) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k_rope) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
  }
  if (warp == kFMma) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kFTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // ---- the row blocks that there are, those with the most keys first (every CTA for itself, all alike)
  int my_blocks = 0;
  PrefillSpan mine{0, 0, 0, 0, 0};
  if (plan.listed && tid < kFMaxList && tid < p.batch) {
    mine = prefill_span(p, tid);
    my_blocks = (mine.nq + kFRows - 1) / kFRows;
    spans[tid] = make_int4(mine.q0, mine.nq, mine.k0, mine.nk);
  }
  int incl = my_blocks;
  if (plan.listed && tid < kFMaxList) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) scan[warp] = incl;
  }
  tc_fence_before();
  __syncthreads();
  int n_blocks = 0;
  uint32_t my_work = 0, my_entry = 0;
  bool by_two = true;  // heads two by two on small blocks
  if (plan.listed) {
    int before = incl - my_blocks;
    for (int i = 0; i < kFMaxList / 32; ++i) {
      before += i < warp ? scan[i] : 0;
      n_blocks += scan[i];
    }
    // (ascending offsets give at most as many as the host has allowed for; others are reported)
    if (n_blocks > kFMaxList) {
      report(p.status, PDA_DEV_BAD_SEQ_LEN);
      n_blocks = kFMaxList;
    }
    // ... unless there is a pair of CTAs for each head of each block: half as many units are no gain then
    by_two = static_cast<int64_t>(n_blocks) * p.num_heads > pairs;
    for (int k = 0; k < my_blocks && before + k < kFMaxList; ++k) {
      const int last = min((k + 1) * kFRows, mine.nq) - 1;
      work[before + k] = min(max(mine.nk - mine.nq_all + last + 1, 0), mine.nk);
      list[before + k] = tid | (k << 7) | (mine.nq - k * kFRows <= kFHalf ? kFSmallBlock : 0u);
    }
    __syncthreads();
    int place = 0;
    if (tid < n_blocks) {
      my_work = work[tid];
      my_entry = list[tid];
      for (int i = 0; i < n_blocks; ++i) place += work[i] > my_work || (work[i] == my_work && i < tid);
    }
    __syncthreads();
    if (tid < n_blocks) list[place] = my_entry;
    __syncthreads();
    uint32_t units = tid < n_blocks ? units_of(list[tid], p.num_heads, by_two) : 0;
    const uint32_t my_units = units;
    if (tid < kFMaxList) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, units, o);
        if (lane >= o) units += u;
      }
      if (lane == 31) scan[warp] = units;
    }
    __syncthreads();
    uint32_t units_before = units - my_units;
    for (int i = 0; i < kFMaxList / 32; ++i) units_before += i < warp ? scan[i] : 0;
    if (tid < n_blocks) work[tid] = units_before;
  }
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // Unit number k of this CTA, for the warps that are told by the producer.
  auto next_unit = [&](int k, FUnit& un) {
    const int slot = k % kFUnitSlots;
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(unit_full + 8 * slot, (k / kFUnitSlots) & 1));
    if (!ok) return false;
    un = units[slot];
    return un.row0 >= 0;
  };
  auto free_unit = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive_tc(unit_empty + 8 * (k % kFUnitSlots));
  };

  // The barrier of a tile, from full_k or v_ready: both halves' tiles, the first half's and the second half's (dual
  // blocks) are counted each for themselves, so that who waits for a set's barriers follows all their phases. (Three
  // tiles of a set are in the ring at most: a barrier's next use comes behind its last one's wait.)
  auto tile_bar = [&](uint32_t first, int set, int count) { return first + 8 * (kFStages * set + count % kFStages); };

  // ================= products of half w =================
  // A warp for each half, which prepares its next products while the other's are being issued (one warp for both
  // spent as long between the products as on them). Where S is taken at once, they take turns: so the halves stay in
  // opposite phase (without, both ran their softmax at the same time and the tensor core waited: 0.89 ms instead of 0.61
  // for the 8192-token prompt).
  auto issue_role = [&](auto half) {
    constexpr int w = decltype(half)::value;
    constexpr uint32_t idesc_s = latent_idesc(256, kFKeys, false, false), idesc_run = latent_idesc(256, kFKeys / 2, false, false),
                       idesc_o = latent_idesc(256, 128, false, true);
    const uint32_t leader = elect_one();
    const uint32_t u_q = uniform(q_sm + w * kFQLines * kFQLine), u_k = uniform(k_sm), u_v = uniform(v_sm), u_tmem = uniform(tmem);
    const uint32_t u_ek = uniform(empty_k), u_ev = uniform(empty_v);
    const uint32_t d_s = u_tmem + 128 * w, d_o = u_tmem + kFTmemO + 128 * w;
    auto wait = [&](uint32_t bar, int phase) {
      if (ok) ok = __all_sync(0xffffffffu, mbar_spin_cluster(bar, phase & 1));
    };
    // S of a tile at once, or of run k of two: of each CTA's 64 keys those from 32 k on
    auto s_product = [&](uint32_t k_addr, int k, uint32_t idesc) {
      const uint64_t q0 = tc_desc(u_q, 16, 1024), k0 = tc_desc(k_addr, 16, 1024) + 256 * k;
#pragma unroll
      for (int ln = 0; ln < kFQLines; ++ln)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          mma2_ss_if(leader, d_s + 64 * k, q0 + ln * (kFQLine / 16) + 2 * ks, k0 + ln * (kFKLine / 16) + 2 * ks, idesc, (ln > 0 || ks > 0) ? 1u : 0u);
      commit2_if(leader, bar_s + 16 * w + 8 * k);
    };
    FUnit un;
    // Before this unit: tiles of the pair; of this half; units of this half; tiles on which the halves take turns.
    int t0 = 0, mine = 0, done = 0, turns = 0;
    int counts[2] = {0, 0};  // tiles of blocks of two halves; of dual ones, this half's
    for (int k = 0; next_unit(k, un); ++k) {
      free_unit(k);
      const int n = uniform(w == 0 ? un.n0 : un.n1), n_other = uniform(w == 0 ? un.n1 : un.n0);
      const int dual = uniform(un.dual);
      const int step = dual ? 2 : 1, own = dual ? w : 0;  // this half's tiles: t0 + step * j + own
      const int set = dual ? 1 + w : 0, c0 = counts[dual ? 1 : 0];  // this unit's tiles on the set's barriers: c0 + j
      // Both halves give a tile of a block of two halves back. The one that does not read it does so as soon as it is
      // there (see tile_bar) and goes on, to the next unit where this was the last tile.
      auto hand_on = [&](uint32_t full, uint32_t empty, int j) {
        wait(tile_bar(full, 0, c0 + j), (c0 + j) / kFStages);
        if (ok && lane < 2) arrive_cluster_tc(in_cta(empty + 8 * ((t0 + j) % kFStages), lane));
        __syncwarp();
      };
      // (a tile of a dual block is given back twice by its half)
      auto give_back = [&](uint32_t bar) {
        commit2_if(leader, bar);
        if (dual) commit2_if(leader, bar);
      };
      if (n > 0) {  // S(0): its place is free, the tensor core works a thread's products off in order
        const int t = t0 + own, sk = t % kFStages;
        wait(bar_q + 8 * w, done);
        wait(tile_bar(full_k, set, c0), c0 / kFStages);
        if (!ok) break;
        tc_fence_after();
        const uint32_t k_addr = uniform(u_k + sk * kFKBytes);
        s_product(k_addr, 0, kRuns ? idesc_run : idesc_s);
        if constexpr (kRuns) s_product(k_addr, 1, idesc_run);
        if (n == 1) commit2_if(leader, bar_qfree + 8 * w);
        give_back(uniform(u_ek + 8 * sk));
      }
      for (int j = 0; j < n; ++j) {
        const int t = t0 + step * j + own, tn = t + step, sv = t % kFStages, sk = tn % kFStages;
        wait(tile_bar(v_ready, set, c0 + j), (c0 + j) / kFStages);
        const uint64_t v0 = tc_desc(uniform(u_v + sv * kFVBytes), 16, 1024);
        const uint32_t k_addr = uniform(u_k + sk * kFKBytes), ev = uniform(u_ev + 8 * sv), ek = uniform(u_ek + 8 * sk);
        const uint32_t acc = uniform(j > 0 ? 1u : 0u);
        if (j == 0 && done > 0) wait(bar_ofree + 8 * w, done - 1);  // the last unit's output has been read
        // turn i: half 0 after half 1's turn i - 1, half 1 after half 0's turn i
        const bool taking_turns = !kRuns && j < n_other;
        const int turn = turns + j;
        const uint32_t turn_bar = taking_turns && (w == 1 || turn > 0) ? bar_turn + 8 * w : 0u;
        const int turn_phase = w == 1 ? turn : turn - 1;
        // (a run's keys: 64 k .. 64 k + 63 of the tile; in two runs 32 k .. 32 k + 31 and the same from 64 on)
        const uint64_t v_lo = v0 + (kRuns ? 256u : 512u), v_hi = v0 + (kRuns ? 256u : 0u);
        wait(bar_p + 16 * w, mine + j);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) mma2_ts_if(leader, d_o, d_s + 8 * ks, (ks < 2 ? v0 : v_hi) + 128 * ks, idesc_o, ks > 0 ? 1u : acc);
        commit2_if(leader, bar_pv + 16 * w);
        if (j + 1 < n) wait(tile_bar(full_k, set, c0 + j + 1), (c0 + j + 1) / kFStages);
        if (kRuns && j + 1 < n) {
          if (!ok) break;
          tc_fence_after();
          s_product(k_addr, 0, idesc_run);  // over these weights: the tensor core works a thread's products off in order
        }
        {  // the other weights and the turn, looked for at once by different lanes
          const bool second = (lane & 1) && turn_bar != 0u;
          wait(second ? turn_bar : bar_p + 16 * w + 8, second ? turn_phase : mine + j);
        }
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) mma2_ts_if(leader, d_o, d_s + kRunP + 8 * ks, (ks < 2 ? v_lo : v_lo + v_hi - v0) + 128 * ks, idesc_o, 1u);
        commit2_if(leader, bar_pv + 16 * w + 8);
        if (j + 1 < n) s_product(k_addr, kRuns ? 1 : 0, kRuns ? idesc_run : idesc_s);
        if (taking_turns && lane == 0) mbar_arrive_tc(bar_turn + 8 * (1 - w));
        if (j + 2 == n) commit2_if(leader, bar_qfree + 8 * w);
        give_back(ev);
        if (j + 1 < n) give_back(ek);
      }
      if (!dual)
        for (int j = n; ok && j < n_other; ++j) {
          hand_on(full_k, empty_k, j);
          hand_on(v_ready, empty_v, j);
        }
      if (!ok) break;
      t0 += dual ? n + n_other : max(n, n_other);
      if (dual) counts[1] += n; else counts[0] += max(n, n_other);
      if (!kRuns) turns += min(n, n_other);
      mine += n;
      if (n > 0) ++done;
    }
    if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    asm volatile(
        "{\n\t.reg .pred pe;\n\tsetp.ne.b32 pe, %1, 0;\n\t"
        "@pe tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar_drain), "r"(leader) : "memory");
    __syncwarp();
    if (!mbar_wait_bounded(bar_drain, 0, 1u << 12) && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
  };

  if (warp >= kFSoftWarps) {
    reg_alloc_dec<kFRegsControl>();
    if (warp == kFProducer) {
      // ================= units, and TMA: this CTA's rows of Q, keys of K, dims of V =================
      const uint32_t leader = elect_one(), first = leader & (rank == 0 ? 1u : 0u);  // (the first CTA expects both CTAs' bytes)
      const uint32_t u_q = uniform(q_sm), u_k = uniform(k_sm), u_v = uniform(v_sm);
      const uint32_t to_q = uniform(in_cta(bar_q, 0));
      const int64_t n_units = plan.slots > 0 ? plan.slots * p.num_heads
                              : !plan.listed ? static_cast<int64_t>(plan.q_blocks) * p.batch * p.num_heads
                              : n_blocks == 0 ? 0 : static_cast<int64_t>(work[n_blocks - 1]) + units_of(list[n_blocks - 1], p.num_heads, by_two);
      int64_t round = 0;
      auto make_unit = [&](FUnit& un, int qb, int h, int4 span) {
        const int nq = span.y, nk = span.w;
        // keys that the last row of half w can see, in tiles (of either CTA: the pair walks together)
        int n[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int from = qb * kFRows + kFHalf * w, last = min(from + kFHalf - 1, nq - 1);
          const int see = from >= nq ? 0 : min(max(nk - nq + last + 1, 0), nk);
          n[w] = (see + kFKeys - 1) / kFKeys;
        }
        int dual = kOneHead;
        if (by_two && nq - qb * kFRows <= kFHalf && h + 1 < p.num_heads) {
          dual = kTwoHeads;
          n[1] = n[0];
        } else if (!by_two && n[0] > 1 && n[1] == 0) {  // (the second half has no rows, and pairs are not short)
          dual = kSplitKeys;
          n[0] = n[1] = (n[0] + 1) / 2;  // (with an odd number the last tile lies behind the last visible key)
        }
        un = FUnit{qb * kFRows, h, span.x, nq, span.z, nk, n[0], n[1], dual};
      };
      // The pair's next unit: every pairs-th of the order, to and fro, so that each pair gets early (long) and late
      // (short) ones. Unlisted blocks may be empty: 32 at a time are looked at.
      auto find_unit = [&](FUnit& un) {
        if (plan.listed) {
          while (round * pairs < n_units) {
            const int r = static_cast<int>(round++), at = r * pairs + (r & 1 ? pairs - 1 - pair : pair);
            if (at >= n_units) continue;
            int entry = -1;  // the last one whose units start at or before this one
#pragma unroll
            for (int i = 0; i < kFMaxList; i += 32)
              entry += __popc(__ballot_sync(0xffffffffu, i + lane < n_blocks && work[i + lane] <= static_cast<uint32_t>(at)));
            const uint32_t e = list[entry];
            const int h = at - static_cast<int>(work[entry]);
            make_unit(un, (e & (kFSmallBlock - 1)) >> 7, by_two && (e & kFSmallBlock) ? 2 * h : h, spans[e & 127]);
            return true;
          }
          return false;
        }
        while (true) {
          const int64_t r = round + lane, at = r * pairs + (r & 1 ? pairs - 1 - pair : pair);
          int qb = 0, b = 0, h = 0;
          PrefillSpan sp{0, 0, 0, 0, 0};
          if (at < n_units) {
            if (plan.slots > 0) {
              // Sequence b's blocks stand from place cu_q[b] / kFRows + b on: the next sequence's come behind them,
              // and all places are one a sequence and one for every kFRows tokens.
              h = static_cast<int>(at % p.num_heads);
              const int64_t place = plan.slots - 1 - at / p.num_heads;
              int hi = p.batch;  // the last sequence whose first place is not behind this one
              while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (p.cu_q[mid] / kFRows + static_cast<int64_t>(mid) <= place) b = mid; else hi = mid;
              }
              const int64_t in_seq = place - (p.cu_q[b] / kFRows + static_cast<int64_t>(b));
              qb = in_seq < 0 || in_seq >= plan.q_blocks ? plan.q_blocks : static_cast<int>(in_seq);
            } else {
              const int64_t in_block = at % (static_cast<int64_t>(p.batch) * p.num_heads);
              qb = plan.q_blocks - 1 - static_cast<int>(at / (static_cast<int64_t>(p.batch) * p.num_heads));
              b = static_cast<int>(in_block / p.num_heads);
              h = static_cast<int>(in_block % p.num_heads);
            }
            if (qb < plan.q_blocks) sp = prefill_span(p, b);
            else qb = 0;  // (no such block: sp has no rows)
          }
          const bool small = by_two && sp.nq - qb * kFRows <= kFHalf;  // heads two by two
          if (small) h *= 2;
          const uint32_t have = __ballot_sync(0xffffffffu, qb * kFRows < sp.nq && h < p.num_heads);
          if (have == 0) {
            // (r grows with the lane, and so does `at` from one pair of rounds to the next)
            if (round * pairs >= n_units) return false;
            round += 32;
            continue;
          }
          const int src = __ffs(have) - 1;
          round += src + 1;
          auto from_lane = [&](int v) { return __shfl_sync(0xffffffffu, v, src); };
          make_unit(un, from_lane(qb), from_lane(h), make_int4(from_lane(sp.q0), from_lane(sp.nq), from_lane(sp.k0), from_lane(sp.nk)));
          return true;
        }
      };
      int t = 0, done[2] = {0, 0};  // tiles so far; units of each half so far
      int counts[3] = {0, 0, 0};    // tiles so far by set of barriers
      for (int k = 0;; ++k) {
        FUnit un;
        const bool more = find_unit(un);
        if (!more) un.row0 = -1;
        const int slot = k % kFUnitSlots;
        if (k >= kFUnitSlots) ok = __all_sync(0xffffffffu, mbar_wait_bounded(unit_empty + 8 * slot, (k / kFUnitSlots - 1) & 1));
        if (!ok) break;
        if (lane == 0) {
          units[slot] = un;
          mbar_arrive_tc(unit_full + 8 * slot);
        }
        __syncwarp();
        if (!more) break;
        const int key0 = un.k0, n_all = un.tiles();
        auto load_q = [&](int w) {
          if (ok && done[w] > 0) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_qfree + 8 * w, (done[w] - 1) & 1));
          if (!ok) return;
          const int head = uniform(un.head(w)), token = uniform(un.q0 + un.first_row(w) + 128 * rank);
          mbar_expect_tx_if(first, bar_q + 8 * w, 2 * kFQLines * kFQLine);
#pragma unroll
          for (int ln = 0; ln < kFQLines; ++ln)
            tma_load_4d_pair_if(leader, u_q + (w * kFQLines + ln) * kFQLine, &maps.q, to_q + 8 * w, ln, head, token);
          ++done[w];
        };
        if (un.n0 > 0) load_q(0);
        for (int i = 0; ok && i < n_all; ++i, ++t) {
          const int u_h = uniform(un.head(un.half_of(i)));
          const int st = uniform(t % kFStages), rnd = t / kFStages;
          if (rnd > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty_k + 8 * st, (rnd - 1) & 1));
          if (!ok) break;
          const int set = un.dual ? 1 + (i & 1) : 0;
          const int count = set == 0 ? counts[0] : set == 1 ? counts[1] : counts[2];
          const uint32_t bar = uniform(tile_bar(full_k, set, count)), to_k = uniform(in_cta(bar, 0));
          if (set == 0) ++counts[0]; else if (set == 1) ++counts[1]; else ++counts[2];
          mbar_expect_tx_if(first, bar, 2 * kFKBytes);
          const int key = uniform(key0 + un.keys_of(i) * kFKeys), my_key = key + 64 * rank;
          const uint32_t kd = u_k + st * kFKBytes;
          tma_load_4d_pair_if(leader, kd, &maps.k_nope, to_k, 0, u_h, my_key);
          tma_load_4d_pair_if(leader, kd + kFKLine, &maps.k_nope, to_k, 1, u_h, my_key);
          tma_load_4d_pair_if(leader, kd + 2 * kFKLine, &maps.k_rope, to_k, 0, 0, my_key);
          if (i == 0 && un.n1 > 0) load_q(1);
          if (ok && rnd > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty_v + 8 * st, (rnd - 1) & 1));
          if (!ok) break;
          mbar_expect_tx_if(leader, full_v + 8 * st, kFVBytes);
          tma_load_4d_if(leader, u_v + st * kFVBytes, &maps.v, full_v + 8 * st, rank, u_h, key);
        }
        if (!ok) break;
      }
      if (!ok) {  // copies in flight end before the CTA does: they are given time (a millisecond; a copy takes microseconds)
        if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
        for (int k = 0; k < 256; ++k) mbar_wait_bounded(bar_never, 0, 1);  // (4 us a poll)
      }
    } else if (warp == kFRelay) {
      // ================= V tiles: cleared behind the sequence's end, then handed to the first CTA =================
      int counts[3] = {0, 0, 0};  // tiles so far by set of barriers
      FUnit un;
      int t = 0;
      for (int k = 0; next_unit(k, un); ++k) {
        free_unit(k);
        const int n_all = un.tiles();
        for (int i = 0; ok && i < n_all; ++i, ++t) {
          const int st = t % kFStages;
          ok = __all_sync(0xffffffffu, mbar_wait_bounded(full_v + 8 * st, (t / kFStages) & 1));
          if (!ok) break;
          const int valid = max(un.nk - un.keys_of(i) * kFKeys, 0);
          if (valid < kFKeys) {
            // (keys behind the end have weight 0, but what they hold may be anything)
            for (int c = lane; c < (kFKeys - valid) * 8; c += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(v_sm + st * kFVBytes + valid * 128 + c * 16), "r"(0));
            fence_proxy_async();
          }
          const int set = un.dual ? 1 + (i & 1) : 0;
          const int count = set == 0 ? counts[0] : set == 1 ? counts[1] : counts[2];
          const uint32_t to = in_cta(tile_bar(v_ready, set, count), 0);
          if (set == 0) ++counts[0]; else if (set == 1) ++counts[1]; else ++counts[2];
          __syncwarp();
          if (lane == 0) {
            if (valid < kFKeys) arrive_cluster(to);  // (with what has been written before it)
            else arrive_cluster_tc(to);
          }
        }
        if (!ok) break;
      }
      if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    } else if (warp == kFMma && rank == 0) {
      issue_role(std::integral_constant<int, 0>{});
    } else if (warp == kFMma + 1 && rank == 0) {
      issue_role(std::integral_constant<int, 1>{});
    } else if (warp == kFMma && pair == 0 && plan.slots > 0) {
      for (int b = lane; b < p.batch; b += 32) prefill_span(p, b);  // (reports sequences that no place leads to)
    }
  } else {
    reg_alloc_inc<kFRegsSoftmax>();
    // ================= softmax and output: thread = row =================
    const int w = warp >> 2;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t my_s = tmem + 128 * w + lane_base, my_o = tmem + kFTmemO + 128 * w + lane_base;
    const float scale_log2 = p.scale * 1.4426950408889634f;
    const uint32_t to_p = in_cta(bar_p + 16 * w, 0), to_ofree = in_cta(bar_ofree + 8 * w, 0);
    const float neg_inf = -INFINITY;
    int t = 0, merges = 0;  // tiles of this half, merges with the second half so far
    for (int unit = 0;; ++unit) {
      int n, seen;  // tiles; columns that this thread's row sees, from the half's first tile on
      // The row's reference, a score as it comes from the product, and the factor that goes with it. A row behind the
      // sequence's last is another sequence's, or anything: its reference is infinite, so that it never asks for the
      // warp's to be raised and has no say in the other rows' rounding.
      float m_ref, c_ref;
      {
        FUnit un;
        if (!next_unit(unit, un)) break;
        n = w == 0 ? un.n0 : un.n1;
        const int row = un.first_row(w) + 128 * rank + (tid & 127);
        // (a warp without any row sees nothing; one with some goes by the mask, so as not to take the slower way)
        seen = row - lane < un.nq ? min(un.nk, un.nk - un.nq + row + 1) - un.key_tile(w, 0) * kFKeys : 0;
        m_ref = row < un.nq ? kFNoMax : INFINITY;
      }
      c_ref = score_factor(m_ref, scale_log2);
      float l = 0.f;
      // One tile; masked: some row of the warp does not see all of it.
      auto tile = [&](auto masked, int j) {
        constexpr bool kMasked = decltype(masked)::value;
        const int vis = seen - j * kFKeys;  // visible columns of this row
        // 64 keys at a time; the first run's products start while the second run is here
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (kRuns || k == 0) {
            if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_s + 16 * w + 8 * k, t & 1));
            if (!ok) return;
            tc_fence_after();
          }
          uint32_t sv[64];
          tmem_ld32(my_s + 64 * k, *reinterpret_cast<uint32_t(*)[32]>(&sv[0]));
          tmem_ld32(my_s + 64 * k + 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[32]));
          tmem_wait_ld();
          // keys of the run's columns: 64 k + e, or 32 k + e, from the 32nd on 32 k + 32 + e
          const int vis_lo = vis - (kRuns ? 32 * k : 64 * k), vis_hi = vis - (kRuns ? 32 * k + 32 : 64 * k);
          if (kMasked) {
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (e >= (e < 32 ? vis_lo : vis_hi)) sv[e] = 0xff800000u;  // -inf
          }
          if (k == 0 && j == 0) {  // the first reference: the maximum of the first 64 scores
            float mx[2] = {neg_inf, neg_inf};
#pragma unroll
            for (int e = 0; e < 64; e += 2) mx[(e >> 1) & 1] = max3(mx[(e >> 1) & 1], __uint_as_float(sv[e]), __uint_as_float(sv[e + 1]));
            m_ref = fmaxf(m_ref, fmaxf(mx[0], mx[1]));
            c_ref = score_factor(m_ref, scale_log2);
          }
          // Weights relative to the reference as it stands, the maximum taken along the way: rarely does it pass the
          // reference by so much that the reference is raised and the weights are taken again.
          uint32_t pk[32];
          float part;
          float top;
          auto weights = [&](auto poly) {
            const float minus_ref = -__fmul_rn(m_ref, c_ref);
            const uint64_t ref2 = f32x2(__float_as_uint(minus_ref), __float_as_uint(minus_ref));
            const uint64_t c2 = f32x2(__float_as_uint(c_ref), __float_as_uint(c_ref));
            uint64_t sum2[2] = {0ull, 0ull};
            float mx[2] = {neg_inf, neg_inf};
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const uint64_t x = fma_f32x2(f32x2(sv[2 * e], sv[2 * e + 1]), c2, ref2);
              mx[e & 1] = max3_nan(mx[e & 1], __uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1]));
              float w0, w1;
              if (decltype(poly)::value && e % kFPolyOf == kFPolyOf - 1) {
                exp2_pair(x, w0, w1);
              } else {
                f32x2_split(x, w0, w1);
                w0 = ex2(w0);
                w1 = ex2(w1);
              }
              sum2[e & 1] = add_f32x2(sum2[e & 1], f32x2(__float_as_uint(w0), __float_as_uint(w1)));
              pk[e] = pack2<false>(w0, w1);
            }
            float s0, s1;
            f32x2_split(add_f32x2(sum2[0], sum2[1]), s0, s1);
            part = s0 + s1;
            top = max3_nan(mx[0], mx[0], mx[1]);
            if (!(top <= 3.4028235e38f)) part = __uint_as_float(0x7fc00000u);  // a NaN or +inf among the scores
          };
          while (true) {
            if (kMasked && __all_sync(0xffffffffu, vis_lo <= 0)) {  // no row of the warp sees any of these
#pragma unroll
              for (int e = 0; e < 32; ++e) pk[e] = 0;
              part = 0.f;
              break;
            }
            weights(std::bool_constant<!kMasked>{});  // (weights of hidden keys are exactly zero)
            if (!__any_sync(0xffffffffu, top * c_ref > m_ref * c_ref + kFRescale)) break;
            const float m_new = fmaxf(m_ref, top), c_new = score_factor(m_new, scale_log2);
            const float a = rescale(m_ref, m_new, c_new);
            m_ref = m_new;
            c_ref = c_new;
            l *= a;
            if (j > 0 || k > 0) {  // O so far: up to the last tile, or to the first run of this one
              if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 16 * w + 8 * (k ^ 1), (k == 0 ? t - 1 : t) & 1));
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < 8; ++c) {
                uint32_t ov[16];
                tmem_ld16(my_o + 16 * c, ov);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * a);
                tmem_st16(my_o + 16 * c, ov);
              }
            }
          }
          if (!ok) return;
          l += part;
          tmem_st32(my_s + kRunP * k, pk);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster_tc(to_p + 8 * k);
        }
      };
      // (the tiles that every row of the warp sees come first)
      const int n_full = min(n, __reduce_min_sync(0xffffffffu, max(seen, 0)) / kFKeys);
      for (int j = 0; ok && j < n_full; ++j, ++t) tile(std::false_type{}, j);
      for (int j = n_full; ok && j < n; ++j, ++t) tile(std::true_type{}, j);
      // ---- output
      if (n > 0) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 16 * w + 8, (t - 1) & 1));
        tc_fence_after();
      }
      const FUnit un = units[unit % kFUnitSlots];  // (read again: it takes registers that the loop above needs)
      free_unit(unit);
      const int row = un.first_row(w) + 128 * rank + (tid & 127);  // query token of the sequence
      const bool split = un.dual == kSplitKeys;
      float* sums = merge_sh + 2 * (tid & 127);  // the row's reference and sum from the second half
      if (split && w == 1) {  // the first half's warp of the same rows takes it from here
        *reinterpret_cast<float2*>(sums) = make_float2(m_ref, l);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_tc(bar_merge + 8 * (warp & 3));
        if (!ok) break;
        continue;
      }
      // (warp-uniform; the second half of a block with at most kFHalf rows has none, unless they are the next head's)
      const bool rows_here = un.first_row(w) + 128 * rank + (warp & 3) * 32 < un.nq;
      if (split) {  // O and the sum of both halves, in the first half's place
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_merge + 8 * (warp & 3), merges & 1));
        tc_fence_after();
        ++merges;
        const float2 other = *reinterpret_cast<const float2*>(sums);
        const float m = fmaxf(m_ref, other.x);
        const float c_new = score_factor(m, scale_log2);
        const float mul = rescale(m_ref, m, c_new), mul_other = rescale(other.x, m, c_new);
        l = l * mul + other.y * mul_other;
#pragma unroll 1
        for (int c = 0; c < 8; ++c) {
          uint32_t ov[16], o2[16];
          tmem_ld16(my_o + 16 * c, ov);
          tmem_ld16(my_o + 128 + 16 * c, o2);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(fmaf(__uint_as_float(o2[e]), mul_other, __uint_as_float(ov[e]) * mul));
          tmem_st16(my_o + 16 * c, ov);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster_tc(to_ofree + 8);  // (the second half's O has been read)
      }
      // A row that sees keys has a score at its reference, of weight 1 or (c r rounded) a little less, unless none of them is
      // finite: then it has no softmax and is NaN. (The polynomial gives such scores 2^-126.)
      const bool some = n > 0 && ok && un.nk - un.nq + row >= 0;
      const float inv = 1.f / (l < 5.4210109e-20f ? NAN : l);  // 2^-64
      __nv_bfloat16* out = p.out + (static_cast<int64_t>(un.q0) + row) * p.out_token_stride + un.head(w) * p.out_head_stride;
      // A thread stores its own row, 32 bytes (a whole sector) at a time where the rows' alignment allows it.
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0 && p.out_token_stride % 16 == 0 && p.out_head_stride % 16 == 0;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t ov[32];
        tmem_ld32(my_o + 32 * c, ov);
        tmem_wait_ld();
        if (c == 3 && n > 0) {  // O is in registers: the next unit's products may write it
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster_tc(to_ofree);
        }
        if (rows_here && row < un.nq) {
#pragma unroll
          for (int e = 0; e < 32; e += 2)
            ov[e >> 1] = some ? pack2<false>(__uint_as_float(ov[e]) * inv, __uint_as_float(ov[e + 1]) * inv) : 0u;
#pragma unroll
          for (int k = 0; k < 16; k += 8) {
            __nv_bfloat16* dst = out + 32 * c + 2 * k;
            if (wide) {
              asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(ov[k]), "r"(ov[k + 1]), "r"(ov[k + 2]),
                           "r"(ov[k + 3]), "r"(ov[k + 4]), "r"(ov[k + 5]), "r"(ov[k + 6]), "r"(ov[k + 7]) : "memory");
            } else {
              reinterpret_cast<uint4*>(dst)[0] = make_uint4(ov[k], ov[k + 1], ov[k + 2], ov[k + 3]);
              reinterpret_cast<uint4*>(dst)[1] = make_uint4(ov[k + 4], ov[k + 5], ov[k + 6], ov[k + 7]);
            }
          }
        }
      }
      if (!ok) break;
    }
    if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
  }

  // ---- teardown: neither CTA leaves while the other may still reach its barriers or tensor memory
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && *cta_err) report(p.status, *cta_err);
  cluster_sync();
  if (warp == kFMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kFTmemCols) : "memory");
  }
}

// [tokens][heads][lines][64]: a copy takes one line of box_tokens tokens of one head
bool encode_rows(EncodeFn enc, CUtensorMap* map, const void* base, int64_t dim, int64_t heads, int64_t tokens, int64_t head_stride,
                 int64_t token_stride, int box_tokens) {
  const cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(dim / 64), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
  // (a dimension of extent 1 is never stepped over)
  const cuuint64_t strides[3] = {128, heads == 1 ? 128 : static_cast<cuuint64_t>(head_stride) * 2,
                                 tokens == 1 ? 128 : static_cast<cuuint64_t>(token_stride) * 2};
  const cuuint32_t box[4] = {64, 1, 1, static_cast<cuuint32_t>(box_tokens)};
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
  if (p.total_q > INT32_MAX - 1024 || p.total_k > INT32_MAX - 1024) return false;
  return static_cast<int64_t>((p.max_q + kFRows - 1) / kFRows) * p.batch <= INT32_MAX;
}

cudaError_t launch_latent_prefill_tc(const LatentPrefillParams& p, cudaStream_t stream) {
  EncodeFn enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  FMaps maps{};
  if (!encode_rows(enc, &maps.q, p.q, 192, p.num_heads, p.total_q, p.q_head_stride, p.q_token_stride, 128) ||
      !encode_rows(enc, &maps.k_nope, p.k_nope, 128, p.num_heads, p.total_k, p.kn_head_stride, p.kn_token_stride, 64) ||
      !encode_rows(enc, &maps.k_rope, p.k_rope, 64, 1, p.total_k, 0, p.kr_token_stride, 64) ||
      !encode_rows(enc, &maps.v, p.v, 128, p.num_heads, p.total_k, p.v_head_stride, p.v_token_stride, kFKeys))
    return cudaErrorNotSupported;
  // One pair of CTAs per two SMs at most; the row blocks of all sequences are at most one a sequence and one for
  // every kFRows query tokens.
  int dev = 0, sms = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  const int q_blocks = (p.max_q + kFRows - 1) / kFRows;
  const int64_t most = std::min(static_cast<int64_t>(p.batch) + p.total_q / kFRows, static_cast<int64_t>(p.batch) * q_blocks);
  // Not listed, the sequences' last possible blocks come first (their keys are the most). Where the sequences differ so
  // much that most of these places would be empty, the places are counted by the tokens instead.
  const int64_t places = static_cast<int64_t>(p.batch) + p.total_q / kFRows;
  const int listed = most <= kFMaxList ? 1 : 0;
  const FPlan plan{q_blocks, listed, !listed && static_cast<int64_t>(p.batch) * q_blocks > 4 * places ? places : 0};
  const int64_t pairs = std::min(most * p.num_heads, static_cast<int64_t>(std::max(sms / 2, 1)));
  // S in two runs where the units have many tiles: very many keys a sequence and rows enough for both halves, or fewer
  // units than pairs of CTAs (then the chain of one half is what is left, not power or copies). Both ways measured (at
  // once, in two runs): a prompt of 8192, 32 heads 625 and 613 us; chunks of 500..1024 behind 1000..16384, 16 heads
  // 170 and 165; 7 chunks of 8..408 behind 1500..3000, 4 heads 62 and 52; but prompts of 1..700, 16 heads 75 and 78;
  // chunks of 700 behind 1500..3000, 16 heads 178 and 188; 40 chunks of 24 behind 2000..4000, 16 heads 316 and 339.
  // (By what the call's totals say, not by max_q: the result does not depend on how loose a bound that is.)
  const bool runs = places * p.num_heads <= sms / 2 ? p.total_k >= 1024ll * p.batch
                                                    : p.total_k >= 4096ll * p.batch && p.total_q >= static_cast<int64_t>(kFHalf) * p.batch;
  const auto kernel = runs ? latent_prefill_tc_kernel<true> : latent_prefill_tc_kernel<false>;
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFSmemBytes)) != cudaSuccess) return e;
  kernel<<<static_cast<unsigned>(2 * pairs), kFThreads, kFSmemBytes, stream>>>(maps, p, plan);
  return cudaGetLastError();
}

}  // namespace pda
