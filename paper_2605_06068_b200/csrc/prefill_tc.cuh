// Attention of packed ragged prompts over the paged cache on tcgen05 + TMEM, with shaped scores.
//
// The query rows of a kv head are (token, head of the group): 128 / group tokens fill the 128 rows (TMEM lanes) of a CTA, so
// that a key tile serves the whole group. A pair of CTAs (a cluster of two SMs, tcgen05 cta_group::2) takes a block of four
// times as many tokens as two halves of 256 rows, 128 of each in either CTA, and walks over the keys 128 at a time (8 pages):
//   S[w] = Q[w] . K^T    M256 N128; of K each CTA holds 64 keys (4 pages)
//   O[w] += P[w] . V     M256 N128; P (bf16) in tensor memory over the S it came from; of V each CTA holds 64 of the 128 dims
//                        (head_dim 64: both hold all 64, and O comes out twice; the exponentials bound that case)
// S[0], S[1], O[0], O[1] fill the 512 TMEM columns. A thread is a row's softmax and takes 64 keys at a time.
// The softmax takes weights relative to a reference per row that is raised (and O rescaled in tensor memory) only when
// the row's maximum passes it by more than 2^32; row sums are kept by the row's thread, of the 32-bit weights.
// Warps of each CTA: 0-3, 4-7 softmax of the halves, 8 TMA producer, 9 and 10 MMA issue of the halves (in the pair's first
// CTA; 9: TMEM), 11 hands V tiles on, clearing what lies behind the sequence's end. All waits are bounded.
// Measured (B200, 32 query and 8 kv heads of 128, a call at a time): a prompt of 8192 tokens 442 us (1.24 PFLOP/s), capped at 50 533,
// biased 519, e4m3 600; 24 prompts of 1..700 tokens 96 us, capped 115; 300 tokens behind 60000 in 72 parts 317 us (860 uncut). Tensor
// pipe 52 % of active clocks, capped 42 %: the softmax's instructions and the products take turns.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "pair_ptx.cuh"
#include "shaped.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_ptx.cuh"

namespace pda {

// What a launch decides for all CTAs.
struct PrefillPlan {
  int q_blocks;   // blocks of max_q
  int tile_rows;  // query tokens of 128 rows
  int listed;     // the row blocks of all sequences are few enough to be listed and sorted in shared memory
  int64_t slots;  // (not listed) row blocks are looked for at this many places
  int cut;        // few units: blocks are cut along the keys, so that every pair has a part
  float scale_log2;
  // Capped scores as polynomials of the product s (each coefficient twice, for pairs of scores): of degree 5 for
  // |s| <= limit[0], of degree 11 for |s| <= limit[1]; u = scale / softcap. relative: poly11 is that of cap_score, in u s, times
  // s, and scores are taken one by one. ref: the fixed reference (capped only), or 0; ref_low: that of rows with low scores, whose
  // products are above low_limit in size.
  float limit[2], ref, ref_low, low_limit, u;
  int relative;
  uint64_t poly5[3], poly11[6];
};
struct PrefillMaps {
  CUtensorMap q, k, v;
};
// Workspace of a cut launch: per pair of CTAs one part's 512 rows of sums (fp32), references and sums, and a record.
struct PrefillRecord {
  int parts, row0, h, q0, nq, pad[3];  // parts of the row block that start here (0: none starts here)
};
constexpr int kPreMaxPairs = 74;       // a device with more SMs uses this many where blocks are cut
constexpr int kPreRows = 512;
constexpr int kPreCutKeys = 2048;      // keys that the block table has room for, below which nothing is cut
__host__ __device__ constexpr int64_t prefill_part_bytes(int head_dim) { return static_cast<int64_t>(kPreRows) * head_dim * 4; }
__host__ __device__ constexpr int64_t prefill_sums_at(int head_dim) { return kPreMaxPairs * prefill_part_bytes(head_dim); }
__host__ __device__ constexpr int64_t prefill_records_at(int head_dim) { return prefill_sums_at(head_dim) + kPreMaxPairs * kPreRows * 8; }

namespace {

constexpr int kGKeys = 128;  // keys per tile
constexpr int kGQLine = 128 * 128, kGKLine = 64 * 128;
constexpr int kGSoftWarps = 8, kGProducer = 8, kGMma = 9, kGRelay = 11, kGConvert = 12;
constexpr int kGScaleSlots = 8;  // tiles whose page scales are kept (e4m3): more than both rings hold together
constexpr int kGBookBytes = 9 * 1024;
constexpr uint32_t kGTmemCols = 512, kGTmemO = 256;
constexpr int kGUnitSlots = 4;   // units the producer may be ahead
constexpr int kGMaxList = 256;   // row blocks that are sorted by their work
constexpr float kGNoMax = -FLT_MAX;
// A row's reference is raised once a score passes it by 2^32: weights and their sums are floating-point numbers of 8 exponent
// bits, whose precision does not depend on their size, and 32 leaves values up to 2^64 room. With 2^8 (scores of +-15: a warp
// raises on half of its tiles) a prompt of 8192 tokens took 934 us instead of 570.
constexpr float kGRescale = 32.f;
constexpr int kGPolyOf = 4;      // every fourth pair of exponentials by polynomial
constexpr int kGMinTiles = 4;    // of a part
// Capped scores that are not biased lie within [-C, C] (ScoreParams): they need no maximum. Their weights are taken relative
// to a reference fixed at max(C - 30, 0), which keeps them within 2^-120 .. 2^30 for C <= 75 (a cap up to 52). A weight is multiplied
// with values, and with their page's scale, that may be small too. So, where weights could be below 2^-60 (C > 45, a cap above 31: kShapeLow),
// a row whose first 64 keys together weigh less than that (as the first tokens of a prompt may, or all, if their scores lie near -C) goes
// on at C - 100, from where it returns once 64 keys weigh more than 2^36: its largest weight is never below 2^-60. Rows whose first
// products are small are not looked at. The code for it costs 2 % of a prompt of 8192 tokens and 4 % of 24 of 1..700, although it
// hardly runs (instruction caches: in front of the weights it cost 5 and 15 %, as a second copy of the loop 7 and 21 %).
constexpr float kGFixedTop = 30.f, kGFixedCap = 75.f, kGFixedFloor = 60.f, kGFixedLow = 100.f;
constexpr float kGFixedLeast = 8.6736174e-19f, kGFixedMost = 68719476736.f;  // 2^-60, 2^36

// How scores are shaped (bits): capped; biased by distance; capped alone, with a fixed reference that rows may lie far below.
enum : int { kShapeNone = 0, kShapeCap = 1, kShapeBias = 2, kShapeLow = 4 };

// e4m3 caches: tiles land in a ring of bytes and are converted to bf16 (exactly) by a warpgroup of their own; the page scales
// go through the softmax.
template <int D, bool kFp8>
struct GCfg {
  static constexpr int kLines = D / 64;
  static constexpr int kStages = kFp8 ? 3 : D == 128 ? 4 : 6;
  static constexpr int kRaw = kFp8 ? 3 : 0;         // tiles as bytes
  static constexpr int kRawBytes = 64 * 128;        // K: 64 keys; V: 64 dims of 128 keys
  static constexpr int kThreads = (kGSoftWarps + 4 + (kFp8 ? 4 : 0)) * 32;
  // 384 threads start with 168 registers (64512 in all), 512 with 128 (65536)
  static constexpr uint32_t kRegsSoftmax = kFp8 ? 184 : 200, kRegsControl = kFp8 ? 72 : 104;
  static_assert(kGSoftWarps * 32 * kRegsSoftmax + (kThreads - kGSoftWarps * 32) * kRegsControl <= kThreads * (kFp8 ? 128 : 168), "registers");
  static constexpr int kKBytes = kLines * kGKLine;  // of its 64 keys
  static constexpr int kVBytes = kGKeys * 128;      // its line (64 dims) of all keys
  static constexpr int kQBytes = kLines * kGQLine;  // of a half
  static constexpr int kRing = 2 * kQBytes;
  static constexpr int kRawAt = kRing + kStages * (kKBytes + kVBytes);
  static constexpr int kBook = kRawAt + kRaw * 2 * kRawBytes;
  static constexpr int kBars = (9 * kStages + 32 + 4 * kRaw + kGScaleSlots + 1) / 2 * 2;
  static constexpr int kSmemBytes = kBook + kGBookBytes + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory");
};

// 2^x for two x <= 2^7 on the FMA units: x = n + f with n the nearest integer, 2^f by the polynomial of degree 3 whose
// largest relative error over [-1/2, 1/2] is least (7.5e-5, by Remez exchange; a weight's rounding to bf16 is 3.9e-3),
// n added to the exponent. x below -126 gives 2^-126, and so does a NaN: that is looked for in the scores' maximum.
__device__ __forceinline__ void exp2_two(uint64_t x, float& w0, float& w1) {
  auto both = [](float v) { return f32x2(__float_as_uint(v), __float_as_uint(v)); };
  float x0, x1;
  f32x2_split(x, x0, x1);
  x = f32x2(__float_as_uint(fmaxf(x0, -126.f)), __float_as_uint(fmaxf(x1, -126.f)));
  const uint64_t t = add_f32x2(x, both(12582912.f));  // 1.5 * 2^23
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
__device__ __forceinline__ uint32_t bits_before(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// Scores that are not shaped stay as they come from the product: weights are 2^(c s - c r), s the scores and r the
// reference, by one fused multiply-add with c r rounded: off by half a step of c r, the same for all of the row, so it
// cancels in the quotient. c is the scale as long as |c r| < 2^28, where that is at most 2^8. Beyond, scores that differ at
// all differ by 16 and more there, so that only the largest one weighs anything in 32 bits, and by any c that is large enough:
// then c is a power of two with 2^31 <= |c r| < 2^32, c r is exact, and other scores are 2^7 and more away.
constexpr float kGFar = 268435456.f;
__device__ __forceinline__ float score_factor(float r, float scale_log2) {
  if (fabsf(r * scale_log2) < kGFar) return scale_log2;
  const uint32_t exponent = (__float_as_uint(r) >> 23) & 255u;
  return __uint_as_float(min(127u + 31u + 127u - min(exponent, 254u), 254u) << 23);
}
// What weights and sums taken at reference `from` are multiplied by to be those at a reference `to` >= from: with the factor that the
// weights were taken with, so that a score of `to` among them, which weighed up to 2^32, comes out as 1, whichever factor `to` goes with.
// scale_log2 = 0: references in the exponent's units, whose factor is always 1.
__device__ __forceinline__ float rescale(float from, float to, float scale_log2) {
  if (scale_log2 == 0.f) return ex2(from - to);
  const float z_from = __fmul_rn(from, scale_log2), z_to = __fmul_rn(to, scale_log2);
  if (fabsf(z_from) < kGFar && fabsf(z_to) < kGFar) return ex2(z_from - z_to);  // (nearly always)
  const float c = score_factor(from, scale_log2);
  if (c == score_factor(to, scale_log2)) return ex2(__fmul_rn(from, c) - __fmul_rn(to, c));
  return ex2(-fmaf(to, c, -__fmul_rn(from, c)));
}

// O of a warp's rows in tensor memory, times `a` (each row its own). Out of line: it is rare, and the hot loop's code has to stay in the
// instruction caches.
template <int D>
__device__ __noinline__ void rescale_columns(uint32_t my_o, float a) {
#pragma unroll 1
  for (int c = 0; c < D / 16; ++c) {
    uint32_t ov[16];
    tmem_ld16(my_o + 16 * c, ov);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * a);
    tmem_st16(my_o + 16 * c, ov);
  }
}

// One row block of one kv head (or a part of its keys), as the producer hands it to the other warps of its CTA. row0 < 0: no
// more. Rows are counted in query tokens of the sequence. dual: the block fits one half and both halves take the same
// rows, with tiles of their own by turns: kTwoHeads: the second half's are the next head's; kSplitKeys: the second half's are
// the later n1 tiles of the same head, and the first half's warps merge the two results.
enum : int { kOneHead = 0, kTwoHeads = 1, kSplitKeys = 2 };
struct GUnit {
  // tile0: first 128 keys; slot >= 0: a part (keys before key_end), its place in the workspace; gaps: there may be keys between that
  // no row sees
  int row0, h, q0, nq, L, prefix, tile0, n0, n1, dual, slot, key_end, bad, gaps;
  __device__ int first_row(int w, int half_rows) const { return row0 + (dual ? 0 : half_rows * w); }
  __device__ int head(int w) const { return h + (dual == kTwoHeads ? w : 0); }
  __device__ int tiles() const { return dual ? n0 + n1 : max(n0, n1); }
  // The pair's i-th tile: whose half's (where that matters), and which 128 keys from tile0 on, the last ones first (down) or the
  // first ones. Of a block of two halves both read the pair's tiles up to their own last one; down, from it on.
  __device__ int half_of(int i) const { return i & 1; }
  __device__ int keys_of(int i, bool down) const {
    if (!dual) return down ? tiles() - 1 - i : i;
    return key_tile(i & 1, down ? (i & 1 ? n1 : n0) - 1 - (i >> 1) : i >> 1);
  }
  __device__ int key_tile(int w, int j) const { return dual == kSplitKeys && w ? n0 + j : j; }
  __device__ int skipped(int w, bool down) const { return dual || !down ? 0 : tiles() - (w ? n1 : n0); }
};
constexpr int kGBuckets = 64;
constexpr uint32_t kGSmallBlock = 1u << 30;  // (in a list entry) fits one half
__device__ __forceinline__ int units_of(uint32_t entry, int heads, bool by_two) {
  return by_two && (entry & kGSmallBlock) ? (heads + 1) / 2 : heads;
}

// A page's line into this CTA, its bytes counted at a barrier of either CTA of the pair. A page number at or beyond the
// cache's is read as zeros.
__device__ __forceinline__ void tma_load_page_pair_if(uint32_t leader, uint32_t dst, const CUtensorMap* map, uint32_t bar, int line, int head,
                                                      int page) {
  asm volatile(
      "{\n\t.reg .pred pe;\n\tsetp.ne.b32 pe, %6, 0;\n\t"
      "@pe cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {0, 0, %3, %4, %5}], [%2];\n\t}"
      ::"r"(dst), "l"(map), "r"(bar), "r"(line), "r"(head), "r"(page), "r"(leader) : "memory");
}

template <int D, int kShape, bool kFp8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GCfg<D, kFp8>::kThreads, 1)
prefill_tc_kernel(const __grid_constant__ PrefillMaps maps, const __grid_constant__ PrefillParams p,
                  const __grid_constant__ PrefillPlan plan) {
  using C = GCfg<D, kFp8>;
  constexpr int kStages = C::kStages;
  constexpr bool kCap = (kShape & kShapeCap) != 0, kBias = (kShape & kShapeBias) != 0;
  constexpr bool kFixed = kCap && !kBias;          // ... and lie within bounds: the reference is fixed
  constexpr bool kLow = (kShape & kShapeLow) != 0;
  // References in the exponent's units: of scores whose factor is not the same for all keys (a bias, e4m3's page scales).
  constexpr bool kExp = kBias || (kFp8 && !kFixed);
  constexpr bool kDown = kBias;                    // a bias has the scores rise from tile to tile: the last tiles come first
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBook);
  uint32_t* work = reinterpret_cast<uint32_t*>(bars + C::kBars);    // [kGMaxList] tiles, then units of the entries before
  uint32_t* list = work + kGMaxList;                                // [kGMaxList] sequence and block, most work first
  GUnit* units = reinterpret_cast<GUnit*>(list + kGMaxList);        // [kGUnitSlots]
  uint32_t* scan = reinterpret_cast<uint32_t*>(units + kGUnitSlots);  // [kGMaxList / 32] by warp, then the sum of all
  uint32_t* tmem_slot = scan + kGMaxList / 32 + 1;
  int* cta_err = reinterpret_cast<int*>(tmem_slot + 1);
  uint32_t* target_sh = reinterpret_cast<uint32_t*>(cta_err + 1);   // tiles of a part
  uint32_t* most_sh = target_sh + 1;                                // tiles of the block that has most
  float* merge_sh = reinterpret_cast<float*>(most_sh + 2);          // [128][2]
  static_assert(sizeof(GUnit) * kGUnitSlots % 8 == 0 && (kGMaxList / 32 + 1 + 5) % 2 == 0, "pairs of floats on 8 bytes");
  float* scales_sh = merge_sh + 256;                                // (e4m3) [kGScaleSlots][8 pages][K, V]
  int4* spans = reinterpret_cast<int4*>(reinterpret_cast<uint8_t*>(bars) + kGBookBytes - kGMaxList * 16);  // listed sequences' q0, nq, L
  uint32_t* hist = reinterpret_cast<uint32_t*>(smem);               // [kGMaxList / 32][kGBuckets], in Q's place, before its first copy
  uint32_t* bucket_sh = hist + kGMaxList / 32 * kGBuckets;          // [kGBuckets]
  static_assert(kGMaxList == 256 && kGMaxList <= (kGSoftWarps + 4) * 32, "sequence numbers of 8 bits, a thread each");
  static_assert(C::kBars * 8 + kGUnitSlots * sizeof(GUnit) + 2 * kGMaxList * 4 + (kGMaxList / 32 + 6) * 4 + 1024 + (kFp8 ? kGScaleSlots * 64 : 0) + kGMaxList * 16 <= kGBookBytes, "shared memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x & 1;  // in the pair
  const int pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  const int half_rows = 2 * plan.tile_rows, block_rows = 4 * plan.tile_rows;  // in query tokens
  const int heads = p.geom.num_kv_heads;
  bool ok = true;

  const uint32_t q_sm = smem_u32(smem), k_sm = q_sm + C::kRing, v_sm = k_sm + kStages * C::kKBytes;
  // Barriers, at the same place in both CTAs. Of the pair's first CTA: full_k (both CTAs' copies), v_ready, bar_q,
  // bar_p, bar_ofree. In each: empty_k, empty_v (both halves' products), full_v (its own copy), bar_s,
  // bar_pv, bar_qfree, the unit slots'. bar_s, bar_p and bar_pv: [half w][run of
  // 64 keys].
  const uint32_t full_k = smem_u32(bars), empty_k = full_k + 24 * kStages, full_v = empty_k + 8 * kStages,
                 empty_v = full_v + 8 * kStages, v_ready = empty_v + 8 * kStages, bar_q = v_ready + 24 * kStages;
  const uint32_t bar_s = bar_q + 16, bar_p = bar_s + 32, bar_pv = bar_p + 32, bar_qfree = bar_pv + 32,
                 bar_ofree = bar_qfree + 16, unit_full = bar_ofree + 16, unit_empty = unit_full + 8 * kGUnitSlots,
                 bar_drain = unit_empty + 8 * kGUnitSlots, bar_never = bar_drain + 8, bar_merge = bar_never + 8,
                 raw_full = bar_merge + 32, raw_empty = raw_full + 16 * C::kRaw, scale_full = raw_empty + 16 * C::kRaw;
  // (e4m3: raw_full and raw_empty [K, V][raw stage], scale_full [scale slot])
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      for (int set = 0; set < 3; ++set) {
        mbar_init(full_k + 8 * (kStages * set + i), kFp8 ? 8 : 1);  // (e4m3: four converting warps of each CTA)
        mbar_init(v_ready + 8 * (kStages * set + i), kFp8 ? 8 : 2);
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
      mbar_init(bar_qfree + 8 * w, 1);
      mbar_init(bar_ofree + 8 * w, 8);
    }
    for (int i = 0; i < kGUnitSlots; ++i) {
      mbar_init(unit_full + 8 * i, 1);
      mbar_init(unit_empty + 8 * i, kGSoftWarps + (kFp8 ? 4 : 1) + (rank == 0 ? 2 : 0));  // softmax, relay or converting, product warps
    }
    for (int i = 0; i < 2 * C::kRaw; ++i) {
      mbar_init(raw_full + 8 * i, 1);
      mbar_init(raw_empty + 8 * i, 4);
    }
    for (int i = 0; kFp8 && i < kGScaleSlots; ++i) mbar_init(scale_full + 8 * i, 1);
    mbar_init(bar_drain, 2);
    mbar_init(bar_never, 1);
    for (int i = 0; i < 4; ++i) mbar_init(bar_merge + 8 * i, 1);
    *cta_err = 0;
    *target_sh = 1u << 30;
    *most_sh = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == kGProducer && elect_one()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
  }
  if (warp == kGMma) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kGTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // The keys that the query tokens `row0` .. `last` of a sequence see where nothing but position, window and prefix matters: none
  // before `lo`, none from `hi` on, and each in between. (documents: the rows one by one, see make_unit)
  auto key_range = [&](int row0, int last, int nq, int L, int prefix, int& lo, int& hi) {
    const int first_pos = L - nq + row0, last_pos = L - nq + last;
    hi = last_pos < 0 ? 0 : max(last_pos + 1, min(prefix, L));
    lo = p.score.window > 0 ? max(max(first_pos, 0) - p.score.window + 1, 0) : 0;  // (rows before the sequence see nothing)
  };
  auto prefix_of = [&](int b) { return p.prefix_lens != nullptr ? p.prefix_lens[b] : 0; };

  // ---- the row blocks that there are, those with the most keys first (every CTA for itself, all alike)
  int my_blocks = 0, my_prefix = 0;
  SeqSpan mine{0, 0, 0};
  if (plan.listed && tid < kGMaxList && tid < p.batch) {
    mine = seq_span(p, tid);
    my_blocks = (mine.nq + block_rows - 1) / block_rows;
    my_prefix = prefix_of(tid);
    spans[tid] = make_int4(mine.q0, mine.nq, mine.L, my_prefix);
  }
  int incl = my_blocks;
  if (plan.listed && tid < kGMaxList) {
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
    for (int i = 0; i < kGMaxList / 32; ++i) {
      before += i < warp ? scan[i] : 0;
      n_blocks += scan[i];
    }
    // (ascending offsets give at most as many as the host has allowed for; others are reported)
    if (n_blocks > kGMaxList) {
      report(p.status, PDA_DEV_BAD_SEQ_LEN);
      n_blocks = kGMaxList;
    }
    // ... unless there is a pair of CTAs for each head of each block: half as many units are no gain then
    by_two = !plan.cut && static_cast<int64_t>(n_blocks) * heads > pairs;
    if (tid < kGMaxList) work[tid] = before;  // blocks of the sequences before
    for (int i = tid; i < kGMaxList / 32 * kGBuckets; i += C::kThreads) hist[i] = 0;
    __syncthreads();
    if (tid < n_blocks) {
      int seq = 0;  // the last sequence whose blocks start at or before this one
#pragma unroll 1
      for (int at = kGMaxList / 2; at > 0; at >>= 1)
        if (seq + at < p.batch && work[seq + at] <= static_cast<uint32_t>(tid)) seq += at;
      const int4 span = spans[seq];
      const int k = tid - static_cast<int>(work[seq]), row0 = k * block_rows;
      int lo, hi;
      key_range(row0, min(row0 + block_rows, span.y) - 1, span.y, span.z, span.w, lo, hi);
      if (p.first_keys != nullptr) lo = max(lo, p.first_keys[span.x + row0]);
      my_work = hi > lo ? (hi + kGKeys - 1) / kGKeys - lo / kGKeys : 0;
      my_entry = seq | (k << 8) | (span.y - row0 <= half_rows ? kGSmallBlock : 0u);
    }
    // Places by buckets of like work (the finest that hold the largest), by number within a bucket: a warp counts its 32 blocks by
    // matching, one adds up. (Each block compared with all: 200 of them 4 us.)
    const uint32_t most = __reduce_max_sync(0xffffffffu, my_work);
    if (lane == 0) atomicMax(most_sh, most);
    __syncthreads();  // (work has been read)
    const int shift = max(32 - __clz(*most_sh) - 6, 0);
    const uint32_t bucket = tid < n_blocks ? kGBuckets - 1 - (my_work >> shift) : kGBuckets + lane;
    const uint32_t same = __match_any_sync(0xffffffffu, bucket);
    const int in_bucket = __popc(same & ((1u << lane) - 1u));
    if (tid < n_blocks) {
      if (in_bucket == 0) hist[warp * kGBuckets + bucket] = __popc(same);
      work[tid] = my_work;
    }
    __syncthreads();
    if (warp == 0) {  // counts become counts before: of the blocks of earlier warps, and of all earlier buckets
      uint32_t total[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t run = 0;
#pragma unroll 1
        for (int i = 0; i < kGMaxList / 32; ++i) {
          const uint32_t x = hist[i * kGBuckets + lane + 32 * h];
          hist[i * kGBuckets + lane + 32 * h] = run;
          run += x;
        }
        total[h] = run;
      }
      uint32_t low = total[0], high = total[1];
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t a = __shfl_up_sync(0xffffffffu, low, o), b = __shfl_up_sync(0xffffffffu, high, o);
        if (lane >= o) low += a, high += b;
      }
      bucket_sh[lane] = low - total[0];
      bucket_sh[lane + 32] = __shfl_sync(0xffffffffu, low, 31) + high - total[1];
    }
    // Few units: the fewest tiles a part with which all parts find a pair each.
    if (plan.cut && warp == 1) {
      uint32_t below = kGMinTiles - 1, t = work[0];  // (below: too small, or not wanted)
      for (int i = lane; i < n_blocks; i += 32) t = max(t, work[i]);
      t = max(__reduce_max_sync(0xffffffffu, t), static_cast<uint32_t>(kGMinTiles));
      while (t - below > 1) {
        const uint32_t mid = (t + below) >> 1;
        uint32_t parts = 0;
        for (int i = lane; i < n_blocks; i += 32) parts += max((work[i] + mid - 1) / mid, 1u);
        if (static_cast<int64_t>(__reduce_add_sync(0xffffffffu, parts)) * heads <= pairs) t = mid; else below = mid;
      }
      if (lane == 0) *target_sh = t;
    }
    __syncthreads();  // (and `work` has been read)
    if (tid < n_blocks) {
      const uint32_t place = bucket_sh[bucket] + hist[warp * kGBuckets + bucket] + in_bucket;
      list[place] = my_entry;
      work[place] = my_work;
    }
    __syncthreads();
    uint32_t units = 0;
    if (tid < n_blocks) units = plan.cut ? heads * max((work[tid] + *target_sh - 1) / *target_sh, 1u) : units_of(list[tid], heads, by_two);
    const uint32_t my_units = units;
    if (tid < kGMaxList) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, units, o);
        if (lane >= o) units += u;
      }
      if (lane == 31) scan[warp] = units;
    }
    __syncthreads();
    uint32_t units_before = units - my_units;
    for (int i = 0; i < kGMaxList / 32; ++i) units_before += i < warp ? scan[i] : 0;
    if (tid < n_blocks) work[tid] = units_before;
    if (tid == 0) {
      uint32_t all = 0;
      for (int i = 0; i < kGMaxList / 32; ++i) all += scan[i];
      scan[kGMaxList / 32] = all;
    }
    fence_proxy_async();  // (the counts lay where Q is copied to)
  }
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // Unit number k of this CTA, for the warps that are told by the producer.
  auto next_unit = [&](int k, GUnit& un) {
    const int slot = k % kGUnitSlots;
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(unit_full + 8 * slot, (k / kGUnitSlots) & 1));
    if (!ok) return false;
    un = units[slot];
    return un.row0 >= 0;
  };
  auto free_unit = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive_tc(unit_empty + 8 * (k % kGUnitSlots));
  };

  // The barrier of a tile, from full_k or v_ready: both halves' tiles, the first half's and the second half's (dual
  // blocks) are counted each for themselves, so that who waits for a set's barriers follows all their phases. (kStages
  // tiles of a set are in the ring at most: a barrier's next use comes behind its last one's wait.)
  auto tile_bar = [&](uint32_t first, int set, int count) { return first + 8 * (kStages * set + count % kStages); };

  // ================= products of half w =================
  // A warp for each half, which prepares its next products while the other's are being issued. S comes in two runs of 64 keys
  // (32 of either CTA's), each taken again as soon as its own P . V is through, so that a half has scores of the next tile before
  // its softmax is done with this one. (S of 128 keys at once, the halves taking turns: 498 us instead of 454 for 8192 tokens.)
  auto issue_role = [&](auto half) {
    constexpr int w = decltype(half)::value;
    constexpr uint32_t idesc_s = latent_idesc(256, kGKeys / 2, false, false), idesc_o = latent_idesc(256, 128, false, true);
    const uint32_t leader = elect_one();
    const uint32_t u_q = uniform(q_sm + w * C::kQBytes), u_k = uniform(k_sm), u_v = uniform(v_sm), u_tmem = uniform(tmem);
    const uint32_t u_ek = uniform(empty_k), u_ev = uniform(empty_v);
    const uint32_t d_s = u_tmem + 128 * w, d_o = u_tmem + kGTmemO + 128 * w;
    auto wait = [&](uint32_t bar, int phase) {
      if (ok) ok = __all_sync(0xffffffffu, mbar_spin_cluster(bar, phase & 1));
    };
    // S of run k of a tile: of each CTA's 64 keys those from 32 k on
    auto s_product = [&](uint32_t k_addr, int k) {
      const uint64_t q0 = tc_desc(u_q, 16, 1024), k0 = tc_desc(k_addr, 16, 1024) + 256 * k;
#pragma unroll
      for (int ln = 0; ln < C::kLines; ++ln)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          mma2_ss_if(leader, d_s + 64 * k, q0 + ln * (kGQLine / 16) + 2 * ks, k0 + ln * (kGKLine / 16) + 2 * ks, idesc_s, (ln > 0 || ks > 0) ? 1u : 0u);
      commit2_if(leader, bar_s + 16 * w + 8 * k);
    };
    GUnit un;
    // Before this unit: tiles of the pair; of this half; units of this half.
    int t0 = 0, mine = 0, done = 0;
    int counts[2] = {0, 0};  // tiles of blocks of two halves; of dual ones, this half's
    for (int k = 0; next_unit(k, un); ++k) {
      free_unit(k);
      const int n = uniform(w == 0 ? un.n0 : un.n1), n_other = uniform(w == 0 ? un.n1 : un.n0);
      const int dual = uniform(un.dual);
      const int step = dual ? 2 : 1, own = dual ? w : 0;  // this half's tiles: t0 + step * j + own
      const int skip = uniform(un.skipped(w, kDown));
      const int set = dual ? 1 + w : 0, c0 = counts[dual ? 1 : 0] + skip;  // this unit's tiles on the set's barriers: c0 + j
      // Both halves give a tile of a block of two halves back. The one that does not read it does so as soon as it is
      // there (see tile_bar) and goes on. (j: counted from this half's first one)
      auto hand_on = [&](uint32_t full, uint32_t empty, int j) {
        wait(tile_bar(full, 0, c0 + j), (c0 + j) / kStages);
        if (ok && lane < 2) arrive_cluster_tc(in_cta(empty + 8 * ((t0 + skip + j) % kStages), lane));
        __syncwarp();
      };
      for (int j = -skip; ok && j < 0; ++j) {
        hand_on(full_k, empty_k, j);
        hand_on(v_ready, empty_v, j);
      }
      if (!ok) break;
      // (a tile of a dual block is given back twice by its half)
      auto give_back = [&](uint32_t bar) {
        commit2_if(leader, bar);
        if (dual) commit2_if(leader, bar);
      };
      if (n > 0) {  // S(0): its place is free, the tensor core works a thread's products off in order
        const int t = t0 + skip + own, sk = t % kStages;
        wait(bar_q + 8 * w, done);
        wait(tile_bar(full_k, set, c0), c0 / kStages);
        if (!ok) break;
        tc_fence_after();
        const uint32_t k_addr = uniform(u_k + sk * C::kKBytes);
        s_product(k_addr, 0);
        s_product(k_addr, 1);
        if (n == 1) commit2_if(leader, bar_qfree + 8 * w);
        give_back(uniform(u_ek + 8 * sk));
      }
      for (int j = 0; j < n; ++j) {
        const int t = t0 + skip + step * j + own, tn = t + step, sv = t % kStages, sk = tn % kStages;
        wait(tile_bar(v_ready, set, c0 + j), (c0 + j) / kStages);
        const uint64_t v0 = tc_desc(uniform(u_v + sv * C::kVBytes), 16, 1024);
        const uint32_t k_addr = uniform(u_k + sk * C::kKBytes), ev = uniform(u_ev + 8 * sv), ek = uniform(u_ek + 8 * sk);
        const uint32_t acc = uniform(j > 0 ? 1u : 0u);
        if (j == 0 && done > 0) wait(bar_ofree + 8 * w, done - 1);  // the last unit's output has been read
        // (run 0: keys 0 .. 31 and 64 .. 95 of the tile; run 1: 32 .. 63 and 96 .. 127)
        wait(bar_p + 16 * w, mine + j);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) mma2_ts_if(leader, d_o, d_s + 8 * ks, v0 + (ks < 2 ? 0 : 256) + 128 * ks, idesc_o, ks > 0 ? 1u : acc);
        commit2_if(leader, bar_pv + 16 * w);
        if (j + 1 < n) wait(tile_bar(full_k, set, c0 + j + 1), (c0 + j + 1) / kStages);
        if (j + 1 < n) {
          if (!ok) break;
          tc_fence_after();
          s_product(k_addr, 0);  // over these weights: the tensor core works a thread's products off in order
        }
        wait(bar_p + 16 * w + 8, mine + j);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) mma2_ts_if(leader, d_o, d_s + 64 + 8 * ks, v0 + (ks < 2 ? 256 : 512) + 128 * ks, idesc_o, 1u);
        commit2_if(leader, bar_pv + 16 * w + 8);
        if (j + 1 < n) s_product(k_addr, 1);
        if (j + 2 == n) commit2_if(leader, bar_qfree + 8 * w);
        give_back(ev);
        if (j + 1 < n) give_back(ek);
      }
      if (!dual && !kDown)
        for (int j = n; ok && j < n_other; ++j) {
          hand_on(full_k, empty_k, j);
          hand_on(v_ready, empty_v, j);
        }
      if (!ok) break;
      t0 += dual ? n + n_other : max(n, n_other);
      if (dual) counts[1] += n; else counts[0] += max(n, n_other);
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

  if (warp >= kGSoftWarps) {
    reg_alloc_dec<C::kRegsControl>();
    if (warp == kGProducer) {
      // ================= units, and TMA: this CTA's rows of Q, pages of K, dims of V =================
      const uint32_t leader = elect_one(), first = leader & (rank == 0 ? 1u : 0u);  // (the first CTA expects both CTAs' bytes)
      const uint32_t u_q = uniform(q_sm), u_k = uniform(k_sm), u_v = uniform(v_sm);
      const uint32_t to_q = uniform(in_cta(bar_q, 0));
      const int64_t n_units = !plan.listed ? plan.slots * heads
                              : n_blocks == 0 ? 0 : static_cast<int64_t>(scan[kGMaxList / 32]);
      int64_t round = 0;
      // b: the unit's sequence. part of parts: of the tiles.
      int b_now = 0, lo_now = 0, hi_now = 0;  // the unit's sequence and keys
      int my_parts = 0;                       // (cut) of the row block whose first part this pair has
      auto make_unit = [&](GUnit& un, int qb, int h, int b, int4 span, int part, int parts, int slot) {
        const int nq = span.y, L = span.z, row0 = qb * block_rows;
        const int rows = min(block_rows, nq - row0);
        int lo, hi_w[2] = {0, 0};  // first key that any row sees; the last ones of the halves' rows
        bool gaps = false;
        if (p.first_keys == nullptr) {
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const int from = row0 + half_rows * w, last = min(from + half_rows, nq) - 1;
            int lo_w;
            if (from < nq) key_range(from, last, nq, L, span.w, lo_w, hi_w[w]);
            if (w == 0) lo = lo_w;
          }
        } else {
          // Rows that see nothing have no say: neither their pages nor the table's entries for them need be any good.
          int lo_min = INT_MAX, first_row = INT_MAX, last_row = -1, own = 0;  // (own: rows that see the key they stand at)
#pragma unroll 1
          for (int i = lane; i < rows; i += 32) {
            const int pos = L - nq + row0 + i;
            int row_lo, row_hi;
            visible_keys(pos, L, p.score.window, p.first_keys[span.x + row0 + i], span.w, row_lo, row_hi);
            if (row_lo >= row_hi) continue;
            lo_min = min(lo_min, row_lo);
            hi_w[0] = i < half_rows ? max(hi_w[0], row_hi) : hi_w[0];
            hi_w[1] = i < half_rows ? hi_w[1] : max(hi_w[1], row_hi);
            first_row = min(first_row, i);
            last_row = i;
            own += row_lo <= pos;
          }
          lo = __reduce_min_sync(0xffffffffu, lo_min);
#pragma unroll
          for (int w = 0; w < 2; ++w) hi_w[w] = __reduce_max_sync(0xffffffffu, hi_w[w]);
          first_row = __reduce_min_sync(0xffffffffu, first_row);
          last_row = __reduce_max_sync(0xffffffffu, last_row);
          // (the keys of rows that see their own ones hang together, if there is no other row between them)
          gaps = __reduce_add_sync(0xffffffffu, own) != last_row - first_row + 1;
          if (last_row < 0) lo = 0, gaps = false;
        }
        const int hi = max(hi_w[0], hi_w[1]);
        int n[2], tile0 = lo / kGKeys, key_end = hi;
#pragma unroll
        for (int w = 0; w < 2; ++w) n[w] = hi_w[w] > lo ? (hi_w[w] + kGKeys - 1) / kGKeys - tile0 : 0;
        if (parts > 1) {  // (both halves' tiles within this part of the block's)
          const int all = max(n[0], n[1]);
          const int from = static_cast<int>(static_cast<int64_t>(all) * part / parts), to = static_cast<int>(static_cast<int64_t>(all) * (part + 1) / parts);
          n[0] = min(max(n[0] - from, 0), to - from);
          n[1] = min(max(n[1] - from, 0), to - from);
          tile0 += from;
          key_end = static_cast<int>(min(static_cast<int64_t>(hi), (static_cast<int64_t>(tile0) + to - from) * kGKeys));
        }
        int dual = kOneHead;
        if (by_two && rows <= half_rows && h + 1 < heads) {
          dual = kTwoHeads;
          n[1] = n[0];
        } else if (!by_two && n[0] > 1 && rows <= half_rows) {  // (the second half has no rows, and pairs are not short)
          dual = kSplitKeys;
          n[0] = n[1] = (n[0] + 1) / 2;  // (with an odd number the last tile lies behind the last key)
        }
        un = GUnit{row0, h, span.x, nq, L, span.w, tile0, n[0], n[1], dual, parts > 1 ? slot : -1, key_end, 0, gaps};
        b_now = b;
        lo_now = lo;
        hi_now = key_end;
      };
      // The pair's next unit: every pairs-th of the order, to and fro, so that each pair gets early (long) and late
      // (short) ones. Unlisted blocks may be empty: 32 at a time are looked at.
      auto find_unit = [&](GUnit& un) {
        if (plan.listed) {
          while (round * pairs < n_units) {
            const int r = static_cast<int>(round++), at = r * pairs + (r & 1 ? pairs - 1 - pair : pair);
            if (at >= n_units) continue;
            int entry = -1;  // the last one whose units start at or before this one
#pragma unroll
            for (int i = 0; i < kGMaxList; i += 32)
              entry += __popc(__ballot_sync(0xffffffffu, i + lane < n_blocks && work[i + lane] <= static_cast<uint32_t>(at)));
            const uint32_t e = list[entry];
            const int units = static_cast<int>(entry + 1 < n_blocks ? work[entry + 1] : n_units) - static_cast<int>(work[entry]);
            const int in_entry = at - static_cast<int>(work[entry]);
            const int parts = plan.cut ? units / heads : 1;
            const int h = in_entry / parts;
            make_unit(un, (e & (kGSmallBlock - 1)) >> 8, by_two && (e & kGSmallBlock) ? 2 * h : h, e & 255, spans[e & 255], in_entry % parts, parts, at);
            if (plan.cut && in_entry % parts == 0 && parts > 1) my_parts = parts;
            return true;
          }
          return false;
        }
        while (true) {
          const int64_t r = round + lane, at = r * pairs + (r & 1 ? pairs - 1 - pair : pair);
          int qb = 0, b = 0, h = 0;
          SeqSpan sp{0, 0, 0};
          if (at < n_units) {
            // Sequence b's blocks stand from place cu_q[b] / block_rows + b on: the next sequence's come behind them,
            // and all places are one a sequence and one for every block_rows tokens.
            h = static_cast<int>(at % heads);
            const int64_t place = plan.slots - 1 - at / heads;
            int hi = p.batch;  // the last sequence whose first place is not behind this one
            while (hi - b > 1) {
              const int mid = (b + hi) >> 1;
              if (p.cu_q[mid] / block_rows + static_cast<int64_t>(mid) <= place) b = mid; else hi = mid;
            }
            const int64_t in_seq = place - (p.cu_q[b] / block_rows + static_cast<int64_t>(b));
            qb = in_seq < 0 || in_seq >= plan.q_blocks ? plan.q_blocks : static_cast<int>(in_seq);
            if (qb < plan.q_blocks) sp = seq_span(p, b);
            else qb = 0;  // (no such block: sp has no rows)
          }
          const bool small = sp.nq - qb * block_rows <= half_rows;  // heads two by two
          if (small) h *= 2;
          const uint32_t have = __ballot_sync(0xffffffffu, qb * block_rows < sp.nq && h < heads);
          if (have == 0) {
            // (r grows with the lane, and so does `at` from one pair of rounds to the next)
            if (round * pairs >= n_units) return false;
            round += 32;
            continue;
          }
          const int src = __ffs(have) - 1;
          round += src + 1;
          auto from_lane = [&](int v) { return __shfl_sync(0xffffffffu, v, src); };
          const int b_src = from_lane(b);
          make_unit(un, from_lane(qb), from_lane(h), b_src, make_int4(from_lane(sp.q0), from_lane(sp.nq), from_lane(sp.L), prefix_of(b_src)), 0, 1, -1);
          return true;
        }
      };
      int t = 0, done[2] = {0, 0};  // tiles so far; units of each half so far
      int counts[3] = {0, 0, 0};    // tiles so far by set of barriers
      for (int k = 0;; ++k) {
        GUnit un;
        const bool more = find_unit(un);
        if (!more) un.row0 = -1;
        if (plan.cut && k == 0 && rank == 0 && lane == 0)  // what the merge finds at this pair's place (it has one unit at most)
          reinterpret_cast<PrefillRecord*>(static_cast<uint8_t*>(p.workspace) + prefill_records_at(D))[pair] =
              PrefillRecord{my_parts, un.row0, more ? un.h : 0, more ? un.q0 : 0, more ? un.nq : 0, {0, 0, 0}};
        const int slot = k % kGUnitSlots;
        if (k >= kGUnitSlots) ok = __all_sync(0xffffffffu, mbar_wait_bounded(unit_empty + 8 * slot, (k / kGUnitSlots - 1) & 1));
        if (!ok) break;
        if (lane == 0) {
          units[slot] = un;
          mbar_arrive_tc(unit_full + 8 * slot);
        }
        __syncwarp();
        if (!more) break;
        // Page numbers, four tiles (32 pages) at a time: of the first half's tiles (or all) and of the second half's where they
        // are others. Pages that no row sees are not looked at and read as zeros, like a page number beyond the cache.
        const int32_t* table = p.block_table + static_cast<int64_t>(b_now) * p.block_table_stride;
        const int tile0 = un.tile0;
        struct Pages {
          int id;
          float ks, vs;  // (e4m3) the page's scales
        };
        // (lanes 8 j .. 8 j + 7: the j-th of four tiles, downwards or upwards)
        auto load_pages = [&](int first_tile, int head) {
          const int tile = first_tile + (kDown ? -(lane >> 3) : lane >> 3);
          const int64_t page = (static_cast<int64_t>(tile0) + tile) * 8 + (lane & 7);
          Pages r{p.geom.num_pages, 0.f, 0.f};
          bool bad = false;
          bool wanted = tile >= 0 && page * kPageSize < hi_now && (page + 1) * kPageSize > lo_now;
          if (wanted && units[slot].gaps) {  // (the unit from shared memory: registers are short here)
            const GUnit& un = units[slot];
            const int rows = min(block_rows, un.nq - un.row0), pos0 = un.L - un.nq + un.row0;
            // Pages before the block's first position: what begins before their end reaches past them. Others: the rows one by one, from the
            // one that stands at the page's first key on, as mostly that one sees it.
            wanted = (page + 1) * kPageSize <= pos0;
            int i = static_cast<int>(min(max(page * kPageSize - pos0, static_cast<int64_t>(0)), static_cast<int64_t>(rows - 1)));
#pragma unroll 1
            for (int k = 0; k < rows && !wanted; ++k, i = i + 1 < rows ? i + 1 : 0) {
              int row_lo, row_hi;
              visible_keys(pos0 + i, un.L, p.score.window, p.first_keys[un.q0 + un.row0 + i], un.prefix, row_lo, row_hi);
              wanted = row_lo < row_hi && row_lo < (page + 1) * kPageSize && row_hi > page * kPageSize;
            }
          }
          if (wanted) {
            const int v = table[page];
            bad = v < 0 || v >= p.geom.num_pages;
            if (!bad) {
              r.id = v;
              if constexpr (kFp8) {
                r.ks = p.k_scale[static_cast<int64_t>(v) * heads + head];
                r.vs = p.v_scale[static_cast<int64_t>(v) * heads + head];
              }
            }
          }
          if (bad) {
            reinterpret_cast<volatile GUnit*>(units)[slot].bad = 1;
            __threadfence_block();
            report(p.status, PDA_DEV_BAD_PAGE);
          }
          __syncwarp();
          return r;
        };
        // (of the second half where it has tiles of its own: other keys, or the same of the next head)
        const int head1 = un.head(1), own0 = un.dual ? un.n0 : un.tiles();
        auto tile_of = [&](int w, int j) { return un.key_tile(w, kDown ? (w ? un.n1 : own0) - 1 - j : j); };
        Pages now0 = load_pages(tile_of(0, 0), un.h), next0 = un.tiles() > 4 ? load_pages(tile_of(0, 4), un.h) : now0;
        Pages now1 = un.dual ? load_pages(tile_of(1, 0), head1) : now0, next1 = un.dual && un.n1 > 4 ? load_pages(tile_of(1, 4), head1) : now0;
        const int n_all = un.tiles();
        auto load_q = [&](int w) {
          if (ok && done[w] > 0) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_qfree + 8 * w, (done[w] - 1) & 1));
          if (!ok) return;
          const int head = uniform(un.head(w) * p.group), token = uniform(un.q0 + un.first_row(w, half_rows) + plan.tile_rows * rank);
          mbar_expect_tx_if(first, bar_q + 8 * w, 2 * C::kLines * plan.tile_rows * p.group * 128);
#pragma unroll
          for (int ln = 0; ln < C::kLines; ++ln)
            tma_load_4d_pair_if(leader, u_q + w * C::kQBytes + ln * kGQLine, &maps.q, to_q + 8 * w, ln, head, token);
          ++done[w];
        };
        if (un.n0 > 0) load_q(0);
        for (int i = 0; ok && i < n_all; ++i, ++t) {
          const int u_h = uniform(un.head(un.half_of(i)));
          const int st = uniform(t % kStages), rnd = t / kStages;
          // this tile's pages in lanes 8 j .. 8 j + 7 of `ids`
          const int j = un.dual ? i >> 1 : i;
          const bool other = un.dual && (i & 1);
          if ((j & 3) == 0 && j > 0) {
            if (other) {
              now1 = next1;
              if (j + 4 < un.n1) next1 = load_pages(tile_of(1, j + 4), head1);
            } else {
              now0 = next0;
              if (j + 4 < own0) next0 = load_pages(tile_of(0, j + 4), un.h);
            }
          }
          const int ids = other ? now1.id : now0.id;
          if constexpr (kFp8) {
            const int rs = uniform(t % C::kRaw), used = t / C::kRaw;
            if (used > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(raw_empty + 8 * rs, (used - 1) & 1));
            if (!ok) break;
            // (the scales' place is free: the tile that had it is kGScaleSlots back, more than the tiles in both rings)
            if ((lane >> 3) == (j & 3))
              reinterpret_cast<float2*>(scales_sh)[(t % kGScaleSlots) * 8 + (lane & 7)] = other ? make_float2(now1.ks, now1.vs) : make_float2(now0.ks, now0.vs);
            __syncwarp();
            if (lane == 0) mbar_arrive_tc(scale_full + 8 * (t % kGScaleSlots));
            const uint32_t kd = uniform(smem_u32(smem) + C::kRawAt + rs * 2 * C::kRawBytes), vd = kd + C::kRawBytes;
            mbar_expect_tx_if(leader, raw_full + 8 * rs, C::kRawBytes);
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
              for (int ln = 0; ln < 2; ++ln)
                tma_load_5d_if(leader, kd + ln * 4096 + g * 1024, &maps.k, raw_full + 8 * rs, ln, u_h, __shfl_sync(0xffffffffu, ids, (j & 3) * 8 + 4 * rank + g));
            if (i == 0 && un.n1 > 0) load_q(1);
            if (ok && used > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(raw_empty + 8 * (C::kRaw + rs), (used - 1) & 1));
            if (!ok) break;
            mbar_expect_tx_if(leader, raw_full + 8 * (C::kRaw + rs), C::kRawBytes);
#pragma unroll
            for (int g = 0; g < 8; ++g)  // (of V the line is the CTA's 64 dims)
              tma_load_5d_if(leader, vd + g * 1024, &maps.v, raw_full + 8 * (C::kRaw + rs), rank, u_h, __shfl_sync(0xffffffffu, ids, (j & 3) * 8 + g));
            continue;
          }
          if (rnd > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty_k + 8 * st, (rnd - 1) & 1));
          if (!ok) break;
          const int set = un.dual ? 1 + (i & 1) : 0;
          const int count = set == 0 ? counts[0] : set == 1 ? counts[1] : counts[2];
          const uint32_t bar = uniform(tile_bar(full_k, set, count)), to_k = uniform(in_cta(bar, 0));
          if (set == 0) ++counts[0]; else if (set == 1) ++counts[1]; else ++counts[2];
          mbar_expect_tx_if(first, bar, 2 * C::kKBytes);
          const uint32_t kd = u_k + st * C::kKBytes;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int page = __shfl_sync(0xffffffffu, ids, (j & 3) * 8 + 4 * rank + g);
#pragma unroll
            for (int ln = 0; ln < C::kLines; ++ln)
              tma_load_page_pair_if(leader, kd + ln * kGKLine + g * 2048, &maps.k, to_k, ln, u_h, page);
          }
          if (i == 0 && un.n1 > 0) load_q(1);
          if (ok && rnd > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty_v + 8 * st, (rnd - 1) & 1));
          if (!ok) break;
          mbar_expect_tx_if(leader, full_v + 8 * st, C::kVBytes);
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const int page = __shfl_sync(0xffffffffu, ids, (j & 3) * 8 + g);
            tma_load_5d_if(leader, u_v + st * C::kVBytes + g * 2048, &maps.v, full_v + 8 * st, D == 128 ? rank : 0, u_h, page);
          }
        }
        if (!ok) break;
      }
      if (!ok) {  // copies in flight end before the CTA does: they are given time (a millisecond; a copy takes microseconds)
        if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
        for (int k = 0; k < 256; ++k) mbar_wait_bounded(bar_never, 0, 1);  // (4 us a poll)
      }
    } else if (kFp8 && warp >= kGConvert) {
      // ================= e4m3 tiles to bf16, in the layout of the copies of bf16 tiles =================
      // A thread takes 16 bytes of a row at a time and stores two 16-byte chunks. V rows behind the sequence's end are zero.
      const int me = tid - kGConvert * 32;
      auto convert = [&](uint32_t src, uint32_t dst0, uint32_t dst1, bool zero) {
        uint32_t r[4], o[8];
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(src));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t h[2];
          e4m3x4_to_f16x2x2(zero ? 0u : r[e], h[0], h[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            o[2 * e + i] = pack2<false>(f.x, f.y);
          }
        }
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst0), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst1), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
      };
      auto swizzled = [](uint32_t line, int row, int chunk) { return line + row * 128 + ((chunk ^ (row & 7)) << 4); };
      int counts[3] = {0, 0, 0};  // tiles so far by set of barriers
      GUnit un;
      int t = 0;
      for (int k = 0; next_unit(k, un); ++k) {
        free_unit(k);
        const int n_all = un.tiles();
        for (int i = 0; ok && i < n_all; ++i, ++t) {
          const int st = t % kStages, rnd = t / kStages, rs = t % (kFp8 ? C::kRaw : 1), used = t / (kFp8 ? C::kRaw : 1);
          const int set = un.dual ? 1 + (i & 1) : 0;
          const int count = set == 0 ? counts[0] : set == 1 ? counts[1] : counts[2];
          if (set == 0) ++counts[0]; else if (set == 1) ++counts[1]; else ++counts[2];
          const int64_t valid = un.L - (static_cast<int64_t>(un.tile0) + un.keys_of(i, kDown)) * kGKeys;
          const uint32_t raw = smem_u32(smem) + C::kRawAt + rs * 2 * C::kRawBytes;
#pragma unroll 1
          for (int v = 0; v < 2; ++v) {  // K, then V
            if (rnd > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded((v ? empty_v : empty_k) + 8 * st, (rnd - 1) & 1));
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(raw_full + 8 * (v * C::kRaw + rs), used & 1));
            if (!ok) break;
            // (K: two lines of 64 rows; V: one of 128, which lies the same way. In a loop, for the instruction caches' sake, which the
            // softmax's code fills: 4 steps unrolled 647 us for 8192 tokens, in a loop 603; the bytes' bits shifted into place and
            // multiplied by 2^120, which is more code, 656)
            const uint32_t to = v ? v_sm + st * C::kVBytes : k_sm + st * C::kKBytes, from = raw + v * C::kRawBytes;
            const int rows = v ? static_cast<int>(min(max(valid, static_cast<int64_t>(0)), static_cast<int64_t>(kGKeys))) : kGKeys;
#pragma unroll 1
            for (int x = me; x < 512; x += 128) convert(from + x * 16, swizzled(to, x >> 2, 2 * (x & 3)), swizzled(to, x >> 2, 2 * (x & 3) + 1), (x >> 2) >= rows);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
              arrive_cluster(in_cta(tile_bar(v ? v_ready : full_k, set, count), 0));
              mbar_arrive_tc(raw_empty + 8 * (v * C::kRaw + rs));
            }
            __syncwarp();
          }
        }
        if (!ok) break;
      }
      if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    } else if (!kFp8 && warp == kGRelay) {
      // ================= V tiles: cleared behind the sequence's end, then handed to the first CTA =================
      int counts[3] = {0, 0, 0};  // tiles so far by set of barriers
      GUnit un;
      int t = 0;
      for (int k = 0; next_unit(k, un); ++k) {
        free_unit(k);
        const int n_all = un.tiles();
        for (int i = 0; ok && i < n_all; ++i, ++t) {
          const int st = t % kStages;
          ok = __all_sync(0xffffffffu, mbar_wait_bounded(full_v + 8 * st, (t / kStages) & 1));
          if (!ok) break;
          const int64_t valid = un.L - (static_cast<int64_t>(un.tile0) + un.keys_of(i, kDown)) * kGKeys;
          const bool partly = valid > 0 && valid < kGKeys;  // (pages behind the end have been read as zeros)
          if (partly) {
            // (keys behind the end have weight 0, but what they hold may be anything)
            for (int c = lane; c < (kGKeys - static_cast<int>(valid)) * 8; c += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(v_sm + st * C::kVBytes + static_cast<int>(valid) * 128 + c * 16), "r"(0));
            fence_proxy_async();
          }
          const int set = un.dual ? 1 + (i & 1) : 0;
          const int count = set == 0 ? counts[0] : set == 1 ? counts[1] : counts[2];
          const uint32_t to = in_cta(tile_bar(v_ready, set, count), 0);
          if (set == 0) ++counts[0]; else if (set == 1) ++counts[1]; else ++counts[2];
          __syncwarp();
          if (lane == 0) {
            if (partly) arrive_cluster(to);  // (with what has been written before it)
            else arrive_cluster_tc(to);
          }
        }
        if (!ok) break;
      }
      if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    } else if (warp == kGMma && rank == 0) {
      issue_role(std::integral_constant<int, 0>{});
    } else if (warp == kGMma + 1 && rank == 0) {
      issue_role(std::integral_constant<int, 1>{});
    } else if (warp == kGMma && pair == 0 && !plan.listed) {
      for (int b = lane; b < p.batch; b += 32) seq_span(p, b);  // (reports sequences that no place leads to)
    }
  } else {
    reg_alloc_inc<C::kRegsSoftmax>();
    // ================= softmax and output: thread = row =================
    const int w = warp >> 2;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t my_s = tmem + 128 * w + lane_base, my_o = tmem + kGTmemO + 128 * w + lane_base;
    const float scale_log2 = kExp || kFixed ? 0.f : plan.scale_log2;  // (see rescale)
    const uint32_t to_p = in_cta(bar_p + 16 * w, 0), to_ofree = in_cta(bar_ofree + 8 * w, 0);
    const float neg_inf = -INFINITY;
    // this thread's row of a unit: query token row_token (from the half's first of this CTA), head row_head of the group
    const int row_token = (tid & 127) / p.group, row_head = (tid & 127) % p.group;
    const bool row_used = row_token < plan.tile_rows;  // (a group that does not divide 128 leaves rows over)
    int t = 0, merges = 0;  // tiles of this half, merges with the second half so far
    int pair_t = 0;         // (e4m3) tiles of the pair before this unit
    for (int unit = 0;; ++unit) {
      int step, own;  // (e4m3) the pair's tiles of this half: pair_t + step j + own
      int n, lo, hi;  // tiles; keys that this thread's row sees, from the half's first tile on
      int full_from, full_to;  // keys that all of the warp's rows see
      // The row's reference and the factor that goes with it. A row that does not exist is another sequence's, or anything:
      // its reference is infinite, so that it never asks for the warp's to be raised and has no say in the other rows' rounding.
      float m_ref, c_ref;
      float slope = 0.f;  // (biased) per key
      int key0_pos = 0;   // the half's first key minus the row's position
      {
        GUnit un;
        if (!next_unit(unit, un)) break;
        n = w == 0 ? un.n0 : un.n1;
        step = un.dual ? 2 : 1;
        own = un.dual ? w : un.skipped(w, kDown);
        const int row = un.first_row(w, half_rows) + plan.tile_rows * rank + row_token, pos = un.L - un.nq + row;
        const bool exists = row_used && row < un.nq;
        lo = hi = 0;
        if (exists) visible_keys(pos, un.L, p.score.window, p.first_keys != nullptr ? p.first_keys[un.q0 + row] : 0, un.prefix, lo, hi);
        const int64_t key0 = (static_cast<int64_t>(un.tile0) + un.key_tile(w, 0)) * kGKeys;
        const auto from_key0 = [&](int key) { return static_cast<int>(max(min(key - key0, static_cast<int64_t>(1 << 30)), static_cast<int64_t>(-(1 << 30)))); };
        lo = from_key0(lo);
        hi = from_key0(min(hi, un.key_end));
        // (biased: keys behind the token itself go the way of masked tiles, which takes the distance's absolute value)
        const int full_hi = kBias && exists ? min(hi, from_key0(pos + 1)) : hi;
        full_from = __reduce_max_sync(0xffffffffu, exists ? lo : -(1 << 30));
        full_to = __reduce_min_sync(0xffffffffu, exists ? full_hi : 1 << 30);
        if (!__any_sync(0xffffffffu, exists)) full_to = -(1 << 30);  // (a warp without any row sees nothing)
        m_ref = kFixed ? plan.ref : exists ? kGNoMax : INFINITY;
        if constexpr (kBias) {
          slope = exists && p.score.slopes != nullptr ? p.score.slopes[un.head(w) * p.group + row_head] * kLog2e : 0.f;
          key0_pos = static_cast<int>(key0 - pos);
        }
      }
      c_ref = kExp || kFixed ? 1.f : score_factor(m_ref, scale_log2);
      float l = 0.f;
      // One tile; masked: some row of the warp does not see all of it.
      auto tile = [&](auto masked, int j, int j_key) {  // j_key: which of the half's tiles by its keys
        constexpr bool kMasked = decltype(masked)::value;
        // 64 keys at a time; the first run's products start while the second run is here. (Not unrolled: both runs' code, masked and
        // not, was more than the instruction caches held: a third of all stalls were for instructions.)
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_s + 16 * w + 8 * k, t & 1));
          if (!ok) return;
          tc_fence_after();
          uint32_t sv[64];
          tmem_ld32(my_s + 64 * k, *reinterpret_cast<uint32_t(*)[32]>(&sv[0]));
          tmem_ld32(my_s + 64 * k + 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[32]));
          tmem_wait_ld();
          // keys of the run's columns: 32 k + e, from the 32nd on 32 k + 32 + e
          const int first_lo = j_key * kGKeys + 32 * k, first_hi = first_lo + 32;
          // (columns of the run that this row sees, a bit each)
          [[maybe_unused]] uint32_t seen[2];
          if (kMasked) {
            seen[0] = bits_before(hi - first_lo) & ~bits_before(lo - first_lo);
            seen[1] = bits_before(hi - first_hi - 32) & ~bits_before(lo - first_hi - 32);
          }
          auto hidden = [&](int e) { return (seen[e >> 5] & (1u << (e & 31))) == 0u; };
          auto both = [](float v) { return f32x2(__float_as_uint(v), __float_as_uint(v)); };
          auto two = [&](int e) { return f32x2(sv[2 * e], sv[2 * e + 1]); };
          uint32_t pk[32];
          float part = 0.f;
          [[maybe_unused]] float2 page_scale[4];  // (e4m3) of keys and values of the run's four pages
          if constexpr (kFp8) {
            const int pt = pair_t + step * j + own;
            if (k == 0) {
              if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(scale_full + 8 * (pt % kGScaleSlots), (pt / kGScaleSlots) & 1));
              if (!ok) return;
            }
            const float2* scales = reinterpret_cast<const float2*>(scales_sh) + (pt % kGScaleSlots) * 8 + 2 * k;
#pragma unroll
            for (int g = 0; g < 4; ++g) page_scale[g] = scales[(g >> 1) * 4 + (g & 1)];
            if constexpr (kShape != kShapeNone) {
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                float s0, s1;
                f32x2_split(mul_f32x2(two(e), both(page_scale[e >> 3].x)), s0, s1);
                sv[2 * e] = __float_as_uint(s0);
                sv[2 * e + 1] = __float_as_uint(s1);
              }
            }
          }
          // (warp-collective) O so far, up to the last tile or to the first run of this one, times `a`; false: the wait for it ran out
          auto rescale_output = [&](float a) {
            if (j == 0 && k == 0) return true;
            if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 16 * w + 8 * (k ^ 1), (k == 0 ? t - 1 : t) & 1));
            if (!ok) return false;
            __syncwarp();
            tc_fence_after();
            rescale_columns<D>(my_o, a);
            return true;
          };
          auto pack = [&](int e, float w0, float w1) {  // (values' page scales go with the weights)
            if constexpr (kFp8) f32x2_split(mul_f32x2(f32x2(__float_as_uint(w0), __float_as_uint(w1)), both(page_scale[e >> 3].y)), w0, w1);
            return pack2<false>(w0, w1);
          };
          if (kMasked && __all_sync(0xffffffffu, hi <= first_lo || lo >= first_hi + 64)) {  // no row of the warp sees any of these
#pragma unroll
            for (int e = 0; e < 32; ++e) pk[e] = 0;
          } else {
            if constexpr (kCap) {
              // The hyperbolic tangent of the cap goes by the row's largest product among the 64: small ones by a polynomial
              // (|x| <= 1/2: degree 5; |x| <= 5/4: degree 11), of the form whose largest error is least (2^-17.5 and 2^-18.7, of
              // 1), others, and infinities and NaN, by exponential and reciprocal: three results of the special-function unit a
              // score with the weight's. A warp takes one of the polynomials, the longer one if any of its rows asks for it.
              // Where the reference is fixed, the weights are taken right behind it.
              // Above kAbsoluteCap each score is taken by itself as in cap_score, since scores may be far below the cap.
              if (kMasked) {
#pragma unroll
                for (int e = 0; e < 64; ++e) sv[e] = hidden(e) ? 0u : sv[e];
              }
              float mx[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int e = 0; e < 32; ++e) mx[e & 3] = max3_nan(mx[e & 3], fabsf(__uint_as_float(sv[2 * e])), fabsf(__uint_as_float(sv[2 * e + 1])));
              const float far = max3_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3], mx[3]);
              const uint64_t minus_ref = both(-m_ref);
              [[maybe_unused]] uint64_t sum2[2] = {0ull, 0ull};
              auto capped = [&](auto shape) {  // (shape: of a pair of products)
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  float z0, z1;
                  f32x2_split(shape(two(e)), z0, z1);
                  if constexpr (kFixed) {
                    float w0 = ex2(z0), w1 = ex2(z1);
                    if (kMasked) {
                      w0 = hidden(2 * e) ? 0.f : w0;
                      w1 = hidden(2 * e + 1) ? 0.f : w1;
                    }
                    sum2[e & 1] = add_f32x2(sum2[e & 1], f32x2(__float_as_uint(w0), __float_as_uint(w1)));
                    pk[e] = pack(e, w0, w1);
                  } else {
                    sv[2 * e] = __float_as_uint(z0);
                    sv[2 * e + 1] = __float_as_uint(z1);
                  }
                }
              };
              auto poly11 = [&](uint64_t t2) {
                uint64_t y = fma_f32x2(t2, plan.poly11[5], plan.poly11[4]);
                y = fma_f32x2(t2, y, plan.poly11[3]);
                y = fma_f32x2(t2, y, plan.poly11[2]);
                y = fma_f32x2(t2, y, plan.poly11[1]);
                return fma_f32x2(t2, y, plan.poly11[0]);
              };
              [[maybe_unused]] const bool watch = kLow && __any_sync(0xffffffffu, (l == 0.f && far > plan.low_limit && hi > lo) || m_ref != plan.ref);
              const bool longer = kMasked || __any_sync(0xffffffffu, far > plan.limit[0] && far <= plan.limit[1] && hi > lo);
              if (!longer && far <= plan.limit[0]) {
                capped([&](uint64_t x) {
                  const uint64_t t2 = mul_f32x2(x, x);
                  const uint64_t y = fma_f32x2(t2, fma_f32x2(t2, plan.poly5[2], plan.poly5[1]), plan.poly5[0]);
                  return kFixed ? fma_f32x2(x, y, minus_ref) : mul_f32x2(x, y);
                });
              } else if (far <= plan.limit[1]) {
                capped([&](uint64_t x) {
                  const uint64_t y = poly11(mul_f32x2(x, x));
                  return kFixed ? fma_f32x2(x, y, minus_ref) : mul_f32x2(x, y);
                });
              } else if (!kFixed && plan.relative) {
                capped([&](uint64_t x) {
                  float x0, x1, z0, z1;
                  const uint64_t ux = mul_f32x2(x, both(plan.u));
                  f32x2_split(ux, x0, x1);
                  f32x2_split(mul_f32x2(x, poly11(mul_f32x2(ux, ux))), z0, z1);
                  auto far_one = [&](float v) { return fmaf(-p.score.cap, 2.f * rcp_approx(ex2(2.f * kLog2e * v) + 1.f), p.score.cap); };
                  if (!(fabsf(x0) <= kTanhReach)) z0 = far_one(x0);
                  if (!(fabsf(x1) <= kTanhReach)) z1 = far_one(x1);
                  return f32x2(__float_as_uint(z0), __float_as_uint(z1));
                });
              } else {
                capped([&](uint64_t x) {
                  float y0, y1;
                  f32x2_split(mul_f32x2(x, both(2.f * kLog2e * plan.u)), y0, y1);
                  const uint64_t r = f32x2(__float_as_uint(rcp_approx(ex2(y0) + 1.f)), __float_as_uint(rcp_approx(ex2(y1) + 1.f)));
                  return fma_f32x2(r, both(-2.f * p.score.cap), both(kFixed ? p.score.cap - m_ref : p.score.cap));
                });
              }
              if constexpr (kFixed) {
                float s0, s1;
                f32x2_split(add_f32x2(sum2[0], sum2[1]), s0, s1);
                part = s0 + s1;
                if constexpr (kLow) {
                  // Where the reference is not the right one it is changed and the run begins again: its scores still stand in tensor memory.
                  // (A row that has nothing yet has no O to be multiplied. A row goes down once and up once.)
                  const bool lower = l == 0.f && part > 0.f && part < kGFixedLeast && m_ref > plan.ref_low && hi > lo;
                  const bool raise = part > kGFixedMost && m_ref < plan.ref;
                  if (__builtin_expect(watch && __any_sync(0xffffffffu, lower || raise), 0)) {
                    const float a = raise ? ex2(m_ref - plan.ref) : 1.f;
                    m_ref = raise ? plan.ref : lower ? plan.ref_low : m_ref;
                    l *= a;
                    if (__any_sync(0xffffffffu, raise) && !rescale_output(a)) return;
                    --k;
                    continue;
                  }
                }
              }
            }
            // Scores that references are taken of. Biased ones and e4m3's are in the exponent's units: mul s + slope (j - p), the slope's
            // part a constant for the first of 16 keys and slope times 0 .. 15 (in masked tiles the distance of each key); e4m3's that are
            // not biased with the page's scale. They are rounded before the reference is taken from them: so a reference is a score itself, none of those it was taken of
            // passes it, and it is raised once at most for 64 keys. (Taken from the product in the same rounding, scores of 2^30 and
            // more passed a reference that could not be raised by so little. Cost 7 %: 508 -> 538 us biased, 577 -> 617 e4m3. A pass of its own
            // for rows with such scores, beside the hot one, gained nothing: 541 and 604, 543 and 613, or, in place, 528 and 664.)
            const auto score = [&](int e) {
              if constexpr (kBias) {
                const int g = e >> 3, i = e & 7;
                // (the distance is taken in whole numbers: near keys' biases are off by little behind long contexts too)
                const float distance = static_cast<float>(key0_pos + (g < 2 ? first_lo : first_hi) + 16 * g);
                uint64_t bias2;
                if constexpr (kMasked) {  // (keys behind the token itself may be among them, of a prefix: the bias goes down on that side too)
                  bias2 = mul_f32x2(both(-slope), f32x2(__float_as_uint(fabsf(distance + 2.f * i)), __float_as_uint(fabsf(distance + (2.f * i + 1.f)))));
                } else {
                  bias2 = fma_f32x2(both(slope), f32x2(__float_as_uint(2.f * i), __float_as_uint(2.f * i + 1.f)), both(slope * distance));
                }
                return kCap ? add_f32x2(two(e), bias2) : fma_f32x2(two(e), both(p.score.mul), bias2);
              } else if constexpr (kExp) {
                return mul_f32x2(two(e), both(p.score.mul * page_scale[e >> 3].x));
              } else {
                return two(e);
              }
            };
            if constexpr (!kFixed) {
              if (kMasked && !kExp) {
#pragma unroll
                for (int e = 0; e < 64; ++e)
                  if (hidden(e)) sv[e] = 0xff800000u;  // -inf
              }
              const auto visible = [&](int e) {
                uint64_t z = score(e);
                if (kMasked && kExp) {
                  float z0, z1;
                  f32x2_split(z, z0, z1);
                  z = f32x2(hidden(2 * e) ? 0xff800000u : __float_as_uint(z0), hidden(2 * e + 1) ? 0xff800000u : __float_as_uint(z1));
                }
                return z;
              };
              // The first reference, where there is none yet: the maximum of these 64 scores.
              if (kExp ? __any_sync(0xffffffffu, m_ref == kGNoMax) : (k == 0 && j == 0)) {
                float mx[2] = {neg_inf, neg_inf};
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  float z0, z1;
                  f32x2_split(visible(e), z0, z1);
                  mx[e & 1] = max3(mx[e & 1], z0, z1);
                }
                const float first = fmaxf(mx[0], mx[1]);
                if (kExp) m_ref = m_ref == kGNoMax && first > neg_inf ? first : m_ref;
                else m_ref = fmaxf(m_ref, first);
                if (!kExp) c_ref = score_factor(m_ref, scale_log2);
              }
              // Weights relative to the reference as it stands, the maximum taken along the way: rarely does it pass the
              // reference by so much that the reference is raised and the weights are taken again.
              float top;
              while (true) {
                const float minus_ref = kExp ? -m_ref : -__fmul_rn(m_ref, c_ref);
                uint64_t sum2[2] = {0ull, 0ull};
                float mx[2] = {neg_inf, neg_inf};
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const uint64_t z = visible(e);
                  const uint64_t x = kExp ? add_f32x2(z, both(minus_ref)) : fma_f32x2(z, both(c_ref), both(minus_ref));
                  float w0, w1;
                  f32x2_split(z, w0, w1);
                  mx[e & 1] = max3_nan(mx[e & 1], w0, w1);
                  if (!kMasked && e % kGPolyOf == kGPolyOf - 1) {  // (weights of hidden keys are exactly zero, the polynomial's are not)
                    exp2_two(x, w0, w1);
                  } else {
                    f32x2_split(x, w0, w1);
                    w0 = ex2(w0);
                    w1 = ex2(w1);
                  }
                  sum2[e & 1] = add_f32x2(sum2[e & 1], f32x2(__float_as_uint(w0), __float_as_uint(w1)));
                  pk[e] = pack(e, w0, w1);
                }
                float s0, s1;
                f32x2_split(add_f32x2(sum2[0], sum2[1]), s0, s1);
                part = s0 + s1;
                top = max3_nan(mx[0], mx[0], mx[1]);
                if (!(top <= 3.4028235e38f)) part = __uint_as_float(0x7fc00000u);  // a NaN or +inf among the scores
                const bool raise = kExp ? top > m_ref + kGRescale : top * c_ref > m_ref * c_ref + kGRescale;
                if (!__any_sync(0xffffffffu, raise)) break;
                // (only the rows that ask for it: a row's rounding does not depend on its neighbours' scores)
                const float m_new = raise ? top : m_ref;
                float a;
                if (kExp) {
                  a = raise ? ex2(m_ref - m_new) : 1.f;
                } else {
                  a = rescale(m_ref, m_new, scale_log2);
                  c_ref = score_factor(m_new, scale_log2);
                }
                m_ref = m_new;
                l *= a;
                if (!rescale_output(a)) break;
              }
            }
          }
          if (!ok) return;
          l += part;
          tmem_st32(my_s + 64 * k, pk);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster_tc(to_p + 8 * k);
        }
      };
      for (int j = 0; ok && j < n; ++j, ++t) {
        const int j_key = kDown ? n - 1 - j : j;
        if (full_from <= j_key * kGKeys && full_to >= (j_key + 1) * kGKeys) tile(std::false_type{}, j, j_key);
        else tile(std::true_type{}, j, j_key);
      }
      // ---- output
      if constexpr (kFp8) pair_t += units[unit % kGUnitSlots].tiles();
      if (n > 0) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv + 16 * w + 8, (t - 1) & 1));
        tc_fence_after();
      }
      GUnit un = units[unit % kGUnitSlots];  // (read again: it takes registers that the loop above needs)
      un.bad = reinterpret_cast<volatile GUnit*>(units)[unit % kGUnitSlots].bad;
      free_unit(unit);
      const int row = un.first_row(w, half_rows) + plan.tile_rows * rank + row_token;  // query token of the sequence
      const bool exists = row_used && row < un.nq;
      const bool split = un.dual == kSplitKeys;
      float* sums = merge_sh + 2 * (tid & 127);  // the row's reference and sum from the second half
      if (split && w == 1) {  // the first half's warp of the same rows takes it from here
        *reinterpret_cast<float2*>(sums) = make_float2(kFixed && l == 0.f ? kGNoMax : m_ref, l);  // (no keys of this half: no say in the reference)
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_tc(bar_merge + 8 * (warp & 3));
        if (!ok) break;
        continue;
      }
      if (split) {  // O and the sum of both halves, in the first half's place
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_merge + 8 * (warp & 3), merges & 1));
        tc_fence_after();
        ++merges;
        const float2 other = *reinterpret_cast<const float2*>(sums);
        if (kFixed && l == 0.f) m_ref = kGNoMax;
        const float m = fmaxf(m_ref, other.x);
        const float mul = rescale(m_ref, m, scale_log2), mul_other = rescale(other.x, m, scale_log2);
        m_ref = m;
        l = l * mul + other.y * mul_other;
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
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
      // finite: then it has no softmax and is NaN. (The polynomial gives such scores 2^-126.) Rows that see nothing are zero.
      bool some = n > 0 && ok && exists && !un.bad;
      if (some) {
        int see_lo, see_hi;
        visible_keys(un.L - un.nq + row, un.L, p.score.window, p.first_keys != nullptr ? p.first_keys[un.q0 + row] : 0, un.prefix, see_lo, see_hi);
        some = see_lo < see_hi;
      }
      const bool partial = un.slot >= 0;
      float inv = 1.f / (!kFixed && l < 5.4210109e-20f ? NAN : l);  // 2^-64
      float* part_o = nullptr;
      if (partial) {  // sums go to the workspace as they are, for the merge
        const int64_t at = static_cast<int64_t>(un.slot) * kPreRows + (2 * w + rank) * 128 + (tid & 127);
        part_o = static_cast<float*>(p.workspace) + at * D;
        float2* ws = reinterpret_cast<float2*>(static_cast<uint8_t*>(p.workspace) + prefill_sums_at(D)) + at;
        // (no tile here, or no page: nothing. A bad page anywhere makes the row zero: marked by a negative sum)
        if (exists) *ws = un.bad ? make_float2(INFINITY, -1.f) : n > 0 ? make_float2(m_ref, l) : make_float2(kGNoMax, 0.f);
        some = n > 0 && ok && !un.bad;
        inv = 1.f;
      }
      __nv_bfloat16* out = p.out + (static_cast<int64_t>(un.q0) + row) * p.out_token_stride + (un.head(w) * p.group + row_head) * p.out_head_stride;
      // A thread stores its own row, 32 bytes (a whole sector) at a time where the rows' alignment allows it.
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0 && p.out_token_stride % 16 == 0 && p.out_head_stride % 16 == 0;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t ov[32];
        tmem_ld32(my_o + 32 * c, ov);
        tmem_wait_ld();
        if (c == D / 32 - 1 && n > 0) {  // O is in registers: the next unit's products may write it
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster_tc(to_ofree);
        }
        if (exists && partial) {
          if (some) {
#pragma unroll
            for (int k = 0; k < 32; k += 8)
              asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(part_o + 32 * c + k), "r"(ov[k]), "r"(ov[k + 1]), "r"(ov[k + 2]),
                           "r"(ov[k + 3]), "r"(ov[k + 4]), "r"(ov[k + 5]), "r"(ov[k + 6]), "r"(ov[k + 7]) : "memory");
          }
        } else if (exists) {
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
        __syncwarp();
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
  if (warp == kGMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kGTmemCols) : "memory");
  }
}

// Joins the parts of row blocks that were cut along the keys. A warp per row; a lane owns D / 32 columns.
template <int D>
__global__ void __launch_bounds__(256) prefill_merge_kernel(const __grid_constant__ PrefillParams p, const __grid_constant__ PrefillPlan plan, float scale_log2, float least) {
  constexpr int kCols = D / 32;
  const uint8_t* ws = static_cast<const uint8_t*>(p.workspace);
  const PrefillRecord rec = reinterpret_cast<const PrefillRecord*>(ws + prefill_records_at(D))[blockIdx.x];
  const int lane = threadIdx.x & 31;
  for (int r = blockIdx.y * 8 + (threadIdx.x >> 5); rec.parts > 0 && r < kPreRows; r += gridDim.y * 8) {
    const int quarter = r >> 7, in_tile = r & 127, token = in_tile / p.group, head = in_tile % p.group;
    const int row = rec.row0 + quarter * plan.tile_rows + token;
    if (token >= plan.tile_rows || row >= rec.nq) continue;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kPreRows + r;
    const float2* sums = reinterpret_cast<const float2*>(ws + prefill_sums_at(D)) + at;
    // A lane takes every 32nd part's reference and sum (parts are kPreMaxPairs at most), and their factors.
    constexpr int kRounds = (kPreMaxPairs + 31) / 32;
    float2 sum[kRounds];
    float m = kGNoMax, l = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      sum[i] = 32 * i + lane < rec.parts ? sums[static_cast<int64_t>(32 * i + lane) * kPreRows] : make_float2(kGNoMax, 0.f);
      m = fmaxf(m, sum[i].y != 0.f ? sum[i].x : kGNoMax);
      bad |= sum[i].y < 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    bad = __any_sync(0xffffffffu, bad);
    float mul[kRounds], acc[kCols];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      mul[i] = bad || sum[i].y == 0.f ? 0.f : rescale(sum[i].x, m, scale_log2);  // (nothing of this row in that part)
      l = fmaf(sum[i].y, mul[i], l);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
    for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int n = min(rec.parts - 32 * i, 32);
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float a = __shfl_sync(0xffffffffu, mul[i], k);
        if (a == 0.f) continue;  // (what stands there may be anything)
        const float* o = reinterpret_cast<const float*>(ws) + (at + static_cast<int64_t>(32 * i + k) * kPreRows) * D + kCols * lane;
        if constexpr (kCols == 4) {
          const float4 v = *reinterpret_cast<const float4*>(o);
          acc[0] = fmaf(v.x, a, acc[0]), acc[1] = fmaf(v.y, a, acc[1]), acc[2] = fmaf(v.z, a, acc[2]), acc[3] = fmaf(v.w, a, acc[3]);
        } else {
          const float2 v = *reinterpret_cast<const float2*>(o);
          acc[0] = fmaf(v.x, a, acc[0]), acc[1] = fmaf(v.y, a, acc[1]);
        }
      }
    }
    const bool zero = bad || l == 0.f;
    const float inv = 1.f / (l < least ? NAN : l);
    uint32_t packed[kCols / 2];
#pragma unroll
    for (int i = 0; i < kCols; i += 2) packed[i / 2] = zero ? 0u : pack2<false>(acc[i] * inv, acc[i + 1] * inv);
    __nv_bfloat16* out = p.out + (static_cast<int64_t>(rec.q0) + row) * p.out_token_stride + (rec.h * p.group + head) * p.out_head_stride + kCols * lane;
    if constexpr (kCols == 4) *reinterpret_cast<uint2*>(out) = make_uint2(packed[0], packed[1]);
    else *reinterpret_cast<uint32_t*>(out) = packed[0];
  }
}

}  // namespace
}  // namespace pda
