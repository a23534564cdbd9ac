// Absorbed attention over the paged latent cache on tcgen05 + TMEM: up to 64 query rows (query tokens x
// heads) per CTA against tiles of 64 cached rows, each tile fetched once and used as keys and as values.
//
// Both products run transposed, so that the query rows are the N of the instruction and the accumulator
// fits tensor memory (O of 128 rows x 512 dims in f32 would be all of it):
//   S^T[64 tokens x N]   = C[64 x (R + 64)] . Q^T      M = 64, A = the tile (K-major), B = Q (K-major)
//   O^T[128 dims x N] (+)= C^T[128 x 64] . P^T         R / 128 of them, M = 128, A = the tile read
//                                                      MN-major, B = P (MN-major, written by the softmax)
// N = 16, 32 or 64, the least that holds the rows (fewer rows: less of the tensor core's time, which for
// 16 rows stays far below the tile's trip from memory). A tile is 64 tokens because two tiles (2 x 72 KB)
// next to Q (72 KB at N = 64) are what shared memory holds; they are filled and freed by the 128-byte
// lines that one O^T instruction group reads, so that the next tile's copies start while P . C runs.
//
// Work: the tiles of all sequences form one list, cut into equal spans, one per group of CTAs (the CTAs of
// a group take the row blocks of the same span at the same time: the tile comes from memory once and
// from L2 for the others). A sequence that lies in several spans leaves partial results (normalised, with
// the reference and the sum of their weights: their logarithm in one number would lose the sum next to a large
// reference) in the workspace, merged by a second kernel; one within a span is written directly. Spans depend on the lengths and the number of SMs only.
//
// Softmax: a thread holds 2 tokens x N / 8 query rows. Weights are taken relative to a reference per row
// that is raised (and O, in tensor memory, rescaled) only when a score passes it by more than 2^8; the
// decision is one vote per tile, so that in the steady state no maximum crosses lanes. Row sums stay in
// registers, per token lane, until the end. Weights are rounded to bf16 for the tensor core (they are at
// most 2^8, and relative to their row's sum the rounding is 2^-8 whatever the reference); sums, scores and
// O are 32-bit.
//
// Measured (B200, 512 + 64, pages of 64): 64 sequences of 512..4096 tokens, 16 heads, 43 us a call (floor from HBM 27);
// 128 such sequences with 128 heads 166 us a call, 151 in a graph, 2900 clocks a tile,
// of which the MMAs keep shared memory busy for 2000 (they read A for 64 columns only: 33 clocks an MMA of S, 49 of O) and the
// tile's arrival for 600: with 64 rows that is the bound, with 16 or 32 it is HBM.
//
// Warps: 0-7 softmax and output, 8 and 12 TMA producers, 9 S issue + TMEM, 10 P . C issue, 11 Q rows. All waits are
// bounded; on a timeout every role leaves its loop, outstanding copies and products are waited for (with a
// limit) and tensor memory is released.
#include <cfloat>
#include <cmath>

#include "latent.cuh"
#include "latent_ptx.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_ptx.cuh"

namespace pda {

namespace {

constexpr int kLTok = 64;                       // tokens per tile
constexpr int kLLineBytes = kLTok * 128;        // one 128-byte line of 64 tokens
constexpr int kLMaxLines = 9;                   // latent 512 + rope 64
constexpr int kLStageBytes = kLMaxLines * kLLineBytes;
constexpr int kLStages = 2;
constexpr int kLGroups = 5;                     // line groups of a stage: rope, then pairs of latent lines
constexpr int kLSoftWarps = 8, kLSoft = kLSoftWarps * 32;  // two warps per 32 lanes of tensor memory, half the columns each
constexpr int kLThreads = kLSoft + 160;
constexpr int kLProducer = 8, kLSIssue = 9, kLPvIssue = 10, kLQLoad = 11, kLProducer2 = 12;
constexpr uint32_t kLTmemCols = 512, kLTmemS = 256;  // O^T: R / 128 blocks of N columns from 0; S^T from 256
constexpr float kLNoMax = -FLT_MAX;             // reference of a row that has seen no finite score yet: the lowest it can be
constexpr float kLRescale = 8.f;                // log2

template <int N>
struct LCfg {
  static constexpr int kQBytes = kLMaxLines * N * 128;
  static constexpr int kQBufs = N <= 32 ? 2 : 1;  // what fits: with two, the next segment's rows arrive during this one
  static constexpr int kPBytes = kLTok * 128;
  static constexpr int kBarBytes = 384;
  // column maxima / sums of the four token quarters (the first row also inverse sums), rescale factors, row offsets
  static constexpr int kRowBytes = 4 * N * 4 + N * 4 + N * 4;
  static constexpr int kSmemBytes = kLStages * kLStageBytes + kQBufs * kQBytes + kPBytes + kRowBytes + kBarBytes + 1024;
};
static_assert(LCfg<64>::kSmemBytes <= 232448 && LCfg<32>::kSmemBytes <= 232448, "shared memory");

struct LPlan {
  int32_t row_blocks, per_pass, passes, groups;  // row blocks per sequence; taken at once; rounds; CTA groups
  int32_t page_shift;                            // log2 of the page size
  int32_t by_sequence;                           // records are indexed by sequence (there are fewer than groups)
  int32_t q_box;                                 // heads per copy of Q (0: rows by plain copies)
};

struct LMaps {
  CUtensorMap line, pair;        // the cache: one line, two lines of a run of slots
  CUtensorMap q_latent, q_rope;  // one line of q_box heads of a token
};

// A sequence that continues behind its first span: see latent_merge_kernel. One per group (the sequence that
// leaves its span), or one per sequence where those are fewer. vseq < 0: none. Every record is written by every
// call, after an expired wait too and whatever *status holds: the merge takes them for addresses.
struct LRecord {
  int32_t vseq, first_slot, n_seg, group;
};

__device__ __forceinline__ int seq_tokens(const LatentParams& p, int b) {
  const int L = p.seq_lens[b];
  return L <= 0 || L > static_cast<int64_t>(p.block_table_stride) * p.geom.page_size ? 0 : L;
}
__device__ __forceinline__ int seq_tiles(int L) { return L <= 0 ? 1 : (L - 1) / kLTok + 1; }  // (an empty one takes a place too)

// One sequence's part of a CTA's span.
struct Segment {
  int b, rb, L;        // sequence, row block (-1: none in this pass), tokens
  int tile0, n_tiles;  // tiles to attend (cut at what the row block can see)
  int off, take;       // tiles of the list it stands for
  int whole;           // tiles of the sequence in the list
  int vseq;
};

struct Walk {
  int vseq, off, rem;
  int L0;  // tokens of the first sequence; -1 behind it
};

template <int N>
__device__ __forceinline__ bool next_segment(const LatentParams& p, const LPlan& plan, int r, Walk& w, Segment& s) {
  if (w.rem <= 0) return false;
  s.vseq = w.vseq;
  s.b = w.vseq % p.batch;
  const int rb = (w.vseq / p.batch) * plan.per_pass + r;
  s.rb = rb < plan.row_blocks ? rb : -1;
  s.L = w.L0 >= 0 ? w.L0 : seq_tokens(p, s.b);
  w.L0 = -1;
  s.whole = seq_tiles(s.L);
  s.off = w.off;
  s.take = min(s.whole - w.off, w.rem);
  const int last_row = min((rb + 1) * N, p.n_q * p.num_q_heads) - 1;
  const int see = min(max(s.L - p.n_q + last_row / p.num_q_heads + 1, 0), s.L);  // what its last row can see
  s.tile0 = w.off;
  s.n_tiles = s.rb < 0 || see == 0 ? 0 : max(0, min(w.off + s.take, seq_tiles(see)) - w.off);
  w.rem -= s.take;
  w.off = 0;
  w.vseq += 1;
  return true;
}

__device__ __forceinline__ void tma_load_4d_hint_if(uint32_t leader, uint32_t dst, const CUtensorMap* map, uint32_t bar, int slot,
                                                    int line, int page, uint64_t policy) {
  asm volatile(
      "{\n\t.reg .pred pe;\n\tsetp.ne.b32 pe, %6, 0;\n\t"
      "@pe cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {0, %3, %4, %5}], [%2], %7;\n\t}"
      ::"r"(dst), "l"(map), "r"(bar), "r"(slot), "r"(line), "r"(page), "r"(leader), "l"(policy) : "memory");
}
__device__ __forceinline__ uint64_t l2_policy_normal() {
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
  return pol;
}
// 16 lanes x 8 J columns: register 4 j + 0, 1: lane t / 4, columns 8 j + 2 (t % 4) + 0, 1; + 2, 3: lane t / 4 + 8
template <int J>
__device__ __forceinline__ void tmem_ld_16x256b(uint32_t taddr, uint32_t (&r)[4 * J]) {
  if constexpr (J == 1) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
  } else if constexpr (J == 2) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr));
  } else {
    static_assert(J == 4);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
  }
}
__device__ __forceinline__ void stsm_x4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void stsm_x2(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("stmatrix.sync.aligned.m8n8.x2.shared.b16 [%0], {%1,%2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool soft_any(bool x) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(static_cast<uint32_t>(x)) : "memory");
  return r != 0;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int N>
__global__ void __launch_bounds__(kLThreads, 1)
latent_tc_kernel(const __grid_constant__ LMaps maps, const __grid_constant__ LatentParams p,
                 const __grid_constant__ LPlan plan) {
  using C = LCfg<N>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* rows_raw = smem + kLStages * kLStageBytes + C::kQBufs * C::kQBytes + C::kPBytes;
  float* wred = reinterpret_cast<float*>(rows_raw);                 // [4][N]
  float* alpha = wred + 4 * N;                                      // [N]
  int32_t* row_off = reinterpret_cast<int32_t*>(alpha + N);         // [N] offset of the row in out, in units of 8 elements; -1: none
  float* inv_l = wred;                                              // [N] (thread n replaces column n of what it has summed)
  uint64_t* bars = reinterpret_cast<uint64_t*>(rows_raw + C::kRowBytes);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 40);
  int* cta_err = reinterpret_cast<int*>(tmem_slot + 1);
  int* span = cta_err + 1;                                          // [4] first sequence, tile, tiles, its tokens
  uint32_t* scan = reinterpret_cast<uint32_t*>(wred);               // (start of the kernel only) warps' sums

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = blockIdx.x / plan.per_pass, r = blockIdx.x % plan.per_pass;
  const LatentGeom& geo = p.geom;
  const int m_tiles = geo.latent_dim / 128, n_groups = m_tiles + 1;
  const uint32_t ring = smem_u32(smem), q_sm = ring + kLStages * kLStageBytes, p_sm = q_sm + C::kQBufs * C::kQBytes;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kLStages * kLGroups;  // [stage][group]
  const uint32_t bar_s = empty0 + 8 * kLStages * kLGroups, bar_sfree = bar_s + 16, bar_p = bar_sfree + 16, bar_pv = bar_p + 8,
                 bar_q = bar_pv + 8, bar_qfree = bar_q + 16, bar_ofree = bar_qfree + 16, bar_drain = bar_ofree + 8;
  // (the set-up that reads nothing runs beside the end of the kernel before this one)
  if (warp == kLProducer && elect_one()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.line) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.pair) : "memory");
  }
  if (warp == kLQLoad && plan.q_box > 0 && elect_one()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q_latent) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q_rope) : "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < kLStages * kLGroups; ++i) {
      mbar_init(full0 + 8 * i, geo.page_size < kLTok ? 2 : 1);  // (one arrival per producer warp)
      mbar_init(empty0 + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_sfree + 8 * i, kLSoftWarps);
      mbar_init(bar_q + 8 * i, 1);      // Q buffer i
      mbar_init(bar_qfree + 8 * i, 1);
    }
    mbar_init(bar_p, kLSoftWarps);
    mbar_init(bar_pv, 1);
    mbar_init(bar_ofree, kLSoftWarps);
    mbar_init(bar_drain, 2);
    *cta_err = 0;
    span[0] = span[1] = span[2] = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (tensor memory only now: a kernel before this one may still have had to ask for its own)
  if (warp == kLSIssue) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kLTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const LatentWorkspace lay = latent_workspace_layout(p.num_q_heads, p.n_q, geo.latent_dim);
  uint8_t* ws = static_cast<uint8_t*>(p.workspace);
  // ---- this group's span of the tile list: every thread sums a run of sequences, then the sums are scanned
  const int per_thread = (p.batch + kLThreads - 1) / kLThreads;
  const int b0 = min(tid * per_thread, p.batch), b1 = min(b0 + per_thread, p.batch);
  uint32_t mine = 0;  // (the host has checked that the list fits 32 bits)
  for (int b = b0; b < b1; ++b) mine += seq_tiles(seq_tokens(p, b));
  uint32_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) scan[warp] = incl;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  uint32_t list = 0, before = 0;
#pragma unroll
  for (int w = 0; w < kLThreads / 32; ++w) {
    before += w < warp ? scan[w] : 0;
    list += scan[w];
  }
  before += incl - mine;
  const uint32_t total = list * plan.passes;
  // Equal spans, but of at least two tiles where sequences have at most two (a merge costs more than a tile: 100
  // tokens 10.2 instead of 11.4 us) or more than 32 (so many parts of one sequence cost more to merge: 8000 tokens,
  // 16 heads 16.7 instead of 20.0 us); in between single tiles are faster (8 x 700 tokens, 32 heads: 14.0, else 18.3 us).
  const uint32_t sequences = static_cast<uint32_t>(p.batch);
  const int span_tiles = max(static_cast<int>((total + plan.groups - 1) / plan.groups),
                             list <= 2 * sequences || list > 32 * sequences ? 2 : 1);
  const int64_t start = static_cast<int64_t>(g) * span_tiles;
  if (start < total) {
    const uint32_t pass = static_cast<uint32_t>(start) / list, in_pass = static_cast<uint32_t>(start) - pass * list;
    if (in_pass >= before && in_pass < before + mine) {  // (one thread)
      uint32_t at = before;
      for (int b = b0; b < b1; ++b) {
        const int L = seq_tokens(p, b);
        const uint32_t n = seq_tiles(L);
        if (in_pass < at + n) {
          span[3] = L;
          span[0] = static_cast<int>(pass) * p.batch + b;
          span[1] = static_cast<int>(in_pass - at);
          span[2] = static_cast<int>(min(static_cast<int64_t>(span_tiles), total - start));
          break;
        }
        at += n;
      }
    }
  }
  __syncthreads();
  const uint32_t tmem = *tmem_slot;
  Walk walk{span[0], span[1], span[2], span[3]};
  Segment s;
  bool ok = true;

  if (warp == kLProducer || (warp == kLProducer2 && geo.page_size < kLTok)) {
    // ================= TMA producer: lines of the tiles, in the order in which they are read and freed ========
    // (pages smaller than a tile: two warps share the copies, even and odd pages; one warp issues its 36
    // copies a tile no faster than one in 75 clocks, which was 4400 clocks a tile against 2700 from memory)
    const int odd = warp == kLProducer2 ? 1 : 0;
    const uint32_t leader = elect_one();
    const int box = uniform(min(geo.page_size, kLTok)), ept = kLTok / box;  // rows per copy, copies per line of a tile
    // row blocks of other CTAs read the same tiles: only a tile that is read once is marked to leave L2 first
    const uint64_t policy = plan.row_blocks == 1 ? l2_policy_evict_first() : l2_policy_normal();
    int i = 0;  // tiles of this CTA
    while (ok && next_segment<N>(p, plan, r, walk, s)) {
      if (s.n_tiles == 0) continue;
      const int32_t* table = p.block_table + static_cast<int64_t>(s.b) * p.block_table_stride;
      const int batch_tiles = 32 / ept;  // tiles whose page ids the lanes hold
      auto load_ids = [&](int t) -> int {  // lane -> copy (t + lane / ept, lane % ept) of this segment
        const int tile = t + lane / ept;
        if (tile >= s.n_tiles) return 0;
        const int tok0 = (s.tile0 + tile) * kLTok;  // (lengths go up to 2^31 - 1: nothing is added up beyond them)
        if ((lane % ept) * box >= s.L - tok0) return 0;
        const int tok = tok0 + (lane % ept) * box;
        const int v = __ldg(table + (tok >> plan.page_shift));
        return v < 0 || v >= geo.num_pages ? 0 : v;  // (the softmax warps look for these and drop the segment)
      };
      int ids = load_ids(0), ids_next = load_ids(batch_tiles);
      for (int t = 0; t < s.n_tiles; ++t, ++i) {
        const int in_batch = t % batch_tiles;
        if (in_batch == 0 && t > 0) {
          ids = ids_next;
          ids_next = load_ids(t + batch_tiles);
        }
        const int tok0 = (s.tile0 + t) * kLTok;
        const int n_copies = uniform((min(kLTok, s.L - tok0) + box - 1) / box);
        const uint32_t st = uniform(i & 1), sb = ring + st * kLStageBytes, bars0 = 8 * (st * kLGroups);
        const uint32_t parity = ((i >> 1) - 1) & 1;
        const uint32_t my_bytes = uniform((ept == 1 ? n_copies : (n_copies + 1 - odd) / 2) * box * 128);
        const int slot = uniform(tok0 & (geo.page_size - 1));
        int pages[2];  // of this warp's copies (a box of fewer than 64 rows is a whole page)
#pragma unroll
        for (int k = 0; k < 2; ++k) pages[k] = __shfl_sync(0xffffffffu, ids, (in_batch * ept + 2 * k + odd) & 31);
        // rope first: it is freed first (by the S product), then the latent pairs as P . C frees them
#pragma unroll
        for (int gr = 0; gr < kLGroups; ++gr) {
          if (gr >= n_groups) break;
          if (i >= kLStages) ok = mbar_spin_bounded(empty0 + bars0 + 8 * gr, parity);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const int line0 = gr == 0 ? 2 * m_tiles : 2 * (gr - 1);
          const uint32_t bar = full0 + bars0 + 8 * gr, dst = sb + line0 * kLLineBytes;
          mbar_expect_tx_if(leader, bar, gr == 0 ? my_bytes : 2 * my_bytes);
          // (a copy of 64 rows takes both lines of a group at once; smaller pages go line by line, so that
          // the rows of a line stay together)
          if (box == kLTok) {
            tma_load_4d_hint_if(leader, dst, gr == 0 ? &maps.line : &maps.pair, bar, slot, line0, pages[0], policy);
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int c = 2 * k + odd;
              if (c >= n_copies) break;
              tma_load_4d_hint_if(leader, dst + c * box * 128, &maps.line, bar, 0, line0, pages[k], policy);
              if (gr > 0) tma_load_4d_hint_if(leader, dst + kLLineBytes + c * box * 128, &maps.line, bar, 0, line0 + 1, pages[k], policy);
            }
          }
        }
        if (!ok) break;
      }
    }
    if (!ok) {  // copies in flight end before the CTA does
      if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
      for (int k = max(i - 1, 0); k <= i; ++k)
        for (int gr = 0; gr < n_groups; ++gr) mbar_wait_bounded(full0 + 8 * ((k & 1) * kLGroups + gr), (k >> 1) & 1, 1u << 12);
    }
  } else if (warp == kLSIssue) {
    // ================= S^T(i) = C . Q^T =================
    constexpr uint32_t idesc = latent_idesc(64, N, false, false);
    const uint32_t leader = elect_one();
    int i = 0, seg = 0;
    while (ok && next_segment<N>(p, plan, r, walk, s)) {
      if (s.n_tiles == 0) continue;
      // (segment seg is the (seg / bufs)-th in its buffer)
      const int qb = seg % C::kQBufs;
      ok = mbar_spin_bounded(bar_q + 8 * qb, (seg / C::kQBufs) & 1);
      for (int t = 0; ok && t < s.n_tiles; ++t, ++i) {
        const int st = i & 1;
        if (i >= 2) ok = mbar_spin_bounded(bar_sfree + 8 * st, ((i >> 1) - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        // (operands warp-uniform by a shuffle, offsets constant: 33 clocks an MMA; computed per thread: 100)
        const uint32_t d = uniform(tmem + kLTmemS + st * N), sb = uniform(ring + st * kLStageBytes), u_q = uniform(q_sm + qb * C::kQBytes);
#pragma unroll
        for (int gr = 0; gr < kLGroups; ++gr) {
          if (gr >= n_groups) break;
          ok = mbar_spin_bounded(full0 + 8 * (st * kLGroups + gr), (i >> 1) & 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const int line0 = gr == 0 ? 2 * m_tiles : 2 * (gr - 1);
          const uint64_t ad = tc_desc(sb + line0 * kLLineBytes, 16, 1024), bd = tc_desc(u_q + line0 * (N * 128), 16, 1024);
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) mma_ss_if(leader, d, ad + 2 * ks, bd + 2 * ks, idesc, (ks > 0 || gr > 0) ? 1u : 0u);
          if (gr > 0) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              mma_ss_if(leader, d, ad + kLLineBytes / 16 + 2 * ks, bd + N * 128 / 16 + 2 * ks, idesc, 1u);
          }
        }
        if (!ok) break;
        tc_commit_if(leader, bar_s + 8 * st);
        tc_commit_if(leader, empty0 + 8 * (st * kLGroups));  // the rope line is only read here
        if (t == s.n_tiles - 1) tc_commit_if(leader, bar_qfree + 8 * qb);
      }
      ++seg;
    }
    if (!ok) {
      if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    }
    tc_commit_if(leader, bar_drain);
  } else if (warp == kLPvIssue) {
    // ================= O^T += C^T . P^T(i) =================
    constexpr uint32_t idesc = latent_idesc(128, N, true, true);
    const uint32_t leader = elect_one();
    int i = 0, seg = 0;
    while (ok && next_segment<N>(p, plan, r, walk, s)) {
      if (s.n_tiles == 0) continue;
      if (seg > 0) ok = mbar_wait_bounded(bar_ofree, (seg - 1) & 1);
      for (int t = 0; ok && t < s.n_tiles; ++t, ++i) {
        const int st = i & 1;
        ok = mbar_spin_bounded(bar_p, i & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint64_t bd = tc_desc(uniform(p_sm), 16, 1024);
        const uint32_t sb = uniform(ring + st * kLStageBytes), d = uniform(tmem), bars0 = uniform(empty0 + 8 * (st * kLGroups + 1));
        const uint32_t acc = uniform(t > 0 ? 1u : 0u);
#pragma unroll
        for (int m = 0; m < kLGroups - 1; ++m) {
          if (m >= m_tiles) break;
          const uint64_t ad = tc_desc(sb + 2 * m * kLLineBytes, kLLineBytes, 1024);
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) mma_ss_if(leader, d + m * N, ad + 128 * ks, bd + 128 * ks, idesc, ks > 0 ? 1u : acc);
          tc_commit_if(leader, bars0 + 8 * m);
        }
        tc_commit_if(leader, bar_pv);
      }
      ++seg;
    }
    if (!ok) {
      if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    }
    tc_commit_if(leader, bar_drain);
  } else if (warp == kLQLoad) {
    // ================= Q rows of a segment: [line][N rows][128 B], swizzled =================
    int seg = 0;
    while (ok && next_segment<N>(p, plan, r, walk, s)) {
      if (s.n_tiles == 0) continue;
      const int qb = seg % C::kQBufs;
      const uint32_t bar_qb = uniform(bar_q + 8 * qb), q_to = uniform(q_sm + qb * C::kQBytes);
      if (seg >= C::kQBufs) {
        ok = mbar_spin_bounded(bar_qfree + 8 * qb, (seg / C::kQBufs - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
      }
      if (plan.q_box > 0) {
        // runs of q_box heads of one token (one query token: N heads, those beyond the last are zero)
        const uint32_t leader = elect_one();
        const int live = min(N, p.n_q * p.num_q_heads - s.rb * N);
        const int runs = (live + plan.q_box - 1) / plan.q_box, lines = 2 * m_tiles + 1;
        if (runs * plan.q_box < N) {
          // rows that there are not are zero: what an earlier segment left there would have its say in when the
          // references are raised, and so in the other rows' rounding
          const int first = runs * plan.q_box;
          for (int k = lane; k < lines * (N - first) * 8; k += 32) {
            const int ln = k / ((N - first) * 8), at = k - ln * (N - first) * 8;
            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(q_to + ln * (N * 128) + first * 128 + at * 16), "r"(0) : "memory");
          }
          fence_proxy_async();
          __syncwarp();
        }
        mbar_expect_tx_if(leader, bar_qb, uniform(runs * plan.q_box * lines * 128));
        for (int k = 0; k < runs; ++k) {
          const int row = s.rb * N + k * plan.q_box;
          const int t = uniform(row / p.num_q_heads), h = uniform(row - t * p.num_q_heads);
          const int token = uniform(s.b * p.n_q + t);
          const uint32_t dst = uniform(q_to + k * plan.q_box * 128);
          for (int ln = 0; ln < lines - 1; ++ln) tma_load_4d_if(leader, dst + ln * (N * 128), &maps.q_latent, bar_qb, ln, h, token);
          tma_load_4d_if(leader, dst + (lines - 1) * (N * 128), &maps.q_rope, bar_qb, 0, h, token);
        }
        ++seg;
        continue;
      }
      const int cv = geo.latent_dim / 8;
      for (int n = 0; n < N; ++n) {
        const int row = s.rb * N + n;
        const bool live = row < p.n_q * p.num_q_heads;
        const int t = row / p.num_q_heads, h = row - t * p.num_q_heads;
        const int64_t token = static_cast<int64_t>(s.b) * p.n_q + t;
        const __nv_bfloat16* ql = live ? p.q_latent + token * p.ql_token_stride + h * p.ql_head_stride : p.q_latent;
        const __nv_bfloat16* qr = live ? p.q_rope + token * p.qr_token_stride + h * p.qr_head_stride : p.q_rope;
        for (int c = lane; c < cv + 8; c += 32) {
          const __nv_bfloat16* src = c < cv ? ql + c * 8 : qr + (c - cv) * 8;
          cp_async16(q_to + (c >> 3) * (N * 128) + n * 128 + (((c & 7) ^ (n & 7)) << 4), live ? src : (c < cv ? ql : qr), live ? 16u : 0u);
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive_tc(bar_qb);
      ++seg;
    }
    if (!ok) {
      if (lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
      for (int k = max(seg - C::kQBufs, 0); k < seg; ++k)
        mbar_wait_bounded(bar_q + 8 * (k % C::kQBufs), (k / C::kQBufs) & 1, 1u << 12);
    }
  } else if (warp < kLSoftWarps) {
    // ================= softmax, output =================
    // After an expired wait a warp goes on without waiting (all eight meet at the same named barriers), and
    // what it writes is zero.
    constexpr int J = N / 16;  // column blocks of 8 of this warp; a thread's columns are col0 + 8 j + {0, 1}
    const int quad = warp & 3, half = warp >> 2;
    const float scale_log2 = p.scale * 1.4426950408889634f;
    const int tok_a = quad * 16 + (lane >> 2), tok_b = tok_a + 8;  // its tokens within the tile
    const int col0 = half * (N / 2) + 2 * (lane & 3);
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    const int rows_total = p.n_q * p.num_q_heads;
    LRecord rec{-1, 0, 0, 0};
    LRecord* records = reinterpret_cast<LRecord*>(ws + lay.records);
    int i = 0;
    bool first_in_span = true;
    while (next_segment<N>(p, plan, r, walk, s)) {
      const bool at_start = first_in_span;
      first_in_span = false;
      const bool is_first = s.off == 0, is_last = s.off + s.take == s.whole;
      if (is_first) {
        const LRecord now{is_last ? -1 : s.vseq, 2 * g + (at_start ? 0 : 1), 1 + (s.whole - s.take - 1) / span_tiles + 1, g};
        if (!is_last) rec = now;
        if (plan.by_sequence && r == 0 && tid == 0) records[s.vseq] = now;
      }
      if (s.rb < 0) continue;
      const bool partial = !(is_first && is_last);
      const int slot = 2 * g + (at_start ? 0 : 1);
      // row addresses; pages and length
      if (tid < N) {
        const int row = s.rb * N + tid;
        const int t = row / p.num_q_heads, h = row - t * p.num_q_heads;
        row_off[tid] = row < rows_total ? static_cast<int32_t>(((static_cast<int64_t>(s.b) * p.n_q + t) * p.out_token_stride +
                                                                h * p.out_head_stride) / 8) : -1;
      }
      bool bad = false;
      {
        const int raw = p.seq_lens[s.b];
        if (raw > 0 && s.L == 0 && tid == 0) report(p.status, PDA_DEV_BAD_SEQ_LEN);
        const int32_t* table = p.block_table + static_cast<int64_t>(s.b) * p.block_table_stride;
        const int64_t tok_end = min(static_cast<int64_t>(s.off + s.take) * kLTok, static_cast<int64_t>(s.L));
        const int pg1 = static_cast<int>((tok_end + geo.page_size - 1) >> plan.page_shift);
        for (int k = static_cast<int>((static_cast<int64_t>(s.off) * kLTok) >> plan.page_shift) + tid; k < pg1; k += kLSoft) {
          const int v = __ldg(table + k);
          bad |= v < 0 || v >= geo.num_pages;
        }
        if (bad) report(p.status, PDA_DEV_BAD_PAGE);
      }
      bad = soft_any(bad);

      float m_ref[2 * J], l[2 * J];
#pragma unroll
      for (int c = 0; c < 2 * J; ++c) { m_ref[c] = kLNoMax; l[c] = 0.f; }
      for (int t = 0; t < s.n_tiles; ++t, ++i) {
        const int st = i & 1;
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_s + 8 * st, (i >> 1) & 1));
        tc_fence_after();
        uint32_t sv[4 * J];
        tmem_ld_16x256b<J>(tmem + kLTmemS + st * N + half * (N / 2) + lane_base, sv);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_tc(bar_sfree + 8 * st);
        const int tok0 = (s.tile0 + t) * kLTok;
        const int valid = s.L - tok0;  // tokens of this tile (may be more than it has)
        float x[4 * J];
#pragma unroll
        for (int c = 0; c < 4 * J; ++c) x[c] = __uint_as_float(sv[c]) * scale_log2;
        if (valid < kLTok + p.n_q - 1) {  // the end of the sequence, or of what some query token may see
#pragma unroll
          for (int c = 0; c < 2 * J; ++c) {
            const int row = s.rb * N + 8 * (c >> 1) + col0 + (c & 1);
            const int lim = p.n_q == 1 ? valid : min(valid, valid - p.n_q + row / p.num_q_heads + 1);
            const int e = 4 * (c >> 1) + (c & 1);
            if (tok_a >= lim) x[e] = -INFINITY;
            if (tok_b >= lim) x[e + 2] = -INFINITY;
          }
          if (valid < kLTok) {
            // rows of the tile behind the sequence's end hold anything (pages' tails, an earlier tile): their
            // weight is 0, and so must be what it multiplies
            for (int k = tid; k < (kLTok - valid) * (geo.latent_dim / 8); k += kLSoft) {
              const int row = valid + k / (geo.latent_dim / 8), ch = k % (geo.latent_dim / 8);
              asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};"
                           ::"r"(ring + st * kLStageBytes + (ch >> 3) * kLLineBytes + row * 128 + (((ch & 7) ^ (row & 7)) << 4)), "r"(0));
            }
          }
        }
        bool above = false;
#pragma unroll
        for (int c = 0; c < 2 * J; ++c) {
          const int e = 4 * (c >> 1) + (c & 1);
          above |= fmaxf(x[e], x[e + 2]) > m_ref[c] + kLRescale;
        }
        const bool raise = soft_any(above);
        if (raise) {
          float mx[2 * J];
#pragma unroll
          for (int c = 0; c < 2 * J; ++c) {
            const int e = 4 * (c >> 1) + (c & 1);
            mx[c] = fmaxf(x[e], x[e + 2]);
          }
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1)
#pragma unroll
            for (int c = 0; c < 2 * J; ++c) mx[c] = fmaxf(mx[c], __shfl_xor_sync(0xffffffffu, mx[c], o));
          if (lane < 4) {
#pragma unroll
            for (int c = 0; c < 2 * J; ++c) wred[quad * N + 8 * (c >> 1) + col0 + (c & 1)] = mx[c];
          }
          soft_sync();
#pragma unroll
          for (int c = 0; c < 2 * J; ++c) {
            const int col = 8 * (c >> 1) + col0 + (c & 1);
            const float m_new = fmaxf(fmaxf(fmaxf(wred[col], wred[N + col]), fmaxf(wred[2 * N + col], wred[3 * N + col])), m_ref[c]);
            const float a = ex2(m_ref[c] - m_new);
            if (quad == 0 && lane < 4) alpha[col] = a;
            l[c] *= a;
            m_ref[c] = m_new;
          }
          soft_sync();
        }
        // weights (P's buffer and, where the reference rose, O are free once the last product is through)
        uint32_t pk[2 * J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float a0 = ex2(x[4 * j] - m_ref[2 * j]), a1 = ex2(x[4 * j + 1] - m_ref[2 * j + 1]);
          const float b0v = ex2(x[4 * j + 2] - m_ref[2 * j]), b1v = ex2(x[4 * j + 3] - m_ref[2 * j + 1]);
          l[2 * j] += a0 + b0v;
          l[2 * j + 1] += a1 + b1v;
          pk[2 * j] = pack2<false>(a0, a1);
          pk[2 * j + 1] = pack2<false>(b0v, b1v);
        }
        if (i > 0) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv, (i - 1) & 1));
        }
        if (raise && t > 0) {
          tc_fence_after();
          for (int cb = half * 16; cb < m_tiles * N; cb += 32) {
            uint32_t ov[16];
            tmem_ld16(tmem + lane_base + cb, ov);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
              const float4 a = *reinterpret_cast<const float4*>(alpha + (cb & (N - 1)) + k);
              ov[k] = __float_as_uint(__uint_as_float(ov[k]) * a.x);
              ov[k + 1] = __float_as_uint(__uint_as_float(ov[k + 1]) * a.y);
              ov[k + 2] = __float_as_uint(__uint_as_float(ov[k + 2]) * a.z);
              ov[k + 3] = __float_as_uint(__uint_as_float(ov[k + 3]) * a.w);
            }
            tmem_st16(tmem + lane_base + cb, ov);
          }
          tmem_wait_st();
          tc_fence_before();
        }
        {
          const int mi = lane >> 3, row = quad * 16 + (mi & 1) * 8 + (lane & 7), ch = half * J;
          if constexpr (J == 1) {
            stsm_x2(p_sm + row * 128 + ((ch ^ (row & 7)) << 4), pk[0], pk[1]);
          } else {
#pragma unroll
            for (int j = 0; j < J; j += 2)
              stsm_x4(p_sm + row * 128 + (((ch + j + (mi >> 1)) ^ (row & 7)) << 4), pk[2 * j], pk[2 * j + 1], pk[2 * j + 2], pk[2 * j + 3]);
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive_tc(bar_p);
      }

      // ---- the segment's result
      soft_sync();  // (alpha and wred: every warp is past the last tile)
#pragma unroll
      for (int o = 4; o <= 16; o <<= 1)
#pragma unroll
        for (int c = 0; c < 2 * J; ++c) l[c] += __shfl_xor_sync(0xffffffffu, l[c], o);
      if (lane < 4) {
#pragma unroll
        for (int c = 0; c < 2 * J; ++c) wred[quad * N + 8 * (c >> 1) + col0 + (c & 1)] = l[c];
      }
      if (quad == 0 && lane < 4) {
#pragma unroll
        for (int c = 0; c < 2 * J; ++c) alpha[8 * (c >> 1) + col0 + (c & 1)] = m_ref[c];
      }
      soft_sync();
      const int64_t part_row0 = (static_cast<int64_t>(slot) * plan.per_pass + r) * N;
      if (tid < N) {
        const float sum = (wred[tid] + wred[N + tid]) + (wred[2 * N + tid] + wred[3 * N + tid]);
        // A sum of zero: the row sees no token of this segment, or none that scores more than -inf. If that is all it has,
        // the first gives zeros and the second (0 * inf) NaN, which of a part the merge finds out.
        const bool sees = s.L - p.n_q + (s.rb * N + tid) / p.num_q_heads + 1 > 0;
        inv_l[tid] = bad || (sum == 0.f && (partial || !sees)) ? 0.f : 1.f / sum;
        // (a sum below zero marks a segment with a bad page: the merge then zeroes the row)
        if (partial) reinterpret_cast<float2*>(ws + lay.part_w)[part_row0 + tid] = make_float2(alpha[tid], bad ? -1.f : sum);
      }
      soft_sync();
      if (s.n_tiles > 0) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_spin_bounded(bar_pv, (i - 1) & 1));
        tc_fence_after();
      }
      for (int x0 = half * 16; x0 < m_tiles * N; x0 += 32) {  // 16 columns at a time, the two warps of 32 lanes in turn
        const int m = x0 / N, cb = x0 % N, dim = m * 128 + quad * 32 + lane;
        {
          uint32_t ov[16];
          tmem_ld16(tmem + lane_base + x0, ov);
          float v[16];
          int32_t off[16];
#pragma unroll
          for (int k = 0; k < 16; k += 4) {
            const float4 f = *reinterpret_cast<const float4*>(inv_l + cb + k);
            const int4 o = *reinterpret_cast<const int4*>(row_off + cb + k);
            v[k] = f.x; v[k + 1] = f.y; v[k + 2] = f.z; v[k + 3] = f.w;
            off[k] = o.x; off[k + 1] = o.y; off[k + 2] = o.z; off[k + 3] = o.w;
          }
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = s.n_tiles > 0 && ok && !bad ? __uint_as_float(ov[k]) * v[k] : 0.f;
          if (partial) {
            float* dst = reinterpret_cast<float*>(ws + lay.part_o) + (part_row0 + cb) * geo.latent_dim + dim;
#pragma unroll
            for (int k = 0; k < 16; ++k)
              if (off[k] >= 0) dst[k * geo.latent_dim] = v[k];
          } else {
            // neighbouring lanes swap, so that each stores two dims of one row
            const bool odd = lane & 1;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              const float other = __shfl_xor_sync(0xffffffffu, odd ? v[k] : v[k + 1], 1);
              const uint32_t w = odd ? pack2<false>(other, v[k + 1]) : pack2<false>(v[k], other);
              const int64_t to = odd ? off[k + 1] : off[k];
              if (to >= 0) *reinterpret_cast<uint32_t*>(p.out + 8 * to + (dim & ~1)) = w;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (s.n_tiles > 0 && lane == 0) mbar_arrive_tc(bar_ofree);
      soft_sync();  // (row_off and inv_l are free again)
    }
    if (!ok && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
    if (r == 0 && tid == 0 && !plan.by_sequence) records[g] = rec;
  }

  // ---- teardown
  __syncwarp();
  if (warp == kLPvIssue && !mbar_wait_bounded(bar_drain, 0, 1u << 12) && lane == 0) atomicMax(cta_err, PDA_DEV_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && *cta_err) report(p.status, *cta_err);
  if (warp == kLSIssue) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kLTmemCols) : "memory");
  }
}

// Rows of the sequences that lie in several spans. Grid: (record, row block, rows). kWide: a CTA per row, its
// warps sharing the row's segments (few sequences, each over many spans); else a warp per row (many
// sequences over two or three spans: a quarter of the CTAs).
constexpr int kMergeRows = 4, kMergeWideWarps = 8;
template <int N, bool kWide>
__global__ void __launch_bounds__(kWide ? kMergeWideWarps * 32 : kMergeRows * 32) latent_merge_kernel(const __grid_constant__ LatentParams p,
                                                                        const __grid_constant__ LPlan plan) {
  constexpr int kMergeWarps = kWide ? kMergeWideWarps : kMergeRows;
  __shared__ float4 acc_sh[kWide ? kMergeWarps - 1 : 1][kWide ? 128 : 1];
  __shared__ float w_sh[kMergeWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const LatentWorkspace lay = latent_workspace_layout(p.num_q_heads, p.n_q, p.geom.latent_dim);
  const uint8_t* ws = static_cast<const uint8_t*>(p.workspace);
  const LRecord rec = reinterpret_cast<const LRecord*>(ws + lay.records)[blockIdx.x];
  if (rec.vseq < 0) return;
  const int r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = kWide ? blockIdx.z : blockIdx.z * kMergeWarps + warp;
  const int row = ((rec.vseq / p.batch) * plan.per_pass + r) * N + n, b = rec.vseq % p.batch;
  if (row >= p.n_q * p.num_q_heads) return;  // (kWide: the whole CTA)
  const int t = row / p.num_q_heads, h = row - t * p.num_q_heads;
  __nv_bfloat16* out = p.out + (static_cast<int64_t>(b) * p.n_q + t) * p.out_token_stride + h * p.out_head_stride;
  const int vecs = p.geom.latent_dim / 4;  // 16-byte vectors of a partial row, a multiple of 32
  const bool sees = seq_tokens(p, b) - p.n_q + t + 1 > 0;
  const float2* wt = reinterpret_cast<const float2*>(ws + lay.part_w);
  const float4* part = reinterpret_cast<const float4*>(ws + lay.part_o);
  const int g0 = rec.group;
  auto row_of = [&](int k) -> int64_t {  // row of the k-th segment: later spans hold theirs in their first slot
    return (static_cast<int64_t>(k == 0 ? rec.first_slot : 2 * (g0 + k)) * plan.per_pass + r) * N + n;
  };
  // The first segments' rows are asked for before the weights are known: the trips to L2 are what this kernel
  // spends its time on.
  constexpr int kStep = kWide ? kMergeWarps : 1, kAhead = 2;
  const int k0 = kWide ? warp : 0;
  float4 x[kAhead][4];
#pragma unroll
  for (int a = 0; a < kAhead; ++a) {
    const int k = k0 + a * kStep;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (k < rec.n_seg && v * 32 < vecs) x[a][v] = part[row_of(k) * vecs + v * 32 + lane];
  }
  float M = kLNoMax;
  float2 mine = make_float2(kLNoMax, 0.f);  // the lane-th segment's reference and sum
  bool bad = false;                         // a bad page in some segment
  for (int k = lane; k < rec.n_seg; k += 32) {
    const float2 y = wt[row_of(k)];
    if (k == lane) mine = y;
    bad |= y.y < 0.f;
    M = fmaxf(M, y.x);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  bad = __any_sync(0xffffffffu, bad);
  const float w_mine = ex2(mine.x - M) * mine.y;
  float4 acc[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  float W = 0.f;
  auto add = [&](float w, const float4 (&y)[4]) {
    W += w;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (v * 32 < vecs) {
        acc[v].x = fmaf(w, y[v].x, acc[v].x); acc[v].y = fmaf(w, y[v].y, acc[v].y);
        acc[v].z = fmaf(w, y[v].z, acc[v].z); acc[v].w = fmaf(w, y[v].w, acc[v].w);
      }
    }
  };
  if (!bad) {  // (the whole warp)
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
      if (k0 + a * kStep < rec.n_seg) add(__shfl_sync(0xffffffffu, w_mine, k0 + a * kStep), x[a]);
#pragma unroll 4
    for (int k = k0 + kAhead * kStep; k < rec.n_seg; k += kStep) {
      const int64_t at = row_of(k);
      float4 y[4];
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (v * 32 < vecs) y[v] = part[at * vecs + v * 32 + lane];
      const float2 f = wt[at];
      add(ex2(f.x - M) * f.y, y);
    }
  }
  if constexpr (kWide) {  // warp 0 adds the warps' sums, in their order
    if (warp > 0) {
#pragma unroll
      for (int v = 0; v < 4; ++v) acc_sh[warp - 1][v * 32 + lane] = acc[v];
      if (lane == 0) w_sh[warp] = W;
    }
    __syncthreads();
    if (warp > 0) return;
    for (int u = 1; u < kMergeWarps; ++u) {
      W += w_sh[u];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float4 x = acc_sh[u - 1][v * 32 + lane];
        acc[v].x += x.x; acc[v].y += x.y; acc[v].z += x.z; acc[v].w += x.w;
      }
    }
  }
  const float inv = bad || (W == 0.f && !sees) ? 0.f : 1.f / W;  // (no finite score among what it sees: 0 * inf, a NaN)
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    if (v * 32 < vecs) {
      uint2 o;
      o.x = pack2<false>(acc[v].x * inv, acc[v].y * inv);
      o.y = pack2<false>(acc[v].z * inv, acc[v].w * inv);
      *reinterpret_cast<uint2*>(out + 4 * (v * 32 + lane)) = o;
    }
  }
}

// How many row blocks run at once, and how often: the choice that keeps most CTAs busy, for at most 37
// row blocks at once (four groups of CTAs), fewer rounds first.
LPlan make_plan(int row_blocks, int ctas) {
  LPlan best{row_blocks, 1, row_blocks, ctas, 0, 0, 0};
  double best_eff = -1.0;
  for (int passes = 1; passes <= row_blocks; ++passes) {
    const int per = (row_blocks + passes - 1) / passes;
    if (per > 37 || per > ctas) continue;
    const int groups = ctas / per;
    const double eff = static_cast<double>(row_blocks) / (static_cast<double>(passes) * per) * groups * per / ctas;
    if (eff > best_eff + 0.02) {
      best_eff = eff;
      best = LPlan{row_blocks, per, passes, groups, 0, 0, 0};
    }
    if (per == 1) break;
  }
  return best;
}

// Map of [pages][lines of 128 bytes][rows][64 elements], box [1][box_lines][box_rows][64].
bool encode_map(EncodeFn enc, CUtensorMap* map, const void* base, int64_t lines, int64_t rows, int64_t outer, int64_t row_stride,
                int64_t outer_stride, int box_lines, int box_rows, bool lines_inner) {
  const cuuint64_t rs = static_cast<cuuint64_t>(row_stride) * 2, os = static_cast<cuuint64_t>(outer_stride) * 2;
  const cuuint64_t nl = lines, nr = rows, no = outer;
  const cuuint64_t dims[4] = {64, lines_inner ? nl : nr, lines_inner ? nr : nl, no};
  const cuuint64_t strides[3] = {lines_inner ? 128 : rs, lines_inner ? rs : 128, os};
  const cuuint32_t bl = box_lines, br = box_rows;
  const cuuint32_t box[4] = {64, lines_inner ? bl : br, lines_inner ? br : bl, 1};
  const cuuint32_t step[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Heads per copy of Q: all N rows at once for one query token, else the largest run of heads that divides
// both a token's heads and a row block and keeps the swizzle's 8-row period; 0 where there is none, or where
// the strides are not a tensor map's.
int q_box_of(const LatentParams& p, int N) {
  const auto fits = [](int64_t stride, int64_t extent) { return extent == 1 || (stride > 0 && stride < (1ll << 38)); };
  const int64_t tokens = static_cast<int64_t>(p.batch) * p.n_q;
  if (!fits(p.ql_token_stride, tokens) || !fits(p.qr_token_stride, tokens) || !fits(p.ql_head_stride, p.num_q_heads) ||
      !fits(p.qr_head_stride, p.num_q_heads))
    return 0;
  if (p.n_q == 1) return N;
  for (int box = N; box >= 8; box /= 2)
    if (p.num_q_heads % box == 0) return box;
  return 0;
}

// Launch attributes: the kernel may be placed while the one before it on the stream ends (both kernels here
// wait for that one's end before they read anything).
struct OverlapConfig {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  OverlapConfig(dim3 grid, int threads, int smem, cudaStream_t stream) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
  }
};

template <int N>
cudaError_t launch_n(EncodeFn enc, LMaps& maps, const LatentParams& p, int sms, cudaStream_t stream) {
  const int rows = p.n_q * p.num_q_heads;
  LPlan plan = make_plan((rows + N - 1) / N, sms < kLatMaxCtas ? sms : kLatMaxCtas);
  plan.by_sequence = static_cast<int64_t>(p.batch) * plan.passes <= plan.groups;
  plan.page_shift = __builtin_ctz(p.geom.page_size);
  plan.q_box = q_box_of(p, N);
  if (plan.q_box > 0) {
    const int64_t tokens = static_cast<int64_t>(p.batch) * p.n_q;
    const auto some = [](int64_t stride, int64_t extent) { return extent == 1 ? int64_t{64} : stride; };  // (never stepped)
    if (!encode_map(enc, &maps.q_latent, p.q_latent, p.geom.latent_dim / 64, p.num_q_heads, tokens,
                    some(p.ql_head_stride, p.num_q_heads), some(p.ql_token_stride, tokens), 1, plan.q_box, true) ||
        !encode_map(enc, &maps.q_rope, p.q_rope, 1, p.num_q_heads, tokens, some(p.qr_head_stride, p.num_q_heads),
                    some(p.qr_token_stride, tokens), 1, plan.q_box, true))
      return cudaErrorNotSupported;
  }
  cudaError_t e = cudaFuncSetAttribute(latent_tc_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, LCfg<N>::kSmemBytes);
  if (e != cudaSuccess) return e;
  OverlapConfig attention(dim3(plan.groups * plan.per_pass), kLThreads, LCfg<N>::kSmemBytes, stream);
  if ((e = cudaLaunchKernelEx(&attention.cfg, latent_tc_kernel<N>, maps, p, plan)) != cudaSuccess) return e;
  // (the spans cut at most groups - 1 sequences: with few sequences those have many segments each)
  const int64_t sequences = static_cast<int64_t>(p.batch) * plan.passes;
  const bool wide = sequences * 4 <= plan.groups;
  OverlapConfig merge(dim3(plan.by_sequence ? static_cast<unsigned>(sequences) : plan.groups, plan.per_pass, wide ? N : N / kMergeRows), 32 * (wide ? kMergeWideWarps : kMergeRows), 0, stream);
  return wide ? cudaLaunchKernelEx(&merge.cfg, latent_merge_kernel<N, true>, p, plan)
              : cudaLaunchKernelEx(&merge.cfg, latent_merge_kernel<N, false>, p, plan);
}

}  // namespace

bool latent_tc_supports(const LatentParams& p) {
  const LatentGeom& g = p.geom;
  if (g.rope_dim != 64 || g.latent_dim % 128 || g.latent_dim > 512 || g.num_pages < 1) return false;
  if (g.page_size < 16 || (g.page_size & (g.page_size - 1))) return false;
  // what a tensor map can describe, and 32-bit tile counts
  if (g.page_stride >= (1ll << 38) || g.slot_stride >= (1ll << 38)) return false;
  const int64_t last_out = (static_cast<int64_t>(p.batch) * p.n_q - 1) * (p.out_token_stride / 8) + (p.num_q_heads - 1) * (p.out_head_stride / 8);
  if (last_out > INT32_MAX) return false;
  const int64_t row_blocks = (static_cast<int64_t>(p.n_q) * p.num_q_heads + kLatMaxRows - 1) / kLatMaxRows;
  // (rounds x sequences, and the tiles of all of them, are counted in 32 bits)
  const int64_t tiles = (static_cast<int64_t>(p.block_table_stride) * g.page_size + kLTok - 1) / kLTok + 1;
  return tiles <= INT32_MAX / (4 * row_blocks * p.batch);
}

cudaError_t launch_latent_tc(const LatentParams& p, cudaStream_t stream) {
  EncodeFn enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  const LatentGeom& g = p.geom;
  LMaps maps{};
  const int box = g.page_size < kLTok ? g.page_size : kLTok, lines = (g.latent_dim + g.rope_dim) / 64;
  if (!encode_map(enc, &maps.line, p.cache, lines, g.page_size, g.num_pages, g.slot_stride, g.page_stride, 1, box, false) ||
      !encode_map(enc, &maps.pair, p.cache, lines, g.page_size, g.num_pages, g.slot_stride, g.page_stride, 2, box, false))
    return cudaErrorNotSupported;
  int dev = 0, sms = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  switch (latent_tile_rows(static_cast<int64_t>(p.n_q) * p.num_q_heads)) {
    case 16: return launch_n<16>(enc, maps, p, sms, stream);
    case 32: return launch_n<32>(enc, maps, p, sms, stream);
    default: return launch_n<64>(enc, maps, p, sms, stream);
  }
}

}  // namespace pda
