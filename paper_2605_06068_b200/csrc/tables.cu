// paged_build_tables: block-table rows, slot map, positions and cumulative token counts of one step.
// Integer work on a few hundred lengths, so the time is launch and latency: one launch, in which every CTA
// scans all lengths by itself (256 or 1024 at a time, one per thread) and then writes its own share of the new
// pages and of the tokens. Nothing is handed from CTA to CTA: a page id is taken from the free list (or,
// for pages that were there before, from the table's untouched part), never read back from what another
// CTA writes. The order of pages and tokens is that of the scan, so results do not depend on timing.
// 256 sequences that grow by a token: 3.6 us in a graph; 96 prompts with 100k tokens: 4.3 us.
#include "latent.cuh"

namespace pda {

namespace {

constexpr int kTabTokensPerThread = 2;  // token entries a CTA writes

struct SeqStep {
  int held, take, start, n;  // pages before, pages taken, position of the first new token, new tokens
  bool bad;
};

__device__ __forceinline__ SeqStep load_step(const TablesParams& p, int b) {
  SeqStep s{0, 0, 0, 0, false};
  if (b >= p.batch) return s;
  const int L = p.seq_lens[b], n = p.new_lens[b];
  const int64_t room = static_cast<int64_t>(p.block_table_stride) * p.page_size;
  if (L < 0 || n < 0 || n > L || L > room) {
    s.bad = true;
    return s;
  }
  s.start = L - n;
  s.n = n;
  s.held = static_cast<int>((static_cast<int64_t>(L) - n + p.page_size - 1) / p.page_size);
  s.take = static_cast<int>((static_cast<int64_t>(L) + p.page_size - 1) / p.page_size) - s.held;
  return s;
}

// Exclusive scan of two counters over the CTA of kWarps warps; `tot` receives the sums.
template <int kWarps, class Acc>
__device__ __forceinline__ void block_scan2(Acc a, Acc b, Acc& ea, Acc& eb, Acc& tot_a, Acc& tot_b, Acc (*scratch)[kWarps]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Acc ia = a, ib = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Acc ua = __shfl_up_sync(0xffffffffu, ia, o), ub = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) { ia += ua; ib += ub; }
  }
  __syncthreads();  // (scratch may still be read by the previous step)
  if (lane == 31) { scratch[0][warp] = ia; scratch[1][warp] = ib; }
  __syncthreads();
  Acc wa = lane < kWarps ? scratch[0][lane] : 0, wb = lane < kWarps ? scratch[1][lane] : 0;
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const Acc ua = __shfl_up_sync(0xffffffffu, wa, o), ub = __shfl_up_sync(0xffffffffu, wb, o);
    if (lane >= o) { wa += ua; wb += ub; }
  }
  tot_a = __shfl_sync(0xffffffffu, wa, kWarps - 1);
  tot_b = __shfl_sync(0xffffffffu, wb, kWarps - 1);
  const Acc ba = __shfl_sync(0xffffffffu, wa, (warp + 31) & 31), bb = __shfl_sync(0xffffffffu, wb, (warp + 31) & 31);
  ea = ia - a + (warp ? ba : 0);
  eb = ib - b + (warp ? bb : 0);
}

// The k-th page of the step is the k-th from the top of the free list.
__device__ __forceinline__ int64_t count_index(int avail, int64_t k) { return avail - 1 - k; }

__device__ __forceinline__ int clamp_i32(int64_t v) { return static_cast<int>(v > INT32_MAX ? INT32_MAX : v); }

// Number of entries e of the ascending array a[0 .. n] with a[e] <= x, minus one: the sequence x falls in.
__device__ __forceinline__ int find(const int32_t* a, int n, int x) {
  int lo = 0, hi = n;  // a[lo] <= x < a[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// write_count: this launch stores free_count_out (it is another address than free_count, or no other CTA
// reads free_count). count_only: nothing but free_count_out is written.
// kThreads: sequences per scan step. Acc: 32 bits where no sum of lengths can pass them.
template <int kTabThreads, class Acc>
__global__ void __launch_bounds__(kTabThreads)
build_tables_kernel(TablesParams p, bool write_count, bool count_only) {
  constexpr int kTabTokensPerCta = kTabTokensPerThread * kTabThreads;
  __shared__ Acc scratch[2][kTabThreads / 32];
  __shared__ int32_t cu_s[kTabThreads + 1], tk_s[kTabThreads + 1], start_s[kTabThreads], held_s[kTabThreads];
  const int tid = threadIdx.x;
  const int avail = min(max(p.free_count[0], 0), p.free_capacity);

  // totals first: either every page that the step needs can be had, or none is taken
  SeqStep s{};
  Acc en = 0, et = 0;
  int64_t tot_n = 0, tot_t = 0;
  bool any_bad = false;
  for (int b0 = 0; b0 < p.batch; b0 += kTabThreads) {
    s = load_step(p, b0 + tid);
    any_bad |= s.bad;
    Acc cn, ct;
    block_scan2<kTabThreads / 32, Acc>(s.n, s.take, en, et, cn, ct, scratch);
    tot_n += cn;
    tot_t += ct;
  }
  const bool pages_ok = tot_t <= avail, slots_ok = tot_n <= p.capacity;
  const bool ok = pages_ok && slots_ok;
  if (blockIdx.x == 0 && !count_only) {
    if (any_bad) report(p.status, PDA_DEV_BAD_SEQ_LEN);
    if (tid == 0 && !pages_ok) report(p.status, PDA_DEV_NO_PAGES);
    if (tid == 0 && !slots_ok) report(p.status, PDA_DEV_NO_SLOTS);
  }
  if (blockIdx.x == 0 && write_count && tid == 0) p.free_count_out[0] = ok ? avail - static_cast<int>(tot_t) : avail;
  if (count_only) return;

  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTabTokensPerCta;
  const int64_t t1 = min(t0 + kTabTokensPerCta, static_cast<int64_t>(p.capacity));
  int64_t base_n = 0, base_t = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kTabThreads) {
    int64_t cn = tot_n, ct = tot_t;
    if (p.batch > kTabThreads) {
      s = load_step(p, b0 + tid);
      Acc sum_n, sum_t;
      block_scan2<kTabThreads / 32, Acc>(s.n, s.take, en, et, sum_n, sum_t, scratch);
      cn = sum_n;
      ct = sum_t;
    }
    if (blockIdx.x == 0 && b0 + tid < p.batch) {
      p.cu_new[b0 + tid] = clamp_i32(base_n + en);
      if (b0 + tid == p.batch - 1) p.cu_new[p.batch] = clamp_i32(base_n + en + s.n);
    }
    if (ok) {  // (all sums are then within 32 bits)
      __syncthreads();
      cu_s[tid] = static_cast<int>(base_n + en);
      tk_s[tid] = static_cast<int>(base_t + et);
      if (tid == kTabThreads - 1) {
        cu_s[kTabThreads] = static_cast<int>(base_n + cn);
        tk_s[kTabThreads] = static_cast<int>(base_t + ct);
      }
      start_s[tid] = s.start;
      held_s[tid] = s.held;
      __syncthreads();
      const int n_here = min(kTabThreads, p.batch - b0);
      // this CTA's share of the new pages
      for (int64_t k = base_t + static_cast<int64_t>(blockIdx.x) * kTabThreads + tid; k < base_t + ct;
           k += static_cast<int64_t>(gridDim.x) * kTabThreads) {
        const int i = find(tk_s, n_here, static_cast<int>(k));
        p.block_table[static_cast<int64_t>(b0 + i) * p.block_table_stride + held_s[i] + (k - tk_s[i])] =
            p.free_pages[count_index(avail, k)];
      }
      // its tokens
      for (int64_t t = max(t0, base_n) + tid; t < min(t1, base_n + cn); t += kTabThreads) {
        const int i = find(cu_s, n_here, static_cast<int>(t));
        const int pos = start_s[i] + static_cast<int>(t - cu_s[i]);
        const int lp = pos / p.page_size;
        const int page = lp >= held_s[i] ? p.free_pages[count_index(avail, tk_s[i] + (lp - held_s[i]))]
                                         : p.block_table[static_cast<int64_t>(b0 + i) * p.block_table_stride + lp];
        const int64_t slot = static_cast<int64_t>(page) * p.page_size + (pos - lp * p.page_size);
        const bool fine = page >= 0 && slot <= INT32_MAX;
        if (!fine) report(p.status, PDA_DEV_BAD_PAGE);
        p.slot_map[t] = fine ? static_cast<int>(slot) : -1;
        if (p.positions) p.positions[t] = pos;
      }
    }
    base_n += cn;
    base_t += ct;
  }
  // entries behind the last token (all of them when nothing could be placed)
  for (int64_t t = max(t0, ok ? tot_n : 0) + tid; t < t1; t += kTabThreads) {
    p.slot_map[t] = -1;
    if (p.positions) p.positions[t] = -1;
  }
  if (blockIdx.x == 0 && p.batch == 0 && tid == 0) p.cu_new[0] = 0;
}

}  // namespace

namespace {
template <int kThreads, class Acc>
cudaError_t launch(const TablesParams& p, cudaStream_t stream) {
  constexpr int kTokens = kTabTokensPerThread * kThreads;
  int64_t ctas = (static_cast<int64_t>(p.capacity) + kTokens - 1) / kTokens;
  if (ctas < 1) ctas = 1;
  // In place (free_count_out == free_count) with several CTAs: the new count is stored by a second launch,
  // after every CTA of the first has read the old one.
  const bool in_place = p.free_count == p.free_count_out && ctas > 1;
  build_tables_kernel<kThreads, Acc><<<static_cast<unsigned>(ctas), kThreads, 0, stream>>>(p, !in_place, false);
  if (in_place) build_tables_kernel<kThreads, Acc><<<1, kThreads, 0, stream>>>(p, true, true);
  return cudaGetLastError();
}
}  // namespace

// Up to 256 sequences fit a CTA of 256 threads, whose scan has two levels of 8 instead of 32.
cudaError_t launch_build_tables(const TablesParams& p, cudaStream_t stream) {
  const bool small_sums = static_cast<int64_t>(p.batch) * p.block_table_stride <= INT32_MAX / p.page_size;
  if (p.batch <= 256) return small_sums ? launch<256, int32_t>(p, stream) : launch<256, int64_t>(p, stream);
  return small_sums ? launch<1024, int32_t>(p, stream) : launch<1024, int64_t>(p, stream);
}

}  // namespace pda
