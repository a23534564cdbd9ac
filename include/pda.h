/* pda.h -- C ABI of the B200 (sm_100a) paged decode attention library (libpda.so).
 *
 * One decode step of one attention layer over a paged KV cache:
 *
 *     kv_append  ->  paged_decode_attention  ( ->  paged_decode_reduce )
 *
 * The operation is the one the serving stacks of the paper run at every decode
 * step on top of their "paged KV cache" with grouped-query attention ("32 query
 * heads sharing 8 key/value heads", Appendix A, Scenario A): for sequence b and
 * query head h, with kv head g = h / (num_q_heads / num_kv_heads),
 *
 *     out[b,h,:] = softmax_j( scale * q[b,h,:] . K_j[g,:] ) . V_j[g,:]
 *
 * over the sequence's tokens j = 0 .. seq_lens[b]-1 in logical order, token j
 * living in physical page block_table[b][j / page_size], slot j % page_size.
 * The paper names these ingredients but defines no layout; everything below is
 * this library's definition.
 *
 * Conventions
 *   - All data pointers are DEVICE pointers unless a comment says "host".
 *   - The caller owns every data buffer: inputs, outputs, partials, workspaces,
 *     status words. TMA descriptors are rebuilt per call on the host and passed by
 *     value. What the library itself owns, per process, is small and listed here:
 *       * per device, a second stream and two events, created by the first
 *         paged_prefix_decode_attention call on that device that is not inside a
 *         stream capture (the cascade's suffix launch runs on it);
 *       * per device, 64 claim counters (256 bytes of the library's device image)
 *         used by the persistent kernel of paged_verify_attention, each left at zero
 *         by the launch that took it;
 *       * per device, the PDA_STATIC_SCRATCH_BYTES array of
 *         paged_decode_attention_static (part of the device image: reserved when the
 *         image is loaded on that device, see there);
 *       * one host-side integer, the threshold of pda_set_persistent_threshold.
 *     No call allocates device memory with cudaMalloc or frees any; nothing else
 *     is kept between calls.
 *   - Every call enqueues work on `stream` (a cudaStream_t passed as void*) and
 *     returns without synchronising. Nothing reads seq_lens or block_table back
 *     to the host, so a step can be captured in a CUDA graph.
 *   - Return value: 0 = PDA_OK; < 0 = PDA_ERR_* detected on the host before
 *     anything was enqueued; > 0 = the cudaError_t of a failed launch.
 *   - `status` (optional, device int32, caller-zeroed): problems found on the
 *     device are recorded as PDA_DEV_*: the largest code stays, PDA_DEV_TIMEOUT
 *     above all others. The affected unit's output is zero-filled; no out-of-bounds
 *     access is ever made. Calls may share one word; while it holds
 *     PDA_DEV_TIMEOUT, the verification and prefix calls do not start their
 *     attention (their output is not to be used), the others work as ever.
 *   - bf16 = upper half of an IEEE binary32. e4m3 = OCP FP8 E4M3 (bias 7, max
 *     finite 448, no infinities, S.1111.111 = NaN).
 */
#ifndef PDA_H_
#define PDA_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PDA_VERSION 100

/* host-side return codes */
#define PDA_OK 0
#define PDA_ERR_INVALID_ARG (-1)  /* null pointer, negative size, inconsistent sizes          */
#define PDA_ERR_UNSUPPORTED (-2)  /* shape / dtype / stride outside the supported set          */
#define PDA_ERR_MISALIGNED (-3)   /* a pointer or stride breaks the 16-byte alignment rule     */
#define PDA_ERR_TOO_LARGE (-4)    /* size beyond a documented fixed maximum                    */

/* device-side status codes (in *status the largest stays, PDA_DEV_TIMEOUT above all) */
#define PDA_DEV_OK 0
#define PDA_DEV_BAD_PAGE 1     /* block_table entry outside [0, num_pages) for a live page     */
#define PDA_DEV_BAD_SEQ_LEN 2  /* seq_lens[b] > block_table_stride * page_size                 */
#define PDA_DEV_TIMEOUT 3      /* a bounded wait on an asynchronous copy expired               */
#define PDA_DEV_NO_PAGES 4     /* paged_build_tables: the free list holds fewer pages than asked */
#define PDA_DEV_NO_SLOTS 5     /* paged_build_tables: more new tokens than slot_map has room for */

/* KV element types */
#define PDA_BF16 0
#define PDA_FP8_E4M3 1

/* flags for paged_decode_attention */
#define PDA_FLAG_FORCE_GENERIC 1u /* use the plain CUDA-core kernel even where the
                                     TMA + tensor-core kernel applies (for testing) */

#define PDA_FLAG_MQ_MMA_SYNC 2u   /* multi-query calls (verify, shared prefix): use the mma.sync
                                     kernel even where the tcgen05 + TMEM kernel applies */
#define PDA_FLAG_MQ_ONE_UNIT 4u   /* paged_verify_attention: one CTA per (sequence, kv head, row block) even
                                     where a persistent tcgen05 kernel applies (unsplit, head_dim 128) */

typedef void* pda_stream_t; /* cudaStream_t */

/* Describes k_cache and v_cache (both have the same geometry).
 * Element (page, head, slot, d) lives at element offset
 *   page*page_stride + head*head_stride + slot*slot_stride + d.
 * The canonical layout is [num_pages, num_kv_heads, page_size, head_dim]
 * contiguous, i.e. slot_stride = head_dim, head_stride = page_size*head_dim,
 * page_stride = num_kv_heads*head_stride; any strides whose byte values are
 * multiples of 16 are accepted. */
typedef struct pda_cache_desc {
  int64_t page_stride;  /* elements */
  int64_t head_stride;  /* elements */
  int64_t slot_stride;  /* elements */
  int32_t num_pages;
  int32_t page_size;    /* tokens per page; supported: 16 */
  int32_t num_kv_heads;
  int32_t head_dim;     /* supported: multiples of 32 up to 256; fast path 64 and 128 */
  int32_t dtype;        /* PDA_BF16 or PDA_FP8_E4M3 */
} pda_cache_desc;

int pda_version(void);
const char* pda_status_string(int code); /* text for a PDA_ERR_* / PDA_DEV_* / 0 code */

/* ceil(max_seq_len / chunk_tokens): the `max_chunks` extent the partial buffers need. */
int pda_max_chunks(int32_t max_seq_len, int32_t chunk_tokens);

/* KV append (this step's scatter of new keys/values into the paged cache; the
 * paper's Appendix A lists the paged KV cache, not its update rule -- this is
 * the plain definition): for every sequence b with L = seq_lens[b] > 0 (length
 * AFTER the append) and every kv head g,
 *     cache[block_table[b][(L-1)/P]][g][(L-1)%P][:] = new[b][g][:]   (bytewise)
 * k_new, v_new: [batch, num_kv_heads, head_dim] bf16, contiguous. bf16 caches
 * only (PDA_ERR_UNSUPPORTED for e4m3). Target slots must be distinct across the
 * batch. A bad page id or length skips that sequence and sets *status.
 * desc is a host pointer, read during the call. */
int kv_append(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
              const pda_cache_desc* desc, const int32_t* block_table,
              int32_t block_table_stride, const int32_t* seq_lens, int32_t batch,
              int32_t* status, pda_stream_t stream);

/* Paged decode attention (definition at the top of this file; GQA head grouping
 * per Appendix A, Scenario A).
 *   q            [batch, num_q_heads, head_dim] bf16, contiguous
 *   k_scale,
 *   v_scale      [num_pages, num_kv_heads] fp32 dequantisation factors for e4m3
 *                caches (value = decode(byte) * scale); NULL for bf16 caches
 *   block_table  [batch, block_table_stride] int32; entries at or beyond
 *                ceil(seq_lens[b]/page_size) are never read
 *   scale        fp32 multiplier of q.k
 *   chunk_tokens 0: whole sequence per unit, result written to `out`
 *                [batch, num_q_heads, head_dim] bf16 (round to nearest even);
 *                a sequence of length 0 gives zeros.
 *                >0 (multiple of page_size): split-KV. Chunk c covers tokens
 *                [c*chunk_tokens, min((c+1)*chunk_tokens, L)); for every c <
 *                ceil(L/chunk_tokens) the kernel writes
 *                  part_o  [batch, num_q_heads, max_chunks, head_dim] fp32,
 *                          normalised within the chunk, and
 *                  part_lse[batch, num_q_heads, max_chunks] fp32 = m + ln(l)
 *                          (natural log of the chunk's softmax denominator);
 *                other entries are left untouched; `out` is not written.
 *                max_chunks * chunk_tokens must cover block_table_stride*page_size
 *                or at least every seq_lens[b] (longer sequences set *status).
 *   flags        PDA_FLAG_* bits
 * Unused slots of a last page, unused pages and table tails may hold any bit
 * pattern (NaN included). e4m3 caches: q is converted to fp16 for the tensor
 * core path, so |q| must stay below 65504.
 * Supported: page_size 16; num_q_heads a multiple of num_kv_heads; any group
 * size and head_dim (multiple of 32, <= 256) on the generic kernel; group size
 * <= 8 with head_dim 64 or 128 on the TMA + tensor-core kernel. */
int paged_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                           const pda_cache_desc* desc, const float* k_scale,
                           const float* v_scale, const int32_t* block_table,
                           int32_t block_table_stride, const int32_t* seq_lens,
                           int32_t batch, int32_t num_q_heads, float scale,
                           int32_t chunk_tokens, void* out, float* part_o, float* part_lse,
                           int32_t max_chunks, uint32_t flags, int32_t* status,
                           pda_stream_t stream);

/* Sliding-window decode attention: paged_decode_attention restricted, for every
 * sequence, to its last `window` tokens j in [max(0, L - window), L) (the
 * sliding-window attention over a paged per-stream cache of the paper's
 * streaming scenario, Appendix A, Scenario D; the paper gives no formula -- this
 * is the same softmax over that token range). window == 0 means no window.
 * Pages wholly before the window are never read, so their block_table entries
 * may be stale (evicted pages). With chunk_tokens > 0 the chunk grid stays the
 * one of the full sequence: chunks wholly before the window get o = 0 and
 * lse = -inf, and paged_decode_reduce merges as usual. Other arguments as in
 * paged_decode_attention. */
int paged_window_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                                  const pda_cache_desc* desc, const float* k_scale,
                                  const float* v_scale, const int32_t* block_table,
                                  int32_t block_table_stride, const int32_t* seq_lens,
                                  int32_t batch, int32_t num_q_heads, float scale, int32_t window,
                                  int32_t chunk_tokens, void* out, float* part_o, float* part_lse,
                                  int32_t max_chunks, uint32_t flags, int32_t* status,
                                  pda_stream_t stream);

/* Append of n_new tokens per sequence (the draft block of a verification step):
 * k_new, v_new are [batch, n_new, num_kv_heads, head_dim] bf16; token i becomes
 * logical token seq_lens[b] - n_new + i (seq_lens = length AFTER the append).
 * n_new == 1 is kv_append. */
int kv_append_tokens(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                     const pda_cache_desc* desc, const int32_t* block_table,
                     int32_t block_table_stride, const int32_t* seq_lens, int32_t batch,
                     int32_t n_new, int32_t* status, pda_stream_t stream);

/* Quantising KV append into e4m3 caches (no counterpart in the paper, whose one
 * remark on KV quantisation is negative; this is the library's policy). k_new,
 * v_new: [batch, num_kv_heads, head_dim] bf16. For K and V separately and every kv
 * head, with slot = (L-1) % page_size of the target page:
 *   slot == 0: scale[page, head] = amax(row) * 2 / 448 (1 if the row is all zero)
 *              is stored -- the page's scale is fixed by its first row;
 *   slot  > 0: the stored scale is reused;
 *   bytes = e4m3(row / scale): IEEE fp32 division, round to nearest even,
 *           saturating at +-448.
 * k_scale, v_scale: [num_pages, num_kv_heads] fp32, read and written. head_dim must
 * be a multiple of 64. Target slots must be distinct across the batch. */
int kv_append_fp8(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                  const pda_cache_desc* desc, float* k_scale, float* v_scale,
                  const int32_t* block_table, int32_t block_table_stride,
                  const int32_t* seq_lens, int32_t batch, int32_t* status, pda_stream_t stream);

/* The same for a block of n_new tokens per sequence (the draft block of a
 * verification step on an e4m3 cache): k_new, v_new are
 * [batch, n_new, num_kv_heads, head_dim] bf16, token i becomes logical token
 * seq_lens[b] - n_new + i, and the one-token rule above is applied to the tokens
 * in this order -- a page opened inside the block takes its scale from the
 * block's own row that lands in its slot 0. n_new == 1 is kv_append_fp8. */
int kv_append_tokens_fp8(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                         const pda_cache_desc* desc, float* k_scale, float* v_scale,
                         const int32_t* block_table, int32_t block_table_stride,
                         const int32_t* seq_lens, int32_t batch, int32_t n_new, int32_t* status,
                         pda_stream_t stream);

/* Verification attention over a block of n_query_tokens draft tokens per sequence
 * (the predicted-output verifier of the paper scores 16-token blocks in one pass:
 * Section 4.2 and Appendix A, Scenario B; the paper prints no formula -- this is
 * causal attention over the paged cache). The cache already holds all seq_lens[b]
 * tokens, the block being the last n_query_tokens of them; query token i stands at
 * position L - n + i and attends tokens j <= L - n + i.
 *   q, out    [batch, n_query_tokens, num_q_heads, head_dim] bf16
 *   chunk_tokens 0: one unit per (sequence, kv head).  > 0: split-KV; the partials
 *             part_o [batch, n, num_q_heads, max_chunks, head_dim] and part_lse
 *             [batch, n, num_q_heads, max_chunks] are scratch and the merge runs
 *             inside this call.  `out` is always written.
 * The query rows of a kv head's group form dense tensor-core tiles (rows = tokens x
 * group size), so each page is fetched once per block, not once per token.
 * bf16 KV with head_dim 128 or 64 and e4m3 KV with head_dim 128 run on tcgen05
 * tensor-core tiles with the accumulators in tensor memory (128 query rows per CTA);
 * PDA_FLAG_MQ_MMA_SYNC selects the mma.sync kernel instead. Unsplit calls with
 * head_dim 128 and up to 1024 sequences run as one persistent CTA per SM that walks
 * through the (sequence, kv head, row block) units, longest sequences first
 * (PDA_FLAG_MQ_ONE_UNIT: one CTA per unit). The bf16 one of these kernels shares out its last
 * units through a counter in device memory which the library owns (a pool of 64,
 * taken in turn by the launches and left at zero by each): up to 64 such launches
 * may be in flight at once on a device; a launch captured in a CUDA graph keeps its
 * counter, so one graph must not run beside itself on two streams.
 * e4m3 on tcgen05: the products are e4m3 x e4m3 on the cache's bytes; q enters as two
 * e4m3 parts (exact for every element within 2^-9 of its row's largest) and the softmax
 * weights as three 8-bit parts that add up to the weight rounded to fp16, the same
 * precision the mma.sync kernel gives them; the page scales go through the softmax.
 * Scales must be finite and non-negative (kv_append_fp8 writes them so). */
int paged_verify_attention(const void* q, const void* k_cache, const void* v_cache,
                           const pda_cache_desc* desc, const float* k_scale,
                           const float* v_scale, const int32_t* block_table,
                           int32_t block_table_stride, const int32_t* seq_lens, int32_t batch,
                           int32_t num_q_heads, int32_t n_query_tokens, float scale,
                           int32_t chunk_tokens, void* out, float* part_o, float* part_lse,
                           int32_t max_chunks, uint32_t flags, int32_t* status,
                           pda_stream_t stream);

/* Decode attention for a batch whose sequences all start with the SAME
 * prefix_tokens tokens stored in the same physical pages (the shared-prefix
 * prompt-caching workload of the paper: Section 4.2 and Appendix A, Scenario C).
 * The result is exactly paged_decode_attention's; the work is reorganised: the
 * prefix's keys/values are read once for the whole batch (all queries of a kv
 * head's groups as one block of rows), each sequence's own suffix is attended
 * separately, and the pieces are merged by their log-sum-exp weights.
 *   block_table    rows must agree on their first prefix_tokens/page_size entries
 *                  (row 0's are used); prefix_tokens is a multiple of page_size and
 *                  <= every seq_lens[b]
 *   prefix_chunk_tokens  split of the prefix for parallelism (multiple of page_size). The
 *                  prefix launch has ceil(batch * group / 128) * num_kv_heads CTAs per chunk,
 *                  each with a fixed cost of several microseconds: fastest with at most one
 *                  CTA per SM and chunks of 1024 tokens or more
 *   chunk_tokens   (> 0) split of the suffixes
 *   part_o, part_lse  scratch [batch, num_q_heads, max_chunks, head_dim] / [.., max_chunks]
 *                  with max_chunks >= ceil(prefix_tokens/prefix_chunk_tokens)
 *                                    + ceil((max seq_len - prefix_tokens)/chunk_tokens)
 *   out            [batch, num_q_heads, head_dim] bf16
 * Three launches (prefix, suffixes, merge), ordered on `stream`; the suffix launch,
 * which is independent of the prefix launch, runs beside it on a stream the
 * library owns (forked from and joined back to `stream` with events, which is
 * also valid while `stream` is being captured; the side stream is created by the
 * first call that is not inside a capture, and until it exists the launches simply
 * follow one another on `stream`). Supported: group size <= 8, head_dim 64/128
 * (bf16) or 128 (e4m3), batch <= 4096. The prefix launch is a multi-query call:
 * the kernel choice, `flags` and the e4m3 precision note of paged_verify_attention
 * apply to it. */
int paged_prefix_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                                  const pda_cache_desc* desc, const float* k_scale,
                                  const float* v_scale, const int32_t* block_table,
                                  int32_t block_table_stride, const int32_t* seq_lens,
                                  int32_t batch, int32_t num_q_heads, float scale,
                                  int32_t prefix_tokens, int32_t prefix_chunk_tokens,
                                  int32_t chunk_tokens, void* out, float* part_o, float* part_lse,
                                  int32_t max_chunks, uint32_t flags, int32_t* status,
                                  pda_stream_t stream);

/* Merge of split-KV partials (the reduce step of flash-decoding; exact algebra):
 *     out[b,h,:] = sum_c w_c part_o[b,h,c,:] / sum_c w_c,
 *     w_c = exp(part_lse[b,h,c] - max_c part_lse[b,h,c]),  c < ceil(L_b/chunk_tokens)
 * out: [batch, num_q_heads, head_dim] bf16. A sequence without chunks gives zeros. */
int paged_decode_reduce(const float* part_o, const float* part_lse, const int32_t* seq_lens,
                        int32_t batch, int32_t num_q_heads, int32_t head_dim,
                        int32_t chunk_tokens, int32_t max_chunks, void* out,
                        pda_stream_t stream);

/* Tuning knob (process-wide, host side): an unsplit paged_decode_step with a workspace
 * and batch <= 256 runs on the persistent kernel (resident CTAs looping over (sequence, kv
 * head) units through the workspace's work ticket, longest first) once there are at least
 * min_units_per_cta units per resident CTA (2 per SM); below that, one CTA per unit is
 * faster. Default 6. 0 always selects the persistent kernel where it applies (tests). */
int pda_set_persistent_threshold(int32_t min_units_per_cta);

/* Number of int32 the `workspace` of paged_decode_step needs: 2 + batch*num_kv_heads. */
int pda_workspace_ints(int32_t batch, int32_t num_kv_heads);

/* One whole decode step of this layer in a single launch: KV append (when k_new
 * and v_new are given; both NULL skips it), paged decode attention and, for
 * chunk_tokens > 0, the merge of the split-KV partials -- the three calls above
 * fused, with the same definitions; `out` [batch, num_q_heads, head_dim] bf16 is
 * always written. The append is applied to the cache and seen by this step's
 * attention.
 *   part_o, part_lse, max_chunks  as in paged_decode_attention (chunk_tokens > 0)
 *   workspace  device int32[pda_workspace_ints(batch, num_kv_heads)], zeroed by the
 *              caller ONCE (e.g. at allocation); every call leaves it zeroed again,
 *              so consecutive calls on one stream may share it. Calls that can
 *              overlap on the GPU need separate workspaces. It carries the work
 *              the work ticket of the persistent kernel (two leading ints)
 *              and the per-(sequence, kv head) chunk counters. May be NULL when chunk_tokens == 0. After a
 *              PDA_DEV_TIMEOUT status, zero it again.
 * If chunk_tokens > 0 and workspace is NULL, or the shape is outside the fused
 * kernel's set (group size > 8, head_dim not 64/128), the step is
 * run as the separate launches instead, with the same result. */
int paged_decode_step(const void* q, const void* k_new, const void* v_new, void* k_cache,
                      void* v_cache, const pda_cache_desc* desc, const float* k_scale,
                      const float* v_scale, const int32_t* block_table,
                      int32_t block_table_stride, const int32_t* seq_lens, int32_t batch,
                      int32_t num_q_heads, float scale, int32_t chunk_tokens, void* out,
                      float* part_o, float* part_lse, int32_t max_chunks, int32_t* workspace,
                      int32_t* status, pda_stream_t stream);

/* seq_lens[b] += delta for every b, on the device and in stream order. Lets a
 * whole decode step -- advance the lengths, then paged_decode_step -- be captured
 * once in a CUDA graph and replayed every token with no host work (CUDA-graph
 * capture of the step is the most frequent single win the paper reports:
 * Section 4.2, Scenarios B, C, D and F). Grids never depend on seq_lens, the
 * caches' addresses are baked into the captured launch, and the block table must
 * already hold the pages the growing sequences will reach. */
int pda_advance_seq_lens(int32_t* seq_lens, int32_t batch, int32_t delta, pda_stream_t stream);

/* One whole decode step driven from HOST buffers (the end-to-end call): copies
 * this step's q, k_new, v_new, seq_lens and block_table from (ideally pinned)
 * host memory into the caller's device staging buffers, runs
 * paged_decode_step (workspace as described there, may be NULL), and copies
 * `out` back to out_host; all on `stream`, without synchronising. The KV cache
 * itself stays resident on the device between steps. *_dev are device buffers
 * of the same sizes as their host counterparts.
 * In place: q_dev, k_new_dev, v_new_dev, block_table_dev, seq_lens_dev and
 * out_dev may each be NULL; the kernel then reads (for out: writes) the host
 * buffer itself over the bus while it streams the cache, and that copy and its
 * launch drop out of the step. This needs pinned host memory that is mapped into
 * the device's address space (cudaHostAlloc, cudaHostRegister);
 * PDA_ERR_INVALID_ARG otherwise. With out_dev == NULL the result exists in
 * out_host only. Every CTA reads seq_lens and its row of block_table at its
 * start, so reading those two in place trades two copies ahead of the launch
 * for a bus round trip inside each CTA's start; the host must not change any
 * in-place buffer before the step has completed. */
int paged_decode_step_host(const void* q_host, const void* k_new_host, const void* v_new_host,
                           const int32_t* block_table_host, const int32_t* seq_lens_host,
                           void* q_dev, void* k_new_dev, void* v_new_dev,
                           int32_t* block_table_dev, int32_t* seq_lens_dev,
                           void* k_cache, void* v_cache, const pda_cache_desc* desc,
                           int32_t block_table_stride, int32_t batch, int32_t num_q_heads,
                           float scale, int32_t chunk_tokens, float* part_o, float* part_lse,
                           int32_t max_chunks, int32_t* workspace, void* out_dev, void* out_host,
                           int32_t* status, pda_stream_t stream);

/* Split-KV attention plus reduce with library-owned scratch. (The paper has no
 * counterpart; this entry point exists for integration reasons only.)
 *
 * Some callers cannot hand the library partial buffers because they cannot get
 * device memory when the call is made: a serving process whose start-up code has
 * already claimed the whole HBM for its KV pool and weights, so that any later
 * cudaMalloc fails; a plug-in that runs inside a host application's context and
 * was given no allocator; or a latency-critical loop in which an allocation's
 * implicit device synchronisation is not acceptable. For them this call does what
 * paged_decode_attention(chunk_tokens > 0) followed by paged_decode_reduce does,
 * but keeps part_o / part_lse in a fixed array of PDA_STATIC_SCRATCH_BYTES
 * compiled into the library's device image. It calls no cudaMalloc, cudaFree or
 * other allocating routine.
 *
 * The array is part of the device code of the library, and the CUDA runtime loads
 * device code lazily: the image that holds the array is loaded on a device -- and
 * its PDA_STATIC_SCRATCH_BYTES of device memory reserved there, until the process
 * exits -- by the FIRST call of this function on that device, which looks up the
 * array's device address (with that device current) and caches it. That first
 * call therefore synchronises like any module load and fails with the runtime's
 * out-of-memory code (a positive return value) if the device has no room left.
 * Make it once per device at start-up: before the process hands the rest of HBM
 * to its pools, and outside any stream capture (a call with batch 0 is enough and
 * enqueues nothing). Every later call on that device reserves nothing: the free
 * memory the runtime reports is the same before and after it.
 *
 * Arguments are those of paged_decode_attention without the partial buffers and
 * flags; `out` is [batch, num_q_heads, head_dim] bf16. The sizes must satisfy
 *   round_up(batch*num_q_heads*max_chunks*head_dim*4, 256)
 *     + batch*num_q_heads*max_chunks*4  <=  PDA_STATIC_SCRATCH_BYTES,
 * otherwise PDA_ERR_TOO_LARGE is returned and nothing is enqueued.
 *
 * The array is shared by all calls and keeps the previous call's contents:
 * nothing in it needs to start at zero (attention writes every entry that reduce
 * reads), but two calls whose kernels can overlap on the GPU (different streams,
 * or different host threads without ordering) race on it. Calls on one stream are
 * ordered and safe. */
#define PDA_STATIC_SCRATCH_BYTES (16u * 1024u * 1024u)
int paged_decode_attention_static(const void* q, const void* k_cache, const void* v_cache,
                                  const pda_cache_desc* desc, const float* k_scale,
                                  const float* v_scale, const int32_t* block_table,
                                  int32_t block_table_stride, const int32_t* seq_lens,
                                  int32_t batch, int32_t num_q_heads, float scale,
                                  int32_t chunk_tokens, int32_t max_chunks, void* out,
                                  int32_t* status, pda_stream_t stream);

/* Diagnostic: decodes all 256 e4m3 bytes with the device decoder the generic
 * kernel uses; out256: device float[256]. */
int pda_debug_e4m3_decode(float* out256, pda_stream_t stream);

/* Diagnostic: makes the kernels' bounded waits run out. (No counterpart in the
 * paper; this exercises the library's own failure handling.) Every wait inside the
 * attention kernels is a wait of a warp on an mbarrier of its own CTA with a poll
 * limit, after which the kernel records PDA_DEV_TIMEOUT in *status, zero-fills the
 * unit's output and returns. This call launches one warp that initialises such a
 * barrier, never arrives at it, and runs the same two wait helpers (the suspended
 * try_wait form of the TMA rings, the spinning test_wait form of the tensor-core
 * hand-offs) with `polls` as their limit instead of the built-in 2^18 (4.0 us per
 * poll: 1.05 s) and 2^24 (21.9 ns per poll: 0.37 s).
 * Nothing faults and nothing waits without a limit; the context stays usable.
 *   polls   1 .. 2^20
 *   status  device int32: receives PDA_DEV_TIMEOUT
 *   result  device uint64[3] or NULL: nanoseconds spent in the suspended and in the
 *           spinning wait, and a mask of the waits that wrongly reported completion
 *           (must be 0). */
int pda_debug_wait_timeout(uint32_t polls, int32_t* status, uint64_t* result, pda_stream_t stream);

/* Diagnostic: read-only streaming probe. Reads `bytes` (a multiple of 16) from the
 * 16-byte aligned device buffer `buf` once with 16-byte loads from 8 CTAs per SM
 * and writes nothing but (practically never) one counter word `sink` (device
 * uint32). Timed by the caller with events, bytes / time is the bandwidth a kernel
 * that only reads HBM can reach on this device: the ceiling beside which the
 * decode kernels' GB/s are to be read (a copy moves half its bytes as writes and
 * is the lower figure). */
int pda_debug_read_probe(const void* buf, uint64_t bytes, uint32_t* sink, pda_stream_t stream);

/* ---- Step tables and latent attention ---------------------------------------------
 *
 * A latent cache holds, for every token, ONE row shared by all query heads:
 *     row = [ c (latent_dim elements) | r (rope_dim elements) ]        bf16
 * c is the compressed vector from which every head's keys and values are projected
 * (k_nope[h] = Wk[h] c, v[h] = Wv[h] c), r the rotary part of the key, the same for
 * all heads. (The paper has no counterpart; the calls below are this library's.) The
 * attention over it has two forms that give the same result:
 *   expanded  keys [k_nope[h] | r] and values v[h] per head, as the projections leave
 *             them: latent_prefill_attention, for prompts;
 *   absorbed  the projections moved to the query and the output (q_latent[h] =
 *             Wk[h]^T q_nope[h], v-part = Wv[h] out[h]), so that the cached rows
 *             themselves are keys and values: paged_latent_attention, for decoding.
 * A step: paged_build_tables -> latent_append -> one of the two. */

/* Element (page, slot, d) of the cache lives at page*page_stride + slot*slot_stride + d,
 * d < latent_dim + rope_dim. Strides in elements, their byte values multiples of 16.
 * page_size 1..1024; latent_dim a multiple of 8, 8..1024; rope_dim a multiple of 8,
 * 0..256. dtype: PDA_BF16. */
typedef struct pda_latent_desc {
  int64_t page_stride;
  int64_t slot_stride;
  int32_t num_pages;
  int32_t page_size;
  int32_t latent_dim;
  int32_t rope_dim;
  int32_t dtype;
} pda_latent_desc;

/* The tables of one step, built on the device from request lengths. With P = page_size,
 * L = seq_lens[b] (length AFTER the step), n = new_lens[b] (tokens of this step, 0..L):
 *     held = ceil((L - n) / P) pages are in block_table[b] already,
 *     need = ceil(L / P); entries [held, need) are written with new pages: page k of the
 *     step, counted in (b, page) order, is free_pages[free_count - 1 - k];
 *     cu_new[b] = n_0 + ... + n_{b-1}, b = 0 .. batch;
 *     token t = cu_new[b] + i (i < n) stands at position L - n + i of sequence b:
 *     positions[t] = L - n + i,
 *     slot_map[t] = block_table[b][positions[t] / P] * P + positions[t] % P;
 *     slot_map[t] = positions[t] = -1 for cu_new[batch] <= t < capacity;
 *     *free_count_out = *free_count - (pages taken).
 *   free_pages      int32[free_capacity], the free page ids, a stack whose top is at
 *                   *free_count - 1 (values beyond free_capacity count as free_capacity,
 *                   negative ones as 0, for *free_count_out too);
 *                   read only: to give pages back, write their ids at *free_count onwards
 *                   and raise it
 *   free_count_out  may be free_count itself
 *   slot_map        int32[capacity]; positions int32[capacity] or NULL
 *   batch           >= 0; page_size 1..1024
 * A sequence with n < 0, n > L, L < 0 or L > block_table_stride * P gets nothing (n counts as
 * 0) and *status PDA_DEV_BAD_SEQ_LEN. Where the free list is too short (PDA_DEV_NO_PAGES) or
 * the tokens are more than capacity (PDA_DEV_NO_SLOTS), no page is taken, the table stays as
 * it was and every slot_map and positions entry is -1 (cu_new counts all the same). A page id below 0, or one whose slots pass 2^31 - 1,
 * gives slot -1 and PDA_DEV_BAD_PAGE. Entries of block_table beyond need are left as they are. */
int paged_build_tables(const int32_t* seq_lens, const int32_t* new_lens, int32_t batch,
                       int32_t page_size, const int32_t* free_pages, int32_t free_capacity,
                       const int32_t* free_count, int32_t* free_count_out, int32_t* block_table,
                       int32_t block_table_stride, int32_t* cu_new, int32_t* slot_map,
                       int32_t* positions, int32_t capacity, int32_t* status, pda_stream_t stream);

/* Rows of n_tokens new tokens into their slots of the latent cache: for slot_map[t] = s >= 0
 *     row(s / P, s % P) = [ f(c_new[t]) | rope_new[t] ],
 *     f(c) = c bytewise (norm_weight NULL), or the root-mean-square norm
 *     f(c) = bf16(c / sqrt(mean(c^2) + eps) * norm_weight), in 32 bits, rounded once.
 *   c_new     [n_tokens, latent_dim] bf16, c_stride elements from token to token
 *   rope_new  [n_tokens, rope_dim] bf16, rope_stride elements from token to token (both may
 *             be parts of one buffer; NULL with rope_dim 0)
 *   slot_map  int32[n_tokens]; entries < 0 are skipped, entries beyond the cache are
 *             skipped with PDA_DEV_BAD_PAGE. Entries >= 0 must be distinct.
 *   eps       >= 0, finite */
int latent_append(const void* c_new, int64_t c_stride, const void* rope_new, int64_t rope_stride,
                  void* cache, const pda_latent_desc* desc, const void* norm_weight, float eps,
                  const int32_t* slot_map, int32_t n_tokens, int32_t* status,
                  pda_stream_t stream);

/* Absorbed attention of n_query_tokens tokens per sequence over the paged latent cache. Query
 * token i of sequence b stands at position L - n + i (L = seq_lens[b], n = n_query_tokens; the
 * cache holds all L rows) and attends tokens j <= L - n + i:
 *     out[b,i,h,:] = softmax_j( scale * (q_latent[b,i,h] . c_j + q_rope[b,i,h] . r_j) ) . c_j
 *   q_latent  [batch, n, num_q_heads, latent_dim] bf16: element (token, head, d) at
 *             token*ql_token_stride + head*ql_head_stride + d, token = b*n + i
 *   q_rope    [batch, n, num_q_heads, rope_dim] bf16, likewise (NULL with rope_dim 0)
 *   out       [batch, n, num_q_heads, latent_dim] bf16, likewise
 *             (strides: multiples of 8 elements, >= 0; out rows must not overlap)
 *   block_table, seq_lens  as in paged_decode_attention, with desc's page size
 *   workspace device memory of pda_latent_workspace_bytes(...) bytes, 256-byte aligned. Need
 *             not be initialised, holds nothing between calls; calls that can overlap on the
 *             GPU (graphs replayed side by side included) need separate ones.
 *   flags     PDA_FLAG_FORCE_GENERIC
 * Rows whose range is empty (L = 0, or i < n - L) are zero. L < 0 counts as 0. A bad page id or
 * length zeroes the sequence's rows and sets *status. Every slot holding a live token must be
 * finite; all other slots, pages and table entries may hold anything.
 * 1 <= n <= 4096, batch * n <= 65535. The tensor-core kernel (tcgen05) takes latent_dim 128, 256,
 * 384 or 512 with rope_dim 64 and page sizes 16, 32, 64, 128 and larger powers of two; other
 * shapes run on a plain kernel, which takes a CTA per query row. Scores are held in 32 bits: a row
 * with a NaN or +inf among those it sees, or with none above -inf, is NaN. Results do not depend on
 * timing: sums are taken in an order fixed by the lengths and the number of SMs. */
int paged_latent_attention(const void* q_latent, int64_t ql_token_stride, int64_t ql_head_stride,
                           const void* q_rope, int64_t qr_token_stride, int64_t qr_head_stride,
                           const void* cache, const pda_latent_desc* desc,
                           const int32_t* block_table, int32_t block_table_stride,
                           const int32_t* seq_lens, int32_t batch, int32_t num_q_heads,
                           int32_t n_query_tokens, float scale, void* out,
                           int64_t out_token_stride, int64_t out_head_stride, void* workspace,
                           int64_t workspace_bytes, uint32_t flags, int32_t* status,
                           pda_stream_t stream);

/* Bytes of workspace that paged_latent_attention needs, or PDA_ERR_INVALID_ARG. */
int64_t pda_latent_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t n_query_tokens,
                                   int32_t latent_dim);

/* Expanded attention of packed ragged sequences (prompts, or chunks of prompts behind a
 * context): sequence b has query tokens cu_q[b] .. cu_q[b+1]-1 and key tokens cu_k[b] ..
 * cu_k[b+1]-1, aligned at their ends: with nq and nk of them, query i attends keys
 * j <= nk - nq + i:
 *     out[i,h,:] = softmax_j( scale * (q[i,h,:nope] . k_nope[j,h] + q[i,h,nope:] . k_rope[j]) ) . v[j,h]
 *   q       [total_q, num_heads, nope_dim + rope_dim] bf16
 *   k_nope  [total_k, num_heads, nope_dim], v [total_k, num_heads, v_dim] bf16 (may be the two
 *           parts of one buffer); k_rope [total_k, rope_dim], one for all heads (NULL with
 *           rope_dim 0)
 *   out     [total_q, num_heads, v_dim] bf16
 *           Strides in elements, multiples of 8, >= 0; rows of out must not overlap.
 *   cu_q, cu_k  device int32[batch + 1], ascending
 *   max_q   an upper bound of the sequences' query tokens (host: the launch is sized by it)
 * Rows without any key are zero. Rows of out outside all sequences are left as they were, and
 * rows of the inputs outside all sequences may hold anything: neither what stands there nor what
 * stands in other sequences changes a bit of a sequence's result (the lengths may: they decide how
 * the work is cut). Within a sequence q and the keys may hold anything (a row with a NaN or +inf
 * among the scores it sees, or with none above -inf, is NaN, and no other row is), but every value
 * v must be finite: on the tensor-core kernel an infinity or NaN in v makes earlier rows NaN too,
 * whose weight for it is 0. Scores are held in 32 bits. A sequence whose ranges do not lie in the
 * arrays or that has more than max_q query tokens is zeroed (as far as its rows lie within the
 * array and max_q) and sets *status PDA_DEV_BAD_SEQ_LEN.
 * nope_dim, v_dim: multiples of 8 up to 512; rope_dim a multiple of 8 up to 256; batch and
 * num_heads <= 65535; the smaller of max_q and total_q times num_heads < 2^31. Dims 128, 64 and
 * 128 run on the tensor-core kernel (tcgen05); other dims, a scale that is not above 0 and finite,
 * token or head strides of 0 (a broadcast) in an extent above 1 and PDA_FLAG_FORCE_GENERIC on a
 * plain kernel, which takes a CTA per query row and head. */
int latent_prefill_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride,
                             const void* k_nope, int64_t kn_token_stride, int64_t kn_head_stride,
                             const void* k_rope, int64_t kr_token_stride, const void* v,
                             int64_t v_token_stride, int64_t v_head_stride, const int32_t* cu_q,
                             const int32_t* cu_k, int32_t batch, int32_t num_heads,
                             int32_t nope_dim, int32_t rope_dim, int32_t v_dim, int32_t max_q,
                             int32_t total_q, int32_t total_k, float scale, void* out,
                             int64_t out_token_stride, int64_t out_head_stride, uint32_t flags,
                             int32_t* status, pda_stream_t stream);

/* ---- Rotated keys into the paged cache, and attention with shaped scores ------------
 *
 * The layer's step around the paged key/value cache of grouped-query attention: what lies
 * between the projection and the cache (rope_kv_append), and attention over the cache for
 * prompts (paged_prefill_attention) and for one token per sequence
 * (paged_biased_decode_attention), whose scores may be capped, biased by distance and
 * masked. (The paper has no counterpart; the calls below are this library's.)
 * A step: paged_build_tables -> rope_kv_append -> one of the two. */

/* From product to score, for query head h at position p and key j:
 *     s = scale * (q . k_j)
 *     s = softcap * tanh(s / softcap)          if softcap > 0
 *     s = s - slopes[h] * |p - j|              if slopes
 * in 32 bits, and the softmax is over the keys that the token sees. window > 0: among them only
 * j > p - window. scale finite, softcap finite and >= 0, slopes finite; log2(e) scale, log2(e) softcap and
 * 2 log2(e) scale / softcap within 32 bits' range too. A cap of any size is off by 2^-20 of the score at most,
 * one up to 128 by 2^-17 of the cap besides. */
typedef struct pda_score_desc {
  float scale;
  float softcap;        /* 0: none */
  const float* slopes;  /* device fp32[num_q_heads], or NULL */
  int32_t window;       /* 0: none */
} pda_score_desc;

/* A step's queries, keys and values as the projection leaves them: for every token t with slot
 * slot_map[t] = s >= 0
 *     q_out[t,h]  = R_t(N(q[t,h], q_norm))     bf16
 *     key row     = R_t(N(k[t,g], k_norm))     into k_cache, page s / 16, slot s % 16, head g
 *     value row   = v[t,g]                     into v_cache
 *   N(x, w)   x / sqrt(mean(x^2) + eps) * w over the head's head_dim elements; x where w is NULL
 *   R_t       rotation of the first rot_dim elements; the others stay. Frequency f of
 *             rot_dim / 2 turns the pair (x_f, x_{f + rot_dim/2}), or with `interleaved`
 *             (x_{2f}, x_{2f+1}), by the angle whose cosine and sine are
 *             cos_sin[p][f] and cos_sin[p][rot_dim/2 + f], p = positions[axis(f)][t]:
 *                 (a, b) -> (a cos - b sin, b cos + a sin)
 *   all of it in 32 bits, rounded once. q_norm, k_norm: bf16[head_dim].
 *   bf16 caches: rows rounded to bf16. e4m3 caches: the rule of kv_append_tokens_fp8, on the 32-bit
 *   rows: a row in slot 0 sets its page's scale, amax * 2 / 448 (1 for a row of zeros), the others take the
 *   stored one; a page that the call opens must have its rows of this call one behind the other in
 *   the token array, in the order of their slots (as paged_build_tables lays them out).
 *   q, k, v     [n_tokens, heads, head_dim] bf16 (may be parts of one buffer)
 *   q_out       likewise; may be q itself
 *               (strides in elements, multiples of 8, >= 0, from head to head below 2^31, the caches'
 *               included; rows of q_out must not overlap)
 *   positions   int32[num_axes][n_tokens], positions_stride elements from axis to axis;
 *               num_axes 1..4. NULL with rot_dim 0
 *   freq_axis   HOST uint8[rot_dim / 2], the axis of each frequency, read during the call; NULL: axis 0
 *   cos_sin     fp32 [table_len][rot_dim], contiguous, 16-byte aligned; NULL with rot_dim 0
 *   rot_dim     0..head_dim, a multiple of 16
 *   slot_map    int32[n_tokens]. A token with an entry < 0 is left out altogether (its row of q_out stays
 *               as it was). An entry beyond the cache: no cache row, PDA_DEV_BAD_PAGE. Entries >= 0
 *               must be distinct.
 * A token with a position outside [0, table_len) among the axes that its frequencies use gets a row of
 * zeros in q_out, no cache row, and PDA_DEV_BAD_SEQ_LEN. desc is that of both caches. */
int rope_kv_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k,
                   int64_t k_token_stride, int64_t k_head_stride, const void* v,
                   int64_t v_token_stride, int64_t v_head_stride, const int32_t* positions,
                   int64_t positions_stride, int32_t num_axes, const uint8_t* freq_axis,
                   const float* cos_sin, int32_t table_len, int32_t rot_dim, int32_t interleaved,
                   const void* q_norm, const void* k_norm, float eps, const int32_t* slot_map,
                   int32_t n_tokens, int32_t num_q_heads, void* q_out, int64_t qo_token_stride,
                   int64_t qo_head_stride, void* k_cache, void* v_cache,
                   const pda_cache_desc* desc, float* k_scale, float* v_scale, int32_t* status,
                   pda_stream_t stream);

/* Attention of packed ragged sequences (prompts, or chunks of prompts behind a context) over the
 * paged cache: sequence b has query tokens cu_q[b] .. cu_q[b+1]-1, the last nq of the seq_lens[b] = L
 * tokens whose keys and values the cache holds. Its i-th query token stands at position
 * p = L - nq + i and sees the keys lo <= j < hi,
 *     hi = max(p + 1, min(prefix_lens[b], L)),  lo = max(0, p - window + 1, first_keys[t]);
 *     out[t,h,:] = softmax_{lo <= j < hi}( score ) . V_j[g,:]       (score: pda_score_desc)
 *   q, out       [total_q, num_q_heads, head_dim] bf16. Strides in elements, multiples of 8,
 *                >= 0; rows of out must not overlap
 *   cu_q         int32[batch + 1], ascending
 *   max_q        an upper bound of the sequences' query tokens (host: the launch is sized by it)
 *   prefix_lens  int32[batch], tokens at the start that every query token sees, or NULL
 *   first_keys   int32[total_q], the first key that a query token sees (its document's start), or NULL
 *   k_scale .. seq_lens  as in paged_decode_attention
 *   workspace    device memory of pda_prefill_workspace_bytes bytes, 256-byte aligned, or NULL. With it,
 *                sequences of few query tokens and many keys are cut along the keys. Need not be
 *                initialised, holds nothing between calls; calls that can overlap on the GPU
 *                (graphs replayed side by side included) need separate ones.
 *   flags        PDA_FLAG_FORCE_GENERIC
 * Rows that see nothing (p < 0, lo >= hi) are zero. Rows of out outside all sequences are left as they
 * were, and rows of q outside all sequences may hold anything. Slots that hold no token < L, unused pages
 * and table entries of pages that no token sees may hold anything; the values of all tokens < L in
 * pages that are seen must be finite (and on the tensor-core kernel below 2^64 in size; e4m3 value scales
 * there 0 or at least 2^-56). A row with a NaN or +inf among the scores it sees is NaN;
 * one with none above -inf is NaN or zero. L < 0 counts as 0. A sequence whose query range does not
 * lie in the arrays, that has more than max_q query tokens or more than block_table_stride * 16 or
 * 2^30 tokens is zeroed (as far as its rows lie within the array and max_q; one that starts below 0 is left
 * out) with PDA_DEV_BAD_SEQ_LEN; rows for
 * which a page id outside the cache is read are zero, with PDA_DEV_BAD_PAGE.
 * batch and num_q_heads <= 65535; the smaller of max_q and total_q times num_q_heads < 2^31. Groups of up
 * to 128 query heads with head_dim 64 and 128 run on the tensor-core kernel (tcgen05; e4m3: head_dim 128);
 * other head_dims, caches without pages, token or head strides of 0 in an extent above 1 and
 * PDA_FLAG_FORCE_GENERIC on a plain kernel, which takes a warp per query row. */
int paged_prefill_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride,
                            const void* k_cache, const void* v_cache, const pda_cache_desc* desc,
                            const float* k_scale, const float* v_scale, const int32_t* block_table,
                            int32_t block_table_stride, const int32_t* seq_lens,
                            const int32_t* cu_q, int32_t batch, int32_t num_q_heads, int32_t max_q,
                            int32_t total_q, const pda_score_desc* score,
                            const int32_t* prefix_lens, const int32_t* first_keys, void* out,
                            int64_t out_token_stride, int64_t out_head_stride, void* workspace,
                            int64_t workspace_bytes, uint32_t flags, int32_t* status,
                            pda_stream_t stream);

/* Bytes of workspace that paged_prefill_attention uses, or PDA_ERR_INVALID_ARG. */
int64_t pda_prefill_workspace_bytes(int32_t num_q_heads, int32_t head_dim);

/* The same for one token per sequence: query b stands at position p = seq_lens[b] - 1 and sees the
 * keys max(0, p - window + 1, first_keys[b]) <= j <= p.
 *   q, out       [batch, num_q_heads, head_dim] bf16, contiguous
 *   first_keys   int32[batch] or NULL
 *   chunk_tokens 0: one unit per (sequence, kv head); > 0 (a multiple of 16): split into chunks of at most
 *                so many tokens, with part_o, part_lse and max_chunks as in paged_decode_attention; they are
 *                scratch, and the merge runs inside this call. Chunks are joined by their log-sum-exp in 32
 *                bits: beside the largest scores' size s a chunk's weight is off by 2^-23 s at most
 *   workspace    (chunk_tokens > 0) int32[pda_workspace_ints(batch, num_kv_heads * ceil(group / 8))] as in
 *                paged_decode_step: zeroed by the caller once, left zeroed, one per stream of overlapping
 *                calls. NULL: the merge is a launch of its own
 *   flags        PDA_FLAG_FORCE_GENERIC
 * `out` is always written: zeros where nothing is seen (an empty sequence). What is not seen may hold
 * anything, in pages that are read too. NaN and infinite scores, lengths and page ids as in
 * paged_prefill_attention. bf16 with head_dim 64, 128 and 256 and e4m3 with head_dim 128 run on the TMA +
 * tensor-core kernel (there e4m3 takes queries in fp16: |q| below 65504, in
 * steps of 2^-24 below 2^-14), groups above 8 heads as several units; other
 * shapes on a plain kernel, which does not split. */
int paged_biased_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                                  const pda_cache_desc* desc, const float* k_scale,
                                  const float* v_scale, const int32_t* block_table,
                                  int32_t block_table_stride, const int32_t* seq_lens,
                                  int32_t batch, int32_t num_q_heads, const pda_score_desc* score,
                                  const int32_t* first_keys, int32_t chunk_tokens, void* out,
                                  float* part_o, float* part_lse, int32_t max_chunks,
                                  int32_t* workspace, uint32_t flags, int32_t* status,
                                  pda_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* PDA_H_ */
