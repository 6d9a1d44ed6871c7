/*
 * ac.h -- C ABI of the B200 (sm_100a) paged decode-attention library (libac.so).
 *
 * One decode step of one attention layer, for a batch of requests that each contribute ONE new
 * token, over a paged KV cache:
 *
 *   ac_rope_kv_append      rotary embedding of the new q and k, then the new k/v are written into
 *                          their cache page through the block table
 *   ac_paged_decode_attn   grouped-query attention of each request's query token over all of its
 *                          cached pages, one CTA per (request, KV head, KV split), online softmax;
 *                          emits per-split partial results (or the final output when 1 split)
 *   ac_splitkv_merge       log-sum-exp merge of the per-split partial results
 *
 * Source of each operation (the paper gives them in prose only): Method, "Principle-Driven LLM
 * Kernel Generator", kernel families (iii) "standalone RoPE kernel" and (iv) "paged decode
 * attention ... online-softmax kernel over paged KV with fused cross-CTA merging"; Method, "Kernel
 * Customization and Multi-Request Adaptation": the kv_append scatter kernel ("writes the new K/V
 * vectors", attention then runs "with the sequence length advanced by one"), the paged KV cache
 * allocated at block granularity, sequence lengths kept on the GPU, and decode steps replayed as
 * bucketed CUDA Graphs (one graph per batch-size bucket).
 *
 * General rules
 *   - Every pointer is a DEVICE pointer owned by the caller unless its name ends in _host or
 *     _out.  The library never allocates or frees device memory, never synchronises and never reads
 *     device memory on the host: each call only validates its arguments and enqueues work on
 *     `stream` (a cudaStream_t passed as void*; NULL = the legacy default stream).  The three kernel
 *     calls may therefore be recorded in a CUDA Graph; ac_init must have been called before capture.
 *   - The kernels are launched with programmatic stream serialization and signal launch completion
 *     early, so that in a chain of calls each kernel's set-up overlaps the tail of the one before.
 *     Before synchronising on the preceding kernel the attention kernels read only context_lens,
 *     block_table and cache tiles below the one holding slot context_lens[b] - 1 (over an 8-bit cache, whose
 *     append also rewrites the slots in front of its own in a block: below the block holding that slot, and
 *     no scales), and the projection kernels only their weights.  The attention and RoPE kernels signal only after their own
 *     synchronisation, so no kernel that writes the cache can still be running two launches back:
 *     consecutive steps on one cache need nothing between them.  The early reads are invisible
 *     unless the kernel enqueued directly before one of these calls BOTH writes context_lens,
 *     block_table or those weights AND itself signals programmatic launch completion before
 *     finishing; such a producer must not signal early (copies and ordinary kernels are always safe).
 *   - Tensors q/k/v/cache/out are bf16 (16-bit patterns); rope tables and partials are fp32;
 *     block_table and context_lens are int32.  The innermost dimension (head_dim) is contiguous.
 *   - Return value: AC_OK (0) or an ac_status > 0.  On any non-zero return nothing was launched.
 *     The library never throws, aborts or exits.
 *   - Supported: head_dim d in {64, 128}; page_size a multiple of 16, <= 256; Hq % Hkv == 0 and
 *     Hq / Hkv <= 16; all base pointers 16-byte aligned; cache strides multiples of 8 elements and
 *     stride_token, stride_head >= d.
 *   - Rows with context_lens[b] < 0 are inactive (batch padding up to a graph bucket): nothing is
 *     written to the cache for them and their output row is +0.
 *   - Query head hq reads KV head hq / (Hq / Hkv).
 */
#ifndef AC_H_
#define AC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    AC_OK = 0,
    AC_ERR_NULL = 1,        /* a required pointer is NULL */
    AC_ERR_SHAPE = 2,       /* a size is non-positive or inconsistent */
    AC_ERR_UNSUPPORTED = 3, /* outside the supported set listed above */
    AC_ERR_ALIGN = 4,       /* pointer or stride alignment */
    AC_ERR_WORKSPACE = 5,   /* workspace too small for num_splits */
    AC_ERR_CUDA = 6,        /* a CUDA call failed; see ac_last_cuda_error() */
    AC_ERR_NOT_INIT = 7,    /* ac_init has not succeeded on the current device */
    AC_ERR_SCRATCH_LIMIT = 8 /* ac_paged_decode_attn_static_scratch: partials exceed AC_STATIC_SCRATCH_BYTES */
} ac_status;

/* Bits the kernels OR into the optional device word `status_flag` (never cleared by the library). */
#define AC_FLAG_PAGE_OOB 1     /* a block-table entry used for the append was outside [0, num_pages) */
#define AC_FLAG_POSITION_OOB 2 /* context_lens[b] >= max_position or its page index >= max_pages_per_seq; in the
                                  single-launch step also context_lens[b] + 1 > the tokens the split grid covers */
#define AC_FLAG_WAIT_TIMEOUT 4 /* a bounded wait on a shared-memory barrier gave up */
#define AC_FLAG_POOL_EXHAUSTED 8 /* ac_cache_reserve / ac_cache_fork: fewer free pages than the call needs */
#define AC_FLAG_REF_COUNT 16 /* a page that a row holds has reference count 0 (released twice, or never taken) */
#define AC_FLAG_ROW_OOB 32 /* a row index outside the block table */

/* Once per device, outside any stream capture, with no other call of this library running on that
 * device: reads the device properties, resolves the driver's tensor-map encoder and sets the
 * dynamic shared-memory limits of every kernel instantiation.  device < 0 means the current device.
 * Idempotent. */
int ac_init(int device);

/* Static, never-freed description of a status code. */
const char* ac_status_string(int status);

/* cudaError_t (or CUresult, for tensor-map encoding) recorded by the last AC_ERR_CUDA on this thread. */
int ac_last_cuda_error(void);

/* Number of SMs of the device ac_init saw last; 0 before any ac_init. */
int ac_sm_count(void);

/* Split plan (host only, pure, needs no GPU).  Chooses how many KV splits the attention kernel
 * should use for `sm_count` SMs (<= 0: the count seen by ac_init, or 148 if none): none when the
 * (request, KV head) pairs alone fill the GPU and contexts are short, chunks of at most 4096 tokens
 * when contexts are long, and otherwise the split count with the smallest estimated time from a
 * small cost model (bandwidth of one CTA, waves of CTAs, partial-result traffic); splits are never
 * shorter than 256 tokens, or 128 where the grid is small enough for the merge inside a cluster.  max_context_len = the largest number of tokens any row attends over in this bucket
 * (cached + new).  Outputs: *num_splits_out >= 1, *split_tokens_out = tokens per split (a multiple
 * of 64; split s of row b covers tokens [s*split_tokens, min((s+1)*split_tokens, n_b)), the last one
 * all that are left), and *workspace_bytes_out = bytes of fp32 workspace the attention + merge calls
 * need for that plan (0 when num_splits == 1).  The paper's kernel merges across CTAs inside the attention kernel and
 * does not state how it sizes the split; this heuristic is this library's own. */
int ac_decode_plan(int B, int Hq, int Hkv, int d, int page_size, int max_context_len, int sm_count,
                   int* num_splits_out, int* split_tokens_out, size_t* workspace_bytes_out);

/* The same plan for a batch whose row lengths the caller knows (a scheduler builds context_lens on
 * the host anyway).  token_counts_host[b] = tokens row b attends over this step (cached + new; <= 0
 * for an inactive row), a HOST array of B entries; max_context_len >= every entry bounds the chunk
 * grid as in ac_decode_plan (counts above it are clipped).  Splits that lie beyond a row's end launch
 * CTAs that exit at once, so a ragged batch can afford more and shorter splits than its longest row
 * alone suggests: the estimate counts only the CTAs that have tokens, the longest of them, and the
 * batch's total bytes.  Same outputs and errors as ac_decode_plan; any plan gives the same results. */
int ac_decode_plan_for_lengths(const int32_t* token_counts_host, int B, int Hq, int Hkv, int d,
                               int page_size, int max_context_len, int sm_count,
                               int* num_splits_out, int* split_tokens_out, size_t* workspace_bytes_out);

/* Tokens per split the attention kernel uses for a given (max_context_len, num_splits): the smallest
 * multiple of 64 whose num_splits-fold covers max_context_len.  Host only, pure. */
int ac_split_tokens(int max_context_len, int num_splits);

/* Largest number of tokens a row is partitioned over under a sliding window with sinks: window + 63, plus
 * sinks rounded up to a multiple of 16 when there are any; INT_MAX for window <= 0 (no bound but the
 * context).  Host only, pure. */
int ac_window_span(int window, int sinks);

/* Workspace bytes for (B, Hq, d, num_splits): partial_o fp32 [B,Hq,num_splits,d] followed by
 * partial_lse fp32 [B,Hq,num_splits]; 0 when num_splits == 1.  Host only, pure. */
size_t ac_workspace_bytes(int B, int Hq, int d, int num_splits);

/* A1 + A2: RoPE on the new q/k and KV append (families (iii) "standalone RoPE kernel" and the
 * kv_append scatter kernel of "Kernel Customization and Multi-Request Adaptation").
 *
 * For every active row b, with p = context_lens[b] (the position of the new token, 0-based):
 *   q_out[b,h,:]  = rope(q_in[b,h,:], p)   for all Hq heads   (q_out may alias q_in)
 *   k_cache[page, slot, h, :] = rope(k_new[b,h,:], p),  v_cache[page, slot, h, :] = v_new[b,h,:]
 *   for all Hkv heads, page = block_table[b, p / page_size], slot = p % page_size.
 * rope pairs element i with i + d/2 (i < d/2):  (x_i, x_{i+d/2}) -> (x_i c - x_{i+d/2} s,
 * x_{i+d/2} c + x_i s) with c = rope_cos[p, i], s = rope_sin[p, i].  Each result is the
 * round-to-nearest-even bf16 of the real value (products exact, one fp64 addition, one rounding), so
 * cache contents are reproducible bit for bit.  v is copied verbatim.
 *
 * Layout: q_in/q_out [B,Hq,d], k_new/v_new [B,Hkv,d] dense; cache element (page, slot, head, j) at
 * page*stride_page + slot*stride_token + head*stride_head + j (strides in elements);
 * block_table [B, max_pages_per_seq]; rope_cos/rope_sin [max_position, d/2].
 * A row whose position or page id is out of range writes nothing and sets status_flag bits (if
 * status_flag != NULL).  Two rows appending into the same slot is a caller error (not detected). */
int ac_rope_kv_append(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                      void* k_cache, void* v_cache,
                      int64_t stride_page, int64_t stride_token, int64_t stride_head,
                      const int32_t* block_table, int max_pages_per_seq,
                      const int32_t* context_lens,
                      const float* rope_cos, const float* rope_sin, int max_position,
                      int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                      int32_t* status_flag, void* stream);

/* Prelude variants of A1 (the paper's attention-prelude family (i) names "optionally ... per-head
 * Q/K RMSNorm"; its per-model adaptations mention partial rotary embeddings).  Zero-initialise. */
typedef struct ac_rope_options {
    int rotary_dim;            /* 0 or d: rotate the whole vector; else even, < d: only elements
                                  [0, rotary_dim) are rotated, the rest pass through; the rope tables
                                  are then [max_position, rotary_dim/2] */
    int interleaved;           /* 0: pair element i with i + rotary_dim/2; 1: pair 2i with 2i + 1 */
    const void* q_norm_weight; /* device bf16 [d] or NULL: RMSNorm of every q head vector before the
                                  rotation: y = bf16(bf16(x / sqrt(mean(x^2) + eps)) * w) */
    const void* k_norm_weight; /* same for k (v is never normalised) */
    float norm_eps;
    int reserved[4];
} ac_rope_options;

/* ac_rope_kv_append with options (NULL = plain call).  Everything else as ac_rope_kv_append; the
 * rotation keeps its exact-then-round arithmetic, the norm is evaluated in fp64 (sum of squares,
 * square root and division correctly rounded) and rounded to bf16 where the formula above says. */
int ac_rope_kv_append_ex(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                         void* k_cache, void* v_cache,
                         int64_t stride_page, int64_t stride_token, int64_t stride_head,
                         const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* context_lens,
                         const float* rope_cos, const float* rope_sin, int max_position,
                         int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                         int32_t* status_flag, void* stream, const ac_rope_options* options);

/* Attention-prelude fusion, the paper's kernel family (i) ("QKV projection + RoPE"), with the KV
 * append of the kv_append kernel folded in: one launch computes
 *   y[b, n] = sum_k x[b, k] * w_qkv[n, k]     (bf16 operands, fp32 accumulation, rounded to bf16)
 * for n over the (Hq + 2 Hkv) * d output features (rows of w_qkv ordered q heads, k heads, v heads,
 * d rows per head; the [N, K] layout of the paper's decode GEMV), rotates the q and k features at
 * position context_lens[b] exactly as ac_rope_kv_append does, writes q to q_out [B,Hq,d] and k, v
 * into the cache slot block_table[b, p / page_size], p % page_size.  x is [B, H] bf16, H % 64 == 0.
 * The projection is not bit-reproducible against an fp64 evaluation (fp32 accumulation order): its
 * bf16 results can differ from the correctly rounded ones by one unit in the last place; the
 * rotation and the stores are exact given those results.  Errors and status bits as
 * ac_rope_kv_append.  Up to 16 batch rows run on a warp-level MMA kernel that streams w_qkv once
 * from HBM; larger batches run on a tcgen05 kernel (batch tiles of up to 128 rows as the M dimension
 * of the instruction, accumulators in tensor memory) that streams w_qkv once per 128 rows.  Both
 * give the same results up to fp32 accumulation order. */
int ac_qkv_rope_kv_append(const void* x, const void* w_qkv, int H, void* q_out,
                          void* k_cache, void* v_cache,
                          int64_t stride_page, int64_t stride_token, int64_t stride_head,
                          const int32_t* block_table, int max_pages_per_seq,
                          const int32_t* context_lens,
                          const float* rope_cos, const float* rope_sin, int max_position,
                          int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                          int32_t* status_flag, void* stream);

/* ac_qkv_rope_kv_append with the prelude variants of ac_rope_kv_append_ex (family (i) names the per-head
 * Q/K RMSNorm as an option of the fused prelude; the per-model adaptations mention partial rotary):
 * the projected, bf16-rounded q and k head vectors are normalised, rotated over their first
 * rotary_dim elements with the chosen pairing and stored, still in one launch.  The CTAs that share a
 * head (d/32 of the warp-MMA kernel, the one or two 32-pair tiles of the tcgen05 kernel) form a
 * thread-block cluster and exchange the sums of squares and the rotation partners through distributed
 * shared memory.  options == NULL (or all defaults) is ac_qkv_rope_kv_append.  The rope tables are
 * [max_position, rotary_dim/2].  Everything else as ac_qkv_rope_kv_append. */
int ac_qkv_rope_kv_append_ex(const void* x, const void* w_qkv, int H, void* q_out,
                             void* k_cache, void* v_cache,
                             int64_t stride_page, int64_t stride_token, int64_t stride_head,
                             const int32_t* block_table, int max_pages_per_seq,
                             const int32_t* context_lens,
                             const float* rope_cos, const float* rope_sin, int max_position,
                             int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                             int32_t* status_flag, void* stream, const ac_rope_options* options);

/* Output-projection fusion, the paper's kernel family (v) ("an output-projection (o_proj) kernel
 * fusing GEMV + residual + post-RMSNorm"), consuming the attention output:
 *   h[b, n]      = bf16( residual_in[b, n] + sum_k attn_out[b, k] * w_o[n, k] )   (fp32 sum, one rounding)
 *   normed[b, :] = RMSNorm(h[b, :]) * norm_weight = bf16( bf16( h / sqrt(mean(h^2) + eps) ) * w )
 * attn_out [B,K] bf16 (K = Hq*d, K % 64 == 0), w_o [N,K] bf16 ([N,K] layout, N % 32 == 0),
 * residual_in/residual_out/normed_out [B,N] bf16 (residual_out may alias residual_in), norm_weight
 * [N] bf16.  Two dependent launches on `stream`: the weight-streaming product with the residual add
 * in its epilogue, then the row norm (it needs all N features of a row); the second starts under the
 * first one's tail.  The norm is exact given h (fp64 sum of squares, correctly rounded sqrt and
 * division); h can differ from the correctly rounded value by one bf16 step (fp32 accumulation).
 * As for ac_qkv_rope_kv_append, B > 16 runs the product on the tcgen05 kernel. */
int ac_oproj_residual_rmsnorm(const void* attn_out, const void* w_o, int K, int N,
                              const void* residual_in, void* residual_out,
                              const void* norm_weight, float norm_eps, void* normed_out,
                              int B, void* stream);

/* A4: paged decode attention, family (iv).  Row b attends over tokens 0 .. n_b - 1 with
 * n_b = context_lens[b] + new_tokens (new_tokens = 1 right after ac_rope_kv_append, 0 to attend
 * over the cached tokens only); token t lives in page block_table[b, t / page_size], slot
 * t % page_size.  For query head hq:  out = softmax(scale * q_rot[b,hq,:] . K[t,:]) V  over those
 * tokens (bf16 operands, fp32 accumulation, fp32 softmax); softmax_scale <= 0 means 1/sqrt(d).
 *
 * Grid: one CTA per (request, KV head, split) holding the whole group of Hq/Hkv query heads.
 * num_splits == 1: the final bf16 result is written to out [B,Hq,d]; workspace may be NULL.
 * num_splits  > 1: out is not touched; split s writes its own normalised result to
 *   partial_o  = (float*)workspace                      [B,Hq,num_splits,d]
 *   partial_lse = partial_o + B*Hq*num_splits*d          [B,Hq,num_splits]  natural-log
 * log-sum-exp of the scaled scores; a split with no tokens writes lse = -inf and leaves its
 * partial_o untouched.  workspace_bytes must be >= ac_workspace_bytes(B,Hq,d,num_splits).
 * max_context_len sizes the splits (split_tokens = ac_split_tokens(max_context_len, num_splits)): it should be
 * >= every n_b.  Where a row is longer all the same, its last split takes the rest: the result is that
 * of the whole row, the call only takes longer.
 * Contents of cache slots at or past n_b, of unreferenced pages and of unused block-table entries
 * never influence the result.  A page id outside [0, num_pages) reads as zeros. */
int ac_paged_decode_attn(const void* q_rot, const void* k_cache, const void* v_cache,
                         int64_t stride_page, int64_t stride_token, int64_t stride_head,
                         const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* context_lens, int new_tokens, float softmax_scale,
                         int num_splits, void* workspace, size_t workspace_bytes, void* out,
                         int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                         int max_context_len, int32_t* status_flag, void* stream);

/* A4 + A5 in one launch: the same attention kernel, but the CTA that finishes last for a (request,
 * KV head) merges that pair's split partials itself and writes the final bf16 rows to out [B,Hq,d]
 * (the "fused cross-CTA merging" of family (iv); Supplementary Implementation Notes: "a fused
 * fence-based merge that removes a separate reduction kernel").  Each CTA publishes its partial,
 * fences, and takes a ticket from a per-(request, KV head) arrival counter; the holder of the last
 * ticket merges and resets the counter.  No CTA ever waits for another.  When a pair's splits number
 * at most 16 and the whole grid is resident at once, the launch instead makes each pair's splits one
 * thread-block cluster: every CTA stages its partial in its own shared memory and the CTA of split 0
 * reads them from there (distributed shared memory, two hardware cluster barriers; no partials in
 * global memory, no ticket); the workspace contract is the same either way.
 *
 * Arguments as ac_paged_decode_attn, except: out is always written; for num_splits > 1 the workspace
 * must hold ac_fused_workspace_bytes(B,Hq,Hkv,d,num_splits) bytes = the partials followed by int32
 * arrival counters [B,Hkv], and the counters must be ZERO on entry.  A launch that completes leaves
 * them zero, so call ac_fused_workspace_reset once after allocating the workspace (and again after
 * any launch that did not complete).  Results differ from the separate merge only in rounding order
 * of the fp32 combination; for fixed inputs and num_splits they are deterministic. */
size_t ac_fused_workspace_bytes(int B, int Hq, int Hkv, int d, int num_splits);
int ac_fused_workspace_reset(void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int d,
                             int num_splits, void* stream);
int ac_paged_decode_attn_fused_merge(const void* q_rot, const void* k_cache, const void* v_cache,
                                     int64_t stride_page, int64_t stride_token, int64_t stride_head,
                                     const int32_t* block_table, int max_pages_per_seq,
                                     const int32_t* context_lens, int new_tokens, float softmax_scale,
                                     int num_splits, void* workspace, size_t workspace_bytes, void* out,
                                     int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                                     int max_context_len, int32_t* status_flag, void* stream);

/* A1 + A2 + A4 + A5 in ONE launch (the step as the paper's families (iii)/(iv) and its kv_append
 * kernel define it, fused): every CTA rotates the query rows of its group in registers (same exact
 * arithmetic as ac_rope_kv_append); the warp whose tile holds the new token's slot rotates k_new,
 * writes k and v into the cache page AND into the tile it just loaded, then attention proceeds over
 * context_lens[b] + 1 tokens and the last CTA of each (request, KV head) merges the splits.  Cache
 * contents after the call are bit-identical to ac_rope_kv_append's; outputs equal those of the
 * three-call sequence up to the fp32 merge order.
 *
 * q_in is the un-rotated query [B,Hq,d]; q_rot_out (optional, may be NULL) receives the rotated
 * rows and must not alias q_in.  Workspace as for ac_paged_decode_attn_fused_merge (counters zero on
 * entry when num_splits > 1).  A row whose position is outside the rope table or the block-table row,
 * whose page id is outside the pool, or whose context_lens[b] + 1 exceeds what the launch's split
 * grid covers (max_context_len too small for it: the new token's slot then lies in no CTA's range)
 * sets the status bits, appends nothing and writes no q_rot_out; its output is then unspecified. */
int ac_decode_step_fused(const void* q_in, void* q_rot_out, const void* k_new, const void* v_new,
                         void* k_cache, void* v_cache,
                         int64_t stride_page, int64_t stride_token, int64_t stride_head,
                         const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* context_lens,
                         const float* rope_cos, const float* rope_sin, int max_position,
                         float softmax_scale, int num_splits, void* workspace, size_t workspace_bytes,
                         void* out, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                         int max_context_len, int32_t* status_flag, void* stream);

/* Options of the _ex entry points.  Zero-initialise; unknown fields must stay zero. */
typedef struct ac_attn_options {
    int window;      /* > 0: sliding-window attention -- row b attends over its last `window` tokens
                        only, i.e. tokens max(0, n_b - window) .. n_b - 1 (the paper wires a sliding
                        window in for one of its model families, "Per-Model Adaptations"); 0: all */
    int fused_merge; /* ac_paged_decode_attn_ex only: non-zero = behave as ac_paged_decode_attn_fused_merge */
    const int32_t* row_order; /* optional device array [B], a permutation of 0..B-1: grid row y serves
                        request row_order[y].  CTAs are dispatched in grid order, so listing the requests
                        by decreasing context length (what a scheduler that knows the lengths can do
                        for free) shortens the tail of grids that are several waves deep.  Any
                        permutation gives the same results.  NULL: the kernel ranks the requests
                        itself when B <= 128 and serves them in index order otherwise. */
    const struct ac_rope_options* rope; /* ac_decode_step_fused_ex only: prelude variants (per-head Q/K
                        RMSNorm, partial rotary, interleaved pairing) applied to q_in and k_new inside the
                        step, with the arithmetic and the table shapes of ac_rope_kv_append_ex; NULL or
                        all-default options = the plain rotation */
    int sinks;       /* >= 0: with a window, the row's first `sinks` tokens stay visible beside it, i.e. the row
                        attends over tokens t < sinks and max(0, n_b - window) .. n_b - 1; no effect
                        without a window (every token is visible then) */
    int reserved[1];
} ac_attn_options;

/* ac_paged_decode_attn / ac_paged_decode_attn_fused_merge / ac_decode_step_fused with options
 * (options == NULL means defaults).  With a window, tokens before the window's start are neither
 * read (whole tiles) nor weighted (the first tile masks them), so their pages may already have been
 * recycled; the splits partition the at most window + 63 tokens from the window's start rounded
 * down to a multiple of 64, so pass min(max_context_len, window + 63) to ac_decode_plan.
 * With sinks > 0 the tokens between the sinks and the window are skipped in the same way (whole tiles
 * of 16 are not read, the tiles at the two borders mask theirs); the splits then partition the at most
 * window + sinks + 30 tokens of the two pieces laid end to end, so pass
 * min(max_context_len, ac_window_span(window, sinks)) to ac_decode_plan.  The softmax scale, the positions
 * of the rotary embedding and the append are those of the row without a window. */
int ac_paged_decode_attn_ex(const void* q_rot, const void* k_cache, const void* v_cache,
                            int64_t stride_page, int64_t stride_token, int64_t stride_head,
                            const int32_t* block_table, int max_pages_per_seq,
                            const int32_t* context_lens, int new_tokens, float softmax_scale,
                            int num_splits, void* workspace, size_t workspace_bytes, void* out,
                            int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                            int max_context_len, int32_t* status_flag, void* stream,
                            const ac_attn_options* options);
int ac_decode_step_fused_ex(const void* q_in, void* q_rot_out, const void* k_new, const void* v_new,
                            void* k_cache, void* v_cache,
                            int64_t stride_page, int64_t stride_token, int64_t stride_head,
                            const int32_t* block_table, int max_pages_per_seq,
                            const int32_t* context_lens,
                            const float* rope_cos, const float* rope_sin, int max_position,
                            float softmax_scale, int num_splits, void* workspace, size_t workspace_bytes,
                            void* out, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                            int max_context_len, int32_t* status_flag, void* stream,
                            const ac_attn_options* options);

/* A5: merge of the split partials ("cross-CTA merging" of family (iv), here as its own kernel):
 *   M = max_s lse_s,  w_s = exp(lse_s - M),  out[b,hq,:] = sum_s w_s partial_o[b,hq,s,:] / sum_s w_s
 * rounded to bf16.  Splits with lse = -inf are skipped (their partial_o is not read); a row whose
 * splits are all empty, or with context_lens[b] < 0 (context_lens may be NULL), gets +0.
 * workspace has the layout written by ac_paged_decode_attn for the same B, Hq, d, num_splits. */
int ac_splitkv_merge(const void* workspace, int num_splits, const int32_t* context_lens, void* out,
                     int B, int Hq, int d, void* stream);

/* The whole step from HOST buffers (for callers that hold the step's inputs on the host, and for
 * end-to-end timing): copies q/k_new/v_new/block_table/context_lens from the *_host buffers (pinned
 * memory recommended) into the caller's device buffers of the same name, resets the arrival
 * counters, enqueues ac_decode_step_fused for the given num_splits (workspace_bytes >=
 * ac_fused_workspace_bytes), and delivers the bf16 result in out AND out_host (when out_host is pinned
 * memory the GPU can address, the kernel's final stores go to both; otherwise a copy from out follows).  When the host
 * buffers are pinned memory the GPU can address and their sizes are multiples of 16 bytes, the five
 * inputs are gathered (and the counters cleared) by ONE small kernel reading host memory directly
 * instead of five copy-engine transfers; otherwise each buffer gets its own cudaMemcpyAsync.  The
 * *_host inputs must be complete when the call is made and stay unchanged until the step has
 * finished: that kernel reads them as soon as it is resident, which may be while earlier work of the
 * stream is still running (it writes the device buffers only after that work has completed).
 * Everything is asynchronous on `stream`; the caller
 * synchronises the stream before reading out_host.  The KV cache pools and rope tables stay on the
 * device (they are the layer's resident state, not a per-step input).  No paper counterpart. */
int ac_decode_step_host(const void* q_host, const void* k_new_host, const void* v_new_host,
                        const int32_t* block_table_host, const int32_t* context_lens_host,
                        void* out_host,
                        void* q, void* k_new, void* v_new, int32_t* block_table,
                        int32_t* context_lens, void* out,
                        void* k_cache, void* v_cache,
                        int64_t stride_page, int64_t stride_token, int64_t stride_head,
                        int max_pages_per_seq,
                        const float* rope_cos, const float* rope_sin, int max_position,
                        float softmax_scale, int num_splits, void* workspace, size_t workspace_bytes,
                        int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                        int max_context_len, int32_t* status_flag, void* stream);

/* Calibration helper (no paper counterpart): enqueues a plain coalesced read-only pass over
 * buffer[0, bytes) -- 16-byte streaming loads, nothing written -- on `stream`.  Timed by the caller
 * (CUDA events around it) it gives the read-only HBM ceiling of the machine, which a benchmark can
 * print beside the copy-measured peak its roofline fractions use.  buffer: device memory, 16-byte
 * aligned, bytes >= 16 (a tail shorter than 16 bytes is not read); sink: optional device word that
 * receives the fold of a thread's loads only if that happens to equal one constant (it keeps the
 * loads alive; expect it untouched).  ac_init must have succeeded on the current device. */
int ac_hbm_read_probe(const void* buffer, size_t bytes, void* sink, void* stream);

/* Size of the library's built-in partial-result array (bytes), held by every GPU that loads the
 * library until the process exits. */
#define AC_STATIC_SCRATCH_BYTES (8u << 20)

/* Split-KV attention and merge in one call, for callers that cannot allocate device memory.  (The
 * paper has no counterpart to this entry point; it exists for the integration cases below.)
 *
 * ac_paged_decode_attn needs a workspace for the split partials, which normally means a cudaMalloc
 * (or a framework allocation) somewhere in the caller.  That is not always possible: an engine that
 * gave all remaining HBM to its KV-cache pool at start-up has nothing left to ask for; code running
 * under a host framework that forbids allocation in the serving loop, or that must not take the
 * driver's allocation lock, cannot call cudaMalloc at all; and a stateless step function has nowhere
 * to keep a buffer from one call to the next.  This entry point calls no cudaMalloc, cudaFree or
 * any allocating routine: the partials go into a fixed array inside the library image, of
 * AC_STATIC_SCRATCH_BYTES bytes per GPU.
 *
 * Arguments are those of ac_paged_decode_attn without workspace/workspace_bytes; the caller still
 * passes every input and the output.  The call runs the attention kernel with num_splits splits
 * (use ac_decode_plan to choose) and then the merge, both on `stream`, and always writes the final
 * bf16 rows to out [B,Hq,d].
 *
 * Limits and rules
 *   - For num_splits > 1, B * Hq * num_splits * (d + 1) * 4 bytes must not exceed
 *     AC_STATIC_SCRATCH_BYTES, otherwise AC_ERR_SCRATCH_LIMIT is returned and nothing is launched.
 *     Lower num_splits, or use ac_paged_decode_attn with your own workspace.  A single split uses
 *     no scratch (the attention kernel writes `out` itself), so no size limit applies to it.
 *   - ac_init must have succeeded on the current device.  The first call on each device also looks
 *     up the array's device address (once; later calls reuse it): make that first call outside any
 *     stream capture.
 *   - All calls on a device share the one array, and it keeps whatever the previous call wrote.
 *     Nothing needs clearing between calls (each call overwrites the log-sum-exp slot of every split
 *     it uses before reading it, and never reads the partial of a split marked empty), but two calls
 *     whose kernels overlap on the GPU -- different streams, or different host threads without
 *     ordering between their streams -- would write the same bytes and corrupt each other.  Order
 *     them on one stream or with events.
 *   - Errors are otherwise those of ac_paged_decode_attn and ac_splitkv_merge. */
int ac_paged_decode_attn_static_scratch(const void* q_rot, const void* k_cache, const void* v_cache,
                                        int64_t stride_page, int64_t stride_token, int64_t stride_head,
                                        const int32_t* block_table, int max_pages_per_seq,
                                        const int32_t* context_lens, int new_tokens,
                                        float softmax_scale, int num_splits, void* out, int B, int Hq,
                                        int Hkv, int d, int page_size, int num_pages,
                                        int max_context_len, int32_t* status_flag, void* stream);

/* ---- the cache held in 4 bits --------------------------------------------------------------------
 *
 * A quarter of the bf16 cache's bytes per token, plus parameters.  A group of `group` consecutive
 * elements (x_0, x_1, ...) of one token and KV head is held as
 *   minimum m = min x_i,  scale s = bf16(fp32((max x_i - m) / 15))  (both bf16; the quotient in fp64),
 *   codes   c_i = clamp(rint((x_i - m) / s), 0, 15)                 (fp64, ties to even; 0 when s = 0),
 * and stands for c_i * s + m.  x is bf16: the rotated, bf16-rounded key, or the value vector.  A group
 * that contains an infinity or a NaN is held as m = NaN, s = 0, c = 0 and reads back as NaN.
 *
 * Codes are two to a byte, element 2i in the low nibble of byte i.  They sit in two pools with caller's
 * strides, like the bf16 cache; the parameters of K and V sit together in one dense pool, in which the
 * slots of one page and head are contiguous whatever the codes' layout. */
typedef struct ac_q4_cache {
    void* k_codes;           /* byte j of (page, slot, head) at page*stride_page + slot*stride_token + head*stride_head + j, */
    void* v_codes;           /* j < d/2; 16-byte aligned bases, strides in BYTES, multiples of 16, token and head >= d/2 */
    void* params;            /* bf16 [num_pages, Hkv, page_size, 2 (K, V), d/group, 2 (s, m)], 16-byte aligned */
    int64_t stride_page, stride_token, stride_head;
    int group;               /* 32, 64 or 128, at most d */
    int reserved[3];
} ac_q4_cache;

/* ac_rope_kv_append_ex into a 4-bit cache: q is rotated into q_out bit for bit as there; k is normalised
 * and rotated as there, rounded to bf16 and then quantised, v is quantised as it is.  Rows that are
 * inactive or out of range behave as there.  Supported shapes, errors and status bits as there; the
 * cache's group must be one of 32, 64, 128 and at most d (AC_ERR_UNSUPPORTED). */
int ac_rope_kv_append_q4(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                         const ac_q4_cache* cache, const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* context_lens, const float* rope_cos, const float* rope_sin,
                         int max_position, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                         int32_t* status_flag, void* stream, const ac_rope_options* options);

/* Quantises many tokens of each row at once (a prompt whose keys are already rotated).  k, v are dense
 * bf16 [total_tokens, Hkv, d]; row b owns the tokens row_offsets[b] .. row_offsets[b+1] - 1 and its i-th
 * one is written to position start_pos[b] + i, i.e. page block_table[b, position / page_size].  row_offsets
 * is device int32 [B + 1], non-decreasing; tokens before row_offsets[0] or at and past row_offsets[B] are ignored, rows with
 * start_pos[b] < 0 are inactive and write nothing.  total_tokens may be 0.  A token whose position or page
 * is out of range writes nothing and sets the status bits of ac_rope_kv_append.  Two tokens of one call in
 * the same slot are a caller error. */
int ac_kv_store_q4(const void* k, const void* v, const ac_q4_cache* cache, const int32_t* block_table,
                   int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                   int total_tokens, int B, int Hkv, int d, int page_size, int num_pages,
                   int32_t* status_flag, void* stream);

/* The reverse: reads the same tokens back as bf16(c * s + m), rounded once, into dense k, v [total_tokens, Hkv, d].
 * Tokens of inactive rows, of no row, or out of range (status bits set) read as +0. */
int ac_kv_load_q4(void* k, void* v, const ac_q4_cache* cache, const int32_t* block_table,
                  int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                  int total_tokens, int B, int Hkv, int d, int page_size, int num_pages,
                  int32_t* status_flag, void* stream);

/* Split plan for ac_paged_decode_attn_q4: arguments and outputs as ac_decode_plan_for_lengths, except that
 * token_counts_host may be NULL (every row then counts max_context_len tokens) and the workspace is the
 * one of the fused merge (ac_fused_workspace_bytes).  Host only, pure; any plan is valid, results of different
 * split counts differ in their low bits. */
int ac_decode_plan_q4(const int32_t* token_counts_host, int B, int Hq, int Hkv, int d, int page_size,
                      int max_context_len, int sm_count, int* num_splits_out, int* split_tokens_out,
                      size_t* workspace_bytes_out);

/* Paged decode attention over the 4-bit cache, merge included: ac_paged_decode_attn_ex with fused_merge
 * set (splits, workspace, inactive rows, window, sinks, row_order and max_context_len as there; options->rope must
 * be NULL; no status bit is set).  K and V enter as the exact values c * s + m; q is bf16, products and sums are
 * fp32, and the softmax weights times a V group's scale are rounded to fp16 (2^-11 relative, or 2^-31 of the
 * largest V scale seen, which counts as 2^-114 at least, whichever is more) for the second product.  Slots at or past n_b, unreferenced pages and
 * unused block-table entries never influence the result; a page id outside [0, num_pages) reads as zeros.
 * Outside the supported range: queries of magnitude 2^116 and more; rows whose tokens times the largest magnitude of V
 * reach 2^118 (the running sums are fp32, and a weight may be up to 2^8 before the final division); and
 * (AC_ERR_UNSUPPORTED) code pools in which 16 tokens of a page start 2^36 bytes or more behind the base, whatever the
 * order of the strides.  The workspace belongs to one call at a time: calls that may overlap need one each. */
int ac_paged_decode_attn_q4(const void* q_rot, const ac_q4_cache* cache, const int32_t* block_table,
                            int max_pages_per_seq, const int32_t* context_lens, int new_tokens,
                            float softmax_scale, int num_splits, void* workspace, size_t workspace_bytes,
                            void* out, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                            int max_context_len, int32_t* status_flag, void* stream,
                            const ac_attn_options* options);

/* ---- the cache held in 8 bits --------------------------------------------------------------------
 *
 * Half of the bf16 cache's bytes per token.  A block of `block` consecutive slots of a page has, for each KV head and for
 * each of K and V, one scale s, a power of two; an element is held as a code c of the format and stands for c * s.
 *   AC_Q8_INT8  c an integer, -127 .. 127 (two's complement; M = 127)
 *   AC_Q8_E4M3  c an 8-bit floating-point number: sign, 4 bits of exponent (bias 7), 3 of fraction, no infinities,
 *               0x7F and 0xFF are NaN (M = 448)
 * The scale is the least s = 2^e with max |x| <= M s over the tokens of the block, -100 <= e <= 121 (INT8) or 119 (E4M3),
 * and c = x / s rounded to the nearest code (ties to even), at most M in magnitude.  x is bf16: the rotated, bf16-rounded key,
 * or the value vector.  A block that holds an infinity or a NaN has s = NaN and reads back as NaN.
 *
 * Writing goes on in a block that is partly filled: a write at a slot that does not begin a block keeps the block's scale
 * where it suffices for the new tokens too; otherwise the scale grows to what they need and the codes of the slots in front
 * become c * (old s / new s), rounded as above.  A scale at least doubles when it grows, so a code that was rounded more than once
 * is off by less than one of its final steps (INT8).  A write at the first slot of a block begins it anew, whatever it held.  What
 * appending one by one and storing at once leave may differ by that.  No other block is touched: a page that rows share is
 * written by none of them (ac_cache_fork copies the partly filled page).  Two rows of a call that write into one block are a
 * caller error.  Attention and load take any finite positive scale. */
#define AC_Q8_INT8 0
#define AC_Q8_E4M3 1
typedef struct ac_q8_cache {
    void* k_codes;           /* byte j of (page, slot, head) at page*stride_page + slot*stride_token + head*stride_head + j, */
    void* v_codes;           /* j < d; 16-byte aligned bases, strides in BYTES, multiples of 16 below 2^40, token and head >= d */
    float* scales;           /* s of (page, head, block, side) at page*stride_scales + (head*(page_size/block) + block)*2 + side,
                                side 0 for K and 1 for V; 16-byte aligned */
    int64_t stride_page, stride_token, stride_head;
    int64_t stride_scales;   /* in floats; even, at least Hkv * (page_size/block) * 2 (a multiple of 4 for ac_page_pool) */
    int block;               /* tokens: a multiple of 16 that divides page_size */
    int format;              /* AC_Q8_INT8 or AC_Q8_E4M3 */
    int reserved[2];
} ac_q8_cache;

/* ac_rope_kv_append_ex into an 8-bit cache: q is rotated into q_out bit for bit as there; k is normalised and rotated as
 * there, rounded to bf16 and then quantised, v is quantised as it is.  Rows that are inactive or out of range behave as there.
 * Supported shapes, errors and status bits as there; an unknown format or a block that is no multiple of 16 is
 * AC_ERR_UNSUPPORTED, one that does not divide the page AC_ERR_SHAPE. */
int ac_rope_kv_append_q8(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                         const ac_q8_cache* cache, const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* context_lens, const float* rope_cos, const float* rope_sin,
                         int max_position, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                         int32_t* status_flag, void* stream, const ac_rope_options* options);

/* ac_kv_store_q4 and ac_kv_load_q4 for the 8-bit cache: arguments, rows, errors and status bits as there.  The tokens that one
 * call writes into a block are one write; where they go on in a partly filled block, what the row holds in front of them
 * must be there. Load gives bf16(c * s), which is exact but where c * s is subnormal. */
int ac_kv_store_q8(const void* k, const void* v, const ac_q8_cache* cache, const int32_t* block_table,
                   int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                   int total_tokens, int B, int Hkv, int d, int page_size, int num_pages,
                   int32_t* status_flag, void* stream);
int ac_kv_load_q8(void* k, void* v, const ac_q8_cache* cache, const int32_t* block_table,
                  int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                  int total_tokens, int B, int Hkv, int d, int page_size, int num_pages,
                  int32_t* status_flag, void* stream);

/* Split plan for ac_paged_decode_attn_q8: arguments and outputs as ac_decode_plan_q4. */
int ac_decode_plan_q8(const int32_t* token_counts_host, int B, int Hq, int Hkv, int d, int page_size,
                      int max_context_len, int sm_count, int* num_splits_out, int* split_tokens_out,
                      size_t* workspace_bytes_out);

/* Paged decode attention over the 8-bit cache, merge included: ac_paged_decode_attn_ex with fused_merge set (splits, workspace,
 * inactive rows, window, sinks, row_order and max_context_len as there; options->rope must be NULL).  K and V enter as the
 * exact values c * s; q is bf16, products and sums are fp32, and the softmax weights times V's scale are rounded to fp16
 * (2^-11 relative, or 2^-31 of the largest V scale seen, which counts as 2^-120 at least, whichever is more) for the second product.  Slots at or past n_b, the
 * scales of blocks in which the row attends over no token, unreferenced pages and unused block-table entries never influence
 * the result; a page id outside [0, num_pages) reads as zeros.  Outside the supported range: as ac_paged_decode_attn_q4
 * says of q and V.  AC_FLAG_WAIT_TIMEOUT is the only status bit.  The workspace belongs to one call at a time: calls that may
 * overlap need one each. */
int ac_paged_decode_attn_q8(const void* q_rot, const ac_q8_cache* cache, const int32_t* block_table,
                            int max_pages_per_seq, const int32_t* context_lens, int new_tokens,
                            float softmax_scale, int num_splits, void* workspace, size_t workspace_bytes,
                            void* out, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                            int max_context_len, int32_t* status_flag, void* stream,
                            const ac_attn_options* options);

/* ---- rotary positions ---------------------------------------------------------------------------- */

/* Frequencies f_i = base^(-2i/R), i < R/2, R = rotary_dim, and what is done to them for contexts longer than the one that they
 * were made for. */
#define AC_ROPE_NONE 0       /* as they are */
#define AC_ROPE_LINEAR 1     /* f_i / factor: positions are squeezed */
#define AC_ROPE_BASE 2       /* base * factor^(R/(R-2)) for base: the lowest frequency is slowed down by factor, the highest stays */
#define AC_ROPE_RAMP 3       /* g f_i + (1 - g) f_i / factor, g = clamp((original * f_i / (2 pi) - low) / (high - low), 0, 1):
                                frequencies that turn more than `high` times in the original context stay, those that turn less
                                than `low` times are slowed down, in between they are blended */
typedef struct ac_rope_scaling {
    int kind;                /* AC_ROPE_... */
    int reserved;
    double base;             /* > 0; no number of the struct, nor the larger base, above 1e300 in magnitude */
    double factor;           /* > 0 (not used for AC_ROPE_NONE) */
    double original;         /* AC_ROPE_RAMP: positions of the original context, > 0 */
    double low, high;        /* AC_ROPE_RAMP: low < high */
    double magnitude;        /* cosines and sines are multiplied by it; 0 means 1 */
} ac_rope_scaling;

/* Tables for ac_rope_kv_append and its relatives and for ac_rope_rows: rope_cos[j, i] = magnitude * cos((first_position + j) f_i),
 * rope_sin likewise, j < positions, fp32 [positions, rotary_dim/2] dense, evaluated in fp64 and rounded: each entry is within
 * magnitude * 2^-45 of the one of an angle that is off by at most (|ln b| + 2 |ln factor| + 12) 2^-53 of itself (2^-48 for bases
 * below 10^8 that stay; b is the larger base for AC_ROPE_BASE), and then rounded once.  AC_ROPE_RAMP with low >= 0: max(factor,
 * 1/factor) * high / (high - low) times that where frequencies are blended.  rotary_dim is even; for AC_ROPE_BASE it is at least 4.
 * positions may be 0. */
int ac_rope_tables(float* rope_cos, float* rope_sin, int64_t first_position, int positions, int rotary_dim,
                   const ac_rope_scaling* scaling, void* stream);

/* A1 for many tokens of each row (prompts): token i of row b, i.e. token row_offsets[b] + i of the packed tensors, is rotated at
 * position start_pos[b] + i exactly as ac_rope_kv_append_ex rotates the new token's q and k (options as there: rotary_dim,
 * interleaved, norm weights).  q_in [total_tokens, Hq, d] and k_in [total_tokens, Hkv, d] are bf16 with dense heads and
 * tokens stride_*_token elements apart (multiples of 8, at least Hq*d or Hkv*d), so that they may be parts of a joint projection's
 * output; q_out and k_out likewise, each either its input with the same stride or apart from both inputs.  Hkv may be 0 (then k_in
 * and k_out are ignored).  row_offsets, start_pos and their rows as ac_kv_store_q4: tokens of inactive rows and of no row are not
 * touched; a token at or past max_position is not written and sets AC_FLAG_POSITION_OOB (AC_FLAG_WAIT_TIMEOUT: a copy of the call did
 * not arrive).  Any Hq and Hkv whose sum is at most
 * 65535; d is 64 or 128. */
int ac_rope_rows(const void* q_in, void* q_out, int64_t stride_q_in_token, int64_t stride_q_out_token,
                 const void* k_in, void* k_out, int64_t stride_k_in_token, int64_t stride_k_out_token,
                 const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hq, int Hkv, int d,
                 const float* rope_cos, const float* rope_sin, int max_position, int32_t* status_flag, void* stream,
                 const ac_rope_options* options);

/* ---- pages ----------------------------------------------------------------------------------------
 *
 * Bookkeeping of a page pool on the device, so that sequences can be grown, forked and dropped between
 * steps without a copy to the host.  State, all int32 in device memory: block_table [rows,
 * max_pages_per_seq], context_lens [rows] (tokens held; < 0: the row is unused) and ref_counts [num_pages]
 * (rows that hold the page; 0: free).  A row holds its first ceil(context_lens / page_size) pages.  What ac_cache_reserve
 * takes for it beyond those is counted in ref_counts but belongs to the row only once context_lens has grown to
 * count it: the other calls do not know of it (ac_cache_release does not return it, ac_cache_compact does not follow
 * it in the table).  ac_cache_trim returns whatever was reserved and not used.
 *
 * Free pages are handed out lowest index first, in the order of the call's list, so every call's
 * result is determined by its inputs.  The pools themselves are opaque bytes: any number of them (K and V
 * of every layer, codes, parameters) can share one block table. */
#define AC_PAGE_WHOLE (-1)
typedef struct ac_page_pool {
    void* base;              /* page p occupies bytes [p*page_bytes, (p+1)*page_bytes); 16-byte aligned */
    int64_t page_bytes;      /* a multiple of 16 * segments */
    int segments;            /* a page is this many equal pieces, each holding the page's slots in order: 1 for
                                [page, slot, head, d], Hkv for [page, head, slot, ...]; or AC_PAGE_WHOLE where its bytes do not
                                follow its slots (the scales of an 8-bit cache): ac_cache_fork then copies all of a partly filled
                                page, and page_bytes is any multiple of 16 */
    int reserved;
} ac_page_pool;

/* Most pools of one call. */
#define AC_MAX_PAGE_POOLS 128

/* Copies whole pages, pairs[i] = (source, destination), device int32 [n, 2], in every pool.  A pair with a
 * page outside [0, num_pages) is skipped and sets AC_FLAG_PAGE_OOB; source == destination is a no-op.  A
 * destination that is listed twice or is also a source is a caller error.  n may be 0. */
int ac_cache_copy_pages(const ac_page_pool* pools, int n_pools, const int32_t* pairs, int n, int num_pages,
                        int32_t* status_flag, void* stream);

/* Bytes of workspace that reserve, fork (n = forks of the call) and compact need; n = 0 but for fork.  It holds
 * nothing from one call to the next; calls that may overlap need one each.  Host only, pure. */
size_t ac_cache_workspace_bytes(int rows, int num_pages, int n);

/* Gives every active row room for new_tokens more tokens: pages ceil(n/page_size) .. ceil((n + new_tokens) /
 * page_size) - 1 of the row are taken from the free pages (reference count 1), rows in order.  Pages are
 * taken again at each call: reserve, then let context_lens grow by new_tokens before reserving anew, or,
 * where rows grow by less (prompts of different lengths, tokens that were not accepted), call ac_cache_trim first.
 * When the free pages run out, the row that does not get all of its pages and every later row that needs
 * any get none, and AC_FLAG_POOL_EXHAUSTED is set; a row whose pages would exceed max_pages_per_seq gets
 * none and sets AC_FLAG_POSITION_OOB. */
int ac_cache_reserve(int32_t* block_table, int max_pages_per_seq, const int32_t* context_lens,
                     int32_t* ref_counts, int new_tokens, int rows, int page_size, int num_pages,
                     void* workspace, size_t workspace_bytes, int32_t* status_flag, void* stream);

/* Forks: pairs[i] = (parent row, child row), device int32 [n, 2].  The child holds the parent's full pages
 * too (reference counts go up) and, where the parent's last page is partly filled, a page of its own
 * with a copy of the filled slots in every pool; context_lens[child] = context_lens[parent].  What else the
 * page and the child's table row held stays as it was.  The child row must be unused before (its
 * old pages are not released); a child listed twice, or that is also a parent, is a caller error (which rows
 * hold which pages is then undefined; lengths are those before the call, and nothing outside the tables is written);
 * one parent may have many children.  A fork whose page the pool cannot supply makes its child unused and sets
 * AC_FLAG_POOL_EXHAUSTED; an unused parent gives an unused child.  n_pools may be 0 (bookkeeping only). */
int ac_cache_fork(const ac_page_pool* pools, int n_pools, int32_t* block_table, int max_pages_per_seq,
                  int32_t* context_lens, int32_t* ref_counts, const int32_t* pairs, int n, int rows,
                  int page_size, int num_pages, void* workspace, size_t workspace_bytes,
                  int32_t* status_flag, void* stream);

/* Drops the rows listed in row_list (device int32 [n]): the reference counts of their pages go down and
 * context_lens[row] becomes -1; the table entries stay, and pages reserved for the rows stay taken (see
 * ac_cache_trim).  A row that is unused, or listed again, is a no-op.  A count that is already 0 stays 0 and sets
 * AC_FLAG_REF_COUNT. */
int ac_cache_release(const int32_t* block_table, int max_pages_per_seq, int32_t* context_lens,
                     int32_t* ref_counts, const int32_t* row_list, int n, int rows, int page_size,
                     int num_pages, int32_t* status_flag, void* stream);

/* Returns what was reserved and not used: every count becomes the number of active rows that hold the page by their
 * lengths, so pages reserved for tokens that did not come, or for rows released since, are free again.  Counts are
 * rebuilt from the table alone: a page that the caller has counted up by itself is free too unless a row holds it.
 * A row longer than its table row counts as far as that goes and sets AC_FLAG_POSITION_OOB, a page outside the pool
 * is skipped and sets AC_FLAG_PAGE_OOB.  Two launches. */
int ac_cache_trim(const int32_t* block_table, int max_pages_per_seq, const int32_t* context_lens,
                  int32_t* ref_counts, int rows, int page_size, int num_pages, int32_t* status_flag, void* stream);

/* Moves the live pages (reference count > 0) to the lowest ids: with L of them, the live pages at ids >= L
 * move, in order, to the free ids < L, in every pool, and the block table entries of the active rows and the
 * reference counts follow; *live_out (optional) = L.  Only free pages are written, so a step in flight
 * that still reads the old table reads the same bytes until those pages are handed out again.  The new
 * table and counts go to block_table_out and ref_counts_out, which may be the inputs themselves or other
 * buffers of the same shape (both or neither aliased); context_lens does not change.  Table entries past a
 * row's pages and rows that are not active are copied as they are: call it with nothing reserved (after
 * ac_cache_trim). */
int ac_cache_compact(const ac_page_pool* pools, int n_pools, const int32_t* block_table,
                     int32_t* block_table_out, int max_pages_per_seq, const int32_t* context_lens,
                     const int32_t* ref_counts, int32_t* ref_counts_out, int rows, int page_size,
                     int num_pages, int32_t* live_out, void* workspace, size_t workspace_bytes,
                     int32_t* status_flag, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AC_H_ */
