/*
 * spf.h -- C ABI of the speculative-prefill scoring / selection library for NVIDIA B200 (sm_100a).
 *
 * The library covers the data-parallel part of "Cross-Family Speculative Prefill" that runs between
 * the draft model's forward pass and the assembly of the compressed prompt text:
 *
 *   spf_score          Appendix A.1.1 / Algorithm 1 "AggregateMaxMean": attention of the lookahead
 *                      queries over the prompt keys, max over (layer, head), mean over lookahead.
 *   spf_chunk_pool     Appendix A.1.2 / Algorithm 1 "AvgPool1D" + "PartitionIntoChunks": smoothing
 *                      and per-chunk mean.
 *   spf_select_topk    Appendix A.1.2 / Algorithm 1 "TopKChunks".
 *   spf_compact_spans  Section 3.2 / Algorithm 1 "MergeAdjacentChunks" + "MapDraftChunksToTextSpans".
 *
 * Before them, on the draft model's side: spf_kv_append (rotates a step's queries and keys and writes a paged cache) and
 * spf_attend (the step's attention over it); spf_kv_weigh and spf_kv_evict (received attention weights, and cuts of the cache to a
 * budget by them).  Around them: spf_keep_count / spf_keep_rate / spf_snap_budget (Section 3.1, keep rate) and spf_concat_with_delim
 * (Algorithm 1 "ConcatWithDelim") on the host; spf_score_paged (paged key cache), spf_score_fp8 (8-bit key cache), spf_score_paged_fp8 (both),
 * spf_score_shard_lse /
 * spf_score_shard_apply (one prompt's keys over several GPUs); spf_score_extra, spf_chunk_pool_edge,
 * spf_select_topk_forced (switches for points the paper leaves open); spf_compress_host (the four calls for host
 * buffers); spf_score_static (no allocation).
 *
 * Symbols: N prompt tokens (the paper's S), m lookahead queries (the paper's N), L layers, Hq query
 * heads (the paper's H), Hkv key heads, G = Hq / Hkv, d head dimension, c chunk size, C = ceil(N / c),
 * k chunks kept, w pooling kernel.
 *
 * General conventions
 *   - Every pointer is DEVICE memory owned by the caller unless its comment says HOST.  The library
 *     never frees or keeps caller memory and allocates nothing per call.
 *   - `cuda_stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).  All work is
 *     enqueued on it; no call synchronises the stream or the device.
 *   - Return value: SPF_OK (0) or a negative spf_status.  Argument checks happen on the host before
 *     anything is launched; a call that fails them launches nothing.  spf_last_error() gives the text of
 *     the calling thread's last failure.
 *   - Conditions only the device can see are written to `dev_status` (see spf_score).
 *   - Nothing here falls back to the CPU: unsupported shapes return SPF_ERR_UNSUPPORTED.
 */
#ifndef SPF_H_
#define SPF_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(_WIN32)
#define SPF_API
#else
#define SPF_API __attribute__((visibility("default")))
#endif

typedef enum {
  SPF_OK = 0,
  SPF_ERR_INVALID_ARG = -1, /* null pointer, non-positive size, misaligned K rows, k > C, ...      */
  SPF_ERR_UNSUPPORTED = -2, /* shape outside what the kernels cover (see spf_score)                 */
  SPF_ERR_WORKSPACE = -3,   /* workspace missing, misaligned or smaller than the size query says    */
  SPF_ERR_CUDA = -4,        /* a CUDA runtime call failed (no device, launch error)                 */
  SPF_ERR_TIMEOUT = -5,     /* device status only: a bounded wait inside a kernel ran out           */
  SPF_ERR_RANGE = -6,       /* device status only: a softmax row sum overflowed fp32 in the fused path */
  SPF_ERR_CACHE = -7        /* device status only: a length, position or block-table entry outside the cache */
} spf_status;

/* Draft-model attention geometry shared by all prompts of a call. */
typedef struct {
  int32_t n_layers;     /* L >= 1                                                                  */
  int32_t n_q_heads;    /* Hq, multiple of n_kv_heads                                              */
  int32_t n_kv_heads;   /* Hkv                                                                     */
  int32_t head_dim;     /* d: 64 or 128                                                            */
  int32_t n_lookahead;  /* m: 1..32, with G * roundup(m, 8) <= 64                                   */
  float softmax_scale;  /* multiplies q.k before the softmax; <= 0 selects 1/sqrt(d)                */
} spf_shape;

/* One prompt.  An array of these expresses a ragged batch; prompts are independent. */
typedef struct {
  int64_t n_tokens;            /* N >= 1                                                            */
  const void* const* k_layers; /* HOST array of L device pointers; layer l is bf16 [Hkv][N][d],
                                  post-RoPE, element (h, s, j) at h*k_stride_head + s*k_stride_tok + j */
  int64_t k_stride_head;       /* in elements                                                       */
  int64_t k_stride_tok;        /* in elements, >= d, multiple of 8 (rows start 16-byte aligned)     */
  const void* q;               /* bf16 [L][Hq][m][d], contiguous, post-RoPE lookahead queries       */
  float* importance;           /* out: fp32 [N], the token importance I                             */
  float* lse;                  /* out, may be NULL: fp32 [L][Hq][m], natural-log sum-exp of each
                                  softmax row, so that p = exp(scale * q.k - lse)                   */
} spf_prompt;

/*
 * Bytes of scratch with which spf_score scores these prompts at full speed (0 on invalid arguments; the reason is left in
 * spf_last_error()): up to 16 consecutive prompts share a launch of the fused path, each with scratch of its own (queries as
 * the tensor cores read them, row sums and log-sum-exps, running maxima).  spf_score also takes less, down to the bytes
 * that this call gives for each prompt alone: then fewer prompts share a launch, and one buffer serves them in turn.
 */
SPF_API size_t spf_score_workspace_bytes(const spf_shape* shape, const spf_prompt* prompts, int32_t n_prompts);

/*
 * Token importance (Appendix A.1.1; Algorithm 1, AggregateMaxMean).  For every prompt:
 *     z[l,h,i,s] = scale * sum_j Q[l,h,i,j] * K[l, h / G, s, j]         (GQA: head h reads key head h / G)
 *     p[l,h,i,s] = exp(z[l,h,i,s]) / sum_{s'} exp(z[l,h,i,s'])           softmax over the N prompt keys
 *     A[i,s]     = max over all (l,h) of p[l,h,i,s]                      max over layer and head first,
 *     I[s]       = (1/m) * sum_i A[i,s]                                  then the mean over lookahead
 * written to prompts[p].importance (and the row log-sum-exps to prompts[p].lse when not NULL).
 * bf16 inputs, fp32 accumulation and softmax.  The attention tensor itself is never stored.
 *
 * `shape`, `prompts` and the k_layers arrays are HOST memory, read during the call only.
 * `workspace`: device, 256-byte aligned, spf_score_workspace_bytes(...) bytes, or at least what that call
 * gives for the most demanding prompt alone; contents on entry are irrelevant, contents on exit
 * unspecified.  Calls that share a workspace must be ordered on one stream.
 * `dev_status`: device int32, may be NULL (device-side conditions then go unreported).  Kernels store a
 * negative spf_status there when a device-side condition occurs; they never trap.  The caller zeroes it
 * before the call and reads it after synchronising.  Conditions:
 *   SPF_ERR_TIMEOUT  a bounded wait of the fused path ran out (2 s): the kernel returned without results.
 *                    The fused kernel needs all its CTAs resident at once and asks the runtime for that at
 *                    launch; the wait can still run out if the GPU is shared so heavily that a hand-over
 *                    between CTAs takes seconds.
 *   SPF_ERR_RANGE    fused path only.  Its first sweep sums exp2(logit - r) per softmax row in fp32, with one
 *                    reference r per (layer, kv-head): 60 base-2 units above the smallest logit that the rows of
 *                    that kv-head have against the key at position N / 2.  No row can underflow (its largest
 *                    term is at least 2^-60, and what is flushed is 2^66 times smaller), whatever the spread
 *                    between the heads of a group.  A row sum overflows when some logit lies about 188 -
 *                    log2(number of such keys) base-2 units -- 157 at the very least, about 109 nats -- above that
 *                    smallest sample logit.  The importance is then invalid and the call should be repeated on
 *                    the general path (spf_set_score_path(1)), which has no such limit.
 * Errors: SPF_ERR_INVALID_ARG, SPF_ERR_UNSUPPORTED (d not 64/128, Hq % Hkv != 0, m > 32,
 * G * roundup(m,8) > 64, L > 128; with the fused path forced, also shapes outside it or a grid that cannot be
 * co-resident on the device), SPF_ERR_WORKSPACE, SPF_ERR_CUDA.  All prompts are validated before the first
 * launch; a shape that only the forced fused path refuses is found when its prompt's turn comes, after earlier
 * prompts of the batch have been enqueued.
 */
SPF_API int32_t spf_score(const spf_shape* shape, const spf_prompt* prompts, int32_t n_prompts, void* workspace,
                          size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * spf_score with a larger softmax denominator -- a switch for a point the paper leaves open (Section 3 describes the
 * attention of each lookahead step "over the prompt", Appendix A.1.1 slices it to the prompt length): in the draft
 * model, lookahead step i also attends to the i - 1 tokens generated before it and to itself, so its probabilities
 * over the prompt sum to less than 1.  `extra_lse` is a HOST array of n_prompts DEVICE pointers (an entry may be
 * NULL), each fp32 [L][Hq][m]: the natural log of sum exp(scale * q.k) over those non-prompt keys of row (l, h, i),
 * as the draft model's attention kernel reports it.  Then
 *     p[l,h,i,s] = exp(z[l,h,i,s]) / (sum_{s'} exp(z[l,h,i,s']) + exp(extra_lse[l,h,i]))
 * and everything downstream is unchanged; prompts[p].lse receives the log of the whole denominator.  With
 * extra_lse == NULL, or all entries NULL, this is spf_score.  Arguments, workspace and errors as for spf_score.
 */
SPF_API int32_t spf_score_extra(const spf_shape* shape, const spf_prompt* prompts, int32_t n_prompts,
                                const float* const* extra_lse, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                void* cuda_stream);

/*
 * spf_score on a PAGED key cache (Section 3.1: the paper's serving system keeps KV caches in 4k-token blocks; a draft
 * model served the same way has its prompt keys scattered over a block pool).  Same computation as spf_score.
 *
 *   k_pools        HOST array of L device pointers; layer l's pool is bf16 [n_pool_blocks][Hkv][block_tokens][d],
 *                  contiguous, 16-byte aligned, post-RoPE
 *   block_tokens   tokens per block, a positive multiple of 128
 *   block_table    DEVICE int32 [ceil(N / block_tokens)]: logical block b of the prompt is pool block block_table[b].
 *                  Entries must lie in [0, n_pool_blocks); the kernels cannot report a bad entry, but its keys then
 *                  read as zeros (or, for the one sampled reference key, from a clamped block) instead of faulting.
 *                  Rows of the last block beyond n_tokens are never used.
 *   q, importance, lse   as in spf_prompt
 *
 * Both kernel paths read paged caches (spf_set_score_path applies); shapes, errors and dev_status as for spf_score.
 * Workspace: spf_score_paged_workspace_bytes(...), rules as for spf_score.
 */
typedef struct {
  int64_t n_tokens;
  const void* const* k_pools;
  int64_t n_pool_blocks;
  int32_t block_tokens;
  const int32_t* block_table;
  const void* q;
  float* importance;
  float* lse;
} spf_paged_prompt;

SPF_API size_t spf_score_paged_workspace_bytes(const spf_shape* shape, const spf_paged_prompt* prompts, int32_t n_prompts);
SPF_API int32_t spf_score_paged(const spf_shape* shape, const spf_paged_prompt* prompts, int32_t n_prompts, void* workspace,
                                size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * spf_score on an 8-BIT key cache (Section 3.1: the paper's serving system keeps KV caches in block-quantised form; a
 * draft model served the same way holds its prompt keys in 8 bits).  The cache format is an input format: key
 * (l, hk, s, j) has the value
 *     k_scale[l * Hkv + hk] * E4M3(byte at k_layers[l] + hk * k_stride_head + s * k_stride_tok + j)
 * with E4M3 the 8-bit floating-point format of 1 sign, 4 exponent (bias 7) and 3 mantissa bits, subnormals, no
 * infinities (the byte patterns 0x7F / 0xFF, NaN, must not occur).  The key scale is folded into the softmax scale of
 * its (layer, kv-head).  Queries are given in bf16.
 *
 *   k_layers       HOST array of L device pointers (8-byte aligned), layer l uint8 [Hkv][N][d]; strides in bytes,
 *                  k_stride_tok >= d, both strides multiples of 8
 *   k_scale        DEVICE fp32 [L][Hkv], positive and finite
 *   others         as in spf_prompt
 *
 * Kernel paths, chosen as in spf_score (spf_set_score_path):
 *   fused     needs 16-byte aligned layer pointers and strides (and a shape spf_score's fused path takes).  The tensor
 *             cores multiply the E4M3 keys by E4M3 operands only, so each bf16 query is handed to them as the sum of two
 *             E4M3 terms after a power-of-two scaling per (layer, kv-head): exact for every element within 2^9 of the
 *             largest |q| of its (layer, kv-head), off by at most 2^-17 of that largest value below.  Accumulation is
 *             fp32.  Range limits and `dev_status` as for spf_score's fused path (SPF_ERR_RANGE, SPF_ERR_TIMEOUT).
 *   general   any cache the layout rules above admit.  Bytes are widened to bf16 exactly; arithmetic and error are
 *             those of spf_score's general path; `dev_status` is not written.
 * With the path left automatic, caches the fused path cannot read go to the general kernels; with the fused path
 * forced they are refused with SPF_ERR_UNSUPPORTED.  Workspace: spf_score_fp8_workspace_bytes(...), rules as for
 * spf_score.
 */
typedef struct {
  int64_t n_tokens;
  const void* const* k_layers;
  int64_t k_stride_head;
  int64_t k_stride_tok;
  const float* k_scale;
  const void* q;
  float* importance;
  float* lse;
} spf_fp8_prompt;

SPF_API size_t spf_score_fp8_workspace_bytes(const spf_shape* shape, const spf_fp8_prompt* prompts, int32_t n_prompts);
SPF_API int32_t spf_score_fp8(const spf_shape* shape, const spf_fp8_prompt* prompts, int32_t n_prompts, void* workspace,
                              size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * The draft model's paged cache of ONE layer, keys and values, as spf_kv_append writes and spf_attend reads it.  The key pool
 * is the pool that spf_score_paged (bf16) and spf_score_paged_fp8 (8 bits) score.
 *
 *   k_pool, v_pool     DEVICE, contiguous [n_pool_blocks][Hkv][block_tokens][d], 16-byte aligned; keys after the rotation.
 *                      16 bits: bf16.  8 bits: E4M3 bytes (see spf_score_fp8).  4 bits: codes 0 ... 15, two to a byte ([...][d / 2] bytes),
 *                      element 2 j in the low half of byte j, 2 j + 1 in the high one
 *   k_scale, v_scale   16 bits: both NULL.
 *                      8 bits: DEVICE fp32 [n_pool_blocks][Hkv][block_tokens / SPF_KV_SCALE_TOKENS]: what the bytes of that many
 *                      consecutive tokens of a block and head are multiplied by, positive and finite.
 *                      4 bits: DEVICE bf16 [n_pool_blocks][Hkv][block_tokens][d / SPF_KV_SCALE_DIMS], 16-byte aligned: an element is worth
 *                      scale * (code - 8), the scale being that of its SPF_KV_SCALE_DIMS consecutive elements of the token; positive and
 *                      finite, with at most five significant bits (an element then is a bf16 number)
 *   block_tokens       a positive multiple of 128
 *   head_dim           d: 64 or 128
 *   bits               of an element: 16, 8 or 4; 0: 16 without scales, 8 with them.  (Since version 0.2.0, where the structure ended in four
 *                      unused bytes, and k_scale and v_scale were float*: programs that do not set the bytes to zero have to be adapted)
 * Limit: n_pool_blocks * Hkv * block_tokens < 2^31.
 */
#define SPF_KV_SCALE_TOKENS 64
#define SPF_KV_SCALE_DIMS 32
typedef struct {
  void* k_pool;
  void* v_pool;
  void* k_scale;
  void* v_scale;
  int64_t n_pool_blocks;
  int32_t block_tokens;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t bits;
} spf_kv_cache;

/*
 * A step of the draft model: some new tokens of each of n_seqs sequences (one, when it generates; a chunk of the prompt;
 * none).  The new tokens of sequence b are rows row_start[b] ... row_start[b + 1] - 1 of the step's arrays and the LAST
 * row_start[b + 1] - row_start[b] of the sequence's seq_lens[b] tokens.  All arrays are DEVICE memory, so that a captured
 * graph can be replayed with other lengths.
 *
 *   n_rows        rows of the step's arrays; rows behind row_start[n_seqs] are not read and left as they were
 *   max_new       HOST hint, >= 1: new tokens of the sequence that has most.  It picks the kernels; sequences with more are
 *                 computed all the same, only slower (2048 tokens after 30720 with a hint of 1: 3.7 ms instead of 0.6)
 *   row_start     int32 [n_seqs + 1], ascending from 0, the last one at most n_rows
 *   seq_lens      int32 [n_seqs], the new tokens included, at most table_stride * block_tokens
 *   block_table   int32 [n_seqs][table_stride]: logical block j of sequence b is pool block block_table[b][j]; entries behind
 *                 a sequence's length are not read
 */
typedef struct {
  int32_t n_seqs;
  int32_t n_rows;
  int32_t max_new;
  int32_t table_stride;
  const int32_t* row_start;
  const int32_t* seq_lens;
  const int32_t* block_table;
} spf_kv_step;

/*
 * Rotation by position.  `table` is DEVICE fp32 [n_positions][rot_dim], row p = the cosines of position p's rot_dim / 2
 * angles, then their sines (whatever base or scaling they were made with).  Pair j of a head, elements (j, j + rot_dim / 2),
 * or (2 j, 2 j + 1) where `interleaved`, becomes
 *     (x cos_j - y sin_j, y cos_j + x sin_j),
 * in fp32 with each product rounded; elements from rot_dim on stay.  rot_dim: a multiple of 16, at most d.  `positions`:
 * DEVICE int32 [n_rows], the table's row for every row of the step, or NULL for a token's place in its sequence.
 */
typedef struct {
  const float* table;
  const int32_t* positions;
  int32_t n_positions;
  int32_t rot_dim;
  int32_t interleaved;
} spf_rope;

/* Rows of a step, element (row, head, j) at row * stride_row + head * stride_head + j; strides in elements, multiples of 8,
 * data 16-byte aligned: a slice of a fused projection's output, or one lookahead token of the [L][Hq][m][d] queries that
 * spf_score reads. */
typedef struct {
  void* data;
  int64_t stride_row;
  int64_t stride_head;
} spf_rows;

/*
 * Appends a step's keys and values to the cache, rotating keys (and queries) on the way.
 *   k, v          bf16, n_kv_heads heads a row
 *   q, q_out      bf16, n_q_heads heads a row: the rotated queries go to q_out, which may be q itself (same strides) and must
 *                 overlap neither it otherwise nor k or v; both NULL: the step's queries are handled elsewhere
 *   rope          NULL: nothing is rotated (q, where given, is copied)
 * bf16 pools: rotated values are rounded to bf16 once.  8-bit pools, for each group of SPF_KV_SCALE_TOKENS tokens and head that
 * receives tokens: scale = the smallest power of two that keeps the new tokens' finite values within 448 times it (at least
 * 2^-100), and no smaller than the scale that tokens of the group from before the step have; where it grows, their bytes are
 * rounded again to the new scale (exact unless they become subnormal).  New values are rounded once, from fp32; infinities
 * become +-448 times the scale, NaN stays NaN (0x7F).
 * 4-bit pools, for each SPF_KV_SCALE_DIMS elements x of a new token and head: scale = the smallest number of five significant bits that
 * keeps the finite ones within 7 times it (at least 2^-100), code = 8 + x * (1 / scale) rounded to the nearest whole number, ties to
 * even, -7 ... 7; fp32 throughout.  Infinities become +-7 times the scale, NaN makes the scale NaN.
 * A block that receives tokens belongs to one sequence of the step only (two that write the same block race).
 * Device conditions: SPF_ERR_CACHE in dev_status (may be NULL) for a row whose position, table row or block lies outside; that
 * row is left out, the others are not affected.
 * Errors: SPF_ERR_INVALID_ARG, SPF_ERR_UNSUPPORTED (head_dim, the limit above), SPF_ERR_CUDA.
 */
SPF_API int32_t spf_kv_append(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rope* rope, const spf_rows* k,
                              const spf_rows* v, const spf_rows* q, const spf_rows* q_out, int32_t n_q_heads,
                              int32_t* dev_status, void* cuda_stream);

/*
 * Attention of a step's tokens over the cache (the new tokens' own keys and values are in it already: spf_kv_append comes
 * first).  Row t, place p in its sequence of n tokens, head h:
 *     out[t,h] = sum_s w_s V[h / G, s],   w = softmax over s of softmax_scale * q[t,h] . K[h / G, s],
 *     s from first_key to p (to n - 1 where see_all)
 * A row without keys gets zeros, and -inf as its lse.  bf16 queries and outputs, fp32 softmax and sums.
 *   q, out        bf16, n_q_heads heads a row (a multiple of the cache's heads); out must not overlap q
 *   softmax_scale <= 0 selects 1/sqrt(d)
 *   options       NULL: causal, from key 0 on, without lse
 *     lse         fp32, element (row, head) at row * lse_stride_row + head * lse_stride_head: the natural log of the sum of
 *                 exp over the keys that the row sees; may be NULL.  With first_keys = the prompt's length it is what
 *                 spf_score_extra takes.
 *     first_keys  DEVICE int32 [n_seqs], may be NULL: the first key that rows of a sequence see (negative: 0)
 *     see_all     nonzero: rows see all n keys, also those behind them (lookahead queries over a prompt)
 *   workspace     DEVICE, 256-byte aligned, spf_attend_workspace_bytes() of a step whose max_new is at least this one's;
 *                 contents irrelevant on entry, unspecified on exit.  Calls that share one must be ordered on one stream.
 * What the pools hold behind a sequence's tokens, or before its first key, does not matter.
 * Roundings: weights of the sum over values are bf16 over bf16 pools (16 bits with up to 8 rows a key head and sequence), fp16 over
 * 8-bit ones; the sum of the weights is fp32, of weights that are not rounded.  4-bit pools, up to 32 rows (16 with 128 dimensions): weights are
 * rounded to bf16, and once more with the values' scales in them, off by up to 2^-8 together; of 128 keys that not every row sees, once, with the
 * scales in them (2^-9).  From 33 (17) rows on: as over bf16 pools.
 * 4-bit pools: elements are exact.  Elements of a query should lie below 2^114 in magnitude, value scales within 2^-40 ... 2^50.
 * 8-bit pools: values of bytes times scales are exact; their scales should lie within 2^-100 ... 2^100.  Elements of a query row are exact
 * within 2^13 of its largest and off by at most 2^-21 of that below.  Weights below 2^-21 of the row's largest (each times its value
 * scale) are off by up to 2^-32 of it.
 * Device conditions (dev_status, may be NULL): SPF_ERR_CACHE: a length beyond the block table, more new tokens than the
 * sequence is long, or a block outside the pool, whose keys and values then read as zeros; SPF_ERR_TIMEOUT as for spf_score.
 * Errors: SPF_ERR_INVALID_ARG, SPF_ERR_UNSUPPORTED (head_dim, heads, the cache's limit), SPF_ERR_WORKSPACE, SPF_ERR_CUDA.
 */
typedef struct {
  float* lse;
  int64_t lse_stride_row;
  int64_t lse_stride_head;
  const int32_t* first_keys;
  int32_t see_all;
} spf_attend_options;

SPF_API size_t spf_attend_workspace_bytes(const spf_kv_cache* cache, int32_t n_q_heads, int32_t max_new);
SPF_API int32_t spf_attend(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rows* q, const spf_rows* out,
                           int32_t n_q_heads, float softmax_scale, const spf_attend_options* options, void* workspace,
                           size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * What a cut of the cache goes by, beside one layer's cache of any format, 16-byte aligned: for each token of a block and head
 *   weight        DEVICE fp32 [n_pool_blocks][Hkv][block_tokens]: the attention weight that the token has received (spf_kv_weigh)
 *   position      DEVICE int32, the same: the token's position in its sequence, whatever was cut before it; NULL: nothing was ever cut, a
 *                 token's position is its place
 * Nothing has to be set beforehand where spf_kv_weigh is called for every step: it writes both for the step's tokens.  Only it does: where it is
 * left out for some steps (chunks of a prompt before the window that a cut is decided by), their tokens' weights and positions are the caller's
 * to set; with a decay of 0 their weights need not be, either.
 */
typedef struct {
  float* weight;
  int32_t* position;
} spf_kv_ledger;

/*
 * Adds to the ledger the attention weights of a step's rows (spf_kv_append and spf_attend of the step come first).  For each key s and
 * key head h of every sequence that has new tokens:
 *     weight[h, s] = decay * weight[h, s] + sum over rows t that see s, heads g of the group of exp(softmax_scale * q[t,g] . K[h, s] - lse[t,g]),
 * where a new token's weight from before is 0.  Rows see keys as in spf_attend.
 *   q             as for spf_attend
 *   attend        as the step's spf_attend had it; lse is required, and read
 *   ledger        position may be NULL; else the new tokens' positions are written to it
 *   options       NULL: decay 1, all rows, a token's place as its position
 *     decay       finite, not negative; 0: what the ledger holds is replaced, whatever it is
 *     last_rows   only the last so many new tokens of a sequence count as rows (0: all of them)
 *     positions   DEVICE int32 [n_rows], the positions of the step's tokens; NULL: a token's place in its sequence
 * A block belongs to one sequence of the step (two that share one race).
 * Sums are fp32, taken in an order that does not change from run to run; over many rows they carry what their additions lose.  (But for a
 * sequence that has more rows than max_new announces, and no more than it announces for all sequences together: up to 2^-25 of a sum is lost for
 * each 8 of them.)  Besides, weights are off by some 1e-7: the roundings of logits, of log-sum-exps and of ex2.
 * A row whose lse is -inf (it saw no key) adds nothing, whatever the keys are; one with NaN makes NaN of the weights of the keys that it sees.
 * Device conditions: SPF_ERR_CACHE in dev_status (may be NULL) as for spf_attend; keys in a block outside the pool are left out.
 * SPF_ERR_TIMEOUT as for spf_score.
 * Errors: SPF_ERR_INVALID_ARG, SPF_ERR_UNSUPPORTED (as for spf_attend), SPF_ERR_CUDA.
 */
typedef struct {
  float decay;
  int32_t last_rows;
  const int32_t* positions;
} spf_kv_weigh_options;

SPF_API int32_t spf_kv_weigh(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rows* q, int32_t n_q_heads,
                             float softmax_scale, const spf_attend_options* attend, const spf_kv_ledger* ledger,
                             const spf_kv_weigh_options* options, int32_t* dev_status, void* cuda_stream);

/*
 * Cuts sequences to a budget: copies what is kept of them, keys, values, their scales and the ledger, to other blocks of the same pools.
 * For each sequence b of seq_lens[b] = n tokens and each key head, min(n, keep[b]) tokens are kept (n if keep[b] is more, none if it is
 * negative) and put one after the other, in the order of their places, into the blocks of to_table.  Kept are those with a position below
 * n_first, or of n_seen[b] - n_recent and above, then those of the largest weight; of equals, and of the former where they are too many, those
 * of the lowest places.  NaN ranks below every number.  Heads keep different tokens; a sequence's length, the same for all of them, goes to to_lens.
 * The blocks that the call reads are left as they were, and may be given up, or kept (a prefix that other sequences share).
 * A place then holds other tokens in each head and layer: such a cache is attended over, but not scored (spf_score_paged and
 * spf_score_paged_fp8 go by places, and do not notice).
 * The time goes by the room that the tables have too, not by the lengths alone, which the host does not see: 32 sequences of 1900 to 2500
 * tokens (4 bits, 8 heads of 128 dimensions) take 55 us where block_table has no more room than they need, 69 with room for 8192 of each, 103 for 32768,
 * 226 for 131072.
 *
 *   n_seqs        1 ... 2^20
 *   seq_lens      DEVICE int32 [n_seqs], at most table_stride * block_tokens
 *   block_table   DEVICE int32 [n_seqs][table_stride], as in spf_kv_step
 *   keep          DEVICE int32 [n_seqs]; at most to_stride * block_tokens of a sequence's tokens are kept
 *   to_table      DEVICE int32 [n_seqs][to_stride]: the blocks that receive the tokens, none of which is one that the call reads, each in one
 *                 place only (blocks that are read and written race)
 *   to_lens       DEVICE int32 [n_seqs], out; may be seq_lens
 *   n_first, n_recent   0 or more
 *   n_seen        DEVICE int32 [n_seqs], how many tokens the sequences have had, or NULL: seq_lens
 *   workspace     DEVICE, 256-byte aligned, spf_kv_evict_workspace_bytes(); contents irrelevant on entry, unspecified on exit.  Calls
 *                 that share one must be ordered on one stream.
 * Places behind a sequence's new length are left as they were.  8-bit pools: a group of SPF_KV_SCALE_TOKENS tokens gets the largest scale of
 * those that its tokens come from, and their bytes are rounded to it (exact between powers of two unless they become subnormal).
 * Device conditions: SPF_ERR_CACHE in dev_status (may be NULL): a length below zero or beyond the table (it is taken to be 0), or a block outside the
 * pool: tokens that should be read from one count as tokens of weight 0 and position 0 and are left out of the copy, as are those that should
 * be written to one.
 * Errors: SPF_ERR_INVALID_ARG, SPF_ERR_UNSUPPORTED (head_dim, the cache's limit, more than 2^20 sequences times heads, tables of more than
 * 2^30 tokens a sequence), SPF_ERR_WORKSPACE, SPF_ERR_CUDA.
 */
typedef struct {
  int32_t n_seqs;
  int32_t table_stride;
  int32_t to_stride;
  int32_t n_first;
  int32_t n_recent;
  const int32_t* seq_lens;
  const int32_t* block_table;
  const int32_t* keep;
  const int32_t* to_table;
  int32_t* to_lens;
  const int32_t* n_seen;
} spf_kv_cut;

SPF_API size_t spf_kv_evict_workspace_bytes(const spf_kv_cache* cache, int32_t n_seqs, int32_t to_stride);
SPF_API int32_t spf_kv_evict(const spf_kv_cache* cache, const spf_kv_ledger* ledger, const spf_kv_cut* cut, void* workspace,
                             size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * spf_score on a PAGED 8-bit key cache, as spf_kv_append writes it: blocks as for spf_score_paged, key s of a prompt, in block
 * block_table[s / block_tokens], worth
 *     k_scales[l][block][hk][(s % block_tokens) / SPF_KV_SCALE_TOKENS] * E4M3(byte).
 *
 *   k_pools    HOST array of L device pointers, layer l uint8 [n_pool_blocks][Hkv][block_tokens][d], contiguous, 16-byte aligned
 *   k_scales   HOST array of L device pointers, layer l fp32 [n_pool_blocks][Hkv][block_tokens / SPF_KV_SCALE_TOKENS], positive
 *              and finite where the prompt has tokens
 *   others     as in spf_paged_prompt
 * Kernel paths, workspace, errors and dev_status as for spf_score_fp8.
 */
typedef struct {
  int64_t n_tokens;
  const void* const* k_pools;
  const float* const* k_scales;
  int64_t n_pool_blocks;
  int32_t block_tokens;
  const int32_t* block_table;
  const void* q;
  float* importance;
  float* lse;
} spf_paged_fp8_prompt;

SPF_API size_t spf_score_paged_fp8_workspace_bytes(const spf_shape* shape, const spf_paged_fp8_prompt* prompts, int32_t n_prompts);
SPF_API int32_t spf_score_paged_fp8(const spf_shape* shape, const spf_paged_fp8_prompt* prompts, int32_t n_prompts, void* workspace,
                                    size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * One long prompt over several GPUs (Appendix A.1.1 is per prompt; this shards its keys).  Each rank holds a contiguous
 * range of the prompt's keys for all layers and describes it as an spf_prompt of its own (n_tokens = the range's
 * length).  A softmax row spans all ranks, so scoring takes two calls with one exchange between them:
 *
 *   spf_score_shard_lse     writes to prompt->lse (required) the natural-log sum-exp of every row over THIS rank's keys;
 *                           prompt->importance is ignored.
 *   (caller)                combines the ranks' values: lse_all = log sum_r exp(lse_r) -- e.g. a max all-reduce and a
 *                           sum all-reduce of exp(lse_r - max), L * Hq * m floats.
 *   spf_score_shard_apply   given lse_all (device fp32 [L][Hq][m]) writes the importance of this rank's keys, exactly
 *                           what spf_score would give them in the whole prompt; prompt->lse is ignored.
 *
 * Pooling needs a halo of pool_kernel / 2 importance values from each neighbour, the top-k needs all ranks' chunk
 * scores; both are the caller's exchanges.  These two calls use the general two-sweep kernels (one sweep each);
 * workspace as spf_score_workspace_bytes for the shard, errors as spf_score.
 */
SPF_API int32_t spf_score_shard_lse(const spf_shape* shape, const spf_prompt* prompt, void* workspace, size_t workspace_bytes,
                                    void* cuda_stream);
SPF_API int32_t spf_score_shard_apply(const spf_shape* shape, const spf_prompt* prompt, const float* lse, void* workspace,
                                      size_t workspace_bytes, void* cuda_stream);

/*
 * The same two calls on the kernels spf_score would pick (spf_set_score_path applies): where the shard's shape allows it,
 * the fused kernel runs with one of its two visits only -- spf_score_shard_lse_ex streams the shard's keys once and
 * leaves the row log-sum-exps, spf_score_shard_apply_ex streams them once and leaves the importance -- so a rank reads
 * its keys at the fused kernel's rate instead of the general kernels'.  `dev_status` as for spf_score: a row sum of the
 * first call can overflow fp32 (SPF_ERR_RANGE: repeat that call with spf_score_shard_lse), a bounded wait can run out
 * (SPF_ERR_TIMEOUT).  Workspace: spf_score_workspace_bytes for the shard.
 */
SPF_API int32_t spf_score_shard_lse_ex(const spf_shape* shape, const spf_prompt* prompt, void* workspace, size_t workspace_bytes,
                                       int32_t* dev_status, void* cuda_stream);
SPF_API int32_t spf_score_shard_apply_ex(const spf_shape* shape, const spf_prompt* prompt, const float* lse, void* workspace,
                                         size_t workspace_bytes, int32_t* dev_status, void* cuda_stream);

/*
 * Chooses the kernels behind spf_score, process-wide: 0 = automatic (the fused single-kernel path when
 * the shape allows it, else the general two-sweep path), 1 = always the general path, 2 = always the
 * fused path (spf_score then returns SPF_ERR_UNSUPPORTED for shapes outside it: G > 8, G rounded up to a
 * power of two times m > 64, more than 64 layers, or a prompt whose running maxima do not fit tensor memory).  Both compute the same function
 * (Appendix A.1.1).  Meant for tests and measurements.  Returns the previous setting; an invalid value
 * changes nothing.
 */
SPF_API int32_t spf_set_score_path(int32_t path);

/*
 * Diagnostic (no counterpart in the paper): checks that a device-side wait of the fused kernel gives up
 * instead of hanging.  Enqueues a one-CTA kernel that waits, with the kernels' own bounded wait and a
 * 20 ms limit, on a barrier nothing ever signals.  After synchronising, *dev_status (device int32, zeroed
 * by the caller) must read SPF_ERR_TIMEOUT and the context must still be usable.
 */
SPF_API int32_t spf_selftest_bounded_wait(int32_t* dev_status, void* cuda_stream);

/*
 * spf_score without a caller-provided workspace (the paper has no counterpart; this exists for
 * deployment reasons only).
 *
 * Some callers cannot hand over scratch memory because they cannot allocate any at the point where
 * they score a prompt: a serving engine that has already given all free HBM to its KV-cache pool, a
 * plugin that runs inside someone else's process under a no-allocation rule, or code on a path where
 * the implicit device-wide synchronisation of cudaMalloc / cudaFree is not acceptable.  For them the
 * library keeps SPF_STATIC_SCRATCH_BYTES of scratch in a static device array of its own (part of the
 * loaded module: every GPU that loads the library holds it until the process exits) and this call
 * uses it in place of `workspace`.  It computes exactly what spf_score computes with the general
 * two-sweep kernels and calls no allocating routine.
 *
 *   - Arguments and results are those of spf_score; inputs and outputs are still the caller's.
 *   - Prompts whose scratch need (spf_score_workspace_bytes gives an upper bound) exceeds
 *     SPF_STATIC_SCRATCH_BYTES are rejected with SPF_ERR_WORKSPACE before anything is launched.
 *   - The first call on each device looks up the array's device address (with that device current)
 *     and caches it.  CUDA loads a library's device code lazily, so that first lookup is also the
 *     moment the array itself (8 MiB) comes to exist on the device: make the first call at start-up,
 *     BEFORE the application hands the remaining HBM to its own pools (afterwards the lookup can fail
 *     with SPF_ERR_CUDA for lack of memory), outside any stream capture, with the device that owns
 *     `cuda_stream` current.  Any small prompt will do for that call.
 *   - Every call on a device shares the one array, and the array keeps whatever the previous call
 *     left in it.  The kernels write each scratch word before they read it, so nothing needs
 *     clearing between calls; but two calls whose kernels overlap on the GPU (different streams,
 *     no ordering) race on it and give wrong results.  Order them on one stream or with events.
 */
#define SPF_STATIC_SCRATCH_BYTES (8u << 20)
SPF_API int32_t spf_score_static(const spf_shape* shape, const spf_prompt* prompts, int32_t n_prompts,
                                 void* cuda_stream);

/*
 * Smoothing and chunk means (Appendix A.1.2; Algorithm 1, AvgPool1D and PartitionIntoChunks;
 * kernel size 13 and chunk size 32 / 128 in Appendix A.3):
 *     S[s]  = (1/w) * sum_{t = s - w/2}^{s + w/2} I[t]      terms outside [0, N) count as zero
 *     cs[j] = mean of S over tokens [j*c, min((j+1)*c, N))
 * importance: fp32 [N] in; chunk_scores: fp32 [ceil(N/c)] out.  pool_kernel w is odd, 1 <= w <= 255
 * (1 = no smoothing); chunk c >= 1.
 */
SPF_API int32_t spf_chunk_pool(const float* importance, int64_t n_tokens, int32_t pool_kernel, int32_t chunk,
                               float* chunk_scores, void* cuda_stream);

/*
 * Top-k chunks (Appendix A.1.2; Algorithm 1, TopKChunks): the indices of the k largest chunk scores,
 * equal scores resolved toward the lower index, written in ascending order.
 * chunk_scores: fp32 [n_chunks] in (finite); kept_chunks: int32 [k] out; 1 <= k <= n_chunks < 2^31.
 */
SPF_API int32_t spf_select_topk(const float* chunk_scores, int64_t n_chunks, int64_t k, int32_t* kept_chunks,
                                void* cuda_stream);

/*
 * Merge and compaction (Section 3.2; Algorithm 1, MergeAdjacentChunks and MapDraftChunksToTextSpans).
 * kept_chunks: int32 [k], ascending, distinct, each in [0, ceil(N/c)) -- as spf_select_topk writes them.
 * Runs of consecutive kept chunks become one token span [a, b) (b clipped to N); its character span
 * is [char_start[a], char_end[b-1]).  Kept tokens keep their original order.
 *   token_ids, char_start, char_end : int32 [N] in (character offsets of each draft token in the text)
 *   out_ids        int32 [>= min(k*c, N)]  kept token ids, n_kept of them
 *   out_pos        int32 [>= min(k*c, N)]  their original positions; may be NULL
 *   out_tok_spans  int32 [k][2]            n_spans rows (a, b)
 *   out_char_spans int32 [k][2]            n_spans rows (char_start[a], char_end[b-1])
 *   out_counts     int64 [2]               {n_kept, n_spans}
 * Rows beyond n_kept / n_spans are left untouched.
 */
SPF_API int32_t spf_compact_spans(const int32_t* kept_chunks, int64_t k, int32_t chunk, int64_t n_tokens,
                                  const int32_t* token_ids, const int32_t* char_start, const int32_t* char_end,
                                  int32_t* out_ids, int32_t* out_pos, int32_t* out_tok_spans,
                                  int32_t* out_char_spans, int64_t* out_counts, void* cuda_stream);

/*
 * spf_select_topk followed by spf_compact_spans in ONE launch (Algorithm 1, TopKChunks ... MapDraftChunksToTextSpans):
 * both steps are latency-bound, and chaining them saves a launch per prompt.  Arguments, layouts and
 * results are those of the two calls (kept_chunks receives the k indices as spf_select_topk writes them); n_chunks must
 * equal ceil(n_tokens / chunk).  Results are identical to the two separate calls.  Prompts of more than 32768 chunks take
 * the two calls' launches.
 */
SPF_API int32_t spf_select_compact(const float* chunk_scores, int64_t n_chunks, int64_t k, int32_t chunk, int64_t n_tokens,
                                   const int32_t* token_ids, const int32_t* char_start, const int32_t* char_end,
                                   int32_t* kept_chunks, int32_t* out_ids, int32_t* out_pos, int32_t* out_tok_spans,
                                   int32_t* out_char_spans, int64_t* out_counts, void* cuda_stream);

/*
 * Batched forms of the three selection calls (Algorithm 1 runs AvgPool1D ... MapDraftChunksToTextSpans per prompt; a
 * serving step has many prompts).  `items` is a HOST array of n_items descriptors, read during the call only; every
 * pointer inside a descriptor is DEVICE memory with the layout and size the single-prompt call states.  One launch
 * serves up to 32 prompts (more are split into several launches); results are identical to n_items single calls.
 * pool_kernel and chunk are shared by the batch.  Errors as the single-prompt calls, reported with the item index
 * before anything is launched.
 */
typedef struct {
  const float* importance; /* fp32 [n_tokens]                  */
  int64_t n_tokens;
  float* chunk_scores;     /* out: fp32 [ceil(n_tokens / chunk)] */
} spf_pool_item;

typedef struct {
  const float* chunk_scores; /* fp32 [n_chunks] */
  int64_t n_chunks;
  int64_t k;
  int32_t* kept_chunks;      /* out: int32 [k], ascending */
} spf_topk_item;

typedef struct {
  const int32_t* kept_chunks;
  int64_t k;
  int64_t n_tokens;
  const int32_t* token_ids;
  const int32_t* char_start;
  const int32_t* char_end;
  int32_t* out_ids;
  int32_t* out_pos;          /* may be NULL */
  int32_t* out_tok_spans;
  int32_t* out_char_spans;
  int64_t* out_counts;
} spf_compact_item;

SPF_API int32_t spf_chunk_pool_batch(const spf_pool_item* items, int32_t n_items, int32_t pool_kernel, int32_t chunk,
                                     void* cuda_stream);
SPF_API int32_t spf_select_topk_batch(const spf_topk_item* items, int32_t n_items, void* cuda_stream);
SPF_API int32_t spf_compact_spans_batch(const spf_compact_item* items, int32_t n_items, int32_t chunk, void* cuda_stream);

/*
 * spf_chunk_pool, spf_select_topk and spf_compact_spans (Algorithm 1, AvgPool1D ... MapDraftChunksToTextSpans) of one or more
 * prompts in ONE launch per 24 prompts; prompts of more than 32768 chunks take the three calls' launches.  `items` is a HOST
 * array, read during the call only; the pointers in it are DEVICE memory with the layouts that the three calls state.
 * edge_rule, force_first and force_last as in spf_chunk_pool_edge and spf_select_topk_forced.  Results are identical to the
 * separate calls.
 */
typedef struct {
  const float* importance; /* fp32 [n_tokens]                    */
  int64_t n_tokens;
  float* chunk_scores;     /* out: fp32 [ceil(n_tokens / chunk)] */
  int64_t k;
  const int32_t* token_ids;
  const int32_t* char_start;
  const int32_t* char_end;
  int32_t* kept_chunks;    /* out: int32 [k], ascending */
  int32_t* out_ids;
  int32_t* out_pos;        /* may be NULL */
  int32_t* out_tok_spans;
  int32_t* out_char_spans;
  int64_t* out_counts;
} spf_path_item;

SPF_API int32_t spf_pool_select_compact(const spf_path_item* items, int32_t n_items, int32_t pool_kernel, int32_t chunk,
                                        int32_t edge_rule, int32_t force_first, int32_t force_last, void* cuda_stream);

/*
 * Variants for two points the paper leaves open (Algorithm 1 names the operations, Appendix A.3 gives kernel 13 and
 * the chunk sizes, nothing else).  Same arguments, layouts and errors as the calls they extend.
 *
 * spf_chunk_pool_edge: edge_rule 0 is spf_chunk_pool (every window is divided by pool_kernel, tokens beyond the
 *   prompt's ends count as zeros); edge_rule 1 divides each window by the number of tokens it really covers, so
 *   the first and last pool_kernel/2 tokens are not damped.  Other values: SPF_ERR_INVALID_ARG.
 * spf_select_topk_forced: the first and / or the last chunk (system prompt / attention sink, and the question at
 *   the end of the prompt) are kept whatever their scores; they count towards k, the remaining k - forced are
 *   the best of the other chunks, ties to the lower index.  k smaller than the number of forced chunks:
 *   SPF_ERR_INVALID_ARG.  With both flags 0 it is spf_select_topk.
 */
SPF_API int32_t spf_chunk_pool_edge(const float* importance, int64_t n_tokens, int32_t pool_kernel, int32_t chunk,
                                    int32_t edge_rule, float* chunk_scores, void* cuda_stream);
SPF_API int32_t spf_select_topk_forced(const float* chunk_scores, int64_t n_chunks, int64_t k, int32_t force_first,
                                       int32_t force_last, int32_t* kept_chunks, void* cuda_stream);

/*
 * The whole path for ONE prompt whose inputs and results live in HOST memory (Algorithm 1 from AggregateMaxMean to
 * MapDraftChunksToTextSpans): copies the inputs to the device, runs spf_score -> spf_pool_select_compact, copies the
 * selection back.  This is the entry for a caller that holds the draft model's tensors on the host or on another
 * device; a caller whose tensors are already on this GPU chains the two calls itself.  Unlike every other call it SYNCHRONISES `cuda_stream` (twice: once to learn the counts, once at the end).
 *
 *   k_layers_host   HOST array of L HOST pointers, layer l bf16 [Hkv][N][d] contiguous (pinned memory copies at full
 *                   PCIe / NVLink-C2C speed, pageable memory works)
 *   q_host          HOST bf16 [L][Hq][m][d]
 *   token_ids_host, char_start_host, char_end_host   HOST int32 [N]
 *   params          chunk size c, pooling kernel w (odd), keep rate rho: k = spf_keep_count(ceil(N / c), rho)
 *   arena           DEVICE scratch owned by the caller, 256-byte aligned, at least spf_compress_host_arena_bytes(...)
 *                   bytes; holds the device copies of the inputs, every intermediate and the scoring workspace
 *   out_ids_host, out_pos_host (may be NULL)   HOST int32 [min(k * c, N)]
 *   out_tok_spans_host, out_char_spans_host     HOST int32 [k][2]
 *   out_counts_host                             HOST int64 [2]: {n_kept, n_spans}; only that many rows are written
 *
 * If the fused scoring kernel reports SPF_ERR_RANGE or SPF_ERR_TIMEOUT the prompt is scored again with the general
 * kernels before anything is written to the caller's buffers.  Errors: as those calls; SPF_ERR_WORKSPACE for a small or misaligned arena;
 * a device-side status that survives the retry is returned as the call's status.
 */
typedef struct {
  int32_t chunk;        /* c >= 1                       */
  int32_t pool_kernel;  /* w, odd, 1..255               */
  double keep_ratio;    /* rho in (0, 1]                */
} spf_select_params;

SPF_API size_t spf_compress_host_arena_bytes(const spf_shape* shape, int64_t n_tokens, const spf_select_params* params);
SPF_API int32_t spf_compress_host(const spf_shape* shape, int64_t n_tokens, const void* const* k_layers_host, const void* q_host,
                                  const int32_t* token_ids_host, const int32_t* char_start_host, const int32_t* char_end_host,
                                  const spf_select_params* params, void* arena, size_t arena_bytes, int32_t* out_ids_host,
                                  int32_t* out_pos_host, int32_t* out_tok_spans_host, int32_t* out_char_spans_host,
                                  int64_t* out_counts_host, void* cuda_stream);

/*
 * Host helper for the keep rate of Section 3.1: the number of chunks a keep rate rho retains,
 * clamp(ceil(rho * n_chunks), 1, n_chunks).  Pure host arithmetic; returns 0 if n_chunks < 1.
 */
SPF_API int64_t spf_keep_count(int64_t n_chunks, double keep_ratio);

/*
 * Host helpers for the keep rate of Section 3.1.  The keep rate is defined on the TARGET model's tokenisation:
 * rho = compressed target length / original target length, per sample.  The paper picks compressed lengths that
 * are whole KV-cache blocks of the serving system (8k, 16k, 24k, 32k tokens with 4k-token blocks).
 *
 * spf_keep_rate:        min(1, budget_tokens / target_tokens); 0 if target_tokens < 1 or budget_tokens < 1.
 * spf_snap_budget:      the largest multiple of block_tokens that is <= desired_tokens, at least one block;
 *                       0 if block_tokens < 1 or desired_tokens < 1.
 * Pure host arithmetic.
 */
SPF_API double spf_keep_rate(int64_t target_tokens, int64_t budget_tokens);
SPF_API int64_t spf_snap_budget(int64_t desired_tokens, int64_t block_tokens);

/*
 * ConcatWithDelim of Algorithm 1 (Section 3.2, Appendix A.3): builds the compressed prompt text from the character
 * spans that spf_compact_spans produced.  Host routine, host pointers throughout.
 *
 *   text, text_bytes     the prompt as UTF-8 (need not be NUL-terminated)
 *   char_spans           int32 [n_spans][2], half-open [start, end) in CHARACTERS (Unicode code points, as a
 *                        tokenizer's offset mapping counts them), ascending and non-overlapping
 *   delim, delim_bytes   UTF-8 delimiter (e.g. "[...]" or "// omitted"); written between consecutive spans only,
 *                        never before the first or after the last; may be empty
 *   out, out_capacity    receives the compressed text (not NUL-terminated); may be NULL with capacity 0 to query
 *
 * Returns the number of bytes of the compressed text.  Nothing is written unless out_capacity is at least that.
 * A negative return is a status code: SPF_ERR_INVALID_ARG for null / negative arguments, spans that are not
 * ascending, overlap or reach beyond the text's last character.  Bytes of the form 10xxxxxx are counted as
 * continuations of the preceding character; the text is not otherwise validated.
 */
SPF_API int64_t spf_concat_with_delim(const char* text, int64_t text_bytes, const int32_t* char_spans, int64_t n_spans,
                                      const char* delim, int64_t delim_bytes, char* out, int64_t out_capacity);

/* Text of a status code (static storage). */
SPF_API const char* spf_status_string(int32_t status);
/* Text of the calling thread's most recent failure ("" if none).  Thread-local storage. */
SPF_API const char* spf_last_error(void);
/* Library version, e.g. "0.2.0". */
SPF_API const char* spf_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SPF_H_ */
