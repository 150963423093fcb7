/*
 * sp.h -- C ABI of the MI355X (gfx950) token-importance library for
 * cross-family speculative prefill.
 *
 * The library computes, on one GPU, the draft-model token-importance pass of
 * the paper "Cross-Family Speculative Prefill": attention of the lookahead
 * queries over the prompt's keys in every draft layer, max/mean aggregation to
 * one score per prompt token, average pooling, chunk means, top-k chunk
 * selection, merging into spans, projection of those spans through character
 * offsets onto another tokenisation, and assembly of the compressed prompt's
 * token and position ids (Algorithm 1; Appendix A.1).
 *
 * Conventions shared by every call
 *  - Pointers named *_dev point to device memory of the current HIP device and
 *    are owned by the caller; pointers named *_host point to host memory that
 *    is read during the call only. The library never allocates or frees device
 *    memory; scratch space comes from the caller's workspace (`ws_dev`), whose
 *    size the *_workspace functions report. Workspaces must be 256-byte aligned.
 *  - All device work is enqueued on `hip_stream` (a hipStream_t passed as
 *    void*; NULL is the default stream). No call synchronises with the host;
 *    outputs, including the n_*_dev counters, are valid once the stream has
 *    been synchronised. Two calls sharing a workspace must be ordered by the
 *    stream.
 *  - Every call returns an sp_status and never aborts. Host-visible arguments
 *    are validated before anything is launched; on an error nothing is
 *    launched and no output is written. sp_last_error() returns a thread-local
 *    description of the last failure.
 *  - Contents of device buffers (offsets non-decreasing, finite scores, the
 *    host and device copies of the batch offsets agreeing) are the caller's
 *    contract and are not checked.
 */
#ifndef SP_H_
#define SP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SP_OK = 0,
    SP_ERR_INVALID_ARG = 1,   /* null pointer, non-positive size, inconsistent sizes */
    SP_ERR_UNSUPPORTED = 2,   /* valid request outside the supported set */
    SP_ERR_WORKSPACE = 3,     /* workspace missing, misaligned or too small */
    SP_ERR_DEVICE = 4         /* a HIP call failed */
} sp_status;

/* How per-layer head maxima are combined (Appendix A.1.1; Algorithm 1
 * "AggregateMaxMean"). SP_LAYER_MAX is the paper's statement: maximum over
 * layers and heads, then mean over the lookahead rows. SP_LAYER_MEAN takes the
 * maximum over heads only and averages over lookahead rows and layers. */
typedef enum { SP_LAYER_MEAN = 0, SP_LAYER_MAX = 1 } sp_layer_agg;

/* Shape of the draft model's attention and of its K cache.
 * Q is dense bf16 [n_layers][n_q_heads][n_q][head_dim] (per prompt).
 * K of one layer is bf16 with head_dim contiguous; element (kv head, token j,
 * e) sits at  kv * k_stride_head + j * k_stride_token + e  (strides in
 * elements, multiples of 8; layer base pointers 16-byte aligned). Query head h
 * reads kv head h / (n_q_heads / n_kv_heads).
 * Supported: head_dim 64 or 128; 1 <= n_q <= 16; n_q_heads a multiple of
 * n_kv_heads with ratio G <= 16; n_layers <= 128; n_layers * n_kv_heads <=
 * 65535; scale finite and > 0; and the kv head's query group must fit the
 * on-chip staging: with R = 32 * ceil(G/4) * ceil(n_q/8) padded query rows,
 * R <= 224 at head_dim 64 and R <= 96 at head_dim 128 (so G = 16 with
 * n_q > 8 at head_dim 64, and G > 12 or G > 4 with n_q > 8 at head_dim 128,
 * are SP_ERR_UNSUPPORTED). */
typedef struct {
    int32_t n_layers;
    int32_t n_q_heads;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t n_q;              /* lookahead query rows (the paper's N) */
    float   scale;            /* logit scale, normally 1/sqrt(head_dim) */
    int32_t layer_agg;        /* sp_layer_agg */
    int64_t k_stride_token;
    int64_t k_stride_head;
} sp_score_desc;

/* Bytes of workspace sp_score / sp_score_batch need for `total_tokens` prompt
 * tokens in `n_prompts` prompts (upper bound; 1 prompt for sp_score).
 * The first 32-bit word of the workspace is the status word of the last score
 * call that used it: once the stream has been synchronised it reads 0 when the
 * scores are valid and 1 when the single-launch kernel gave up (see sp_score);
 * a caller that cannot scan the scores for NaN can copy this word back. */
sp_status sp_score_workspace(const sp_score_desc *desc, int64_t total_tokens,
                             int32_t n_prompts, size_t *bytes);

/*
 * Token importance of one prompt (Appendix A.1.1; Algorithm 1, the
 * ForwardWithAttn loop's attention and AggregateMaxMean).
 * For every layer l, query head h and lookahead row n the row
 *   p[l,h,n,j] = softmax_j( scale * <Q[l,h,n,:], K[l,h/G,j,:]> ),  j in [0,L)
 * is formed over exactly the L prompt keys (no mask: lookahead rows follow the
 * prompt), and scores_dev[j] receives
 *   SP_LAYER_MAX :  (1/n_q)          sum_n max_{l,h} p[l,h,n,j]
 *   SP_LAYER_MEAN:  (1/(n_q*Lyr))    sum_l sum_n max_h p[l,h,n,j].
 * q_dev: bf16 Q as described above. k_layers_host: host array of n_layers
 * device pointers. scores_dev: float[L]. L == 0 is a no-op returning SP_OK.
 * The softmax is exact (row maximum and sum over all L keys, fp32); the result
 * is deterministic: the same inputs give bit-identical scores.
 * The single-launch kernel needs all its workgroups resident at once, which an
 * otherwise idle device guarantees; if other work occupies the device, its waits
 * on other workgroups are bounded and it gives up. It never hangs.
 *  - Calls for which sp_score_is_fused answers 1 wait for about a second and
 *    have then failed as a whole: every score of the call is NaN and the
 *    workspace's status word (see sp_score_workspace) is 1. A failed call means
 *    "run again", never a wrong value.
 *  - Every other call never fails: some of them use the single-launch kernel too
 *    where it is faster, but give up after some 30 ms, and a last launch then
 *    computes the scores without it (tens of milliseconds to a second).
 * Calls of one process on several streams take turns on the device with it (the
 * first ones after a change of stream may not be able to: they never fail either).
 * On a stream with a compute-unit mask no call fails.
 * Calls recorded into a graph take no turns: such a call uses the single-launch kernel
 * only where sp_score_is_fused (sp_score_batch_is_fused) announces it, and its replays
 * must then not overlap another such call or replay. Its scores may differ from the eager
 * call's by rounding: elsewhere the recorded call takes the three-kernel path, and in a
 * single launch it runs the layers one after another where the eager call may run ranges
 * of them side by side, so that SP_LAYER_MEAN adds them up in another order. Batches
 * announced for several launches run recorded exactly as they do eagerly.
 */
sp_status sp_score(const sp_score_desc *desc, const void *q_dev,
                   const void *const *k_layers_host, int64_t L,
                   float *scores_dev, void *ws_dev, size_t ws_bytes,
                   void *hip_stream);

/*
 * sp_score with the lookahead tokens' own keys in the softmax (Algorithm 1, the
 * ForwardWithAttn loop: the forward pass of lookahead step i also attends to
 * the tokens generated in steps 1 .. i-1). Row n (0-based) of every head is
 * normalised over the L prompt keys and the lookahead keys 0 .. n-1, plus key n
 * itself when look_self is 1 (0 or 1; anything else is SP_ERR_INVALID_ARG):
 *   p[l,h,n,j] = exp(s[l,h,n,j]) / ( sum_{j'<L} exp(s[l,h,n,j'])
 *                                    + sum_{m visible} exp(scale*<Q[l,h,n,:], Klook[l,h/G,m,:]>) )
 * Only prompt tokens are scored; aggregation as in sp_score.
 * k_look_dev: device, bf16, dense [n_layers][n_kv_heads][n_q][head_dim],
 * 16-byte aligned, not null, only read. Everything else as in sp_score (same
 * workspace size, same kernels, same determinism and failure behaviour).
 */
sp_status sp_score_look(const sp_score_desc *desc, const void *q_dev,
                        const void *const *k_layers_host, int64_t L,
                        const void *k_look_dev, int32_t look_self,
                        float *scores_dev, void *ws_dev, size_t ws_bytes,
                        void *hip_stream);

/*
 * sp_score over a paged key cache (Section 3.1 describes KV caches kept in
 * fixed-size blocks of 4k tokens). Token j of layer l lives in page
 * block_table_dev[j / page_tokens] of that layer's pool k_pools_host[l]:
 *   K[l, kv, j, e] = pool_l[ page * page_stride + kv * k_stride_head
 *                            + (j % page_tokens) * k_stride_token + e ]
 * with desc's strides now describing one page (e.g. head-major pages:
 * k_stride_token = head_dim, k_stride_head = page_tokens * head_dim,
 * page_stride = n_kv_heads * page_tokens * head_dim). One block table serves all
 * layers, as in paged decoders. block_table_dev: device, int32,
 * ceil(L / page_tokens) entries, only read. page_tokens: a positive multiple of
 * 512; page_stride: elements, a multiple of 8; every page is allocated whole
 * (rows of the last page beyond L may be read, their contents are ignored).
 * Same result as sp_score on the gathered keys, same kernels, same workspace.
 */
sp_status sp_score_paged(const sp_score_desc *desc, const void *q_dev,
                         const void *const *k_pools_host,
                         const int32_t *block_table_dev, int64_t page_tokens,
                         int64_t page_stride, int64_t L, float *scores_dev,
                         void *ws_dev, size_t ws_bytes, void *hip_stream);

/*
 * sp_score over keys stored as 8-bit floating point (Section 3.1: the deployment
 * keeps its KV cache in blocks on the accelerator; a quantised cache halves the
 * bytes this pass streams). k8_layers_host[l] points at layer l's keys as OCP
 * E4M3 codes (1 sign, 4 exponent bits with bias 7, 3 mantissa bits, finite
 * only; one byte per element), addressed with desc's strides counted in
 * elements, i.e. bytes (multiples of 8, layer bases 16-byte aligned).
 * kscale_dev: device, float [n_layers][n_kv_heads], positive and finite, only
 * read: the key vector of (l, kv, j) is kscale[l][kv] * E4M3(code), and the
 * scores are those of sp_score on exactly these dequantised keys (the queries
 * stay bf16; products are exact, sums are fp32). NaN codes are the caller's to
 * avoid. Contiguous keys of one prompt only; same workspace size and the same
 * choice between the two implementations as sp_score (sp_score_fp8_is_fused;
 * the single-launch kernel fetches codes in 16-byte pieces and so needs both
 * strides to be multiples of 16), same status word and failure behaviour.
 */
sp_status sp_score_fp8(const sp_score_desc *desc, const void *q_dev,
                       const void *const *k8_layers_host, const float *kscale_dev,
                       int64_t L, float *scores_dev, void *ws_dev, size_t ws_bytes,
                       void *hip_stream);

/* Whether sp_score needs the device's compute units to itself for this shape and
 * length on the current device, i.e. can fail (see there): 1 = it relies on the
 * single-launch kernel, which keeps K on chip and reads it from HBM once, 0 = the
 * call never fails: the three-kernel path or, where that is faster, the single-launch
 * kernel with a stand-in: the layers in ranges side by side (shorter prompts), two
 * tiles a workgroup (longer ones), or two blocks of query rows at head_dim 128 (33 to
 * 64 padded rows, up to 8 lookahead rows); -1 = invalid or unsupported desc.
 * In the calls answered with 1 the kernel takes one workgroup per compute unit, each owning T keys:
 * head_dim 64: T = 512, query groups of up to 64 padded rows, 64 to 256
 * workgroups (about 32K to 128K tokens); head_dim 128: T = 256, up to 32 padded
 * rows, 96 to 256 workgroups (about 24K to 64K tokens). Results are the same
 * either way (to rounding); this is for reporting. Host-only. */
int32_t sp_score_is_fused(const sp_score_desc *desc, int64_t L);
/* The same for sp_score_fp8: its single-launch variants need key strides that are
 * multiples of 16 elements; shapes and lengths as above. */
int32_t sp_score_fp8_is_fused(const sp_score_desc *desc, int64_t L);

/*
 * The same for a ragged batch of B prompts whose keys are packed back to back
 * along the token axis: prompt b owns tokens [offsets[b], offsets[b+1]) of each
 * layer's K and of scores_dev; its queries are q_dev + b * (one prompt's Q).
 * offsets_host and offsets_dev hold the same B+1 non-decreasing values with
 * offsets[0] == 0; empty prompts are allowed. Each prompt is softmaxed over
 * its own keys only. 1 <= B <= 4096.
 */
sp_status sp_score_batch(const sp_score_desc *desc, const void *q_dev,
                         const void *const *k_layers_host,
                         const int64_t *offsets_host, const int64_t *offsets_dev,
                         int32_t B, float *scores_dev, void *ws_dev,
                         size_t ws_bytes, void *hip_stream);

/* How sp_score_batch runs this batch on the current device: n > 0 = on the
 * single-launch kernel in n launches (every prompt empty or at least T tokens
 * long and no longer than T tokens per compute unit, T as above; at least 64
 * workgroups in all; prompts share launches, each with all its keys in one, and
 * packed as full as they get no launch has more blocks of four padded query rows
 * than workgroups; several launches may be more than the fewest, run on a half to
 * a quarter of the compute units with two to four ranges of the layers side by
 * side; recorded calls make the same n launches, calls on a stream with a
 * compute-unit mask the fewest, or the three-kernel path's),
 * 0 = a call that never fails (see sp_score_is_fused): the three-kernel path or,
 * where that is faster, the single-launch kernel with a stand-in; -1 = invalid
 * arguments. Same results either way (to rounding). Host-only. */
int32_t sp_score_batch_is_fused(const sp_score_desc *desc,
                                const int64_t *offsets_host, int32_t B);

/* Number of chunks to keep for a keep rate keep_num/keep_den (Section 3.1: the
 * top-K chunks make up a fraction rho of the draft sequence):
 * clamp(ceil(n_chunks * keep_num / keep_den), 1, n_chunks) in integer
 * arithmetic. Returns -1 on invalid arguments (n_chunks < 1, keep_den < 1,
 * keep_num < 0). Host-only. */
int64_t sp_keep_count(int64_t n_chunks, int64_t keep_num, int64_t keep_den);

/* Bytes of workspace sp_select needs for a prompt of L tokens and this chunk size. */
sp_status sp_select_workspace(int64_t L, int32_t chunk, size_t *bytes);

/*
 * Chunk selection (Algorithm 1: AvgPool1D, PartitionIntoChunks, TopKChunks,
 * MergeAdjacentChunks; Appendix A.1.2; Appendix A.3 for pool 13, chunk 32/128).
 *  - pooled[j] = (1/pool_w) * sum of scores over the pool_w-wide window centred
 *    on j, zeros outside [0,L), divisor always pool_w (pool_w odd, >= 1);
 *  - chunk i covers tokens [i*chunk, min((i+1)*chunk, L)); its score is the
 *    mean of pooled over its true size; C = ceil(L/chunk);
 *  - the k chunks with the largest scores are kept, equal scores resolved in
 *    favour of the lower chunk index (compared as fp32, -0 == +0);
 *  - sel_chunks_dev[k]: kept chunk indices, ascending;
 *  - spans_dev[k][2]: maximal runs of adjacent kept chunks as draft-token
 *    ranges [begin, end), ascending; *n_spans_dev of them are written;
 *  - chunk_scores_dev: optional float[C] copy of the chunk scores (may be NULL).
 * Requires 1 <= k <= C, 1 <= chunk, L >= 1. Scores must not be NaN.
 */
sp_status sp_select(const float *scores_dev, int64_t L, int32_t pool_w,
                    int32_t chunk, int64_t k, int32_t *sel_chunks_dev,
                    int64_t *spans_dev, int32_t *n_spans_dev,
                    float *chunk_scores_dev, void *ws_dev, size_t ws_bytes,
                    void *hip_stream);

/*
 * sp_select for a ragged batch of B prompts in one or two launches (Algorithm 1, the
 * same four steps, each prompt on its own: pooling windows and chunks never
 * cross a prompt's end). scores_dev is packed as sp_score_batch leaves it:
 * prompt b owns [offsets[b], offsets[b+1]). kept_off holds the prefix sums of the
 * prompts' chunk counts to keep, kept_off[0] = 0: prompt b keeps
 * k_b = kept_off[b+1] - kept_off[b] chunks, 1 <= k_b <= ceil(L_b / chunk), or 0
 * for an empty prompt (the caller fills it with sp_keep_count). offsets and
 * kept_off are each given twice with the same B+1 values, in host and in device
 * memory. Outputs, packed by kept_off:
 *  - sel_chunks_dev[kept_off[B]]: prompt b's k_b kept chunk indices (relative to
 *    the prompt), ascending, from kept_off[b] on;
 *  - spans_dev[kept_off[B]][2]: its spans as token ranges relative to the prompt,
 *    from kept_off[b] on; n_spans_dev[b] of them are written;
 *  - chunk_scores_dev: optional; prompt b's chunk scores start at
 *    offsets[b] / chunk + b (so total / chunk + B + 1 floats in all).
 * Workspace: sp_select_batch_workspace(offsets[B], B, chunk). 1 <= B <= 4096.
 */
sp_status sp_select_batch_workspace(int64_t total_tokens, int32_t B, int32_t chunk,
                                    size_t *bytes);
sp_status sp_select_batch(const float *scores_dev, const int64_t *offsets_host,
                          const int64_t *offsets_dev, int32_t B, int32_t pool_w,
                          int32_t chunk, const int64_t *kept_off_host,
                          const int64_t *kept_off_dev, int32_t *sel_chunks_dev,
                          int64_t *spans_dev, int32_t *n_spans_dev,
                          float *chunk_scores_dev, void *ws_dev, size_t ws_bytes,
                          void *hip_stream);

/*
 * sp_select for callers that cannot allocate device memory or pass a workspace:
 * code recorded into a HIP graph, tight serving loops, harnesses that forbid
 * hipMalloc. Same arguments, kernels and results as sp_select, without ws_dev /
 * ws_bytes: the chunk scores go to an array that is part of the library's
 * device image (SP_SELECT_STATIC_MAX_CHUNKS floats = 1 MiB, held on every
 * device the library is used on until the process ends). The call allocates
 * and frees nothing. More than SP_SELECT_STATIC_MAX_CHUNKS chunks is
 * SP_ERR_UNSUPPORTED (use sp_select). The first call on a device looks the
 * array's address up (a host-only query; make that call outside a graph
 * capture). All calls on one device share the array: calls that may overlap
 * on the device (different streams without ordering) race; calls ordered by a
 * stream or by events do not, and nothing has to be cleared between them.
 */
#define SP_SELECT_STATIC_MAX_CHUNKS (1 << 18)
sp_status sp_select_static(const float *scores_dev, int64_t L, int32_t pool_w,
                           int32_t chunk, int64_t k, int32_t *sel_chunks_dev,
                           int64_t *spans_dev, int32_t *n_spans_dev,
                           float *chunk_scores_dev, void *hip_stream);

/* Bytes of workspace sp_select_budget needs (SP_ERR_UNSUPPORTED beyond 65536 chunks). */
sp_status sp_select_budget_workspace(int64_t L, int32_t chunk, size_t *bytes);

/*
 * Chunk selection for a fixed target-side length (Section 3.1: compressed
 * prompts of 8k .. 32k target tokens, multiples of the KV block size; the
 * paper derives the keep rate from that length and notes that the result only
 * lands near it). Here k is searched on the device: the largest k in 1..C such
 * that the top-k chunks, merged into spans and projected onto the target
 * tokenisation exactly as sp_project does, keep at most `budget` target
 * tokens; k = 1 if a single chunk already keeps more. Pooling, chunk scores,
 * ranking and tie-breaking are those of sp_select, and the outputs are what
 * sp_select would write for that k, except that the buffers must hold the
 * worst case: sel_chunks_dev[C], spans_dev[C][2] (C = ceil(L/chunk) <= 65536).
 *  - draft_off_dev[L+1], target_off_dev[M+1]: character offsets as in sp_project;
 *  - *k_dev: the chosen k (also the number of entries of sel_chunks_dev written);
 *  - *n_kept_dev: optional, the target tokens kept at that k (what sp_project
 *    reports for the written spans);
 *  - chunk_scores_dev: optional float[C].
 * Requires L >= 1, 1 <= M < 2^31, budget >= 0. Integer work after the chunk
 * scores: exact and deterministic.
 */
sp_status sp_select_budget(const float *scores_dev, int64_t L, int32_t pool_w,
                           int32_t chunk, const int64_t *draft_off_dev,
                           const int64_t *target_off_dev, int64_t M,
                           int64_t budget, int32_t *sel_chunks_dev,
                           int64_t *spans_dev, int32_t *n_spans_dev,
                           int64_t *k_dev, int64_t *n_kept_dev,
                           float *chunk_scores_dev, void *ws_dev,
                           size_t ws_bytes, void *hip_stream);

/*
 * Projection of kept draft-token spans onto the target model's tokenisation
 * (Algorithm 1: MapDraftChunksToTextSpans and the target tokenisation of the
 * kept text; Section 3.1), in character-offset form. Both tokenisations are
 * given as non-decreasing character offsets into the same text:
 * draft_off_dev[L+1] and target_off_dev[M+1]. Draft span [a,b) covers
 * characters [draft_off[a], draft_off[b]); target token t is kept iff
 *      target_off[t] < draft_off[b]  and  target_off[t+1] > draft_off[a]
 * for some span. spans_dev is a buffer of max_spans entries whose first
 * *n_spans_dev (at most max_spans) are ascending, disjoint spans, as written by
 * sp_select; the kernels may read the entries after them (so all max_spans
 * must be readable device memory) and do not use what they hold.
 *  - tspans_dev[max_spans][2]: kept target tokens as maximal ranges
 *    [begin, end), ascending, disjoint and non-adjacent (ranges that overlap or
 *    touch are merged); *n_tspans_dev of them are written (with max_spans > 1024
 *    or M >= 258048, entries behind them, as many as there are spans, may hold
 *    intermediate values);
 *  - keep_mask_dev: optional uint8[M], 1 for kept target tokens (may be NULL);
 *  - *n_kept_dev: number of kept target tokens.
 * Requires L >= 1, M >= 1, 1 <= max_spans <= 2^24.
 */
sp_status sp_project(const int64_t *draft_off_dev, int64_t L,
                     const int64_t *target_off_dev, int64_t M,
                     const int64_t *spans_dev, const int32_t *n_spans_dev,
                     int32_t max_spans, int64_t *tspans_dev,
                     int32_t *n_tspans_dev, uint8_t *keep_mask_dev,
                     int64_t *n_kept_dev, void *hip_stream);

/*
 * sp_project for a ragged batch in one launch (Algorithm 1, the same mapping,
 * each prompt on its own text). Packed inputs: prompt b's L_b + 1 draft offsets
 * start at draft_off_dev[offsets[b] + b], its M_b + 1 target offsets at
 * target_off_dev[moffsets[b] + b] (moffsets = prefix sums of the prompts' target
 * token counts), its spans at spans_dev[kept_off[b]] with n_spans_dev[b] of them
 * valid, as sp_select_batch writes them. Packed outputs: prompt b's target ranges
 * (relative to its own target tokens) from tspans_dev[kept_off[b]] on,
 * n_tspans_dev[b] of them; its mask bytes at keep_mask_dev[moffsets[b]] (optional);
 * n_kept_dev[b]. offsets, moffsets and kept_off are each given in host and in
 * device memory with the same B+1 values, first value 0. A prompt may have at
 * most 1024 spans and fewer than 258048 target tokens (SP_ERR_UNSUPPORTED
 * otherwise: call sp_project for it). 1 <= B <= 4096.
 */
sp_status sp_project_batch(const int64_t *draft_off_dev, const int64_t *offsets_host,
                           const int64_t *offsets_dev, const int64_t *target_off_dev,
                           const int64_t *moffsets_host, const int64_t *moffsets_dev,
                           int32_t B, const int64_t *spans_dev,
                           const int32_t *n_spans_dev, const int64_t *kept_off_host,
                           const int64_t *kept_off_dev, int64_t *tspans_dev,
                           int32_t *n_tspans_dev, uint8_t *keep_mask_dev,
                           int64_t *n_kept_dev, void *hip_stream);

/* Bytes of workspace sp_assemble needs for up to max_spans kept ranges. */
sp_status sp_assemble_workspace(int32_t max_spans, size_t *bytes);

/*
 * Compressed target prompt in token-id form (Algorithm 1: ConcatWithDelim, the
 * target tokenisation of the compressed text and the new contiguous position
 * ids; Section 3.2; Appendix A.3 names the delimiters). target_ids_dev[M] is
 * the target tokenisation of the original text; tspans_dev holds
 * *n_tspans_dev (at most max_spans) ascending, disjoint ranges [begin, end) of
 * kept target tokens, as written by sp_project; delim_ids_dev[n_delim] is the
 * delimiter's own tokenisation (n_delim may be 0, then the pointer may be NULL).
 * The output is the kept ranges in order with the delimiter's ids between
 * consecutive ranges (none before the first or after the last):
 *  - *out_len_dev = kept tokens + (ranges - 1) * n_delim  (0 for no range),
 *    the full length even when it exceeds out_capacity;
 *  - the first min(out_len, out_capacity) entries are written of
 *    out_ids_dev (token ids), out_pos_dev (position ids 0, 1, 2, ...: the
 *    compressed prompt is renumbered, original positions are not restored) and
 *    the optional out_src_dev (original target index of each output token, -1
 *    for delimiter tokens; may be NULL).
 * Requires M >= 1, 1 <= max_spans <= 2^24, 0 <= n_delim <= 1024,
 * 1 <= out_capacity < 2^31. Range bounds are not checked beyond clamping to [0, M].
 */
sp_status sp_assemble(const int32_t *target_ids_dev, int64_t M,
                      const int64_t *tspans_dev, const int32_t *n_tspans_dev,
                      int32_t max_spans, const int32_t *delim_ids_dev,
                      int32_t n_delim, int64_t out_capacity,
                      int32_t *out_ids_dev, int32_t *out_pos_dev,
                      int64_t *out_src_dev, int64_t *out_len_dev,
                      void *ws_dev, size_t ws_bytes, void *hip_stream);

/* ---- the draft model's forward pass around the importance pass ----
 *
 * What sp_score reads is left behind by a draft model's forward pass: the cache
 * of the prompt's keys and the lookahead rows' queries (Algorithm 1,
 * ForwardWithAttn). The calls below are that pass's work on the cache and on the
 * logits, one decoder layer at a time: new keys and values go into a paged
 * cache (sp_cache_append), queries attend over it (sp_attend), and the next
 * token and the probabilities of given ones are read off the logits
 * (sp_logprobs). Projections can be products in 4 bits (sp_mx4_quantise,
 * sp_mx4_matmul), and a cache can be held to a budget: what its tokens draw is
 * added up (sp_attend_weights) and the rest is dropped (sp_cache_evict). A bf16
 * cache with pages of a multiple of 512 tokens is what sp_score_paged reads
 * afterwards.
 */

/* How a paged cache holds its elements. SP_CACHE_BF16: as they are.
 * SP_CACHE_E4M3: OCP E4M3 codes, one byte each, with one float scale for every
 * SP_CACHE_BLOCK consecutive tokens of a page and kv head: value = scale * E4M3(code).
 * SP_CACHE_MX4: microscaled 4-bit elements (OCP MXFP4): E2M1 codes (1 sign, 2 exponent
 * bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the lower element in the
 * lower bits, with one scale for every SP_MX4_GROUP consecutive elements of a token and
 * head: a byte e that stands for 2^(e - 127), or for NaN (as does every element of the
 * group then) where it is 255. */
typedef enum { SP_CACHE_BF16 = 0, SP_CACHE_E4M3 = 1, SP_CACHE_MX4 = 3 } sp_cache_type;
#define SP_CACHE_BLOCK 32
#define SP_MX4_GROUP 32

/* A layer's paged cache: two pools (keys, values) of n_pages pages each with the
 * same strides, in elements, head_dim contiguous:
 *   K[b, kv, j, e] = k_pool[ page * page_stride + kv * stride_head
 *                            + (j % page_tokens) * stride_token + e ],
 *   page = block_table_dev[b * table_stride + j / page_tokens]
 * block_table_dev: device, int32; table_stride entries for each request. E4M3
 * pools come with dense float scale arrays
 * [n_pages][n_kv_heads][page_tokens / SP_CACHE_BLOCK], MX4 pools with dense byte scale
 * arrays [n_pages][n_kv_heads][page_tokens][head_dim / SP_MX4_GROUP], 16-byte aligned
 * (k_scale, v_scale; null for bf16). Pools, queries, keys and values are 16-byte aligned.
 * Query head h reads kv head h / (n_q_heads / n_kv_heads).
 * Supported: head_dim 64 or 128; n_q_heads a multiple of n_kv_heads with ratio
 * G <= 16; n_kv_heads <= 4096; page_tokens a positive multiple of SP_CACHE_BLOCK, at most
 * 2^24; strides multiples of 32 (MX4), 16 (E4M3) or 8 (bf16) elements, stride_token >=
 * head_dim and <= 2^24, none above 2^40; 1 <= n_pages < 2^31. */
typedef struct {
    int32_t n_q_heads;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t cache_type;       /* sp_cache_type */
    int64_t n_pages;
    int64_t page_tokens;
    int64_t page_stride;
    int64_t stride_head;
    int64_t stride_token;
} sp_cache_desc;

/* Pairs that the rotation turns: SP_ROTATE_HALF elements (i, i + rot_dim/2),
 * SP_ROTATE_PAIRS elements (2i, 2i + 1); i in [0, rot_dim/2). */
typedef enum { SP_ROTATE_HALF = 0, SP_ROTATE_PAIRS = 1 } sp_rotate_style;

/*
 * Appends the keys and values of new tokens to a paged cache and rotates keys and
 * (optionally) queries to their positions on the way. Request b brings tokens
 * [offsets[b], offsets[b+1]) of the packed inputs (offsets in host and in device
 * memory, the same B+1 non-decreasing values, offsets[0] == 0; 0 <= B <= 4096,
 * requests without new tokens are allowed; (new tokens / 32 + 2 B) * n_kv_heads < 2^24).
 * Its i-th new token becomes token start_dev[b] + i of its cache.
 *  - k_dev, v_dev: bf16, token t at t * k_stride (v_stride), n_kv_heads * head_dim
 *    contiguous elements each; strides in elements, multiples of 8 (so keys, values and
 *    queries can be parts of one projection's output);
 *  - q_dev, q_out_dev: optional (both or neither): bf16 queries, n_q_heads * head_dim
 *    contiguous elements a token at t * q_stride, and dense bf16
 *    [tokens][n_q_heads][head_dim] for the rotated ones. q_out_dev may be q_dev if that is dense.
 *  - rot_dim: rotated elements of each head, 0 (no rotation) or a multiple of 16 up to
 *    head_dim; with c = cos_dev[p][i], s = sin_dev[p][i] (float, [n_pos][rot_dim/2],
 *    16-byte aligned) the pair (x, y) of index i becomes (x c - y s, y c + x s), products and
 *    sums rounded to float one by one. p = positions_dev[t] (device, int32, one for each packed
 *    token), or without it (null) the token's index in its cache; p is clamped to [0, n_pos).
 *  - bf16 caches take the result rounded to nearest. E4M3 caches: of the tokens of one block
 *    of SP_CACHE_BLOCK slots and kv head that this call brings, the largest magnitude m gives
 *    the smallest power of two s >= 2^-64 with m <= 448 s; a block that already holds tokens
 *    before start_dev[b] keeps the larger of s and its present scale, and the codes of those
 *    tokens are brought to it (exactly where that scale was a power of two, but for values that fall among
 *    E4M3's subnormals); new codes are E4M3(x / s), rounded to nearest, x / s in float. Results that are not
 *    finite are stored as NaN codes and do not count for m. MX4 caches: each group of a token by itself,
 *    by the rule of sp_mx4_quantise; no other token's codes or scales are looked at.
 * Slots at and behind start + new tokens are not touched, except that a new token may lie in a
 * slot that is in use: then it is replaced (a rejected lookahead token), and, in an E4M3 cache, with it
 * whatever follows it in its block. Tokens whose slot lies beyond the block table's row, or whose page is not
 * in [0, n_pages), are not stored (their queries are still rotated). Two requests
 * of one call must not append to the same page's same block (MX4 and bf16: slot).
 */
sp_status sp_cache_append(const sp_cache_desc *desc, const void *k_dev, int64_t k_stride,
                          const void *v_dev, int64_t v_stride, const void *q_dev,
                          int64_t q_stride, void *q_out_dev, const int64_t *offsets_host,
                          const int64_t *offsets_dev, int32_t B, const int32_t *start_dev,
                          const int32_t *positions_dev, const int32_t *block_table_dev,
                          int64_t table_stride, const float *cos_dev, const float *sin_dev,
                          int64_t n_pos, int32_t rot_dim, int32_t rot_style,
                          void *k_pool_dev, void *v_pool_dev, void *k_scale_dev,
                          void *v_scale_dev, void *hip_stream);

/* Bytes of workspace sp_attend needs for these queries and contexts of at most
 * max_len tokens (0 where it needs none). They are enough for every smaller max_len too, so
 * a program asks once, for its longest context. The queries count as they are given: other
 * offsets, with fewer rows or requests among them, may need more. */
sp_status sp_attend_workspace(const sp_cache_desc *desc, const int64_t *offsets_host,
                              int32_t B, int64_t max_len, size_t *bytes);

/*
 * Attention of ragged queries over a paged cache. Request b has query rows
 * [offsets[b], offsets[b+1]) (n_b of them; offsets as in sp_cache_append) of q_dev, dense
 * bf16 [rows][n_q_heads][head_dim], and a context of lens_dev[b] tokens (device, int32),
 * which normally counts the new tokens that were appended before. Row r of request b
 * sees key j iff j < lens[b] and, with causal = 1, j <= p and (window = 0 or
 * j > p - window), where p = lens[b] - n_b + r is the row's own token. With
 * causal = 0 the window must be 0.
 *   out_dev[row, h] = sum_j p_j V[b, h/G, j],  p_j = softmax_j( scale * <q, K[b, h/G, j]> )
 * as dense bf16 [rows][n_q_heads][head_dim], and lse_dev[row, h] (float, optional) the natural
 * logarithm of the softmax's denominator. A row that sees no key gets zeros and an lse
 * of minus infinity. Slots that no row of the request sees (those of a last page past the
 * context among them) may hold anything, NaN included.
 * What a row sees should be finite: logits below 2^120, values below 2^90 in magnitude, scales
 * finite and not negative (a value scale below 2^-64 may count as 2^-64: zero is in order for a block
 * of zeros); scale bytes of MX4 caches stand for less than 2^90. A row that sees a NaN becomes
 * NaN, and other rows of its request may.
 * At most 2^26 query tokens and contexts of at most 2^30 tokens; requests times kv heads, and tiles of 256
 * query rows times kv heads, below 2^23.
 * max_len bounds the contexts from the host's side (a longer lens[b] counts as
 * max_len, a negative one as 0) and must not exceed table_stride * page_tokens; the call reads the table entries
 * of the tokens below lens[b] only. The probabilities of the second product are rounded to bf16; sums and statistics are held in fp32. The
 * result does not change from call to call on the same inputs. 0 < scale <= 2.3e38. Scale times a key scale
 * counts as about 2^-127 where it is less and as about 2^127 where it is more.
 */
sp_status sp_attend(const sp_cache_desc *desc, const void *q_dev,
                    const int64_t *offsets_host, const int64_t *offsets_dev, int32_t B,
                    const int32_t *lens_dev, int64_t max_len,
                    const int32_t *block_table_dev, int64_t table_stride,
                    const void *k_pool_dev, const void *v_pool_dev,
                    const void *k_scale_dev, const void *v_scale_dev, float scale,
                    int32_t causal, int64_t window, void *out_dev, float *lse_dev,
                    void *ws_dev, size_t ws_bytes, void *hip_stream);

/*
 * How much attention the tokens of a paged cache have drawn: the weight that decides which of them
 * sp_cache_evict keeps. Queries, contexts, masks and the cache's keys are those of an sp_attend
 * call, whose lse_dev this call takes; the values are not looked at:
 *   weights_dev[b, h, j] = old + sum over rows r of request b that see key j, and over the query
 *                          heads g of kv head h, of exp( scale * <q[r, g], K[b, h, j]> - lse_dev[r, g] )
 * for j < lens[b]; entries behind are left as they were. weights_dev: float
 * [B][n_kv_heads][weights_stride], weights_stride >= max_len.
 * old = old_dev[b, h, j] (the same layout; may be weights_dev itself, else they must not overlap)
 * for tokens that were there before the rows' own: j < lens[b] - n_b with causal = 1, all with
 * causal = 0; 0 for the others and where old_dev is null. A request without rows keeps its old
 * weights. Rows with an lse of minus infinity add nothing.
 * Arithmetic is in fp32, in an order that is fixed by the offsets, the lengths and max_len.
 * A row that sees a NaN, or whose lse is NaN, makes NaN of the weights that it adds to, and of
 * others of its request.
 * Limits as in sp_attend; requests times kv heads at most 65535.
 */
sp_status sp_attend_weights(const sp_cache_desc *desc, const void *q_dev, const int64_t *offsets_host,
                            const int64_t *offsets_dev, int32_t B, const int32_t *lens_dev, int64_t max_len,
                            const int32_t *block_table_dev, int64_t table_stride, const void *k_pool_dev,
                            const void *k_scale_dev, float scale, int32_t causal, int64_t window,
                            const float *lse_dev, const float *old_dev, float *weights_dev,
                            int64_t weights_stride, void *hip_stream);

/*
 * Eviction: the cached tokens of most weight, of each kv head by itself, into other pages. Request
 * b has lens_dev[b] tokens and a budget of budget_dev[b] (device, int32; a negative one counts as
 * 0, one above max_budget as max_budget). With n = min(len, budget):
 *   - a context of at most the budget is kept whole;
 *   - else the first s = min(sinks, budget) tokens, the last r = min(recent, budget - s), and of
 *     those between the budget - s - r with the largest weights_dev[b, h, j], equal weights in
 *     favour of the earlier token. Weights are compared as numbers, a positive NaN above and a
 *     negative one below all others, -0 equal to 0.
 * The kept tokens of kv head h, in their order, become tokens 0 .. n - 1 of the pages that
 * dst_table_dev names:
 *   - their keys and values (v_pool_dev and v_scale_dev as in sp_attend). bf16 and MX4 as they
 *     are, with their scales. E4M3: a block takes the largest scale s among those of its tokens (a
 *     NaN counts as the largest), codes are brought to it, E4M3(code * (scale / s)): exactly where
 *     scales are powers of two, but for what falls among the subnormals;
 *   - kept_dev[b, h, i] (int32 [B][n_kv_heads][max_budget]): which token it was;
 *   - new_weights_dev[b, h, i] (optional, float [B][n_kv_heads][max_budget], not overlapping
 *     weights_dev): its weight, bit for bit.
 * new_lens_dev[b] = n (int32, neither lens_dev nor budget_dev itself). Entries and slots at and
 * behind n are left as they were, but for the scale of the E4M3 block that holds slot n - 1.
 * Keys keep the rotation of their old position: new tokens go on from there (sp_cache_append's
 * positions_dev), while attention's masks and windows count slots.
 * The pages of dst_table must be different ones for all requests, and not among those that
 * block_table names (for any request): source pages are only read, and free afterwards; pages that
 * requests share stay as they are. Tokens whose destination lies beyond dst_table's row, or whose
 * destination page is not in [0, n_pages), are not moved.
 * weights_dev: float [B][n_kv_heads][weights_stride], weights_stride >= max_len. Contexts are
 * bounded by max_len as in sp_attend. sinks, recent >= 0. 0 <= max_budget <= 2^30,
 * min(max_len, max_budget) <= 2^29 - 32; requests times kv heads at most 65535. The result does
 * not change from call to call.
 */
sp_status sp_cache_evict(const sp_cache_desc *desc, int32_t B, const int32_t *lens_dev, int64_t max_len,
                         const int32_t *budget_dev, int64_t max_budget, int64_t sinks, int64_t recent,
                         const float *weights_dev, int64_t weights_stride,
                         const int32_t *block_table_dev, int64_t table_stride,
                         const int32_t *dst_table_dev, int64_t dst_stride, void *k_pool_dev, void *v_pool_dev,
                         void *k_scale_dev, void *v_scale_dev, int32_t *new_lens_dev, int32_t *kept_dev,
                         float *new_weights_dev, void *hip_stream);

/* Type of logits, and of what goes into and comes out of a product in 4 bits. */
typedef enum { SP_LOGITS_F32 = 0, SP_LOGITS_BF16 = 1 } sp_logits_type;

/* Largest number of alternatives sp_logprobs reports. */
#define SP_LOGPROBS_MAX_TOP 32

/* Bytes of workspace that sp_logprobs needs at most for n_rows rows or fewer, of either type
 * (0 where it needs none): a program asks once, for its most rows. A call that needs none
 * itself (many rows, short rows) may go without. */
sp_status sp_logprobs_workspace(int64_t n_rows, int64_t vocab, int32_t n_top, size_t *bytes);

/*
 * Log probabilities of rows of logits x (dtype an sp_logits_type, row r at r * row_stride
 * elements, vocab of them; row_stride >= vocab; only element alignment is needed).
 * With lse = log sum_v exp(x_v), lp_v = x_v - lse and p_v = exp(lp_v):
 *  - logprob_dev[r]  = lp of token targets_dev[r] (int32; both may be null); 0 for a target
 *    outside [0, vocab), which is how rows without one are marked;
 *  - entropy_dev[r]  = - sum_v p_v lp_v (optional);
 *  - top_ids_dev[r][n_top], top_logprobs_dev[r][n_top]: the n_top likeliest tokens,
 *    likeliest first, equal logits in favour of the lower token (0 <= n_top <=
 *    SP_LOGPROBS_MAX_TOP, n_top <= vocab; n_top = 0: both may be null). The greedy
 *    next token is top_ids[r][0].
 * Minus infinity marks forbidden tokens (p = 0, lp = -inf). A row of nothing else has
 * lp = -inf throughout and entropy 0. Logits must not be NaN or plus infinity.
 * All arithmetic is in fp32, and the result does not change from call to call.
 * 0 <= n_rows < 2^31, 1 <= vocab < 2^31.
 */
sp_status sp_logprobs(const void *logits_dev, int32_t dtype, int64_t n_rows, int64_t vocab,
                      int64_t row_stride, const int32_t *targets_dev, int32_t n_top,
                      float *logprob_dev, float *entropy_dev, int32_t *top_ids_dev,
                      float *top_logprobs_dev, void *ws_dev, size_t ws_bytes,
                      void *hip_stream);

/*
 * Rows of numbers to microscaled 4-bit elements (as in SP_CACHE_MX4 caches). Of each SP_MX4_GROUP
 * elements x of a row the largest magnitude m gives the smallest power of two s >= 2^-64 with
 * m <= 6 s; scales_dev[r][k / 32] = log2 s + 127, and codes are E2M1(x / s), rounded to nearest,
 * halfway to the even code, the sign of zero kept. A group that holds a NaN or an infinity gets
 * scale byte 255 and codes of zero.
 * x_dev: float or bf16 (dtype an sp_logits_type), row r at r * row_stride elements (row_stride >=
 * K, a multiple of 8, rows 16-byte aligned). codes_dev: [rows][K / 2] bytes, scales_dev:
 * [rows][K / 32] bytes, both dense, codes 16-byte, scales 4-byte aligned. K is a positive multiple
 * of 32 below 2^31. 0 <= rows < 2^31; rows * K < 2^35. x_dev, codes_dev and scales_dev must not
 * overlap.
 */
sp_status sp_mx4_quantise(const void *x_dev, int32_t dtype, int64_t rows, int64_t K, int64_t row_stride,
                          void *codes_dev, void *scales_dev, void *hip_stream);

/*
 * Product of two microscaled 4-bit matrices, a projection's activations and weights:
 *   out_dev[m][n] = sum_k A[m][k] W[n][k],  0 <= m < M, 0 <= n < N
 * with A and W as sp_mx4_quantise leaves them: a_codes_dev [M][K / 2], a_scales_dev [M][K / 32],
 * w_codes_dev [N][K / 2], w_scales_dev [N][K / 32], dense, codes 16-byte, scales 4-byte aligned.
 * out_dev: float or bf16 (dtype an sp_logits_type), row m at m * out_stride elements (out_stride
 * >= N), not overlapping the operands. Products are exact, sums are held in fp32 in an order that
 * the sizes fix, the result is rounded once. Rows with a NaN scale give NaN. K is a positive
 * multiple of 32 below 2^31, 0 <= M, N < 2^31; (M / 16 + 1) * (N / 16 + 1) < 2^24.
 */
sp_status sp_mx4_matmul(const void *a_codes_dev, const void *a_scales_dev, int64_t M, const void *w_codes_dev,
                        const void *w_scales_dev, int64_t N, int64_t K, void *out_dev, int32_t dtype, int64_t out_stride,
                        void *hip_stream);

/*
 * Measurement aid: streams `bytes` bytes of buf_dev (device, 16-byte aligned,
 * bytes a positive multiple of 16) with plain wide loads and XORs what it read
 * into *sink_dev (device, 64 bits: lanes fold their 16-byte chunks to 64 bits
 * as (x ^ z) << 32 | (y ^ w) of the four 32-bit words; not cleared first).
 * The rate at which this call reads is the device's achievable streaming-read
 * bandwidth: the practical ceiling, next to the datasheet figure, for
 * sp_score, which streams the K cache once (Appendix A.1.1's attention of the
 * lookahead rows over the whole prompt). Enqueued on hip_stream like every
 * other call.
 */
sp_status sp_hbm_read_probe(const void *buf_dev, size_t bytes, uint64_t *sink_dev,
                            void *hip_stream);

/* Test hook for the failure path of the single-launch score kernel; not for
 * production use. Launches that follow give a wait up after `spin_limit` polls
 * (default 1 << 20), and with force_miss == 1 the waves that combine partial
 * results treat them as never arriving, so that the bounded waits give up on an
 * idle device and every kernel still runs to its end; force_miss == 2 + b does so
 * in the launches that hold prompt b of their call only. force_miss == -1 leaves
 * out the last workgroup of a launch instead, as if it had found no compute unit:
 * only what waits for it gives up. Process-wide. */
void sp_debug_fused_giveup(uint32_t spin_limit, int32_t force_miss);

/* Test hook: how the calling thread's last score call (of more than no tokens)
 * was launched. 0 = the three-kernel path; otherwise the single-launch kernel:
 * bits 0-7 tiles of keys a workgroup owns, bits 8-15 layer ranges side by side,
 * bits 16-23 launches, bit 24 set if the call's last launch can stand in for it. */
int32_t sp_debug_score_path(void);

/* Description of the last error raised on the calling thread ("" if none).
 * The string lives in thread-local storage owned by the library. */
const char *sp_last_error(void);

/* Library version string (static storage). */
const char *sp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SP_H_ */
