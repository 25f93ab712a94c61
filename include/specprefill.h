/*
 * specprefill.h -- C ABI of the SpecPrefill token-importance path for AMD MI355X (gfx950).
 *
 * Method: "Speculative Prefill" (arXiv 2502.02789).  A draft model's stored queries
 * (the last prompt token and/or N look-ahead tokens) score every prompt token by
 * attention against the draft's K cache (Sec. 3.2 equation); scores are aggregated
 * over heads, layers and queries (Sec. 3.2.2), smoothed by 1-D average pooling and
 * cut to the top-k contiguous chunks (Sec. 3.2.3); kept tokens travel to the base
 * model with their ORIGINAL position ids (Sec. 3.2.4).  Algorithm 1 names these
 * steps compute_attention_score, aggregate_attention_score,
 * chunk_select_from_smoothed_attention and restore_pos_ids.
 *
 * Conventions for every entry point
 *   - Pointers named d_* are DEVICE pointers owned by the caller; everything else
 *     (the structs themselves, k_layers[], h_* arrays) is HOST memory.
 *   - The library allocates and frees no device memory; scratch space is the
 *     caller's workspace (size from the *_workspace_bytes query).  It never
 *     synchronises the stream: all work is enqueued on `hip_stream`
 *     (a hipStream_t passed as void*, NULL = the default stream).
 *   - Return value: SP_OK (0) or a negative sp_status.  On an argument error
 *     nothing is launched and no output is written.
 *   - Sequence b owns prompt tokens [cu_seqlens[b], cu_seqlens[b+1]) of the flat
 *     token axis of length T = cu_seqlens[B]; empty sequences are allowed.
 *   - NaN/Inf in Q or K, and token ids outside [0, V), are precondition violations
 *     (undefined values, no fault for NaN/Inf; ids are NOT range-checked on device).
 *   - Calls that share a workspace must not overlap in time.
 *   - One-time set-up per device (kernel attributes, occupancy queries, the address of the
 *     library's static scratch) happens inside the first call made on that device, under a
 *     lock; that first call must not be made while the stream is being captured into a graph.
 */
#ifndef SPECPREFILL_H
#define SPECPREFILL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SP_API __attribute__((visibility("default")))

typedef enum {
  SP_OK = 0,
  SP_EINVAL = -1,       /* a size, rate or enum is out of range                  */
  SP_ENULL = -2,        /* a required pointer is NULL                            */
  SP_EALIGN = -3,       /* a pointer or stride breaks the 16-byte alignment rule */
  SP_EWORKSPACE = -4,   /* workspace missing or smaller than *_workspace_bytes   */
  SP_EUNSUPPORTED = -5, /* valid request this build has no kernel for            */
  SP_ELAUNCH = -6,      /* the HIP runtime refused a launch                      */
  SP_ETIMEOUT = -7      /* a bounded device-side wait expired (see sp_score_check) */
} sp_status;

/* How per-layer values are combined (Sec. 3.2.2).  The paper takes the maximum over
 * heads AND layers; the alternative keeps the maximum over heads but averages layers. */
typedef enum { SP_LAYER_MAX = 0, SP_LAYER_MEAN = 1 } sp_layer_reduce;

/* How the K cache stores its elements.  SP_K_FP8_E4M3: one byte per element, OCP 8-bit floating point,
 * format E4M3 (1 sign, 4 exponent, 3 mantissa bits, bias 7, subnormals, no infinities, S.1111.111 = NaN,
 * largest finite value 448), and the key the paper's Sec. 3.2 equation sees is
 *     K_l[i, g, t] = d_k_scale[l * H_kv + g] * decode(byte)
 * (one fp32 scale per layer and KV head, as an engine with an 8-bit KV cache keeps them).  Every E4M3
 * value is a bf16 value, so the products with the bf16 queries are formed exactly as for a bf16 cache and
 * accumulated in fp32; the scale joins the logit scale.  Scores therefore meet the same tolerance against
 * the definition evaluated on the decoded keys as a bf16 cache does.  NaN codes are a precondition
 * violation like NaN in a bf16 cache. */
typedef enum { SP_K_BF16 = 0, SP_K_FP8_E4M3 = 1 } sp_k_dtype;

#define SP_MAX_LAYERS 128
#define SP_MAX_QUERIES 16

/* sp_score_args.flags */
#define SP_SCORE_EXCLUSIVE_DEVICE 1u /* The caller promises that nothing else runs on the GPU while
                                        sp_score runs (no other stream, no other process).  The
                                        single-pass kernels that share one prompt among workgroups
                                        read the K cache once but exchange softmax row statistics between
                                        workgroups that must all be resident together; with the
                                        flag they wait for one another as long as that can
                                        sensibly take.  That may concern one prompt of more than 3072 keys,
                                        from 2048 keys on where layers times KV heads are 128 or more,
                                        and of any length where they are fewer than 64; no other call
                                        waits.  (From 3073 keys on the same kernels run without the
                                        flag; below, scores with and without it agree to the
                                        tolerance of fp32 summation order, not bit for bit.)
                                        If the promise is broken a bounded wait can
                                        expire; the call's scores are then NaN (see
                                        sp_score_check and sp_pool_select), never silently
                                        wrong.
                                        Without the flag the scores are valid whatever else runs on
                                        the GPU: where a workgroup has waited for the others about
                                        one and a half to three times as long as the call takes
                                        undisturbed (and 50 microseconds), the call gives up waiting
                                        as a whole, and its second launch (which returns at once
                                        otherwise) forms the results again from the row statistics,
                                        which are all there by then.  At worst K is read twice. */
#define SP_SCORE_WORKSPACE_KEPT 2u   /* The caller promises that args->d_workspace was last written by
                                        an sp_score call with the same shape fields (B, T, N, L, H,
                                        H_kv, d, layer_reduce, paging) and SP_SCORE_EXCLUSIVE_DEVICE
                                        set that completed without SP_ETIMEOUT, and has not been
                                        touched since (not by sp_score_general or
                                        sp_score_pool_select either: they write it too).  A single-pass
                                        call leaves its exchange area ready for the next call, so
                                        the kernel that re-initialises it can then be skipped (a
                                        few microseconds per call in a serving loop that keeps its
                                        workspace).  The first call on a workspace, and the call
                                        after a time-out, must not set it.  Other kernels ignore
                                        it.  With a broken promise waits expire or scores are
                                        wrong. */

/* ---------------------------------------------------------------------------
 * sp_score: compute_attention_score + aggregate_attention_score (Algorithm 1),
 * i.e. for every prompt token i of sequence b
 *     s[l,h,n,i] = scale * <Q[l,b,n,h,:], K_l[i, h / (H/H_kv), :]>
 *     a[l,h,n,i] = exp(s[l,h,n,i] - logsumexp_{i' in sequence b} s[l,h,n,i'])   (Sec. 3.2 eq.)
 *     SP_LAYER_MAX : score[i] = mean_{n < n_valid[b]} max_{l,h} a               (Sec. 3.2.2)
 *     SP_LAYER_MEAN: score[i] = mean_{n < n_valid[b]} mean_l max_h a
 * The softmax runs over the prompt keys of the token's own sequence only.
 * Probabilities below 2^-126 (fp32's subnormal range) may count as 0.
 * Q and K are taken as stored by the draft model (already position-encoded) unless
 * rope_theta > 0 asks for the rotary encoding to be applied here.
 * --------------------------------------------------------------------------- */
typedef struct {
  int32_t B;                 /* sequences, >= 1                                           */
  int32_t N;                 /* query rows per sequence, 1..SP_MAX_QUERIES                */
  int32_t L;                 /* layers, 1..SP_MAX_LAYERS                                  */
  int32_t H;                 /* query heads                                               */
  int32_t H_kv;              /* key heads; H % H_kv == 0, H / H_kv <= 8                   */
  int32_t d;                 /* head dim: 64 or 128                                       */
  int64_t T;                 /* total prompt tokens = cu_seqlens[B], < 2^31               */
  const void* d_q;           /* bf16 [L, B, N, H, d] contiguous, 16-byte aligned          */
  const void* const* k_layers; /* HOST array of L device pointers; layer l holds bf16
                                  K_l[i, g, t] at element offset i*k_token_stride +
                                  g*k_head_stride + t (t contiguous); 16-byte aligned     */
  int64_t k_token_stride;    /* elements, multiple of 8                                   */
  int64_t k_head_stride;     /* elements, multiple of 8                                   */
  const int32_t* d_cu_seqlens; /* int32 [B+1], cu[0] = 0, non-decreasing, cu[B] = T       */
  const int32_t* d_n_valid;  /* int32 [B] with 1 <= n_valid[b] <= N, or NULL (= N): only the
                                first n_valid[b] query rows count (EOS validity, Sec. 3.3)  */
  float scale;               /* logit scale; the model's own attention uses 1/sqrt(d)     */
  int32_t layer_reduce;      /* sp_layer_reduce                                           */
  float rope_theta;          /* 0: Q and K are stored already position-encoded (what a serving
                                cache holds; the fast path).  > 0: Q and K are stored
                                un-rotated and are rotated here, rotate-half pairing
                                (t, t + d/2), angle pos * theta^(-2t/d): key i of a sequence
                                at position i, query row n of sequence b at d_q_pos[b*N+n];
                                cosine/sine in fp32 (angle formed in fp64), the two products
                                and their sum separate fp32 operations, rotated values
                                rounded to bf16 (nearest even): bit for bit what a cache
                                rotated that way would hold, then everything as for
                                rope_theta = 0.  Runs the two-pass kernels (the keys are
                                turned in registers on their way to the matrix cores; the
                                single-pass kernels take rotated caches only) and needs the
                                larger workspace the size query reports.                    */
  const int32_t* d_q_pos;    /* int32 [B, N] query positions if rope_theta > 0, else NULL  */
  float* d_scores;           /* out fp32 [T]                                              */
  float* d_lse;              /* out fp32 [L, B, N, H] row log-sum-exp, or NULL            */
  void* d_workspace;         /* device scratch, 256-byte aligned                          */
  size_t workspace_bytes;
  /* Paged K cache (Sec. 3.3: the draft's keys are fetched through the serving engine's slot
   * mapping).  d_block_table == NULL: token i of sequence b is row cu_seqlens[b] + i of every
   * layer, as described at k_layers.  Otherwise every layer is a pool of pages and token i of
   * sequence b is row (i % page_size) of page d_block_table[b*blocks_per_seq + i/page_size]:
   * element offset page*k_page_stride + (i % page_size)*k_token_stride + g*k_head_stride + t.
   * The table must cover every sequence and hold valid page numbers (not checked: a wrong
   * entry reads outside the pool).  Scores are still indexed by cu_seqlens[b] + i. */
  const int32_t* d_block_table; /* int32 [B, blocks_per_seq] page numbers, or NULL             */
  int32_t page_size;         /* tokens per page: a power of two >= 8 (ignored if not paged)   */
  int32_t blocks_per_seq;    /* row length of the table, >= 1                                 */
  int64_t k_page_stride;     /* elements, multiple of 8                                       */
  uint32_t flags;            /* SP_SCORE_* bits, 0 = none                                     */
  int32_t max_seqlen;        /* 0: nothing stated.  > 0: the caller's promise that no sequence has more
                                prompt tokens than this (the lengths themselves live on the device, where
                                the host side of sp_score cannot see them; with B == 1 the length is T and
                                nothing need be stated).  With it sp_score can take, for
                                batches of prompts of up to 8192 keys (4096 with 5..8 query rows per KV
                                head, 3072 with 9..32), a kernel that reads the K cache once and keeps all
                                logits of a sequence on chip.  (Rows: queries times the heads per KV head,
                                those counted as four up to four and as eight beyond.)  A sequence longer
                                than the kernel holds is not scored: all of its scores (and its rows of
                                d_lse) are NaN, which sp_pool_select reports in band; never silently
                                wrong.  Nothing else depends on the promise.                            */
  int32_t k_dtype;           /* sp_k_dtype, 0 = bf16.  With SP_K_FP8_E4M3 the layers hold bytes: the strides
                                (token, head, page) still count ELEMENTS and must then be multiples of 16;
                                rope_theta must be 0 (SP_EUNSUPPORTED otherwise).  The same kernels run as for a
                                bf16 cache (half the bytes per pass).                                    */
  const float* d_k_scale;    /* fp32 [L, H_kv] scales of an SP_K_FP8_E4M3 cache, finite, zero and negative ones
                                included, or NULL (all 1)                                                  */
} sp_score_args;

/* Bytes of workspace sp_score needs for these shapes (pointers are not read).
 * Returns 0 if the shape fields are invalid (flags and max_seqlen are shape fields here: they
 * decide which kernels run).  The size grows with T: per-tile row statistics
 * (L*N*H*8 bytes per 64 tokens) always, plus, for batches whose KV heads have at most eight
 * query rows (H/H_kv * N <= 8), 16 or 32 bytes per token, layer and KV head of logits kept
 * between the two passes (0.7 GB for 167K tokens of a 32-layer, 8-KV-head model), or, for the
 * kernels that take up to 32 rows, a result of 4 bytes per token and query for every run of
 * (layer, KV head) slabs the work is cut into (256 runs for one short prompt of a 32-layer, 8-KV-head
 * model, 16 for 32K tokens on an idle device; never more than there are slabs). */
SP_API size_t sp_score_workspace_bytes(const sp_score_args* args);

/* Enqueue the scoring on hip_stream.  Errors: SP_ENULL, SP_EINVAL (shape limits above),
 * SP_EALIGN, SP_EWORKSPACE, SP_ELAUNCH. */
SP_API sp_status sp_score(const sp_score_args* args, void* hip_stream);

/* Same contract and results as sp_score, but always runs the general two-pass kernels
 * (sp_score picks a faster single-pass kernel when the shape allows).  Meant for
 * cross-checking the two implementations of the Sec. 3.2 / 3.2.2 arithmetic. */
SP_API sp_status sp_score_general(const sp_score_args* args, void* hip_stream);

/* Optional post-check of the most recent sp_score call that used args->d_workspace.  The
 * single-pass kernels (SP_SCORE_EXCLUSIVE_DEVICE) exchange row statistics between workgroups
 * that must all be resident on the device at once.  Their waits are bounded: a workgroup whose
 * wait expired records the event in the workspace instead of hanging, and all of the call's scores
 * become NaN.  (Without the flag such a call has completed itself: SP_OK.)  This call SYNCHRONISES hip_stream (the only entry point that does), reads
 * that record and returns SP_ETIMEOUT if a wait expired, SP_OK otherwise.  Recovery: call
 * sp_score again without the flag (or sp_score_general). */
SP_API sp_status sp_score_check(const sp_score_args* args, void* hip_stream);

/* Upper bound on the polls a workgroup may spend waiting for other workgroups during one sp_score
 * call (process-wide, applies to later calls; default 65536, about 0.1 s; calls without
 * SP_SCORE_EXCLUSIVE_DEVICE also have a bound in time, see there).
 * 0 makes every wait give up at once, which turns every score of a single-pass call with that flag into
 * NaN, and takes one without it through its second launch: that is how the failure paths are
 * exercised without ever making a kernel hang.  Returns the previous value;
 * a negative argument only queries. */
SP_API int32_t sp_set_wait_budget(int32_t polls);

/* ---------------------------------------------------------------------------
 * sp_pool_select: chunk_select_from_smoothed_attention (Algorithm 1, Sec. 3.2.3).
 * Per sequence (length M): average-pool the scores with an odd window clipped to the
 * sequence (divisor = in-range count); split into ceil(M/chunk) contiguous chunks and
 * take each chunk's mean over its actual length; keep the
 * k = clamp(ceil(keep_rate * n_chunks - 1e-9), 1, n_chunks) best chunks (keep rate =
 * ratio of chunks, Sec. 4.1), equal scores resolved to the lower chunk index; emit the
 * tokens of the kept chunks in ascending order.  Arithmetic is fp64 on the fp32 input.
 * A NaN among the scores (sp_score writes NaN where a device-side wait expired) is reported
 * in band: cu_keep[0] = 0, cu_keep[1..B] = -1, and no kept index is written, so that neither
 * this call nor sp_gather after it hands on a keep set made from invalid scores.
 * --------------------------------------------------------------------------- */
typedef struct {
  int32_t B;
  int64_t T;
  const int32_t* d_cu_seqlens;  /* int32 [B+1]                                             */
  const float* d_scores;        /* fp32 [T]                                                */
  int32_t chunk;                /* >= 1                                                    */
  int32_t pool_window;          /* odd, >= 1 (1 = no smoothing)                            */
  double keep_rate;             /* in (0, 1]                                               */
  int32_t* d_kept_idx;          /* out int32 [kept_capacity]: flat token indices, ascending;
                                   entries at and beyond cu_keep[B] are left untouched     */
  int64_t kept_capacity;        /* >= number of kept tokens; T always suffices, see
                                   sp_keep_upper_bound.  Writes beyond it are suppressed.  */
  int32_t* d_cu_keep;           /* out int32 [B+1]: kept tokens of sequence b are
                                   kept_idx[cu_keep[b] .. cu_keep[b+1])                    */
  float* d_chunk_scores;        /* optional out fp32 [sum_b ceil(M_b/chunk)], NULL to skip */
  void* d_workspace;
  size_t workspace_bytes;
} sp_pool_select_args;

/* Host helper: an upper bound on the kept-token count from HOST sequence lengths
 * (sum over sequences of min(M_b, k_b * chunk)); -1 on invalid arguments. */
SP_API int64_t sp_keep_upper_bound(int32_t B, const int32_t* h_seqlens, int32_t chunk, double keep_rate);

SP_API size_t sp_pool_select_workspace_bytes(const sp_pool_select_args* args);
SP_API sp_status sp_pool_select(const sp_pool_select_args* args, void* hip_stream);

/* For callers that cannot allocate device memory (code under HIP-graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same operation and results as sp_pool_select, but
 * the scratch space is a fixed array inside the library's device image instead of a caller
 * workspace (d_workspace / workspace_bytes are ignored).  Limits: B <= SP_STATIC_MAX_SEQS and
 * T / chunk + B <= SP_STATIC_MAX_CHUNKS, else SP_EUNSUPPORTED.  Calls nothing that allocates.
 * Every call on one GPU shares that GPU's array: calls that overlap in time on one GPU race
 * (serialise them on one stream).  The array (SP_STATIC_SCRATCH_BYTES per GPU) lives until the
 * process ends. */
#define SP_STATIC_MAX_SEQS 4096
#define SP_STATIC_MAX_CHUNKS 131072
#define SP_STATIC_SCRATCH_BYTES (2u << 20)
SP_API sp_status sp_pool_select_static(const sp_pool_select_args* args, void* hip_stream);

/* ---------------------------------------------------------------------------
 * sp_score_pool_select: sp_score followed by sp_pool_select for ONE SHORT prompt, in a single
 * kernel launch (Sec. 3.2 equation, Sec. 3.2.2 and Sec. 3.2.3 in one go; the case of the paper's
 * variants without look-ahead on short contexts, Sec. 4.3, where the separate calls are bound by
 * their launches).  `score` and `select` are filled exactly as for the separate calls and must
 * describe the same prompt (select->B == score->B, select->T == score->T, select->d_scores ==
 * score->d_scores, select->d_cu_seqlens == score->d_cu_seqlens).  score->d_workspace must hold
 * sp_score_workspace_bytes(score) bytes as for sp_score (the logits pass through it; SP_EWORKSPACE
 * otherwise); select's workspace fields are ignored.  Outputs: everything the two calls write
 * (scores, optional lse, kept_idx, cu_keep, optional chunk_scores); scores agree with sp_score's
 * to the tolerance of fp32 summation order (probabilities below 2^-126, which sp_score may return as 0, keep their
 * subnormal values here), the selection is sp_pool_select's on these scores.
 * The workgroups of the launch never wait for one another (the last one to finish its share
 * completes the call), so nothing depends on what else runs on the device; they do count their
 * arrivals in one word per device, so two of these calls must not overlap on one GPU.
 * Supported: B == 1, 1 <= T <= 2048, H/H_kv * N <= 16, L * H * N <= 4096, rope_theta == 0, a bf16 cache, no
 * block table, at most 2048 chunks; anything else returns SP_EUNSUPPORTED and launches nothing (use the
 * separate calls).  The part after the logits is done by one workgroup: the call pays while
 * L * H * N * T stays small (a few layers of a few thousand keys); the separate calls, which use
 * the whole device throughout, overtake it beyond that.
 * --------------------------------------------------------------------------- */
SP_API sp_status sp_score_pool_select(const sp_score_args* score, const sp_pool_select_args* select, void* hip_stream);

/* ---------------------------------------------------------------------------
 * sp_gather: restore_pos_ids (Algorithm 1, Sec. 3.2.4) plus the gathers the base
 * model's prefill needs.  For kept slot s of sequence b:
 *     kept_pos[s]  = kept_idx[s] - cu_seqlens[b]      (position in the ORIGINAL prompt)
 *     kept_ids[s]  = token_ids[kept_idx[s]]
 *     out_embed[s] = embed[kept_ids[s], :]
 *     decode_pos[b] = M_b   (the first decoded token sits at the full prompt length)
 * Integer outputs and copied rows are exact.
 * --------------------------------------------------------------------------- */
typedef struct {
  int32_t B;
  const int32_t* d_cu_seqlens;  /* int32 [B+1]                                            */
  const int32_t* d_cu_keep;     /* int32 [B+1] from sp_pool_select                        */
  const int32_t* d_kept_idx;    /* int32 [>= cu_keep[B]]                                  */
  const int32_t* d_token_ids;   /* int32 [T], or NULL (then d_kept_ids/d_embed unused)    */
  const void* d_embed;          /* bf16 [V, D] row-major, 16-byte aligned, or NULL        */
  int32_t V;
  int32_t D;                    /* multiple of 8 when d_embed != NULL                     */
  int32_t* d_kept_ids;          /* out int32 [kept_capacity], NULL iff d_token_ids NULL   */
  int32_t* d_kept_pos;          /* out int32 [kept_capacity]                              */
  int32_t* d_decode_pos;        /* out int32 [B]                                          */
  void* d_out_embed;            /* out bf16 [kept_capacity, D] or NULL to skip the rows   */
  int64_t kept_capacity;        /* slots at and beyond min(cu_keep[B], capacity) untouched */
} sp_gather_args;

SP_API sp_status sp_gather(const sp_gather_args* args, void* hip_stream);

/* ---------------------------------------------------------------------------
 * The cache between the calls above and the two models: sp_cache_append fills it (the draft's, which sp_score reads,
 * or the base model's, whose prefill takes the kept tokens at their ORIGINAL positions, Sec. 3.2.4), sp_attend
 * attends over it.  Both work on one layer and take the cache as sp_score does:
 *   paged       d_block_table int32 [B, blocks_per_seq]; token i of sequence b is row i % page_size of page
 *               d_block_table[b*blocks_per_seq + i/page_size]: element offset page*cache_page_stride +
 *               (i % page_size)*cache_token_stride + g*cache_head_stride + t for KV head g; page_size a power of two >= 8
 *   contiguous  d_block_table NULL; token i of sequence b is row d_cu_cache[b] + i at row*cache_token_stride +
 *               g*cache_head_stride + t; sequence b owns the rows up to d_cu_cache[b+1] (int32 [B+1], non-decreasing)
 * Keys and values are two arrays of the same layout and type (sp_k_dtype); 8-bit elements stand for
 * scale[g] * decode(byte), one fp32 scale per KV head (finite) for the keys and one for the values, NULL = all 1.
 * n_rows is the number of token rows of the pool (pages * page_size) or of the contiguous cache.  Nothing outside it
 * is read or written, whatever the tables hold: a page number outside the pool or a row outside the cache is answered as
 * stated at each call.  New tokens of sequence b are rows [d_cu_new[b], d_cu_new[b+1]) of a flat axis with
 * room for T_new tokens (d_cu_new[0] = 0, non-decreasing, d_cu_new[B] <= T_new; rows at and beyond d_cu_new[B] are
 * neither read nor written).  Limits: d 64 or 128, H <= 1024, H % H_kv == 0,
 * H / H_kv <= 16, T_new * H < 2^31, T_new of an append <= 2^25.  With T_new = 0 the pointers to new tokens may be NULL.
 * Pointers to bf16 or 8-bit data are 16-byte aligned; strides count elements and are multiples of 8
 * (of an 8-bit cache: 16).
 * --------------------------------------------------------------------------- */

/* sp_cache_append: for new token j of sequence b (flat row t = cu_new[b] + j), at cache index i = cache_len[b] + j and
 * position p = pos[t] (NULL: p = i):
 *     q_out[t, h, :] = R_p(q[t, h, :]),   K[i, g, :] = R_p(k[t, g, :]),   V[i, g, :] = v[t, g, :]
 * R_p turns the pair (m, m + d/2) by the angle p * f_m, f_m = inv_freq[m] or rope_theta^(-2m/d): the angle in fp64, its
 * cosine and sine rounded to fp32, the products and their sum separate fp32 operations.  Results are rounded once: to
 * bf16 (nearest even), or divided by the scale in fp32 and rounded to E4M3 (nearest even; beyond +-448 the largest finite
 * value; NaN stays NaN; a scale of zero stores zeros).  A bf16 cache filled so holds bit for bit what
 * sp_score with rope_theta > 0 makes of an unrotated one.
 * A token whose cache index is negative or outside its sequence's room (blocks_per_seq * page_size tokens, or its rows of a
 * contiguous cache) or whose page number lies outside the pool is not written to the cache; its row of q_out is.
 * No two tokens of a call may have the same place in the cache: keys and values are different arrays, the cache's strides are at
 * least d where there are several heads, tokens or pages (SP_EINVAL), and its layout keeps all rows apart.  q_out, unless it is d_q itself, and the
 * cache overlap no input. */
typedef struct {
  int32_t B;                 /* sequences, >= 1                                                       */
  int32_t H;                 /* query heads (ignored if d_q is NULL)                                  */
  int32_t H_kv;              /* key and value heads                                                   */
  int32_t d;                 /* head dim: 64 or 128                                                   */
  int64_t T_new;             /* rows of q, k, v and q_out                                             */
  const void* d_q;           /* bf16 [T_new, H, d], any token and head strides, or NULL (keys and values only) */
  int64_t q_token_stride;
  int64_t q_head_stride;
  const void* d_k;           /* bf16 [T_new, H_kv, d], any token and head strides                     */
  int64_t k_token_stride;
  int64_t k_head_stride;
  const void* d_v;           /* bf16 [T_new, H_kv, d], any token and head strides                     */
  int64_t v_token_stride;
  int64_t v_head_stride;
  const int32_t* d_cu_new;   /* int32 [B+1]                                                           */
  const int32_t* d_cache_len;/* int32 [B]: tokens the cache holds before the call, or NULL (none)     */
  const int32_t* d_pos;      /* int32 [T_new] positions, or NULL; NULL without rotation               */
  float rope_theta;          /* > 0: frequencies theta^(-2m/d); 0: no rotation unless d_inv_freq      */
  const double* d_inv_freq;  /* fp64 [d/2] frequencies (scaled rotary encodings), or NULL; not with rope_theta > 0 */
  void* d_q_out;             /* out bf16 [T_new, H, d] contiguous, NULL iff d_q is; may be d_q itself if that is contiguous */
  void* d_k_cache;           /* out                                                                   */
  void* d_v_cache;           /* out                                                                   */
  int64_t cache_token_stride;
  int64_t cache_head_stride;
  int64_t cache_page_stride; /* (ignored if not paged)                                                */
  const int32_t* d_cu_cache; /* contiguous cache: int32 [B+1], else NULL                              */
  const int32_t* d_block_table; /* paged cache: int32 [B, blocks_per_seq], else NULL                  */
  int32_t page_size;         /* (ignored if not paged)                                                */
  int32_t blocks_per_seq;    /* (ignored if not paged)                                                */
  int64_t n_rows;            /* token rows of the cache, < 2^31                                       */
  int32_t cache_dtype;       /* sp_k_dtype                                                            */
  const float* d_k_scale;    /* fp32 [H_kv] of an 8-bit cache, or NULL (all 1)                        */
  const float* d_v_scale;    /* fp32 [H_kv] of an 8-bit cache, or NULL (all 1)                        */
} sp_cache_append_args;

/* Enqueue the append on hip_stream.  Needs no workspace. */
SP_API sp_status sp_cache_append(const sp_cache_append_args* args, void* hip_stream);

/* sp_attend: attention of the new tokens over the cache, causal.  Sequence b has kv_len[b] tokens in the cache, its
 * n_b new ones (appended before the call) the last of them, so new token j sees the first
 * n_vis = clamp(kv_len[b] - n_b + j + 1, 0, kv_len[b]) tokens.  For query head h and KV head g = h / (H/H_kv), t = cu_new[b] + j:
 *     s_i = scale * k_scale[g] * <q[t, h, :], K[i, g, :]>,  i < n_vis
 *     out[t, h, :] = sum_i softmax(s)_i * v_scale[g] * V[i, g, :]   (rounded once to bf16),   lse[t, h] = log sum_i exp(s_i)
 * A row that sees no token gets out = 0 and lse = -infinity.  Logits, maxima, sums and the accumulation of out are
 * fp32; the weights exp(s_i - m) are rounded to bf16 for the product with the values, as the values are.
 * NaN/Inf among the queries, or the keys and values of the first kv_len[b] tokens, are precondition violations
 * (undefined values in rows of that sequence, or of its group), and so are logits beyond fp32's range on the positive side; one that overflows to
 * -infinity has weight 0.  What lies behind the first kv_len[b] tokens in the cache is never used.
 *
 * Shared prefixes: sequences d_cu_group[g] .. d_cu_group[g+1]-1 form a group whose members hold the same first
 * d_prefix_len[g] tokens (the same pages, or copies).  Results are those of the definition; the keys and values of those
 * tokens are read through the FIRST member's block table, once for all members, where that pays.  A
 * prefix is cut to what every query of the group sees.  Paged caches only.
 *
 * Two calls: sp_attend_plan turns the lengths (which only the device knows) into the list of pieces of work, once per
 * step; sp_attend runs it, once per layer.  Both take the same struct; sp_attend_plan reads the shape fields and d_cu_new,
 * d_kv_len, d_cu_cache, d_cu_group, d_prefix_len and writes d_plan.  sp_attend may be given other queries, caches, scales,
 * outputs, strides and another workspace, but the shape fields B, H, H_kv, d, T_new, n_groups, page_size, blocks_per_seq,
 * n_rows, cache_dtype must be those of the plan, and whether it is paged: on a plan made for others, or on none,
 * every row of out and lse becomes NaN.  Lengths are those at the time of the plan.  A plan may be used by several
 * sp_attend calls at once if each has a workspace of its own.
 * Answered with NaN in out and lse: sequences whose kv_len is negative or beyond their room (all rows), and rows whose
 * part of the work met a page number outside the pool.
 * Limits: n_rows and blocks_per_seq * page_size <= 2^31 - 2^16, cache_token_stride < 2^26, and lists of work that one launch has
 * threads for (about T_new * H < 2^31 for prompts, B * H_kv < 2^23 for single tokens): SP_EINVAL beyond.
 * Rows of a contiguous cache are those that d_cu_cache names at the time of the plan.  d_out overlaps no input, and no two of its rows
 * overlap (strides below d, where there are several heads or rows: SP_EINVAL).
 * Both calls may be captured into graphs: nothing depends on lengths on the host. */
typedef struct {
  int32_t B;                 /* sequences, >= 1                                                       */
  int32_t H;                 /* query heads                                                           */
  int32_t H_kv;              /* key and value heads                                                   */
  int32_t d;                 /* head dim: 64 or 128                                                   */
  int64_t T_new;             /* rows of q, out and lse                                                */
  int32_t n_groups;          /* groups of sequences that share a prefix, 0: none                      */
  const int32_t* d_cu_new;   /* int32 [B+1]                                                           */
  const int32_t* d_kv_len;   /* int32 [B]: tokens in the cache, the new ones included                 */
  const int32_t* d_cu_group; /* int32 [n_groups+1] first sequences of the groups, 0 .. B, non-decreasing; NULL iff n_groups is 0 */
  const int32_t* d_prefix_len; /* int32 [n_groups] shared tokens, NULL iff n_groups is 0              */
  const int32_t* d_cu_cache; /* contiguous cache: int32 [B+1], else NULL                              */
  const int32_t* d_block_table; /* paged cache: int32 [B, blocks_per_seq], else NULL                  */
  int32_t page_size;         /* (ignored if not paged)                                                */
  int32_t blocks_per_seq;    /* (ignored if not paged)                                                */
  int64_t n_rows;            /* token rows of the cache                                               */
  int32_t cache_dtype;       /* sp_k_dtype                                                            */
  const void* d_q;           /* bf16 [T_new, H, d] (rotated), any token and head strides              */
  int64_t q_token_stride;
  int64_t q_head_stride;
  const void* d_k_cache;
  const void* d_v_cache;
  int64_t cache_token_stride;
  int64_t cache_head_stride;
  int64_t cache_page_stride; /* (ignored if not paged)                                                */
  const float* d_k_scale;    /* fp32 [H_kv] of an 8-bit cache, or NULL (all 1)                        */
  const float* d_v_scale;    /* fp32 [H_kv] of an 8-bit cache, or NULL (all 1)                        */
  float scale;               /* logit scale, finite, > 0                                              */
  void* d_out;               /* out bf16 [T_new, H, d], any token and head strides                    */
  int64_t out_token_stride;
  int64_t out_head_stride;
  float* d_lse;              /* out fp32 [T_new, H], or NULL                                          */
  void* d_plan;              /* 256-byte aligned                                                      */
  size_t plan_bytes;
  void* d_workspace;         /* 256-byte aligned; not read by sp_attend_plan                          */
  size_t workspace_bytes;
} sp_attend_args;

/* Bytes of d_plan and of d_workspace for the shape fields (pointers are not read); 0 if these are invalid. */
SP_API size_t sp_attend_plan_bytes(const sp_attend_args* args);
SP_API size_t sp_attend_workspace_bytes(const sp_attend_args* args);
SP_API sp_status sp_attend_plan(const sp_attend_args* args, void* hip_stream);
SP_API sp_status sp_attend(const sp_attend_args* args, void* hip_stream);

/* Static, never-NULL description of a status code. */
SP_API const char* sp_strerror(sp_status status);

/* Library version as major*10000 + minor*100 + patch. */
SP_API int32_t sp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SPECPREFILL_H */
