/*
 * sbw.h -- C ABI of the B200 (sm_100a) library for Stateless Bernoulli Watermarking (SBW).
 *
 * The library is the data-parallel hot path of the method: the per-decode-step logits bias
 * (Section 2.2, Eq. 1 and Eq. 2 of the paper), the same bias fused with temperature softmax and
 * Gumbel-max sampling, and batch detection (Section 2.2 "Detection", Eq. 5).  Every step runs
 * in hand-written CUDA kernels; there is no CPU fallback and no other backend.
 *
 * Conventions for every call
 *   - Pointers are DEVICE pointers owned by the caller unless a parameter says "host".
 *   - The library allocates nothing, frees nothing and never synchronises: work is enqueued on
 *     `stream` (a cudaStream_t passed as void*, NULL = the legacy default stream) and the call
 *     returns at once.  Scratch memory, where a call needs it, is passed in as `workspace`.
 *   - Return value: SBW_OK or a negative SBW_ERR_* code.  Nothing is enqueued when an argument
 *     is rejected.  After SBW_ERR_CUDA, sbw_last_cuda_error() returns the cudaError_t seen by
 *     the calling thread.  No exceptions, no exit(), no device-side traps.
 *   - Token ids are reinterpreted as unsigned 32-bit values; any bit pattern gives a
 *     deterministic result and is never used as an address.
 *   - B == 0 or N == 0 is SBW_OK and launches nothing.
 *
 * Readings taken where the paper names an operation without printing it ("SBW-spec v1"):
 *   Jenkins hash J      (Section 2.3)  a=(a+0x7ed55d16)+(a<<12); a=(a^0xc761c23c)^(a>>19);
 *                                      a=(a+0x165667b1)+(a<<5);  a=(a+0xd3a2646c)^(a<<9);
 *                                      a=(a+0xfd7046c5)+(a<<3);  a=(a^0xb55a4f09)^(a>>16)
 *   CBRNG               (Section 2.2)  x = word 0 of Philox4x32-10(counter (v,0,0,0),
 *                                      key (lo32 r, hi32 r)), v = vocab_offset + column
 *   green               (Eq. 1)        x < ceil(gamma * 2^32)   (strict, integer compare)
 *   seed r, CONTEXT     (Table 12, "additive")          r = key * (sum of the ctx ids)  mod 2^64
 *   seed r, SELFSALT    (Table 12, "anchored minhash";  r = key * J(v) * min(J(v), min_i J(ctx_i))
 *                        Section 5.2, every candidate)      mod 2^64, J(.)J(.) taken in 64 bits
 *   bias                (Eq. 2)        green: one round-to-nearest-even add of delta in the
 *                                      logits' precision (bf16: delta rounded to bf16 first);
 *                                      not green: value unchanged
 */
#ifndef SBW_H
#define SBW_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SBW_OK 0
#define SBW_ERR_INVALID_ARG (-1) /* null required pointer, size < 0, ld < V, gamma outside (0,1), ... */
#define SBW_ERR_UNSUPPORTED (-2) /* a value the ABI reserves but this build does not implement */
#define SBW_ERR_WORKSPACE (-3)   /* workspace missing, misaligned or too small */
#define SBW_ERR_CUDA (-4)        /* a CUDA runtime call failed; see sbw_last_cuda_error() */
#define SBW_ERR_TOO_LARGE (-5)   /* the problem exceeds a fixed built-in capacity (see the call) */

#define SBW_SCHEME_CONTEXT 0  /* seed from the preceding tokens only (SBW-1, SBW-4) */
#define SBW_SCHEME_SELFSALT 1 /* seed from the preceding tokens and the candidate (SBW-ss-V) */

#define SBW_DTYPE_F32 0  /* IEEE binary32 logits */
#define SBW_DTYPE_BF16 1 /* bfloat16 logits */

#define SBW_MAX_CTX_WIDTH 8

/* Library version string (static storage, host). */
const char *sbw_version(void);

/* cudaError_t recorded by the calling thread's last call that returned SBW_ERR_CUDA, else 0. */
int sbw_last_cuda_error(void);

/*
 * sbw_bias_logits -- Eq. 1 + Eq. 2, one decode step, in place, one pass, no mask tensor
 * (Section 5.1: in-place mutation, a single CBRNG evaluation per token, no CPU synchronisation).
 *
 *   logits       in/out, device, [B, ld] row-major, element type `dtype`; columns 0..V-1 of each
 *                row are biased, columns V..ld-1 are neither read nor written.  Any alignment is
 *                accepted; rows that start on 16-byte boundaries take the vectorised path.
 *   B, V, ld     rows, vocabulary columns, row stride in elements (ld >= V > 0, B >= 0).
 *   vocab_offset global id of column 0 (>= 0; non-zero when the vocabulary is sharded);
 *                vocab_offset + V may not exceed 2^32 (ids are 32-bit), else SBW_ERR_UNSUPPORTED.
 *   ctx_tokens   device, [B, ctx_width] int32: the ctx_width tokens preceding the one being
 *                generated, per row.  1 <= ctx_width <= SBW_MAX_CTX_WIDTH.
 *   key          64-bit secret key.      gamma  green fraction, 0 < gamma < 1.
 *   delta        bias added to green logits (any finite float; 0 leaves every bit unchanged).
 *   scheme       SBW_SCHEME_*.           stream cudaStream_t.
 * NaN logits stay NaN (payload unspecified); +-inf follow IEEE addition.
 */
int sbw_bias_logits(void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                    const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma,
                    float delta, int scheme, void *stream);

/*
 * sbw_bias_logits_topk -- the paper's SBW-ss scheme (Table 1: Bernoulli list, self-salt, candidates
 * "top-40"; Section 5.2 describes the top-k restriction it inherits from KGW): per row only the
 * top_k largest logits are tested (Eq. 1) and biased (Eq. 2); every other element of the row
 * keeps its bits.  "Largest" is the total order on order-encoded bit patterns -- +NaN > +inf >
 * ... > +0 > -0 > ... > -inf > -NaN -- with ties to the lowest column (the paper states no tie
 * rule).  Arguments as for sbw_bias_logits; top_k >= 1; top_k >= V is the full-vocabulary call.
 * Needs no workspace.  Fast for ordinary rows and top_k <= 256; rows of mostly equal values or
 * larger top_k take a slow, exact fallback (top_k block reductions per row).
 */
int sbw_bias_logits_topk(void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                         const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma,
                         float delta, int scheme, int64_t top_k, void *stream);

/*
 * sbw_bias_logits_host -- the same step for callers whose logits live in HOST memory: copies
 * B*ld elements and the context tokens to the device staging buffer, runs sbw_bias_logits on
 * it, and copies the logits back, all enqueued on `stream` (the copies are asynchronous only if
 * the host buffers are page-locked).  The paper has the logits on the GPU already; this entry
 * exists so that end-to-end cost including the PCIe transfers can be measured.
 *
 *   logits_host  in/out, HOST, [B, ld].        ctx_tokens_host  HOST, [B, ctx_width] int32.
 *   staging      device scratch of at least sbw_bias_logits_host_staging_bytes(...) bytes,
 *                256-byte aligned; owned by the caller, contents undefined afterwards.
 * The results are in logits_host once `stream` has been synchronised by the caller.
 */
size_t sbw_bias_logits_host_staging_bytes(int dtype, int64_t B, int64_t ld, int ctx_width);
int sbw_bias_logits_host(void *logits_host, int dtype, int64_t B, int64_t V, int64_t ld,
                         int64_t vocab_offset, const int32_t *ctx_tokens_host, int ctx_width,
                         uint64_t key, double gamma, float delta, int scheme, void *staging,
                         size_t staging_bytes, void *stream);

/*
 * sbw_bias_sample -- the bias of Eq. 1 + Eq. 2 fused with temperature softmax statistics and
 * Gumbel-max sampling, one pass over read-only logits.  The paper leaves sampling to the
 * serving engine (Section 5.1 speaks of absorbing the watermark into existing logit
 * post-processing); this call is that absorption.  Per row b, with l'_v the biased logit in the
 * logits' own precision and tau = temperature:
 *     m  = max_v l'_v                      Z = sum_v exp((l'_v - m) / tau)
 *     id = argmax_v fmaf(l'_v, 1/tau, g_v)  (fp32, 1/tau rounded once; ties -> lowest v)
 *     p  = exp((l'_id - m) / tau) / Z
 * g_v = -L(-L(u_v)) is a standard Gumbel variate from a counter-based stream of its own:
 *     y   = word (vg & 3) of Philox4x32-10(counter (vg >> 2, b, lo32 rng_step, hi32 rng_step),
 *           key (lo32 rng_seed, hi32 rng_seed)),  vg = vocab_offset + v
 *     u_v = ((y >> 9) + 0.5) * 2^-23
 * and L is a fixed fp32 logarithm made of exactly rounded operations (see sbw_sample.cu), so
 * that `out_tokens` is reproducible bit for bit on any IEEE machine.
 *
 *   logits        device, read only, [B, ld] of `dtype`.
 *   temperature   tau > 0.                 rng_seed, rng_step  select the Gumbel stream; use a
 *                 new rng_step for every decode step.
 *   out_tokens    device [B] int32: sampled column index (0-based within this shard).
 *   out_max, out_sumexp, out_prob   device [B] float, each may be NULL: m, Z, p.
 *   out_probs     device [B, V] float or NULL: the full softmax of the biased logits
 *                 (costs a second pass; meant for tests and small batches).
 *                 With all four NULL only the ids are produced, and the green test is evaluated
 *                 only for candidates whose Gumbel variate could make them win (same ids, about
 *                 twice the throughput).
 *   workspace     device scratch, 256-byte aligned, at least
 *                 sbw_sample_workspace_bytes(B, V) bytes; contents undefined afterwards.
 *                 Calls that share a workspace must not overlap on the GPU.
 * Rows whose logits are all -inf return id 0; m, Z, p of such rows, and every output of rows
 * that contain NaN or +inf, are unspecified.
 */
size_t sbw_sample_workspace_bytes(int64_t B, int64_t V);
int sbw_bias_sample(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                    int64_t vocab_offset, const int32_t *ctx_tokens, int ctx_width, uint64_t key,
                    double gamma, float delta, int scheme, float temperature, uint64_t rng_seed,
                    uint64_t rng_step, int32_t *out_tokens, float *out_max, float *out_sumexp,
                    float *out_prob, float *out_probs, void *workspace, size_t workspace_bytes,
                    void *stream);

/*
 * sbw_bias_sample_shard / sbw_sample_combine -- fused sampling of rows whose vocabulary is split
 * over S shards (tensor-parallel language-model heads).  The paper states that every device can
 * derive identical green lists from the shared key (Limitations) and leaves it unvalidated; with
 * these two calls no shard reads another shard's logits and 32 bytes per row and shard are all
 * that has to be exchanged.
 *
 * sbw_bias_sample_shard is sbw_bias_sample on one shard: `logits` holds columns vocab_offset ..
 * vocab_offset+V-1 of rows row_offset .. row_offset+B-1 (row_offset enters the Gumbel counter, so
 * a shard of the rows draws the same variates as the whole batch would; sbw_bias_sample uses 0).
 *   out_shard   device, 16-byte aligned, [B, 8] float: per row (m, Z, best score s, GLOBAL id of
 *               the best candidate as int bits, its biased logit, 0, 0, 0) of this shard.
 *   out_tokens  device [B] int32: the shard-local column of that candidate (required).
 *   vocab_offset + V may not exceed 2^31 here (the summary holds the global id as a signed
 *   32-bit value), else SBW_ERR_UNSUPPORTED.
 * sbw_sample_combine merges S such summaries laid out [S, B, 8] (shard-major, e.g. the result of
 * an all-gather): m = max m_r, Z = sum Z_r exp((m_r - m)/tau) in fp64, id = the global id with
 * the largest s (ties -> lowest global id), p = exp((l_id - m)/tau)/Z.  out_max / out_sumexp /
 * out_prob may be NULL.  The combined id, m, and (to 1e-6 relative) Z and p equal what
 * sbw_bias_sample returns on the unsplit rows.
 */
int sbw_bias_sample_shard(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                          int64_t vocab_offset, int64_t row_offset, const int32_t *ctx_tokens,
                          int ctx_width, uint64_t key, double gamma, float delta, int scheme,
                          float temperature, uint64_t rng_seed, uint64_t rng_step, float *out_shard,
                          int32_t *out_tokens, void *workspace, size_t workspace_bytes, void *stream);
int sbw_sample_combine(const float *shards, int64_t S, int64_t B, float temperature,
                       int32_t *out_tokens, float *out_max, float *out_sumexp, float *out_prob,
                       void *stream);

/*
 * sbw_bias_sample_shard_ids -- sbw_bias_sample_shard for callers that want the global ids only:
 * same arguments and summary layout, but the summary carries no statistics (m = -inf, Z = 0), so
 * the shard takes the ids-only path of sbw_bias_sample (the green test runs only for candidates
 * that could win).  sbw_sample_combine on such summaries gives the same out_tokens; its m, Z and
 * p outputs must then be NULL.
 */
int sbw_bias_sample_shard_ids(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                              int64_t vocab_offset, int64_t row_offset, const int32_t *ctx_tokens,
                              int ctx_width, uint64_t key, double gamma, float delta, int scheme,
                              float temperature, uint64_t rng_seed, uint64_t rng_step, float *out_shard,
                              int32_t *out_tokens, void *workspace, size_t workspace_bytes, void *stream);

/*
 * sbw_bias_sample_noalloc -- sbw_bias_sample for callers that cannot hand over a workspace.
 * The paper has no counterpart for this call; it exists for deployment.  Some users of this
 * library cannot allocate device memory at all: a logits processor plugged into a serving
 * engine that gave every free byte of the GPU to its KV-cache pool at start-up, or a component
 * that runs inside another process under a fixed memory budget.  For them cudaMalloc either
 * fails or stalls the whole device, so this variant needs none: the scratch that
 * sbw_bias_sample takes as `workspace` lives in a fixed array inside the library instead
 * (256 KiB of device memory, held by every GPU that loads the library until the process exits).
 *
 * Arguments and results are exactly those of sbw_bias_sample without `workspace` and
 * `workspace_bytes`; inputs and outputs are still the caller's.  Differences:
 *   - B may be at most SBW_NOALLOC_MAX_ROWS; a larger batch returns SBW_ERR_TOO_LARGE and
 *     enqueues nothing (split it, or use sbw_bias_sample).  The other arguments are checked
 *     first, so a call that is wrong in another way as well reports that.
 *   - The first call on each device looks up the array's device address (with that device
 *     current) before launching; make that first call outside any stream capture.
 *   - All calls on a device share the one array.  The library clears what has to start at zero
 *     on every call, but two calls that overlap on the GPU (different streams, no ordering
 *     between them) race on it and give undefined results: order them.
 * The call itself allocates nothing: no cudaMalloc, no cudaFree, no allocating library routine.
 */
#define SBW_NOALLOC_MAX_ROWS 4096
int sbw_bias_sample_noalloc(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                            int64_t vocab_offset, const int32_t *ctx_tokens, int ctx_width,
                            uint64_t key, double gamma, float delta, int scheme, float temperature,
                            uint64_t rng_seed, uint64_t rng_step, int32_t *out_tokens,
                            float *out_max, float *out_sumexp, float *out_prob, float *out_probs,
                            void *stream);

/*
 * sbw_detect -- batch detection (Section 2.2 "Detection": one membership test per token, no
 * green list is built; Eq. 5 for the score).  For sequence s with tokens t_0..t_{L-1}:
 *     scored positions  i = W .. L-1  (the first W = ctx_width tokens only seed), T = max(L-W, 0)
 *     Y_i = green(seed(t_{i-W..i-1}[, t_i]), v = t_i),   G = sum Y_i
 *     z   = (G - gamma T) / sqrt(T gamma (1 - gamma))     in fp64;  T = 0 gives G = 0, z = 0.
 *
 *   tokens        device, int32, the N sequences back to back (total_tokens ids).
 *   lengths       device [N] int32 (negative values count as 0).
 *   offsets       device [N+1] int64 start of each sequence in `tokens`, or NULL: the library
 *                 then scans `lengths` into the workspace first.
 *   total_tokens  number of ids in `tokens`; positions at or beyond it are never read, and a
 *                 sequence that would run past it is scored only up to it.
 *   out_counts    device [N] int32: G.    out_T  device [N] int32 or NULL: T.
 *   out_z         device [N] double: z.
 *   workspace     device scratch, 256-byte aligned, at least sbw_detect_workspace_bytes(N) bytes
 *                 (may be NULL with size 0 when `offsets` is given).
 */
size_t sbw_detect_workspace_bytes(int64_t N);
int sbw_detect(const int32_t *tokens, const int32_t *lengths, const int64_t *offsets, int64_t N,
               int64_t total_tokens, int ctx_width, uint64_t key, double gamma, int scheme,
               int32_t *out_counts, int32_t *out_T, double *out_z, void *workspace,
               size_t workspace_bytes, void *stream);

/*
 * sbw_detect_bits -- sbw_detect that also keeps the per-token indicators Y_i of Section 3 (the
 * paper's robustness study, Appendix G, scores cut and edited text; partly watermarked text needs
 * more than one count per sequence).  Arguments and results as for sbw_detect, plus
 *   out_bits   device, uint32[sbw_detect_bits_words(N, total_tokens)].  The bits of sequence s
 *              start at word (offset_s >> 5) + 2 s; scored position i (token W + i) is bit i & 31
 *              of word i >> 5 of that region; ceil(T / 32) words per sequence are written, unused
 *              high bits of the last one are 0, other words are left as they were.
 * When `offsets` is NULL the scanned int64[N + 1] offsets are left at the start of `workspace`,
 * where sbw_window_z can read them.
 *
 * sbw_window_z -- windowed detection on those bits: per sequence, the window of `window`
 * consecutive scored positions (all T of them if T < window) with the most green tokens, ties to
 * the earliest start, and Eq. 5 on that window.  T = 0 gives count 0, start 0, z 0.
 *   bits, lengths, offsets (required, device), total_tokens, ctx_width  as used by sbw_detect_bits.
 *   prefix_scratch  device, uint32[sbw_detect_bits_words(N, total_tokens)], contents undefined after.
 *   out_count, out_start  device [N] int32;  out_z  device [N] double.
 */
size_t sbw_detect_bits_words(int64_t N, int64_t total_tokens);
int sbw_detect_bits(const int32_t *tokens, const int32_t *lengths, const int64_t *offsets, int64_t N,
                    int64_t total_tokens, int ctx_width, uint64_t key, double gamma, int scheme,
                    int32_t *out_counts, int32_t *out_T, double *out_z, uint32_t *out_bits,
                    void *workspace, size_t workspace_bytes, void *stream);
int sbw_window_z(const uint32_t *bits, const int32_t *lengths, const int64_t *offsets, int64_t N,
                 int64_t total_tokens, int ctx_width, int64_t window, double gamma,
                 uint32_t *prefix_scratch, int32_t *out_count, int32_t *out_start, double *out_z,
                 void *stream);

/*
 * sbw_prefix_z -- detection on truncated text (the paper's robustness study, Appendix G, cuts
 * text to a prefix): Eq. 5 over the first keep[s] tokens of sequence s only, from the bits
 * sbw_detect_bits stored.  keep is clamped to [0, length]; T = max(keep - W, 0); T = 0 gives z 0.
 *   bits, lengths, offsets (required, device), total_tokens, ctx_width  as used by sbw_detect_bits.
 *   keep        device [N] int32.
 *   out_counts  device [N] int32;  out_T  device [N] int32 or NULL;  out_z  device [N] double.
 */
int sbw_prefix_z(const uint32_t *bits, const int32_t *lengths, const int64_t *offsets, const int32_t *keep,
                 int64_t N, int64_t total_tokens, int ctx_width, double gamma, int32_t *out_counts,
                 int32_t *out_T, double *out_z, void *stream);

/*
 * sbw_detect_unique -- sbw_detect that scores every distinct (context, token) tuple of a sequence
 * once (what KGW-family detectors call "ignore repeated n-grams"; Section 3 of the paper treats the
 * indicators Y_i as independent trials, which repeated text is not).  A scored position t counts
 * iff no earlier scored position of the same sequence has the same W + 1 tokens tok[t-W .. t];
 * out_T is the number of such positions, out_counts the green ones among them, out_z Eq. 5 on
 * the two.  Arguments as for sbw_detect, plus
 *   max_length  an upper bound on every length.  Sequences with more than 1536 scored tokens keep
 *               their hash set in the workspace; the workspace holds room for that only if
 *               max_length says such sequences exist.  A sequence longer than max_length that
 *               needs that room is not scored: count -1, T -1, z NaN.
 *   workspace   device, 256-byte aligned, at least
 *               sbw_detect_unique_workspace_bytes(N, total_tokens, max_length) bytes (always
 *               required; 16 bytes per token more when max_length > 1537).
 */
size_t sbw_detect_unique_workspace_bytes(int64_t N, int64_t total_tokens, int64_t max_length);
int sbw_detect_unique(const int32_t *tokens, const int32_t *lengths, const int64_t *offsets, int64_t N,
                      int64_t total_tokens, int64_t max_length, int ctx_width, uint64_t key, double gamma,
                      int scheme, int32_t *out_counts, int32_t *out_T, double *out_z, void *workspace,
                      size_t workspace_bytes, void *stream);

/*
 * sbw_roc_auc -- Section 4.3: area under the ROC curve of z-scores as a detector of label 1
 * (watermarked) against label 0, computed exactly as the pair statistic
 *   AUC = (2 #{z_pos > z_neg} + #{z_pos == z_neg}) / (2 n_pos n_neg),
 * which equals the trapezoid area under the (FPR, TPR) curve swept over every threshold.  NaN
 * scores are left out of both classes; -0 and +0 tie.
 *   z          device [n] double;  labels  device [n] uint8 (0 or non-zero);  n <= 2^31.
 *   out_auc    device double[1]; NaN when a class is empty.
 *   out_stats  device uint64[4] or NULL: {pairs greater, pairs equal, n_pos, n_neg}.
 *   workspace  device, 256-byte aligned, at least sbw_roc_auc_workspace_bytes(n) bytes.
 */
size_t sbw_roc_auc_workspace_bytes(int64_t n);
int sbw_roc_auc(const double *z, const uint8_t *labels, int64_t n, double *out_auc, uint64_t *out_stats,
                void *workspace, size_t workspace_bytes, void *stream);

/*
 * sbw_roc_auc_batched -- M independent ROC-AUCs in one launch (the paper's Table 4 holds one AUC per
 * configuration, each over 500 watermarked and 500 unmarked texts).  Problem i is the scores and
 * labels [offsets[i], offsets[i + 1]) of the flat arrays; each result is what sbw_roc_auc gives on
 * that slice.  One CTA per problem: meant for many problems of up to a few ten thousand scores.
 *   z, labels   device, flat;  offsets  device int64[M + 1], non-decreasing.
 *   out_auc     device double[M];  out_stats  device uint64[4 M] or NULL.
 * Needs no workspace.
 */
int sbw_roc_auc_batched(const double *z, const uint8_t *labels, const int64_t *offsets, int64_t M,
                        double *out_auc, uint64_t *out_stats, void *stream);

/*
 * sbw_bias_sample_filtered -- sbw_bias_sample on the top-k / top-p truncated distribution (the
 * paper's Appendix F samples with temperature 0.7 and top_p = 0.8; the paper gives no arithmetic
 * for the truncation, the one below is this library's).  Per row, with l' the biased logits of Eq. 2:
 *   order    candidates are ranked by order-encoded bit pattern, descending, ties to the lowest
 *            column (the order of sbw_bias_logits_topk); m is the first one's value.
 *   top_k    > 0 keeps the first min(top_k, V) of the order; 0 switches the filter off.
 *   top_p    < 1 keeps candidate i of what top_k left iff the integer weights of the candidates
 *            before it sum to S with S 2^32 < floor(top_p 2^32) Z, Z being the sum over all of
 *            them; >= 1 switches the filter off; must be > 0.  The weight of a candidate is 2^40
 *            for the bits of m, else with c = (float)(log2(e) / (double)temperature), y = (l' - m) c
 *            in fp32: 0 if not y >= -41, else trunc(2^(40 + n) P(y - n)), n = rintf(y), P the
 *            degree-7 Taylor polynomial of 2^f with coefficients rounded to fp32, evaluated by
 *            Horner's rule with fused multiply-adds.  The sums are exact, so the kept set does
 *            not depend on the order of addition.
 *   sample   arg max over the kept candidates of fmaf(l', 1 / temperature, g), g the Gumbel
 *            variate sbw_bias_sample draws for (rng_seed, rng_step, row, vocab_offset + column),
 *            ties to the lowest column.  With both filters off the ids equal sbw_bias_sample's.
 * Arguments as for sbw_bias_sample (logits are not modified), plus
 *   out_tokens  device [B] int32: the sampled column per row.
 *   out_kept    device [B] int32 or NULL: the number of candidates left per row.
 *   workspace   device, 256-byte aligned, at least sbw_sample_filtered_workspace_bytes(dtype, B, V)
 *               bytes (a biased copy of the logits); contents undefined afterwards.
 * With top_k set and 16-byte aligned rows the full-vocabulary hash is not evaluated: the columns that
 * can reach the biased top-k are found on the unbiased logits (l >= k-th largest l - |delta|) and only
 * they are hashed; the result is the same.
 * Rows that contain NaN are not supported (the result is some kept column).  V <= 2^21
 * (SBW_ERR_UNSUPPORTED beyond: the weight histogram's counters hold that many candidates).
 */
size_t sbw_sample_filtered_workspace_bytes(int dtype, int64_t B, int64_t V);
int sbw_bias_sample_filtered(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                             int64_t vocab_offset, const int32_t *ctx_tokens, int ctx_width, uint64_t key,
                             double gamma, float delta, int scheme, float temperature, int64_t top_k,
                             double top_p, uint64_t rng_seed, uint64_t rng_step, int32_t *out_tokens,
                             int32_t *out_kept, void *workspace, size_t workspace_bytes, void *stream);

/*
 * sbw_token_logprobs -- log probabilities of given tokens, with what goes with an answer: the
 * entropy of each row, the token's rank and the row's most probable alternatives, in one pass over
 * read-only logits and one launch.  (The paper scores texts by perplexity, Table 5; a server
 * returns these numbers beside the sampled tokens; an entropy-weighted detector takes the
 * entropies, see sbw_detect_weighted.)  Per row b, with l' the biased logits of Eq. 2 in the logits'
 * own precision -- the logits themselves where delta is 0 in it -- tau = temperature, t = tokens[b]:
 *     m = max_v l'_v        Z = sum_v exp((l'_v - m) / tau)        (as sbw_bias_sample returns them)
 *     log p_v = (l'_v - m) / tau - ln Z
 *     logprob = log p_t     entropy = - sum_v p_v log p_v  (in nats; 0 log 0 = 0)
 *     rank    = 1 + #{v : l'_v > l'_t} + #{v < t : l'_v = l'_t}
 *     alternatives: the top_n first columns by l' descending, ties to the lowest column (a token
 *     of rank r <= top_n is alternative r - 1), and their log p.
 * For this order -0 equals +0 and NaN counts as -inf.
 *
 *   logits, dtype, B, V, ld, vocab_offset, key, gamma, scheme   as for sbw_bias_sample; rows of any
 *                 alignment take the vectorised path.  vocab_offset only numbers the columns for
 *                 the hash: the probabilities are those over the V columns given, so a row has to hold
 *                 its whole vocabulary.  Vocabulary shards are not joined here, as
 *                 sbw_sample_combine joins them: a shard without the token would take its row for a padded one.
 *   ctx_tokens, ctx_width   as for sbw_bias_sample; ctx_tokens may be NULL where delta is 0.
 *   delta         0: no watermark (nothing is hashed).
 *   temperature   tau, 1e-6 .. 1e6 (SBW_ERR_INVALID_ARG beyond).
 *   tokens        device [B] int32 column indices (0-based, vocab_offset not added, as sbw_bias_sample
 *                 returns them), or NULL: no out_logprob and no out_rank then.  A token outside
 *                 [0, V) marks a padded row: its logits do not count, its outputs are 0, its
 *                 alternatives ids -1 with log probability -inf.
 *   top_n         0 .. SBW_MAX_TOP_LOGPROBS (SBW_ERR_TOO_LARGE beyond).  With top_n > V the places
 *                 from V on are id -1, log probability -inf.
 *   out_logprob, out_entropy, out_max, out_sumexp   device [B] float;  out_rank  device [B] int32;
 *   out_top_ids, out_top_logprobs   device [B, top_n] int32 / float.  Each may be NULL, not all.
 * A row whose logits are all -inf: every log p is -inf, entropy 0, m -inf, Z 0.  A row with a NaN or
 * +inf among its biased logits: logprob, entropy, m, Z and the alternatives' log p are NaN.
 * Statistics are fp32 sums of fp32 exponentials in chains of at most 39 additions, whatever V, joined in
 * fp64: log p is within 8e-6 + 2^-21 (H + |log p|) of its exact value, the entropy H within
 * 16e-6 (1 + H); a tenth of that is usual.  The order of a row's sums depends on B, V, dtype, the
 * scheme (or no watermark), whether top_n is 0, the row's address modulo 16 and the device's number of SMs, and on
 * nothing else: calls that are equal in these give equal bits, others may differ in the last ones.
 * No workspace; calls on different streams may overlap.  V <= 2^31 - 1.
 *
 * sbw_token_logprobs_backward -- the gradient of those log probabilities and entropies with respect
 * to the logits (straight through the watermark's addition: d l'_v / d l_v = 1):
 *     d_v = (1/tau) [ g (1[v = t] - p_v) - h p_v (log p_v + H) ],  g = grad_logprob[b], h = grad_entropy[b]
 * with p_v = exp((l'_v - m) / tau) / Z and H the saved entropy.
 *   max, sumexp, entropy   device [B] float: m, Z, H of the forward call (m and Z may come from
 *                 sbw_bias_sample too); entropy may be NULL where grad_entropy is.
 *   grad_logprob, grad_entropy   device [B] float; one of them may be NULL (0).  tokens may be NULL
 *                 where grad_logprob is.
 *   grad_logits   device [B, grad_ld] of `dtype`: every element of columns 0 .. V-1 is written, the
 *                 rest of a row is not; rounded once.  It may be `logits` itself (grad_ld = ld): the gradient then
 *                 takes the logits' place.  Any other overlap of the two is SBW_ERR_INVALID_ARG, and so are
 *                 rows that lie between each other's with different strides (they are not told apart).
 * Padded rows and rows whose logits are all -inf get zeros; rows with NaN or +inf get NaN.  p_v is an
 * fp32 exponential: relative error below 2^-21 + 2^-22 (m - l'_v) / tau (below 2^-126 it is 0).
 */
#define SBW_MAX_TOP_LOGPROBS 64
int sbw_token_logprobs(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                       const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma, float delta,
                       int scheme, float temperature, const int32_t *tokens, int64_t top_n,
                       float *out_logprob, float *out_entropy, int32_t *out_rank, float *out_max,
                       float *out_sumexp, int32_t *out_top_ids, float *out_top_logprobs, void *stream);
int sbw_token_logprobs_backward(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                                int64_t vocab_offset, const int32_t *ctx_tokens, int ctx_width, uint64_t key,
                                double gamma, float delta, int scheme, float temperature,
                                const int32_t *tokens, const float *max, const float *sumexp,
                                const float *entropy, const float *grad_logprob, const float *grad_entropy,
                                void *grad_logits, int64_t grad_ld, void *stream);

/*
 * sbw_detect_weighted -- sbw_detect with a weight per token (entropy-weighted detection: positions
 * where the model had a choice say more than positions where it had none; 0/1 weights score a
 * chosen part of a text).  Over the scored positions i of a sequence, with Y_i as for sbw_detect:
 *     G = sum w_i Y_i     S1 = sum w_i     S2 = sum w_i^2     (fp64)
 *     z = (G - gamma S1) / sqrt(S2 gamma (1 - gamma));  S2 = 0 gives z = 0.
 * With every weight 1 this is sbw_detect's z, bit for bit.
 *   weights     device [total_tokens] float, one per token of `tokens`, in its place; those of the
 *               first ctx_width tokens of a sequence are not read into any sum.  Any finite value; a
 *               NaN or an infinity among a sequence's scored weights makes its z NaN.
 *   out_green, out_weight, out_weight2   device [N] double: G, S1, S2; each may be NULL.
 *   out_z       device [N] double.
 * Other arguments, lengths, offsets and workspace as for sbw_detect
 * (sbw_detect_workspace_bytes(N) where offsets is NULL).  The order of the sums is fixed by N, the
 * lengths, total_tokens and the device's number of SMs: equal calls give equal bits.
 */
int sbw_detect_weighted(const int32_t *tokens, const float *weights, const int32_t *lengths,
                        const int64_t *offsets, int64_t N, int64_t total_tokens, int ctx_width, uint64_t key,
                        double gamma, int scheme, double *out_green, double *out_weight, double *out_weight2,
                        double *out_z, void *workspace, size_t workspace_bytes, void *stream);

/*
 * sbw_quantize_fp8 -- values to e4m3 (the finite 8-bit format with 4 exponent bits, largest value 448) with
 * one fp32 scale for each block of 128 columns: the form in which sbw_head_logits takes its operands.
 * Over the elements of a block, amax the largest magnitude:
 *     scale = max(amax / 448, 2^-126)      code = e4m3(x / scale)
 * (both divisions in fp32 and correctly rounded, the code rounded to nearest even and held within +-448; a zero keeps
 * its sign).  x is within half an e4m3 step of code * scale.  A block that holds a NaN or an infinity has a scale that
 * is not finite, and code times scale is NaN throughout it.
 *   x           device, [R, ld] of `dtype`, R >= 0 rows, K > 0 columns, ld >= K; any alignment of an element
 *               (rows that start on 16-byte boundaries, and on 8-byte ones in `out`, take the vectorised path).
 *   block_rows  1: a scale per row and 128 columns (hidden states).  128: a scale per 128 x 128 block (weights).
 *   out         device, [R, ld_out] bytes, ld_out >= K; columns K .. ld_out - 1 are not written.
 *   scales      device, [ceil(R / block_rows), ld_scales] float, ld_scales >= ceil(K / 128).
 * x, out and scales may not overlap.
 *
 * sbw_head_logits -- the projection of hidden states to the vocabulary, with the bias of Eq. 1 + Eq. 2 on the
 * way out (the paper's Section 5.1 speaks of absorbing the watermark into existing steps; this step makes the
 * logits).  With x and w in e4m3:
 *     l[b, v] = sum_kb x_scales[b, kb] w_scales[v / 128, kb] sum_{k in block kb} x[b, k] w[v, k]
 * summed in fp32 (a block's sum on the tensor cores, the blocks in order by fused multiply-add with the product
 * of the two scales), rounded once to `dtype`; green logits then get delta as in sbw_bias_logits: the result has
 * the bits of sbw_head_logits with delta 0 followed by sbw_bias_logits.
 *   x           device, [B, ld_x] e4m3 codes, 16-byte aligned, ld_x >= K a multiple of 16 (any from K on where B is 1);
 *               x_scales device [B, ld_x_scales] float, ld_x_scales >= ceil(K / 128).
 *   w           device, [V, ld_w] e4m3 codes, one row per vocabulary entry, aligned likewise;
 *               w_scales device [ceil(V / 128), ld_w_scales] float.
 *   logits      device, [B, ld] of `dtype`; columns 0 .. V-1 of every row are written, the others are not.
 *               It may not overlap the operands.
 *   delta       0: the plain product; ctx_tokens may be NULL then (and where delta is 0 in the logits' precision).
 *   vocab_offset, ctx_tokens, ctx_width, key, gamma, scheme   as for sbw_bias_logits (a shard of the vocabulary is a
 *               slice of w's rows that starts at a multiple of 128, with its first row's id in vocab_offset).
 * An e4m3 NaN or a scale that is not finite makes the logits that it enters NaN or infinite.  Equal calls give
 * equal bits; a row's logits do not depend on the other rows.  The gradient of the hidden states is the same product
 * with the transposed weights (codes and scales both transposed; blocks of 128 x 128 stay blocks):
 * d_x = d_l w, with d_l quantized in blocks of one row.  The caller makes and keeps the transposed copy.
 * A product of two scales beyond fp32's range is infinite or 0, as fp32 has it.
 * No workspace; calls on different streams may overlap.
 * The kernel hands tiles on inside each CTA.  A wait there that does not end within two seconds of running (which no
 * call is known to reach) gives up: the call still ends, the rest of that CTA's logits are NaN, and sbw_head_gave_up
 * counts the CTA.
 *
 * sbw_head_gave_up -- the number of CTAs in which such a wait gave up, on the current device since the library was
 * loaded: a number that grew over a call means that its logits are not whole.  (sbw_sample_given takes NaN as
 * -inf, so that it would draw from what is left.)
 *   out_ctas    host.  Waits for the work before it in `stream`; SBW_ERR_UNSUPPORTED while `stream` is captured.
 */
int sbw_quantize_fp8(const void *x, int dtype, int64_t R, int64_t K, int64_t ld, int64_t block_rows, void *out,
                     int64_t ld_out, float *scales, int64_t ld_scales, void *stream);
int sbw_head_logits(const void *x, int64_t ld_x, const float *x_scales, int64_t ld_x_scales, const void *w,
                    int64_t ld_w, const float *w_scales, int64_t ld_w_scales, int64_t B, int64_t V, int64_t K,
                    void *logits, int dtype, int64_t ld, int64_t vocab_offset, const int32_t *ctx_tokens,
                    int ctx_width, uint64_t key, double gamma, float delta, int scheme, void *stream);
int sbw_head_gave_up(uint64_t *out_ctas, void *stream);

/*
 * sbw_sample_given -- one token per row from a random number that the caller gives, with temperature, top-k, top-p
 * and min-p of its own for every row (a serving batch in which each request has its settings; random numbers from
 * the caller's generator, or shared with another sampler).  Per row b, with l' the biased logits of Eq. 2 in the logits' own
 * precision (the logits themselves where delta is 0 in it):
 *   order    candidates are ranked by value, descending, equal ones by column (-0 equals +0; NaN counts as -inf);
 *            m is the first one's value.
 *   weights  with tau = temperature[b], c = (float)(log2(e) / (double)tau), y = (l' - m) c in fp32: W = 0 if not
 *            y >= -41, else trunc(2^(40 + n) P(y - n)), n = rintf(y), P as in sbw_bias_sample_filtered (which has the
 *            same weights).  Sums of weights are exact.  A candidate of weight 0 is never kept.
 *   min_p    > 0 drops the candidates with y < (float)log2((double)min_p[b]) (values above 1 count as 1: what equals
 *            m stays).
 *   top_k    > 0 keeps the first top_k[b] of what is left.
 *   top_p    < 1 keeps a candidate of what is left then iff the weights before it sum to S with
 *            S 2^32 < max(1, floor(top_p[b] 2^32)) Z, Z being the sum over all of them.
 *   draw     with Z the sum over what is kept: the first kept candidate, in the order above, at which the running weight
 *            exceeds floor(u 2^32) Z / 2^32, u = uniforms[b] (values below 0 and NaN count as 0, values from 1 on as
 *            the largest number below).  u = 0 is the most probable candidate.
 * A temperature below 1e-6, or NaN, is greedy: the first candidate of the order.  A NaN among min_p or top_p switches
 * that filter off for its row, as do min_p <= 0, top_k <= 0 and top_p >= 1.
 *   logits, dtype, B, V, ld, vocab_offset, ctx_tokens, ctx_width, key, gamma, delta, scheme   as for
 *               sbw_token_logprobs (read only; rows of any alignment take the vectorised path; a row holds its whole
 *               vocabulary).  V <= 327680 (SBW_ERR_TOO_LARGE beyond).
 *   uniforms, temperature   device [B] float.
 *   top_k       device [B] int32;  top_p, min_p  device [B] float; each may be NULL: off for every row.
 *   out_tokens  device [B] int32: the column drawn.
 *   out_prob    device [B] float or NULL: its weight over Z (its probability among what is kept).
 *   out_kept    device [B] int32 or NULL: the number of candidates kept.
 * A row without a value above -inf: token 0, probability 0, kept 0.  +inf among the logits: those share the whole weight.
 * No workspace; calls on different streams may overlap.
 */
int sbw_sample_given(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                     const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma, float delta, int scheme,
                     const float *uniforms, const float *temperature, const int32_t *top_k, const float *top_p,
                     const float *min_p, int32_t *out_tokens, float *out_prob, int32_t *out_kept, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SBW_H */
