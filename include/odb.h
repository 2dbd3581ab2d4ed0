/* odb.h - C ABI of the MI355X (gfx950) block-decode / cache-refresh library.
 *
 * The library computes the model step of ODB-dLLM (arXiv 2511.21759):
 *   - odb_prefill: the full-sequence bidirectional forward that refreshes the
 *     K/V cache and yields a decoding attempt for every response position
 *     (Sec. 2.1 "DualCache" refresh; Sec. 4.1, first paragraph);
 *   - odb_block_step: the forward of S mutually invisible drafts of one
 *     response block against the cached K/V of every position outside the
 *     block, followed by the confidence-threshold acceptance
 *     (Sec. 3 Observation 3; Sec. 4.2 and Fig. 8 for the drafts);
 * and, built on those two, the paper's controllers: odb_predict_length (Sec. 4.1),
 * odb_accept_jump (Sec. 4.2.1) and its form for eight blocks, odb_speculative_jump,
 * odb_block_step_shared (Sec. 4.2.2) and the whole block-wise loop, odb_generate
 * (Sec. 2.1).
 *
 * Conventions
 *   - "dev" pointers are device (HBM) addresses on the current HIP device,
 *     "host" pointers are ordinary host memory.  The caller owns every buffer
 *     it passes; the library owns models, caches and its internal scratch.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Calls with a stream argument are asynchronous on it unless they say
 *     otherwise (odb_generate is synchronous): outputs are valid once the caller
 *     has synchronised the stream.  Calls that use the same model must be issued
 *     on one stream at a time (they share scratch).  A model's scratch grows with the largest call it has served
 *     and is freed with the model; beside the activations of that call it holds 32 MiB of partial sums for split
 *     projections, with many rows up to 96 MiB (16 bytes per row and channel; 32 MiB where more cannot be had).
 *     While a stream is captured into a graph scratch cannot grow (ODB_E_UNSUPPORTED: make the call once before);
 *     that of a captured call stays where it is when a larger call takes new scratch later.
 *   - Every function returns ODB_OK (0) or a negative ODB_E_* code; a message
 *     for the last failure on the calling thread is kept in odb_last_error().
 *     Arguments are validated on the host before any kernel is launched, so an
 *     invalid call launches nothing.
 *   - There is no CPU fallback: without a usable gfx950 device calls fail with
 *     ODB_E_HIP.
 */
#ifndef ODB_H
#define ODB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ODB_OK 0
#define ODB_E_INVALID_ARG (-1)
#define ODB_E_NOMEM (-2)
#define ODB_E_HIP (-3)
#define ODB_E_UNSUPPORTED (-4)
#define ODB_E_NO_PROGRESS (-5)   /* odb_generate: a decode step left the block's MASK count unchanged */

typedef struct odb_model odb_model;
typedef struct odb_cache odb_cache;

/* Architecture of the masked-diffusion transformer.  The paper names the LLaDA
 * 8B models (Sec. 5.1) without listing the architecture; this library fixes
 * pre-norm residual blocks, RMSNorm, rotate-half RoPE on the full head
 * dimension, SwiGLU, an untied LM head and no biases.
 * Requirements: d_model = n_heads*head_dim; head_dim is 64 or 128; d_model and
 * d_ff are multiples of 256; vocab is a multiple of 16; 0 <= mask_id < vocab. */
typedef struct {
    int n_layers, d_model, n_heads, head_dim, d_ff, vocab;
    float rope_base; /* pair j of a head turns by pos * rope_base^(-2j/head_dim) */
    float rms_eps;
    int mask_id;     /* token id of [MASK] */
} odb_config;

/* Optional device allocator (e.g. backed by torch.empty(device="cuda")).
 * alloc returns a device pointer aligned to 256 B or NULL. */
typedef struct {
    void *(*alloc)(size_t bytes, void *user);
    void (*free)(void *dev_ptr, void *user);
    void *user;
} odb_allocator;

/* Tensor ids for odb_model_set_tensor / odb_model_get_tensor.  Logical shapes
 * are row-major [out, in]: EMBED and LM [vocab, d]; WQ WK WV WO [d, d]; WG WU
 * [d_ff, d]; WD [d, d_ff]; the gains G1 (before attention), G2 (before the
 * MLP) and GF (before the LM head) are [d].  `layer` is ignored for EMBED, LM
 * and GF. */
enum {
    ODB_T_EMBED = 0, ODB_T_WQ, ODB_T_WK, ODB_T_WV, ODB_T_WO, ODB_T_WG, ODB_T_WU,
    ODB_T_WD, ODB_T_LM, ODB_T_G1, ODB_T_G2, ODB_T_GF, ODB_T_COUNT
};

/* Creates a model and allocates its weights in HBM (private tiled layout).
 * allocator may be NULL (hipMalloc/hipFree are used).  Weights are
 * uninitialised until odb_model_init_random or odb_model_set_tensor. */
int odb_model_create(const odb_config *cfg, const odb_allocator *allocator,
                     odb_model **out);
void odb_model_destroy(odb_model *m);

/* Fills every weight with bf16_rne(float(std * x)), x ~ N(0,1) drawn by the
 * counter-based generator below from the element's logical flat index, and
 * sets all gains to 1.  Element i of tensor t at layer l uses
 *   key = SM(SM(seed) + (t << 32 | l)),   z = SplitMix64 output i of state key,
 *   u1 = (hi32(z)+0.5)/2^32, u2 = (lo32(z)+0.5)/2^32,
 *   x = sqrt(-2 ln u1) cos(2 pi u2)   evaluated in binary64,
 * where SM(s) is the first SplitMix64 output for state s.  Asynchronous on
 * `stream`. */
int odb_model_init_random(odb_model *m, uint64_t seed, double std, void *stream);

/* Replaces / reads back one tensor as bf16 bit patterns in logical row-major
 * order (host memory, n = number of elements, must match the shape).
 * Synchronous.  Inside the library the projection matrices are held as IEEE
 * binary16, which represents every bf16 value of magnitude 2^-16 .. 65504
 * exactly; smaller magnitudes are rounded to a multiple of 2^-24 (an absolute
 * error below 3e-8).  A projection matrix with an element beyond that range (or
 * a NaN) is rejected with ODB_E_UNSUPPORTED and the model is left unchanged; the
 * embedding table and the gains are kept as given (bf16 / float). */
int odb_model_set_tensor(odb_model *m, int tensor_id, int layer,
                         const uint16_t *host_bf16, size_t n);
int odb_model_get_tensor(const odb_model *m, int tensor_id, int layer,
                         uint16_t *host_bf16, size_t n);

/* K/V cache for `batch` sequences of up to max_len positions: post-RoPE K and
 * V, two bytes per element (binary16), for every layer, head and position
 * (Sec. 2.1). */
int odb_cache_create(odb_model *m, int batch, int max_len, odb_cache **out);
void odb_cache_destroy(odb_cache *c);
/* Current sequence length set by the last odb_prefill (0 before). */
int odb_cache_length(const odb_cache *c);
/* Cuts the cached sequences to new_len positions (ODB-dLLM Sec. 4.1: the response is
 * truncated at the predicted end): positions new_len .. length-1 stop being keys of later
 * decode steps; the K/V of the kept positions stay as the last odb_prefill wrote them.
 * Host-side bookkeeping only; takes effect for calls issued afterwards.  Errors:
 * ODB_E_INVALID_ARG for a NULL cache or new_len outside [1, current length]. */
int odb_cache_truncate(odb_cache *c, int new_len);

/* Cache refresh (Sec. 2.1; Sec. 4.1).  tokens: dev int32 [batch, L], ids in
 * [0, vocab).  Runs the bidirectional forward over all L positions of every
 * sequence (positions 0..L-1), stores post-RoPE K and V of all of them in the
 * cache (its length becomes L) and writes, for response positions i >=
 * resp_off, conf (dev float [batch, L-resp_off]) = probability of the greedy
 * token and argmax (dev int32, same shape) = greedy token id, lowest id on
 * ties.  1 <= L <= max_len, 0 <= resp_off < L. */
int odb_prefill(odb_model *m, odb_cache *c, const int32_t *tokens_dev, int L,
                int resp_off, float *conf_dev, int32_t *argmax_dev, void *stream);

/* Block-decode step (Sec. 3 Obs. 3; Sec. 4.2).  drafts: dev int32
 * [batch, S, b]: S versions of the block at positions block_off ..
 * block_off+b-1 (all drafts share these position ids).  Each draft's b rows
 * attend to the cached K/V of positions outside the block and to the draft's
 * own fresh K/V; the cache entries at the block's positions are ignored and
 * the cache is not modified.  Outputs, all dev [batch, S, b]: conf (float),
 * argmax (int32) and unmask (uint8): 1 iff the draft holds mask_id there and
 * (conf > tau or the position is the draft's most confident masked position,
 * lowest index on ties).  Requires a prefilled cache, 0 <= block_off,
 * block_off + b <= cache length, 1 <= b <= 256, 1 <= S. */
int odb_block_step(odb_model *m, const odb_cache *c, const int32_t *drafts_dev,
                   int block_off, int b, int S, float tau, float *conf_dev,
                   int32_t *argmax_dev, uint8_t *unmask_dev, void *stream);

/* Run-time switches of a model.
 *   ODB_OPT_KSPLIT_REDUCE (default 1): workgroups of one launch may exchange partial sums, through
 *     device-scope stores and counters.  Projections with few rows and a long K split K over four
 *     workgroups of the streaming kernel, the last of which to arrive adds all sums in slice order and
 *     none of which waits.  Beyond 128 rows the blocks of a last round of workgroups may be shared by
 *     two each, the second of which waits inside the kernel for the sums of the first, a workgroup that
 *     already runs and waits for nobody.  Results do not depend on timing.
 *     0 routes these projections to kernels that exchange nothing inside a launch: the plain streaming
 *     kernel, the tile kernel with a separate reduction pass, or, beyond 128 rows, blocks of another
 *     shape.  Sums are then added in another order, in refreshes and steps alike.
 * Errors: ODB_E_INVALID_ARG for a NULL model, an unknown option or a value outside its range. */
enum { ODB_OPT_KSPLIT_REDUCE = 0 };
int odb_set_option(odb_model *m, int option, int value);

/* Synchronises the device, reads the model's status word and clears it.  Returns ODB_OK, or
 *   ODB_E_UNSUPPORTED  an activation left the binary16 range since the last check.  Between the
 *       kernels activations travel as binary16: Q, K, V, the SwiGLU output and, because the
 *       RMSNorm is folded into its neighbours, the un-normalised residual stream times the
 *       norm's gain, h[i] * g[i].  All of them must stay within +-65504 (for h * g that is a
 *       bound on the residual stream of the model, about 3e3 times what the 8B-shaped synthetic
 *       weights reach); a value beyond is clamped and flagged, as is a NaN.  Outputs of the
 *       calls since the last check are then not to be trusted;
 *   ODB_E_INVALID_ARG  odb_block_step_shared met a block with more MASK positions than n_masked. */
int odb_model_status(odb_model *m);

/* odb_block_step for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * kernels and same results as odb_block_step, but every intermediate buffer lives in a fixed
 * area of ODB_STATIC_SCRATCH_BYTES bytes that is part of the loaded library (one per GPU,
 * held until the process ends; 32 MiB beside it take the partial sums of split projections, so
 * that they are added in the order of odb_block_step); the call itself allocates and frees nothing.
 * A step whose rows need more than that area is rejected with ODB_E_UNSUPPORTED before
 * anything is launched (at the 8B shape of the paper's models, d = 4096, d_ff = 12288,
 * vocab = 126464, the area holds steps of up to 352 rows in blocks of 32).  All models on one GPU share the
 * area and every call overwrites what the last one left there: calls on one GPU that overlap
 * in time, on whatever streams or models, race; issue them one after the other on one
 * stream.  Other errors as odb_block_step. */
#define ODB_STATIC_SCRATCH_BYTES (32u << 20)
int odb_block_step_static(odb_model *m, const odb_cache *c, const int32_t *drafts_dev,
                          int block_off, int b, int S, float tau, float *conf_dev,
                          int32_t *argmax_dev, uint8_t *unmask_dev, void *stream);

/* Test-only variants that materialise the logits (dev float, row-major
 * [batch, L-resp_off, vocab] resp. [batch, S, b, vocab]) through an unfused
 * store instead of the fused confidence/argmax reduction. */
int odb_prefill_logits(odb_model *m, odb_cache *c, const int32_t *tokens_dev,
                       int L, int resp_off, float *logits_dev, void *stream);
int odb_block_step_logits(odb_model *m, const odb_cache *c,
                          const int32_t *drafts_dev, int block_off, int b, int S,
                          float *logits_dev, void *stream);

/* Adaptive length prediction after a refresh (ODB-dLLM Sec. 4.1).  The refresh's
 * decoding attempt (the conf / argmax that odb_prefill wrote for response positions
 * resp_off .. L-1) is scanned per sequence for [EOS]: the response as currently
 * drafted holds tokens[p] where position p is decoded and argmax where it still holds
 * the model's MASK id; an attempted [EOS] counts only if its confidence exceeds
 * truncate_thr (strictly), a decoded one counts as it stands.  new_len_dev[b] = index
 * of the earliest such position + 1 (the [EOS] stays the last position of the
 * sequence), or L when there is none.  The paper prints neither the threshold nor the
 * [EOS] id: both are arguments.
 *   tokens_dev  device int32 [batch, L]          the tokens the refresh ran on
 *   conf_dev    device float [batch, L-resp_off] \ outputs of odb_prefill
 *   argmax_dev  device int32 [batch, L-resp_off] /
 *   new_len_dev device int32 [batch]             written
 * Asynchronous on `stream`; all buffers are the caller's.  Errors: ODB_E_INVALID_ARG
 * for NULL pointers, batch < 1, L < 1, resp_off outside [0, L), eos_id outside
 * [0, vocab) or equal to the MASK id. */
int odb_predict_length(const odb_model *m, const int32_t *tokens_dev, const float *conf_dev,
                       const int32_t *argmax_dev, int batch, int L, int resp_off, int eos_id,
                       float truncate_thr, int32_t *new_len_dev, void *stream);

/* Decode step in the decoded-share stage (ODB-dLLM Sec. 4.2.2, Fig. 8 caption).
 * drafts_dev [batch, S, b] as for odb_block_step, with S >= 2 and b <= 64; the drafts of a
 * sequence must agree with its block_0 (draft 0) wherever block_0 holds a decoded token.
 * block_0 is forwarded in full, exactly as odb_block_step does it.  A speculative block
 * s >= 1 is reduced to the positions that block_0 still has MASKed (position ids kept); at
 * every layer its rows attend to the cached K/V outside the block, to block_0's fresh K/V
 * of the decoded positions, and to their own fresh K/V - not to other speculative blocks,
 * not to block_0's rows at masked positions.  So the decoded tokens are computed once per
 * step and the step has b + (S-1) * n_masked rows per sequence (each of the two parts
 * padded to a multiple of 16) instead of S * b.
 *   n_masked    host value: upper bound of the MASK positions in block_0 of any sequence
 *               (sets the row count; a block with more raises an error that
 *               odb_model_status reports as ODB_E_INVALID_ARG, its outputs are then invalid)
 *   conf_dev, argmax_dev, unmask_dev [batch, S, b] as for odb_block_step; for s >= 1 the
 *               entries at decoded positions are not computed and read conf 0,
 *               argmax = the token held there, unmask 0
 * Asynchronous on `stream`; does not modify the cache.  Errors as odb_block_step, plus
 * ODB_E_INVALID_ARG for b > 64, S outside [2, 64], n_masked outside [0, b]. */
int odb_block_step_shared(odb_model *m, const odb_cache *c, const int32_t *drafts_dev,
                          int block_off, int b, int S, int n_masked, float tau,
                          float *conf_dev, int32_t *argmax_dev, uint8_t *unmask_dev, void *stream);

/* Test aid: rows of a decoded-share step (block_0 of every sequence, padded to 16, then
 * per sequence its speculative blocks one after the other, together padded to 16), or a
 * negative error code. */
int odb_block_step_shared_rows(int batch, int b, int S, int n_masked);
/* Test aid: the logits of every row of the decoded-share step, float [rows, vocab], and for
 * every row its index into [batch, S, b] (-1 for padding rows), int32 [rows]; both device
 * buffers of the caller. */
int odb_block_step_shared_logits(odb_model *m, const odb_cache *c, const int32_t *drafts_dev,
                                 int block_off, int b, int S, int n_masked, float *logits_dev,
                                 int32_t *rowout_dev, void *stream);

/* Accept-jump controller (ODB-dLLM Sec. 4.2.1): decides which of the four drafts of
 * the last block step is adopted and builds the drafts of the next one, on the device.
 * The step ran on drafts[.,0] = block_0 (the block as it stood), [.,1] = block_0 with
 * candidate B unmasked beforehand, [.,2] = with candidate D, [.,3] = with both
 * (cand_pos / cand_tok: position inside the block and speculated token of B and D;
 * position -1 = no such candidate, as in the first step of a block).  A candidate is
 * verified in a draft when that draft's step unmasks its position with exactly the
 * speculated token.  Both verified in block_0: block_3 is adopted.  Only one: the draft
 * that had it unmasked beforehand is taken, and block_3 instead if the other candidate is
 * verified there.  Neither: block_0.  Adopting a draft = its tokens plus every position
 * its own step unmasked (with that step's greedy token); that is new_drafts[.,0].  The
 * next candidates are the two most confident positions of the adopted draft that are
 * still MASK afterwards (lower index first on equal confidence; -1 / token 0 if fewer
 * remain), their tokens that draft's greedy tokens, and new_drafts[.,1..3] unmask them.
 *   drafts_dev, argmax_dev  device int32 [batch, 4, b]     inputs / outputs of odb_block_step
 *   conf_dev device float [batch, 4, b], unmask_dev device uint8 [batch, 4, b]
 *   cand_pos_dev, cand_tok_dev       device int32 [batch, 2]
 *   chosen_dev device int32 [batch] (0..3), new_drafts_dev device int32 [batch, 4, b],
 *   new_cand_pos_dev, new_cand_tok_dev device int32 [batch, 2]             written
 * Output buffers must not overlap input buffers.  Asynchronous on `stream`; all buffers
 * are the caller's.  Errors: ODB_E_INVALID_ARG for NULL pointers, batch < 1, b < 1. */
int odb_accept_jump(const odb_model *m, const int32_t *drafts_dev, const float *conf_dev,
                    const int32_t *argmax_dev, const uint8_t *unmask_dev,
                    const int32_t *cand_pos_dev, const int32_t *cand_tok_dev, int batch, int b,
                    int32_t *chosen_dev, int32_t *new_drafts_dev, int32_t *new_cand_pos_dev,
                    int32_t *new_cand_tok_dev, void *stream);

/* The jump rule over the S = 4 or 8 blocks of a step (ODB-dLLM Sec. 4.2.1, carried over to the
 * eight blocks of Sec. 4.2.2; the paper states the rule for the two candidates B and D only).
 * With the candidates ranked by confidence, block s holds the block with these candidates
 * unmasked beforehand: s = 0 none, 1 {B}, 2 {D}, 3 {B, D}, 4 {third}, 5 {B, D, third},
 * 6 {fourth}, 7 {all four}.  The walk starts at block_0.  At a block with candidate set X the
 * verified set is X plus every other candidate whose position this block's own step unmasks
 * with exactly the speculated token; the block whose set lies strictly above X inside the
 * verified set and holds the most candidates (the lowest number among equals) is visited
 * next, and the block at which no such block exists is adopted.  For S = 4 this is the rule
 * of odb_accept_jump.  The adopted block plus every position its own step unmasked is
 * new_drafts[.,0]; the n_next / 2 most confident positions still MASK there (lower index
 * first on equal confidence; -1 / token 0 where fewer remain, and in the entries behind
 * n_next / 2) are the next candidates and new_drafts[.,1 .. n_next) the blocks built on them.
 *   drafts_dev, argmax_dev  device int32 [batch, S, b]; conf_dev float, unmask_dev uint8, same shape
 *   cand_pos_dev, cand_tok_dev  device int32 [batch, 4] (the first S / 2 are read)
 *   chosen_dev device int32 [batch], new_drafts_dev device int32 [batch, n_next, b],
 *   new_cand_pos_dev, new_cand_tok_dev device int32 [batch, 4]                 written
 * Output buffers must not overlap input buffers.  Asynchronous on `stream`; all buffers are
 * the caller's.  Errors: ODB_E_INVALID_ARG for NULL pointers, batch < 1, b < 1, S or n_next
 * other than 4 and 8. */
int odb_speculative_jump(const odb_model *m, const int32_t *drafts_dev, const float *conf_dev,
                         const int32_t *argmax_dev, const uint8_t *unmask_dev,
                         const int32_t *cand_pos_dev, const int32_t *cand_tok_dev, int batch, int b,
                         int S, int n_next, int32_t *chosen_dev, int32_t *new_drafts_dev,
                         int32_t *new_cand_pos_dev, int32_t *new_cand_tok_dev, void *stream);

/* Block-wise generation of one response (ODB-dLLM Sec. 2.1, with the adaptive length
 * prediction of Sec. 4.1 and the jump-share decoding of Sec. 4.2 switched on by the
 * parameters).  The host loop is the library's; every decision is taken by kernels and the
 * host reads back sixteen 32-bit words per forward.
 *
 * The response starts as resp_len MASK tokens behind the prompt and is decoded block by
 * block, front to back.  A block cycle opens with a refresh (odb_prefill over the whole
 * sequence: the cache is rebuilt and every response position attempted).  Then
 *   1. if eos_id >= 0, the attempt is scanned as odb_predict_length does and the sequence
 *      is cut at once: dropped positions leave the token sequence and, as for
 *      odb_cache_truncate, stop being keys of this cycle's steps;
 *   2. the attempt at the current block goes through the acceptance rule of odb_block_step
 *      (MASK positions whose confidence exceeds tau, and always the most confident one), so
 *      the refresh is also the block's first decoding iteration;
 *   3. decode steps follow until the block holds no MASK.  n_drafts = 1: odb_block_step on
 *      the block alone.  n_drafts = 4: the four accept-jump drafts and odb_accept_jump (the
 *      first candidates are the two most confident positions the refresh left MASKed); once
 *      share_from positions of the block are decoded the step is odb_block_step_shared
 *      on the same four drafts.  n_drafts = 8 (needs share_from >= 0): as n_drafts = 4 until
 *      share_from positions are decoded, then odb_block_step_shared on eight blocks - the four
 *      most confident positions left MASKed are the candidates (Sec. 4.2.2: the third, the top
 *      three, the fourth and the top four join B, D and B + D) - and odb_speculative_jump;
 *      with row_budget > 0 a step of that stage whose eight blocks would come to more rows
 *      runs on the four accept-jump blocks instead.
 *      A step that leaves the block's MASK count unchanged (an untrained model may attempt
 *      the MASK token itself) ends the call with ODB_E_NO_PROGRESS rather than repeating for ever.
 * Generation ends when the next block would start at or behind the end of the sequence.
 * None of the parameter values is printed in the paper.
 *
 *   tokens_dev  device int32 [prompt_len + resp_len]; the caller fills the prompt, the call
 *               writes the MASKs and then the decoded tokens; positions behind the final
 *               length are left as they were when they were cut
 *   c           a cache for batch 1 with max_len >= prompt_len + resp_len; left holding the
 *               last refresh, cut to the final length
 *   stats       host, written (counts, lengths, host wall-clock of the two phases)
 *   events      host array of max_events records or NULL: one record per forward, in order
 *   event_tokens_dev  device int32 [max_events, prompt_len + resp_len] or NULL: the token
 *               sequence after every forward (test aid; costs one device copy per forward)
 * Synchronous: returns after the last forward has finished; the stream is synchronised
 * once per forward.  Working buffers come from the model's allocator and are released
 * before returning.  Errors: ODB_E_INVALID_ARG for NULL handles / tokens / params / stats,
 * prompt_len < 1, resp_len < 1, a cache of batch != 1 or too short, block_len outside
 * [1, 256] (or > 64 with share_from >= 0), n_drafts other than 1, 4 and 8 (or 8 with
 * share_from < 0), eos_id >= vocab or
 * equal to the MASK id; more than max_events forwards stop being recorded (stats.n_events
 * still counts them).  On an error of an inner call its code is returned and tokens_dev is
 * left partly decoded. */
enum { ODB_EV_REFRESH = 0, ODB_EV_STEP = 1, ODB_EV_STEP_SHARED = 2 };
typedef struct {
    int block_len;        /* positions per block (32 in the paper's runs) */
    int n_drafts;         /* 1: threshold decoding; 4: accept-jump (Sec. 4.2.1); 8: accept-jump, then
                             eight blocks in the decoded-share stage (Sec. 4.2.2) */
    float tau;            /* acceptance threshold */
    int eos_id;           /* < 0: no length prediction */
    float truncate_thr;   /* Sec. 4.1 */
    int share_from;       /* decoded positions of the block from which steps run in the
                             decoded-share stage (Sec. 4.2.2); < 0: never */
    int row_budget;       /* n_drafts = 8: a decoded-share step forwards eight blocks only if its
                             block_len + 7 * masked rows fit this budget, else the four accept-jump
                             blocks (Sec. 4.2: the step has to stay memory-bound; Sec. 4.2.2: the
                             shrinking blocks make room for the extra candidates); <= 0: always eight */
} odb_generate_params;
typedef struct {
    int kind;             /* ODB_EV_* */
    int length;           /* sequence length after the event */
    int block_off, block_len;   /* block_len 0: the cut fell into what was already decoded */
    int chosen;           /* adopted draft (0 for a refresh and for n_drafts = 1) */
    int n_masked;         /* MASK positions left in the block */
    int cand_pos[4], cand_tok[4];   /* the candidates handed to the next step, best first (-1 / 0:
                                       none; n_drafts < 8 uses two) */
} odb_generate_event;
typedef struct {
    int n_refresh, n_step, n_step_shared, final_len, n_events;
    long long refresh_positions;    /* sum of the refreshed lengths */
    long long step_rows;            /* rows forwarded by the steps (padding not counted) */
    double refresh_ms, step_ms, total_ms;   /* host wall-clock, each phase up to its read-back */
} odb_generate_stats;
int odb_generate(odb_model *m, odb_cache *c, int32_t *tokens_dev, int prompt_len, int resp_len,
                 const odb_generate_params *params, odb_generate_stats *stats,
                 odb_generate_event *events, int32_t *event_tokens_dev, int max_events,
                 void *stream);

/* ---- Paged K/V: requests of different lengths share a pool of pages ------------------------------------------
 * The cache above holds sequences of one length.  Where requests of different lengths come, grow by blocks and are
 * cut behind a predicted end (odb_predict_length), K/V live in pages: a page holds page_size consecutive positions of
 * every K/V head of one layer, and a request's row of `tables` names its pages in order.  The caller owns all memory.
 * These calls need no model and run on the current device.  They allocate and synchronise nothing, so they can be
 * captured into a graph; several may run at once as long as what one writes no other reads or writes.
 * What they read from device memory (lengths, tables, slots, positions) is checked there: an entry outside its
 * range is taken as said below and never leads outside the buffers described. */
enum { ODB_F16 = 0, ODB_BF16 = 1, ODB_F32 = 2 };

/* The pool of one layer: element (page, head, position inside the page, channel) of k and of v lies at
 * page * page_stride + head * head_stride + position * pos_stride + channel elements.
 * Requirements: page_size a power of two from 16 to 4096; head_dim 64, 128 or 256; dtype ODB_F16 or ODB_BF16; strides
 * not negative and multiples of 8, pos_stride below 2^24; k and v aligned to 16 bytes; n_pages * page_size < 2^31. */
typedef struct {
    void *k, *v;          /* dev */
    int n_pages, page_size, n_kv_heads, head_dim, dtype;
    long long page_stride, head_stride, pos_stride;
} odb_pages;

/* Page tables and slot maps of a step, from the requests' lengths.  For request r (of n, 1 to 4096): held[r] positions own
 * pages so far, wanted[r] shall.  A request that wants fewer gives its last pages back, which go on top of the stack
 * free_pages (in order of the requests); then those that want more take pages off its top, again in order.  A request is
 * refused, and keeps what it holds, if the pages taken by it and all before it exceed those that are there (so that after
 * the first refused one no other gets pages either), or if wanted[r] is negative or beyond columns * page_size.
 *   held, wanted   dev int32 [n]; held is clamped to [0, columns * page_size]
 *   tables         dev int32 [n, columns], read and written: entries of pages that were taken; all others stay as they are
 *   free_pages     dev int32 [n_pages], read and written; n_free dev int32 [1]: how many of its entries are free pages
 *   row_first, row_count   dev int32 [n]: the positions that the step computes, row_count[r] of them from row_first[r] on;
 *                  either may be NULL: held[r], and wanted[r] - held[r] (none where that is negative or wanted[r] no length of the table)
 * written:
 *   len            dev int32 [n]: wanted[r], or held[r] where refused
 *   cu_rows        dev int32 [n + 1]: rows in front of each request; all are capped at rows_cap
 *   slots, positions   dev int32 [rows_cap]: for every row its position and its slot, page * page_size + position inside the
 *                  page; -1 where the position lies outside [0, len[r]) or its page outside the pool.  Entries behind the last row stay:
 *                  those of an earlier, longer step, say.  Where such a step's whole buffers go on, cu_rows + n is the row_end of
 *                  odb_qk_norm_rope.
 *   state          dev int32 [4]: free pages afterwards (the next call's n_free), pages taken, given back, requests refused
 * Pages are not counted: one that several tables name (a prefix that requests share) is given back as often as requests that
 * hold it get shorter, so shared pages are kept out of what is given back.
 * The same call with the same inputs writes the same values again.  Buffers must not overlap.  Asynchronous on `stream`.
 * Errors: ODB_E_INVALID_ARG for NULL buffers, n outside [1, 4096], columns < 1, columns * page_size > 2^30, rows_cap outside
 * [1, 2^24], n_pages < 1, a page size or a pool outside the requirements above, or buffers that overlap. */
int odb_page_tables(const int32_t *held_dev, const int32_t *wanted_dev, int n, int page_size, int32_t *tables_dev,
                    int columns, int32_t *free_pages_dev, int n_pages, const int32_t *n_free_dev,
                    const int32_t *row_first_dev, const int32_t *row_count_dev, int32_t *len_dev,
                    int32_t *cu_rows_dev, int32_t *slots_dev, int32_t *positions_dev, int rows_cap,
                    int32_t *state_dev, void *stream);

/* Rotary angles.  Pair j of rot_dim / 2 turns by p * f_j at position p, f_j = base^(-2j/rot_dim), and for contexts longer than
 * the original one
 *   ODB_ROPE_LINEAR  f_j / factor
 *   ODB_ROPE_NTK     base * factor^(rot_dim / (rot_dim - 2)) instead of base (rot_dim = 2: unchanged)
 *   ODB_ROPE_YARN    f_j (w + (1 - w) / factor), w = (original_len * f_j / 2 pi - beta_slow) / (beta_fast - beta_slow)
 *                    clamped to [0, 1] (YaRN, arXiv 2309.00071: by the turns that a pair makes in the original context; a ramp over
 *                    the pairs' numbers between two bounds, as some configurations have it, is not expressed so) */
enum { ODB_ROPE_PLAIN = 0, ODB_ROPE_LINEAR, ODB_ROPE_NTK, ODB_ROPE_YARN };
typedef struct {
    double base;
    int scaling;
    double factor;                  /* >= 1; ignored by ODB_ROPE_PLAIN */
    int original_len;               /* ODB_ROPE_YARN: positions of the original context */
    double beta_fast, beta_slow;    /* ODB_ROPE_YARN: 32 and 1 in the paper */
    double magnitude;               /* cosines and sines are multiplied by it; 0: 0.1 ln(factor) + 1 for YARN, else 1 */
} odb_rope;

/* table[p][j] = (cos, sin) of pair j at position p, dev float [n_pos, rot_dim / 2, 2]; rounded once from 64 bits.
 * Asynchronous on `stream`.  Errors: ODB_E_INVALID_ARG for NULL, n_pos outside [1, 2^22], rot_dim odd or outside [2, 256],
 * base <= 1, factor < 1, beta_fast <= beta_slow, beta_slow < 0, original_len < 1, a negative magnitude, numbers that are not finite. */
int odb_rope_table(float *table_dev, int n_pos, int rot_dim, const odb_rope *rope, void *stream);

/* Norms and rotation of queries and keys, K/V to their pages, in one pass over the projection's output.  For every row:
 * q and k of each head are divided by their root mean square, sqrt(mean of squares + eps), and multiplied by the gain
 * (skipped where the gain is NULL); then the first rot_dim channels of each head turn by the angles of the row's
 * position: pairs are (j, j + rot_dim / 2), or with `interleaved` (2j, 2j + 1).  Queries go to q_out, keys and values to the
 * row's slot.  All in 32 bits with one rounding at the end, to an infinity beyond the type's range.
 *   q [rows, n_heads, head_dim], k, v [rows, n_kv_heads, head_dim]: dev, in_dtype ODB_F32 or the pages' dtype; the heads of a
 *       row follow each other, rows are q_row, k_row, v_row elements apart (three parts of one buffer, say)
 *   table       dev float [n_pos, rot_dim / 2, 2] as odb_rope_table writes it
 *   positions, slots   dev int32 [rows].  A position outside [0, n_pos) marks a padding row: its queries become zero, nothing
 *               is stored.  A slot outside the pool stores nothing.  Slots must differ: of two rows with the same slot
 *               either's values may remain, piece by piece.
 *   q_out       dev [rows, n_heads, head_dim] of the pages' dtype, rows q_out_row elements apart; may be q itself
 *               (same dtype and stride; k and v then lie beside it, between its rows only with its stride), otherwise its
 *               range, from the first row's beginning to the last one's end, must not overlap those of q, k and v
 *   row_end     dev int32 [1] or NULL: rows from this one on are padding rows, whatever their positions and slots (a captured step of
 *               fixed size whose number of rows is known on the device alone)
 * Requirements: buffers aligned to 16 bytes, row strides multiples of 8, rot_dim a multiple of 16 in [16, head_dim].
 * Asynchronous on `stream`.  rows = 0 launches nothing.  Errors: ODB_E_INVALID_ARG, also where rows * ceil((n_heads + 2 n_kv_heads)
 * * head_dim / 1024) reaches 2^26. */
typedef struct {
    const void *q, *k, *v;
    int in_dtype, rows, n_heads;
    long long q_row, k_row, v_row;
    const float *q_gain, *k_gain;   /* dev [head_dim] each, or both NULL */
    float eps;
    const float *table;
    int n_pos, rot_dim, interleaved;
    const int32_t *positions, *slots;
    void *q_out;
    long long q_out_row;
    const int32_t *row_end;
} odb_qk_rows;
int odb_qk_norm_rope(const odb_qk_rows *rows, const odb_pages *pages, void *stream);

/* Attention of new rows over their requests' pages: out = softmax(scale * q k^T over the visible keys) v.
 * Request r has rows cu_rows[r] .. cu_rows[r + 1] - 1 at positions first_pos[r], first_pos[r] + 1, ...; a row at position p
 * sees key i (whatever the pages hold there, the rows' own K/V included once they are stored) iff
 *   i < kv_len[r],  and with causal i <= p,  and with window > 0  |p - i| < window or i < sinks.
 * A row that sees no key becomes zero.  What lies at positions that a row does not see has no influence on it, not even
 * if it is infinite or no number; a key whose score is minus infinity counts as one that is not seen.  Query head h reads K/V head h / (n_heads / n_kv_heads).
 *   q, out   dev [rows, n_heads, head_dim] of the pages' dtype, rows q_row / out_row elements apart
 *   cu_rows  dev int32 [n + 1], rising from 0; NULL: one row per request (rows = n).  Rows that belong to no request stay.
 *   kv_len   dev int32 [n], clamped to [0, columns * page_size];  tables dev int32 [n, columns]: an entry outside the
 *            pool stands for positions that nobody sees
 *   first_pos  dev int32 [n], or NULL: the rows are the last positions, kv_len[r] - their number
 *   max_rows, max_len   upper bounds of a request's rows and positions, or 0 where none are known (rows; columns *
 *            page_size).  They choose the way of computing; a bound that does not hold costs time, not correctness, and so does
 *            none: max_rows is 1 for single tokens, with cu_rows or without (24 of 1000 positions 26 us, with 0 34).
 *   workspace  dev, odb_paged_attention_workspace() bytes, aligned to 256, NULL where that says 0; holds the
 *            sums of keys that are split over workgroups, means nothing between calls, must not be shared by calls that
 *            overlap in time
 * Scores and sums are 32-bit; probabilities are rounded to the pages' dtype for the product with V.  The largest score that a row
 * sees, times scale * log2(e), has to stay below 2^29 in magnitude (the results of a row where it does not are no numbers).  The order of all
 * additions follows from the arguments and the lengths alone, so the same call gives the same bits.
 * Asynchronous on `stream`.  Errors: ODB_E_INVALID_ARG for NULL buffers, n outside [1, 4096], rows outside [0, 2^24] (0: nothing is
 * launched), n_heads no multiple of n_kv_heads, columns < 1, columns * page_size > 2^30, a scale that is not positive or, times
 * log2(e), not finite, window or sinks negative or above 2^30, a workspace that is too small, buffers not aligned to 16 bytes, row
 * strides that are no multiples of 8, out's range overlapping q's, rows * n_heads above 2^30, pools
 * outside the requirements above. */
typedef struct {
    const void *q;
    void *out;
    long long q_row, out_row;
    const int32_t *cu_rows, *first_pos, *kv_len, *tables;
    int columns, n, rows, n_heads;
    float scale;
    int causal, window, sinks, max_rows, max_len;
    void *workspace;
    size_t workspace_bytes;
} odb_attention;
int odb_paged_attention(const odb_attention *a, const odb_pages *pages, void *stream);
/* Bytes of workspace that the call needs (fields that are device buffers are not read, workspace is ignored), or a negative error code. */
long long odb_paged_attention_workspace(const odb_attention *a, const odb_pages *pages);

/* The model's forward over paged K/V: n requests of different lengths, b rows each, in one pass.  Row i of request r is the token
 * tokens[r][i] at position positions[r * b + i]; its K and V go to the pages (slots, as odb_qk_norm_rope stores them), and it attends
 * in both directions to positions 0 .. kv_len[r] - 1 of its request as the pages then hold them: the rows' own and those that
 * earlier calls stored.  With b the whole sequence it is the cache refresh of one or more requests (odb_prefill), with a block's
 * rows at first_pos[r] a decode step (odb_block_step with one draft) whose requests need neither the same length nor the same
 * block; the block's K/V in the pages are then those of this step.  odb_page_tables makes slots and positions from row_first =
 * first_pos and row_count = b; rows that pad a request have position and slot -1 and mean nothing in the outputs.
 * Inside the pages a head's K has the channel order of an interleaved rotation (channel j of the model at 2j, j + head_dim / 2 at
 * 2j + 1).
 *   tokens      dev int32 [n, b]; first_pos, kv_len dev int32 [n]; tables dev int32 [n, columns]; positions, slots dev int32 [n * b]
 *   table       dev float [n_pos, head_dim / 2, 2] as odb_rope_table writes it (base: the model's rope_base)
 *   layer0      the first layer's pool, binary16, n_heads heads; those of the next layers lie layer_stride elements further each
 *   n_layers    how many layers the pools were made for: the model's number, a call with another one is refused
 *   skip        rows of each request in front of those that conf and argmax are written for (a prompt's)
 *   conf, argmax   dev float / int32 [n, b - skip]; both NULL: only K/V are wanted
 *   unmask      dev uint8 [n, b] or NULL: the acceptance of odb_block_step with threshold tau, for b <= 256 and skip 0
 *   max_len     upper bound of kv_len as for odb_paged_attention
 * Q, K and V beyond the binary16 range are clamped and reported by odb_model_status, as in the dense calls (what padding rows
 * hold is not).  Uses the model's scratch (see the conventions above).  Asynchronous on `stream`.  Errors: ODB_E_INVALID_ARG for NULL inputs,
 * n * b outside [1, 65536], pools that do not fit the model, and what odb_paged_attention refuses. */
typedef struct {
    const int32_t *tokens;
    int n, b;
    const int32_t *first_pos, *kv_len, *tables;
    int columns;
    const int32_t *positions, *slots;
    const float *table;
    int n_pos;
    long long layer_stride;
    int skip, max_len;
    float tau;
    float *conf;
    int32_t *argmax;
    uint8_t *unmask;
    int n_layers;
} odb_paged_rows;
int odb_step_paged(odb_model *m, const odb_paged_rows *rows, const odb_pages *layer0, void *stream);

/* ---- Paged K/V in 8 bits ---------------------------------------------------------------------------------------
 * Pages as above, at half the bytes: an element is a code, and its value is code * scale, with one scale, float >= 0, for every `group`
 * consecutive positions of a page and K/V head, K and V each their own.  Codes are ODB_INT8, -127 .. 127, or ODB_E4M3 (four bits of
 * exponent, three of mantissa, largest 448; the codes 0x7f and 0xff are no numbers and are never stored).
 * Element (page, head, position inside the page, channel) of k and of v lies at page * page_stride + head * head_stride + position *
 * pos_stride + channel bytes, its scale at page * scale_page_stride + head * scale_head_stride + position / group floats.
 * Requirements: page_size, head_dim and n_pages as for odb_pages; group 1, 16, 32 or 64, at most page_size; strides not negative, those of codes
 * multiples of 16, pos_stride below 2^24, with group 1 those of scales multiples of 4; all four buffers aligned to 16 bytes.  Scales must be
 * finite numbers that are not negative where positions are visible; what codes and scales hold elsewhere means nothing. */
enum { ODB_INT8 = 3, ODB_E4M3 = 4 };
typedef struct {
    void *k, *v;                    /* dev: codes */
    float *k_scale, *v_scale;       /* dev */
    int n_pages, page_size, n_kv_heads, head_dim, codes, group;
    int dtype;                      /* of queries and results: ODB_F16 or ODB_BF16 */
    long long page_stride, head_stride, pos_stride, scale_page_stride, scale_head_stride;
} odb_quant_pages;

/* odb_qk_norm_rope into such pages: norms of queries and keys, their rotation, and K/V to codes in one pass over the projection's output.
 * Request r (of n) has rows cu_rows[r] .. cu_rows[r + 1] - 1, at positions first_pos[r], first_pos[r] + 1, ... of its pages, as for
 * odb_paged_attention; kv_len[r] is its length with them.  For every group of positions that rows fall into, and every K/V head:
 *   a = the largest magnitude of the new values;  s = a / M (M = 127 or 448), or the scale that is there if that is larger and other
 *   positions of the group below kv_len[r] stay;  codes of the new values = value / s to the nearest code, ties to even (value * M / a
 *   in 32 bits, so that the rounding of s moves no tie);  where s grows, codes that stay are rounded anew to it, else they are left alone.
 * A group whose values are all below 2^-100, with nothing that stays, has codes and scale zero; a scale below 2^-110 counts as zero.  Positions of the group that are not
 * below kv_len[r] are left alone.  The same call again writes the same codes and scales.
 * Of values that are not finite, infinities become the largest code of their sign (zero where nothing else gives the group a scale) and no numbers
 * become zero; they do not count for a, and *odd is set to 1 (it is never cleared).
 *   q, k, v, in_dtype, rows, n_heads, strides, gains, eps, table, n_pos, rot_dim, interleaved, q_out   as for odb_qk_norm_rope; in_dtype is
 *               ODB_F32 or the pages' dtype, which q_out has
 *   positions   dev int32 [rows]: of the angles.  A position outside [0, n_pos) marks a padding row: its queries become zero, nothing is stored
 *   cu_rows     dev int32 [n + 1], rising from 0, or NULL: one row per request (rows = n).  Rows that belong to no request are padding
 *   first_pos   dev int32 [n], or NULL: the rows are the last positions
 *   kv_len      dev int32 [n], tables dev int32 [n, columns], as for odb_paged_attention.  Rows at positions that are not below kv_len[r], or
 *               in no page of the pool, are not stored.  No group may hold new rows of two requests, or new rows of one and positions
 *               that another reads (a prefix that requests share ends with a group)
 *   odd         dev int32 [1] or NULL
 * Asynchronous on `stream`.  rows = 0 launches nothing.  Errors: ODB_E_INVALID_ARG, also for sizes beyond one launch (2^24 workgroups). */
typedef struct {
    const void *q, *k, *v;
    int in_dtype, rows, n_heads;
    long long q_row, k_row, v_row;
    const float *q_gain, *k_gain;
    float eps;
    const float *table;
    int n_pos, rot_dim, interleaved;
    const int32_t *positions;
    void *q_out;
    long long q_out_row;
    const int32_t *cu_rows, *first_pos, *kv_len, *tables;
    int columns, n;
    int32_t *odd;
} odb_quant_rows;
int odb_qk_norm_rope_quant(const odb_quant_rows *rows, const odb_quant_pages *pages, void *stream);

/* Values of positions: k_out and v_out, dev [rows, n_kv_heads, head_dim] of out_dtype (ODB_F16, ODB_BF16 or ODB_F32), rows k_row and v_row elements
 * apart.  slots dev int32 [rows] as odb_page_tables writes them; a slot outside the pool gives zeros.  code * scale in 32 bits, rounded
 * once, to an infinity beyond the type's range.  (pages->dtype is not looked at.)  Requirements: outputs aligned to 16 bytes, strides multiples of 8,
 * outputs that do not overlap.  Asynchronous on `stream`.  rows = 0 launches nothing.  Errors: ODB_E_INVALID_ARG, also where rows * n_kv_heads *
 * head_dim reaches 2^33. */
int odb_paged_read_quant(const odb_quant_pages *pages, const int32_t *slots, int rows, int out_dtype, void *k_out, void *v_out, long long k_row,
                         long long v_row, void *stream);

/* odb_paged_attention over such pages: the same arguments and masks, and the same errors; q and out have pages->dtype.
 * Queries meet the codes in binary16, which holds every code (bfloat16 queries as multiples of a power of two of their row's largest, within
 * 2^-33 of it), probabilities times V's scales are rounded to binary16; scores and sums are 32-bit.  A position adds to a row to within 2^-31 of
 * the largest value that V's scales in its sight can stand for (a scale of 2^-126 at least), beside the relative roundings.  V's scales that are
 * visible have to be below 2^127, K's below 2^64 and times scale * log2(e) finite in 32 bits.  The largest score that a row sees, times
 * scale * log2(e), has to stay below 2^27 in magnitude (the results of a row where it does not are no numbers). */
int odb_paged_attention_quant(const odb_attention *a, const odb_quant_pages *pages, void *stream);
long long odb_paged_attention_quant_workspace(const odb_attention *a, const odb_quant_pages *pages);

/* odb_step_paged over such pages (dtype ODB_F16): K and V of the rows are stored as odb_qk_norm_rope_quant stores them, at first_pos[r] + i, where that is
 * below kv_len[r] and the row's position is in the table of angles; slots is not looked at.  The codes of the next layers lie rows->layer_stride
 * bytes further each (a multiple of 16), the scales scale_layer_stride floats (a multiple of 4).  Queries beyond the binary16 range, K or
 * V that are not finite, and answers of the attention beyond the binary16 range, are reported by odb_model_status (K and V beyond it that are finite
 * are stored as they are).  Else as odb_step_paged. */
int odb_step_paged_quant(odb_model *m, const odb_paged_rows *rows, const odb_quant_pages *layer0, long long scale_layer_stride, void *stream);

/* Copies cached K (kv = 0, post-RoPE, logical channel order) or V (kv = 1) of
 * positions pos0 .. pos0+n-1 of one sequence and layer to host memory as
 * float [n, n_heads, head_dim].  Synchronous (device-wide). */
int odb_cache_read(const odb_cache *c, int layer, int kv, int batch_index,
                   int pos0, int n, float *host_f32);

/* Measurement aid.  Between odb_profile_begin and odb_profile_end every launch
 * of the kernel class `kernel_class` made by calls on this model is bracketed
 * by a pair of HIP events recorded on the launch stream (at most max_launches
 * pairs; further launches are not timed).  odb_profile_end synchronises the
 * device, returns the number of timed launches and the sum of their durations
 * in milliseconds, and releases the events.  A pair also spans the latency
 * from its first event to the start of the kernel, which a kernel trace does
 * not count: behind every pair a third event is recorded, and empty_pairs_ms
 * (may be NULL) receives the sum of the intervals between second and third
 * events - what a pair measures with nothing in between.  The events serialise
 * nothing but do cost a few microseconds each: do not time whole steps while
 * enabled. */
enum {
    ODB_K_GEMM_QKV = 0, ODB_K_ATTENTION, ODB_K_GEMM_O, ODB_K_GEMM_GATE_UP,
    ODB_K_GEMM_DOWN, ODB_K_GEMM_LM_HEAD, ODB_K_RMSNORM, ODB_K_COUNT
};
int odb_profile_begin(odb_model *m, int kernel_class, int max_launches);
int odb_profile_end(odb_model *m, int *n_launches, float *total_ms, float *empty_pairs_ms);

const char *odb_strerror(int code);
const char *odb_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ODB_H */
