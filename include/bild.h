/*
 * bild.h - C ABI of the MI355X (gfx950) Big Little Decoder library.
 *
 * The calls follow the paper's problem statement (Section 3.2) and Algorithm 1:
 * a small model drafts tokens autoregressively, a large model reviews a block
 * of drafts in one non-autoregressive pass.  Every numerical step runs in HIP
 * kernels on the device; the host side of this library only owns memory and
 * launches.  There is no CPU fallback.
 *
 * Conventions
 *   - every function returns BILD_OK (0) or a negative BILD_E* code; nothing
 *     throws or aborts across this boundary; on error the object passed in is
 *     left as it was;
 *   - pointers named host_* / src / out / draft are HOST memory owned by the
 *     caller and only read or written during the call;
 *   - all device memory is owned by the library behind the opaque handles;
 *   - a handle is not thread-safe; distinct states are independent but calls
 *     on states sharing one stream serialise on it;
 *   - a call that runs a decoder pass returns once the pass's results have
 *     reached the host; the stream may still be retiring that pass's last
 *     kernel, so work the caller adds must go through the same stream or
 *     wait for it (bild_encode and the bench/profile calls do wait for the stream);
 *   - token ids are int32 in [0, vocab).
 *
 * Sequence model held by a bild_state
 *   y[0..y_len)       the sequence so far: <s> (encoder-decoder pairs) or the
 *                     prompt (decoder-only pairs) followed by generated tokens
 *   draft_start       y[draft_start..y_len) are small-model drafts the large
 *                     model has not reviewed yet
 *   len_small/large   number of leading tokens of y each model has consumed
 *                     into its KV cache (cache row p holds K/V of y[p])
 * A pass of a model consumes rows y[len..y_len) at positions len.. and yields,
 * for each row, the distribution of the token that follows it.
 *
 * Environment (read when a bild_state is created)
 *   BILD_NO_GRAPH=1      launch every kernel of a pass directly instead of replaying a captured
 *                        HIP graph (needed under rocprofv3, which cannot follow graph launches)
 */
#ifndef BILD_H
#define BILD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BILD_OK      0
#define BILD_EINVAL (-1) /* bad argument (null pointer, size out of range, token id >= vocab, unsupported shape) */
#define BILD_ESTATE (-2) /* call not valid in the current state (e.g. step before encode, nothing to consume) */
#define BILD_ECAP   (-3) /* capacity exceeded (source longer than max_src, sequence longer than max_len, n > max rows) */
#define BILD_EHIP   (-4) /* a HIP runtime call failed */
#define BILD_ENOMEM (-5) /* host or device allocation failed */

#define BILD_ACT_RELU        0 /* relu(x W_in) W_out                       */
#define BILD_ACT_GATED_GELU  1 /* (gelu_tanh(x W_in) * (x W_up)) W_out     */
#define BILD_ACT_SWIGLU      2 /* (silu(x W_in) * (x W_up)) W_out          */
#define BILD_POS_SINUSOIDAL  0 /* PE added to the embedding                */
#define BILD_POS_ROPE        1 /* rotary on q and k, pairs (2i, 2i+1)      */
#define BILD_POS_RELATIVE    2 /* learned bias on self-attention scores by clamped key-query distance */
#define BILD_DT_F32          0
#define BILD_DT_BF16         1 /* weights and cached K/V stored as bf16    */

#define BILD_MAX_ROWS 32       /* most rows one decoder pass processes     */

/* Architecture of one network.  The paper fixes only layer counts and widths
 * (Table 2); the rest is this benchmark's model contract:
 *   x = embed_scale*E[(tok+tie_shift) mod vocab] (+ sinusoidal PE; relative-position
 *   models add nothing here and bias their self-attention scores instead); pre-RMSNorm
 *   sublayers x += f(norm(x)) in the order self-attn, cross-attn, FFN; scores
 *   scaled by 1/sqrt(d_head); logits = logit_scale * norm(x) E_out^T.
 * d_model, n_heads*d_head and d_ff must be multiples of 32. */
typedef struct bild_model_config {
    int32_t n_enc_layers;   /* 0: no encoder of its own                                     */
    int32_t n_dec_layers;
    int32_t d_model;
    int32_t n_heads;
    int32_t d_head;         /* 64 or 128 or any multiple of 8 up to 128                     */
    int32_t d_ff;
    int32_t act;            /* BILD_ACT_*                                                   */
    int32_t pos;            /* BILD_POS_*                                                   */
    int32_t vocab;
    int32_t tied_head;      /* 1: the LM head is the embedding matrix                       */
    int32_t dtype;          /* BILD_DT_*                                                    */
    int32_t cross_attn;     /* 1: decoder layers have a cross-attention sublayer            */
    int32_t bos;            /* first token of y for encoder-decoder pairs                   */
    int32_t tie_shift;      /* row offset of the embedding lookup, 0 = ordinary             */
    float   logit_scale;
    float   embed_scale;
    float   norm_eps;
    float   rope_base;
    int32_t rel_max_dist;   /* BILD_POS_RELATIVE: distances are clamped to [-rel_max_dist, rel_max_dist] */
} bild_model_config;

/* Counters of one bild_generate call (Table 4 reports fallback and rollback
 * rates; the paper does not define their denominators, so raw counts are given). */
typedef struct bild_stats {
    int32_t small_steps;        /* small-model passes                                  */
    int32_t large_calls;        /* large-model passes (= fallbacks of both kinds)      */
    int32_t rows_verified;      /* rows processed by large-model passes                */
    int32_t fallbacks_conf;     /* fallbacks because max p_S < alpha_FB                */
    int32_t fallbacks_forced;   /* fallbacks because n_max drafts were pending         */
    int32_t rollbacks;          /* reviews that rejected a draft                       */
    int32_t tokens_discarded;   /* drafts removed by rollbacks                         */
    int32_t n_generated;
} bild_stats;

typedef struct bild_model bild_model; /* one network's weights on the device, immutable            */
typedef struct bild_pair  bild_pair;  /* {small, large}; borrows both models                       */
typedef struct bild_state bild_state; /* one request: y, both KV caches, cross K/V, control block  */

/* Number of entries bild_model_create expects in host_tensors for this config. */
int bild_model_num_tensors(const bild_model_config* cfg);

/* Uploads one network.  host_tensors[i] are fp32 host arrays in this order
 * (entries that do not exist for the config are simply absent from the list):
 *   emb [vocab][d]; head [vocab][d] (only if !tied_head);
 *   enc_final_norm [d] (only if n_enc_layers > 0); dec_final_norm [d];
 *   (BILD_POS_RELATIVE only) enc_rel_bias (only if n_enc_layers > 0), dec_rel_bias: [n_heads][2*rel_max_dist+1],
 *     entry [h][r + rel_max_dist] is added to the self-attention score of head h for a key r positions after
 *     the query (r clamped to +-rel_max_dist); one table per stack, shared by its layers; kept in fp32;
 *   per encoder layer: ln1 [d], wq [d][I], wk [d][I], wv [d][I], wo [I][d], ln2 [d],
 *                      w_in [d][F], w_up [d][F] (gated only), w_out [F][d];
 *   per decoder layer: ln1, wq, wk, wv, wo, then (cross_attn only) lnc [d], cwq [d][I],
 *                      cwk [d][I], cwv [d][I], cwo [I][d], then ln2, w_in, w_up (gated only), w_out.
 * Matrices are row-major [inputs][outputs] (a layer computes x W); I = n_heads*d_head, F = d_ff.
 * For BILD_DT_BF16 values are rounded to bf16 (nearest even) on upload.  The
 * arrays are copied; the caller may free them on return. */
int bild_model_create(const bild_model_config* cfg, const float* const* host_tensors, int n_tensors,
                      bild_model** out);
int bild_model_destroy(bild_model* m);

/* Pairs two models (Section 3.5.1: the only requirement is a shared
 * vocabulary).  Fails with BILD_EINVAL if vocab sizes or cross_attn differ, or if the
 * small model has cross-attention but no encoder and its d_model differs from the
 * large one's (it then attends to the large model's encoder output, the early-exit
 * arrangement of Section 4.4).  The pair borrows the models: destroy it first. */
int bild_pair_create(bild_model* small_model, bild_model* large_model, bild_pair** out);

/* Early-exit pair (Section 4.4, "Early Exiting Strategy in the BiLD Framework"): the small model IS the
 * first k decoder layers of `large` followed by the large model's final norm and its LM head (the shared
 * prediction head), with a logit scale of its own.  No weights are copied.  A state of such a pair keeps
 * ONE K/V cache for those k layers and remembers the hidden state each consumed token left after layer k,
 * so a pass of the large model runs layers k..L-1 only; if the trunk has not yet consumed the rows a
 * large pass needs, the library runs it first.  Results equal those of bild_pair_create on a separately
 * uploaded copy of the first k layers up to summation order.  1 <= k < n_dec_layers, else BILD_EINVAL.
 * The pair borrows `large`: destroy the pair first. */
int bild_pair_create_early_exit(bild_model* large_model, int k, float small_logit_scale, bild_pair** out);
int bild_pair_destroy(bild_pair* p);

/* Allocates the per-request device state: room for max_src source/prompt tokens
 * and a sequence y of at most max_len tokens (including <s> or the prompt).
 * n_max: cap on consecutive small-model tokens (appendix: 10); 0 disables it.
 * hip_stream: a hipStream_t to launch on, or NULL for a stream the state creates. */
int bild_state_create(const bild_pair* p, int max_src, int max_len, int n_max, void* hip_stream,
                      bild_state** out);
int bild_state_destroy(bild_state* s);

/* Starts a request (Section 3.2: both models map the input x and the partial output y_1..n-1 to a distribution
 * over the next token; this call does the part of that map which depends on x alone, once per request).
 * Encoder-decoder pairs: runs the encoder(s) over src[0..n_src)
 * and fills every decoder layer's cross-attention K/V; y = [bos].  Decoder-only
 * pairs: y = src (the prompt) and both caches are prefilled with its first
 * n_src-1 tokens.  Requires 1 <= n_src <= max_src. */
int bild_encode(bild_state* s, const int32_t* src, int n_src);

/* One autoregressive pass of the small model (Algorithm 1, lines 3-6): consumes the
 * unconsumed tail of y, takes token = argmax p_S and
 *   fallback_flag = (max p_S < alpha_fb) or (n_max drafts already pending).
 * If the flag is 0 the token is appended to y as a draft; if 1 it is returned
 * for diagnostics only and y is unchanged.  BILD_ESTATE if nothing is unconsumed
 * (two steps in a row after a fallback), BILD_ECAP if y is full.
 * max_prob (nullable) receives max p_S. */
int bild_small_step(bild_state* s, float alpha_fb, int32_t* token, int32_t* fallback_flag, float* max_prob);

/* One non-autoregressive pass of the large model over the pending drafts
 * (Algorithm 1, lines 9-16; rollback policy of Section 3.4 with d = -ln p_L(draft)).
 * draft == NULL reviews the n = y_len - draft_start drafts pending in the state
 * (n is then ignored).  draft != NULL first replaces the pending block by
 * draft[0..n) (tests and stress runs drive arbitrary blocks this way; the small
 * cache is cut back to the reviewed prefix).  n + 1 <= BILD_MAX_ROWS.
 * On return rollback_pos = r in [0, n]: the first draft with -ln p_L > alpha_rb,
 * or n if none; out_tokens (capacity n+1) receives the r accepted drafts followed
 * by the large model's token for position r; *n_out = r + 1.  y and both caches
 * are committed accordingly.  nll (nullable, capacity n) receives -ln p_L of each draft. */
int bild_large_verify(bild_state* s, const int32_t* draft, int n, float alpha_rb, int32_t* out_tokens,
                      int32_t* n_out, int32_t* rollback_pos, float* nll);

/* Sampling variant (Appendix, "BiLD with Sampling"): with top_p in (0, 1] every token either model commits
 * is DRAWN from the nucleus of its distribution instead of being the argmax; the fallback and the rollback
 * tests are unchanged.  Nucleus: the smallest set of most likely tokens whose probability reaches top_p,
 * plus any token tied with its least likely member.  Draw: the members are walked in increasing token id and
 * the first whose running probability exceeds u * P(nucleus) is taken.  The uniform numbers are the caller's:
 * u_small[p] / u_large[p] in [0, 1) is used when the small / large model commits the token at position p of
 * the sequence (host arrays of n >= max_len floats, copied).  top_p <= 0 switches back to argmax (the arrays
 * may then be NULL).  BILD_EINVAL for top_p > 1, a missing array, n < max_len or a number outside [0, 1). */
int bild_set_sampling(bild_state* s, float top_p, const float* u_small, const float* u_large, int n);

/* Acceptance rule of the review (Section 4.2 and the appendix comparison with speculative decoding, Tables 3-4).
 * BILD_ACCEPT_THRESHOLD (the default) is the paper's rollback policy, Section 3.4: the first draft with
 * -ln p_L(draft) > alpha_RB is rolled back.  BILD_ACCEPT_REJECTION is the stochastic rule of the methods the paper
 * compares with; it needs the sampling variant (bild_set_sampling called first, else BILD_ESTATE): with p_S the nucleus
 * distribution the small model drew a draft x from and p_L the large model's nucleus distribution of the same position,
 * x is kept iff u_accept[position] * p_S(x) < p_L(x); the first refused draft is replaced by a draw (the large model's
 * uniform number of that position, ids walked in increasing order) from the normalised positive part of p_L - p_S, and
 * if none is refused the next token is drawn from p_L as usual; alpha_RB is ignored.  The fallback policy is unchanged
 * (alpha_FB = 0 with n_max = w gives the fixed window w of those methods).  u_accept: host array of n >= max_len
 * numbers in [0, 1), copied; may be NULL for BILD_ACCEPT_THRESHOLD.  The library then keeps the small model's logits
 * of every pending draft (32 x vocabulary floats of device memory).  BILD_EINVAL for an unknown rule, a missing or
 * short array or a number outside [0, 1). */
#define BILD_ACCEPT_THRESHOLD 0
#define BILD_ACCEPT_REJECTION 1
int bild_set_acceptance(bild_state* s, int rule, const float* u_accept, int n);

/* Lowers a cache length (Algorithm 1, the rollback step y <- y[:m] + [large model's token]; Section 3.4: the
 * predictions after the rolled-back position are discarded): which = 1 small, 2 large, 3 both; the cache(s) keep
 * their first pos rows (O(1): only a length changes).  BILD_EINVAL if pos exceeds
 * the current length of a selected cache.  y is not changed; a later pass simply
 * re-consumes the rows that were cut. */
int bild_kv_truncate(bild_state* s, int which, int pos);

/* Cuts the sequence to its first n_keep tokens (n_keep >= the initial length),
 * with draft_start and both caches cut to match, so that decoding continues
 * as if only that prefix had been generated. */
int bild_seq_truncate(bild_state* s, int n_keep);

/* Driver hook for tests and stress runs: overwrites y[first .. first+n) with
 * tokens (n may be 0), sets y_len = first + n and draft_start, and cuts both caches
 * back to the rows that are still valid (len_small <= first, len_large <=
 * min(first, draft_start - 1)); later passes re-consume what was cut.  Requires
 * initial length <= first <= y_len, initial length <= draft_start <= first + n,
 * first + n < max_len.  No model runs. */
int bild_force_tokens(bild_state* s, int first, const int32_t* tokens, int n, int draft_start);

/* Algorithm 1 end to end: encode(src), then small steps / large reviews until
 * max_new tokens exist or the last token equals eos (eos < 0: none).  out
 * (capacity max_new) receives the generated tokens without <s> / the prompt.
 * Equals the composition of the calls above.  src == NULL skips the encode step
 * and continues from the state as it is (max_new then counts all tokens after
 * the initial <s> / prompt); the same holds for bild_greedy. */
int bild_generate(bild_state* s, const int32_t* src, int n_src, float alpha_fb, float alpha_rb, int max_new,
                  int32_t eos, int32_t* out, int32_t* n_out, bild_stats* stats /* nullable */);

/* Vanilla inference with one model alone (which = 1 small, 2 large): greedy
 * autoregressive decoding, the baseline the paper normalises speedups to. */
int bild_greedy(bild_state* s, int which, const int32_t* src, int n_src, int max_new, int32_t eos,
                int32_t* out, int32_t* n_out);

/* The vocabulary sweep of a decoder pass as a call of its own (Section 3.2: each model maps its hidden state to
 * a distribution over the entire vocabulary; Sections 3.3 and 3.4 test max p and -ln p(draft) of it).  For each of
 * `rows` hidden rows (1..BILD_MAX_ROWS) the final RMSNorm of model m, its LM head and logit scale are applied and the
 * row's statistics are written: zmax = largest logit, lse = ln sum exp(logit), argmax (lowest id among equal
 * maxima) and z_target = logit of targets_dev[row] (NaN without targets or for an id outside the vocabulary), so
 * that max p = exp(zmax - lse) and -ln p(target) = lse - z_target.  Logits are never written to memory.
 * x_dev [rows][d_model] fp32 (16-byte aligned), targets_dev [rows] int32 (nullable) and out_dev [rows] are DEVICE
 * memory of the caller, read and written by kernels on hip_stream (NULL: the default stream), behind what is on that
 * stream already.  The call takes a scratch buffer for its kernels' partial results from a pool of the model's, or
 * allocates one, and returns when the results are in memory: the kernels then read and write nothing of the caller's
 * or of the scratch any more.  The stream itself may still be retiring the launches (hipStreamQuery: not ready), and an
 * error that the runtime finds afterwards is reported by the next call that waits for the stream.  The host polls for
 * the results for up to 2 ms and then waits for the stream. */
typedef struct bild_row_stats {
    float zmax;
    float lse;
    int32_t argmax;
    float z_target;
} bild_row_stats;
int bild_head_stats(const bild_model* m, const float* x_dev, int rows, const int32_t* targets_dev,
                    bild_row_stats* out_dev, void* hip_stream);
/* bild_head_stats for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): same arguments, same results, but the scratch buffer is a
 * 4 MiB device array inside the library (one per GPU, held until the process ends), and the call neither allocates
 * nor frees anything and does not wait for the stream: it returns once its two kernels (the head, the merge of its
 * workgroups' statistics) are enqueued on hip_stream.
 * Limit: the head's launch must not have more than 8191 workgroups (one 512-byte block of partial statistics each),
 * else BILD_ECAP; vocabularies up to 250112 at widths of 512 and 1024 are well inside it.  Every call on a GPU uses
 * that GPU's one array, which keeps the previous call's contents (the head writes all that the merge reads): calls
 * that overlap on one GPU - two streams, two threads - race; calls on one stream are ordered and safe. */
int bild_head_stats_static(const bild_model* m, const float* x_dev, int rows, const int32_t* targets_dev,
                           bild_row_stats* out_dev, void* hip_stream);

/* ======================================================================= operators on rows
 * Like bild_head_stats these work on rows that the caller holds: x, y, src, dst, logits and every other array of a call's struct is
 * DEVICE memory of the caller, read and written by kernels on hip_stream (NULL: the default stream) behind what is on that stream
 * already.  The calls allocate nothing, do not wait for the stream and may be captured into a graph; what the struct points to then
 * has to stay where it is.  They run on the device of their handle, or of the stream (bild_rotary_apply), and leave the caller's
 * current device as it was.  Strides are in elements, may be anything that keeps the rows apart, and ask for no alignment beyond the type's
 * (rows whose addresses are multiples of 16 bytes are faster).  Unless an entry says that it may be, what a call writes must not overlap what it reads. */
#define BILD_DT_F16 2 /* rows and scales of the operators, besides BILD_DT_F32 and BILD_DT_BF16; no model has it */

/* ---- products with a matrix in 4 bits ----
 * w[n][k] = (code[n][k] - zero[n][k / group]) * scale[n][k / group], zero = 8 where there are no zeros.  The last group of a feature may be short. */
typedef struct bild_quant bild_quant; /* the matrix on the device, immutable */

/* Rounds an fp32 matrix (HOST memory, [n][k]; inputs_first: [k][n], the order of bild_model_create's matrices) to such a matrix: codes [n][(k + 1) / 2],
 * input 2j in the low and 2j + 1 in the high half of byte j (an odd k leaves the last half zero); scales [n][groups], groups = ceil(k / group), of type
 * scale_dtype (BILD_DT_F16 or BILD_DT_BF16); zeros [n][groups], one of 0..15 a byte, or NULL.  Without zeros the scale is the group's largest magnitude / 7,
 * with zeros the group's range (widened to hold 0) / 15; codes and zeros are the nearest.  No value moves by more than half a scale, but for what the scale's own rounding adds
 * at the ends of the range.  (A scale below what fp16 has becomes its smallest, 2^-24; in bf16 a group whose scale is 2^-134 or less becomes zeros.)  BILD_EINVAL for a value
 * that is not finite or a scale beyond the type. */
int bild_quant_round(const float* host_w, int n, int k, int inputs_first, int group, int scale_dtype, uint8_t* host_codes, void* host_scales,
                     uint8_t* host_zeros /* nullable */);
/* Uploads a matrix given as above.  The arrays may be in host or in device memory (whatever wrote them there has to be done) and are copied.  group is 32, 64 or 128.
 * BILD_EINVAL for another group, a scale type that is not 16 bits wide, a zero above 15, or bf16 scales so far apart that no power of two makes all of
 * them fp16 (a factor of 2^32 between the largest and the smallest that is not zero always fits); the matrix lies on the current device. */
int bild_quant_create(int n, int k, int group, const uint8_t* codes, const void* scales, int scale_dtype, const uint8_t* zeros /* nullable */,
                      bild_quant** out);
int bild_quant_destroy(bild_quant* w); /* nothing that uses it may still run */

/* y[r][n] = scale * sum over k of xh[r][k] * w[n][k], xh = x, or with gain x[r][k] * gain[k] / sqrt(mean over k of x[r][k]^2 + eps): the RMSNorm in front of
 * a projection or an LM head.  Products are those of the values themselves (none is rounded on the way, but x * gain to 24 bits, and what fp32 inputs and x * gain
 * have below 2^-133), sums are fp32, that of the squares too, y is rounded once.  A row with an infinite input or NaN has no finite result and
 * leaves the others alone: all NaN, but for fp16 rows of a prompt in blocks, which have the formula's infinities.  Inputs whose sum at twice their size is beyond fp32 may be
 * taken for infinite; a row whose squares' sum is becomes zeros behind a gain.
 * rows 1 .. 2097120: those of a decoder pass, of a
 * prompt (16 bits without gain from 96 blocks of 64 rows x 128 features on, if k is a multiple of 8 and rows begin at multiples of 16 bytes, in a kernel made for it). */
typedef struct bild_quant_call {
    const void* x;      /* [rows][k], row r at x + r * x_stride               */
    int64_t x_stride;
    void* y;            /* [rows][n]                                          */
    int64_t y_stride;
    const float* gain;  /* [k], nullable: no norm                             */
    int32_t rows;
    int32_t x_dtype;    /* BILD_DT_F32, BILD_DT_BF16 or BILD_DT_F16           */
    int32_t y_dtype;
    float eps;
    float scale;
} bild_quant_call;
int bild_quant_matmul(const bild_quant* w, const bild_quant_call* call, void* hip_stream);

/* ---- rotary positions ----
 * The first rot_dim dimensions of a head are pairs that turn by position * f_i, i = 0 .. rot_dim / 2 - 1; the others are copied.
 *   layout   BILD_ROTARY_PAIRS: pair i is (2i, 2i + 1); BILD_ROTARY_HALVES: (i, i + rot_dim / 2)
 *   scaling  f_i = base^(-2i / rot_dim), and for long contexts
 *     LINEAR  f_i / factor
 *     BASE    with base * factor^(rot_dim / (rot_dim - 2)) for base
 *     BANDS   by the turns t_i = original * f_i / 2 pi in the original context: f_i from `high` turns on, f_i / factor up to `low`,
 *             in between the mean weighted by (t_i - low) / (high - low)
 *     YARN    f_i below the pair that makes `high` turns in the original context, f_i / factor above the one that makes `low`, a ramp over the
 *             pairs' index in between; cos and sin are multiplied by `magnitude`, 0: 0.1 ln(factor) + 1
 * A configuration with a frequency above 131072 radians a position (bases far below one) is refused.
 * original, low, high and magnitude are read by the last two alone (magnitude by YARN); low = high = 0 stands for 1 and 4 (BANDS), 1 and 32 (YARN). */
#define BILD_ROTARY_PAIRS  0
#define BILD_ROTARY_HALVES 1
#define BILD_ROTARY_NONE   0
#define BILD_ROTARY_LINEAR 1
#define BILD_ROTARY_BASE   2
#define BILD_ROTARY_BANDS  3
#define BILD_ROTARY_YARN   4
typedef struct bild_rotary_config {
    int32_t layout;
    int32_t rot_dim;    /* even, 2 .. 256  */
    int32_t scaling;
    int32_t original;   /* positions the unscaled frequencies were made for */
    float   base;
    float   factor;     /* >= 1 */
    float   low, high;
    float   magnitude;
} bild_rotary_config;
typedef struct bild_rotary bild_rotary; /* the frequencies, in host memory: one handle serves any stream and device, and several threads */

/* The frequencies f_i (HOST memory, rot_dim / 2 doubles) and the factor on cos and sin (nullable). */
int bild_rotary_frequencies(const bild_rotary_config* cfg, double* frequencies, double* magnitude);
int bild_rotary_create(const bild_rotary_config* cfg, bild_rotary** out);
int bild_rotary_destroy(bild_rotary* r);

/* Turns the rows of up to two arrays (queries and keys, each with heads of its own) by the positions of their tokens: dst[t][h] =
 * turned src[t][h].  inverse turns back (without dividing by the magnitude): the gradient of src from that of dst.  dst may be src with the same strides.  Angles are
 * formed in 64 bits, the products in fp32, results are rounded once. */
typedef struct bild_rotary_rows {
    const void* src;       /* head h of token t at src + t * src_token + h * src_head, its d_head dimensions side by side */
    void* dst;
    int64_t src_token, src_head, dst_token, dst_head;
    int32_t heads;         /* 0: the array is not there */
    int32_t reserved;      /* 0 */
} bild_rotary_rows;
typedef struct bild_rotary_call {
    bild_rotary_rows q, k;
    const int32_t* positions;  /* [tokens], nullable: first, first + 1, .. */
    int32_t first;
    int32_t tokens;
    int32_t d_head;            /* rot_dim .. 1024 */
    int32_t dtype;
    int32_t inverse;
    int32_t reserved;          /* 0 */
} bild_rotary_call;
int bild_rotary_apply(const bild_rotary* r, const bild_rotary_call* call, void* hip_stream);

/* bild_model_create for a network (pos = BILD_POS_ROPE) whose positions are those of `rotary` (rot_dim <= d_head; cfg->rope_base is not read but has to be
 * valid).  Every pass of such a model turns queries and keys accordingly. */
int bild_model_create_rotary(const bild_model_config* cfg, const bild_rotary_config* rotary, const float* const* host_tensors, int n_tensors,
                             bild_model** out);

/* ---- rules on logits ----
 * For each row, in this order and in fp32:
 *   an id that the row's tokens hold:            z = z > 0 ? z / repetition : z * repetition
 *   one they hold c > 0 times from `starts` on:  z = z - frequency * c, then z = z - presence
 *   an id with a bias:                           z = z + bias (the entry that stands last, if there are several)
 *   an id whose mask bit is 0:                   z = -infinity, whatever stood there
 * and the statistics of what is left, as bild_head_stats gives them, of the values before they are rounded to the rows' type: zmax, lse, argmax (lowest id among equal maxima; -1 where no id is
 * above -infinity, zmax and lse are -infinity then) and z_target (NaN without targets or for an id outside the vocabulary).  +infinity makes lse +infinity; without one a NaN that the
 * rules leave makes lse NaN, zmax and argmax are those of the numbers. */
typedef struct bild_penalties {
    float repetition;  /* 1: none */
    float frequency;   /* 0: none */
    float presence;    /* 0: none */
} bild_penalties;
typedef struct bild_rules_call {
    const void* logits;              /* [rows][vocab]                                                            */
    int64_t logits_stride;
    void* out;                       /* [rows][vocab] of the same type; may be logits (same stride); NULL: statistics only */
    int64_t out_stride;
    const int32_t* targets;          /* [rows], nullable                                                         */
    bild_row_stats* stats;           /* [rows], nullable: logits only                                            */
    const int32_t* tokens;           /* row r's tokens at tokens + r * tokens_stride (0: the rows share them); nullable: no penalties */
    int64_t tokens_stride;
    const int32_t* lengths;          /* [rows]: how many of them count; limited to 0 .. max_tokens. Ids outside the vocabulary are passed over. */
    const int32_t* starts;           /* [rows], nullable (0): the first that frequency and presence count        */
    const bild_penalties* penalties; /* [rows], or one for all rows (penalties_stride 0); needed with tokens     */
    int64_t penalties_stride;        /* 0 or 1                                                                   */
    const int32_t* bias_ids;         /* row r's ids at bias_ids + r * bias_stride (0: shared); nullable: no biases. Ids outside the vocabulary are passed over. */
    const float* bias;               /* their values, laid out the same; needed with bias_ids                    */
    int64_t bias_stride;
    const int32_t* bias_counts;      /* [rows], nullable (max_bias): how many of them count; limited to 0 .. max_bias */
    const uint32_t* mask;            /* bit id % 32 of word id / 32, row r's words at mask + r * mask_stride (0: shared); nullable: all allowed */
    int64_t mask_stride;
    int32_t rows;                    /* 1 .. the handle's max_rows                                               */
    int32_t dtype;
    int32_t max_tokens;              /* up to 1048575 */
    int32_t max_bias;                /* up to 1023    */
} bild_rules_call;
typedef struct bild_rules bild_rules; /* device memory for the statistics of rows that several workgroups share */
/* A handle's calls have to follow each other (one stream, or ordered by the caller): two streams, or two captured graphs, that may
 * run at the same time take a handle each. */
int bild_rules_create(int vocab /* up to 2^24 */, int max_rows /* up to 65535 */, bild_rules** out);
int bild_rules_destroy(bild_rules* r);
int bild_rules_apply(bild_rules* r, const bild_rules_call* call, void* hip_stream);

/* ---- a cache of keys and values in 8 bits, in pages ----
 * For callers with sequences of their own (batches, beams, drafts): keys and values of any number of sequences in one pool of pages that sequences may share.
 * A page holds page_tokens consecutive positions of a sequence: for each layer, keys and values and each key head their codes in one piece, and a scale, the
 * value that code 127 stands for (not negative, at most 2^90): code c is c * scale / 127.  The arrays are DEVICE memory of the caller, who may read them, save them and bring them back, and has to keep them
 * where they are while the handle lives.  An empty cache has lengths and refs of 0 and -1 throughout the table; of a page that no sequence holds, codes and scales are not read.
 * Entries of the table that are no page's number count as none, also where a row would see them; lengths are limited to 0 .. max_pages * page_tokens.
 * Sequences are grown, cut, forked and freed on the device, by numbers that a device array may hold (a beam's parents), so none of these calls waits, and all may be
 * captured.  Wherever a call has `sequences`, entries outside 0 .. sequences - 1 are passed over, and none may stand twice.  A handle's calls have to follow each other
 * (one stream, or ordered by the caller). */
typedef struct bild_cache_config {
    int8_t* codes;       /* [pages][layers][2: keys, values][heads][page_tokens][d_head], 16-byte aligned */
    float* scales;       /* [pages][layers][2][heads]                                            */
    int32_t* table;      /* [sequences][max_pages]: the page of each page_tokens positions, -1: none */
    int32_t* lengths;    /* [sequences]                                                          */
    int32_t* refs;       /* [pages]: how many entries of the table name the page; 0: it is free  */
    int32_t pages;       /* 1 .. 2^24                                                            */
    int32_t page_tokens; /* 32, 64 or 128                                                        */
    int32_t layers;      /* 1 .. 1024                                                            */
    int32_t heads;       /* key heads, 1 .. 1024                                                 */
    int32_t d_head;      /* a multiple of 8, 16 .. 256                                           */
    int32_t sequences;   /* 1 .. 65535                                                           */
    int32_t max_pages;   /* of a sequence; max_pages * page_tokens <= 2^30, sequences * max_pages <= 2^28 */
    int32_t reserved;    /* 0                                                                    */
} bild_cache_config;
typedef struct bild_cache bild_cache; /* the geometry, and device memory for what the calls' kernels hand on: 18, 35, 69 MB for d_head up to 64, 128, 256, and 4 x (sequences x (max_pages + 7) + 6 x pages) bytes */
int bild_cache_create(const bild_cache_config* cfg, bild_cache** out);
int bild_cache_destroy(bild_cache* c); /* nothing that uses it may still run */

/* Cuts and grows sequences.  First each is cut to `cut` positions (where that is less than it has) and gives back the pages behind; with a window, so it does with the pages that no row from
 * the cut on sees (bild_cache_attend; a later cut must not reach behind those).  Then each gets room for its new rows: free pages, lowest number first, in the order of the list; where new
 * rows would go into a page that others hold too, a copy of its positions below the cut (the last in the list keeps the page, if nobody else is left on it).  Either all sequences
 * grow or, if the pages are not enough, a sequence would become longer than max_pages, or one has no page where it was cut, none does; until the next call bild_cache_append then writes nothing. */
typedef struct bild_cache_extend_call {
    const int32_t* sequences; /* [n], nullable: 0 .. n - 1                                       */
    const int32_t* cut;       /* [n], nullable: nothing is cut                                   */
    const int32_t* starts;    /* [n + 1], nullable: sequence i gets starts[i + 1] - starts[i] rows; else `rows` each */
    int32_t* granted;         /* nullable: 1 if the sequences have grown, else 0                 */
    int32_t n;                /* 1 .. sequences                                                  */
    int32_t rows;             /* >= 0                                                            */
    int32_t window;           /* 0: none                                                         */
    int32_t sinks;
} bild_cache_extend_call;
int bild_cache_extend(bild_cache* c, const bild_cache_extend_call* call, void* hip_stream);

/* Entry i of the list becomes a copy of entry parents[i] of its group (of `group` consecutive entries, 0: all n), all at the same time and sharing pages; a parent that is not in 0 .. group - 1: empty. */
int bild_cache_fork(bild_cache* c, const int32_t* sequences /* [n], nullable */, const int32_t* parents, int n, int group, void* hip_stream);

/* Moves pages so that those in use are the lowest: the i-th free page among them takes what the i-th page behind them held (of all layers), and the tables follow.  used (device memory,
 * nullable): how many there are. */
int bild_cache_compact(bild_cache* c, int32_t* used, void* hip_stream);

/* Writes keys and values of one layer for the last rows of each sequence, which bild_cache_extend has made room for.  A page's scale grows to the largest magnitude that it has held (a cut does not
 * lower it, a page that is given away anew begins at 0); the positions that were there are rounded once more if it does: codes are the nearest to 127 x / scale (fp32), with scale, the products and quotients in fp32.
 * Magnitudes beyond 2^90 are limited to it, NaN counts as 0.  Pages that several sequences hold are not written. */
typedef struct bild_cache_append_call {
    const void* k;            /* head h of row t at k + t * k_token + h * k_head, its d_head values side by side */
    const void* v;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t* sequences; /* [n], nullable: 0 .. n - 1                                        */
    const int32_t* starts;    /* [n + 1], nullable: sequence i has the rows starts[i] .. starts[i + 1] - 1; else i * rows .. (i + 1) * rows - 1 */
    int32_t n;
    int32_t rows;             /* of a sequence; with starts: the most that one is expected to have (a choice of kernels goes by it) */
    int32_t tokens;           /* with starts: rows in all; rows behind are not touched            */
    int32_t layer;
    int32_t dtype;
    int32_t reserved;         /* 0 */
} bild_cache_append_call;
int bild_cache_append(bild_cache* c, const bild_cache_append_call* call, void* hip_stream);

/* Attention of one layer: row t of sequence i stands at position length - (rows of i) + its place among them and sees the keys j up to its own position, with a window those with j > position - window
 * and the first `sinks`; without `causal` all of the sequence (window 0 then).
 *   out[t][h] = sum over j of p_j v_j,  p = softmax of scale * q[t][h] k_j,  lse = ln of the sum of e^(scale * q k_j)
 * Query head h has the key head h / (heads / key heads).  A row that sees nothing: out 0, lse -infinity.  Products are those of q as fp16, times a power of two that puts the largest of its row below 2^15
 * (fp32: two fp16 parts), with the codes themselves; weights of the values, for many rows with the ratio of their page's scale to others, are fp16 (fp32 rows: two parts); sums are fp32; out is
 * rounded once.  Where a sequence has many rows, values of a page may count as 0 whose scale is 2^80 times smaller than that of another of its pages.  Weights (times that ratio)
 * below 2^-25 of a row's largest may count as 0 for the values, not for lse.  What a row gives whose q has an infinity or NaN, or whose products go beyond fp32, is not defined (as a rule NaN); it
 * leaves the others alone.  out may not overlap q. */
typedef struct bild_cache_attend_call {
    const void* q;            /* head h of row t at q + t * q_token + h * q_head                  */
    void* out;
    float* lse;               /* [tokens][heads], nullable                                        */
    int64_t q_token, q_head, out_token, out_head;
    const int32_t* sequences; /* as above                                                         */
    const int32_t* starts;
    int32_t n;
    int32_t rows;
    int32_t tokens;           /* as above; n * rows or `tokens` times heads is below 2^31         */
    int32_t layer;
    int32_t heads;            /* of q: a multiple of the cache's, up to 64 times as many          */
    int32_t dtype;            /* of q and out                                                     */
    float scale;
    int32_t window;           /* 0: none                                                          */
    int32_t sinks;
    int32_t causal;
} bild_cache_attend_call;
int bild_cache_attend(bild_cache* c, const bild_cache_attend_call* call, void* hip_stream);

/* ---- beams ----
 * The best continuations of each of `batch` groups of `beams` rows.  A beam that has not ended goes on with any id v: its sum is scores + logit - lse of its row (lse in fp32, sums in 64 bits from there),
 * its length one more.  One that has ended goes on with `pad` alone, sum and length unchanged.  The `choices` best by sum / max(length, 1)^penalty come out in that order, of equals the lower beam and id first.  Beams
 * whose score is -infinity or NaN (that have not ended: no finite number), rows without finite lse and ids of logit -infinity offer nothing; choices that nobody offers: parent and token -1, score -infinity, length 0, ended.
 * Nothing that is written may overlap what is read. */
typedef struct bild_beams_call {
    const void* logits;        /* [batch * beams][vocab]                                          */
    int64_t logits_stride;
    const float* scores;       /* [batch * beams]                                                 */
    const int32_t* lengths;    /* [batch * beams], nullable: 0                                    */
    const int32_t* finished;   /* [batch * beams], nullable: none has ended                       */
    float* out_scores;         /* [batch * choices], rounded to fp32                              */
    int32_t* out_parents;      /* beams of the group, 0 .. beams - 1                              */
    int32_t* out_tokens;
    int32_t* out_lengths;      /* nullable                                                        */
    int32_t* out_finished;     /* nullable: 1 if the parent had ended or the token is eos         */
    const int32_t* history;    /* nullable: the `steps` tokens of each beam so far                */
    int64_t history_stride;
    int32_t* out_history;      /* with history: those of the parents and the new token behind (-1 throughout where nobody offers) */
    int64_t out_history_stride;
    int32_t batch;
    int32_t choices;           /* 1 .. 64                                                         */
    int32_t dtype;
    int32_t eos;               /* -1: none                                                        */
    int32_t pad;
    int32_t steps;
    float penalty;             /* 0: by sums                                                      */
    int32_t reserved;          /* 0 */
} bild_beams_call;
typedef struct bild_beams bild_beams; /* device memory for the statistics of rows that several workgroups share; its calls have to follow each other (one stream, or ordered by the caller) */
int bild_beams_create(int vocab /* up to 2^24 */, int max_batch, int beams /* 1 .. 64; max_batch * beams up to 65535 */, bild_beams** out);
int bild_beams_destroy(bild_beams* b);
int bild_beams_select(bild_beams* b, const bild_beams_call* call, void* hip_stream);

/* ---- the operators inside a state's passes ----
 * The LM head of model `which` (1 small, 2 large) of this state's passes becomes `head` (n = vocab, k = d_model, else BILD_EINVAL), behind the model's final
 * norm and times its logit scale; NULL: the model's own again.  Everything that is read off the logits (policies, draws, acceptance) follows.  The matrix is
 * borrowed and has to outlive the state or the next call.  The passes then keep their logits in device memory (32 x vocabulary floats a model).
 * (bild_bench.h's counts of bytes stay those of the model's own head.) */
int bild_set_quant_head(bild_state* s, int which, const bild_quant* head /* nullable */);
/* Penalties (NULL: none) and biases (n 0: none; id i gets bias[i], the last entry of an id counts; finite, at most 1023, ids in the vocabulary) for every token that
 * either model of the state proposes from now on, as bild_rules_apply has them: the row's tokens are the sequence up to the row, drafts
 * included; frequency and presence count from the first generated token on.  repetition > 0.  HOST memory, copied.  Both none: back to unchanged logits (masks stay).
 * bild_small_step's max_prob, the fallback and rollback tests, draws and bild_debug_logits are those of the changed logits.  BILD_ECAP for penalties where
 * max_len is above 1048575. */
int bild_set_rules(bild_state* s, const bild_penalties* penalties /* nullable */, const int32_t* bias_ids, const float* bias, int n_bias);
/* Masks for the tokens at positions first .. first + n - 1 of the sequence (0 <= first, first + n <= max_len): bit id % 32 of word id / 32 of a row of ceil(vocab / 32) words
 * says whether the id may stand there.  masks [n][words]: HOST memory, copied; NULL: all ids may.  They hold until changed, also for later requests.  BILD_EINVAL for
 * a row that allows no id.  The first call allocates (max_len + 1) rows of device memory.  While no position keeps an id out, passes are those of a state without masks. */
int bild_set_masks(bild_state* s, int first, int n, const uint32_t* masks);

/* Introspection (host copies of the control block). */
int bild_get_lengths(bild_state* s, int32_t* y_len, int32_t* draft_start, int32_t* len_small, int32_t* len_large);
int bild_get_sequence(bild_state* s, int32_t* out, int cap, int32_t* n);

/* Test/debug: when enabled, each pass also writes its rows' full logits to a device
 * buffer that bild_debug_logits copies out ([rows][vocab] fp32, rows of the last pass
 * of model `which`).  Off by default: the product path never materialises logits. */
int bild_debug_enable_logits(bild_state* s, int enable);
int bild_debug_logits(bild_state* s, int which, int row, float* out_vocab);
/* Test/debug: copies cached self-attention keys (is_v = 0) or values (is_v = 1) of decoder layer `layer` of model
 * `which` for positions pos0 .. pos0+n-1 to out ([n][n_heads*d_head] fp32, host; bf16 storage is widened exactly).
 * Positions must lie below the model's consumed length.  BILD_EINVAL otherwise. */
int bild_debug_kv(bild_state* s, int which, int layer, int is_v, int pos0, int n, float* out);

const char* bild_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* BILD_H */
