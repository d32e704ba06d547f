/*
 * lfmmi.h - C ABI of the MI355X (gfx950) LF-MMI forward-backward library.
 *
 * The library computes, for a batch of unequal-length sequences, the HMM
 * forward-backward over a graph shared by the batch (denominator) or over one
 * graph per sequence (numerators): the per-sequence log-likelihood
 * log P(X | G) of Eq. 2 and the pdf occupancies gamma of Eq. 3, which are the
 * derivative of that log-likelihood with respect to the network output.
 *
 * Model (Section 3.3, Section 3.4 / Algorithm 1):
 *   an arc goes from state src to state dst, emits pdf-id pdf and has
 *   probability w = exp(logw); frame t of a sequence multiplies an arc by
 *   exp(logits[b, t, pdf]); a graph has initial probabilities init_prob[s]
 *   (a unique initial state is the one-hot case) and final probabilities
 *   final_prob[s], applied at the sequence's own last frame. The leaky HMM the
 *   paper refers to is taken as: at t = 0 and after every frame each state s
 *   additionally receives leak * (total mass) * init_prob[s].
 *
 * Conventions: every function returns an lfmmi_status (never throws, never
 * aborts); on failure lfmmi_last_error() describes the reason (thread-local).
 * Inputs are never modified. "HOST" / "DEVICE" says where a pointer lives.
 */
#ifndef LFMMI_H
#define LFMMI_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lfmmi_graph lfmmi_graph; /* opaque; owns host and device copies */

typedef enum {
    LFMMI_OK = 0,
    LFMMI_ERR_INVALID_ARG = 1, /* null pointer, negative size, shape mismatch   */
    LFMMI_ERR_BAD_GRAPH = 2,   /* state / pdf id out of range, non-finite weight */
    LFMMI_ERR_OOM = 3,         /* host or device allocation failed               */
    LFMMI_ERR_HIP = 4,         /* a HIP runtime call failed (no GPU, launch...)  */
    LFMMI_ERR_UNSUPPORTED = 5  /* size beyond what the kernels hold in LDS       */
} lfmmi_status;

/*
 * Graph packing (Section 3.3: the transition list sorted by from-state and by
 * to-state with per-state index ranges; here three sliced-ELL orderings -
 * by to-state, by from-state, by pdf-id - built once on the host).
 *
 * All pointers HOST, copied. Arcs in any order, duplicates allowed.
 *   src, dst [num_arcs] in [0, num_states); pdf [num_arcs] in [0, num_pdfs);
 *   logw [num_arcs] natural-log weight, finite (drop an arc instead of -inf);
 *   init_prob, final_prob [num_states] linear, >= 0, finite, not normalised.
 * Limits (the recursion keeps two state vectors and two emission rows in the
 * 160 KB of LDS of a compute unit): num_states <= 16384, num_pdfs <= 16384 and
 * 8 * (num_states rounded up to 64) + 8 * (num_pdfs rounded up to 64) + 128
 * <= 163840 bytes, else LFMMI_ERR_UNSUPPORTED. num_arcs may be 0.
 * When some state has final_prob == 0 or init_prob == 0 (left-to-right graphs:
 * numerators, or any graph entered through one state) the state vectors, trellis
 * and scales are kept in fp64 and the limit above counts 16 bytes per state;
 * when every state is initial and final they are fp32. The environment variable
 * LFMMI_PRECISION=32 or 64, read when a graph is packed, overrides that choice:
 * it changes results (32 on a left-to-right graph can lose posterior mass to
 * underflow, which lfmmi_forward_backward then reports in status).
 * lfmmi_graph_create packs and uploads to the current HIP device.
 * lfmmi_graph_pack only packs (no HIP call): for host-side inspection; such a
 * handle is refused by lfmmi_forward_backward until lfmmi_graph_upload.
 */
lfmmi_status lfmmi_graph_create(int32_t num_states, int32_t num_pdfs, int64_t num_arcs,
                                const int32_t *src, const int32_t *dst,
                                const int32_t *pdf, const float *logw,
                                const float *init_prob, const float *final_prob,
                                lfmmi_graph **out);
lfmmi_status lfmmi_graph_pack(int32_t num_states, int32_t num_pdfs, int64_t num_arcs,
                              const int32_t *src, const int32_t *dst,
                              const int32_t *pdf, const float *logw,
                              const float *init_prob, const float *final_prob,
                              lfmmi_graph **out);

/*
 * n graphs in one handle (Section 3.3, the batch of numerator graphs; ragged
 * offsets instead of zero padding). Graph g owns states
 * [state_off[g], state_off[g+1]) of init_prob / final_prob and arcs
 * [arc_off[g], arc_off[g+1]); src / dst are local to the graph
 * (0 .. its state count - 1). All graphs share num_pdfs.
 */
lfmmi_status lfmmi_graph_create_batch(int32_t n, int32_t num_pdfs,
                                      const int64_t *state_off, const int64_t *arc_off,
                                      const int32_t *src, const int32_t *dst,
                                      const int32_t *pdf, const float *logw,
                                      const float *init_prob, const float *final_prob,
                                      lfmmi_graph **out);
lfmmi_status lfmmi_graph_pack_batch(int32_t n, int32_t num_pdfs,
                                    const int64_t *state_off, const int64_t *arc_off,
                                    const int32_t *src, const int32_t *dst,
                                    const int32_t *pdf, const float *logw,
                                    const float *init_prob, const float *final_prob,
                                    lfmmi_graph **out);
lfmmi_status lfmmi_graph_upload(lfmmi_graph *graph);
/* Frees host and device memory, including the cached workspace. NULL is a no-op.
 * Synchronises the device. */
void lfmmi_graph_destroy(lfmmi_graph *graph);

/*
 * Batched forward-backward (Algorithm 1 and its mirrored backward pass; Eq. 3).
 *
 *   graph    one graph (shared by all sequences) or a batch handle with n == B
 *            (graph b goes with sequence b).
 *   logits   DEVICE, float32 [B, T, P] row-major contiguous; rows t >= lengths[b]
 *            are never read.
 *   lengths  HOST, int32 [B], 0 <= lengths[b] <= T, any order.
 *   P        must equal the graph's num_pdfs.
 *   leak     leaky-HMM coefficient >= 0 (0 = plain HMM).
 *   objf     DEVICE float32 [B]:      objf[b]      (=|+=) grad_scale * log Z_b
 *   grad     DEVICE float32 [B, T, P]: grad[b,t,:] (=|+=) grad_scale * gamma_t
 *            accumulate == 0 overwrites (rows t >= lengths[b] become 0),
 *            accumulate != 0 adds (those rows are left alone). The full
 *            objective of Eq. 2 / Eq. 3 is: numerators with (+1, 0), then the
 *            denominator with (-1, 1).
 *   status   DEVICE int32 [B] or NULL: 0 ok; bit 0: zero total probability
 *            (log Z = -inf, gamma rows 0); bit 1: a non-finite logit was read
 *            (objf NaN, gamma rows 0); bit 2: the alpha pass and the beta pass
 *            disagree on log Z by more than 1e-3, i.e. one of them lost mass to
 *            underflow (fp32 state vectors with leak == 0, or forced by
 *            LFMMI_PRECISION=32): objf and gamma are written but not to be trusted.
 *   hip_stream  hipStream_t (NULL = default stream). The call only enqueues
 *            work; it does not synchronise. It may allocate (and so
 *            synchronise) when the handle's cached workspace has to grow.
 *            Internally the sequences are cut by length into up to four buckets
 *            whose kernels run on three streams the library keeps per device (default
 *            priority) between an event recorded on hip_stream and events
 *            hip_stream then waits for: all of the call's work is ordered on
 *            hip_stream as if it ran there. (The buckets overlap only while their
 *            streams sit on hardware queues of their own; HIP gives a process four
 *            by default, GPU_MAX_HW_QUEUES, and streams that share one run their
 *            kernels one after the other. LFMMI_BUCKETS=1..4 sets the bucket count.)
 *            A call with the same B, T and lengths as the handle's last one, and
 *            a workspace that is large enough already, copies nothing from the
 *            host and allocates nothing: it enqueues kernels, event records and
 *            event waits only, and may be captured into a HIP graph (relaxed
 *            capture mode, because of the library's own streams).
 * B == 0 or T == 0 with all lengths 0 are valid. Calls on one handle must be
 * ordered on one stream (they share the handle's workspace). The device the
 * graph was uploaded to must be the current one (LFMMI_ERR_INVALID_ARG if not).
 */
lfmmi_status lfmmi_forward_backward(const lfmmi_graph *graph, const float *logits,
                                    const int32_t *lengths, int32_t B, int32_t T,
                                    int32_t P, float leak, float grad_scale,
                                    int accumulate, float *objf, float *grad,
                                    int32_t *status, void *hip_stream);

/*
 * lfmmi_forward_backward for callers that cannot allocate: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc. Same arguments,
 * same results; the call's workspace (emission values, both trellises, per-frame
 * scales, descriptors) lies in a static device array of
 * LFMMI_STATIC_WORKSPACE_BYTES that every GPU the library runs on holds from the
 * first graph upload on that GPU until the process ends, instead of in memory the
 * handle allocates. The call makes no hipMalloc / hipFree / hipHostMalloc, creates
 * no stream or event and copies nothing from the host: the lengths travel as a
 * kernel argument, all kernels run on hip_stream in one bucket, and there is no
 * per-kernel timing (lfmmi_profile_enable does not apply).
 * Limits: B <= LFMMI_STATIC_MAX_BATCH, and the workspace the call needs - about
 *   4 * B * T * P + 4 * sum_b (lengths[b] + 1) * (rows_fwd + rows_bwd + 5) bytes
 * (8 instead of 4 in the second term for fp64 graphs; rows = the padded row counts
 * lfmmi_graph_ordering_info reports as 64 * info[1]) - must fit the array, else
 * LFMMI_ERR_UNSUPPORTED with the two sizes in lfmmi_last_error().
 * All calls on one GPU share that GPU's array, whatever their handle or stream:
 * calls that overlap on one GPU race, so order them (one stream, or events).
 * Nothing in the array has to survive between calls; what must start at zero is
 * cleared by the call's own kernels.
 */
#define LFMMI_STATIC_WORKSPACE_BYTES (64u << 20)
#define LFMMI_STATIC_MAX_BATCH 256
lfmmi_status lfmmi_forward_backward_static(const lfmmi_graph *graph, const float *logits,
                                           const int32_t *lengths, int32_t B, int32_t T,
                                           int32_t P, float leak, float grad_scale,
                                           int accumulate, float *objf, float *grad,
                                           int32_t *status, void *hip_stream);

/*
 * The whole objective of Eq. 2 and its gradient, Eq. 3, in one call:
 *   objf[b]     = log P(X_b | numerator graph b) - log P(X_b | denominator graph)
 *   grad[b,t,:] = numerator occupancies - denominator occupancies (rows t >= lengths[b]: 0)
 *   status[b]   = the two passes' flags or-ed together (may be NULL)
 * exactly what lfmmi_forward_backward(num, ..., +1, 0, ...) followed by
 * lfmmi_forward_backward(den, ..., -1, 1, ...) leaves in the three arrays (bit for
 * bit). Where the recursion workgroups of both passes fit the chip together (4 B
 * at most its compute units: B <= 64), no sequence is empty and the batch has 8
 * sequences or one of 256 frames, the passes run at the same time, the numerators'
 * on a stream of the library's that hip_stream waits for (LFMMI_BESIDE=0: never; nor
 * while either handle collects events, see lfmmi_profile_enable: what they time is the
 * passes in turn; nor with fewer than 4 sequences under capture).
 * Otherwise the numerators' pass is enqueued first, then the denominator's, both on
 * hip_stream, and the emission values exp(logit - row maximum) are computed once,
 * by the numerators' pass; the denominator's reads them from that handle's
 * workspace. If the denominator's pass is refused (an error code comes back) the
 * numerators' pass is already enqueued and the three arrays are left holding its
 * results alone: treat them as undefined.
 * (With more sequences, side by side was measured 13 to 24 % slower on the
 * 128-sequence workload: the numerators' workgroups then take compute units from
 * the denominator's longest sequences, whose recursion decides when the call ends,
 * and HIP streams of one priority give no say in that.)
 * num: a batch handle with B graphs (or one graph for all); den: usually one shared
 * graph; the two must be different handles.
 * Arguments and errors otherwise as lfmmi_forward_backward.
 */
lfmmi_status lfmmi_loss(const lfmmi_graph *num, const lfmmi_graph *den, const float *logits,
                        const int32_t *lengths, int32_t B, int32_t T, int32_t P, float leak,
                        float *objf, float *grad, int32_t *status, void *hip_stream);

/* ---- log probabilities of given tokens, and gradients --------------------
 * What a trainer uses beside the sequence loss. No handle: the calls keep nothing. */

/* Types of the arrays below. */
typedef enum { LFMMI_F32 = 0, LFMMI_BF16 = 1, LFMMI_F16 = 2 } lfmmi_dtype;

/*
 * Log probabilities of given tokens (or pdfs, of a frame alignment), with the entropy and
 * the best alternatives of every row. For row (b, t) with logits x, m = max_i x_i,
 * d_i = scale * (x_i - m) and s = sum_i exp(d_i):
 *   logp[b,t]    = d_target - ln s
 *   entropy[b,t] = ln s - (sum_i d_i exp(d_i)) / s        (a logit of -inf adds nothing)
 *   top_id[b,t,:], top_logp[b,t,:]  the top_k largest logits' indices and log
 *                  probabilities, largest first, equal ones by index, lowest first
 *   stats[b,t,:] = (m, ln s), what lfmmi_token_logprobs_backward takes
 *
 *   logits   DEVICE, [B, T, V] of `dtype` (lfmmi_dtype): element (b, t, i) at
 *            b * stride_b + t * stride_t + i, strides >= 0 in elements (0 repeats),
 *            aligned to an element at least. V >= 1.
 *   lengths  HOST int32 [B], 0 <= lengths[b] <= T, or NULL (all T).
 *   targets  DEVICE int32 or int64 (target_bytes 4 or 8) [B, T], or NULL: no logp.
 *            Rows t >= lengths[b] and rows with a negative target are not scored: their
 *            logits are never read, their outputs are 0 and their top_id -1.
 *   scale    what logits are multiplied by (an acoustic scale, the inverse of a
 *            temperature), 1e-6 <= scale <= 1e6.
 *   top_k    0 <= top_k <= LFMMI_MAX_TOP and <= V.
 *   logp, entropy float32 [B, T]; stats float32 [B, T, 2]; top_id int32 and top_logp
 *            float32 [B, T, top_k]; status int32 [B, T]: all DEVICE, any may be NULL
 *            (logp must be if targets is).
 *   status   0 ok; bit 0: every logit is -inf (logp and top_logp -inf, entropy 0);
 *            bit 1: a NaN or +inf logit was read (logp, entropy, stats and top_logp NaN,
 *            top_id -1); bit 2: the target is not below V (logp NaN).
 *   workspace DEVICE, at least the bytes that lfmmi_token_logprobs_workspace gives for
 *            the same dtype, B, T, V and top_k (0: may be NULL), aligned to 16; its content
 *            before and after the call is of no account. Calls that may run at the same
 *            time, replays of captured graphs among them, need one each.
 * The call enqueues kernels on hip_stream and nothing else: it does not allocate or
 * synchronise and may be captured into a HIP graph. Arrays lie on the current device.
 * The same inputs at the same alignment give the same bits. B == 0 or T == 0 is valid.
 */
#define LFMMI_MAX_TOP 64
lfmmi_status lfmmi_token_logprobs(const void *logits, int32_t dtype, int32_t B, int32_t T,
                                  int32_t V, int64_t stride_b, int64_t stride_t,
                                  const int32_t *lengths, const void *targets,
                                  int32_t target_bytes, float scale, int32_t top_k,
                                  float *logp, float *entropy, float *stats, int32_t *top_id,
                                  float *top_logp, int32_t *status, void *workspace,
                                  int64_t workspace_bytes, void *hip_stream);
lfmmi_status lfmmi_token_logprobs_workspace(int32_t dtype, int32_t B, int32_t T, int32_t V,
                                            int32_t top_k, int64_t *bytes);

/*
 * The gradient of a loss with respect to the logits, given its gradients with respect to
 * logp (grad_logp) and entropy (grad_entropy), DEVICE float32 [B, T], either may be NULL
 * (taken as 0). With l_i = d_i - ln s and p_i = exp(l_i):
 *   grad[b,t,i] = scale * (grad_logp * (delta_{i,target} - p_i)
 *                          - grad_entropy * p_i * (l_i + entropy))
 * Rows that are not scored, and rows with a flag in status, become 0. stats and entropy
 * (needed with grad_entropy) are what lfmmi_token_logprobs gave for the same logits, lengths,
 * targets and scale. targets may be NULL (then grad_logp must be). grad: DEVICE [B, T, V]
 * contiguous, of the logits' type; it may be the logits' own array if those are contiguous,
 * and must not overlap them otherwise. Streams, capture, errors as above; no workspace.
 */
lfmmi_status lfmmi_token_logprobs_backward(const void *logits, int32_t dtype, int32_t B,
                                           int32_t T, int32_t V, int64_t stride_b,
                                           int64_t stride_t, const int32_t *lengths,
                                           const void *targets, int32_t target_bytes,
                                           float scale, const float *stats,
                                           const float *entropy, const float *grad_logp,
                                           const float *grad_entropy, void *grad,
                                           void *hip_stream);

/*
 * The norm of n gradient tensors taken together, sqrt(sum of all squares), and gradients
 * scaled so that it is at most max_norm:
 *   norm       DEVICE float32 [1]
 *   outs[i]    = grads[i] * min(1, max_norm / norm)
 * grads, outs, counts, dtypes are HOST arrays [n], copied: DEVICE pointers (aligned to an
 * element at least; NULL where the count is 0), numbers of values (0 is valid) and
 * lfmmi_dtype codes. outs NULL, or outs[i] == grads[i], scales in place (nothing is written
 * if norm <= max_norm); otherwise nothing written may overlap any other array of the call,
 * nor may gradients scaled in place be listed twice (LFMMI_ERR_INVALID_ARG); norm and
 * workspace are written by both calls. Squares are
 * summed in fp64, in a fixed order (the same inputs at the same alignment give the same
 * bits): values whose squares overflow fp32 do not upset the norm. A norm that is not finite
 * (a NaN or infinite gradient; a norm beyond fp32 counts as infinite) makes every value of
 * outs 0, so that none of it reaches the weights, and `norm` says so: plain gradient descent then
 * does nothing, an optimiser with momentum or weight decay still moves unless the step is left
 * out. max_norm >= 0, may be infinite.
 * workspace: DEVICE, LFMMI_GRAD_WORKSPACE_BYTES(n) bytes, aligned to 16; otherwise as for
 * lfmmi_token_logprobs. The calls enqueue kernels on hip_stream and nothing else.
 */
#define LFMMI_GRAD_WORKSPACE_BYTES(n) (16384 + 32 * ((int64_t)(n) + 1))
lfmmi_status lfmmi_grad_norm(int32_t n, const void *const *grads, const int64_t *counts,
                             const int32_t *dtypes, float *norm, void *workspace,
                             int64_t workspace_bytes, void *hip_stream);
lfmmi_status lfmmi_clip_grads(int32_t n, const void *const *grads, void *const *outs,
                              const int64_t *counts, const int32_t *dtypes, float max_norm,
                              float *norm, void *workspace, int64_t workspace_bytes,
                              void *hip_stream);

/* ---- around an output layer ----------------------------------------------
 * What stands in front of the layer whose logits the calls above take, and behind it: token
 * embeddings, dropout, the end of a residual block, verification of drafted tokens. No handle:
 * the calls keep nothing, enqueue kernels on hip_stream and nothing else, do not allocate or
 * synchronise, and may be captured into a HIP graph. Arrays are DEVICE and lie on the current
 * device, aligned to their elements, contiguous where no stride is given; lengths are HOST,
 * copied. What is written may overlap no other array of a call but where that is said
 * (LFMMI_ERR_INVALID_ARG). Workspaces as for lfmmi_token_logprobs: aligned to 16, the bytes that
 * the call of that name gives for the same sizes, one for each call that may run at the same
 * time, replays of captured graphs among them. The same inputs give the same bits. Sums are
 * taken in 32 bits or more and rounded to an array's type once. */

/*
 * Rows of a table for given tokens: out[b,t,:] = scale * table[tokens[b,t],:]
 *   table    [V, D] of `dtype`, row v at v * stride elements (stride >= 0).
 *   tokens   int32 or int64 (token_bytes 4 or 8) [B, T]. Rows with a negative token and rows
 *            t >= lengths[b] (lengths HOST int32 [B], or NULL: all T) are 0; the tokens of the
 *            latter are never read. A token that is not below V makes its row NaN.
 *   scale    1e-6 <= scale <= 1e6
 *   out      [B, T, D]
 *   status   int32 [B, T] or NULL: 0 ok; bit 2: the token is not below V.
 * 1 <= D <= 2^24.
 */
lfmmi_status lfmmi_embed_tokens(const void *table, int32_t dtype, int32_t V, int32_t D,
                                int64_t stride, const void *tokens, int32_t token_bytes,
                                int32_t B, int32_t T, const int32_t *lengths, float scale,
                                void *out, int32_t *status, void *hip_stream);
/*
 * The gradient of the table, given that of out:
 *   grad[v,:] (=|+=) scale * sum of grad_out[b,t,:] over the positions whose token is v
 * summed in fp32, in an order that the tokens alone decide; rows without a position are 0, or
 * with accumulate != 0 left as they are. Negative tokens, tokens that are not below V and rows
 * t >= lengths[b] add nothing, and those rows of grad_out are never read.
 *   grad_out [B, T, D] of `dtype`, row (b, t) at b * stride_b + t * stride_t, strides >= 0
 *   grad     [V, D] of `dtype`
 */
lfmmi_status lfmmi_embed_tokens_backward(const void *grad_out, int32_t dtype, int32_t V, int32_t D,
                                         int64_t stride_b, int64_t stride_t, const void *tokens,
                                         int32_t token_bytes, int32_t B, int32_t T,
                                         const int32_t *lengths, float scale, int accumulate,
                                         void *grad, void *workspace, int64_t workspace_bytes,
                                         void *hip_stream);
lfmmi_status lfmmi_embed_tokens_workspace(int32_t V, int32_t D, int32_t B, int32_t T,
                                          int64_t *bytes);

/*
 * Dropout of rows: y[r,c] = kept ? x[r,c] / (1 - p') : 0, whatever x is where it is dropped.
 * p' is p rounded to a multiple of 2^-16, 0 <= p <= 1 (1: everything is dropped). What is kept is
 * a function of (seed, draw, r, c) alone, draw = offset + *step modulo 2^64 (step DEVICE int64
 * [1] or NULL: 0; a captured graph draws anew when a kernel has counted it up): with the four
 * words w of
 * Philox4x32-10 for the counter (c / 8, r, low and high word of draw) and the key (low and high
 * word of seed), c is kept if the 16 bits c % 8 of w (the low half of w[0] first) are at least
 * 65536 p'. No mask is stored: the gradient is the same call on the gradient of y.
 *   x        [R, D] of `dtype`, D <= 2^30, row r at r * stride elements (stride >= 0)
 *   y        [R, D]; or x itself, laid out as it is (stride >= D)
 */
lfmmi_status lfmmi_dropout(const void *x, int32_t dtype, int32_t R, int32_t D, int64_t stride,
                           float p, uint64_t seed, uint64_t offset, const int64_t *step, void *y,
                           void *hip_stream);

/*
 * The end of a residual block: the residual's addition and a root-mean-square norm, with dropout
 * on the way and the output in 8 bits if wanted. For row (b, t):
 *   sum    = residual + dropout(x), rounded to `dtype` (row b * T + t of lfmmi_dropout)
 *   rstd   = 1 / sqrt(mean_c sum_c^2 + eps)
 *   y_c    = sum_c * rstd * weight_c
 *   q_scale = max(max_c |y_c| / 448, 2^-126),  q_c = y_c / q_scale rounded to e4m3 (OCP, no infinities)
 *
 *   x, residual [B, T, D] of `dtype`, rows at their strides (>= 0); residual may be NULL (0).
 *   weight   [D] of `dtype` or float32 (weight_dtype), or NULL (1)
 *   lengths  HOST int32 [B], or NULL: rows t >= lengths[b] are never read, their outputs are 0
 *   eps      1e-30 <= eps <= 1e20
 *   p, seed, offset, step  as for lfmmi_dropout
 *   sum      [B, T, D]; may be NULL where it would be x itself (no residual, nothing dropped).
 *            It may be x or residual, where the rows of that one follow each other.
 *   y        [B, T, D] of `dtype`, rstd float32 [B, T]: may be NULL
 *   q        bytes [B, T, D], q_scale float32 [B, T]: both or none. A row with a NaN has a
 *            q_scale of NaN.
 * 1 <= D <= 2^24. Squares are summed in fp32; where that overflows, of the values times 2^-80.
 */
lfmmi_status lfmmi_add_rms_norm(const void *x, int64_t stride_b, int64_t stride_t,
                                const void *residual, int64_t residual_stride_b,
                                int64_t residual_stride_t, int32_t dtype, int32_t B, int32_t T,
                                int32_t D, const int32_t *lengths, const void *weight,
                                int32_t weight_dtype, float eps, float p, uint64_t seed,
                                uint64_t offset, const int64_t *step, void *sum, void *y,
                                float *rstd, void *q, float *q_scale, void *hip_stream);
/*
 * Its gradients, given those of y (grad_y) and of sum (grad_sum), either may be NULL (0). With
 * n = sum * rstd and g = weight * grad_y:
 *   d             = grad_sum + rstd * (g - n * mean_c(g_c n_c))
 *   grad_residual = d,  grad_x = dropout(d) with the forward call's p, seed, offset and step
 *   grad_weight   = sum over the rows of grad_y * n, in fp32, in an order that sizes and type decide
 * sum (or x, where that is it; rows at their strides) and rstd: what the forward call read and
 * gave. grad_x, grad_residual [B, T, D] of `dtype` and grad_weight [D] of weight_dtype may be
 * NULL; either of the first two may be grad_y or grad_sum. Rows t >= lengths[b] become 0 and add
 * nothing (where x stands for sum, grad_sum is x's gradient there too, and the caller's to add).
 * workspace: needed with grad_weight.
 */
lfmmi_status lfmmi_add_rms_norm_backward(const void *sum, int64_t stride_b, int64_t stride_t,
                                         int32_t dtype, int32_t B, int32_t T, int32_t D,
                                         const int32_t *lengths, const void *weight,
                                         int32_t weight_dtype, const float *rstd,
                                         const void *grad_y, const void *grad_sum, float p,
                                         uint64_t seed, uint64_t offset, const int64_t *step,
                                         void *grad_x, void *grad_residual, void *grad_weight,
                                         void *workspace, int64_t workspace_bytes,
                                         void *hip_stream);
lfmmi_status lfmmi_add_rms_norm_workspace(int32_t B, int32_t T, int32_t D, int64_t *bytes);

/*
 * Drafted tokens against the logits of the model they are drafted for. Sequence b has n =
 * lengths[b] drafted tokens d_0 .. d_{n-1} (HOST int32 [B], 0 <= n <= K; NULL: K) and the target's
 * logits in rows 0 .. n: row i is what follows the first i drafted tokens. With p_i the softmax of
 * scale * logits[b,i,:], q_i that of draft_scale * draft_logits[b,i,:] (NULL: q_i is 1 at d_i, 0
 * elsewhere) and u = uniforms[b,:], float32 [B, K + 1] in [0, 1):
 *   d_i is taken if all before it are and u_i q_i(d_i) < p_i(d_i);
 *   the first that is not, d_r, is replaced by a token drawn from max(0, p_r - q_r), normalised
 *   (from p_r where that is 0 everywhere; where p_r and q_r agree but for rounding it is what
 *   rounding leaves);
 *   if all are taken (r = n), a token drawn from p_n follows.
 * Drawn means: the first token at which the running sum of what it is drawn from, in the order of
 * the tokens, passes u_K times the whole (a number of 1 or more: the last token of any
 * weight). All of it is in fp64, with exponentials that are off by 7e-12 of themselves at most; a
 * probability below 2^-1000 times the largest of its row counts as 0. The tokens that come out are
 * distributed as p says. With K = 0 the call draws one token a sequence.
 * uniforms NULL: greedy. d_i is taken if it is the first largest logit of row i, which replaces
 * or follows the others too; draft_logits must be NULL.
 *
 *   logits   [B, K + 1, V], draft_logits [B, K, V], of `dtype`: rows at their strides (>= 0)
 *   drafted  int32 or int64 (token_bytes 4 or 8) [B, K]
 *   accepted int32 [B]: r.  tokens int32 [B, K + 1]: d_0 .. d_{r-1}, the token drawn, then -1
 *   status   int32 [B] or NULL: 0 ok; otherwise row r could not be judged, tokens[b,r] is -1: bit 0:
 *            every logit of a row is -inf; bit 1: a NaN or +inf logit; bit 2: d_r is not in
 *            [0, V). Rows behind r do not matter.
 */
lfmmi_status lfmmi_verify_tokens(const void *logits, int32_t dtype, int32_t B, int32_t K, int32_t V,
                                 int64_t stride_b, int64_t stride_t, const void *draft_logits,
                                 int64_t draft_stride_b, int64_t draft_stride_t,
                                 const void *drafted, int32_t token_bytes, const int32_t *lengths,
                                 float scale, float draft_scale, const float *uniforms,
                                 int32_t *accepted, int32_t *tokens, int32_t *status,
                                 void *workspace, int64_t workspace_bytes, void *hip_stream);
lfmmi_status lfmmi_verify_tokens_workspace(int32_t B, int32_t K, int32_t V, int64_t *bytes);

/* Thread-local description of the last failure on this thread ("" if none). */
const char *lfmmi_last_error(void);

/* ---- introspection (host side; used by tests and the benchmark) ---------- */

enum { LFMMI_ORD_FWD = 0, LFMMI_ORD_BWD = 1, LFMMI_ORD_OCC = 2 };

/* info[0] number of graphs, [1] num_pdfs, [2] total states, [3] total arcs,
 * [4] waves per workgroup of the recursion kernel, [5] waves of the occupancy
 * kernel, [6] flags (bit 0: uploaded; bit 1: state vectors kept in fp64, which
 * is chosen when some state has final_prob 0 or init_prob 0; bit 2: every arc
 * carries the pdf-id of the state it enters - graphs expanded from HMMs whose
 * states emit, Section 4.2 - and the recursion runs without an emission gather per
 * arc: alpha multiplies a row by its emission once, beta folds the emission into
 * the stored vector; not set for graphs of one short slice a wave, per-utterance
 * numerators, whose straight-line variant does the same), [7] workspace bytes held. */
lfmmi_status lfmmi_graph_info(const lfmmi_graph *graph, int64_t info[8]);

/* Packed ordering `ord` of graph `g`: info[0] rows, [1] slices (64 rows each),
 * [2] waves, [3] total slots (sum of slice widths), [4] max slots of one wave,
 * [5] arc slots of a wave the recursion kernel keeps in registers (0: all streamed),
 * [6] 1 if the emission row is replicated per LDS bank, [7] how the leak meets an init_prob
 * that is not uniform: 1 the arcs carry a factor each, 2 state values are kept divided by
 * init_prob and the arcs need none (0: init_prob is uniform), [8] modelled LDS cycles of the
 * gathers of one frame (per slot and half-wave, the largest number of distinct
 * addresses in one of the 32 banks), [9] 1 if every FWD / BWD slice ends in a
 * closing slot (packed so when init_prob is not uniform), [10] number of hub
 * slices (see below), [11] FWD / BWD: rows (slices * 64) one state vector of the
 * chosen recursion kernel's fixed LDS map holds, 0 when that kernel sizes its LDS
 * by the graph (arcs streamed). The kernel is chosen so that info[1] * 64 fits. */
lfmmi_status lfmmi_graph_ordering_info(const lfmmi_graph *graph, int32_t g,
                                       int32_t ord, int64_t info[12]);
/* Copies the packed ordering out (any pointer may be NULL):
 *   slice_off  [slices + 1] first slot of each slice
 *   wave_first [waves + 1]  first slice of each wave
 *   key, w     [total slots * 64] arc records, lane-minor; key = x-index * 4 in
 *              the low 16 bits, y-index * 4 in the high 16 bits; padding has w 0 (its
 *              key points wherever no bank conflict arises).
 *              With closing slots (info[9]) the last slot of every FWD / BWD
 *              slice holds no arc: its key is 0 and its w is the row's leak-dot
 *              weight (FWD: 1 on real rows; BWD: init_prob of the row's state)
 *   row_id     [slices * 64] the state (FWD: to-state, BWD: from-state) or
 *              pdf-id (OCC) a row stands for, -1 for padding rows
 *   slice_hub  [slices] 1 for a hub slice (FWD / BWD): a state with at least 64
 *              arcs and far more than the others gets a slice of its own; its
 *              row is that of lane 0, the arcs in all 64 lanes of the slice are
 *              its arcs (the kernels add the lanes' sums up), and the other 63
 *              rows are padding rows
 *   x-index / y-index: FWD (from-state in FWD numbering, pdf), BWD (to-state in
 *   BWD numbering, pdf), OCC (from-state in FWD numbering, to-state in BWD
 *   numbering), where a state's number in an ordering is the row it owns. */
lfmmi_status lfmmi_graph_ordering_copy(const lfmmi_graph *graph, int32_t g, int32_t ord,
                                       int32_t *slice_off, int32_t *wave_first,
                                       uint32_t *key, float *w, int32_t *row_id,
                                       int32_t *slice_hub);

/* Per-kernel timing with HIP events. While enabled, every lfmmi_forward_backward
 * on this handle records events around its kernels, on the streams they run on:
 * one emission, one recursion and one occupancy launch per bucket of sequences
 * (see lfmmi_forward_backward). enable: 0 off; 1 events around every kernel;
 * 2 around the recursion launches only (half the events: they cost about 3 % of
 * a call on the WSJ-shaped workload at level 1). Calls recorded at one level
 * must be read before the level changes. lfmmi_profile_read waits for the
 * events and returns mean durations per launch in milliseconds - ms[0] emission
 * (0 at level 2); [1] recursion (alpha and beta, and the scales, which the last
 * workgroup of a sequence computes); [2] 0; [3] occupancy + gradient (0 at
 * level 2) - with the number of calls in *calls and of launches of each kernel
 * in *launches (either may be NULL), then forgets them. Launches of one call
 * overlap: the means do not add up to the time of a call. While events are collected
 * lfmmi_loss runs its two passes in turn (results are the same bits). */
lfmmi_status lfmmi_profile_enable(lfmmi_graph *graph, int enable);
lfmmi_status lfmmi_profile_read(lfmmi_graph *graph, float ms[4], int32_t *calls,
                                int32_t *launches);

#ifdef __cplusplus
}
#endif
#endif /* LFMMI_H */
