/*
 * dv.h -- vocabulary alignment and masked greedy decoding on one MI355X.
 *
 * C ABI of libdv.so.  Two operations, from "Guiding LLMs The Right Way: Fast,
 * Non-Invasive Constrained Generation" (DOMINO, ICML 2024):
 *
 *   dv_align        the offline vocabulary alignment of Sec. 3.3 /
 *                   Algorithm 2 for a regular (DFA) constraint walked to full
 *                   depth (Sec. 3.5, lookahead k = infinity): every scanner
 *                   state is walked through every token's bytes.
 *   dv_masked_step  one step of Algorithm 1: look up the mask of each
 *                   sequence's current state, apply it to the logits, decode
 *                   greedily (Algorithm 3's argmax over the admissible set)
 *                   and advance the state with the chosen token.
 *   dv_align_eos    dv_align with an end-of-sequence token that is allowed
 *                   exactly in accepting states.
 *   dv_masked_step_opportunistic
 *                   dv_masked_step that checks the model's own choice first
 *                   (opportunistic masking, Sec. 3.5).
 *   dv_masked_sample
 *                   the sampled decode at temperature T over the allowed
 *                   tokens, reproducible from a seed and an offset.
 *   dv_spec_walk,   the speculative chain check of Sec. 3.6: how many
 *   dv_spec_verify  proposed tokens the constraint admits, and greedy
 *                   verification of the proposals against the model's logits
 *                   at every proposed position.
 *   dv_head_loss,   training a proposer or a model under the same constraint:
 *   dv_distill_loss, softmax cross entropy over the allowed tokens from hidden
 *   dv_embed and    states and head weights, divergence from a teacher's top
 *   their _backward logits, and the embedding, each with its gradients.
 *   dv_rms_norm,    from a model's last hidden states to the logits that the
 *   dv_quantize_f8, steps above read: the last norm with the residual's
 *   dv_product_f8,  addition, the head's product in 8 bits (both with their
 *   dv_adjust_logits  gradients), and penalties, biases and the grammar's mask.
 *
 * Conventions shared by every call:
 *   - Every array argument is a DEVICE pointer (hipMalloc'd or a torch CUDA
 *     tensor's data_ptr) owned by the caller.  The library allocates nothing,
 *     keeps no pointer after it returns, and has no global state except a
 *     per-thread error message.
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = the null stream)
 *     and runs asynchronously to the host.  Outputs are valid once the stream
 *     has reached the call; inputs must stay unchanged until then.  Two calls
 *     that share a workspace must be ordered on one stream.
 *   - Arguments are checked on the host before any HIP call.  On a failed
 *     check nothing is enqueued and the call returns an error status; a
 *     message is available from dv_last_error() on the calling thread.
 *   - The alphabet is bytes (256 symbols).  DV_DEAD (-1) is the dead state:
 *     a sentinel, never a table row.  A transition target or an input state
 *     outside [0, num_states) reads as DV_DEAD; nothing leaves DV_DEAD.
 */
#ifndef DV_H
#define DV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define DV_API __attribute__((visibility("default")))
#else
#define DV_API
#endif

#define DV_DEAD (-1)

/* Limits checked by every call (inclusive). */
#define DV_MAX_STATES 65535        /* num_states  in [1, DV_MAX_STATES]  */
#define DV_MAX_TOKENS 16777216     /* num_tokens  in [1, DV_MAX_TOKENS]  */
#define DV_MAX_BATCH  1048576      /* batch       in [0, DV_MAX_BATCH]   */
#define DV_MAX_PROPOSED 1024       /* num_proposed in [0, DV_MAX_PROPOSED];
                                      batch * (num_proposed + 1) <= DV_MAX_BATCH */
#define DV_NOALLOC_MAX_BATCH 65536 /* batch of dv_masked_step_noalloc          */
#define DV_MAX_HIDDEN 65536        /* hidden      in [1, DV_MAX_HIDDEN]  */
#define DV_MAX_TOP    1024         /* num_top     in [1, DV_MAX_TOP]     */
#define DV_MAX_DEPTH  4194304      /* depth       in [128, DV_MAX_DEPTH] */
#define DV_MAX_BIAS   1024         /* num_bias    in [0, DV_MAX_BIAS]    */
#define DV_MAX_HISTORY 1048575     /* max_history in [0, DV_MAX_HISTORY] */
#define DV_EXACT_SUMS 256          /* beside dv_product_f8's dtype: no products are cut */
#define DV_SCALE_BLOCK 128         /* columns, or rows and columns, of an 8-bit operand's scale */

typedef enum dv_status {
    DV_OK = 0,
    DV_ERR_INVALID_ARG = 1,  /* a required pointer is NULL                         */
    DV_ERR_SHAPE = 2,        /* a size is outside its limit or ld_logits < V       */
    DV_ERR_DTYPE = 3,        /* unknown logits dtype                               */
    DV_ERR_ALIAS = 4,        /* an output overlaps an input or another output      */
    DV_ERR_WORKSPACE = 5,    /* workspace missing, too small or misaligned         */
    DV_ERR_HIP = 6           /* a HIP launch or runtime call failed                */
} dv_status;

typedef enum dv_dtype {
    DV_F32 = 0,              /* IEEE binary32 logits                               */
    DV_BF16 = 1              /* bfloat16 logits (high half of a binary32)          */
} dv_dtype;

/*
 * dv_align_workspace_bytes -- device workspace dv_align / dv_align_eos need
 * for `num_states` states and `num_tokens` tokens (the compacted transition
 * table, the byte-class map and per-token byte classes).  Returns 0 when a
 * size is outside its limit.
 */
DV_API size_t dv_align_workspace_bytes(int32_t num_states, int32_t num_tokens);

/*
 * dv_align -- the vocabulary alignment table (Sec. 3.3, Algorithm 2, at
 * full depth as in Sec. 3.5).
 *
 * For every state s in [0, S) and every token t in [0, V):
 *     next_state[s*V + t] = the state reached by reading the bytes of token t
 *                           one by one from s, or DV_DEAD if a transition on
 *                           the way is dead (the walk stops there);
 *     bit (t % 32) of allow[s*W + t/32] = 1 exactly when next_state != DV_DEAD,
 * with W = ceil(V/32).  Bits for t >= V are written as 0.  A zero-length
 * token leaves the state unchanged (next_state = s, allowed).
 *
 * Inputs (device, read only):
 *   trans      [S][256] int32, row-major: trans[s*256 + b] is the move of
 *              state s on byte b.  Values outside [0, S) read as DV_DEAD.
 *   offsets    [V+1] int32, offsets[0] = 0, non-decreasing, offsets[V] <=
 *              the size of bytes (a precondition this call does not check:
 *              dv_validate_vocab does): token t is bytes[offsets[t] ..
 *              offsets[t+1]); a decreasing pair reads as an empty token.
 *   bytes      [offsets[V]] uint8, the concatenated token strings.  May be
 *              NULL only when every token is empty.
 * Outputs (device, written in full):
 *   next_state [S][V] int32; allow [S][W] uint32.
 * Workspace: at least dv_align_workspace_bytes(S, V) bytes of device memory,
 *   256-byte aligned; contents on entry are ignored, on exit undefined.
 * Errors: DV_ERR_INVALID_ARG (NULL pointer), DV_ERR_SHAPE (S or V out of
 *   range), DV_ERR_ALIAS (next_state/allow overlap each other or an input,
 *   checked on the address ranges implied by S and V), DV_ERR_WORKSPACE,
 *   DV_ERR_HIP.
 */
DV_API dv_status dv_align(const int32_t *trans, int32_t num_states,
                   const int32_t *offsets, const uint8_t *bytes, int32_t num_tokens,
                   int32_t *next_state, uint32_t *allow,
                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_align_eos -- dv_align with an end-of-sequence token (Algorithm 1 stops
 * on EOS; Sec. 3.2 treats EOS as one more terminal of the scanner, so it may
 * follow wherever a terminal sequence may end).
 *
 * Every token except `eos_token` is aligned exactly as by dv_align.  For the
 * EOS column (its bytes are ignored):
 *     next_state[s*V + eos_token] = s        if accepting[s] != 0,
 *                                   DV_DEAD  otherwise,
 * with the allow bit set exactly when it is not DV_DEAD, so the masked step
 * can choose EOS only where the constraint may end; the state is left
 * unchanged and the caller stops decoding the sequence.
 *
 * accepting  [S] uint8 (device), nonzero for states where the constraint may
 *            end (accepting states; the start state if the empty output is
 *            valid).  NULL means no state accepts: EOS is never allowed.
 * eos_token  in [0, V).
 * Workspace, outputs and errors as dv_align (DV_ERR_SHAPE also for an
 * eos_token outside [0, V)).
 */
DV_API dv_status dv_align_eos(const int32_t *trans, int32_t num_states,
                       const int32_t *offsets, const uint8_t *bytes, int32_t num_tokens,
                       const uint8_t *accepting, int32_t eos_token,
                       int32_t *next_state, uint32_t *allow,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_validate_vocab -- checks the CSR layout of a vocabulary on the device:
 * the precondition of dv_align / dv_align_eos, whose kernels read
 * bytes[offsets[t] .. offsets[t+1]) without bounds checks.
 *
 * Writes to *first_bad (device, one int32) -1 when offsets[0] = 0, offsets
 * is non-decreasing and offsets[V] <= num_bytes; otherwise the smallest t
 * in [0, V] at which that fails (t = 0: offsets[0] != 0; t >= 1:
 * offsets[t] < offsets[t-1] or offsets[t] > num_bytes).  The result is
 * valid once the stream has reached the call.
 *
 * offsets    [V+1] int32 (device), num_tokens = V in [1, DV_MAX_TOKENS];
 * num_bytes  the number of bytes the caller's bytes array holds (>= 0).
 * (dv_align itself reads a decreasing pair as an empty token, never as
 * anything else; bytes past the array are the case only this check
 * catches.)
 * Errors: DV_ERR_INVALID_ARG (NULL), DV_ERR_SHAPE, DV_ERR_ALIAS (first_bad
 *   inside offsets), DV_ERR_HIP.
 */
DV_API dv_status dv_validate_vocab(const int32_t *offsets, int32_t num_tokens, int64_t num_bytes,
                                   int32_t *first_bad, void *stream);

/*
 * dv_masked_step_workspace_bytes -- device workspace dv_masked_step needs for
 * `batch` rows of `num_tokens` logits, for either dtype: where a row is
 * split over several blocks, they meet there (up to four blocks per row in
 * pairs, one 64-bit word per pair; more through a running maximum and an
 * arrival count per row; the block that finishes the row writes its
 * outputs and puts its words back to zero).  For one num_tokens the size
 * never falls as batch grows: a workspace made for a batch serves every
 * smaller one.  Returns 0 when a size is outside its limit.
 */
DV_API size_t dv_masked_step_workspace_bytes(int32_t batch, int32_t num_tokens);

/*
 * dv_masked_step -- one greedy constrained decoding step (Algorithm 1:
 * mask, apply, decode, update; the argmax of Algorithm 3 restricted to the
 * admissible tokens).
 *
 * For every row b in [0, B):
 *     s = states[b];  if s is outside [0, S) the row is dead;
 *     token[b] = the index i in [0, V) with allow bit (s, i) set whose logit
 *                logits[b*ld_logits + i] is largest; ties go to the lowest
 *                index; NaN ranks as -infinity; -0.0 equals +0.0;
 *                -1 when the row is dead or has no allowed token;
 *     new_state[b] = next_state[s*V + token[b]], or DV_DEAD when token = -1.
 *
 * Inputs (device, read only):
 *   next_state [S][V] int32 and allow [S][ceil(V/32)] uint32 as written by
 *              dv_align (any table with that layout is accepted; new_state
 *              is read from it as is).
 *   states     [B] int32.
 *   logits     [B][ld_logits] of `dtype` (dv_dtype), row stride ld_logits
 *              elements (ld_logits >= V); the pointer must be aligned to
 *              the element size.  Rows of any such alignment take the
 *              vector path (the elements before the row's first 16-byte
 *              boundary are read one by one).
 * Outputs (device): token [B] int32, new_state [B] int32.  They must not
 *   overlap each other or any input (callers ping-pong two state buffers).
 * Workspace: at least dv_masked_step_workspace_bytes(B, V) bytes of device
 *   memory, 256-byte aligned, all zero before its first use (clear it once,
 *   e.g. with hipMemset); every call leaves it all zero again, so it can be
 *   reused by any later call of any size without clearing.  Calls that share
 *   a workspace must be ordered on one stream.
 * B = 0 is valid and enqueues nothing; states, logits, token and new_state
 *   may then be NULL (the pointers of empty tensors).
 * Errors: DV_ERR_INVALID_ARG (also for logits not aligned to the element
 *   size), DV_ERR_SHAPE (S, V, B out of range or ld_logits < V),
 *   DV_ERR_DTYPE, DV_ERR_ALIAS, DV_ERR_WORKSPACE, DV_ERR_HIP.
 */
DV_API dv_status dv_masked_step(const int32_t *next_state, const uint32_t *allow,
                         int32_t num_states, int32_t num_tokens,
                         const int32_t *states, const void *logits, int32_t dtype,
                         int32_t batch, int64_t ld_logits,
                         int32_t *token, int32_t *new_state,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_masked_step_noalloc -- dv_masked_step without a workspace argument, for
 * callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation).  Results are
 * exactly those of dv_masked_step.
 *
 * Split rows meet in a scratch array the library holds on each GPU it runs
 * on (768 KiB, enough for DV_NOALLOC_MAX_BATCH rows; kept until the process
 * ends).  The first call on a device looks the array up and enqueues a
 * kernel on `stream` that clears it; every call leaves it all zero.  The
 * call allocates nothing.  All calls on one GPU share the array: calls that
 * may overlap on one GPU (other streams, other threads) race and must be
 * ordered by the caller; give concurrent work dv_masked_step with a
 * workspace each.
 *
 * Arguments as dv_masked_step, without workspace and workspace_bytes.
 * Errors as dv_masked_step; DV_ERR_SHAPE also for batch >
 *   DV_NOALLOC_MAX_BATCH; DV_ERR_HIP if the scratch array cannot be found or
 *   cleared.
 */
DV_API dv_status dv_masked_step_noalloc(const int32_t *next_state, const uint32_t *allow,
                         int32_t num_states, int32_t num_tokens,
                         const int32_t *states, const void *logits, int32_t dtype,
                         int32_t batch, int64_t ld_logits,
                         int32_t *token, int32_t *new_state, void *stream);

/*
 * dv_masked_step_opportunistic -- dv_masked_step with opportunistic masking
 * (Sec. 3.5, further optimizations): the model's own greedy choice over all
 * V logits is found first, without reading the mask, and checked against
 * the mask; only when it is not allowed is the masked choice computed.
 *
 * The outputs are exactly those of dv_masked_step (an allowed overall
 * maximum at the lowest index is also the masked one), so the two are
 * interchangeable; this one reads less memory when the model mostly picks
 * allowed tokens and reads a row twice when it does not.  The check runs
 * first for bf16 rows of batches >= 256, or >= 64 with rows of at most 32768
 * tokens, where one block covers a row (always for rows of at most 24576
 * tokens); other shapes (fp32 rows, rows split over several blocks) take
 * dv_masked_step's kernels.
 * Arguments, workspace (dv_masked_step_workspace_bytes) and errors as
 *   dv_masked_step.
 */
DV_API dv_status dv_masked_step_opportunistic(const int32_t *next_state, const uint32_t *allow,
                         int32_t num_states, int32_t num_tokens,
                         const int32_t *states, const void *logits, int32_t dtype,
                         int32_t batch, int64_t ld_logits,
                         int32_t *token, int32_t *new_state,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_masked_sample_workspace_bytes -- device workspace dv_masked_sample needs
 * for `batch` rows of `num_tokens` logits; for one num_tokens it never falls
 * as batch grows.  Returns 0 when a size is outside its limit.
 */
DV_API size_t dv_masked_sample_workspace_bytes(int32_t batch, int32_t num_tokens);

/*
 * dv_masked_sample -- one sampled constrained decoding step (Algorithm 1's
 * decode "argmax or sample"; the paper samples at temperature 1.0, Sec. 4).
 *
 * For every row b with a live state s (as dv_masked_step), the token is
 * drawn from softmax(logits / T) restricted to the allowed tokens, as the
 * Gumbel-max choice
 *     token[b] = argmax over allowed i of  fma(x_i, inv_temperature, G_i)
 * in binary32 (x_i the logit, widened exactly from bf16), NaN ranking as
 * -infinity and ties going to the lowest index, with the noise
 *     G_i = -ln(-ln U_i),  U_i = (2 (w >> 9) + 1) 2^-24,
 *     w = word (i mod 4) of Philox4x32-10 (Salmon et al., SC 2011) with
 *         key (seed mod 2^32, seed >> 32) and
 *         counter (i / 4, b, offset mod 2^32, offset >> 32),
 * and ln evaluated in binary32 by fixed IEEE steps (x = m 2^e with m in
 * [sqrt(1/2), sqrt(2)); z = (m - 1) r, r = 1/(m + 1) by four Newton steps
 * t = fma(-d, r, 1), r = fma(r, t, r) from r = 1/2; ln m = 2 h with
 * h = fma(z^3, p, z), p = 1/3 + w (1/5 + w (1/7 + w/9)) by fused
 * multiply-adds, w = z^2; ln x = fma(e, ln 2, ln m)), so the draw is the
 * same on every device.  new_state[b] = next_state[s*V + token[b]]; a dead
 * row or a row with nothing allowed gives token -1 and DV_DEAD.  Rows are
 * independent draws; use a different `offset` for every step (the pair
 * (seed, offset) names one draw of the whole batch).
 *
 * inv_temperature = 1/T, finite and > 0 (T -> 0 approaches dv_masked_step).
 * Other arguments and errors as dv_masked_step (DV_ERR_SHAPE also for a
 * bad inv_temperature); workspace: dv_masked_sample_workspace_bytes(B, V),
 * zero before its first use and left zero, as for dv_masked_step.
 */
DV_API dv_status dv_masked_sample(const int32_t *next_state, const uint32_t *allow,
                         int32_t num_states, int32_t num_tokens,
                         const int32_t *states, const void *logits, int32_t dtype,
                         int32_t batch, int64_t ld_logits, float inv_temperature,
                         uint64_t seed, uint64_t offset,
                         int32_t *token, int32_t *new_state,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_spec_walk -- speculative chain check (Sec. 3.6): how many of a row's
 * proposed tokens the constraint admits, one after the other.
 *
 * For every row b in [0, B), with s = num_proposed proposals
 * p_j = proposals[b*ld_proposals + j] and q_0 = states[b] (DV_DEAD if
 * outside [0, S)):
 *     p_j is admitted when q_j is a state in [0, S), p_j is in [0, V) and
 *         the allow bit (q_j, p_j) is set; then q_{j+1} = next_state[q_j*V + p_j];
 *     accepted[b]    = the number a of leading admitted proposals;
 *     final_state[b] = the table entry reached by the last admitted proposal
 *                      (q_0 when a = 0).
 * Proposal ids outside [0, V) are not errors: they are not admitted.
 *
 * Inputs (device, read only): next_state, allow, states as for
 *   dv_masked_step; proposals [B][ld_proposals] int32 (ld_proposals >= s;
 *   may be NULL when s = 0).
 * Outputs (device): accepted [B], final_state [B] int32; they must not
 *   overlap each other or any input.  No workspace.
 * B = 0 is valid and enqueues nothing (then only next_state and allow must
 *   be non-NULL).
 * Errors: DV_ERR_INVALID_ARG, DV_ERR_SHAPE (S, V, B or s out of range,
 *   ld_proposals < s), DV_ERR_ALIAS, DV_ERR_HIP.
 */
DV_API dv_status dv_spec_walk(const int32_t *next_state, const uint32_t *allow,
                       int32_t num_states, int32_t num_tokens,
                       const int32_t *states, const int32_t *proposals,
                       int32_t num_proposed, int64_t ld_proposals, int32_t batch,
                       int32_t *accepted, int32_t *final_state, void *stream);

/*
 * dv_spec_verify_workspace_bytes -- device workspace dv_spec_verify needs for
 * `batch` rows of `num_proposed` proposals over `num_tokens` logits (the
 * state of every position and the masked step's meeting entries).  Returns 0
 * when a size is outside its limit.
 */
DV_API size_t dv_spec_verify_workspace_bytes(int32_t batch, int32_t num_proposed,
                                             int32_t num_tokens);

/*
 * dv_spec_verify -- verification of proposed tokens with greedy decoding
 * (Sec. 3.6: the model scores all proposed positions in one pass and the
 * proposals it does not confirm are discarded; its choice at a position is
 * the masked greedy decode of Algorithm 1).
 *
 * Row b proposes s = num_proposed tokens p_j = proposals[b*ld_proposals + j].
 * The logits the model gives at position j (j = 0 .. s, after reading the
 * first j proposals) are V elements at logits[b*ld_row + j*ld_pos].  With
 * q_j the state after the first j proposals as defined by dv_spec_walk, and
 * DV_DEAD once a proposal was not admitted:
 *     token[b*(s+1) + j] = the masked greedy choice of dv_masked_step in
 *                          state q_j for position j's logits (-1 when q_j is
 *                          DV_DEAD or allows nothing);
 *     accepted[b]        = the first j < s whose choice is -1 or differs from
 *                          p_j, else s: the proposals p_0 .. p_{a-1} agree with
 *                          the model and token[b][0 .. a] are the tokens
 *                          plain greedy decoding emits (a + 1 of them, a if
 *                          token[b][a] = -1);
 *     new_state[b]       = next_state[q_a*V + token[b][a]], or DV_DEAD when
 *                          token[b][a] = -1.
 * The tokens emitted are exactly those of one-step-at-a-time decoding with
 * dv_masked_step on the same logits; an end-of-sequence token among them
 * ends the sequence at that point (the caller truncates there).
 *
 * Inputs (device, read only): next_state, allow, states as for
 *   dv_masked_step; proposals [B][ld_proposals] int32 (ld_proposals >= s;
 *   may be NULL when s = 0; ids outside [0, V) are never confirmed);
 *   logits of `dtype`, aligned to the element size, any non-negative
 *   ld_row and ld_pos (a model's [B][s+1][V] output is ld_row = (s+1)*V,
 *   ld_pos = V).
 * Outputs (device): token [B][s+1], accepted [B], new_state [B] int32; they
 *   must not overlap each other, an input or the workspace.
 * Workspace: at least dv_spec_verify_workspace_bytes(B, s, V) bytes of
 *   device memory, 256-byte aligned, all zero before its first use and left
 *   all zero by every call (as for dv_masked_step).  Calls that share a
 *   workspace must be ordered on one stream.
 * B = 0 is valid and enqueues nothing.
 * Errors: DV_ERR_INVALID_ARG (also for misaligned logits), DV_ERR_SHAPE
 *   (S, V, B or s out of range, B*(s+1) > DV_MAX_BATCH, ld_proposals < s,
 *   a negative or too large stride), DV_ERR_DTYPE, DV_ERR_ALIAS,
 *   DV_ERR_WORKSPACE, DV_ERR_HIP.
 */
DV_API dv_status dv_spec_verify(const int32_t *next_state, const uint32_t *allow,
                         int32_t num_states, int32_t num_tokens,
                         const int32_t *states, const int32_t *proposals,
                         int32_t num_proposed, int64_t ld_proposals,
                         const void *logits, int32_t dtype, int64_t ld_row, int64_t ld_pos,
                         int32_t batch, int32_t *token, int32_t *accepted, int32_t *new_state,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Training under a constraint
 * ---------------------------
 * The calls below take rows instead of sequences: row n (a token position of
 * a batch, `rows` of them in [0, DV_MAX_BATCH]) has an automaton state, and
 * the tokens its state allows are the only ones with a probability:
 *
 *   allow, num_states, states   allow [S][ceil(V/32)] uint32 as written by
 *       dv_align and states [rows] int32: row n's allowed tokens A_n are those
 *       with bit (states[n], v) set; none when states[n] is outside [0, S).
 *       allow = NULL (states then also NULL, num_states 0): every token.
 *
 * What is masked has no effect on any result, whatever its logit (infinities
 * and NaN included).  Elements are of `dtype` (DV_F32 or DV_BF16) and aligned
 * to their size; every array with a row stride ld_* (in elements, at least the
 * row's length) has unit stride along its rows, and rows may start at any
 * alignment.  Products, sums, softmax statistics and losses are in fp32, each
 * result rounded once; no call adds with atomics: the same call gives the same
 * bits.  Workspaces hold nothing between calls and need no clearing; 256-byte
 * aligned; calls that share one must be ordered on one stream.  Outputs must
 * not overlap each other, an input or the workspace, except where said.
 */

/*
 * dv_head_loss_workspace_bytes -- device workspace of dv_head_loss, for
 * operands of any stride and alignment.  Returns 0 when an argument is outside
 * its limit.
 *
 * Operands are multiplied where they lie if hidden is a multiple of 64, their
 * rows start on 16-byte boundaries and are at most 2^20 elements apart; else
 * copies take their place: of x whole, of the weights a piece at a time (2^27 + 2^19
 * rows elements, or 8,192 tokens if those are more).  dv_head_loss_workspace_bytes_for
 * is the workspace of a call with these operands, without copies of what needs
 * none; the pointers are not dereferenced.
 */
DV_API size_t dv_head_loss_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens, int32_t dtype);
DV_API size_t dv_head_loss_workspace_bytes_for(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                                               int32_t dtype, int32_t rows, int32_t hidden, int32_t num_tokens);

/*
 * dv_head_loss -- softmax cross entropy over the allowed tokens, from hidden
 * states and head weights, without the logits in memory.
 *
 * For row n with z_v = sum_d x[n][d] weight[v][d] and t = targets[n]:
 *     lse[n]  = ln sum over v in A_n of exp(z_v), -infinity when A_n is empty;
 *     loss[n] = lse[n] - z_t where t is in A_n; else (t outside [0, V), not
 *               allowed, or a dead row) the row takes no part: loss[n] = 0.
 *
 * x [rows][ld_x], weight [V][ld_weight] of `dtype`; targets [rows] int32.
 * fp32 operands are multiplied as sums of three bf16 parts each: the products
 * of parts below 2^-22 of the whole are left out.  They must be finite and at
 * most 2^127 (1.7e38) in magnitude: an fp32 element beyond, infinities among
 * them, makes NaN of its row's logits (of x) or its token's (of weight), and of
 * no other.  bf16 operands take infinities as they are.
 * loss, lse [rows] fp32.
 * rows = 0 is valid and enqueues nothing.
 * Errors: DV_ERR_INVALID_ARG (NULL, misaligned elements, or only one of allow
 *   and states), DV_ERR_SHAPE, DV_ERR_DTYPE, DV_ERR_ALIAS, DV_ERR_WORKSPACE,
 *   DV_ERR_HIP.
 */
DV_API dv_status dv_head_loss(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight, int32_t dtype,
                              int32_t rows, int32_t hidden, int32_t num_tokens, const int32_t *targets,
                              const uint32_t *allow, int32_t num_states, const int32_t *states,
                              float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_head_loss_backward_workspace_bytes -- device workspace of
 * dv_head_loss_backward, for operands of any stride and alignment: what
 * dv_head_loss copies, G of a piece of the vocabulary (2^27 elements of 4 bytes, or
 * 4,096 tokens if those are more) and the gradients' partial sums.  Returns 0 when an
 * argument is outside its limit.  dv_head_loss_backward_workspace_bytes_for: of
 * a call with these operands.
 */
DV_API size_t dv_head_loss_backward_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens, int32_t dtype);
DV_API size_t dv_head_loss_backward_workspace_bytes_for(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                                                        int32_t dtype, int32_t rows, int32_t hidden,
                                                        int32_t num_tokens);

/*
 * dv_head_loss_backward -- the gradients of sum_n grad_loss[n] loss[n].
 *
 * With G[n][v] = grad_loss[n] (exp(z_v - lse[n]) - [v = targets[n]]) for v in
 * A_n of rows that take part, 0 elsewhere:
 *     grad_x[n]      = sum_v G[n][v] weight[v]     [rows][hidden]
 *     grad_weight[v] = sum_n G[n][v] x[n]          [V][hidden]
 * both contiguous, of `dtype`; either may be NULL and is then not computed.
 * lse [rows] fp32 as dv_head_loss wrote it for the same inputs; grad_loss
 * [rows] fp32.  The logits are computed again a piece at a time.  For bf16
 * inputs G goes into the two products as the sum of two bf16 parts (a relative
 * error below 2^-16 of each term): what the outputs lose is their own rounding.
 * x and weight must be finite.
 * rows = 0 is valid: grad_weight is filled with zeros.
 * Errors as dv_head_loss.
 */
DV_API dv_status dv_head_loss_backward(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                                       int32_t dtype, int32_t rows, int32_t hidden, int32_t num_tokens,
                                       const int32_t *targets, const uint32_t *allow, int32_t num_states,
                                       const int32_t *states, const float *lse, const float *grad_loss, void *grad_x,
                                       void *grad_weight, void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_distill_loss_workspace_bytes -- device workspace of dv_distill_loss and
 * dv_distill_loss_backward (for either dtype).  Returns 0 when an argument is
 * outside its limit.  For one num_top it never falls as rows grow.
 */
DV_API size_t dv_distill_loss_workspace_bytes(int32_t rows, int32_t num_tokens, int32_t num_top);

/*
 * dv_distill_loss -- divergence of a model's distribution over the allowed
 * tokens from a teacher's top logits.
 *
 * With c = inv_temperature = 1/T and row n's entries k in [0, num_top),
 * L_n = {k : teacher_ids[n][k] in A_n and teacher_logits[n][k] > -infinity}:
 *     q_k = softmax of c teacher_logits[n] over L_n,
 *     p_v = softmax of c logits[n] over A_n,
 *     loss[n] = sum over L_n of q_k (ln q_k - ln p_{id_k}).
 * An id listed more than once counts with the sum of its entries.  Where L_n is
 * empty, or no allowed logit is above -infinity, the row takes no part: loss 0.
 *
 * logits [rows][ld_logits] of `dtype`; teacher_ids [rows][num_top] int32 (ids
 * outside [0, V) take no part), teacher_logits [rows][num_top] fp32; loss
 * [rows] fp32.  inv_temperature > 0 and at most 2.3e38 (its product
 * with log2(e), in fp32, has to be finite).
 * rows = 0 is valid and enqueues nothing.
 * Errors as dv_head_loss.
 */
DV_API dv_status dv_distill_loss(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows,
                                 int32_t num_tokens, const int32_t *teacher_ids, const float *teacher_logits,
                                 int32_t num_top, float inv_temperature, const uint32_t *allow, int32_t num_states,
                                 const int32_t *states, float *loss, void *workspace, size_t workspace_bytes,
                                 void *stream);

/*
 * dv_distill_loss_backward -- the gradient of sum_n grad_loss[n] loss[n], and
 * the loss with it, in one call (a training step needs no dv_distill_loss):
 *     grad[n][v] = grad_loss[n] c (p_v - sum of q_k with id_k = v)  on A_n,
 *                  0 elsewhere and on rows that take no part.
 * grad [rows][ld_grad] of `dtype`; it may be the logits themselves (the same
 * address and row stride), which are then overwritten.  loss may be NULL;
 * grad_loss [rows] fp32.  Other arguments and errors as dv_distill_loss.
 */
DV_API dv_status dv_distill_loss_backward(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows,
                                          int32_t num_tokens, const int32_t *teacher_ids,
                                          const float *teacher_logits, int32_t num_top, float inv_temperature,
                                          const uint32_t *allow, int32_t num_states, const int32_t *states,
                                          const float *grad_loss, float *loss, void *grad, int64_t ld_grad,
                                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_embed -- rows of a table by token, scaled:
 *     out[n] = scale weight[ids[n]], zeros where ids[n] is outside [0, V).
 * weight [V][ld_weight] and out [rows][hidden] (contiguous) of `dtype`, ids
 * [rows] int32.  rows = 0 is valid and enqueues nothing.
 * Errors as dv_head_loss (no workspace; DV_ERR_SHAPE also for a scale that is
 *   not finite).
 */
DV_API dv_status dv_embed(const void *weight, int64_t ld_weight, int32_t dtype, int32_t num_tokens, int32_t hidden,
                          const int32_t *ids, int32_t rows, float scale, void *out, void *stream);

/*
 * dv_embed_backward_workspace_bytes -- device workspace of dv_embed_backward;
 * for one hidden it never falls as rows grow.  Returns 0 when an argument is
 * outside its limit.
 */
DV_API size_t dv_embed_backward_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens);

/*
 * dv_embed_backward -- the table's gradient, rows added in their order:
 *     grad_weight[v] = scale * (sum over n with ids[n] = v of grad_out[n]),
 * zeros for tokens that no row names; with accumulate != 0 added to what
 * grad_weight holds (a table shared with the head: after
 * dv_head_loss_backward), and rows of tokens that no row names stay as they are.
 * grad_out [rows][ld_grad_out] and grad_weight [V][hidden] (contiguous) of
 * `dtype`.  rows = 0 is valid: zeros, or nothing with accumulate.
 * Errors as dv_embed, and DV_ERR_WORKSPACE.
 */
DV_API dv_status dv_embed_backward(const void *grad_out, int64_t ld_grad_out, int32_t dtype, int32_t rows,
                                   int32_t hidden, const int32_t *ids, int32_t num_tokens, float scale,
                                   int32_t accumulate, void *grad_weight, void *workspace, size_t workspace_bytes,
                                   void *stream);

/*
 * From the last layer to the logits
 * ---------------------------------
 * The calls below lead from a model's last hidden states to the logits that the
 * steps above decode from (and, with their gradients, from the head loss back to
 * the last layer).  Conventions are those of the training calls: rows of any
 * stride and alignment where a stride is an argument, sums in fp32, each result
 * rounded once, the same call the same bits, no atomics in memory.
 *
 * 8-bit operands.  An e4m3 matrix (the OCP format: largest 448, no infinities,
 * NaN 0x7F) of n rows over k columns is stored as rows of K bytes, K the next
 * multiple of 128 of k, zeros beyond k, with fp32 scales:
 *   by rows    one for each row and 128 columns, stored [K/128][n];
 *   by tiles   one for each 128 rows and 128 columns, stored [ceil(n/128)][K/128].
 * A block of values x is quantized as
 *     scale = max(largest |x| of the block, 2^-100) / 448   (in fp32)
 *     q     = the e4m3 value nearest to the fp32 quotient x / scale, ties to even;
 * a block that holds an infinity or a NaN becomes NaN, its scale too.  A zero of
 * either sign becomes +0; what rounds to zero keeps its sign.
 */

/*
 * dv_rms_norm -- root-mean-square norm with the residual's addition.
 *
 * For every row, with D = hidden:
 *     h    = x + residual, rounded to the type (h = x where residual is NULL)
 *     rstd = 1 / sqrt(sum_d h_d^2 / D + eps)
 *     y_d  = h_d rstd weight_d
 *
 * x, residual [rows][ld_*], weight [D] of `dtype`.  Outputs, each NULL if not
 * wanted, contiguous: total [rows][D] = h of `dtype`; out [rows][D] = y of
 * `dtype`; rstd [rows] fp32; q and scales (both or none) = y as an 8-bit operand by
 * rows, quantized from fp32.  q 8-byte aligned.  total may be the residual or x
 * itself (the same address, row stride D).  At least one of out and q is wanted.
 * eps >= 0 and finite.  A row of zeros with eps = 0 gives NaN.  rstd is infinite where it
 * passes fp32's largest (a root mean square below 2^-128, eps = 0 or hardly more): out is
 * as defined there, the gradients are not.
 * rows = 0 is valid and enqueues nothing.
 * Errors as dv_head_loss (no workspace).
 */
DV_API dv_status dv_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, const void *weight,
                             int32_t dtype, int32_t rows, int32_t hidden, float eps, void *total, void *out, float *rstd,
                             void *q, float *scales, void *stream);

/*
 * dv_rms_norm_backward_workspace_bytes -- device workspace of
 * dv_rms_norm_backward; for one hidden it never falls as rows grow.  Returns 0
 * when an argument is outside its limit.
 */
DV_API size_t dv_rms_norm_backward_workspace_bytes(int32_t rows, int32_t hidden);

/*
 * dv_rms_norm_backward -- gradients of sum(grad_out y) + sum(grad_total h).
 *
 *     grad_x      = rstd g - h rstd^3 / D (sum_d g_d h_d) + grad_total,  g = grad_out weight
 *                   [rows][D]: the gradient of x, and of the residual
 *     grad_weight = sum over rows of grad_out h rstd   [D]
 * both contiguous, of `dtype`; either may be NULL and is then not computed.
 * total [rows][ld_total]: h as dv_rms_norm wrote it (x where there was no
 * residual), rstd as it wrote it; grad_total [rows][ld_grad_total] or NULL
 * (zeros): what reaches h past the norm.
 * rows = 0 is valid: grad_weight is filled with zeros.
 * Errors as dv_head_loss.
 */
DV_API dv_status dv_rms_norm_backward(const void *grad_out, int64_t ld_grad_out, const void *total, int64_t ld_total,
                                      const void *weight, const float *rstd, const void *grad_total,
                                      int64_t ld_grad_total, int32_t dtype, int32_t rows, int32_t hidden, void *grad_x,
                                      void *grad_weight, void *workspace, size_t workspace_bytes, void *stream);

/*
 * dv_quantize_f8 -- a matrix as an 8-bit operand: as it lies, transposed, or both.
 *
 * x [rows][ld_x] of `dtype`, `cols` columns.  tile = 1: by rows; tile = 128: by
 * tiles.  q [rows][up(cols)] with scales; t_q [cols][up(rows)] with t_scales is
 * the operand of the transposed matrix (by rows: blocks of 128 rows of a column);
 * up(): the next multiple of 128.  One of the pairs may be NULL.  q and t_q 16-byte aligned.
 * rows in [0, DV_MAX_TOKENS], cols in [1, DV_MAX_TOKENS], fewer than 2^24 tiles
 * of 128 x 128.  rows = 0 is valid and enqueues nothing.
 * Errors as dv_head_loss (no workspace; DV_ERR_SHAPE for another tile).
 */
DV_API dv_status dv_quantize_f8(const void *x, int64_t ld_x, int32_t dtype, int32_t rows, int32_t cols, int32_t tile,
                                void *q, float *scales, void *t_q, float *t_scales, void *stream);

/*
 * dv_product_f8_workspace_bytes -- device workspace of dv_product_f8 (sums of
 * parts of a long depth) with these sizes.  Returns 0 when an argument is outside its limit, and
 * may return 0 otherwise: then none is needed.  It falls where more rows fill the
 * card without parts: a workspace for calls of different rows takes the next query.
 */
DV_API size_t dv_product_f8_workspace_bytes(int32_t rows, int32_t cols, int32_t depth);

/*
 * dv_product_f8_workspace_bytes_up_to -- device workspace that serves
 * dv_product_f8 with any rows up to `rows`; for one cols and depth it never falls
 * as rows grow.  (It looks at every 128 rows: a question for when memory is
 * laid out, up to some milliseconds at 2^20 rows.)  0 as above.
 */
DV_API size_t dv_product_f8_workspace_bytes_up_to(int32_t rows, int32_t cols, int32_t depth);

/*
 * dv_product_f8 -- the matrix product of two 8-bit operands:
 *     out[m][n] = sum over blocks kb of a_scales(kb, m) b_scales(kb, n)
 *                 * (sum over the block's 128 k of a[m][k] b[n][k]).
 *
 * a [rows][ld_a] with scales by rows; b [cols][ld_b] with scales by rows (tile =
 * 1) or by tiles (tile = 128); depth: a multiple of 128.  Row starts on 16-byte
 * boundaries (ld_* multiples of 16, at least depth and at most DV_MAX_DEPTH).
 * out [rows][ld_out] of `dtype`.  A head's logits: a the hidden states, b the
 * weights by tiles.  Gradients of out = x w^T: of x, a = the gradient's q, b = w's
 * t_q by tiles; of w, a = the gradient's t_q, b = x's t_q by rows.
 * Scales of any size: what fp32 can hold is not lost where a_scales b_scales, or a
 * block's sum under one of them, would leave its range (a tile of results that meets
 * such scales is summed twice).
 * Products of fp32 results, and of bf16 results of at most 256 rows, are exact and
 * their sums in fp32; with dtype DV_BF16 | DV_EXACT_SUMS those of more rows are too, at about
 * half the rate.  bf16 results of more rows without it: of eight neighbouring products
 * what lies below 2^-13 of the largest is cut off before the sum (at most 7 * 2^-13
 * of the magnitudes; 1.4e-5 of a sum of normal values, before the result's
 * rounding by 2^-9).
 * rows = 0 is valid and enqueues nothing; rows * cols < 2^36.
 * Errors as dv_head_loss.
 */
DV_API dv_status dv_product_f8(const void *a, int64_t ld_a, const float *a_scales, const void *b, int64_t ld_b,
                               const float *b_scales, int32_t tile, int32_t rows, int32_t cols, int32_t depth,
                               int32_t dtype, void *out, int64_t ld_out, void *workspace, size_t workspace_bytes,
                               void *stream);

/*
 * dv_adjust_logits -- logits with each sequence's penalties, biases and mask.
 *
 * Row n's history is history[n*ld_history ..] of lengths[n] tokens (clamped to
 * [0, max_history]), the first prompt_lengths[n] of them its prompt (NULL: none),
 * the others its output; ids outside [0, V) take no part.  For a token v with
 * logit z, in fp32:
 *     v in the history:        z = z / repetition[n] if z > 0, else z * repetition[n]
 *     v c > 0 times in the output:  z = z - c frequency[n] - presence[n]
 *     then                     z = z + the sum of bias[n][i] over the i, in their
 *                              order, with bias_ids[n][i] = v
 *     v not allowed:           z = -infinity, whatever it was
 * rounded once to the type; a token that nothing names keeps its logit's bits.
 *
 * logits [rows][ld_logits], out [rows][ld_out] of `dtype`; out may be the logits
 * themselves (the same address and stride): then, without a mask, only the tokens
 * that something names are read and written.  history [rows][ld_history] int32
 * (NULL with max_history 0), lengths, prompt_lengths [rows] int32, repetition (> 0),
 * presence, frequency [rows] fp32, each NULL for none; bias_ids [rows][num_bias]
 * int32 and bias [rows][num_bias] fp32, contiguous; allow, num_states, states as
 * for the training calls (NULL: every token is allowed).
 * rows * ceil(V / 4096) < 2^24.  rows = 0 is valid and enqueues nothing.
 * Errors as dv_head_loss (no workspace).
 */
DV_API dv_status dv_adjust_logits(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows, int32_t num_tokens,
                                  const int32_t *history, int64_t ld_history, int32_t max_history, const int32_t *lengths,
                                  const int32_t *prompt_lengths, const float *repetition, const float *presence,
                                  const float *frequency, const int32_t *bias_ids, const float *bias, int32_t num_bias,
                                  const uint32_t *allow, int32_t num_states, const int32_t *states, void *out,
                                  int64_t ld_out, void *stream);

/* Static, human-readable name of a status code ("DV_OK", ...). */
DV_API const char *dv_status_string(int32_t status);

/* Detail of the last error returned on the calling thread ("" if none).
 * The string stays valid until the next dv_* call on that thread. */
DV_API const char *dv_last_error(void);

/* Library ABI version: major * 10000 + minor * 100 + patch. */
DV_API int32_t dv_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DV_H */
