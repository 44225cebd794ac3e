/*
 * Host-side beam-search selection step (section 4.5.1 "Host-side Optimization", paragraph "Beam Search
 * Optimization"): out of the beam_width * top_k candidate continuations of a request's beam_width
 * sequences, pick the beam_width best and return them in descending order of score.  xbeam_select
 * runs on the CPU: every pointer of it is a HOST pointer.  The candidates come from xbeam_logprobs, which runs
 * on the GPU.  Same status codes and error text (xattn_last_error) as xattn.h.
 */
#ifndef XBEAM_H_
#define XBEAM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* flags */
enum { XBEAM_FULL_SORT = 1,      /* baseline for comparison: score and sort all candidates, no heap, no early exit */
       XBEAM_CHECK_INPUT = 2 };  /* verify the precondition on cand_lp (costs a pass over all candidates) */

/*
 * Candidate (w, k) of request r has score beam_lp[r][w] + cand_lp[r][w][k], added in fp32.  The result
 * is the first beam_width candidates in the order "score descending, then w ascending, then k
 * ascending" (so it is unique, also among equal scores).
 *
 * Method: one min-heap of beam_width entries per request; the sequences are visited in order, each
 * one's candidates in order of k; a candidate that does not beat the heap's worst entry ends the visit
 * of its sequence, since cand_lp[r][w][:] is descending; finally the heap is emptied worst-first into
 * the output from the back.  No allocation after the first call on a thread (the heap is reused), and
 * the outputs are the caller's arrays.
 *
 * beam_lp   HOST fp32 [n_req, beam_width]         log-probability of each live sequence
 * cand_lp   HOST fp32 [n_req, beam_width, top_k]  log-probabilities of its top_k next tokens, DESCENDING
 *                                                 along the last axis; -inf allowed, NaN not
 * cand_tok  HOST int32 [n_req, beam_width, top_k] the tokens, or NULL (then out_tok receives k)
 * out_lp    HOST fp32 [n_req, beam_width]         scores of the selected candidates, descending
 * out_parent HOST int32 [n_req, beam_width]       w of each selected candidate
 * out_tok   HOST int32 [n_req, beam_width]        its token
 * visited   HOST int64 [n_req] or NULL            candidates examined (beam_width * top_k without early exit)
 * Outputs must not overlap inputs.  n_req >= 0, 1 <= beam_width <= 65536, 1 <= top_k <= 65536.
 * Returns XATTN_OK, or XATTN_EINVAL (bad sizes, NULL, or, with XBEAM_CHECK_INPUT, an ascending step or a
 * NaN in cand_lp / beam_lp) with nothing written for the offending request and those after it.
 */
int xbeam_select(const float* beam_lp, const float* cand_lp, const int32_t* cand_tok, int n_req, int beam_width,
                 int top_k, int flags, float* out_lp, int32_t* out_parent, int32_t* out_tok, int64_t* visited);

/*
 * Log-probabilities of rows of logits: of a given token of each row, of its top_k alternatives, and the entropy.  With
 * x_i = scale * logit_i (scale: one over a temperature) and lse = ln sum exp(x_i):
 *     lp_i = x_i - lse        entropy = -sum exp(lp_i) lp_i
 * The alternatives are the first top_k in the order "logit descending, then index ascending"; with rows = n_req * beam_width,
 * top_lp and top_tok are what xbeam_select takes as cand_lp and cand_tok (after a copy to the host).
 *
 * logits    DEVICE [rows, >= vocab] of `dtype`, rows row_stride values apart (any stride from vocab on), aligned to their type
 * dtype     XBEAM_BF16, XBEAM_FP16 or XBEAM_FP32
 * scale     positive, 2^-20 to 2^20
 * tokens    DEVICE int32[rows], with token_lp, or both NULL.  A negative token (padding) gets 0, one from vocab on NaN.
 * token_lp  DEVICE fp32[rows]
 * top_k     0..512, at most vocab; with top_lp DEVICE fp32 [rows, top_k] and top_tok DEVICE int32 [rows, top_k], both NULL for 0
 * lse, entropy  DEVICE fp32[rows], each may be NULL
 * Logits of -inf, or of a type's lowest value, are forbidden tokens: probability 0 beside others, last among the alternatives.  In a row
 * of nothing but -inf, lse is -inf, entropy and log-probabilities are NaN, the alternatives are the first indices.  With +inf in a
 * row, or NaN, lse, entropy and log-probabilities are NaN; a NaN is no alternative: where a row has fewer than top_k others,
 * the rest of top_tok is -1 (top_lp NaN).  Sums are kept in fp32, of differences of logits: how far a row lies from 0 takes no digits of
 * its log-probabilities and entropy, and no log-probability is above 0.
 * rows 1..2^22, vocab 1..2^24.  Asynchronous on `stream`, which it may be captured on.  Where rows are few they are cut into parts, whose
 * results meet in the stream's workspace (xattn_set_workspace; xbeam_logprobs_workspace_bytes: what one call needs of it),
 * with the rules that xattn_decode states.
 */
enum { XBEAM_BF16 = 0, XBEAM_FP16 = 1, XBEAM_FP32 = 2 };
int xbeam_logprobs(const void* logits, int dtype, int64_t row_stride, int rows, int vocab, float scale, const int32_t* tokens,
                   int top_k, float* token_lp, float* top_lp, int32_t* top_tok, float* lse, float* entropy, void* stream);
size_t xbeam_logprobs_workspace_bytes(int rows, int vocab, int top_k);

/*
 * Verification of drafted tokens (speculative decoding: section 4.4.1's m + 1 query tokens are checked with one pass of the model).  A
 * sequence's q_len rows of target logits are the model's behind its last token and behind each of its drafts; row t judges draft t, and the
 * row behind the last draft that stands gives a token of its own.  With p_t = softmax(scale * target row t) and q_t =
 * softmax(draft_scale * draft row t), what the drafts were drawn from:
 *     draft x_t stands if all before it do and u[t] * q_t(x_t) < p_t(x_t)
 *     new token: where draft t falls, from w = max(0, p_t - q_t); where none falls, from w = p behind the last draft
 *                the least i with sum_{j <= i} w_j > u[q_len - 1] * sum_j w_j
 * so that the tokens given are distributed as the target's alone, whatever the drafts.  Without draft logits (draft NULL: drafts looked up
 * in a text, say) q_t is 1 at x_t.  With XBEAM_GREEDY a draft stands if it is the first of row t's largest logits, which is the new token too.
 *
 * target       DEVICE [batch * q_len, >= vocab] of `dtype`, rows target_stride values apart (any stride from vocab on), aligned to their type
 * draft        DEVICE [batch * (q_len - 1), >= vocab] of `dtype`, rows draft_stride apart, or NULL.  Not looked at with XBEAM_GREEDY.
 * dtype        XBEAM_BF16, XBEAM_FP16 or XBEAM_FP32
 * scale, draft_scale  positive, 2^-20 to 2^20 (one over a temperature; draft_scale counts with draft logits only)
 * draft_tokens DEVICE int32 [batch, q_len - 1]; may be NULL with q_len 1.  A token below 0 or from vocab on falls.
 * n_drafts     DEVICE int32 [batch], how many drafts each sequence has (cut to 0 .. q_len - 1), or NULL: q_len - 1.  Rows behind them are not read.
 * uniforms     DEVICE fp32 [batch, q_len], in [0, 1): one for each draft, the last for the new token; may be NULL with XBEAM_GREEDY
 * tokens       DEVICE int32 [batch, q_len]: the drafts that stand, the new token, then -1
 * n_accepted   DEVICE int32 [batch]: drafts that stand; a sequence keeps kv_len - (q_len - 1 - n_accepted) rows of its cache
 * token_lp     DEVICE fp32 [batch, q_len] or NULL: ln p of every token given, 0 behind them
 * Outputs do not overlap the inputs or each other.
 * Logits of -inf are forbidden tokens, and finite ones may have any size.  A target row with +inf or NaN, or of nothing but -inf, has no probabilities: its draft falls, and the new
 * token is -1 (token_lp NaN).  At a draft row without probabilities the draft falls and w = p.  Where rounding alone let a draft fall, p being
 * nowhere above q, w = p.
 * Numerics: whether a draft stands is decided with sums in 32 bits: p and q are off by 2^-20 of them at most, and 2^-25 for every power of two
 * below 1.  The new token's sums are kept in 64 bits, since the borders between tokens lie closer together than 32 bits tell; that of
 * w = max(0, p_t - q_t) is off by 2^-30 of it at most.  Every call with the same inputs gives the same bits.
 * batch 1..4096, q_len 1..16, vocab 1..2^24.  Asynchronous on `stream`, which it may be captured on; takes the stream's workspace
 * (xattn_set_workspace; xbeam_verify_workspace_bytes: what one call needs of it), with the rules that xattn_decode states.
 */
enum { XBEAM_GREEDY = 1 };
int xbeam_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int dtype, int vocab, float scale,
                 float draft_scale, const int32_t* draft_tokens, const int32_t* n_drafts, const float* uniforms, int batch, int q_len,
                 int flags, int32_t* tokens, int32_t* n_accepted, float* token_lp, void* stream);
size_t xbeam_verify_workspace_bytes(int batch, int q_len, int vocab);

#ifdef __cplusplus
}
#endif
#endif
