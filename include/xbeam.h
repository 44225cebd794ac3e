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

#ifdef __cplusplus
}
#endif
#endif
