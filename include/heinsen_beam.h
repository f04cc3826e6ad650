/*
 * libheinsen_scan -- C ABI of beam search over models whose memory is a pool of states (heinsen_attention.h, heinsen_delta.h):
 * the choice of the next beams, and the states that follow them.
 */
#ifndef HEINSEN_BEAM_H_
#define HEINSEN_BEAM_H_

#include "heinsen_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * For each of `batch` groups of `beams` beams: the `keep` best of the beams * vocabulary candidates
 *
 *         value(w, n) = scores[w] + logits[w, n] - log sum_m exp(logits[w, m])
 *
 * best first, equal ones in the order of w * vocabulary + n (of one beam, larger logits first where only their values are equal).
 * A beam with ended[w] != 0 goes on with the token end_token alone, at value scores[w]; its other candidates count as -inf.  So do all
 * candidates of a beam whose score is not finite or whose logits have no finite log-sum (a NaN or +inf among them, or nothing but
 * -inf).  Candidates of -inf fill up where there are no others.
 *
 * logits: float32 or bf16 [batch, beams, vocabulary], the last dimension contiguous, strides of the others in elements; scores
 * float32 [batch, beams] and ended (1 byte each, or NULL) contiguous.  Outputs, contiguous [batch, keep]: out_scores float32, out_parents
 * (the beam w) and out_tokens (n) int32.  1 <= beams <= 64, 1 <= keep <= 64, keep <= beams * vocabulary, vocabulary <= 2^31 - 2^20;
 * 0 <= end_token < vocabulary where ended is given.  Values are formed and compared in 64 bits, with log-sums whose exponentials are
 * float32's own, up to 32 of them added in float32 and those sums in 64 bits: a log-sum is off by less than 2^-18, whatever the logits.
 * Beams of a call that have the same logits have the same log-sum to the last bit, wherever their rows begin.
 * workspace: 256-byte aligned scratch of heinsen_beam_workspace_bytes.  Asynchronous on `stream`.
 */
typedef struct {
    int64_t batch, vocabulary;
    int32_t beams, keep;
    hs_dtype dtype; /* of logits */
    const void* logits;
    int64_t batch_stride, beam_stride;
    const float* scores;
    const uint8_t* ended;
    int64_t end_token;
} heinsen_beam_problem;

hs_status heinsen_beam_select(const heinsen_beam_problem* p, float* out_scores, int32_t* out_parents, int32_t* out_tokens, void* workspace,
                              size_t workspace_bytes, void* stream);
/* 0 for sizes the library does not accept. */
size_t heinsen_beam_workspace_bytes(const heinsen_beam_problem* p);

/*
 * The states follow their beams, in place: row slots[b, w] of the pool becomes what row slots[b, parents[b, w]] held before the call,
 * for every beam w of every group b (slots NULL: beam w of group b has row b * beams + w).  state: [pool, row_bytes], contiguous;
 * parents, slots: int32 [batch, beams].  No two beams of a call may share a row.  A beam whose parent is not one of 0 .. beams - 1, or whose own or
 * parent's slot is negative or >= pool, keeps what it has.  1 <= beams <= 64.  A row that is its own parent's is neither read nor written.
 * Asynchronous; no workspace.
 */
hs_status heinsen_beam_reorder(void* state, int64_t pool, int64_t row_bytes, const int32_t* parents, const int32_t* slots, int64_t batch,
                               int32_t beams, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HEINSEN_BEAM_H_ */
