/*
 * libheinsen_scan -- C ABI of the delta rule with a decay: the recurrence of heinsen_attention.h, where every token first takes
 * out of the state what it already answers for the token's key.
 *
 *         S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T ,   o_t = scale * S_t^T q_t ,   a_t = exp(log_a_t)
 *
 * Conventions are those of heinsen_attention.h (tensors, strides, shared heads, states, lengths, workspaces).  Beyond them
 *   - beta is float32, given by its strides for (batch, token, head); any finite number is taken.  The recurrence does not grow
 *     where 0 <= beta_t |k_t|^2 <= 2 and decays lie between 0 and 1; layers of this kind have keys of length one and beta in 0..1 or
 *     0..2.  Outside of that values grow from token to token, as the formula says.
 *   - Tokens are worked on in chunks of up to 64: what is said there of 128 tokens (decays above one, what a NaN spoils) holds
 *     for 64.
 *   - Products are formed on the tensor cores from bf16 terms.  Float32 tensors count with 24 bits (three terms a factor).  Of
 *     bf16 tensors states, the writes v - a S^T k and the gradients of the gates, of v and of state0 count with 24 bits, what meets a
 *     query or a key in o, dq and dk (the state, its gradient, the weights between a chunk's tokens) with 16.  A float32 number beyond 3.38e38 in magnitude counts as infinite, one below 2^-100 may count as zero.
 */
#ifndef HEINSEN_DELTA_H_
#define HEINSEN_DELTA_H_

#include "heinsen_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    heinsen_attention_problem a;  /* q, k, v, log_a, state0, lengths and sizes */
    heinsen_attention_tensor beta;
} heinsen_delta_problem;

/* o_t for every token of every sequence and the state after the last one, as heinsen_attention_forward. */
hs_status heinsen_delta_forward(const heinsen_delta_problem* p, const heinsen_attention_tensor* o, float* state, void* workspace,
                                size_t workspace_bytes, void* stream);

/*
 * The gradients of every input, as heinsen_attention_backward.  dbeta: float32 [batch, tokens, heads], contiguous.  dlog_a, dbeta
 * and dstate0 may be NULL.
 */
hs_status heinsen_delta_backward(const heinsen_delta_problem* p, const heinsen_attention_tensor* d_o, const float* d_state, void* dq,
                                 void* dk, void* dv, float* dlog_a, float* dbeta, float* dstate0, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Scratch in bytes for either call on these very tensors (what TMA cannot load is laid out anew there); 0 for sizes the library
 * does not accept.  Of each (batch, head) pair a chunk of 64 tokens takes 27 KB forward and 243 KB backward where keys and values are 128
 * wide and bf16 (47 KB of weights, the state before the chunk and its gradient after it 64 KB each, the errors and theirs 32 KB each, sums
 * 4 KB), and a backward call room for a copy of dO: 1.06 GB for 8 x 2048 tokens of 16 heads.  Nothing is kept between the calls. */
size_t heinsen_delta_workspace_bytes(const heinsen_delta_problem* p, int backward);

/* As heinsen_attention_check, for the calls of this file. */
hs_status heinsen_delta_check(void* stream);

/* One token for each sequence on a pool of states, as heinsen_attention_step. */
hs_status heinsen_delta_step(const heinsen_delta_problem* p, const heinsen_attention_tensor* o, float* pool_state, int64_t pool,
                             const int32_t* slots, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HEINSEN_DELTA_H_ */
