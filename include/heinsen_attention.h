/*
 * libheinsen_scan -- C ABI of the recurrence with a matrix state, and of the norms around a block built on it.
 *
 * The recurrence x_t = a_t * x_{t-1} + b_t of heinsen_scan.h, with a rank-one b_t and one decay for each head:
 *
 *         S_t = exp(log_a_t) * S_{t-1} + k_t v_t^T ,     o_t = scale * S_t^T q_t ,        S_t : [k_dim, v_dim]
 *
 * (attention without a softmax; "attention with a decay for each head").  As in heinsen_scan.h the decays are given
 * as logarithms and are only ever summed and subtracted before an exponential is taken, so products of many decays
 * neither underflow early nor lose what is near them; log 0 = -inf is a legal decay and forgets the state, whatever it holds.
 *
 * Conventions beyond those of heinsen_scan.h
 *   - Tokens are rows: q [batch, tokens, q_heads, k_dim], k [batch, tokens, k_heads, k_dim],
 *     v [batch, tokens, v_heads, v_dim], o [batch, tokens, heads, v_dim], with the last dimension contiguous and the
 *     strides of the other three given in elements (batch, token, head).
 *   - heads is a multiple of q_heads, k_heads and v_heads; head h reads head h * q_heads / heads of q, and so on.
 *   - Outputs do not overlap inputs, nor each other, but where it is said that they may.
 *   - States are float32, contiguous [.., heads, k_dim, v_dim]; decays are float32.
 *   - 1 <= k_dim, v_dim <= 256; batch, tokens, heads >= 0 with batch * tokens * heads * max(k_dim, v_dim) < 2^62 and
 *     tokens < 2^31 - 2^20, batch * heads < 2^31.
 *   - lengths (optional, int32 [batch]): row b has lengths[b] tokens (clamped to 0..tokens).  What lies behind them is
 *     not part of the sequence: it is never used, whatever it holds; o and the gradients are zero there.
 *   - Decays are meant to lie between 0 and 1.  A positive log decay is taken as it is, as long as every sum of consecutive log
 *     decays within 128 tokens that holds no -inf lies between -40 and 40: factors of such a sum are formed by themselves.
 *   - Tokens are worked on in chunks of up to 128, counted from a sequence's first.  A NaN or an infinity in q, k or v, or a NaN
 *     or +inf in log_a, gives unspecified values in the heads that read it from the beginning of its chunk on: up to 127 tokens
 *     before it, and behind it whatever decays follow, so in other sequences too where several are packed into one row with
 *     decays of zero between them.  Other rows of the batch and other heads are not affected.
 */
#ifndef HEINSEN_ATTENTION_H_
#define HEINSEN_ATTENTION_H_

#include "heinsen_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A [batch, tokens, heads', dim] tensor: base pointer and strides in elements (the last dimension is contiguous). */
typedef struct {
    const void* ptr;
    int64_t batch_stride, token_stride, head_stride;
} heinsen_attention_tensor;

typedef struct {
    int64_t batch, tokens;
    int32_t heads, q_heads, k_heads, v_heads, k_dim, v_dim;
    hs_dtype dtype;      /* of q, k, v, o and their gradients: HS_F32 or HS_BF16 */
    float scale;         /* finite, not zero */
    heinsen_attention_tensor q, k, v;
    heinsen_attention_tensor log_a; /* float32; all three strides: log_a of (batch, token, head); batch and token
                                       stride 0 = one fixed decay for each head */
    const float* state0;            /* [batch, heads, k_dim, v_dim] before the first token, or NULL for zeros */
    const int32_t* lengths;         /* [batch], or NULL */
} heinsen_attention_problem;

/*
 * o_t for every token of every sequence, and the state after the last one (`state`, may be NULL).
 * `state` may be `state0` itself.  o.ptr is written through its strides.  Asynchronous on `stream`.
 * workspace: 256-byte aligned device scratch of heinsen_attention_workspace_bytes(p, 0) bytes.  heinsen_scan_check(workspace,
 * stream) returns HS_ERR_COPY_TIMEOUT where a bounded wait of the last call on it ran out: its outputs are not valid then.
 */
hs_status heinsen_attention_forward(const heinsen_attention_problem* p, const heinsen_attention_tensor* o, float* state,
                                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradients of every input.  d_o is the gradient of o (strides as given); d_state that of the last state, or NULL.
 * Nothing of the forward call is needed again.  Outputs, all contiguous: dq, dk, dv in the shapes of q, k, v (summed over the
 * heads that share a head), 16-byte aligned; dlog_a float32 [batch, tokens, heads], or [heads] where the decay is fixed (batch
 * and token stride 0); dstate0 float32.  dlog_a and dstate0 may be NULL.  Where d_state is given 1 / scale has to be finite.
 * Without sequences or heads, gradients that have elements all the same are zeros.  Asynchronous; workspace of
 * heinsen_attention_workspace_bytes(p, 1) bytes, checked as above.
 */
hs_status heinsen_attention_backward(const heinsen_attention_problem* p, const heinsen_attention_tensor* d_o,
                                     const float* d_state, void* dq, void* dk, void* dv, float* dlog_a,
                                     float* dstate0, void* workspace, size_t workspace_bytes, void* stream);

/* Scratch in bytes for either call; 0 for sizes the library does not accept. */
size_t heinsen_attention_workspace_bytes(const heinsen_attention_problem* p, int backward);

/*
 * Synchronises `stream` and returns HS_ERR_COPY_TIMEOUT where a bounded wait of any forward or backward call on the current
 * device, whatever its workspace, has run out since this was last asked (outputs of such calls are not valid); HS_OK otherwise.
 * It finds what calls that completed before it have met.
 */
hs_status heinsen_attention_check(void* stream);

/*
 * One token for each of `batch` sequences (problem with tokens == 1; lengths and state0 must be NULL).  The states are
 * rows of a pool [pool, heads, k_dim, v_dim] that is updated in place: sequence b uses row slots[b], or row b where
 * slots is NULL (pool >= batch).  A slot that is negative or >= pool has no state: nothing is read or written for it and
 * its o is zero.  No two sequences of a call may share a slot.  No workspace; asynchronous.
 */
hs_status heinsen_attention_step(const heinsen_attention_problem* p, const heinsen_attention_tensor* o, float* pool_state,
                                 int64_t pool, const int32_t* slots, void* stream);

/*
 * The norms before and after a block, fused with the block's gate and residual scale.  For each of `rows` rows of `dim`:
 *
 *         n = branch / sqrt(mean(branch^2) + eps) * post_weight      (no division and no weight where post_weight is NULL)
 *         r = x + scale * gate * n                                   (no gate where gate is NULL)
 *         y = r / sqrt(mean(r^2) + eps) * pre_weight
 *
 * x is the residual stream, branch the block's output, r the stream after the block and y the next block's input.
 * x, branch, r, y: contiguous [rows, dim]; gate: contiguous [rows / gate_rows, dim], each of its rows serves gate_rows
 * neighbours (1 = a gate for each row; rows is a multiple of gate_rows); weights [dim].  All of `dtype`, weights of
 * `weight_dtype` (the same or HS_F32).  Sums and norms in float32.  1 <= dim <= 16384.  y is the norm of r before its
 * rounding to `dtype`.
 */
typedef struct {
    int64_t rows, gate_rows;
    int32_t dim;
    hs_dtype dtype, weight_dtype;
    float scale, eps;
    const void *x, *branch, *gate, *pre_weight, *post_weight;
} heinsen_norms_problem;

hs_status heinsen_block_norms_forward(const heinsen_norms_problem* p, void* r, void* y, void* stream);
/*
 * Gradients, given those of r and y (d_r may be NULL for zeros).  dx, dbranch [rows, dim]; dgate as gate; dpre, dpost
 * [dim] (NULL where the input is).  x itself is read again: r is formed anew in float32.
 */
hs_status heinsen_block_norms_backward(const heinsen_norms_problem* p, const void* d_r, const void* d_y, void* dx,
                                       void* dbranch, void* dgate, void* dpre, void* dpost, void* workspace,
                                       size_t workspace_bytes, void* stream);
/* 0 for sizes the library does not accept; of the pointers only whether there is a gate matters. */
size_t heinsen_block_norms_workspace_bytes(const heinsen_norms_problem* p);

/*
 * The gated norm of a block's heads: y = x / sqrt(mean(x^2) + eps) * weight * silu(gate) over rows of `dim`
 * (a row is one head of one token).  x, gate, y contiguous [rows, dim]; weight [dim].  Fields branch, post_weight, scale
 * and gate_rows of the problem are not used; gate may be NULL (no factor).  1 <= dim <= 16384.
 */
hs_status heinsen_gated_norm_forward(const heinsen_norms_problem* p, void* y, void* stream);
hs_status heinsen_gated_norm_backward(const heinsen_norms_problem* p, const void* d_y, void* dx, void* dgate,
                                      void* dweight, void* workspace, size_t workspace_bytes, void* stream);
size_t heinsen_gated_norm_workspace_bytes(const heinsen_norms_problem* p);

#ifdef __cplusplus
}
#endif
#endif /* HEINSEN_ATTENTION_H_ */
