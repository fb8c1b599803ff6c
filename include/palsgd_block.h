/*
 * palsgd_block.h -- C ABI of the block operators: what the K workers of palsgd.h run to MAKE their gradients.
 *
 * Every operator runs the K workers' replicas in one call, each worker with weights of its own (the rows of the
 * parameter buffers of palsgd.h) and its own batch, and writes each worker's gradients where its gradient buffer is:
 *
 *   - the gated feed-forward block, forward and backward               palsgd_ffn_forward / _backward
 *   - activation checkpoints in 8 bits                                 palsgd_act8_pack / _unpack
 *   - the norm of queries and keys for each head with the position
 *     rotation in the same pass, forward and backward                  palsgd_qk_norm_rope_forward / _backward
 *   - the matrix product with bias, activation and residual, forward
 *     and backward                                                     palsgd_linear_forward / _backward
 *   - the layer norm with the residual added, forward and backward     palsgd_layer_norm_forward / _backward
 *   - the cross entropy over a vocabulary, forward and backward        palsgd_cross_entropy_forward / _backward
 *
 * General rules (as in palsgd.h unless stated here)
 *   - Every entry point returns a palsgd_status, never throws, never exits.  Arguments are checked before anything is
 *     enqueued.  `stream` is a cudaStream_t as void*.  Work is asynchronous; entry points keep no state between calls,
 *     so calls on distinct streams and host threads are independent as long as their outputs and workspaces are.
 *   - All buffers are DEVICE memory of the caller.  Nothing is allocated.  Outputs and the workspace must not overlap each
 *     other or an input: EINVAL, told exactly from addresses, sizes and strides (interleaved layouts are no overlap), but
 *     for layouts of unlike strides so entangled that the search would take long.  The one exception: a head matrix that
 *     palsgd_qk_norm_rope_* writes may be exactly one that it reads (q_out = q; dq = dq_out or q): work in place.
 *   - `precision` fixes the storage type of activations, weights and gradients: PALSGD_PREC_FP32 = float,
 *     PALSGD_PREC_BF16_MASTER = bfloat16.  Sums, norms and activations are taken in binary32; each result is rounded
 *     once to the storage type.  What is rounded in between is stated at each call.
 *   - A matrix for K workers is a palsgd_mat: element (k, r, c) at data + k*worker_stride + r*row_stride + c, strides
 *     in ELEMENTS.  The last axis is contiguous.  Any strides >= 0 are accepted for inputs (worker_stride 0: all
 *     workers read one matrix); the rows of an output may not overlap.  Buffers need only natural element alignment:
 *     matrices whose base is 16-byte aligned and whose strides are multiples of 16 bytes are read in place by the
 *     copy engines of the matrix kernels; any other is first copied, by one more kernel, into the workspace.
 *     Unaligned rows are read by whole aligned 16-byte blocks that hold a byte of the row: up to 15 bytes before its
 *     first and behind its last byte are read (and not used), never across a multiple of 16 bytes.
 */
#ifndef PALSGD_BLOCK_H_
#define PALSGD_BLOCK_H_

#include "palsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct palsgd_mat {
    void*   data;
    int64_t worker_stride;    /* elements */
    int64_t row_stride;       /* elements */
} palsgd_mat;

/*
 * 8-bit activation checkpoints.  The last axis is cut into groups of 32 (the last one may be shorter); a group holds
 * one exponent byte E and an int8 q for each value, and stands for q * 2^(E-127):
 *   E = 127 + the smallest e with rint(max|x| / 2^e) <= 127, at least 1;     q = rint(x / 2^e)   (ties to even)
 * so the step is a power of two: no division, and every value that a checkpoint stands for has at most eight
 * significant bits -- exact in bfloat16, which is what the tensor cores take.  8.25 bits a value.
 * A group that holds an infinity, a NaN, or a value that rounds to 2^128 in this form has E = 255, q = 0 and reads back
 * as NaN (an overflow stays visible).
 * q: rows of `cols` int8; e: rows of ceil(cols / 32) uint8.
 */
#define PALSGD_ACT8_GROUP 32u
int palsgd_act8_pack(int32_t precision, uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* x,
                     const palsgd_mat* q, const palsgd_mat* e, void* stream);
int palsgd_act8_unpack(int32_t precision, uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* q,
                       const palsgd_mat* e, const palsgd_mat* x, void* stream);

/*
 * Gated feed-forward block of worker k, x [tokens, d_model], w_gate and w_up [d_ff, d_model], w_down [d_model, d_ff]:
 *   g = x w_gate^T;  u = x w_up^T;  h = act(g) * u;  y = h w_down^T
 * act: SILU g/(1+e^-g);  GELU g Phi(g);  GELU_TANH g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3)));  RELU max(g, 0).
 * g and u stay in binary32 up to h.  BF16: h is rounded to bfloat16 once, for the second product.
 *
 * `save` names what the forward call keeps for the backward call (and the form the backward call finds it in):
 *   NONE   nothing                         (gate, up, gate_e, up_e are NULL)
 *   FULL   gate, up: g and u in the storage type
 *   8BIT   gate, up: int8, gate_e, up_e: uint8 -- the 8-bit checkpoints of g and u, taken from the binary32 sums
 *
 * Backward, at the saved g and u (the values that they stand for):
 *   dh = dy w_down;  du = dh act(g);  dg = dh u act'(g);  h = act(g) u
 *   dx = dg w_gate + du w_up;  dw_gate = dg^T x;  dw_up = du^T x;  dw_down = dy^T h
 * BF16: dg, du and h are rounded to bfloat16 once, for the products.  act'(0) of RELU is 0; a NaN in g gives NaN in act
 * and act' of all four.  With save = 8BIT, x_e may be given: x is then the int8 of an 8-bit checkpoint of x, x_e its
 * exponents (x_e = NULL: x in the storage type).
 * Outputs are overwritten.  tokens = 0: the weight gradients are zero.  dx may be NULL (first layer).
 *
 * FP32 products are formed on the tensor cores from three bfloat16 parts of each operand (24 bits together), all six
 * products of parts that reach above 2^-24 of the whole, summed in binary32 with a rounding to nearest every 256 terms.
 * An infinite operand gives NaN there where a product of binary32 would be infinite, and operands below about 2^-110 lose
 * the bits of their parts below 2^-133.  Results do not depend on timing: the same call gives the same bits.
 *
 * Workspace: call with workspace = NULL to learn *workspace_bytes (nothing is enqueued; all other arguments as in the
 * call to come); then pass at least that many bytes, 256-byte aligned.  Contents need no preparation.  A workspace that
 * is too small is refused with EINVAL, and *workspace_bytes says what is needed: never 0, with tokens = 0 neither, so
 * that a call to do the work cannot look like one that asks.
 * Errors: EINVAL (NULL, K = 0 or > 64, d_model or d_ff = 0, a size >= 2^31, bad enum, negative or overlapping strides,
 * overlapping buffers, small workspace); EALIGN; ECUDA.
 */
enum { PALSGD_ACT_SILU = 0, PALSGD_ACT_GELU = 1, PALSGD_ACT_GELU_TANH = 2, PALSGD_ACT_RELU = 3 };
enum { PALSGD_SAVE_NONE = 0, PALSGD_SAVE_FULL = 1, PALSGD_SAVE_8BIT = 2 };

typedef struct palsgd_ffn_shape {
    uint32_t K;
    int32_t  precision, activation, save;
    uint64_t tokens, d_model, d_ff;
} palsgd_ffn_shape;

int palsgd_ffn_forward(const palsgd_ffn_shape* s, const palsgd_mat* x, const palsgd_mat* w_gate, const palsgd_mat* w_up,
                       const palsgd_mat* w_down, const palsgd_mat* y, const palsgd_mat* gate, const palsgd_mat* up,
                       const palsgd_mat* gate_e, const palsgd_mat* up_e, void* workspace, size_t* workspace_bytes,
                       void* stream);
int palsgd_ffn_backward(const palsgd_ffn_shape* s, const palsgd_mat* dy, const palsgd_mat* x, const palsgd_mat* x_e,
                        const palsgd_mat* w_gate, const palsgd_mat* w_up, const palsgd_mat* w_down,
                        const palsgd_mat* gate, const palsgd_mat* up, const palsgd_mat* gate_e, const palsgd_mat* up_e,
                        const palsgd_mat* dx, const palsgd_mat* dw_gate, const palsgd_mat* dw_up,
                        const palsgd_mat* dw_down, void* workspace, size_t* workspace_bytes, void* stream);

/*
 * The matrix kernels' waits for their own copies and products are bounded (a few seconds).  One that gave up -- which
 * no input should bring about -- leaves its outputs unspecified and a note on the device: this call returns
 * PALSGD_ECUDA once if there is one, else PALSGD_OK.  SYNCHRONISES the stream.
 */
int palsgd_block_status(void* stream);

/*
 * Norm of queries and keys for each head, with the position rotation in the same pass.  For worker k, token t, head h
 * of q (and, with its own weights, of k), x in R^head_dim:
 *   r = 1 / sqrt(mean(x^2) + eps), eps as a float;  n = x r w;   the first rotary_dim values of n are rotated by pairs:
 *   (a, b) -> (a c_i - b s_i, b c_i + a s_i),  c_i = cos_table[pos][i], s_i = sin_table[pos][i], pos = positions[k][t]
 *   pair i is (i, i + rotary_dim/2), or (2i, 2i+1) with interleaved = 1;  0 <= i < rotary_dim/2.
 * Backward:  dn = the gradient rotated back;  xh = x r;
 *   dx = r (w dn - xh mean(w dn xh));   dw = sum over tokens and heads of dn xh   (in a fixed order: bitwise repeatable)
 * Heads are palsgd_heads: element (k, t, h, c) at data + k*worker_stride + t*token_stride + h*head_stride + c, so q and
 * k may be views of one fused projection.  heads_q or heads_k may be 0 (its pointers may then be NULL).  The tables are
 * float [table_rows, rotary_dim/2], contiguous; positions int32, one row per worker at pos_worker_stride (0: one row for
 * all).  w: rows of head_dim in the storage type, one per worker (row_stride unused).  A token whose position is
 * outside 0..table_rows-1 gets NaN outputs (and NaN gradients, dw included).
 * dw are overwritten; with tokens = 0, or no heads, they are zero.  Workspace (backward only): as for the feed-forward block.
 * Errors: EINVAL (NULL, K, odd rotary_dim or rotary_dim > head_dim, head_dim = 0, eps negative or not finite,
 * overlapping buffers, small workspace); EUNSUPPORTED (head_dim > 512); EALIGN; ECUDA.
 */
typedef struct palsgd_heads {
    void*   data;
    int64_t worker_stride, token_stride, head_stride;     /* elements */
} palsgd_heads;

typedef struct palsgd_qk_shape {
    uint32_t K;
    int32_t  precision;
    uint64_t tokens;
    uint32_t heads_q, heads_k, head_dim, rotary_dim;
    int32_t  interleaved;
    uint32_t reserved_;       /* set to 0 */
    uint64_t table_rows;
    int64_t  pos_worker_stride;
    double   eps;
} palsgd_qk_shape;

int palsgd_qk_norm_rope_forward(const palsgd_qk_shape* s, const palsgd_heads* q, const palsgd_heads* k,
                                const palsgd_mat* w_q, const palsgd_mat* w_k, const float* cos_table,
                                const float* sin_table, const int32_t* positions, const palsgd_heads* q_out,
                                const palsgd_heads* k_out, void* stream);
int palsgd_qk_norm_rope_backward(const palsgd_qk_shape* s, const palsgd_heads* dq_out, const palsgd_heads* dk_out,
                                 const palsgd_heads* q, const palsgd_heads* k, const palsgd_mat* w_q,
                                 const palsgd_mat* w_k, const float* cos_table, const float* sin_table,
                                 const int32_t* positions, const palsgd_heads* dq, const palsgd_heads* dk,
                                 const palsgd_mat* dw_q, const palsgd_mat* dw_k, void* workspace,
                                 size_t* workspace_bytes, void* stream);

/*
 * Matrix product with bias, activation and residual of worker k, x [tokens, d_in], w [d_out, d_in], b [d_out]:
 *   z = x w^T + b;   y = act(z) + residual
 * act: one of the four above, or NONE (z itself).  bias and residual [tokens, d_out] may be NULL.  z stays in binary32 up to y.
 * `save` names what is kept of z for the backward call, as in the feed-forward block: NONE; FULL: pre, in the storage type;
 * 8BIT: pre, pre_e, the 8-bit checkpoint taken from the binary32 values.  With act = NONE the backward call needs none of it, and
 * save has to be NONE there and here.  b: rows of d_out in the storage type, one per worker (row_stride unused).
 *
 * Backward, at the saved z (the value that it stands for), x in the storage type or, where x_e is given, as a checkpoint:
 *   dz = dy act'(z);   dx = dz w;   dw = dz^T x;   db = sum over tokens of dz;   the residual's gradient is dy itself
 * BF16: dz is rounded to bfloat16 once, for the products; db sums the unrounded values.  dx and db may be NULL.  Outputs are
 * overwritten.  tokens = 0: dw and db are zero.  Sums have a fixed order: the same call gives the same bits.
 * FP32 products as in the feed-forward block; small calls sum in binary32 multiply-adds throughout, and keep dz in binary32.
 * An activation and its slope are off by at most 2^-21 (1 + |z|) each before they are rounded, in either type.  Far below zero that is
 * more than they are, and calls of few and of many tokens differ there: GELU of the former is 0 below about -5.6, of the latter e^(-z^2 / 2)
 * small, in fp32 to some 100 units in its last place.
 * Workspace and errors as for the feed-forward block (d_in or d_out = 0: EINVAL).
 */
enum { PALSGD_ACT_NONE = 4 };

typedef struct palsgd_linear_shape {
    uint32_t K;
    int32_t  precision, activation, save;
    uint64_t tokens, d_in, d_out;
} palsgd_linear_shape;

int palsgd_linear_forward(const palsgd_linear_shape* s, const palsgd_mat* x, const palsgd_mat* w, const palsgd_mat* bias,
                          const palsgd_mat* residual, const palsgd_mat* y, const palsgd_mat* pre, const palsgd_mat* pre_e,
                          void* workspace, size_t* workspace_bytes, void* stream);
int palsgd_linear_backward(const palsgd_linear_shape* s, const palsgd_mat* dy, const palsgd_mat* x, const palsgd_mat* x_e,
                           const palsgd_mat* w, const palsgd_mat* pre, const palsgd_mat* pre_e, const palsgd_mat* dx,
                           const palsgd_mat* dw, const palsgd_mat* db, void* workspace, size_t* workspace_bytes, void* stream);

/*
 * Layer norm of every token of worker k, x [tokens, width], w and b [width]:
 *   h = x + residual (residual NULL: h = x);   m = mean(h);   r = 1 / sqrt(mean((h - m)^2) + eps), eps as a float
 *   y = (h - m) r w + b
 * h stays in binary32 up to y; total (given exactly where residual is) receives h in the storage type: the residual stream.
 * mean, rstd: rows of `tokens` floats, one per worker (row_stride unused); either may be NULL.  w, b: rows of width in the
 * storage type.
 * Backward, x being the normed input (total, where there was a residual), at the given mean and rstd:
 *   xh = (x - m) r;   g = dy w;   dx = r (g - mean(g) - xh mean(g xh)) + dtotal;   dw = sum over tokens of dy xh;   db = sum of dy
 * dtotal (may be NULL): the gradient that reaches the residual stream past the norm; dx is then the gradient of x and of the
 * residual alike.  Sums have a fixed order (bitwise repeatable).  dw and db are overwritten; with tokens = 0 they are zero.
 * A row that holds an infinity or a NaN gives NaN.  Workspace (backward only): as for the feed-forward block.
 * Errors: EINVAL (NULL, K, width = 0, a size >= 2^31, eps negative or not finite, residual without total or the reverse,
 * overlapping buffers, small workspace); EUNSUPPORTED (width > 16384); EALIGN; ECUDA.
 */
typedef struct palsgd_norm_shape {
    uint32_t K;
    int32_t  precision;
    uint64_t tokens, width;
    double   eps;             /* forward */
} palsgd_norm_shape;

int palsgd_layer_norm_forward(const palsgd_norm_shape* s, const palsgd_mat* x, const palsgd_mat* residual, const palsgd_mat* w,
                              const palsgd_mat* b, const palsgd_mat* y, const palsgd_mat* total, const palsgd_mat* mean,
                              const palsgd_mat* rstd, void* stream);
int palsgd_layer_norm_backward(const palsgd_norm_shape* s, const palsgd_mat* dy, const palsgd_mat* x, const palsgd_mat* w,
                               const palsgd_mat* mean, const palsgd_mat* rstd, const palsgd_mat* dtotal, const palsgd_mat* dx,
                               const palsgd_mat* dw, const palsgd_mat* db, void* workspace, size_t* workspace_bytes, void* stream);

/*
 * Cross entropy of every token of worker k, logits [tokens, vocab], targets int32 (one row per worker at
 * target_worker_stride; 0: one row for all):
 *   lse = log(sum of e^z);   loss = lse - z_target
 * loss, lse, dloss: rows of `tokens` floats, one per worker (row_stride unused).
 *   target < 0: the token does not count: loss 0, gradient 0 whatever its logits are.   target >= vocab: loss and gradient NaN.
 * Logits of -infinity take no part (a target of that logit: loss +infinity).  A row that holds NaN or +infinity, or nothing
 * above -infinity, gives NaN in loss and gradient; its lse is NaN, or -infinity where nothing is above that.
 * Backward, at the given lse:  dlogits = (e^(z - lse) - [target]) dloss.  dlogits may be exactly logits: work in place.
 * The given lse is rounded to binary32, which the exponential feels as 2^-24 |lse| of itself.  From |lse| = 1024 on, one within 2^-22 of
 * itself of the row's own is taken as the row's own before rounding, formed again from the row (1 / vocab for a row of nothing but the
 * type's lowest value); rows of such an lse take five to seven times as long as others.
 * Sums in binary32, in a fixed order; dlogits are rounded once to the storage type.
 * Errors: EINVAL (NULL, K, vocab = 0, a size >= 2^31, overlapping buffers); EUNSUPPORTED (backward: more than 2^31 - 1
 * parts of rows of up to 2048 16-byte pieces, of a worker); EALIGN; ECUDA.
 */
typedef struct palsgd_loss_shape {
    uint32_t K;
    int32_t  precision;
    uint64_t tokens, vocab;
    int64_t  target_worker_stride;
} palsgd_loss_shape;

int palsgd_cross_entropy_forward(const palsgd_loss_shape* s, const palsgd_mat* logits, const int32_t* targets,
                                 const palsgd_mat* loss, const palsgd_mat* lse, void* stream);
int palsgd_cross_entropy_backward(const palsgd_loss_shape* s, const palsgd_mat* dloss, const palsgd_mat* logits,
                                  const int32_t* targets, const palsgd_mat* lse, const palsgd_mat* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PALSGD_BLOCK_H_ */
