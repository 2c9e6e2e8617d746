/*
 * c3c_layers.h -- operators of a recurrent layer, of libc3c for AMD Instinct
 * MI355X (gfx950).
 *
 * The cached causal Conv3D of c3c.h remembers its stream in a few frames; the
 * attention of c3c_tokens.h in a cache that grows with it.  A layer of linear
 * attention remembers it in a state of constant size.  The operators that such
 * a layer has beside those of c3c_tokens.h:
 *
 *   c3c_linear_attention    linear attention with a decay for each head: prompts
 *                           by chunks, single tokens by the recurrence
 *   c3c_linear_i8_epilogue  c3c_linear_i8 with an activation, a gate and a
 *                           residual in its epilogue
 *   c3c_gated_linear_i8     both projections of a gated feed-forward block, the
 *                           activation and their product
 *
 * Conventions are those of c3c_tokens.h: status codes, device pointers that the
 * caller owns, asynchronous work on `stream`, the workspace of the context,
 * float dtypes, contiguous tensors but for the strides that a call takes,
 * alignment to the element, sizes below 2^31 and tensors below 2^40 elements.
 */
#ifndef C3C_LAYERS_H
#define C3C_LAYERS_H

#include "c3c_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- linear attention */
/* A state for each head, fp32 [slots][heads][dim_k][dim_v]; dim_k and dim_v are
 * multiples of 16, at most 256. */
typedef struct c3c_state_cache {
  float* state;
  int64_t slots, heads, dim_k, dim_v;
} c3c_state_cache;

/* For the tokens t of a sequence in order, and every head h:
 *   S     <-  exp(g) S + k_t v_t^T        k_t (dim_k), v_t (dim_v)
 *   out_t  =  scale * q_t S
 * The sequences are packed as c3c_kv_batch says: the new tokens of sequence b
 * are rows cu[b] .. cu[b+1] of q, k, v, the last of its len[b].  The batch's
 * table and cols are not read.  Its state lies in slot[b] (int32 [B]; NULL: in
 * slot b) and is updated in place; where the call holds all of a sequence's
 * tokens (len[b] <= cu[b+1] - cu[b]), the state begins at zero, whatever the
 * slot holds.  A sequence without new tokens leaves its state alone.  What lies
 * on the device is not trusted: rows outside [0, T) are cut off; a sequence
 * whose slot is outside [0, slots) begins at zero and its state is not stored.
 * Slots of a call must differ.
 *   q, k: [T][qk_heads][dim_k], v: [T][heads][dim_v]; ld_q, ld_k, ld_v elements
 *   between tokens, below 2^23; head h reads query and key head h / (heads / qk_heads).
 *   log_decay (g): fp32, [heads] with ld_decay 0, or [T][heads] with ld_decay
 *   elements between tokens.  At most 0; -infinity forgets.  A decay is held to
 *   exp(-110), which is 0 in fp32, and a weight below 2^-126 counts as 0.  Larger
 *   ones are taken as they come while their sums stay below 87, over any 32 tokens
 *   in a row and, where a sequence is split, over all of its new ones; beyond that
 *   results may be infinite or NaN where the recurrence's are finite.
 *   out: [T][heads][dim_v] contiguous.  Rows of no sequence are left alone.
 * A token does not reach the tokens before it, NaN included; what a NaN or an
 * infinity reaches becomes NaN or infinite (an infinity may become a NaN).
 *
 * States and sums are fp32.  Products of a chunk of tokens run on the matrix
 * cores with operands split into bf16 terms of 8 bits: inputs into as many as
 * hold them exactly (1 for bf16, 2 for f16, 3 for f32); what multiplies them in
 * out into 2 (3 for f32) terms; in the state into 3.  A value beyond 3.38e38, the
 * largest of bf16, counts as infinite; what is below 2^-133, its smallest, is lost
 * of a term, so values and products of queries and keys below about 2^-108 keep
 * fewer bits.
 *
 * max_new bounds the new tokens of a sequence; it only plans the work.
 * Workspace (c3c_linear_attention_workspace_bytes): the states between the
 * parts of sequences that are split because heads and sequences are too few for
 * the device; with a smaller one the call runs unsplit.  It does not grow steadily
 * with the tokens or the sequences: ask for every size that is used.
 * EINVAL: NULL ctx, states, batch or required tensor; sizes out of range;
 * unknown dtype; qk_heads not dividing heads; heads or B > 65535; a stride too
 * small; scale not finite; an output overlapping an input or another; the
 * workspace overlapping a tensor. */
int c3c_linear_attention_workspace_bytes(const c3c_state_cache* states, const c3c_kv_batch* batch,
                                         int dtype, int64_t qk_heads, size_t* bytes);
int c3c_linear_attention(c3c_ctx* ctx, const c3c_state_cache* states, const c3c_kv_batch* batch,
                         const int32_t* slot, int dtype, int64_t qk_heads, const void* q,
                         int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         const float* log_decay, int64_t ld_decay, float scale, void* out,
                         void* stream);

/* ---------------------------------------------------------------- products with an epilogue */
/* NONE z;  SILU z / (1 + exp(-z));  GELU z/2 (1 + erf(z / sqrt 2));  GELU_TANH
 * z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
enum { C3C_ACT_NONE = 0, C3C_ACT_SILU = 1, C3C_ACT_GELU = 2, C3C_ACT_GELU_TANH = 3 };

/* z = c3c_linear_i8's result, before its rounding; for token m and channel n
 *   y = alpha * residual[m][n] + gate[m / rows_per_gate][n] * act(z)
 * residual [M][N], gate [ceil(M / rows_per_gate)][N], both of y_dtype and
 * contiguous; NULL: no residual, a gate of ones.  y may be the residual itself.
 * Codes of float activations, here and in c3c_gated_linear_i8: the integers
 * nearest to 127 x / max|x| themselves, ties to even; 0 in rows whose scale
 * rounds to 0.  c3c_linear_i8 and c3c_quantize_rows divide by the rounded scale
 * instead, which differs by one step for the few values next to a half, by more
 * where the scale is subnormal: a caller who needs one set of codes for several
 * products quantises once and passes int8.  With C3C_ACT_NONE, no gate and no
 * residual the call is c3c_linear_i8, its codes included; every call of
 * c3c_gated_linear_i8 takes the codes stated here.
 * Activations are relatively accurate where they tend to 0 as well, down to
 * magnitudes of 2^-118, below which they may be 0.
 * The workspace is that of c3c_linear_i8 (c3c_linear_i8_workspace_bytes).
 * EINVAL: as c3c_linear_i8; NULL e; unknown act; alpha not finite;
 * rows_per_gate < 1 with a gate; y overlapping a residual that it is not. */
typedef struct c3c_epilogue {
  const void *gate, *residual;
  int64_t rows_per_gate;
  float alpha;
  int32_t act;
} c3c_epilogue;
int c3c_linear_i8_epilogue(c3c_ctx* ctx, const c3c_linear_desc* d, const c3c_epilogue* e,
                           const void* x, const float* x_scale, const int8_t* w,
                           const float* w_scale, const float* bias, void* y, void* stream);

/* y[m][n] = act(z[m][n]) * z[m][N + n], z the product with all 2 N rows of w
 * (int8 [2 N][K]: the gate's rows, then the others), as c3c_linear_i8 forms it:
 * w_scale [2 N], bias [2 N] or NULL.  d->N is N, the channels of y.  Workspace
 * and refusals as c3c_linear_i8; 2 N is below 2^31. */
int c3c_gated_linear_i8_workspace_bytes(const c3c_linear_desc* d, size_t* bytes);
int c3c_gated_linear_i8(c3c_ctx* ctx, const c3c_linear_desc* d, int act, const void* x,
                        const float* x_scale, const int8_t* w, const float* w_scale,
                        const float* bias, void* y, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* C3C_LAYERS_H */
