/*
 * c3c_tokens.h -- token operators of libc3c for AMD Instinct MI355X (gfx950).
 *
 * The cached causal Conv3D of c3c.h decodes a stream chunk by chunk.  What
 * makes those chunks is a causal transformer over the same stream: it takes
 * tokens (one, or a frame's worth) and keeps keys and values where the
 * decoder keeps frames.  The four operators of one layer of it:
 *
 *   c3c_linear_i8        matrix product in 8-bit integers, with a scale for
 *                        every token and every output channel
 *   c3c_kv_append        rotation of queries and keys by their positions;
 *                        keys and values into a paged cache held in 8 bits
 *   c3c_paged_attention  attention over that cache
 *   c3c_norm_gate        norm after a block, gate, scaled residual and norm
 *                        before the next block
 *
 * and c3c_quantize_rows, the quantisation that c3c_linear_i8 applies to
 * float activations, for weights and other rows.
 *
 * Conventions are those of c3c.h: status codes, device pointers that the
 * caller owns, asynchronous work on `stream`, a context that is used by one
 * host thread at a time, a workspace attached with c3c_ctx_set_workspace that
 * calls overlapping in time must not share.  The calls count in no route
 * counter.  Sums, softmax statistics and norms are held in fp32 (integer
 * products in int32) and rounded once, to nearest even, at each output.
 * `dtype` is C3C_DTYPE_BF16, _F16 or _F32 and holds for every float tensor
 * that is not declared `float`.  Tensors are contiguous but for the strides
 * that a call takes, and aligned to their element; the cache's code tensors
 * are aligned to 16 bytes.  Every size is below 2^31 and every tensor below
 * 2^40 elements (EINVAL beyond).
 */
#ifndef C3C_TOKENS_H
#define C3C_TOKENS_H

#include "c3c.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit integer rows with a scale for each row (c3c_linear_i8's x) */
enum { C3C_DTYPE_I8 = 16 };

/* ---------------------------------------------------------------- 8-bit rows */
/* For every row t of x [T][C]:  scale[t] = max_c |x[t][c]| / 127,
 * q[t][c] = x[t][c] / scale[t] rounded to the nearest integer, ties to even.
 * A row of zeros (or whose scale rounds to 0 in fp32) has scale 0 and codes 0.
 * A row that holds a NaN or an infinity has scale NaN and codes 0, so that
 * every product with it is NaN.  ld_x: elements between rows (>= C); q is
 * contiguous.
 * EINVAL: NULL ctx or a NULL tensor of nonzero size; T < 0, C < 1, ld_x < C;
 * unknown dtype; q or scale overlapping x or each other. */
int c3c_quantize_rows(c3c_ctx* ctx, int64_t T, int64_t C, int64_t ld_x, int dtype, const void* x,
                      int8_t* q, float* scale, void* stream);

/* ---------------------------------------------------------------- linear */
/* y[m][n] = (sum_k q[m][k] w[n][k]) * s[m] * w_scale[n] + bias[n]
 *
 * w: int8 [N][K], w_scale: [N].  x is [M][K], ld_x elements between rows:
 *   x_dtype C3C_DTYPE_I8   the codes q, with x_scale [M] = s;
 *   a float dtype          the call quantises x by the rule of
 *                          c3c_quantize_rows (x_scale NULL).
 * y: [M][N] of y_dtype, contiguous.  bias: fp32 [N] or NULL.  The sum is exact
 * in int32, hence K <= 131071.
 *
 * Workspace (c3c_linear_i8_workspace_bytes, 0 where none is used): the
 * quantised rows of float activations, copies of rows that are no multiple of
 * 16 bytes, and the partial sums of a product that is split along K because
 * its tiles are too few for the device.  A call of float activations whose
 * context has less than the quantised rows' bytes is EINVAL, also where few
 * tokens are quantised without them; with those but not the others it runs
 * without copies or unsplit.  Results are the same bits
 * either way (integer sums).
 * EINVAL: NULL ctx, desc or a NULL tensor of nonzero size; M < 0, N < 1,
 * K < 1 or > 131071, ld_x < K; unknown dtypes; x_scale given with a float x
 * or missing with int8; y overlapping an input; the workspace overlapping a
 * tensor. */
typedef struct c3c_linear_desc {
  int64_t M, N, K, ld_x;
  int32_t x_dtype, y_dtype;
} c3c_linear_desc;

int c3c_linear_i8_workspace_bytes(const c3c_linear_desc* d, size_t* bytes);
int c3c_linear_i8(c3c_ctx* ctx, const c3c_linear_desc* d, const void* x, const float* x_scale,
                  const int8_t* w, const float* w_scale, const float* bias, void* y, void* stream);

/* ---------------------------------------------------------------- norms and gate */
/* For every token t:
 *   n(v)[c] = v[c] / sqrt(mean_c v[c]^2 + eps)
 *   h'      = alpha * h + gate[t / rows_per_gate] * (post * n(y))
 *   u       = pre * n(h')
 * h (the residual stream), y (the block's output), h_out (h'), u: [T][C];
 * gate [ceil(T / rows_per_gate)][C] of the same dtype; post and pre: fp32 [C].
 *   post NULL    no norm after the block: h' = alpha h + gate * y
 *   gate NULL    a gate of ones
 *   y NULL       no block before (a first layer): h' = alpha h; post and gate
 *                are then NULL
 *   h_out NULL   h' is not stored; h_out may be h itself
 *   pre NULL     no norm before the next block: u, u_q, u_scale are NULL
 *   u_q          u by the rule of c3c_quantize_rows, int8 [T][C] with u_scale
 *                [T], as c3c_linear_i8 takes it; u and u_q may both be given
 * u is formed from h' before its rounding.
 * EINVAL: NULL ctx, desc or h; no output; T < 0, C < 1, rows_per_gate < 1
 * with a gate; unknown dtype; alpha or eps not finite, eps < 0; u_q without
 * u_scale or the reverse; an output overlapping an input (but h_out == h) or
 * another output. */
typedef struct c3c_norm_desc {
  int64_t T, C, rows_per_gate;
  float alpha, eps;
  int32_t dtype, reserved;
} c3c_norm_desc;

int c3c_norm_gate(c3c_ctx* ctx, const c3c_norm_desc* d, const void* h, const void* y,
                  const void* gate, const float* post, const float* pre, void* h_out, void* u,
                  int8_t* u_q, float* u_scale, void* stream);

/* ---------------------------------------------------------------- the paged cache */
/* Pages of `page` tokens (a multiple of 16), for `heads` key/value heads of
 * `dim` channels (a multiple of 16, at most 256).  Every block of 16
 * consecutive tokens of a page and every head has a scale, a power of two, and
 * e4m3 codes (the OCP 8-bit float with 4 exponent and 3 fraction bits, largest
 * value 448): value = code * scale.
 *   k        [pages][heads][page][dim]           codes, 16-byte aligned
 *   v        [pages][heads][page / 16][dim][16]  codes, 16-byte aligned: the
 *            tokens of a block side by side, as the second product reads them
 *   k_scale, v_scale  [pages][heads][page / 16]
 * A floating code makes the scale a matter of range alone: with a power of
 * two, a block whose scale has to grow when tokens are added keeps its codes
 * exactly but for those that fall below the normal range. */
#define C3C_KV_BLOCK 16
typedef struct c3c_kv_cache {
  void *k, *v;
  float *k_scale, *v_scale;
  int64_t pages, heads, page, dim;
} c3c_kv_cache;

/* The sequences of a call, packed: sequence b has the rows cu[b] .. cu[b+1]
 * of q, k, v, which are the last tokens of its len[b].  Token p of sequence b
 * lies in page table[b][p / page].  Device memory: table [B][cols], cu [B+1]
 * ascending from 0 to T, len [B].  max_new: no sequence has more new tokens
 * (attention leaves the output of rows past it undefined); max_len: no
 * sequence is longer (it only plans the work).  What lies on the device is not trusted: rows outside
 * [0, T) are cut off, a token whose page is outside [0, pages) or past the
 * table's columns is not stored and not seen (so -1 marks an evicted page). */
typedef struct c3c_kv_batch {
  const int32_t *table, *cu, *len;
  int64_t B, cols, T, max_new, max_len;
} c3c_kv_batch;

/* Rotation of the first `rot` channels (even, <= dim) of every head: with
 * c, s = cos[r][i], sin[r][i] (fp32 [rows][rot / 2]), the pair (a, b) becomes
 * (a c - b s, b c + a s).  pairs 0: channels (i, i + rot/2); 1: (2i, 2i + 1).
 * r = pos[t] (int32 [T]) or, with pos NULL, the token's place in its sequence;
 * a token whose r lies outside [0, rows) becomes NaN. */
typedef struct c3c_rope {
  const float *cos, *sin;
  const int32_t* pos;
  int64_t rows, rot;
  int32_t pairs, reserved;
} c3c_rope;

/* Rotates the new tokens' queries and keys and stores keys and values.
 * k, v: [T][heads][dim], ld_k / ld_v elements between tokens (>= heads * dim).
 * q: [T][q_heads][dim], ld_q between tokens, or NULL (then q_out is NULL);
 * q_out: [T][q_heads][dim] contiguous, the rotated queries; it may be q itself
 * when ld_q is q_heads * dim.  rope NULL: no rotation (q is copied).
 *
 * Scale of a block: 2^e with the least e >= -126 such that no finite new
 * element exceeds 448 * 2^e, and no less than the block's present scale where
 * the block holds earlier tokens of the sequence; where it grows, their codes
 * are scaled and rounded again.  Codes: nearest, ties to even.  NaN and
 * infinities are stored as NaN and leave the scale alone.
 * Blocks that are written must belong to one sequence only.
 * EINVAL: NULL ctx, cache, batch or required tensor; sizes out of range;
 * unknown dtype; heads or q_heads < 1; heads, q_heads or B > 65535; ld too
 * small; misaligned codes; outputs overlapping inputs or one another. */
int c3c_kv_append(c3c_ctx* ctx, const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                  const c3c_rope* rope, int dtype, int64_t q_heads, const void* q, int64_t ld_q,
                  const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* q_out,
                  void* stream);

/* Attention of the new tokens' queries over the cache, which holds the new
 * tokens already.  q: [T][q_heads][dim], ld_q between tokens; query head h
 * reads key/value head h / (q_heads / heads).  The query in row cu[b] + i is
 * token p = len[b] - new[b] + i and sees token j < len[b] if its page is
 * valid and
 *   causal:      j <= p
 *   window > 0:  j > p - window
 *   out[h]  = sum_j softmax_j(scale * q . k_j) v_j
 *   lse[h]  = log sum_j exp(scale * q . k_j)      (fp32 [T][q_heads], or NULL)
 * A query that sees no token has out 0 and lse -infinity.  What a query does
 * not see does not reach it, NaN included; blocks that no query of the call
 * sees may hold anything, scales included.  out: [T][q_heads][dim] contiguous,
 * dtype.  Rows of q that belong to no sequence leave theirs undefined.
 * Probabilities enter the matrix cores as sums of 1 (bf16), 2 (f16) or 3 (f32)
 * f16 terms of 11 bits each, and are held to 2^-32 of the row's largest.  Where
 * the scale of a value's block is 2^d, d > 15, below the largest value scale
 * that the call's queries see of its sequence and head, its probability is
 * held to 2^(d - 47) of the row's largest.
 *
 * Workspace (c3c_paged_attention_workspace_bytes): the partial results of a
 * call whose sequences are split because there are too few queries for the
 * device; with a smaller workspace it runs unsplit.
 * EINVAL: as c3c_kv_append; heads not dividing q_heads; T * q_heads / heads of
 * 2^31 - 2048 or more; scale not finite and positive; causal not 0 or 1;
 * window < 0; the workspace overlapping a tensor.  EDEVICE also: 2^31 or more
 * workgroups, of which each sequence and key/value head has one for every 64 or
 * 128 of the most queries that any sequence may have. */
int c3c_paged_attention_workspace_bytes(const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                                        int dtype, int64_t q_heads, int causal, int64_t window,
                                        size_t* bytes);
int c3c_paged_attention(c3c_ctx* ctx, const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                        int dtype, int64_t q_heads, const void* q, int64_t ld_q, float scale,
                        int causal, int64_t window, void* out, float* lse, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* C3C_TOKENS_H */
