/*
 * c3_replay.h -- operators of a replayed transformer layer, and of the model around
 * it, on MI355X (gfx950).
 *
 * A replay runs a layer's forward and backward again on every replica and
 * votes on the outputs and gradients (SCOUT, arXiv 2608.11034, Sec. 6).  Exact
 * C3 then needs operators whose bits are a function of their inputs alone:
 * every sum here runs in an order fixed by the sizes, and no result goes
 * through an atomic.
 *
 * Conventions are those of c3.h: device pointers belong to the caller, every
 * call enqueues work on `stream` and returns, errors are negative
 * c3_status_t, nothing is launched when an argument check fails, host arrays
 * are consumed before the call returns.  Strides count elements.  Element
 * types are C3_F32, C3_BF16 and C3_F16; attention and the loss over a vocabulary take
 * the two 16-bit types.
 * Sums, softmax statistics and norms are held in 32 bits.
 */
#ifndef C3_REPLAY_H_
#define C3_REPLAY_H_

#include "c3.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------- */
/* Rotary positions                                                        */
/* ---------------------------------------------------------------------- */

/* One tensor [batch][length][heads][dim], last dimension contiguous. */
typedef struct {
    const void *in;
    void *out;              /* may be `in` with the same strides; no other overlap */
    int64_t in_stride[3];   /* batch, token, head */
    int64_t out_stride[3];
    int64_t heads;
} c3_heads_t;

/* Which elements of a head form pair i of rot / 2. */
typedef enum {
    C3_ROTARY_HALF = 0,       /* (i, i + rot / 2) */
    C3_ROTARY_INTERLEAVED = 1 /* (2 i, 2 i + 1)   */
} c3_rotary_layout_t;

/*
 * c3_rotary -- turns pair i of every head by the angle position * freqs[i]:
 *     (a, b) -> amplitude * (a cos - b sin, b cos + a sin)
 * in 32 bits, rounded once; elements from `rot` on are copied.  `inverse`
 * turns back, which with the same amplitude is the gradient.
 *
 *   tensors   host array [n], n = 1 or 2 (queries and keys share one call).
 *   positions device [batch][length], strides pos_stride (batch, token; 0
 *             repeats), 4-byte (pos_bytes 4) or 8-byte signed integers.
 *   freqs     device [rot / 2] fp64, radians a position.  The angle is formed
 *             in fp64 and reduced by whole turns before it is rounded, so long
 *             contexts lose nothing.
 *   rot       even, 0 < rot <= dim, dim <= 4096.
 * Errors: C3_E_INVAL, C3_E_ALIGN (a pointer not aligned to its element),
 * C3_E_UNSUPPORTED (element type), C3_E_HIP.  Can be captured.
 */
int c3_rotary(const c3_heads_t *tensors, int n, int dtype, int64_t batch, int64_t length,
              int64_t dim, const void *positions, int pos_bytes, const int64_t pos_stride[2],
              const double *freqs, int64_t rot, int layout, int inverse, double amplitude,
              c3_stream_t stream);

/* ---------------------------------------------------------------------- */
/* Attention                                                               */
/* ---------------------------------------------------------------------- */

/* Sizes, mask and scale of one attention. */
typedef struct {
    int32_t dtype;          /* C3_BF16 or C3_F16                               */
    int32_t heads;          /* query heads, a multiple of kv_heads             */
    int32_t kv_heads;       /* query head h reads key head h / (heads/kv_heads)*/
    int32_t dim;            /* multiple of 8, at most 128                      */
    int32_t causal;         /* query i sees key j only if j <= i + k_len - q_len*/
    int32_t window;         /* > 0: also j > i + k_len - q_len - window        */
    float scale;            /* factor of q . k, positive and finite            */
    int32_t batch;          /* sequences                                       */
    int64_t q_tokens;       /* per sequence, or of all where packed            */
    int64_t k_tokens;
    int32_t packed;         /* 1: tokens of the sequences follow each other    */
    int32_t reserved;
    const int32_t *q_lens;  /* host [batch] or NULL (all q_tokens long)        */
    const int32_t *k_lens;  /* both or neither; required where packed, with    */
                            /* the sums q_tokens and k_tokens                  */
} c3_attention_t;

/* A tensor [batch][tokens][heads][dim] (packed: [tokens][heads][dim], stride[0]
 * unused), last dimension contiguous; pointers 16-byte aligned and strides
 * multiples of 8 elements (that of a dimension with one entry is not looked at).  Of k
 * and v 64 tokens span less than 2^31 bytes; of the gradient's q and dout 64 tokens
 * together with the heads that share a key head (C3_E_UNSUPPORTED).  Results overlap
 * neither inputs nor each other; one that starts where another tensor does is
 * C3_E_INVAL. */
typedef struct {
    void *ptr;
    int64_t stride[3];      /* batch, token, head */
} c3_attn_tensor_t;

/* Sequences whose lengths go along with a kernel's arguments.  Longer lists are
 * staged through host memory that later calls use again, so a stream under graph
 * capture refuses them (C3_E_UNSUPPORTED): a replay would read another call's list. */
#define C3_ATTENTION_CAPTURE_SEQUENCES 112

/* Device workspace bytes of c3_attention and of c3_attention_grad (256 at
 * least; 0 on invalid arguments). */
size_t c3_attention_workspace_size(const c3_attention_t *a);
size_t c3_attention_grad_workspace_size(const c3_attention_t *a);

/*
 * c3_attention -- out = softmax(scale q k^T over the keys that the mask
 * leaves) v, and per query and head lse = log of the sum of exp of the scaled
 * scores.  A query that sees no key gets out = 0 and lse = -inf, as does one
 * behind its sequence's q_len (the padding of a dense batch).  Keys behind
 * k_len, and whatever they hold, are not looked at; neither do values of keys
 * that the mask hides reach a query, infinities and NaN included.
 *
 *   q, out [..][heads][dim]; k, v [..][kv_heads][dim]; lse fp32 contiguous
 *   [batch][q_tokens][heads] (packed: [q_tokens][heads]).
 *   ws  256-byte aligned, c3_attention_workspace_size(a) bytes, not used by
 *       another call at the same time.
 * Can be captured, with lengths of C3_ATTENTION_CAPTURE_SEQUENCES sequences at most.
 * Errors: C3_E_INVAL, C3_E_ALIGN, C3_E_UNSUPPORTED (type, dim, 2^24 tiles of rows or
 * blocks of keys over all key heads or more, capture with more sequences),
 * C3_E_WORKSPACE, C3_E_HIP.
 */
int c3_attention(const c3_attention_t *a, const c3_attn_tensor_t *q, const c3_attn_tensor_t *k,
                 const c3_attn_tensor_t *v, const c3_attn_tensor_t *out, float *lse, void *ws,
                 size_t ws_bytes, c3_stream_t stream);

/*
 * c3_attention_grad -- gradients of c3_attention for the output gradient
 * `dout`.  The probabilities are recomputed from lse; with delta = the sum of
 * dout * out over a head,
 *     dv = P^T dout,  dS = P (dout v^T - delta),
 *     dq = scale dS k,  dk = scale dS^T q,
 * key heads summing over the query heads that share them.  Where a query of a tile sees
 * 16 keys or fewer, or the tile spans at most two blocks of 64 keys, its delta is the sum
 * of P * dout v^T, which the output's rounding does not enter.  out and lse are those of c3_attention for the same arguments.
 * Padding rows get zeros.  Results are deterministic.  Workspace and errors as c3_attention.
 */
int c3_attention_grad(const c3_attention_t *a, const c3_attn_tensor_t *dout,
                      const c3_attn_tensor_t *q, const c3_attn_tensor_t *k,
                      const c3_attn_tensor_t *v, const c3_attn_tensor_t *out, const float *lse,
                      const c3_attn_tensor_t *dq, const c3_attn_tensor_t *dk,
                      const c3_attn_tensor_t *dv, void *ws, size_t ws_bytes, c3_stream_t stream);

/* ---------------------------------------------------------------------- */
/* Tokens to their experts and back                                        */
/* ---------------------------------------------------------------------- */

#define C3_MAX_EXPERTS 512
#define C3_MAX_EXPERT_TOP 64

/* Device workspace bytes of c3_expert_sort (256 at least; 0 if invalid). */
size_t c3_expert_sort_workspace_size(int64_t choices, int experts);

/*
 * c3_expert_sort -- the order in which tokens go to experts: choices sorted
 * by expert, those of one expert in the order of their index (stable).
 *
 *   ids      device [choices] i32, choice c = token * top + t.  A value outside
 *            [0, experts) drops the choice.
 *   offsets  device [experts + 1] i32: expert e's rows are places
 *            offsets[e] .. offsets[e + 1] - 1.
 *   source   device [choices] i32: the choice at each place, -1 from
 *            offsets[experts] on.
 *   slot     device [choices] i32: each choice's place, -1 where dropped.
 *   0 <= choices < 2^31, 1 <= experts <= C3_MAX_EXPERTS; ws 256-byte aligned.
 */
int c3_expert_sort(const int32_t *ids, int64_t choices, int experts, int32_t *offsets,
                   int32_t *source, int32_t *slot, void *ws, size_t ws_bytes,
                   c3_stream_t stream);

/* Sizes shared by the calls that move rows: `tokens` rows of `hidden`
 * elements, `top` choices a token, slot [tokens][top] and `kept` (device, one
 * i32, offsets + experts) as c3_expert_sort wrote them.  Token-side rows are
 * token_stride elements apart, the tokens * top sorted rows sorted_stride.
 * Rows from *kept on hold no token: they are written as zeros, and what they
 * hold enters no result. */
typedef struct {
    int32_t dtype;
    int32_t top;            /* 1..C3_MAX_EXPERT_TOP */
    int64_t tokens;
    int64_t hidden;
    int64_t token_stride;
    int64_t sorted_stride;
    const int32_t *slot;
    const int32_t *kept;
} c3_expert_rows_t;

/* sorted[slot[t][i]] = x[t]. */
int c3_expert_dispatch(const c3_expert_rows_t *r, const void *x, void *sorted, c3_stream_t stream);

/* out[t] = sum over i of weights[t][i] * sorted[slot[t][i]], in the order of i;
 * dropped choices add nothing.  weights device fp32 [tokens][top] or NULL
 * (ones, which is c3_expert_dispatch's gradient). */
int c3_expert_combine(const c3_expert_rows_t *r, const void *sorted, const float *weights,
                      void *out, c3_stream_t stream);

/* Gradients of c3_expert_combine for dout [tokens][hidden]:
 * dsorted[slot[t][i]] = weights[t][i] * dout[t] (weights NULL: ones) and, where
 * dweights is not NULL, dweights[t][i] = <dout[t], sorted[slot[t][i]]> (0 where
 * dropped).  `sorted` may be NULL without dweights. */
int c3_expert_combine_grad(const c3_expert_rows_t *r, const void *dout, const void *sorted,
                           const float *weights, void *dsorted, float *dweights,
                           c3_stream_t stream);

/* ---------------------------------------------------------------------- */
/* Embedding                                                               */
/* ---------------------------------------------------------------------- */

/* Sizes of a lookup of `tokens` rows out of a table of `rows`, and of its
 * gradient.  Strides count elements and are not looked at where there is one row. */
typedef struct {
    int32_t dtype;          /* C3_F32, C3_BF16 or C3_F16                       */
    int32_t id_bytes;       /* 4 or 8: signed integers                         */
    int64_t tokens;
    int64_t rows;           /* of the table, 1 .. 2^31 - 1                     */
    int64_t hidden;         /* elements of a row                               */
    int64_t row_stride;     /* of the tokens' side: out, dout                  */
    int64_t table_stride;
    float scale;            /* finite                                          */
    int32_t reserved;
} c3_embedding_t;

/* c3_embedding -- out[t] = scale * table[ids[t]], rounded once; zeros for an id
 * outside [0, rows).  ids device [tokens].  `out` does not overlap the table. */
int c3_embedding(const c3_embedding_t *a, const void *ids, const void *table, void *out,
                 c3_stream_t stream);

/* Device workspace bytes of c3_embedding_grad (256 at least; 0 if invalid). */
size_t c3_embedding_grad_workspace_size(const c3_embedding_t *a);

/*
 * c3_embedding_grad -- dtable[v] = scale * the sum of dout[t] over the tokens
 * with ids[t] = v, rounded once; ids outside [0, rows) add nothing.  Tokens are
 * sorted by row; a row's sum runs in the order of its tokens, in parts that its
 * place in the sorted list fixes.
 *
 *   dtable       [rows][hidden] of dtype or of C3_F32 (table_dtype), table_stride
 *                apart; all rows are written, those without a token as zeros.
 *   accumulate   not 0: rows with tokens get their sum added, others are left as
 *                they are (a table that is also the output's weights).
 *   ws           256-byte aligned, not used by another call at the same time.
 * Can be captured.  dtable overlaps no input.
 */
int c3_embedding_grad(const c3_embedding_t *a, const void *dout, const void *ids, void *dtable,
                      int table_dtype, int accumulate, void *ws, size_t ws_bytes,
                      c3_stream_t stream);

/* ---------------------------------------------------------------------- */
/* Residual sum and norms around a block                                   */
/* ---------------------------------------------------------------------- */

#define C3_MAX_NORM_HIDDEN 16384

typedef enum {
    C3_GATE_NONE = 0,
    C3_GATE_CHANNELS = 1,   /* [hidden], the same for every token */
    C3_GATE_TOKENS = 2      /* [tokens][hidden]                   */
} c3_gate_t;

/* Sizes and types of c3_residual_norm.  Strides as in c3_embedding_t. */
typedef struct {
    int32_t dtype;          /* of y, gate, weight, post, n and their gradients  */
    int32_t residual;       /* of x, h, dh and dx: dtype or C3_F32              */
    int64_t tokens;
    int64_t hidden;         /* 1 .. C3_MAX_NORM_HIDDEN                          */
    float scale;            /* of the block's output, finite                    */
    float eps;              /* added to the mean of squares, >= 0               */
    int32_t gate;           /* c3_gate_t                                        */
    int32_t reserved;
} c3_residual_norm_t;

/* Rows [tokens][hidden], last dimension contiguous; ptr NULL: not there. */
typedef struct {
    void *ptr;
    int64_t stride;
} c3_rows_t;

/*
 * c3_residual_norm -- joins a block's output y to the residual stream x and
 * norms the sum for the next block:
 *     z = post * y / rms(y)      (without post: z = y)
 *     h = x + scale * gate * z   (without y: h = x, not written)
 *     n = weight * h / rms(h)    with rms(a) = sqrt(mean of a^2 + eps),
 * in 32 bits, n from h before it is rounded.
 *
 *   y      may be missing, and then has neither gate nor post.
 *   gate   [hidden] (stride unused) or rows, by a->gate.
 *   weight, post  device [hidden], post may be NULL.
 *   h      may be x with the same stride; no other overlaps.
 *   stats  device fp32 [tokens][2]: 1 / rms(h), and 1 / rms(y) (1 without post).
 * Can be captured.
 */
int c3_residual_norm(const c3_residual_norm_t *a, const c3_rows_t *x, const c3_rows_t *y,
                     const c3_rows_t *gate, const void *weight, const void *post,
                     const c3_rows_t *h, const c3_rows_t *n, float *stats, c3_stream_t stream);

/* Device workspace bytes of c3_residual_norm_grad (256 at least; 0 if invalid). */
size_t c3_residual_norm_grad_workspace_size(const c3_residual_norm_t *a);

/*
 * c3_residual_norm_grad -- gradients for dn, that of n, and dh, that of h from
 * what else reads it (ptr NULL: zeros).  stats are those of c3_residual_norm.
 * dx is the gradient of x (and of h as a whole); dy, and dgate as rows, are there
 * where y and such a gate are.  Sums over the tokens go to sums, device fp32
 * [3][hidden]: of weight, of post (left alone without post) and of a gate of
 * channels (left alone without one).  They run in an order that the sizes fix.
 *   dx may be dh with the same stride, dy may be dn with the same stride; results
 *   overlap nothing else.  ws as c3_embedding_grad.  Can be captured.
 */
int c3_residual_norm_grad(const c3_residual_norm_t *a, const c3_rows_t *dn, const c3_rows_t *dh,
                          const c3_rows_t *x, const c3_rows_t *y, const c3_rows_t *gate,
                          const void *weight, const void *post, const float *stats,
                          const c3_rows_t *dx, const c3_rows_t *dy, const c3_rows_t *dgate,
                          float *sums, void *ws, size_t ws_bytes, c3_stream_t stream);

/* ---------------------------------------------------------------------- */
/* Loss over a vocabulary                                                  */
/* ---------------------------------------------------------------------- */

/* Sizes and types of a softmax cross entropy of hidden states x [tokens][hidden] over
 * the rows of weight [rows][hidden].  Pointers of x, weight, dx and dweight are 16-byte
 * aligned, their last dimension contiguous and their strides (elements; not looked at
 * where there is one row) multiples of 8 below 2^22. */
typedef struct {
    int32_t dtype;          /* C3_BF16 or C3_F16                               */
    int32_t target_bytes;   /* 4 or 8: signed integers                         */
    int64_t tokens;
    int64_t hidden;         /* a multiple of 8 below 2^20                      */
    int64_t rows;           /* of the vocabulary                               */
    int64_t x_stride;
    int64_t weight_stride;
    float scale;            /* of the logits, finite                           */
    int32_t reserved;
} c3_vocab_loss_t;

/* Device workspace bytes of c3_vocab_loss and of c3_vocab_loss_grad (256 at least; 0 if
 * invalid).  The gradient's holds d for a piece of the vocabulary: up to 512 MiB, or beyond
 * 131,072 tokens 4 KiB a token. */
size_t c3_vocab_loss_workspace_size(const c3_vocab_loss_t *a);
size_t c3_vocab_loss_grad_workspace_size(const c3_vocab_loss_t *a);

/*
 * c3_vocab_loss -- with the logits l = scale * x[t] . weight[v], which are not kept,
 *     lse[t] = log of the sum over v of exp(l[t][v]),  loss[t] = lse[t] - l[t][targets[t]].
 * A token whose target is outside [0, rows) takes no part: its loss and lse are 0 and
 * what its row of x holds is not looked at.
 *   targets device [tokens]; loss, lse device fp32 [tokens].
 *   ws      256-byte aligned, not used by another call at the same time.
 * Can be captured.  Errors: C3_E_INVAL, C3_E_ALIGN, C3_E_UNSUPPORTED (type, hidden,
 * stride, 2^26 tokens, 2^28 rows or 2^22 tiles of 256 by 256 between any two of tokens,
 * rows and hidden, or more), C3_E_WORKSPACE, C3_E_HIP.
 */
int c3_vocab_loss(const c3_vocab_loss_t *a, const void *x, const void *weight, const void *targets,
                  float *loss, float *lse, void *ws, size_t ws_bytes, c3_stream_t stream);

/*
 * c3_vocab_loss_grad -- gradients of c3_vocab_loss for dloss fp32 [tokens], dloss_stride
 * elements apart (0: one number for all): with d = scale * dloss[t] * (exp(l - lse[t]) -
 * onehot(targets[t])), dx = d weight and dweight = d^T x.  d, relative to the largest
 * finite dloss, is rounded to 16 bits on its way into the products; what rounding leaves
 * of the target's entry, and up to 128 tokens of all of a token's, enters both results as
 * well.  In C3_F16 steps of d are no smaller than 2^-37 of that dloss.  All sums are fp32,
 * in an order that the sizes and the targets fix: from 129 tokens on dweight's run over
 * the tokens in the order of their targets.  lse is that of c3_vocab_loss.  dx and dweight
 * are of a->dtype; rows of dx whose token takes no part are zeros.  Results overlap
 * neither inputs nor each other.  Workspace and errors as c3_vocab_loss.  Can be captured.
 */
int c3_vocab_loss_grad(const c3_vocab_loss_t *a, const float *dloss, int64_t dloss_stride,
                       const void *x, const void *weight, const void *targets, const float *lse,
                       void *dx, int64_t dx_stride, void *dweight, int64_t dweight_stride, void *ws,
                       size_t ws_bytes, c3_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* C3_REPLAY_H_ */
