/*
 * adascale_ops.h - C ABI of the language-model operators that stand beside the AdaScale step
 * (adascale.h) on one NVIDIA B200 (sm_100a).
 *
 * The step consumes S gradient rows of a model; these calls produce the parts of such a row, and
 * of the training step around it, that a library's matrix products and attention do not:
 *
 *   adascale_embed, adascale_embed_grad            token table: scaled lookup, gradient by sorted tokens
 *   adascale_distill                               loss against a teacher's top logits, with its gradient
 *   adascale_residual_norm, ..._residual_norm_grad block boundary: norm, gate, residual scale, norm
 *   adascale_position_softmax, ..._grad            attention weights with a relative position bias by buckets
 *   adascale_expert_matmul, ..._grad               products with experts' weights over ragged groups of rows
 *   adascale_clip_grads                            global norm of many gradients, clipping on the way into a row's slots
 *
 * Conventions (those of adascale.h, and)
 *   - Every call takes one struct of arguments (host pointer, read during the call) and a
 *     cudaStream_t as void* (NULL = default stream).  It enqueues on that stream and returns; it
 *     never waits for the device, allocates nothing and keeps nothing, so it can be captured into
 *     a graph and called from several threads and streams at once, as long as each call in flight
 *     has its own workspace.
 *   - The device is the calling thread's current one; all pointers are device pointers on it.
 *   - Matrices are row-major with a row stride `ld_*` in elements (>= the row's length); elements of a row
 *     are adjacent.  Rows that start on 16-byte boundaries are fastest; any alignment to the
 *     element's own size is accepted.
 *   - dtype fields are adascale_dtype (ADASCALE_F32, ADASCALE_BF16).  All arithmetic, sums and
 *     statistics are 32-bit or wider; a bf16 result is rounded once, to nearest even, when it is stored.
 *   - What a gradient call has enqueued last does not let the stream's next kernel start before it has stored its results, so
 *     adascale_step may follow directly, with ADASCALE_FLAG_GRADS_READY too.
 *   - Results are the same bits from run to run: no sum depends on the order in which blocks run.
 *   - Inputs and outputs must not overlap unless a field says so.
 *   - Waits inside a kernel (for its own copies and instructions) are bounded, by seconds in which it gets no further: results that
 *     were not computed because one ran out are NaN, and the kernel ends when its copies in flight have come.  The call has
 *     returned by then: no status tells of it.
 *   - Errors: INVALID_ARG (null pointer, negative size, unknown enum, stride below the row's length,
 *     non-finite constant, workspace too small), ALIGNMENT (a pointer not aligned to its element size),
 *     TOO_LARGE (beyond a maximum below), CUDA (a launch failed).  Nothing is enqueued after an error of the first three kinds.
 *     A size of zero rows or tokens is no error.
 */
#ifndef ADASCALE_OPS_H_
#define ADASCALE_OPS_H_

#include "adascale.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ADASCALE_I32 = 0, ADASCALE_I64 = 1 } adascale_itype; /* token ids and labels */

#define ADASCALE_OPS_MAX_ROWS 2147483647LL /* tokens or rows of one call, vocabulary size - 1 */
#define ADASCALE_EMBED_MAX_DIM 1073741824LL /* width of a token table */
#define ADASCALE_DISTILL_MAX_K 1024        /* entries of a teacher's list */
#define ADASCALE_NORM_MAX_DIM 16384        /* width of a block boundary */
#define ADASCALE_POSITION_MAX_BUCKETS 128  /* buckets of relative positions */
#define ADASCALE_POSITION_MAX_DISTANCE 16384 /* distance from which on all are in the last bucket */
#define ADASCALE_EXPERT_MAX_EXPERTS 1024   /* experts of one product */
#define ADASCALE_EXPERT_MAX_DIM 1048576    /* width of an expert's input or output */
#define ADASCALE_CLIP_MAX_TENSORS 65536    /* gradients of one norm */

/*
 * out[n, :] = scale * table[token[n], :].  A token outside 0 .. vocab-1 gives a row of zeros (and
 * has no gradient).  Reads the tokens and the rows that they name, writes n_tokens x dim.
 */
typedef struct {
    const void *tokens; /* [n_tokens] of token_type */
    const void *table;  /* [vocab, dim] */
    void *out;          /* [n_tokens, dim] */
    int64_t n_tokens, vocab, dim;
    int64_t ld_table, ld_out;
    int32_t token_type; /* adascale_itype */
    int32_t table_dtype, out_dtype;
    float scale;
} adascale_embed_args;
adascale_status adascale_embed(const adascale_embed_args *args, void *cuda_stream);

/*
 * grad[v, :] (+)= scale * sum over n with token[n] = v, in the order of n, of dout[n, :].
 * Without `accumulate` the whole table's gradient is written, zeros where no token points; with it
 * the sums are added to what grad holds and rows of absent tokens are not touched (a tied table
 * whose output projection has already left its part, or several batches into one gradient row).
 * Adding to a float32 grad is one addition per element by the L2 cache, which takes subnormal numbers for zeros: below
 * 2^-126 what grad holds, or the result, may be lost.
 * Tokens equal to padding_idx (-1: none) or outside 0 .. vocab-1 have no part in it.
 * The tokens are sorted first (stable, so the order of every sum is fixed); a row with many
 * tokens is cut into pieces whose sums are joined in order.
 * workspace: at least adascale_embed_grad_workspace(n_tokens, dim) bytes, 16-byte aligned, contents
 * neither expected nor kept.
 */
typedef struct {
    const void *tokens; /* [n_tokens] of token_type */
    const void *dout;   /* [n_tokens, dim] */
    void *grad;         /* [vocab, dim] */
    void *workspace;
    int64_t workspace_bytes;
    int64_t n_tokens, vocab, dim;
    int64_t ld_dout, ld_grad;
    int64_t padding_idx;
    int32_t token_type; /* adascale_itype */
    int32_t dout_dtype, grad_dtype;
    int32_t accumulate;
    float scale;
} adascale_embed_grad_args;
adascale_status adascale_embed_grad(const adascale_embed_grad_args *args, void *cuda_stream);
/* Bytes of workspace for the sizes; 0 for sizes that the call would refuse. */
int64_t adascale_embed_grad_workspace(int64_t n_tokens, int64_t dim);

/*
 * Distillation from a teacher's top logits, mixed with the cross entropy of labels.  For row n, with
 * student logits z (vocab), teacher logits t and token ids i of its list (n_top entries), label y:
 *
 *   q_k   = exp(t_k / T) / sum_j exp(t_j / T)           over the list's valid entries
 *   p^T_v = exp(z_v / T) / sum_u exp(z_u / T)
 *   row_loss = weight * [ alpha T^2 sum_k q_k (log q_k - log p^T_{i_k})  -  beta log p^1_y ]
 *   dlogits_v = weight * [ alpha T (p^T_v - sum_{k: i_k = v} q_k)  +  beta (p^1_v - [v = y]) ]
 *   loss  = sum of row_loss
 *
 * dlogits is the gradient of `loss`; an upstream factor per row goes into `weight`.
 * - A list entry whose id is outside 0 .. vocab-1 or whose logit is -inf is left out (lists of
 *   different lengths are filled up with id -1); an id may occur twice.  A row without valid entries has no
 *   alpha part, a row whose label is outside 0 .. vocab-1 (or -100) no beta part.
 * - A row with weight 0, or with neither part, or whose logits are all -inf, has loss 0 and a
 *   gradient of zeros whatever its logits hold; logits of weight-0 rows are not read.
 * - Masked vocabulary entries may hold -inf or the type's lowest value.  NaN or +inf in a live row
 *   make that row's loss and gradient NaN, and `loss` with it.  NaN or +inf among the teacher's logits of valid
 *   entries makes q NaN: the row's loss, and the gradient of every entry that the list names.
 * - Probabilities below 2^-126 count as 0, gradients below it may be 0.
 * - dlogits (type of logits) may be NULL: the loss alone.  It may be logits itself (same ld).
 * - teacher_logits and teacher_ids may be NULL when n_top = 0; labels and weight may be NULL.
 */
typedef struct {
    const void *logits;         /* [n_rows, vocab] of dtype */
    void *dlogits;              /* [n_rows, vocab] of dtype, or NULL */
    const void *teacher_logits; /* [n_rows, n_top] of teacher_dtype */
    const void *teacher_ids;    /* [n_rows, n_top] of id_type */
    const void *labels;         /* [n_rows] of label_type, or NULL */
    const float *weight;        /* [n_rows], or NULL (1) */
    float *row_loss;            /* [n_rows] */
    float *loss;                /* [1] */
    int64_t n_rows, vocab, n_top;
    int64_t ld_logits, ld_dlogits, ld_teacher, ld_ids;
    int32_t dtype, teacher_dtype;
    int32_t id_type, label_type; /* adascale_itype */
    float temperature;           /* T, within 1e-3 .. 1e3 */
    float alpha, beta;           /* finite, >= 0 */
} adascale_distill_args;
adascale_status adascale_distill(const adascale_distill_args *args, void *cuda_stream);

/*
 * Block boundary of a Transformer.  With the residual stream x, the block's output y, residual
 * scale s and gate G:
 *
 *   u  = post(y)                          norm after the block   (NONE, RMS or LAYER)
 *   x' = x + s * G * u                    G = 1, g[d] per channel, or sigmoid(a[n, d])
 *   h  = pre(x')                          norm before the next block  (RMS or LAYER)
 *
 *   RMS(v)   = v / sqrt(mean(v^2) + eps) * w
 *   LAYER(v) = (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * w + b
 *
 * y may be NULL: then x' = x, x_new is not written (it may be NULL) and h = pre(x): the norm
 * before the first block.  x_new may be x itself (same ld), h may be y itself.  b_* are read for
 * LAYER only and may be NULL (0).  The stream (x, x_new) and the block's side (y, gate matrix, h)
 * have a type each; weights and the channel gate are float32.
 */
typedef enum { ADASCALE_NORM_NONE = 0, ADASCALE_NORM_RMS = 1, ADASCALE_NORM_LAYER = 2 } adascale_norm_kind;
typedef enum { ADASCALE_GATE_NONE = 0, ADASCALE_GATE_CHANNEL = 1, ADASCALE_GATE_SIGMOID = 2 } adascale_gate_kind;

typedef struct {
    const void *x;       /* [n_rows, dim] of x_dtype */
    const void *y;       /* [n_rows, dim] of y_dtype, or NULL */
    void *x_new;         /* [n_rows, dim] of x_dtype */
    void *h;             /* [n_rows, dim] of y_dtype */
    const void *gate;    /* CHANNEL: float32 [dim]; SIGMOID: [n_rows, dim] of y_dtype */
    const float *w_post, *b_post, *w_pre, *b_pre; /* [dim] */
    int64_t n_rows, dim;
    int64_t ld_x, ld_y, ld_x_new, ld_h, ld_gate;
    int32_t x_dtype, y_dtype;
    int32_t post, pre, gate_kind;
    float res_scale, eps;
} adascale_residual_norm_args;
adascale_status adascale_residual_norm(const adascale_residual_norm_args *args, void *cuda_stream);

/*
 * Its gradient, from the stream after the block (x' of the forward call) and the block's output; the
 * rows' statistics are worked out again.  With dx' arriving at the stream (NULL: none) and dh at h:
 *
 *   dx = dx' + pre^T(dh)                  gradient of x (and of x' as a whole)
 *   dy = post^T(s G dx),  dG = s u dx;  SIGMOID: da = dG G (1 - G), CHANNEL: column sums of dG
 *   dw, db: column sums over the rows, written in wgrad_dtype (the gradient row's type)
 *
 * dx may be dx_new itself, dy may be dh itself (same ld).  Outputs other than dx may be NULL and are then left out.
 * workspace: at least adascale_residual_norm_grad_workspace(n_rows, dim) bytes, 16-byte aligned, contents
 * neither expected nor kept.
 */
typedef struct {
    const void *x_new;   /* [n_rows, dim] of x_dtype: the stream after the block */
    const void *y;       /* [n_rows, dim] of y_dtype, or NULL (then only dx, dw_pre, db_pre) */
    const void *dx_new;  /* [n_rows, dim] of x_dtype, or NULL */
    const void *dh;      /* [n_rows, dim] of y_dtype */
    const void *gate;    /* as in the forward call */
    const float *w_post, *b_post, *w_pre; /* [dim]; b_post only with a gate */
    void *dx;            /* [n_rows, dim] of x_dtype */
    void *dy;            /* [n_rows, dim] of y_dtype */
    void *dgate;         /* SIGMOID: [n_rows, dim] of y_dtype; CHANNEL: [dim] of wgrad_dtype */
    void *dw_post, *db_post, *dw_pre, *db_pre; /* [dim] of wgrad_dtype */
    void *workspace;
    int64_t workspace_bytes;
    int64_t n_rows, dim;
    int64_t ld_x_new, ld_y, ld_dx_new, ld_dh, ld_gate, ld_dx, ld_dy, ld_dgate;
    int32_t x_dtype, y_dtype, wgrad_dtype;
    int32_t post, pre, gate_kind;
    float res_scale, eps;
} adascale_residual_norm_grad_args;
adascale_status adascale_residual_norm_grad(const adascale_residual_norm_grad_args *args, void *cuda_stream);
int64_t adascale_residual_norm_grad_workspace(int64_t n_rows, int64_t dim);

/*
 * Attention weights from scores, with a learned bias by relative position.  For batch b, head h, query i at position
 * start[b] + i, key j at position j:
 *
 *   p[b,h,i,j] = softmax over the live keys j of  scale * s[b,h,i,j] + table[bucket(j - (start[b] + i)), h]
 *
 * Live are the keys with j < length[b] and, if causal, j <= start[b] + i.  Others get 0, whatever the scores hold there (they
 * are not used); a query without live keys, or whose live keys all have -inf, gets zeros.  NaN or +inf at a live key makes
 * its query's row NaN (at the live keys).  scale * s + bias is 32-bit arithmetic: the type's lowest value swallows the bias.
 *
 * Buckets: with m = n_buckets (half of them if bidirectional), e = m / 2 and n = |distance| (not bidirectional: the distance
 * back, 0 for keys ahead), n < e has bucket n, and n >= e the bucket e + floor((m - e) log(n / e) / log(max_distance / e)),
 * m - 1 at most, without rounding: a distance that lies on a border belongs to the bucket above it.  Bidirectional: keys ahead
 * have m more.  n_buckets is even and at least 4 if bidirectional, at least 2 otherwise; max_distance > e.
 *
 * probs may be scores itself (same strides).  Strides are in elements and may be 0 for inputs; rows of probs do not overlap; the
 * keys of a row are adjacent.  n_queries and n_keys are at most 2^29.  lengths and starts are clamped: to 0 .. n_keys and to
 * +-2^30.  Weights below 2^-126 may be 0.
 */
typedef struct {
    const void *scores;  /* [batch, heads, n_queries, n_keys] of dtype */
    void *probs;         /* the same, of dtype */
    const float *table;  /* [n_buckets, heads] */
    const void *lengths; /* [batch] of length_type, or NULL (n_keys) */
    const void *starts;  /* [batch] of start_type, or NULL (0) */
    int64_t batch, heads, n_queries, n_keys;
    int64_t scores_stride_b, scores_stride_h, scores_stride_q;
    int64_t probs_stride_b, probs_stride_h, probs_stride_q;
    int64_t ld_table;
    int32_t dtype;
    int32_t length_type, start_type; /* adascale_itype */
    int32_t n_buckets, max_distance, bidirectional, causal;
    float scale;
} adascale_position_softmax_args;
adascale_status adascale_position_softmax(const adascale_position_softmax_args *args, void *cuda_stream);

/*
 * Its gradient from the weights p of the forward call and dp arriving at them; lengths, starts and causal as there:
 *
 *   g = p (dp - sum over the live j of p dp),   dscores = scale * g
 *   dtable[k, h] (+)= sum of g over all b, i and live j in bucket k, written in wgrad_dtype
 *
 * Keys that are not live get 0 and are not used.  Without `accumulate` dtable is written, with it the sums are added to what it
 * holds (a table that several layers share).  dscores may be dprobs or probs itself (same strides).  dscores or dtable may be
 * NULL.  workspace: at least adascale_position_softmax_grad_workspace(heads, n_buckets) bytes, 16-byte aligned, contents
 * neither expected nor kept.
 */
typedef struct {
    const void *probs, *dprobs; /* [batch, heads, n_queries, n_keys] of dtype */
    void *dscores;              /* the same, or NULL */
    void *dtable;               /* [n_buckets, heads] of wgrad_dtype, or NULL */
    const void *lengths;        /* [batch] of length_type, or NULL */
    const void *starts;         /* [batch] of start_type, or NULL */
    void *workspace;
    int64_t workspace_bytes;
    int64_t batch, heads, n_queries, n_keys;
    int64_t probs_stride_b, probs_stride_h, probs_stride_q;
    int64_t dprobs_stride_b, dprobs_stride_h, dprobs_stride_q;
    int64_t dscores_stride_b, dscores_stride_h, dscores_stride_q;
    int64_t ld_dtable;
    int32_t dtype, wgrad_dtype;
    int32_t length_type, start_type; /* adascale_itype */
    int32_t n_buckets, max_distance, bidirectional, causal;
    int32_t accumulate;
    float scale;
} adascale_position_softmax_grad_args;
adascale_status adascale_position_softmax_grad(const adascale_position_softmax_grad_args *args, void *cuda_stream);
int64_t adascale_position_softmax_grad_workspace(int64_t heads, int64_t n_buckets);

/*
 * Products with experts' weights over ragged groups of rows: for the rows r of expert e, offsets[e] <= r < offsets[e + 1],
 *
 *   y[r, :] = w[e] x[r, :]
 *
 * x and w are bf16; sums are 32-bit, y is rounded once.  The tensor cores cut where they add: a sum of terms of one sign comes out too small
 * by up to 2e-6 of itself before it is stored as float32, 1e-4 (a twentieth of the rounding) as bf16, whatever its length.  offsets has n_experts + 1 ascending numbers on the device;
 * rows before the first or behind the last, up to n_rows, are neither used nor written.  Offsets outside 0 .. n_rows are
 * clamped, and one below an earlier one counts as that.  An expert may have no rows.
 * The rows of x and w start on 16-byte boundaries (ALIGNMENT otherwise): strides are multiples of 8 elements.  Widths may be odd.
 */
typedef struct {
    const void *x;       /* [n_rows, in_dim] of bf16 */
    const void *w;       /* [n_experts, out_dim, in_dim] of bf16 */
    void *y;             /* [n_rows, out_dim] of y_dtype */
    const void *offsets; /* [n_experts + 1] of offset_type */
    int64_t n_rows, n_experts, in_dim, out_dim;
    int64_t ld_x, ld_w, stride_w, ld_y; /* stride_w: from expert to expert */
    int32_t offset_type;                /* adascale_itype */
    int32_t y_dtype;
} adascale_expert_matmul_args;
adascale_status adascale_expert_matmul(const adascale_expert_matmul_args *args, void *cuda_stream);

/*
 * Its gradients from dy [n_rows, out_dim] of bf16:
 *
 *   dx[r, :] = w[e]^T dy[r, :]                          for the rows r of expert e
 *   dw[e]  (+)= sum over the rows r of e of dy[r, :] x[r, :]^T     in dw_dtype
 *
 * Without `accumulate` all of dw is written, zeros for experts without rows; with it the sums are added to what dw holds and
 * experts without rows are not touched.  Adding to a float32 dw may be one addition per element by the L2 cache, which takes subnormal
 * numbers for zeros.  w = NULL leaves dx out, x = NULL dw.  Rows of dy, x and w start on 16-byte boundaries.  With n_rows = 0 none of dy, x
 * and dx is looked at, and dw, where it is not NULL, is all zeros without `accumulate`, whether x is NULL or not.
 */
typedef struct {
    const void *dy;      /* [n_rows, out_dim] of bf16 */
    const void *x;       /* [n_rows, in_dim] of bf16, or NULL (no dw) */
    const void *w;       /* [n_experts, out_dim, in_dim] of bf16, or NULL (no dx) */
    void *dx;            /* [n_rows, in_dim] of dx_dtype */
    void *dw;            /* [n_experts, out_dim, in_dim] of dw_dtype */
    const void *offsets; /* [n_experts + 1] of offset_type */
    int64_t n_rows, n_experts, in_dim, out_dim;
    int64_t ld_dy, ld_x, ld_w, stride_w, ld_dx, ld_dw, stride_dw;
    int32_t offset_type; /* adascale_itype */
    int32_t dx_dtype, dw_dtype, accumulate;
} adascale_expert_matmul_grad_args;
adascale_status adascale_expert_matmul_grad(const adascale_expert_matmul_grad_args *args, void *cuda_stream);

/*
 * Global 2-norm of many gradients, and clipping by it:
 *
 *   norm = sqrt(sum over all tensors and elements of g^2)
 *   out  = c g,   c = min(1, max_norm / (norm + eps))
 *
 * grads, out, numels, grad_dtypes and out_dtypes are HOST arrays of n_tensors entries, read during the call (which uses host memory
 * of their size until it returns): device
 * addresses, element counts (0 is allowed, its addresses are not looked at) and adascale_dtype of each tensor, whose elements are
 * adjacent.  out = NULL: the norm alone.  out[k] may be grads[k] itself with the same type (if c = 1 nothing is written
 * then); otherwise it overlaps neither another output nor a gradient.  No output may be given twice.
 * Sums are 64-bit joins of 32-bit sums of a few terms; where squares leave the 32-bit range they are 64-bit throughout.  A NaN
 * anywhere makes norm and all of out NaN; with an infinity and no NaN norm is inf, c 0, and out 0, NaN in the infinity's place.
 * A call per gradient row clips each row by its own norm: what adascale_step then sees, and its gain is of, are clipped gradients.
 * workspace: at least adascale_clip_grads_workspace(n_tensors) bytes, 16-byte aligned, contents neither expected nor kept.
 */
typedef struct {
    const void *const *grads;
    void *const *out;           /* or NULL */
    const int64_t *numels;
    const int32_t *grad_dtypes; /* adascale_dtype of each */
    const int32_t *out_dtypes;  /* of each; NULL with out = NULL */
    float *norm;                /* [1] */
    void *workspace;
    int64_t workspace_bytes;
    int64_t n_tensors;
    float max_norm, eps;        /* finite, >= 0; only with out */
} adascale_clip_grads_args;
adascale_status adascale_clip_grads(const adascale_clip_grads_args *args, void *cuda_stream);
int64_t adascale_clip_grads_workspace(int64_t n_tensors);

#ifdef __cplusplus
}
#endif
#endif /* ADASCALE_OPS_H_ */
