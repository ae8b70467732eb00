/*
 * gockpt_model.h -- operators of a language model's own forward and backward:
 * the head's cross entropy with its gradients, activations kept in 8 bits for
 * the backward pass, and the layers that keep them so.
 *
 * They stand between the lookup and the clip of gockpt_ops.h: the head reads
 * the table that the lookup reads, its gradient and the linear layers' go into
 * their parts of the flat 16-bit gradient (or into fp32 sums that the clip
 * rounds into it), and gockpt_step follows.
 *
 * Conventions are those of gockpt_ops.h: int status, the text of a failing call
 * from gockpt_last_error(NULL) on the calling thread, caller-owned buffers, no
 * C++ exception crosses.  Every call is asynchronous on `stream`, launches
 * kernels only and may be captured in a HIP graph.  The same inputs in the same
 * layout give the same bits on every call.  Workspaces are 256-byte aligned, of
 * the bytes that the call's own size function tells for the same arguments, and
 * in use until the call's kernels have run; what a call reads must not overlap
 * what it writes.
 *
 * Products run on the matrix cores in the inputs' 16-bit type with fp32 sums.
 * Matrices whose data and row stride are multiples of 16 bytes and whose columns
 * are a multiple of 8 are read in place; others are first copied into the
 * workspace.
 */
#ifndef GOCKPT_MODEL_H
#define GOCKPT_MODEL_H

#include "gockpt_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the head's cross entropy ---------------------------------------------- */

/* hidden: one row for each token, table: one row for each class, as many
 * columns, both bf16 or both fp16.  Token t has the logits l[t][v] = scale *
 * <hidden row t, table row v>.  Its target's class is targets[t]; it counts
 * when that is not ignore_id and lies in [first_id, first_id + table.rows), or,
 * with classes > 0, in [0, classes): then the table is this rank's range of so
 * many classes.  Any other token (padding marked by -1, say) is masked: no
 * loss, no gradient, and what its hidden row holds does not matter. */
typedef struct {
    gockpt_matrix hidden, table;
    gockpt_token_ids targets; /* as many as hidden has rows */
    int64_t ignore_id;        /* INT64_MIN: none */
    int64_t classes;          /* 0, or the classes of all ranks' tables */
    float scale;
    int32_t reserved_;
} gockpt_head;

/* How token losses make the loss. */
#define GOCKPT_EACH 0 /* one for each token */
#define GOCKPT_SUM 1
#define GOCKPT_MEAN 2 /* over the tokens that count; 0 where none does */

/* Workspace bytes of gockpt_head_loss.  Host only.  Errors: EINVAL. */
int gockpt_head_loss_bytes(const gockpt_head* head, size_t* bytes);

/* lse[t] = log sum over the table's rows v of exp l[t][v]; logit[t] =
 * l[t][target], 0 where the target is not in the table; loss[t] = lse[t] -
 * logit[t], or their sum or mean; all zeros for masked tokens.  Each may be NULL
 * (device, fp32).  The logits are not kept: each tile of them leaves its rows'
 * maximum and sum of exponentials.  With classes > 0, loss must be NULL: the
 * ranks put their lse (log of the sum of exp) and logit (sum) together.
 * Errors: EINVAL, ENOMEM (workspace), EHIP. */
int gockpt_head_loss(const gockpt_head* head, int reduction, float* loss, float* lse, float* logit, void* workspace,
                     size_t workspace_bytes, void* stream);

/* Workspace bytes of gockpt_head_grad; grad_hidden and grad_table are those of
 * the call (NULL: not wanted).  Host only.  Errors: EINVAL. */
int gockpt_head_grad_bytes(const gockpt_head* head, const gockpt_matrix* grad_hidden,
                           const gockpt_matrix* grad_table, size_t* bytes);

/* The gradients of the loss, from lse over all classes: with z[t][v] = g[t] *
 * (exp(l[t][v] - lse[t]) - [v is t's target]),
 *   grad_hidden row t = round(scale * sum over v of z[t][v] * table row v),
 *   grad_table row v  = round(scale * sum over t of z[t][v] * hidden row t).
 * g: grad[t] with GOCKPT_EACH, else grad[0], with GOCKPT_MEAN over the number
 * of tokens that count.  Either may be NULL; of any of the three types.  With
 * accumulate grad_table becomes round(old + its sum).  Logits are computed
 * again in pieces of the vocabulary; z is rounded to the inputs' type, scaled
 * by a power of two so that fp16 keeps what a loss scale lifts, and all sums are
 * fp32.  For grad_hidden with GOCKPT_EACH each token has a power of two of its
 * own; for grad_table all share one, and in fp16 each z is off by up to 2^-38 of
 * the largest |g|.
 * Errors: EINVAL, ENOMEM (workspace), EHIP. */
int gockpt_head_grad(const gockpt_head* head, const float* lse, int reduction, const float* grad,
                     const gockpt_matrix* grad_hidden, const gockpt_matrix* grad_table, int accumulate,
                     void* workspace, size_t workspace_bytes, void* stream);

/* ---- activations in 8 bits ------------------------------------------------- */

#define GOCKPT_ACT8_BLOCK 32

/* rows x cols values: each 32 columns of a row (the last block of a row may
 * have fewer) share a scale 2^e, e the least with max |x| <= 127 * 2^e and at
 * least -126; a value is kept as the code nearest to x / 2^e (ties to even) and
 * stands for code * 2^e, which bf16, fp16 and fp32 all hold exactly (fp16 within
 * its range: values of another type beyond it are rounded).  Row r has
 * its codes (int8) at codes + r * 32 * blocks, zeros behind its last column, and
 * its scales (e + 127 as a byte) at scales + r * blocks, blocks = ceil(cols /
 * 32).  A block with an inf or NaN has the scale 255 and stands for NaN.  (Where
 * 64 * 2^e would be beyond the source's type the code is at most 63.) */
typedef struct {
    void* codes;  /* device, 16-byte aligned */
    void* scales; /* device */
    int64_t rows, cols;
} gockpt_act8;

/* Errors of both: EINVAL, EHIP. */
int gockpt_act8_pack(const gockpt_matrix* x, const gockpt_act8* out, void* stream);
int gockpt_act8_unpack(const gockpt_act8* x, const gockpt_matrix* out, void* stream);

/* ---- linear layer that keeps its input in 8 bits ---------------------------- */

/* out = round(x weight^T): x has one row for each token, weight one for each
 * output; both bf16 or both fp16, out of any of the three types.  keep: where x
 * goes in 8 bits (NULL: nowhere).  Errors: EINVAL, ENOMEM (workspace), EHIP. */
int gockpt_linear8_bytes(const gockpt_matrix* x, const gockpt_matrix* weight, size_t* bytes);
int gockpt_linear8(const gockpt_matrix* x, const gockpt_matrix* weight, const gockpt_matrix* out,
                   const gockpt_act8* keep, void* workspace, size_t workspace_bytes, void* stream);

/* grad_x = round(grad_out weight), grad_weight = round(grad_out^T kept), with
 * accumulate round(old + it).  Either may be NULL; weight may be NULL without
 * grad_x, keep without grad_weight.  grad_out is of the weight's type, and of
 * bf16 or fp16, and kept is multiplied in that type; the gradients are of any of
 * the three.  Errors: EINVAL, ENOMEM (workspace), EHIP. */
int gockpt_linear8_grad_bytes(const gockpt_matrix* grad_out, const gockpt_matrix* weight, const gockpt_act8* keep,
                              const gockpt_matrix* grad_x, const gockpt_matrix* grad_weight, size_t* bytes);
int gockpt_linear8_grad(const gockpt_matrix* grad_out, const gockpt_matrix* weight, const gockpt_act8* keep,
                        const gockpt_matrix* grad_x, const gockpt_matrix* grad_weight, int accumulate,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- activation that keeps its inputs in 8 bits ------------------------------ */

#define GOCKPT_SILU 0      /* x / (1 + exp(-x)) */
#define GOCKPT_GELU 1      /* x (1 + erf(x / sqrt 2)) / 2 */
#define GOCKPT_GELU_TANH 2 /* x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2 */

/* out = round(act(x) * factor), or round(act(x)) where factor is NULL; all of
 * one type, any of the three.  Before it is rounded a 16-bit act(x) is off by up
 * to 2^-15 of itself, with GOCKPT_GELU_TANH 2^-14 (where it is at least 2^-126).  keep_x and keep_factor: where x and factor go in
 * 8 bits (both NULL: nowhere; keep_factor NULL without a factor).
 * Errors: EINVAL, EHIP. */
int gockpt_gate8(int kind, const gockpt_matrix* x, const gockpt_matrix* factor, const gockpt_matrix* out,
                 const gockpt_act8* keep_x, const gockpt_act8* keep_factor, void* stream);

/* With a and b for what keep_x and keep_factor stand for: grad_x =
 * round(grad_out * act'(a) * b), grad_factor = round(grad_out * act(a)); without
 * keep_factor, grad_x = round(grad_out * act'(a)) and grad_factor is NULL.
 * Either may be NULL; all of grad_out's type.  Errors: EINVAL, EHIP. */
int gockpt_gate8_grad(int kind, const gockpt_matrix* grad_out, const gockpt_act8* keep_x,
                      const gockpt_act8* keep_factor, const gockpt_matrix* grad_x, const gockpt_matrix* grad_factor,
                      void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GOCKPT_MODEL_H */
