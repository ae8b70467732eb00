/*
 * gockpt_ops.h -- operators around the optimizer step of gockpt.h: the norm of
 * a list of gradient tensors, clipping, the embedding lookup and its gradient.
 *
 * A backward pass ends with the embedding's gradient, a table whose rows are
 * sums over the tokens that looked them up; the training loop then takes the
 * norm of all gradients, scales them down where it is too large, and calls
 * gockpt_step on the flat 16-bit gradient buffer.  These calls do that: the
 * embedding's gradient is written straight into its part of the flat buffer,
 * and clipping scales the other tensors in place or rounds them (fp32 sums
 * over micro-batches, say) into theirs.  The norm's found_inf is what
 * gockpt_config.found_inf takes, and gockpt_scale_ptr gives the loss scale
 * that the norm divides by, so nothing here waits for the device.
 *
 * Conventions are those of gockpt.h: int status, the text of a failing call
 * from gockpt_last_error(NULL) on the calling thread, caller-owned buffers, no
 * C++ exception crosses.  Every call but gockpt_grads_create is asynchronous
 * on `stream` (a hipStream_t, NULL: the null stream), launches kernels only
 * and may be captured in a HIP graph.  The same inputs in the same layout give
 * the same bits on every call: no sum depends on the order in which blocks run.
 */
#ifndef GOCKPT_OPS_H
#define GOCKPT_OPS_H

#include "gockpt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define GOCKPT_BF16 0
#define GOCKPT_FP16 1
#define GOCKPT_FP32 2

/* ---- norm and clipping of many gradient tensors --------------------------- */

/* One gradient tensor: rows x cols elements, row r at data + r * stride
 * elements (a vector has one row).  dst: where clipping writes the rows one
 * after another, rounded to dst_dtype, or NULL: in place (dst_dtype is then
 * ignored).  Pointers are aligned to their element.  A dst must overlap no
 * other tensor of the list, and its own data only where both are the same
 * contiguous memory and type, which is the same as NULL. */
typedef struct {
    const void* data;  /* device */
    void* dst;         /* device, nullable */
    int64_t rows, cols, stride;  /* rows, cols >= 0; stride >= cols if rows > 1 */
    int32_t dtype, dst_dtype;    /* GOCKPT_BF16, GOCKPT_FP16 or GOCKPT_FP32 */
} gockpt_grad_tensor;

/* What a norm leaves on the device (32 bytes, 8-byte aligned). */
typedef struct {
    double sumsq;     /* sum of squares of the elements as stored */
    float norm;       /* sqrt(sumsq) / scale */
    float found_inf;  /* 1 when some element is inf or NaN, or times coef is rounded to inf in its dst, else 0 */
    float coef;       /* min(1, max_norm / (norm + 1e-6)); 1 when some element is inf or NaN */
    /* [0]: largest magnitude of the elements that go to fp16 from a wider type and
     * are, unscaled, too large for it, [1]: of such that go to bf16 (0: none); [2]: 0 */
    float reserved_[3];
} gockpt_grad_result;

typedef struct gockpt_grads gockpt_grads;

/* Device workspace bytes of a list.  Host only.  Errors: EINVAL. */
int gockpt_grads_bytes(const gockpt_grad_tensor* tensors, int64_t count, size_t* bytes);

/* A handle over `count` tensors (0 is allowed: norm 0).  Writes the list's
 * table into the workspace (256-byte aligned, kept by the caller as long as
 * the handle) on `stream` and waits for it.  The handle holds the tensors'
 * addresses, never their contents.  Errors: EINVAL (types, sizes, alignment),
 * ENOMEM (workspace too small), EHIP. */
int gockpt_grads_create(const gockpt_grad_tensor* tensors, int64_t count, void* workspace,
                        size_t workspace_bytes, void* stream, gockpt_grads** out);

/* Releases the handle (host memory only; work it queued may still run).
 * Accepts NULL. */
int gockpt_grads_destroy(gockpt_grads* list);

/* The norm over all tensors of the list into *result (device).  scale: device
 * float, the loss scale the gradients carry (NULL: 1).  max_norm >= 0, for
 * coef (INFINITY: coef is 1).  Squares are summed in fp32 over at most 32
 * elements and in fp64 beyond; a group whose fp32 sum leaves [2^-100, 2^126)
 * is summed again in fp64, so no finite gradients overflow or vanish.  The
 * calls of one list use its workspace: one at a time, in stream order (calls
 * that overlap all the same end, with results of no meaning).
 * Errors: EINVAL, EHIP. */
int gockpt_grads_norm(gockpt_grads* list, const float* scale, double max_norm,
                      gockpt_grad_result* result, void* stream);

/* dst = round(element * result->coef) for every element, one fp32 product
 * rounded once to the destination's type, to nearest even; beyond that type's
 * range: infinity, which the found_inf of this list's norm tells.  In place, a
 * coefficient of 1 leaves the memory untouched.  Errors: EINVAL, EHIP. */
int gockpt_grads_scale(gockpt_grads* list, const gockpt_grad_result* result, void* stream);

/* gockpt_grads_norm, then gockpt_grads_scale by its coef.  Gradients with an
 * inf or NaN are written unscaled (the step skips them by found_inf). */
int gockpt_grads_clip(gockpt_grads* list, const float* scale, double max_norm,
                      gockpt_grad_result* result, void* stream);

/* norm, found_inf and coef again from result->sumsq and reserved_, as a norm
 * left them: for ranks that hold different parameters, have added up their
 * sumsq and, where a dst is narrower than its data, taken the maximum of each
 * of reserved_[0] and [1].  Errors: EINVAL, EHIP. */
int gockpt_grads_result(gockpt_grad_result* result, const float* scale, double max_norm, void* stream);

/* Device address of the context's loss scale (the one the next gockpt_step
 * divides by; written on its compute stream).  Errors: EINVAL. */
int gockpt_scale_ptr(const gockpt_ctx* ctx, const float** out);

/* ---- embedding ------------------------------------------------------------ */

/* The tokens: batch x length ids, token b * length + l at ids[b * stride + l]
 * (device, 32 or 64 bits).  An id in [first_id, first_id + rows) stands for
 * row id - first_id of the table; any other is masked: its output is zero and
 * it adds to no gradient (padding marked by -1, and the ids of other ranks
 * where each holds a range of the vocabulary). */
typedef struct {
    const void* ids;
    int64_t batch, length, stride;  /* batch * length < 2^31; stride >= length if batch > 1 */
    int64_t first_id;
    int32_t bits, reserved_;
} gockpt_token_ids;

/* A matrix: rows x cols of dtype, row r at data + r * stride elements. */
typedef struct {
    const void* data;
    int64_t rows, cols, stride;  /* stride >= cols if rows > 1 */
    int32_t dtype, reserved_;
} gockpt_matrix;

/* out row t = round(scale * table row of token t), one fp32 product rounded
 * once to nearest even; zeros where the token is masked.  out has batch *
 * length rows and the table's columns.  Errors: EINVAL, EHIP. */
int gockpt_embedding(const gockpt_matrix* table, const gockpt_token_ids* tokens, float scale,
                     const gockpt_matrix* out, void* stream);

/* Workspace bytes of gockpt_embedding_grad for these shapes (0 for few
 * tokens).  Host only.  Errors: EINVAL. */
int gockpt_embedding_grad_bytes(int64_t tokens, int64_t rows, int64_t cols, size_t* bytes);

/* The table's gradient: row v = round(scale * sum of grad_out rows of the
 * tokens with id first_id + v).  accumulate = 0 writes every row (zeros where
 * no token has it); 1 adds to what the row holds, round(old + scale * sum), and
 * touches only rows that some token has (a head that shares the table has
 * written its gradient there).  Tokens with padding_id add nothing (INT64_MIN:
 * none).  Sums are fp32, in token order over chunks of at most 128 tokens, those
 * sums then in order; no atomics.  grad_out has batch * length rows, the table
 * at most 4194304.  workspace: 256-byte aligned, gockpt_embedding_grad_bytes; in
 * use until the call's kernels have run.  Errors: EINVAL, ENOMEM (workspace),
 * EHIP. */
int gockpt_embedding_grad(const gockpt_matrix* grad_out, const gockpt_token_ids* tokens, int64_t padding_id,
                          float scale, int accumulate, const gockpt_matrix* grad_table, void* workspace,
                          size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GOCKPT_OPS_H */
