/* The operators from plain C: an embedding's gradient written into a flat
 * bf16 buffer, and the norm and clip over it and an fp32 tensor, against sums
 * made on the host in double.  Only gockpt_ops.h and the HIP runtime. */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "gockpt_ops.h"

#define ROWS 60
#define COLS 24
#define TOKENS 200
#define OTHER 5001

#define CHECK(x)                                                                              \
    do {                                                                                      \
        int rc_ = (int)(x);                                                                   \
        if (rc_ != 0) {                                                                       \
            fprintf(stderr, "%s: %d (%s)\n", #x, rc_, gockpt_last_error(NULL));               \
            return 1;                                                                         \
        }                                                                                     \
    } while (0)

static float value(int i) { return (float)((i * 37) % 101 - 50) / 64.0f; } /* exact in bf16 */

static uint16_t to_bf16(float f) {
    uint32_t u;
    memcpy(&u, &f, 4);
    u += 0x7FFFu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}

static double from_bf16(uint16_t b) {
    uint32_t u = (uint32_t)b << 16;
    float f;
    memcpy(&f, &u, 4);
    return f;
}

int main(void) {
    static float grad_out[TOKENS * COLS], other[OTHER];
    static double table[ROWS * COLS];
    static int32_t ids[TOKENS];
    static uint16_t flat[ROWS * COLS + OTHER];
    void *d_grad, *d_ids, *d_other, *d_flat, *d_ws, *d_list, *d_result;
    size_t ws_bytes, list_bytes;
    gockpt_grads* list;
    gockpt_grad_result r;
    hipStream_t s;
    double sum = 0.0, norm, max_norm = 3.0;
    int i, c;

    for (i = 0; i < TOKENS; ++i) ids[i] = i % 9 == 0 ? -1 : (i * i) % 41 + 5;
    for (i = 0; i < TOKENS * COLS; ++i) grad_out[i] = value(i);
    for (i = 0; i < OTHER; ++i) other[i] = value(i + 7) * 1.001f;
    for (i = 0; i < TOKENS; ++i)
        for (c = 0; c < COLS; ++c)
            if (ids[i] >= 0) table[ids[i] * COLS + c] += 0.5 * grad_out[i * COLS + c];
    /* multiples of 1/128 well within fp32: the sums are exact, the bf16 rounding known */
    for (i = 0; i < ROWS * COLS; ++i) {
        table[i] = from_bf16(to_bf16((float)table[i]));
        sum += table[i] * table[i];
    }
    for (i = 0; i < OTHER; ++i) sum += (double)other[i] * other[i];
    norm = sqrt(sum);

    CHECK(hipStreamCreate(&s));
    CHECK(gockpt_embedding_grad_bytes(TOKENS, ROWS, COLS, &ws_bytes));
    CHECK(hipMalloc(&d_grad, sizeof grad_out));
    CHECK(hipMalloc(&d_ids, sizeof ids));
    CHECK(hipMalloc(&d_other, sizeof other));
    CHECK(hipMalloc(&d_flat, sizeof flat));
    CHECK(hipMalloc(&d_ws, ws_bytes + 256));
    CHECK(hipMalloc(&d_result, sizeof r));
    CHECK(hipMemcpy(d_grad, grad_out, sizeof grad_out, hipMemcpyHostToDevice));
    CHECK(hipMemcpy(d_ids, ids, sizeof ids, hipMemcpyHostToDevice));
    CHECK(hipMemcpy(d_other, other, sizeof other, hipMemcpyHostToDevice));
    {
        gockpt_matrix grad = {d_grad, TOKENS, COLS, COLS, GOCKPT_FP32, 0};
        gockpt_matrix into = {d_flat, ROWS, COLS, COLS, GOCKPT_BF16, 0};
        gockpt_token_ids tokens = {d_ids, 1, TOKENS, TOKENS, 0, 32, 0};
        gockpt_grad_tensor tensors[2] = {
            {d_flat, NULL, 1, ROWS * COLS, ROWS * COLS, GOCKPT_BF16, 0},
            {d_other, (uint16_t*)d_flat + ROWS * COLS, 1, OTHER, OTHER, GOCKPT_FP32, GOCKPT_BF16}};
        CHECK(gockpt_embedding_grad(&grad, &tokens, INT64_MIN, 0.5f, 0, &into, d_ws, ws_bytes, s));
        CHECK(gockpt_grads_bytes(tensors, 2, &list_bytes));
        CHECK(hipMalloc(&d_list, list_bytes));
        CHECK(gockpt_grads_create(tensors, 2, d_list, list_bytes, s, &list));
        CHECK(gockpt_grads_clip(list, NULL, max_norm, (gockpt_grad_result*)d_result, s));
        if (gockpt_grads_clip(list, NULL, -1.0, (gockpt_grad_result*)d_result, s) != GOCKPT_EINVAL) return 2;
        tokens.bits = 8;
        if (gockpt_embedding(&into, &tokens, 1.0f, &grad, s) != GOCKPT_EINVAL) return 2;
    }
    CHECK(hipStreamSynchronize(s));
    CHECK(hipMemcpy(&r, d_result, sizeof r, hipMemcpyDeviceToHost));
    CHECK(hipMemcpy(flat, d_flat, sizeof flat, hipMemcpyDeviceToHost));
    CHECK(gockpt_grads_destroy(list));
    if (fabs(r.norm - norm) > 2e-6 * norm || r.found_inf != 0.0f) {
        fprintf(stderr, "norm %g, expected %g\n", r.norm, norm);
        return 3;
    }
    for (i = 0; i < ROWS * COLS + OTHER; ++i) {
        const float x = i < ROWS * COLS ? (float)table[i] : other[i - ROWS * COLS];
        if (flat[i] != to_bf16(x * r.coef) && x != 0.0f) {
            fprintf(stderr, "element %d: %x, expected %x\n", i, flat[i], to_bf16(x * r.coef));
            return 4;
        }
    }
    printf("ok norm %.6f coef %.6f\n", r.norm, r.coef);
    return 0;
}
