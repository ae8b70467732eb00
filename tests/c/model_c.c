/* The model's operators from plain C: loss and gradients of a head, a linear
 * layer that keeps its input in 8 bits and an activation behind it, against sums
 * made on the host in double.  Only gockpt_model.h and the HIP runtime. */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "gockpt_model.h"

#define TOKENS 40
#define COLS 24
#define CLASSES 50
#define BLOCKS 1 /* of 32 columns */

#define CHECK(x)                                                                              \
    do {                                                                                      \
        int rc_ = (int)(x);                                                                   \
        if (rc_ != 0) {                                                                       \
            fprintf(stderr, "%s: %d (%s)\n", #x, rc_, gockpt_last_error(NULL));               \
            return 1;                                                                         \
        }                                                                                     \
    } while (0)

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

/* multiples of 1/64 up to 127/64: exact in bf16, and in 8 bits (a block's largest is made 127/64) */
static double value(int i) { return ((i * 37) % 255 - 127) / 64.0; }

static void* upload(const void* from, size_t n) {
    void* p = NULL;
    if (hipMalloc(&p, n) != hipSuccess || hipMemcpy(p, from, n, hipMemcpyHostToDevice) != hipSuccess) exit(9);
    return p;
}

int main(void) {
    static uint16_t x16[TOKENS * COLS], w16[CLASSES * COLS], y16[TOKENS * CLASSES], dx16[TOKENS * COLS];
    static float dw[CLASSES * COLS], gate[TOKENS * COLS];
    static double x[TOKENS * COLS], w[CLASSES * COLS], z[TOKENS * CLASSES];
    static int32_t ids[TOKENS];
    void *d_x, *d_w, *d_ids, *d_y, *d_dx, *d_dw, *d_loss, *d_lse, *d_codes, *d_scales, *d_ws, *d_one, *d_gate;
    size_t loss_bytes, grad_bytes, linear_bytes, most;
    double loss = 0.0, got_loss, err, worst = 0.0;
    float got, one = 1.0f;
    int t, v, c, kept = 0;
    hipStream_t s;

    for (t = 0; t < TOKENS; ++t) {
        for (c = 0; c < COLS; ++c) x[t * COLS + c] = c == 0 ? 127.0 / 64.0 : value(t * 31 + c);
        ids[t] = t % 7 == 0 ? -1 : (t * t) % CLASSES;
    }
    for (v = 0; v < CLASSES * COLS; ++v) w[v] = value(v + 5) / 4.0;
    for (t = 0; t < TOKENS * COLS; ++t) x16[t] = to_bf16((float)x[t]);
    for (v = 0; v < CLASSES * COLS; ++v) w16[v] = to_bf16((float)w[v]);
    for (t = 0; t < TOKENS; ++t) {
        double sum = 0.0, l[CLASSES];
        for (v = 0; v < CLASSES; ++v) {
            l[v] = 0.0;
            for (c = 0; c < COLS; ++c) l[v] += 0.25 * x[t * COLS + c] * w[v * COLS + c];
            sum += exp(l[v]);
        }
        for (v = 0; v < CLASSES; ++v) z[t * CLASSES + v] = ids[t] < 0 ? 0.0 : exp(l[v]) / sum - (v == ids[t]);
        if (ids[t] >= 0) {
            loss += log(sum) - l[ids[t]];
            ++kept;
        }
    }

    CHECK(hipStreamCreate(&s));
    d_x = upload(x16, sizeof x16);
    d_w = upload(w16, sizeof w16);
    d_ids = upload(ids, sizeof ids);
    d_y = upload(y16, sizeof y16);
    d_dx = upload(dx16, sizeof dx16);
    d_dw = upload(dw, sizeof dw);
    d_one = upload(&one, sizeof one);
    d_gate = upload(gate, sizeof gate);
    CHECK(hipMalloc(&d_loss, 4));
    CHECK(hipMalloc(&d_lse, TOKENS * 4));
    CHECK(hipMalloc(&d_codes, TOKENS * BLOCKS * GOCKPT_ACT8_BLOCK));
    CHECK(hipMalloc(&d_scales, TOKENS * BLOCKS));
    {
        gockpt_matrix mx = {d_x, TOKENS, COLS, COLS, GOCKPT_BF16, 0}, mw = {d_w, CLASSES, COLS, COLS, GOCKPT_BF16, 0};
        gockpt_matrix my = {d_y, TOKENS, CLASSES, CLASSES, GOCKPT_BF16, 0};
        gockpt_matrix mdx = {d_dx, TOKENS, COLS, COLS, GOCKPT_BF16, 0};
        gockpt_matrix mdw = {d_dw, CLASSES, COLS, COLS, GOCKPT_FP32, 0};
        gockpt_matrix mg = {d_gate, TOKENS, COLS, COLS, GOCKPT_FP32, 0};
        gockpt_act8 keep = {d_codes, d_scales, TOKENS, COLS};
        gockpt_head head;
        memset(&head, 0, sizeof head);
        head.hidden = mx;
        head.table = mw;
        head.targets.ids = d_ids;
        head.targets.batch = 1;
        head.targets.length = head.targets.stride = TOKENS;
        head.targets.bits = 32;
        head.ignore_id = INT64_MIN;
        head.scale = 0.25f;
        CHECK(gockpt_head_loss_bytes(&head, &loss_bytes));
        CHECK(gockpt_head_grad_bytes(&head, &mdx, &mdw, &grad_bytes));
        CHECK(gockpt_linear8_bytes(&mx, &mw, &linear_bytes));
        most = loss_bytes > grad_bytes ? loss_bytes : grad_bytes;
        if (linear_bytes > most) most = linear_bytes;
        CHECK(hipMalloc(&d_ws, most));
        CHECK(gockpt_head_loss(&head, GOCKPT_MEAN, (float*)d_loss, (float*)d_lse, NULL, d_ws, most, s));
        CHECK(gockpt_head_grad(&head, (const float*)d_lse, GOCKPT_MEAN, (const float*)d_one, &mdx, &mdw, 0, d_ws, most, s));
        CHECK(gockpt_linear8(&mx, &mw, &my, &keep, d_ws, most, s));
        CHECK(gockpt_act8_unpack(&keep, &mg, s));
        if (gockpt_head_loss(&head, 9, (float*)d_loss, NULL, NULL, d_ws, most, s) != GOCKPT_EINVAL) return 2;
        if (gockpt_linear8(&mx, &mw, &mdw, NULL, d_ws, most, s) != GOCKPT_EINVAL) return 2;
    }
    CHECK(hipStreamSynchronize(s));
    CHECK(hipMemcpy(&got, d_loss, 4, hipMemcpyDeviceToHost));
    CHECK(hipMemcpy(dx16, d_dx, sizeof dx16, hipMemcpyDeviceToHost));
    CHECK(hipMemcpy(dw, d_dw, sizeof dw, hipMemcpyDeviceToHost));
    CHECK(hipMemcpy(y16, d_y, sizeof y16, hipMemcpyDeviceToHost));
    CHECK(hipMemcpy(gate, d_gate, sizeof gate, hipMemcpyDeviceToHost));
    got_loss = got;
    if (fabs(got_loss - loss / kept) > 1e-5 * loss / kept) {
        fprintf(stderr, "loss %g, expected %g\n", got_loss, loss / kept);
        return 3;
    }
    for (t = 0; t < TOKENS; ++t) /* z rounded to bf16, half a step of 2^-8, over sums of |z w|, |z x| */
        for (c = 0; c < COLS; ++c) {
            double want = 0.0, size = 0.0;
            for (v = 0; v < CLASSES; ++v) {
                want += 0.25 / kept * z[t * CLASSES + v] * w[v * COLS + c];
                size += 0.25 / kept * fabs(z[t * CLASSES + v] * w[v * COLS + c]);
            }
            err = fabs(from_bf16(dx16[t * COLS + c]) - want);
            if (err > (size + fabs(want)) / 256.0 + 1e-7) return 4;
            if (gate[t * COLS + c] != (float)x[t * COLS + c]) return 5; /* 8 bits hold these */
        }
    for (v = 0; v < CLASSES; ++v)
        for (c = 0; c < COLS; ++c) {
            double want = 0.0, size = 0.0;
            for (t = 0; t < TOKENS; ++t) {
                want += 0.25 / kept * z[t * CLASSES + v] * x[t * COLS + c];
                size += 0.25 / kept * fabs(z[t * CLASSES + v] * x[t * COLS + c]);
            }
            err = fabs(dw[v * COLS + c] - want);
            if (err > size / 256.0 + 1e-7) return 6;
            if (err > worst) worst = err;
        }
    for (t = 0; t < TOKENS; ++t)
        for (v = 0; v < CLASSES; ++v) {
            double want = 0.0;
            for (c = 0; c < COLS; ++c) want += x[t * COLS + c] * w[v * COLS + c];
            /* products of multiples of 1/64 and 1/256, small sums: exact in fp32 */
            if (y16[t * CLASSES + v] != to_bf16((float)want) && want != 0.0) return 7;
        }
    printf("ok loss %.6f, table's gradient within %.3g\n", got_loss, worst);
    return 0;
}
