// gockpt_linear8.hip -- the linear layer that keeps its input in 8 bits.
//
// The weight's gradient restores the input to its 16-bit type (which holds it
// exactly) in the workspace and multiplies that: 21 and 373 us for 16384 x 2048
// values by 8192 (395 among a training step's other products).  A product that took
// the codes themselves, widened between global memory and LDS, needed 673 us with the
// conversion before each tile's barrier and 539 with it between the matrix
// instructions: each of the 32 tiles along the outputs converts all codes again.
#include "gockpt_mma.h"
#include "gockpt_model_internal.h"

namespace gockpt {

namespace {

StoreArgs store_to(const gockpt_matrix& out, int accumulate) {
    StoreArgs o{};
    o.out = static_cast<uint8_t*>(const_cast<void*>(out.data));
    o.stride = (out.rows > 1 ? out.stride : out.cols) * dtype_bytes(out.dtype);
    o.dtype = out.dtype;
    o.accumulate = accumulate != 0;
    o.alpha = 1.0f;
    return o;
}

// The most slices whose fp32 sums are worth their memory.
constexpr int kMostSplits = 64;

int64_t slice_bytes(const ProductPlan& p, int64_t rn, int64_t cn) {
    return p.splits > 1 ? p.splits * rn * cn * 4 : 0;
}

// out = the product, in slices at `slices` that a second kernel joins, or at once.
void product_into(int kind, int dtype, const ProductPlan& p, MmaArgs& a, const gockpt_matrix& out, int accumulate,
                  uint8_t* slices, hipStream_t s) {
    StoreArgs o = store_to(out, accumulate);
    if (p.splits == 1) return launch_product(kind, dtype, p, a, o, s);
    o.slices = reinterpret_cast<float*>(slices);
    launch_product(kind, dtype, p, a, o, s);
    FinishArgs f{};
    f.slices = o.slices;
    f.slice_step = int64_t{a.rn} * a.cn;
    f.count = p.splits;
    f.rows = a.cn;
    f.cols = a.rn;
    f.out = o.out;
    f.stride = o.stride;
    f.dtype = o.dtype;
    f.accumulate = o.accumulate;
    f.alpha = 1.0f;
    launch_finish(f, s);
}

struct ForwardPlan {
    ProductPlan product;
    size_t x, weight, slices, bytes;
};

ForwardPlan plan_forward(const gockpt_matrix& x, const gockpt_matrix& w) {
    ForwardPlan p{};
    Parts parts;
    p.product = plan_product(kAlongAlong, w.rows, x.rows, x.cols, kMostSplits);
    p.x = parts.take(copy_bytes(x));
    p.weight = parts.take(copy_bytes(w));
    p.slices = parts.take(slice_bytes(p.product, w.rows, x.rows));
    p.bytes = parts.bytes;
    return p;
}

struct BackwardPlan {
    ProductPlan by_x, by_weight;
    size_t grad, weight, slices_x, input, slices_weight, bytes;
};

BackwardPlan plan_backward(const gockpt_matrix& g, const gockpt_matrix* w, const gockpt_act8* keep, bool by_x,
                           bool by_weight) {
    BackwardPlan p{};
    Parts parts;
    p.grad = parts.take(copy_bytes(g));
    if (by_x) {
        p.by_x = plan_product(kAcrossAlong, w->cols, g.rows, g.cols, kMostSplits);
        p.weight = parts.take(copy_bytes(*w));
        p.slices_x = parts.take(slice_bytes(p.by_x, w->cols, g.rows));
    }
    if (by_weight) {
        p.by_weight = plan_product(kAcrossAcross, keep->cols, g.cols, g.rows, kMostSplits);
        p.input = parts.take(g.rows * copy_stride(keep->cols) * 2);
        p.slices_weight = parts.take(slice_bytes(p.by_weight, keep->cols, g.cols));
    }
    p.bytes = parts.bytes;
    return p;
}

int check_forward(const char* name, const gockpt_matrix* x, const gockpt_matrix* w) {
    int rc = check_model_matrix(name, "x", x, kHalfTypes);
    if (rc == GOCKPT_OK) rc = check_model_matrix(name, "weight", w, kHalfTypes);
    if (rc != GOCKPT_OK) return rc;
    if (x->dtype != w->dtype)
        return ops_fail(GOCKPT_EINVAL, "%s: x of dtype %d, weight of %d", name, x->dtype, w->dtype);
    if (x->cols != w->cols)
        return ops_fail(GOCKPT_EINVAL, "%s: x of %lld columns, weight of %lld", name, static_cast<long long>(x->cols),
                        static_cast<long long>(w->cols));
    if (w->rows > kMaxWidth)
        return ops_fail(GOCKPT_EINVAL, "%s: weight of %lld rows", name, static_cast<long long>(w->rows));
    return GOCKPT_OK;
}

int check_blocks(const char* name, const ProductPlan& p) {
    if (too_many_blocks(p))
        return ops_fail(GOCKPT_EINVAL, "%s: a product of %u x %u tiles", name, p.tiles_r, p.tiles_c);
    return GOCKPT_OK;
}

int check_backward(const char* name, const gockpt_matrix* g, const gockpt_matrix* w, const gockpt_act8* keep,
                   const gockpt_matrix* gx, const gockpt_matrix* gw) {
    int rc = check_model_matrix(name, "grad_out", g, kHalfTypes);
    if (rc == GOCKPT_OK && gx != nullptr) {
        rc = check_model_matrix(name, "grad_x", gx, kAnyType);
        if (rc == GOCKPT_OK) rc = check_model_matrix(name, "weight", w, kHalfTypes);
        if (rc == GOCKPT_OK && w->dtype != g->dtype)
            rc = ops_fail(GOCKPT_EINVAL, "%s: grad_out of dtype %d, weight of %d", name, g->dtype, w->dtype);
        if (rc == GOCKPT_OK && (w->rows != g->cols || gx->rows != g->rows || gx->cols != w->cols))
            rc = ops_fail(GOCKPT_EINVAL, "%s: grad_out %lld x %lld, weight %lld x %lld, grad_x %lld x %lld", name,
                          static_cast<long long>(g->rows), static_cast<long long>(g->cols),
                          static_cast<long long>(w->rows), static_cast<long long>(w->cols),
                          static_cast<long long>(gx->rows), static_cast<long long>(gx->cols));
    }
    if (rc == GOCKPT_OK && gw != nullptr) {
        rc = check_model_matrix(name, "grad_weight", gw, kAnyType);
        if (rc == GOCKPT_OK) rc = check_act8(name, "keep", keep, g->rows, gw->cols);
        if (rc == GOCKPT_OK && gw->rows != g->cols)
            rc = ops_fail(GOCKPT_EINVAL, "%s: grad_out of %lld columns, grad_weight of %lld rows", name,
                          static_cast<long long>(g->cols), static_cast<long long>(gw->rows));
    }
    return rc;
}

}  // namespace

}  // namespace gockpt

using namespace gockpt;

extern "C" {

int gockpt_linear8_bytes(const gockpt_matrix* x, const gockpt_matrix* weight, size_t* bytes) {
    const char* name = "gockpt_linear8_bytes";
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *bytes = 0;
    int rc = check_forward(name, x, weight);
    if (rc != GOCKPT_OK) return rc;
    const ForwardPlan p = plan_forward(*x, *weight);
    rc = check_blocks(name, p.product);
    if (rc == GOCKPT_OK) *bytes = p.bytes;
    return rc;
}

int gockpt_linear8(const gockpt_matrix* x, const gockpt_matrix* weight, const gockpt_matrix* out,
                   const gockpt_act8* keep, void* workspace, size_t workspace_bytes, void* stream) {
    const char* name = "gockpt_linear8";
    int rc = check_forward(name, x, weight);
    if (rc == GOCKPT_OK) rc = check_model_matrix(name, "out", out, kAnyType);
    if (rc == GOCKPT_OK && (out->rows != x->rows || out->cols != weight->rows))
        rc = ops_fail(GOCKPT_EINVAL, "%s: out of %lld x %lld for %lld tokens and %lld outputs", name,
                      static_cast<long long>(out->rows), static_cast<long long>(out->cols),
                      static_cast<long long>(x->rows), static_cast<long long>(weight->rows));
    if (rc == GOCKPT_OK && keep != nullptr) rc = check_act8(name, "keep", keep, x->rows, x->cols);
    if (rc != GOCKPT_OK) return rc;
    const ForwardPlan p = plan_forward(*x, *weight);
    rc = check_blocks(name, p.product);
    if (rc == GOCKPT_OK) rc = check_workspace(name, workspace, workspace_bytes, p.bytes);
    if (rc != GOCKPT_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const bool needed = out->rows > 0 && out->cols > 0;
    const bool with_keep = keep != nullptr && needed && !in_place(*x);
    if (keep != nullptr) {
        rc = pack_and_copy(name, x, keep, with_keep ? ws + p.x : nullptr, s);
        if (rc != GOCKPT_OK) return rc;
    }
    if (!needed) return GOCKPT_OK;
    Copies copies;
    const Source sx = with_keep ? copied(*x, ws + p.x) : copies.source_of(*x, ws + p.x);
    const Source sw = copies.source_of(*weight, ws + p.weight);
    copies.launch(s);
    MmaArgs a{};
    a.r = sw.data;
    a.r_stride = sw.stride;
    a.c = sx.data;
    a.c_stride = sx.stride;
    a.rn = static_cast<int32_t>(weight->rows);
    a.cn = static_cast<int32_t>(x->rows);
    a.k = static_cast<int32_t>(x->cols);
    product_into(kAlongAlong, x->dtype, p.product, a, *out, 0, ws + p.slices, s);
    return ops_launched(name);
}

int gockpt_linear8_grad_bytes(const gockpt_matrix* grad_out, const gockpt_matrix* weight, const gockpt_act8* keep,
                              const gockpt_matrix* grad_x, const gockpt_matrix* grad_weight, size_t* bytes) {
    const char* name = "gockpt_linear8_grad_bytes";
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *bytes = 0;
    int rc = check_backward(name, grad_out, weight, keep, grad_x, grad_weight);
    if (rc != GOCKPT_OK) return rc;
    const BackwardPlan p = plan_backward(*grad_out, weight, keep, grad_x != nullptr, grad_weight != nullptr);
    rc = check_blocks(name, p.by_x);
    if (rc == GOCKPT_OK) rc = check_blocks(name, p.by_weight);
    if (rc == GOCKPT_OK) *bytes = p.bytes;
    return rc;
}

int gockpt_linear8_grad(const gockpt_matrix* grad_out, const gockpt_matrix* weight, const gockpt_act8* keep,
                        const gockpt_matrix* grad_x, const gockpt_matrix* grad_weight, int accumulate,
                        void* workspace, size_t workspace_bytes, void* stream) {
    const char* name = "gockpt_linear8_grad";
    int rc = check_backward(name, grad_out, weight, keep, grad_x, grad_weight);
    if (rc != GOCKPT_OK) return rc;
    const BackwardPlan p = plan_backward(*grad_out, weight, keep, grad_x != nullptr, grad_weight != nullptr);
    rc = check_blocks(name, p.by_x);
    if (rc == GOCKPT_OK) rc = check_blocks(name, p.by_weight);
    if (rc == GOCKPT_OK) rc = check_workspace(name, workspace, workspace_bytes, p.bytes);
    if (rc != GOCKPT_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const bool by_x = grad_x != nullptr && grad_x->rows > 0 && grad_x->cols > 0;
    const bool by_weight = grad_weight != nullptr && grad_weight->rows > 0 && grad_weight->cols > 0;
    if (!by_x && !by_weight) return GOCKPT_OK;
    Copies copies;
    const Source sg = copies.source_of(*grad_out, ws + p.grad);
    const Source sw = by_x ? copies.source_of(*weight, ws + p.weight) : Source{};
    copies.launch(s);
    if (by_x) {
        MmaArgs a{};
        a.r = sw.data;
        a.r_stride = sw.stride;
        a.c = sg.data;
        a.c_stride = sg.stride;
        a.rn = static_cast<int32_t>(weight->cols);
        a.cn = static_cast<int32_t>(grad_out->rows);
        a.k = static_cast<int32_t>(grad_out->cols);
        product_into(kAcrossAlong, grad_out->dtype, p.by_x, a, *grad_x, 0, ws + p.slices_x, s);
    }
    if (by_weight) {
        const gockpt_matrix input{ws + p.input, keep->rows, keep->cols, copy_stride(keep->cols), grad_out->dtype, 0};
        rc = gockpt_act8_unpack(keep, &input, stream);
        if (rc != GOCKPT_OK) return rc;
        MmaArgs a{};
        a.r = ws + p.input;
        a.r_stride = input.stride * 2;
        a.c = sg.data;
        a.c_stride = sg.stride;
        a.rn = static_cast<int32_t>(keep->cols);
        a.cn = static_cast<int32_t>(grad_out->cols);
        a.k = static_cast<int32_t>(grad_out->rows);
        product_into(kAcrossAcross, grad_out->dtype, p.by_weight, a, *grad_weight, accumulate, ws + p.slices_weight, s);
    }
    return ops_launched(name);
}

}  // extern "C"
