// gockpt_products.hip -- the matrix products of the head's gradients and the
// linear layers: which tile and how many slices of k, the launches, the join of
// slices, and copies of matrices that products cannot read in place.
#include "gockpt_mma.h"
#include "gockpt_model_internal.h"

namespace gockpt {

namespace {

template <class M>
__global__ __launch_bounds__(M::kThreads) void product_kernel(MmaArgs a, StoreArgs o) {
    GOCKPT_MMA_LDS(M)
    const int cn = a.cn_dev != nullptr ? *a.cn_dev : a.cn;
    MmaPlace p;
    if (!mma_place(a, cn, M::kBR, M::kBC, p)) return;
    const int k = a.k_dev != nullptr ? *a.k_dev : a.k;
    typename M::Acc acc;
    GOCKPT_MMA_RUN(M, a, p, cn, k, acc);
    if constexpr (M::kFixes)
        if ((M::kBothAcross ? o.seen : o.owner) != nullptr && p.split == 0) add_fixes<M>(a, o, p, cn, k, acc);
    M::sync();
    store_tile<M>(GOCKPT_MMA_STORE(M), a, o, p, cn, acc);
}

template <class M, int kShape>
void start(const MmaArgs& a, const StoreArgs& o, hipStream_t s) {
    static_assert(M::kThreads == product_threads(kShape), "what too_many_blocks counts");
    hipLaunchKernelGGL(product_kernel<M>, dim3(a.tiles_r * a.tiles_c * a.splits), dim3(M::kThreads), 0, s, a, o);
}

template <int kT, int kR, int kC>
void start_shape(int shape, const MmaArgs& a, const StoreArgs& o, hipStream_t s) {
    if (shape == kWide) return start<Mma<kT, kR, kC, 256, 256, 2, 4>, kWide>(a, o, s);
    if (shape == kMid) return start<Mma<kT, kR, kC, 128, 128, 2, 2>, kMid>(a, o, s);
    if constexpr (kR == kAlongK)
        start<Stream<kT>, kThin>(a, o, s);
    else if constexpr (kC == kAlongK)
        start<Mma<kT, kR, kC, 128, 32, 4, 1>, kThin>(a, o, s);
}

template <int kT>
void start_kind(int kind, int shape, const MmaArgs& a, const StoreArgs& o, hipStream_t s) {
    if (kind == kAlongAlong) return start_shape<kT, kAlongK, kAlongK>(shape, a, o, s);
    if (kind == kAcrossAlong) return start_shape<kT, kAcrossK, kAlongK>(shape, a, o, s);
    start_shape<kT, kAcrossK, kAcrossK>(shape, a, o, s);
}

// ---- the join of slices ---------------------------------------------------------

__global__ __launch_bounds__(256) void finish_kernel(FinishArgs f) {
    const int64_t groups = (f.cols + 3) / 4, all = groups * f.rows;
    const float alpha = f.alpha * (f.beta != nullptr ? *f.beta : 1.0f);
    for (int64_t at = blockIdx.x * int64_t{256} + threadIdx.x; at < all; at += gridDim.x * int64_t{256}) {
        const int64_t row = at / groups;
        const int col = static_cast<int>(at - row * groups) * 4, n = min(4, f.cols - col);
        const int64_t c = f.of_row != nullptr ? f.of_row[row] : row;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c >= 0) {
            const float* p = f.slices + c * f.cols + col;
            for (int k = 0; k < f.count; ++k, p += f.slice_step) {
                if (n == 4) {
                    sum += *reinterpret_cast<const f32x4_any*>(p);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (i < n) sum[i] += p[i];
                }
            }
            if (f.fix != nullptr && f.fix_row[c] >= 0) {
                const float x = f.fix[c];
                const u32x2 w =
                    *reinterpret_cast<const u32x2*>(f.fix_from + f.fix_row[c] * f.fix_stride + int64_t{col} * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t b = w[i / 2] >> (16 * (i & 1)) & 0xffff;
                    sum[i] += x * (f.fix_dtype == kBF16 ? elem_to_f32<kBF16>(b) : elem_to_f32<kFP16>(b));
                }
            }
            sum *= f.up != nullptr ? alpha / f.up[c] : alpha;
        }
        store4(f.out + row * f.stride + static_cast<int64_t>(col) * dtype_bytes(f.dtype), f.dtype, f.accumulate != 0,
               sum, n);
    }
}

// ---- copies ---------------------------------------------------------------------

// 8 columns a thread: rows that start anywhere become rows of whole 16-byte
// pieces, copy_stride apart.  An index past the source's columns is never read.
// The first blocks have the first matrix.
__global__ __launch_bounds__(256) void rows_kernel(Copies c) {
    const bool second = blockIdx.x >= c.one[0].blocks;
    const Copies::One& a = c.one[second];
    const uint32_t block = blockIdx.x - (second ? c.one[0].blocks : 0);
    const int64_t groups = (a.cols + 7) / 8;
    const int64_t all = groups * (a.count != nullptr ? *a.count : a.n);
    for (int64_t at = block * int64_t{256} + threadIdx.x; at < all; at += a.blocks * int64_t{256}) {
        const int64_t row = at / groups;
        const int col = static_cast<int>(at - row * groups) * 8;
        const int64_t from = a.rows != nullptr ? a.rows[row] : row;
        const uint8_t* p = a.src + from * a.stride + static_cast<int64_t>(col) * 2;
        *reinterpret_cast<u32x4*>(a.dst + row * a.dst_stride + col * 2) = load8(p, a.cols - col);
    }
}

uint32_t copy_grid(int64_t items) {
    return static_cast<uint32_t>(std::min<int64_t>((items + 255) / 256, kUnits * 16));
}

}  // namespace

void launch_finish(const FinishArgs& f, hipStream_t s) {
    const int64_t items = (int64_t{f.cols} + 3) / 4 * f.rows;
    if (items > 0) hipLaunchKernelGGL(finish_kernel, dim3(copy_grid(items)), dim3(256), 0, s, f);
}

Source Copies::rows_of(const gockpt_matrix& src, const int32_t* rows, const int32_t* count, int64_t n, uint8_t* dst) {
    const int64_t items = (src.cols + 7) / 8 * n;
    const Source to = copied(src, dst);
    if (items > 0)
        one[many++] = {static_cast<const uint8_t*>(src.data), src.stride * 2, to.stride, rows, count, dst,
                       static_cast<int32_t>(src.cols), static_cast<int32_t>(n), copy_grid(items)};
    return to;
}

void Copies::launch(hipStream_t s) const {
    if (many > 0) hipLaunchKernelGGL(rows_kernel, dim3(one[0].blocks + one[1].blocks), dim3(256), 0, s, *this);
}

namespace {

// Microseconds of so many blocks that take k each.  They run in rounds of as many
// as fit the device; a tile's time has a fixed part (its first copies, its stores)
// and a part for each k, which is less where a unit has one block instead of two,
// or the last round leaves units idle and the others their clock.  Measured, 20 ms
// apart (wide, mid): 8192 x 8192 x 8192 (r x c x k, both along k) 746, 960; 8192 x 16384
// x 2048 406, 515; 4096 x 2048 x 4096 83, 66; 4096 x 1024 x 4096 76, 47; 256 x 128 x
// 4096 68, 32; 3088 x 3000 x 1160 36, 48; 2048 x 8192 x 16384 (across) 373, 475; 1160 x
// 3088 x 3000 (across) 59, 37.  Streamed, 32000 x 1 x 4096: 46.
double blocks_us(int shape, bool streamed, int64_t blocks, double k) {
    const auto over = [](int64_t n, int64_t slots) { return static_cast<double>(n) / static_cast<double>(slots); };
    if (shape == kWide) {
        const int64_t rounds = blocks / kUnits, rest = blocks % kUnits;
        return static_cast<double>(rounds) * (4.5 + 0.0222 * k) +
               (rest > 0 ? 4.0 + (0.0165 + 0.0057 * over(rest, kUnits)) * k : 0.0);
    }
    if (shape == kMid) {
        const int64_t rounds = blocks / (2 * kUnits), rest = blocks % (2 * kUnits);
        return static_cast<double>(rounds) * (4.0 + 0.0166 * k) +
               (rest > kUnits ? 4.0 + 0.0166 * k : rest > 0 ? 3.0 + (0.0075 + 0.003 * over(rest, kUnits)) * k : 0.0);
    }
    const double rounds = static_cast<double>((blocks + 4 * kUnits - 1) / (4 * kUnits));
    return rounds * (streamed ? 2.0 + 0.003 * k : 3.0 + 0.012 * k);
}

}  // namespace

ProductPlan plan_product(int kind, int64_t rn, int64_t cn, int64_t k, int most_splits) {
    const bool along = kind == kAlongAlong || kind == kAcrossAlong;
    const double least = 2.0 * static_cast<double>(rn + cn) * static_cast<double>(k) / 5.5e6;  // to read both
    ProductPlan best{};
    best.us = -1.0;
    for (int shape = kWide; shape <= kThin; ++shape) {
        if ((shape == kThin) != (along && cn <= 32)) continue;  // few c: memory's time, which wider tiles do not reach
        const bool streamed = shape == kThin && kind == kAlongAlong;
        const int64_t br = shape == kWide ? 256 : streamed ? 32 : 128, bc = shape == kWide ? 256 : shape == kMid ? 128 : 32;
        const int64_t tr = (rn + br - 1) / br, tc = (cn + bc - 1) / bc, tiles = tr * tc;
        const int64_t slots = int64_t{kUnits} * (shape == kWide ? 1 : shape == kMid ? 2 : 4);
        for (int want = 1; want <= most_splits; want *= 2) {
            // a power of two, and as many as fill the slots
            for (int fill = 0; fill < (want > 1 ? 2 : 1); ++fill) {
                int64_t splits = want;
                if (fill == 1)
                    splits = std::min<int64_t>(most_splits, std::max<int64_t>(1, slots / std::max<int64_t>(1, tiles)));
                const int64_t split_k = std::max<int64_t>(64, up((k + splits - 1) / splits, 64));
                splits = std::max<int64_t>(1, (k + split_k - 1) / split_k);
                double us = std::max(
                    blocks_us(shape, streamed, tiles * splits, static_cast<double>(std::min(split_k, k))), least);
                if (splits > 1)  // the slices' sums, written and read
                    us += 4.0 + 8.0 * static_cast<double>(splits) * static_cast<double>(rn) * static_cast<double>(cn) / 4.5e6;
                if (best.us < 0.0 || us < best.us) {
                    best.shape = shape;
                    best.splits = static_cast<int>(splits);
                    best.split_k = static_cast<int32_t>(split_k);
                    best.tiles_r = static_cast<uint32_t>(tr);
                    best.tiles_c = static_cast<uint32_t>(tc);
                    best.us = us;
                }
            }
        }
    }
    return best;
}

void launch_product(int kind, int dtype, const ProductPlan& p, MmaArgs& a, const StoreArgs& o, hipStream_t s) {
    a.tiles_r = p.tiles_r;
    a.tiles_c = p.tiles_c;
    a.splits = p.splits;
    a.split_k = p.split_k;
    if (a.tiles_r == 0 || a.tiles_c == 0) return;
    if (dtype == kBF16)
        start_kind<kBF16>(kind, p.shape, a, o, s);
    else
        start_kind<kFP16>(kind, p.shape, a, o, s);
}

// ---- checks -----------------------------------------------------------------------

int check_model_matrix(const char* name, const char* what, const gockpt_matrix* m, int types) {
    if (m == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null %s", name, what);
    if (!dtype_ok(m->dtype) || (types >> m->dtype & 1) == 0)
        return ops_fail(GOCKPT_EINVAL, "%s: %s dtype %d", name, what, m->dtype);
    if (m->rows < 0 || m->cols < 0 || m->rows > kMaxExtent || m->cols > kMaxWidth)
        return ops_fail(GOCKPT_EINVAL, "%s: %s of %lld x %lld", name, what, static_cast<long long>(m->rows),
                        static_cast<long long>(m->cols));
    if (m->rows > 1 && (m->stride < m->cols || m->stride > (int64_t{1} << 46) / m->rows))
        return ops_fail(GOCKPT_EINVAL, "%s: %s stride %lld for rows of %lld", name, what,
                        static_cast<long long>(m->stride), static_cast<long long>(m->cols));
    if (m->rows > 0 && m->cols > 0 && (m->data == nullptr || !elem_aligned(m->data, m->dtype)))
        return ops_fail(GOCKPT_EINVAL, "%s: %s is null or not aligned to its element", name, what);
    return GOCKPT_OK;
}

int check_act8(const char* name, const char* what, const gockpt_act8* a, int64_t rows, int64_t cols) {
    if (a == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null %s", name, what);
    if (a->rows != rows || a->cols != cols)
        return ops_fail(GOCKPT_EINVAL, "%s: %s of %lld x %lld, expected %lld x %lld", name, what,
                        static_cast<long long>(a->rows), static_cast<long long>(a->cols), static_cast<long long>(rows),
                        static_cast<long long>(cols));
    if (rows > 0 && cols > 0 &&
        (a->codes == nullptr || a->scales == nullptr || reinterpret_cast<uintptr_t>(a->codes) % 16 != 0))
        return ops_fail(GOCKPT_EINVAL, "%s: %s is null or its codes are not aligned to 16 bytes", name, what);
    return GOCKPT_OK;
}

int check_workspace(const char* name, const void* workspace, size_t have, size_t need) {
    if (need == 0) return GOCKPT_OK;
    if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
        return ops_fail(GOCKPT_EINVAL, "%s: the workspace must be 256-byte aligned", name);
    if (have < need) return ops_fail(GOCKPT_ENOMEM, "%s: workspace of %zu bytes, %zu needed", name, have, need);
    return GOCKPT_OK;
}

}  // namespace gockpt
