// gockpt_model_internal.h -- what the operators of gockpt_model.h share on the
// host: checks of arguments, workspaces, and the products of gockpt_mma.h.
#pragma once

#include <algorithm>

#include "../../include/gockpt_model.h"
#include "gockpt_ops_internal.h"

namespace gockpt {

struct MmaArgs;
struct StoreArgs;

constexpr int64_t kMaxExtent = int64_t{1} << 30;  // rows and columns: sums of tiles stay in 32 bits
constexpr int64_t kMaxWidth = int64_t{1} << 22;   // columns of what products read
constexpr int kUnits = 256;                       // compute units

constexpr int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A matrix of an operator; `types` tells which it may have (a bit each).
constexpr int kAnyType = 7, kHalfTypes = 1 << kBF16 | 1 << kFP16;
int check_model_matrix(const char* name, const char* what, const gockpt_matrix* m, int types);
int check_act8(const char* name, const char* what, const gockpt_act8* a, int64_t rows, int64_t cols);

// Parts of a workspace, one after another at multiples of 256 bytes.
struct Parts {
    size_t bytes = 0;
    size_t take(int64_t n) {
        const size_t at = bytes;
        bytes += static_cast<size_t>(up(n, 256));
        return at;
    }
};
int check_workspace(const char* name, const void* workspace, size_t have, size_t need);

// Read in place by a product: 16-byte pieces of 8 columns, at offsets of 32
// bits within a tile.
inline bool in_place(const gockpt_matrix& m) {
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && m.cols % 8 == 0 &&
           (m.rows <= 1 || (m.stride % 8 == 0 && m.stride < (int64_t{1} << 23)));
}

// Elements from one row of a copy to the next: whole cache lines where that costs
// little, as a tile's 128 bytes of a row else lie in two (1865 x 32000 logits of 1160
// columns 146 us, of 1152 125, of 1216 131).
inline int64_t copy_stride(int64_t cols) { return up(cols, cols > 256 ? 64 : 8); }

// A 16-bit matrix as a product reads it: in place, or copied to `copy` with
// rows of `cols` rounded up to 8, zeros behind the last column.
struct Source {
    const uint8_t* data;
    int64_t stride;  // bytes
};
inline int64_t copy_bytes(const gockpt_matrix& m) { return in_place(m) ? 0 : m.rows * copy_stride(m.cols) * 2; }
inline Source copied(const gockpt_matrix& m, uint8_t* copy) { return {copy, copy_stride(m.cols) * 2}; }

// The copies that a call needs, of at most two matrices, in one launch.
struct Copies {
    // Row c of dst = row rows[c] of src (null: row c), for c < *count (null: n).
    struct One {
        const uint8_t* src;
        int64_t stride, dst_stride;
        const int32_t *rows, *count;
        uint8_t* dst;
        int32_t cols, n;
        uint32_t blocks;
    } one[2] = {};
    int many = 0;

    Source source_of(const gockpt_matrix& m, uint8_t* copy) {
        if (in_place(m)) return {static_cast<const uint8_t*>(m.data), (m.rows > 1 ? m.stride : m.cols) * 2};
        return rows_of(m, nullptr, nullptr, m.rows, copy);
    }
    Source rows_of(const gockpt_matrix& src, const int32_t* rows, const int32_t* count, int64_t n, uint8_t* dst);
    void launch(hipStream_t s) const;
};

// gockpt_act8_pack, and x copied as above with it (copy not null: 16-bit x).
int pack_and_copy(const char* name, const gockpt_matrix* x, const gockpt_act8* out, uint8_t* copy, hipStream_t s);

// The products by how their operands lie (R, C).
enum ProductKind : int { kAlongAlong = 0, kAcrossAlong = 1, kAcrossAcross = 2 };
// 256 x 256, 128 x 128 and 128 x 32 tiles of r x c, the last one 32 x 32 where both lie along k
enum Shape : int { kWide = 0, kMid = 1, kThin = 2 };

struct ProductPlan {
    int shape;
    int splits;       // slices of k; more than 1: fp32 sums that finish_kernel joins
    int32_t split_k;
    uint32_t tiles_r, tiles_c;
    double us;        // expected
};
// most_splits 1: not split.
ProductPlan plan_product(int kind, int64_t rn, int64_t cn, int64_t k, int most_splits);

// Threads of a block of each shape.
constexpr int product_threads(int shape) { return shape == kWide ? 512 : 256; }

// A launch has fewer than 2^32 threads.
inline bool too_many_blocks(const ProductPlan& p) {
    const uint64_t most = ((uint64_t{1} << 32) - 1) / static_cast<uint64_t>(product_threads(p.shape));
    return p.splits > 0 && uint64_t{p.tiles_r} * p.tiles_c > most / static_cast<uint64_t>(p.splits);
}

// Starts the product of the operands in `a`, which the plan completes.
void launch_product(int kind, int dtype, const ProductPlan& p, MmaArgs& a, const StoreArgs& o, hipStream_t s);

// out row t = round(alpha * beta * sum over the slices of their row c), c =
// of_row[t] (null: t; negative: zeros), added to what is there with accumulate.
// With fix: fix[c] times row fix_row[c] of a 16-bit matrix (none where that is
// negative) is added to the slices' sum.
struct FinishArgs {
    const float* slices;
    int64_t slice_step;  // elements from one slice to the next
    int32_t count;       // slices
    int32_t rows, cols;
    const int32_t* of_row;
    uint8_t* out;
    int64_t stride;  // bytes
    int32_t dtype, accumulate;
    float alpha;
    const float* beta;
    const float* fix;
    const int32_t* fix_row;
    const uint8_t* fix_from;
    int64_t fix_stride;  // bytes; rows of whole pieces of 8
    int32_t fix_dtype;
    const float* up;  // row c's sum is up[c] times too large, a power of two (null: none is)
};
void launch_finish(const FinishArgs& f, hipStream_t s);

}  // namespace gockpt
