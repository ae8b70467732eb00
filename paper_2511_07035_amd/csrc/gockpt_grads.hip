// gockpt_grads.hip -- norm and clipping of a list of gradient tensors.
//
//   sumsq_kernel   reads every tensor once: S = sum of squares, one fp64
//                  partial a block.
//   result_kernel  one block: adds the partials in a fixed order;
//                  norm = sqrt(S) / scale, found_inf, and the clipping
//                  coefficient min(1, max_norm / (norm + 1e-6)).
//   scale_kernel   element * coef, rounded to the destination's type.
//
// The host cuts the tensors into tiles of at most 1024 units of 16 source
// bytes (16 KiB) once, when the list is made; a tensor of any size, type,
// stride or start is a few entries of one table, and one launch covers all.
#include <math.h>

#include <new>
#include <vector>

#include "gockpt_ops_internal.h"

#pragma clang fp contract(off)

namespace gockpt {

namespace {

constexpr int kThreads = 256;
constexpr int kUnitsPerThread = 4;
constexpr int kTileUnits = kThreads * kUnitsPerThread;
constexpr int kMaxBlocks = 2048;  // 8 blocks of 4 wavefronts on each of 256 compute units
constexpr double kClipEps = 1e-6;

// Rows of one tensor, or a piece of one row.  Unit u of a tile is unit u %
// per_row of row u / per_row; every unit but a row's last holds 16 bytes.
struct GradTile {
    const uint8_t* src;
    uint8_t* dst;
    int64_t stride;    // bytes from a row to the next
    int64_t dst_row;   // the same in dst
    int32_t units;     // of the tile, at most kTileUnits
    int32_t per_row;   // units of a row
    uint32_t magic;    // per_row > 1: floor(2^32 / per_row) + 1, u / per_row is the high word of u * magic
    int16_t last;      // bytes in a row's last unit, 2 to 16
    int8_t dtype, dst_dtype;
};
static_assert(sizeof(GradTile) == 48, "table entry");

// u * magic >> 32 is u / d for every u <= kTileUnits: the product exceeds
// u * 2^32 / d by at most u, and u * d <= kTileUnits^2 < 2^32.
__device__ __forceinline__ void unit_place(const GradTile& t, uint32_t u, uint32_t& row, uint32_t& k) {
    if (t.units == t.per_row) {
        row = 0;
        k = u;
    } else if (t.per_row == 1) {
        row = u;
        k = 0;
    } else {
        row = __umulhi(u, t.magic);
        k = u - row * static_cast<uint32_t>(t.per_row);
    }
}

// Unit u of the tile; zeros in the places behind the row's end.
__device__ __forceinline__ u32x4 load_unit(const GradTile& t, uint32_t u) {
    uint32_t row, k;
    unit_place(t, u, row, k);
    const uint8_t* p = t.src + row * t.stride + k * 16u;
    if (k + 1 < static_cast<uint32_t>(t.per_row) || t.last == 16) return *reinterpret_cast<const u32x4_any*>(p);
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    u32x4 raw = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (2 * i < t.last) raw[i / 2] |= static_cast<uint32_t>(h[i]) << (16 * (i & 1));
    return raw;
}

__device__ __forceinline__ void load_tile(const GradTile& t, u32x4 (&raw)[kUnitsPerThread]) {
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        const uint32_t u = i * kThreads + threadIdx.x;
        raw[i] = (u32x4){0u, 0u, 0u, 0u};
        if (u < static_cast<uint32_t>(t.units)) raw[i] = load_unit(t, u);
    }
}

template <int kT, class F>
__device__ __forceinline__ void each_elem(u32x4 raw, F&& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kT == kFP32) {
            f(__uint_as_float(raw[i]));
        } else {
            f(elem_to_f32<kT>(raw[i] & 0xFFFFu));
            f(elem_to_f32<kT>(raw[i] >> 16));
        }
    }
}

// Sum of squares of a thread's units (at most 32 elements).  In fp32 unless
// that may have lost something: an fp32 sum in [2^-100, 2^126) has overflowed
// nowhere, and what its terms lost below 2^-149 is under 2^-44 of it.
// Otherwise (or where it is NaN), and if some element is not zero, the squares
// are added again in fp64, where those of fp32 values neither overflow nor
// vanish and the sum is finite exactly when every element is.
template <int kT>
__device__ __forceinline__ double square_sum(const u32x4 (&raw)[kUnitsPerThread]) {
    float s = 0.0f;
    uint32_t any = 0u;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        any |= raw[i][0] | raw[i][1] | raw[i][2] | raw[i][3];
        each_elem<kT>(raw[i], [&](float x) { s = __builtin_fmaf(x, x, s); });
    }
    if ((s >= 0x1p-100f && s < 0x1p126f) || any == 0u) return static_cast<double>(s);
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i)
        each_elem<kT>(raw[i], [&](float x) { d = __builtin_fma(static_cast<double>(x), static_cast<double>(x), d); });
    return d;
}

__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[kThreads / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(kThreads) void sumsq_kernel(const GradTile* __restrict__ tiles, int ntiles,
                                                         double* __restrict__ parts) {
    double acc = 0.0;
    for (int i = blockIdx.x; i < ntiles; i += gridDim.x) {
        const GradTile t = tiles[i];
        u32x4 raw[kUnitsPerThread];
        load_tile(t, raw);
        if (t.dtype == kBF16)
            acc += square_sum<kBF16>(raw);
        else if (t.dtype == kFP16)
            acc += square_sum<kFP16>(raw);
        else
            acc += square_sum<kFP32>(raw);
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0) parts[blockIdx.x] = acc;
}

__device__ __forceinline__ void finish_result(double sumsq, const float* scale, double max_norm,
                                              gockpt_grad_result* out) {
    const double norm = sqrt(sumsq) / (scale != nullptr ? static_cast<double>(*scale) : 1.0);
    const bool finite = isfinite(sumsq);
    const double coef = max_norm / (norm + kClipEps);
    out->sumsq = sumsq;
    out->norm = static_cast<float>(norm);
    out->found_inf = finite ? 0.0f : 1.0f;
    out->coef = finite && coef < 1.0 ? static_cast<float>(coef) : 1.0f;
    out->reserved_[0] = out->reserved_[1] = out->reserved_[2] = 0.0f;
}

__global__ __launch_bounds__(kThreads) void result_kernel(const double* __restrict__ parts, int nparts,
                                                          const float* __restrict__ scale, double max_norm,
                                                          gockpt_grad_result* __restrict__ out) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kThreads) acc += parts[i];
    acc = block_sum(acc);
    if (threadIdx.x == 0) finish_result(acc, scale, max_norm, out);
}

__global__ void result_again_kernel(gockpt_grad_result* out, const float* scale, double max_norm) {
    finish_result(out->sumsq, scale, max_norm, out);
}

// One unit times coef to its place in dst.
template <int kS, int kD>
__device__ __forceinline__ void scale_unit(u32x4 raw, float coef, uint8_t* d, int last) {
    constexpr int kN = kS == kFP32 ? 4 : 8;
    constexpr int kB = kD == kFP32 ? 4 : 2;
    float x[kN];
    int n = 0;
    each_elem<kS>(raw, [&](float v) { x[n++] = v * coef; });
    if (last == 16) {
        if constexpr (kD == kFP32) {
#pragma unroll
            for (int i = 0; i < kN; i += 4)
                *reinterpret_cast<u32x4_any*>(d + 4 * i) =
                    (u32x4){__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                            __float_as_uint(x[i + 3])};
        } else if constexpr (kN == 8) {
            *reinterpret_cast<u32x4_any*>(d) = (u32x4){pack2<kD>(x[0], x[1]), pack2<kD>(x[2], x[3]),
                                                       pack2<kD>(x[4], x[5]), pack2<kD>(x[6], x[7])};
        } else {
            *reinterpret_cast<u32x2_any*>(d) = (u32x2){pack2<kD>(x[0], x[1]), pack2<kD>(x[2], x[3])};
        }
    } else {
        const int m = last / (kS == kFP32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (i < m) store_elem<kD>(d + kB * i, x[i]);
    }
}

template <int kS, int kD>
__device__ __forceinline__ void scale_tile(const GradTile& t, float coef) {
    u32x4 raw[kUnitsPerThread];
    load_tile(t, raw);
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        const uint32_t u = i * kThreads + threadIdx.x;
        if (u >= static_cast<uint32_t>(t.units)) break;
        uint32_t row, k;
        unit_place(t, u, row, k);
        const int last = k + 1 < static_cast<uint32_t>(t.per_row) ? 16 : t.last;
        constexpr uint32_t kUnitOut = 16u * (kD == kFP32 ? 4 : 2) / (kS == kFP32 ? 4 : 2);
        scale_unit<kS, kD>(raw[i], coef, t.dst + row * t.dst_row + k * kUnitOut, last);
    }
}

__global__ __launch_bounds__(kThreads) void scale_kernel(const GradTile* __restrict__ tiles, int ntiles,
                                                         const gockpt_grad_result* __restrict__ result) {
    const float coef = result->coef;
    for (int i = blockIdx.x; i < ntiles; i += gridDim.x) {
        const GradTile t = tiles[i];
        if (t.dst == t.src && coef == 1.0f) continue;
        switch (t.dtype * 3 + t.dst_dtype) {
            case kBF16 * 3 + kBF16: scale_tile<kBF16, kBF16>(t, coef); break;
            case kBF16 * 3 + kFP16: scale_tile<kBF16, kFP16>(t, coef); break;
            case kBF16 * 3 + kFP32: scale_tile<kBF16, kFP32>(t, coef); break;
            case kFP16 * 3 + kBF16: scale_tile<kFP16, kBF16>(t, coef); break;
            case kFP16 * 3 + kFP16: scale_tile<kFP16, kFP16>(t, coef); break;
            case kFP16 * 3 + kFP32: scale_tile<kFP16, kFP32>(t, coef); break;
            case kFP32 * 3 + kBF16: scale_tile<kFP32, kBF16>(t, coef); break;
            case kFP32 * 3 + kFP16: scale_tile<kFP32, kFP16>(t, coef); break;
            default: scale_tile<kFP32, kFP32>(t, coef); break;
        }
    }
}

// ---- host: the table ---------------------------------------------------------

constexpr int64_t kMaxElems = int64_t{1} << 46;
constexpr size_t kPartsBytes = kMaxBlocks * sizeof(double);

// A tensor as the tiles see it: rows that follow one another are one row.
struct Flat {
    int64_t rows, cols, stride;
};

int check_tensor(const char* name, int64_t i, const gockpt_grad_tensor& t, Flat* flat) {
    const long long at = static_cast<long long>(i);
    if (!dtype_ok(t.dtype)) return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dtype %d", name, at, t.dtype);
    if (t.dst != nullptr && !dtype_ok(t.dst_dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst_dtype %d", name, at, t.dst_dtype);
    if (t.rows < 0 || t.cols < 0 || t.rows > kMaxElems || t.cols > kMaxElems ||
        (t.cols > 0 && t.rows > kMaxElems / t.cols))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: %lld x %lld elements", name, at,
                        static_cast<long long>(t.rows), static_cast<long long>(t.cols));
    if (t.rows > 1 && (t.stride < t.cols || t.stride > kMaxElems / t.rows))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: stride %lld for rows of %lld", name, at,
                        static_cast<long long>(t.stride), static_cast<long long>(t.cols));
    *flat = {0, 0, 0};
    if (t.rows == 0 || t.cols == 0) return GOCKPT_OK;
    if (t.data == nullptr || !elem_aligned(t.data, t.dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: data is null or not aligned to its element", name, at);
    if (t.dst != nullptr && !elem_aligned(t.dst, t.dst_dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst is not aligned to its element", name, at);
    if (t.dst == t.data && (t.dst_dtype != t.dtype || (t.rows > 1 && t.stride != t.cols)))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst is data of another type or layout", name, at);
    *flat = t.rows == 1 || t.stride == t.cols ? Flat{1, t.rows * t.cols, 0} : Flat{t.rows, t.cols, t.stride};
    return GOCKPT_OK;
}

// Calls f(first row, rows, first element of the row, elements) for each tile.
template <class F>
void each_tile(const Flat& x, int dtype, F&& f) {
    const int64_t per_unit = 16 / dtype_bytes(dtype);
    const int64_t units = (x.cols + per_unit - 1) / per_unit;
    if (units <= 0) return;
    if (x.rows == 1 || units * 2 > kTileUnits) {  // pieces of a row
        for (int64_t r = 0; r < x.rows; ++r)
            for (int64_t c = 0; c < x.cols; c += kTileUnits * per_unit)
                f(r, int64_t{1}, c, x.cols - c < kTileUnits * per_unit ? x.cols - c : kTileUnits * per_unit);
    } else {  // several rows
        const int64_t n = kTileUnits / units;
        for (int64_t r = 0; r < x.rows; r += n) f(r, x.rows - r < n ? x.rows - r : n, int64_t{0}, x.cols);
    }
}

int64_t count_tiles(const Flat& x, int dtype) {
    const int64_t per_unit = 16 / dtype_bytes(dtype);
    const int64_t units = (x.cols + per_unit - 1) / per_unit;
    if (units <= 0) return 0;
    if (x.rows == 1 || units * 2 > kTileUnits) return x.rows * ((units + kTileUnits - 1) / kTileUnits);
    const int64_t n = kTileUnits / units;
    return (x.rows + n - 1) / n;
}

int count_list(const char* name, const gockpt_grad_tensor* tensors, int64_t count, int64_t* ntiles) {
    *ntiles = 0;
    if (count < 0 || (count > 0 && tensors == nullptr)) return ops_fail(GOCKPT_EINVAL, "%s: tensor list", name);
    for (int64_t i = 0; i < count; ++i) {
        Flat x;
        const int rc = check_tensor(name, i, tensors[i], &x);
        if (rc != GOCKPT_OK) return rc;
        *ntiles += count_tiles(x, tensors[i].dtype);
        if (*ntiles > (int64_t{1} << 30)) return ops_fail(GOCKPT_EINVAL, "%s: too many elements", name);
    }
    return GOCKPT_OK;
}

}  // namespace

}  // namespace gockpt

using namespace gockpt;

struct gockpt_grads {
    double* parts;
    const GradTile* tiles;
    int ntiles, blocks;
};

extern "C" {

int gockpt_grads_bytes(const gockpt_grad_tensor* tensors, int64_t count, size_t* bytes) {
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "gockpt_grads_bytes: null argument");
    *bytes = 0;
    int64_t ntiles;
    const int rc = count_list("gockpt_grads_bytes", tensors, count, &ntiles);
    if (rc == GOCKPT_OK) *bytes = (kPartsBytes + ntiles * sizeof(GradTile) + 255) / 256 * 256;
    return rc;
}

int gockpt_grads_create(const gockpt_grad_tensor* tensors, int64_t count, void* workspace, size_t workspace_bytes,
                        void* stream, gockpt_grads** out) {
    const char* name = "gockpt_grads_create";
    if (out == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *out = nullptr;
    int64_t ntiles;
    const int rc = count_list(name, tensors, count, &ntiles);
    if (rc != GOCKPT_OK) return rc;
    if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
        return ops_fail(GOCKPT_EINVAL, "%s: the workspace must be 256-byte aligned", name);
    if (workspace_bytes < kPartsBytes + ntiles * sizeof(GradTile))
        return ops_fail(GOCKPT_ENOMEM, "%s: workspace of %zu bytes", name, workspace_bytes);
    std::vector<GradTile> table;
    try {
        table.reserve(static_cast<size_t>(ntiles));
        for (int64_t i = 0; i < count; ++i) {
            const gockpt_grad_tensor& t = tensors[i];
            Flat x;
            check_tensor(name, i, t, &x);
            const bool in_place = t.dst == nullptr || t.dst == t.data;
            const int dst_dtype = in_place ? t.dtype : t.dst_dtype;
            const int64_t sb = dtype_bytes(t.dtype), db = dtype_bytes(dst_dtype);
            const int64_t dst_cols = in_place ? x.stride : x.cols;
            uint8_t* dst = static_cast<uint8_t*>(in_place ? const_cast<void*>(t.data) : t.dst);
            const uint8_t* src = static_cast<const uint8_t*>(t.data);
            each_tile(x, t.dtype, [&](int64_t r, int64_t rows, int64_t c, int64_t cols) {
                GradTile g{};
                g.src = src + (r * x.stride + c) * sb;
                g.dst = dst + (r * dst_cols + c) * db;
                g.stride = x.stride * sb;
                g.dst_row = dst_cols * db;
                g.per_row = static_cast<int32_t>((cols * sb + 15) / 16);
                g.units = static_cast<int32_t>(rows) * g.per_row;
                g.magic = g.per_row > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / g.per_row) + 1u : 0u;
                g.last = static_cast<int16_t>(cols * sb - (g.per_row - 1) * 16);
                g.dtype = static_cast<int8_t>(t.dtype);
                g.dst_dtype = static_cast<int8_t>(dst_dtype);
                table.push_back(g);
            });
        }
    } catch (...) {
        return ops_fail(GOCKPT_ENOMEM, "%s: out of host memory", name);
    }
    gockpt_grads* list = new (std::nothrow) gockpt_grads;
    if (list == nullptr) return ops_fail(GOCKPT_ENOMEM, "%s: out of host memory", name);
    list->parts = static_cast<double*>(workspace);
    list->tiles = reinterpret_cast<const GradTile*>(static_cast<uint8_t*>(workspace) + kPartsBytes);
    list->ntiles = static_cast<int>(table.size());
    list->blocks = list->ntiles < kMaxBlocks ? list->ntiles : kMaxBlocks;
    if (!table.empty()) {
        hipStream_t s = static_cast<hipStream_t>(stream);
        hipError_t e = hipMemcpyAsync(const_cast<GradTile*>(list->tiles), table.data(),
                                      table.size() * sizeof(GradTile), hipMemcpyHostToDevice, s);
        const hipError_t w = hipStreamSynchronize(s);
        if (e == hipSuccess) e = w;
        if (e != hipSuccess) {
            delete list;
            return ops_fail(GOCKPT_EHIP, "%s: %s", name, hipGetErrorString(e));
        }
    }
    *out = list;
    return GOCKPT_OK;
}

int gockpt_grads_destroy(gockpt_grads* list) {
    delete list;
    return GOCKPT_OK;
}

static int check_norm(const char* name, const void* scale, double max_norm, const void* result) {
    if (result == nullptr || reinterpret_cast<uintptr_t>(result) % 8 != 0)
        return ops_fail(GOCKPT_EINVAL, "%s: the result must be 8-byte aligned device memory", name);
    if (reinterpret_cast<uintptr_t>(scale) % 4 != 0) return ops_fail(GOCKPT_EINVAL, "%s: scale alignment", name);
    if (!(max_norm >= 0.0)) return ops_fail(GOCKPT_EINVAL, "%s: max_norm %g", name, max_norm);
    return GOCKPT_OK;
}

int gockpt_grads_norm(gockpt_grads* list, const float* scale, double max_norm, gockpt_grad_result* result,
                      void* stream) {
    const char* name = "gockpt_grads_norm";
    if (list == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null list", name);
    const int rc = check_norm(name, scale, max_norm, result);
    if (rc != GOCKPT_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (list->blocks > 0)
        hipLaunchKernelGGL(sumsq_kernel, dim3(list->blocks), dim3(kThreads), 0, s, list->tiles, list->ntiles,
                           list->parts);
    hipLaunchKernelGGL(result_kernel, dim3(1), dim3(kThreads), 0, s, list->parts, list->blocks, scale, max_norm,
                       result);
    return ops_launched(name);
}

int gockpt_grads_scale(gockpt_grads* list, const gockpt_grad_result* result, void* stream) {
    const char* name = "gockpt_grads_scale";
    if (list == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null list", name);
    const int rc = check_norm(name, nullptr, 0.0, result);
    if (rc != GOCKPT_OK) return rc;
    if (list->blocks > 0)
        hipLaunchKernelGGL(scale_kernel, dim3(list->blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream),
                           list->tiles, list->ntiles, result);
    return ops_launched(name);
}

int gockpt_grads_clip(gockpt_grads* list, const float* scale, double max_norm, gockpt_grad_result* result,
                      void* stream) {
    const int rc = gockpt_grads_norm(list, scale, max_norm, result, stream);
    return rc != GOCKPT_OK ? rc : gockpt_grads_scale(list, result, stream);
}

int gockpt_grads_result(gockpt_grad_result* result, const float* scale, double max_norm, void* stream) {
    const char* name = "gockpt_grads_result";
    const int rc = check_norm(name, scale, max_norm, result);
    if (rc != GOCKPT_OK) return rc;
    hipLaunchKernelGGL(result_again_kernel, dim3(1), dim3(1), 0, static_cast<hipStream_t>(stream), result, scale,
                       max_norm);
    return ops_launched(name);
}

}  // extern "C"
