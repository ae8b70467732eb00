// gockpt_act8.hip -- activations in 8 bits: packing, restoring, and the (gated)
// activation that keeps its inputs so.
//
// Four lanes share a block of 32 columns, 8 each: a lane's 16-bit values are one
// 16-byte load, the block's largest magnitude takes two exchanges between
// neighbours, and a lane's codes are one 8-byte store.  All of it is one pass
// over the data, bound by memory: 65536 x 5120 bf16 values are packed in 184 us
// (5.5 TB/s) and restored in 172 (5.9), 14000 x 11008 gated ones take 208 us
// forward and 199 back (6.0 and 6.25 TB/s).  One group of 8 a thread, and as many
// blocks as that makes: with 8 or 64 blocks a compute unit that go on to the next
// groups the same calls take 207, 194, 246, 233 and 194, 187, 233, 225 us.
#include "gockpt_model_internal.h"

namespace gockpt {

namespace {

constexpr int kThreads = 256;
constexpr int kLaneCols = 8;

struct Rows {
    uint8_t* p;      // row r at p + r * stride bytes
    int64_t stride;
};

struct Kept {
    uint8_t* codes;
    uint8_t* scales;
};

// A lane's place: 8 columns of a row, of which `n` are there (0 or less: none).
struct Place {
    int64_t row, block;  // block: among all of the matrix
    int32_t col, n;
};

__device__ __forceinline__ Place place_of(int64_t group, int32_t blocks, int32_t cols) {
    Place p;
    p.block = group >> 2;
    // 32-bit division where it will do: a 64-bit one costs ten times as much
    p.row = p.block <= INT32_MAX ? static_cast<uint32_t>(p.block) / static_cast<uint32_t>(blocks) : p.block / blocks;
    p.col = static_cast<int32_t>(p.block - p.row * blocks) * GOCKPT_ACT8_BLOCK +
            static_cast<int32_t>(group & 3) * kLaneCols;
    p.n = min(cols - p.col, kLaneCols);
    return p;
}

// 16 bytes; past the caches where `far`.
__device__ __forceinline__ u32x4 load16(const uint8_t* p, bool far) {
    const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p);
    return far ? __builtin_nontemporal_load(q) : *q;
}

__device__ __forceinline__ void store16(uint8_t* p, u32x4 x, bool far) {
    u32x4_any* q = reinterpret_cast<u32x4_any*>(p);
    if (far)
        __builtin_nontemporal_store(x, q);
    else
        *q = x;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// A lane's 8 values (zeros for missing ones), and the bits, as fp32's, of the
// largest magnitude: infinity and NaN above all others.
template <int kT>
__device__ __forceinline__ void load8(const uint8_t* p, int n, bool far, float (&x)[8], uint32_t& top) {
    top = 0;
    if (n == kLaneCols) {
        if constexpr (kT == kFP32) {
            const u32x4 a = load16(p, far), b = load16(p + 16, far);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __uint_as_float(a[i]);
                x[4 + i] = __uint_as_float(b[i]);
                top = max(top, max(a[i] & 0x7fffffffu, b[i] & 0x7fffffffu));
            }
        } else {
            const u32x4 a = load16(p, far);
            u16x2 most = {0, 0};  // magnitudes of 16 bits compare as their bits do, two at a time
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = elem_to_f32<kT>(a[i] & 0xffff);
                x[2 * i + 1] = elem_to_f32<kT>(a[i] >> 16);
                most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, a[i] & 0x7fff7fffu));
            }
            top = __float_as_uint(elem_to_f32<kT>(max(most.x, most.y)));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = 0.0f;
        if (i < n) {
            if constexpr (kT == kFP32)
                x[i] = reinterpret_cast<const float*>(p)[i];
            else
                x[i] = elem_to_f32<kT>(reinterpret_cast<const uint16_t*>(p)[i]);
        }
        top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    }
}

template <int kT>
__device__ __forceinline__ void store8(uint8_t* p, int n, bool far, const float (&x)[8]) {
    if (n == kLaneCols) {
        if constexpr (kT == kFP32) {
            u32x4 a, b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = __float_as_uint(x[i]);
                b[i] = __float_as_uint(x[4 + i]);
            }
            store16(p, a, far);
            store16(p + 16, b, far);
        } else {
            u32x4 a;
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = pack2<kT>(x[2 * i], x[2 * i + 1]);
            store16(p, a, far);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) store_elem<kT>(p + i * dtype_bytes(kT), x[i]);
}

// The largest of four neighbouring lanes' values.
__device__ __forceinline__ uint32_t max_of_4(uint32_t x) {
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0xB1, 0xf, 0xf, true)));  // 1 0 3 2
    return max(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x4E, 0xf, 0xf, true)));  // 2 3 0 1
}

// Four codes: the lowest byte of each number in turn.
__device__ __forceinline__ uint32_t bytes_of(const uint32_t (&b)[8], int i) {
    return __builtin_amdgcn_perm(b[i + 1], b[i], 0x0c0c0400) | __builtin_amdgcn_perm(b[i + 3], b[i + 2], 0x04000c0c);
}

// Codes and the scale's byte of a block that four lanes hold.  The largest
// magnitude m * 2^q, 1 <= m < 2, is at most 127 * 2^(q - 6) where m is at most
// 127 / 64, that is where its fraction's bits are at most 0x7e0000.  x / 2^e is
// exact, so its sum with 1.5 * 2^23 rounds it to the nearest whole number, ties to
// even, and leaves that in two's complement in the lowest bits.
template <int kT>
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], uint32_t top, u32x2& codes) {
    const uint32_t most = max_of_4(top);
    const int scale = max(1, static_cast<int>(most >> 23) - ((most & 0x7fffffu) <= 0x7e0000u ? 6 : 5));
    // up to here 64 times the scale is within the type's range
    constexpr int kTop = kT == kFP16 ? 127 + 9 : 127 + 121;
    const float down = __uint_as_float(static_cast<uint32_t>(254 - scale) << 23);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__builtin_fmaf(x[i], down, 12582912.0f));
    if (scale > kTop) {  // at the end of the type's range, or beyond it
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = max(-63, min(63, static_cast<int>(b[i] << 24) >> 24));
            b[i] = static_cast<uint32_t>(c);
        }
    }
    codes = u32x2{bytes_of(b, 0), bytes_of(b, 4)};
    if (most >= 0x7f800000u) codes = u32x2{0, 0};
    return most >= 0x7f800000u ? 255 : static_cast<uint32_t>(scale);
}

__device__ __forceinline__ void keep8(const Kept& k, int64_t group, bool far, u32x2 codes, uint32_t scale) {
    u32x2* p = reinterpret_cast<u32x2*>(k.codes + group * kLaneCols);
    if (far)
        __builtin_nontemporal_store(codes, p);
    else
        *p = codes;
    if ((group & 3) == 0) k.scales[group >> 2] = static_cast<uint8_t>(scale);
}

// (128 s, which would save an instruction, need not be finite.)
__device__ __forceinline__ void decode8(u32x2 codes, uint32_t scale, float (&x)[8]) {
    const float s = __uint_as_float(scale << 23 | (scale == 255 ? 0x400000u : 0u));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(static_cast<int8_t>(codes[i / 4] >> (8 * (i & 3)))) * s;
}

__device__ __forceinline__ void restore8(const Kept& k, int64_t group, float (&x)[8]) {
    decode8(*reinterpret_cast<const u32x2*>(k.codes + group * kLaneCols), k.scales[group >> 2], x);
}

// ---- activations ------------------------------------------------------------------

// exp, and 1 / (1 + exp(-x)).  Outputs of 16 bits take the hardware's exp2 of the
// product with log2(e).  The constant is off by 0.23 2^-24 of itself and the
// rounding of the product by 2^-24, the result so by 1.23 |x| 2^-24 of itself and by
// the instruction's own 2^-23: 2^-17 in all where anything is left of the result (|x|
// up to 88).  fp32 outputs take the library's exp.
template <int kT>
__device__ __forceinline__ float exp_of(float x) {
    if constexpr (kT == kFP32)
        return expf(x);
    else
        return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}

template <int kT>
__device__ __forceinline__ float sigmoid(float x) {
    const float e = exp_of<kT>(-x);
    if constexpr (kT == kFP32)
        return 1.0f / (1.0f + e);
    else
        return __builtin_amdgcn_rcpf(1.0f + e);
}

// Phi(x) = (1 + erf(x / sqrt 2)) / 2 and phi(x), its derivative.  16-bit outputs take
// the tail as exp(-x^2 / 2) / 2 times erfcx(z) = exp(z^2) erfc(z), z = |x| / sqrt 2,
// which falls as 1 / z: t P(t) with t = 1 / (1 + 0.435 z).  P is of the fifth degree,
// fitted here to the least largest relative error over 0 <= z <= 10, 2^-17.7 of the
// tail.  With the exponential's (1.12 x^2 2^-24, its argument's two roundings and the
// constant's) that is 2^-15 at most wherever the result is a bf16, x > -13.7: far
// below half a step also in the far tail, where an error that is small against 1 is
// not small against the result.
template <int kT>
__device__ __forceinline__ void normal(float x, float& cdf, float& pdf) {
    const float e = exp_of<kT>(-0.5f * x * x);
    pdf = 0.398942280401432677940f * e;
    if constexpr (kT == kFP32) {
        cdf = 0.5f * erfcf(-0.707106781186547524401f * x);
    } else {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.435f * 0.707106781186547524401f * fabsf(x));
        float p = 0.3812965552f - 0.1508592834f * t;
        p = p * t + 0.01285750788f;
        p = p * t + 0.2734441863f;
        p = p * t + 0.2373346605f;
        p = p * t + 0.2459255198f;
        const float tail = 0.5f * p * t * e;
        cdf = x < 0.0f ? tail : 1.0f - tail;
    }
}

// act(x) and, where kSlope, its derivative.
template <int kT, int kKind, bool kSlope>
__device__ __forceinline__ void activate(float x, float& y, float& slope) {
    if constexpr (kKind == GOCKPT_GELU) {
        float c, d;
        normal<kT>(x, c, d);
        y = x * c;
        if (kSlope) slope = c + x * d;
    } else {
        float inner = x, inner_slope = 1.0f;
        if constexpr (kKind == GOCKPT_GELU_TANH) {  // (1 + tanh(u)) / 2 = sigmoid(2 u)
            constexpr float kA = 1.59576912160573071176f, kB = 0.044715f;
            // beyond 64 both are at their limits, and the square of a large x is inf
            const float c = fmaxf(-64.0f, fminf(64.0f, x)), s = c * c;
            inner = kA * c * (1.0f + kB * s);
            inner_slope = kA * (1.0f + 3.0f * kB * s);
        }
        const float s = sigmoid<kT>(inner);
        y = x * s;
        if (kSlope) slope = s + y * (1.0f - s) * inner_slope;
    }
}

// ---- kernels ----------------------------------------------------------------------

struct PackArgs {
    Rows x, copy;  // copy: of 16-bit x (null: none), whole pieces of 8
    Kept kept;
    int64_t groups;  // of 8 columns, blocks' missing ones among them
    int32_t blocks, cols;
};

template <int kT>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs a) {
    for (int64_t g = blockIdx.x * int64_t{kThreads} + threadIdx.x; g < a.groups; g += gridDim.x * int64_t{kThreads}) {
        const Place p = place_of(g, a.blocks, a.cols);
        float x[8];
        uint32_t top;
        load8<kT>(a.x.p + p.row * a.x.stride + int64_t{p.col} * dtype_bytes(kT), p.n, false, x, top);
        u32x2 codes;
        const uint32_t scale = encode8<kT>(x, top, codes);
        keep8(a.kept, g, false, codes, scale);
        if constexpr (kT != kFP32)
            if (a.copy.p != nullptr && p.n > 0)
                store8<kT>(a.copy.p + p.row * a.copy.stride + int64_t{p.col} * 2, kLaneCols, false, x);
    }
}

template <int kT>
__global__ __launch_bounds__(kThreads) void unpack_kernel(PackArgs a) {
    for (int64_t g = blockIdx.x * int64_t{kThreads} + threadIdx.x; g < a.groups; g += gridDim.x * int64_t{kThreads}) {
        const Place p = place_of(g, a.blocks, a.cols);
        if (p.n <= 0) continue;
        float x[8];
        restore8(a.kept, g, x);
        store8<kT>(a.x.p + p.row * a.x.stride + int64_t{p.col} * dtype_bytes(kT), p.n, false, x);
    }
}

struct GateArgs {
    Rows x, factor, out;  // backward: grad_x, grad_factor, grad_out
    Kept keep_x, keep_factor;
    int64_t groups;
    int32_t blocks, cols;
    int32_t far;
};

template <int kT, int kKind, bool kGated>
__global__ __launch_bounds__(kThreads) void gate_kernel(GateArgs a) {
    const bool far = a.far != 0;
    for (int64_t g = blockIdx.x * int64_t{kThreads} + threadIdx.x; g < a.groups; g += gridDim.x * int64_t{kThreads}) {
        const Place p = place_of(g, a.blocks, a.cols);
        const int64_t at = int64_t{p.col} * dtype_bytes(kT);
        float x[8], f[8], y[8], unused;
        uint32_t top_x, top_f;
        load8<kT>(a.x.p + p.row * a.x.stride + at, p.n, far, x, top_x);
        if (kGated) load8<kT>(a.factor.p + p.row * a.factor.stride + at, p.n, far, f, top_f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            activate<kT, kKind, false>(x[i], y[i], unused);
            if (kGated) y[i] *= f[i];
        }
        if (p.n > 0) store8<kT>(a.out.p + p.row * a.out.stride + at, p.n, far, y);
        if (a.keep_x.codes != nullptr) {
            u32x2 codes;
            uint32_t scale = encode8<kT>(x, top_x, codes);
            keep8(a.keep_x, g, far, codes, scale);
            if (kGated) {
                scale = encode8<kT>(f, top_f, codes);
                keep8(a.keep_factor, g, far, codes, scale);
            }
        }
    }
}

template <int kT, int kKind, bool kGated>
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(GateArgs a) {
    const bool far = a.far != 0;
    for (int64_t g = blockIdx.x * int64_t{kThreads} + threadIdx.x; g < a.groups; g += gridDim.x * int64_t{kThreads}) {
        const Place p = place_of(g, a.blocks, a.cols);
        if (p.n <= 0) continue;
        const int64_t at = int64_t{p.col} * dtype_bytes(kT);
        float dy[8], x[8], f[8], dx[8], df[8];
        uint32_t unused;
        load8<kT>(a.out.p + p.row * a.out.stride + at, p.n, far, dy, unused);
        restore8(a.keep_x, g, x);
        if (kGated) restore8(a.keep_factor, g, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y, slope;
            activate<kT, kKind, true>(x[i], y, slope);
            dx[i] = dy[i] * slope;
            if (kGated) {
                dx[i] *= f[i];
                df[i] = dy[i] * y;
            }
        }
        if (a.x.p != nullptr) store8<kT>(a.x.p + p.row * a.x.stride + at, p.n, far, dx);
        if (kGated && a.factor.p != nullptr) store8<kT>(a.factor.p + p.row * a.factor.stride + at, p.n, far, df);
    }
}

// ---- host -------------------------------------------------------------------------

Rows rows_of(const gockpt_matrix* m) {
    if (m == nullptr) return {nullptr, 0};
    return {static_cast<uint8_t*>(const_cast<void*>(m->data)),
            (m->rows > 1 ? m->stride : m->cols) * dtype_bytes(m->dtype)};
}

Kept kept_of(const gockpt_act8* a) {
    if (a == nullptr) return {nullptr, nullptr};
    return {static_cast<uint8_t*>(a->codes), static_cast<uint8_t*>(a->scales)};
}

int32_t blocks_of(int64_t cols) { return static_cast<int32_t>((cols + GOCKPT_ACT8_BLOCK - 1) / GOCKPT_ACT8_BLOCK); }

dim3 grid_of(int64_t groups) {
    return dim3(static_cast<uint32_t>(std::min<int64_t>((groups + kThreads - 1) / kThreads, int64_t{1} << 23)));
}

// The activation's loads and stores go past the caches where a matrix is larger
// than this (14000 x 11008: 208 us forward instead of 227, 199 back instead of
// 209); a smaller one's next reader finds it there.
constexpr int64_t kFarBytes = int64_t{96} << 20;
int32_t far(const gockpt_matrix* m) { return m->rows * m->cols * dtype_bytes(m->dtype) > kFarBytes; }

template <int kT, int kKind>
void start_gate(bool backward, bool gated, const GateArgs& a, hipStream_t s) {
    if (backward)
        hipLaunchKernelGGL((gated ? gate_grad_kernel<kT, kKind, true> : gate_grad_kernel<kT, kKind, false>),
                           grid_of(a.groups), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((gated ? gate_kernel<kT, kKind, true> : gate_kernel<kT, kKind, false>), grid_of(a.groups),
                           dim3(kThreads), 0, s, a);
}

template <int kT>
void start_gate_kind(int kind, bool backward, bool gated, const GateArgs& a, hipStream_t s) {
    if (kind == GOCKPT_SILU) return start_gate<kT, GOCKPT_SILU>(backward, gated, a, s);
    if (kind == GOCKPT_GELU) return start_gate<kT, GOCKPT_GELU>(backward, gated, a, s);
    start_gate<kT, GOCKPT_GELU_TANH>(backward, gated, a, s);
}

void launch_gate(int dtype, int kind, bool backward, bool gated, const GateArgs& a, hipStream_t s) {
    if (dtype == kBF16) return start_gate_kind<kBF16>(kind, backward, gated, a, s);
    if (dtype == kFP16) return start_gate_kind<kFP16>(kind, backward, gated, a, s);
    start_gate_kind<kFP32>(kind, backward, gated, a, s);
}

// A second matrix of a call: of the first one's type and size.
int check_like(const char* name, const char* what, const gockpt_matrix* m, const char* first, const gockpt_matrix* f) {
    const int rc = check_model_matrix(name, what, m, kAnyType);
    if (rc != GOCKPT_OK) return rc;
    if (m->dtype != f->dtype || m->rows != f->rows || m->cols != f->cols)
        return ops_fail(GOCKPT_EINVAL, "%s: %s of %lld x %lld, dtype %d, for %s of %lld x %lld, dtype %d", name, what,
                        static_cast<long long>(m->rows), static_cast<long long>(m->cols), m->dtype, first,
                        static_cast<long long>(f->rows), static_cast<long long>(f->cols), f->dtype);
    return GOCKPT_OK;
}

int check_kind(const char* name, int kind) {
    if (kind < GOCKPT_SILU || kind > GOCKPT_GELU_TANH) return ops_fail(GOCKPT_EINVAL, "%s: kind %d", name, kind);
    return GOCKPT_OK;
}

}  // namespace

int pack_and_copy(const char* name, const gockpt_matrix* x, const gockpt_act8* out, uint8_t* copy, hipStream_t s) {
    int rc = check_model_matrix(name, "x", x, kAnyType);
    if (rc == GOCKPT_OK) rc = check_act8(name, "out", out, x->rows, x->cols);
    if (rc != GOCKPT_OK || x->rows == 0 || x->cols == 0) return rc;
    PackArgs a{rows_of(x), Rows{copy, copy_stride(x->cols) * 2}, kept_of(out), x->rows * blocks_of(x->cols) * 4,
               blocks_of(x->cols), static_cast<int32_t>(x->cols)};
    auto kernel = x->dtype == kBF16 ? pack_kernel<kBF16> : x->dtype == kFP16 ? pack_kernel<kFP16> : pack_kernel<kFP32>;
    hipLaunchKernelGGL(kernel, grid_of(a.groups), dim3(kThreads), 0, s, a);
    return ops_launched(name);
}

}  // namespace gockpt

using namespace gockpt;

extern "C" {

int gockpt_act8_pack(const gockpt_matrix* x, const gockpt_act8* out, void* stream) {
    return pack_and_copy("gockpt_act8_pack", x, out, nullptr, static_cast<hipStream_t>(stream));
}

int gockpt_act8_unpack(const gockpt_act8* x, const gockpt_matrix* out, void* stream) {
    const char* name = "gockpt_act8_unpack";
    int rc = check_model_matrix(name, "out", out, kAnyType);
    if (rc == GOCKPT_OK) rc = check_act8(name, "x", x, out->rows, out->cols);
    if (rc != GOCKPT_OK || out->rows == 0 || out->cols == 0) return rc;
    PackArgs a{rows_of(out), Rows{}, kept_of(x), out->rows * blocks_of(out->cols) * 4, blocks_of(out->cols),
               static_cast<int32_t>(out->cols)};
    auto kernel = out->dtype == kBF16 ? unpack_kernel<kBF16>
                                      : out->dtype == kFP16 ? unpack_kernel<kFP16> : unpack_kernel<kFP32>;
    hipLaunchKernelGGL(kernel, grid_of(a.groups), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    return ops_launched(name);
}

int gockpt_gate8(int kind, const gockpt_matrix* x, const gockpt_matrix* factor, const gockpt_matrix* out,
                 const gockpt_act8* keep_x, const gockpt_act8* keep_factor, void* stream) {
    const char* name = "gockpt_gate8";
    int rc = check_kind(name, kind);
    if (rc == GOCKPT_OK) rc = check_model_matrix(name, "x", x, kAnyType);
    if (rc == GOCKPT_OK && factor != nullptr) rc = check_like(name, "factor", factor, "x", x);
    if (rc == GOCKPT_OK) rc = check_like(name, "out", out, "x", x);
    if (rc == GOCKPT_OK && keep_x != nullptr) rc = check_act8(name, "keep_x", keep_x, x->rows, x->cols);
    if (rc == GOCKPT_OK && keep_factor != nullptr) rc = check_act8(name, "keep_factor", keep_factor, x->rows, x->cols);
    if (rc == GOCKPT_OK && (keep_factor != nullptr) != (keep_x != nullptr && factor != nullptr))
        rc = ops_fail(GOCKPT_EINVAL, "%s: keep_x and keep_factor do not go with x and factor", name);
    if (rc != GOCKPT_OK || x->rows == 0 || x->cols == 0) return rc;
    const GateArgs a{rows_of(x),
                     rows_of(factor),
                     rows_of(out),
                     kept_of(keep_x),
                     kept_of(keep_factor),
                     x->rows * blocks_of(x->cols) * 4,
                     blocks_of(x->cols),
                     static_cast<int32_t>(x->cols),
                     far(x)};
    launch_gate(x->dtype, kind, false, factor != nullptr, a, static_cast<hipStream_t>(stream));
    return ops_launched(name);
}

int gockpt_gate8_grad(int kind, const gockpt_matrix* grad_out, const gockpt_act8* keep_x,
                      const gockpt_act8* keep_factor, const gockpt_matrix* grad_x, const gockpt_matrix* grad_factor,
                      void* stream) {
    const char* name = "gockpt_gate8_grad";
    int rc = check_kind(name, kind);
    if (rc == GOCKPT_OK) rc = check_model_matrix(name, "grad_out", grad_out, kAnyType);
    if (rc == GOCKPT_OK) rc = check_act8(name, "keep_x", keep_x, grad_out->rows, grad_out->cols);
    if (rc == GOCKPT_OK && keep_factor != nullptr)
        rc = check_act8(name, "keep_factor", keep_factor, grad_out->rows, grad_out->cols);
    if (rc == GOCKPT_OK && grad_x != nullptr) rc = check_like(name, "grad_x", grad_x, "grad_out", grad_out);
    if (rc == GOCKPT_OK && grad_factor != nullptr)
        rc = check_like(name, "grad_factor", grad_factor, "grad_out", grad_out);
    if (rc == GOCKPT_OK && grad_factor != nullptr && keep_factor == nullptr)
        rc = ops_fail(GOCKPT_EINVAL, "%s: grad_factor without keep_factor", name);
    if (rc != GOCKPT_OK || grad_out->rows == 0 || grad_out->cols == 0) return rc;
    if (grad_x == nullptr && grad_factor == nullptr) return GOCKPT_OK;
    const GateArgs a{rows_of(grad_x),
                     rows_of(grad_factor),
                     rows_of(grad_out),
                     kept_of(keep_x),
                     kept_of(keep_factor),
                     grad_out->rows * blocks_of(grad_out->cols) * 4,
                     blocks_of(grad_out->cols),
                     static_cast<int32_t>(grad_out->cols),
                     far(grad_out)};
    launch_gate(grad_out->dtype, kind, true, keep_factor != nullptr, a, static_cast<hipStream_t>(stream));
    return ops_launched(name);
}

}  // extern "C"
