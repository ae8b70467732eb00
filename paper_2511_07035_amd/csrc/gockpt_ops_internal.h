// gockpt_ops_internal.h -- element types and errors shared by the operators of
// gockpt_ops.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <string>

#include "../../include/gockpt_ops.h"
#include "gockpt_contract.h"

namespace gockpt {

void set_host_error(const std::string& msg);

// Status `rc` with its text for gockpt_last_error(NULL).  A failure to hold
// the text (memory) leaves the status alone to tell.
__attribute__((format(printf, 2, 3))) inline int ops_fail(int rc, const char* fmt, ...) noexcept {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        set_host_error(buf);
    } catch (...) {
    }
    return rc;
}

// The status of the kernels launched so far by the call `name`.
inline int ops_launched(const char* name) noexcept {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GOCKPT_OK : ops_fail(GOCKPT_EHIP, "%s: %s", name, hipGetErrorString(e));
}

enum DType : int { kBF16 = GOCKPT_BF16, kFP16 = GOCKPT_FP16, kFP32 = GOCKPT_FP32 };

constexpr bool dtype_ok(int t) { return t == kBF16 || t == kFP16 || t == kFP32; }
constexpr int dtype_bytes(int t) { return t == kFP32 ? 4 : 2; }

inline bool elem_aligned(const void* p, int dtype) {
    return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(dtype_bytes(dtype)) == 0;
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Vectors at any 2-byte address.  gfx950 loads and stores 8 and 16 bytes at
// any alignment in one instruction, so rows of odd length and tensors that
// start anywhere in a flat buffer take the same path as aligned ones.
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <int kT>
__device__ __forceinline__ float elem_to_f32(uint32_t bits) {
    if constexpr (kT == kFP32)
        return __uint_as_float(bits);
    else if constexpr (kT == kFP16)
        return fp16_to_f32(static_cast<uint16_t>(bits));
    else
        return bf16_to_f32(static_cast<uint16_t>(bits));
}

// Two fp32 values to two 16-bit ones in a word, to nearest even, in hardware
// for bf16 (v_cvt_pk_bf16_f32; a NaN stays a NaN); fp16 values too large
// become infinities.
template <int kT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    static_assert(kT != kFP32, "16-bit types");
    const f32x2 x = {a, b};
    if constexpr (kT == kFP16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// One element at p from fp32.
template <int kT>
__device__ __forceinline__ void store_elem(uint8_t* p, float x) {
    if constexpr (kT == kFP32)
        *reinterpret_cast<float*>(p) = x;
    else
        *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(pack2<kT>(x, x));
}

}  // namespace gockpt
