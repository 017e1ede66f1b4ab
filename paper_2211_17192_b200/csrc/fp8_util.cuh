// Rows in 8 bits with a scale: what the kernels that write them have in common.
//
// A row y is held as codes c and one fp32 scale s, value = c * s.  With a = max |y|: s = 1 for a row of zeros, else a times the
// rounded reciprocal of 448 (e4m3: the largest code) or of 127 (int8), as an elementwise program divides by a constant, and not
// below 2^-80: 1 / s stays finite and a product of two scales too.
// c = y * (1 / s) rounded to the nearest code, ties to even; the one reciprocal per row instead of a division per element
// moves a code only where y / s lies within two roundings of a tie.  The maximum is taken of bit patterns, in which a NaN is
// the largest: a row with a NaN or an infinity in it has a scale that is none, and every value read back from it is NaN.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace spec {

constexpr float kE4m3Top = 448.0f, kInt8Top = 127.0f;
constexpr float kLeastScale = 0x1p-80f;

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ float row_scale(uint32_t largest, float top) {
    if (largest == 0u) return 1.0f;
    const float s = __fmul_rn(__uint_as_float(largest), 1.0f / top);
    return s < kLeastScale ? kLeastScale : s;  // (a NaN stays)
}

// Two codes, the first in the low byte.
__device__ __forceinline__ uint32_t codes_e4m3(float x, float y) {
    return __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t codes_int8(float x, float y) {
    const int a = max(-127, min(127, __float2int_rn(x))), b = max(-127, min(127, __float2int_rn(y)));
    return (a & 0xff) | ((b & 0xff) << 8);
}

__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(float v) { return v; }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// N elements from memory as fp32, and back; `wide`: the address is aligned to 16 bytes, or to all of them where they are fewer.
template <int N, typename T>
__device__ __forceinline__ void load_row(const T* p, bool wide, float (&v)[N]) {
    constexpr int kBytes = N * sizeof(T);
    __align__(16) T t[N];
    if (wide) {
        if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(t) = *reinterpret_cast<const uint2*>(p);
        else
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_float(t[i]);
}
template <int N, typename T>
__device__ __forceinline__ void store_row(T* p, bool wide, const float (&v)[N]) {
    constexpr int kBytes = N * sizeof(T);
    __align__(16) T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = from_float<T>(v[i]);
    if (wide) {
        if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(t);
        else
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = t[i];
    }
}

inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool float_dtype(int dtype) { return dtype == SPEC_DTYPE_FP32 || dtype == SPEC_DTYPE_BF16 || dtype == SPEC_DTYPE_FP16; }
inline int dtype_bytes(int dtype) { return dtype == SPEC_DTYPE_FP32 ? 4 : dtype == SPEC_DTYPE_E4M3 || dtype == SPEC_DTYPE_INT8 ? 1 : 2; }

}  // namespace spec
