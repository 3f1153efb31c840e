// Elements of the sequence operators' matrices: float, IEEE binary16 or bfloat16, sixteen bytes at a time, at any element's address.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "tbe_device.h"

namespace tbe {

// Two floats rounded to nearest even into one word, the first in its lower half.
__device__ __forceinline__ uint32_t pack2(const __half*, const float a, const float b) {
    return (uint32_t)__half_as_ushort(__float2half_rn(a)) | (uint32_t)__half_as_ushort(__float2half_rn(b)) << 16;
}
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(const bf16_t*, const float a, const float b) {   // (one instruction on gfx950)
    f32x2_t x;
    x.x = a; x.y = b;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
}

template <typename T>
__device__ __forceinline__ float elem_float(T x);
template <>
__device__ __forceinline__ float elem_float(const float x) { return x; }
template <>
__device__ __forceinline__ float elem_float(const __half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float elem_float(const bf16_t x) { return bf16_to_float(x.bits); }
template <typename T>
__device__ __forceinline__ T elem_round(float x);
template <>
__device__ __forceinline__ float elem_round<float>(const float x) { return x; }
template <>
__device__ __forceinline__ __half elem_round<__half>(const float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ bf16_t elem_round<bf16_t>(const float x) { return bf16_t{float_to_bf16_rn(x)}; }

// one element of a vector whose type (TBE_IO_*) is known at run time only
__device__ __forceinline__ float param_load(const void* p, const int io, const int64_t i) {
    return io == 0 ? static_cast<const float*>(p)[i]
                   : (io == 1 ? __half2float(static_cast<const __half*>(p)[i]) : bf16_to_float(static_cast<const bf16_t*>(p)[i].bits));
}
__device__ __forceinline__ void param_store(void* p, const int io, const int64_t i, const float x) {
    if (io == 0) static_cast<float*>(p)[i] = x;
    else if (io == 1) static_cast<__half*>(p)[i] = __float2half_rn(x);
    else static_cast<bf16_t*>(p)[i].bits = float_to_bf16_rn(x);
}

// Sixteen bytes from an address that is a multiple of the element's size only: the memory path takes such addresses, so rows of
// odd lengths need no loads of single elements but at their end.
typedef uint32_t u32x4_a4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_a2_t __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
struct Frag {   // 16-bit types
    static constexpr int kN = 8;
    static __device__ __forceinline__ uint4 load(const T* p) {
        const u32x4_a2_t v = *reinterpret_cast<const u32x4_a2_t*>(p);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    static __device__ __forceinline__ void store(T* p, const float (&x)[8]) {
        u32x4_a2_t v;
        v.x = pack2(p, x[0], x[1]); v.y = pack2(p, x[2], x[3]);
        v.z = pack2(p, x[4], x[5]); v.w = pack2(p, x[6], x[7]);
        *reinterpret_cast<u32x4_a2_t*>(p) = v;
    }
    static __device__ __forceinline__ void unpack(const uint4 r, float (&x)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2 && __is_same(T, bf16_t)) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                x[2 * i] = __half2float(__ushort_as_half((unsigned short)(w[i] & 0xFFFFu)));
                x[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
            }
        }
    }
};
template <>
struct Frag<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ uint4 load(const float* p) {
        const u32x4_a4_t v = *reinterpret_cast<const u32x4_a4_t*>(p);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    static __device__ __forceinline__ void store(float* p, const float (&x)[4]) {
        u32x4_a4_t v;
        v.x = __float_as_uint(x[0]); v.y = __float_as_uint(x[1]);
        v.z = __float_as_uint(x[2]); v.w = __float_as_uint(x[3]);
        *reinterpret_cast<u32x4_a4_t*>(p) = v;
    }
    static __device__ __forceinline__ void unpack(const uint4 r, float (&x)[4]) {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y);
        x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
};

// Sum of p[i * stride] for i = first, first + step, ... below n: eight loads under way together, added in their order.
__device__ __forceinline__ float strided_sum(const float* __restrict__ p, const int64_t stride, int64_t first, const int64_t n, const int64_t step) {
    float s = 0.f;
    for (; first + 7 * step < n; first += 8 * step) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = p[(first + k * step) * stride];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[k];
    }
    for (; first < n; first += step) s += p[first * stride];
    return s;
}

}  // namespace tbe
