// Element types of the dense feed-forward kernels, and microscaled 4-bit floating point on the device.
//
// A row of a 4-bit matrix is blocks of 32 elements; a block has one scale byte s (2^(s - 127), 255: NaN) and 16 bytes of codes,
// the even element of a byte in its low bits: sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.  The conversions of gfx950 take the
// scale as the exponent field of a float, byte 0 included (2^-127), and keep every value exactly; binary16 results are rounded.
#pragma once
#include "device.hpp"

namespace rsh {

typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef int int8v_t __attribute__((ext_vector_type(8)));

constexpr int kBlock = 32;         // elements that share a scale
constexpr int kBlockBytes = 16;    // their codes

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

struct F16 {
    static __device__ __forceinline__ float16_t mfma32(uint4_t a, uint4_t b, float16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma16(uint4_t a, uint4_t b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float widen(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint32_t pair(float a, float b) {
        return __builtin_bit_cast(uint32_t, (half2_t){(_Float16)a, (_Float16)b});
    }
    template <int SEL>
    static __device__ __forceinline__ uint32_t from_codes(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
    }
};

struct BF16 {
    static __device__ __forceinline__ float16_t mfma32(uint4_t a, uint4_t b, float16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma16(uint4_t a, uint4_t b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint32_t pair(float a, float b) {
        return __builtin_bit_cast(uint32_t, (bf2_t){(__bf16)a, (__bf16)b});
    }
    template <int SEL>
    static __device__ __forceinline__ uint32_t from_codes(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
    }
};

// Eight codes as eight elements.
template <class T>
__device__ __forceinline__ uint4_t from_codes8(uint32_t codes, float scale) {
    return (uint4_t){T::template from_codes<0>(codes, scale), T::template from_codes<1>(codes, scale), T::template from_codes<2>(codes, scale),
                     T::template from_codes<3>(codes, scale)};
}

// Eight elements of a row from p, of which `valid` exist (any number); the others are zero.  Any alignment of the element's.
__device__ __forceinline__ uint4_t load8(const uint16_t* p, int64_t valid) {
    if (valid >= 8) return *reinterpret_cast<const uint4_a2*>(p);
    uint4_t v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < valid) v[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
}

// Four finished elements of a row, of which `valid` exist.
__device__ __forceinline__ void store4(uint16_t* p, uint2_t v, int64_t valid) {
    if (valid >= 4) {
        *reinterpret_cast<uint2_a2*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < valid) p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
    }
}

}  // namespace rsh
