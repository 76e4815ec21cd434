// Rows of fp32, binary16 or bfloat16 on the device, eight elements at a time, and the random bits of dropout.
#pragma once
#include "../../include/rsh_spmm.h"
#include "mx4.hpp"

namespace rsh {

struct Eight {
    float v[8];
};

struct F32 {
    static constexpr int kSize = 4;
};
template <class T> constexpr int size_of() { return 2; }
template <> constexpr int size_of<F32>() { return 4; }

template <class T>
__device__ __forceinline__ Eight widen8(uint4_t x) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = T::widen((uint16_t)(x[i / 2] >> (16 * (i & 1))));
    return e;
}

// Eight elements from element `at` on, of which `valid` exist (any number); the others are zero.  Any alignment of the element's.
template <class T>
__device__ __forceinline__ Eight load_eight(const void* base, int64_t at, int valid) {
    if constexpr (std::is_same<T, F32>::value) {
        const float* const p = (const float*)base + at;
        Eight e;
        if (valid >= 8) {
            const float4_t a = *reinterpret_cast<const float4_a4*>(p), b = *reinterpret_cast<const float4_a4*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) e.v[i] = a[i], e.v[4 + i] = b[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e.v[i] = i < valid ? p[i] : 0.f;
        }
        return e;
    } else {
        return widen8<T>(load8((const uint16_t*)base + at, valid));
    }
}

template <class T>
__device__ __forceinline__ void store_eight(void* base, int64_t at, const Eight& e, int valid) {
    if constexpr (std::is_same<T, F32>::value) {
        float* const p = (float*)base + at;
        if (valid >= 8) {
            *reinterpret_cast<float4_a4*>(p) = (float4_t){e.v[0], e.v[1], e.v[2], e.v[3]};
            *reinterpret_cast<float4_a4*>(p + 4) = (float4_t){e.v[4], e.v[5], e.v[6], e.v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < valid) p[i] = e.v[i];
        }
    } else {
        uint16_t* const p = (uint16_t*)base + at;
        const uint4_t x = {T::pair(e.v[0], e.v[1]), T::pair(e.v[2], e.v[3]), T::pair(e.v[4], e.v[5]), T::pair(e.v[6], e.v[7])};
        if (valid >= 8) {
            *reinterpret_cast<uint4_a2*>(p) = x;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < valid) p[i] = (uint16_t)(x[i / 2] >> (16 * (i & 1)));
        }
    }
}

// The same where the type is known at run time only, alike for the launch: parameters.
__device__ __forceinline__ Eight load_eight(int type, const void* base, int64_t at, int valid) {
    if (type == RSH_F32) return load_eight<F32>(base, at, valid);
    return type == RSH_F16 ? load_eight<F16>(base, at, valid) : load_eight<BF16>(base, at, valid);
}
__device__ __forceinline__ void store_eight(int type, void* base, int64_t at, const Eight& e, int valid) {
    if (type == RSH_F32) store_eight<F32>(base, at, e, valid);
    else if (type == RSH_F16) store_eight<F16>(base, at, e, valid);
    else store_eight<BF16>(base, at, e, valid);
}

// Dropout's random numbers: Philox4x32 of ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011).  Eight elements of a row share a block: 16 bits each, the low half of a word before its high half.  The counter is (place of
// the eight in the row, row, both halves of the offset), the key the seed's halves: an element's bits depend on nothing else, so the
// backward pass draws them again and no mask is stored.  A product of 32 by 32 bits is a multiplication at a quarter of the rate, 20
// of them a block: 16 bits an element keep that below what the memory takes.
struct Random {
    uint32_t k0, k1, c2, c3, share;
    float keep;        // what is kept is multiplied by it: 1 / (1 - share / 65536)
    __device__ __forceinline__ Random(const rsh_drop_t& d) {
        const uint64_t seed = d.seed_dev && d.share ? *d.seed_dev : d.seed;
        k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32), c2 = (uint32_t)d.offset, c3 = (uint32_t)(d.offset >> 32), share = d.share;
        keep = 65536.f / (float)(share < 65536u ? 65536u - share : 1u);
    }
    __device__ __forceinline__ uint4_t bits(uint32_t place, uint32_t row) const {
        uint32_t a = place, b = row, c = c2, d = c3, x = k0, y = k1;
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
            a = (uint32_t)(q >> 32) ^ b ^ x;
            b = (uint32_t)q;
            c = (uint32_t)(p >> 32) ^ d ^ y;
            d = (uint32_t)p;
            x += 0x9E3779B9u;
            y += 0xBB67AE85u;
        }
        return (uint4_t){a, b, c, d};
    }
    // What is dropped becomes zero, infinities and NaN too; what is kept is multiplied by `factor`.
    __device__ __forceinline__ void drop(Eight& e, int col, int64_t row, float factor) const {
        const uint4_t r = bits((uint32_t)col / 8, (uint32_t)row);
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (i & 1 ? r[i / 2] >> 16 : r[i / 2] & 0xffffu) >= share ? e.v[i] * factor : 0.f;
    }
};

}  // namespace rsh
