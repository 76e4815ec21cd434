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

// Eight elements as they lie in memory.
template <class T>
struct Raw {
    uint4_t v[size_of<T>() / 2];
};
template <class T>
__device__ __forceinline__ Eight widen(const Raw<T>& r) {
    if constexpr (std::is_same<T, F32>::value) {
        Eight e;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = r.v[i / 4][i % 4];
            e.v[i] = __uint_as_float(w);
        }
        return e;
    } else {
        return widen8<T>(r.v[0]);
    }
}

// Byte `at` of a row whose address is alike in all lanes.  Loops over rows would otherwise have the sums ready, two registers for every
// vector and run, and an access would no longer have its address in scalar registers and an offset.
__device__ __forceinline__ const uint8_t* byte_of(const void* row, uint32_t at) {
    asm volatile("" : "+v"(at));
    return (const uint8_t*)row + at;
}

// Elements col .. col + 7 of a row of d, to be settled before they are used.  Every lane makes the same whole loads, the last of a row that
// is no multiple of eight from where the row's last eight lie: a load under a condition of its own would have to arrive before the two
// ways meet again, and one whose result is looked at here before the next goes out.  SHORT: the row may have less than eight.
template <class T, bool SHORT>
__device__ __forceinline__ Raw<T> load_raw(const void* row, int col, int d) {
    constexpr int N = size_of<T>() / 2;
    Raw<T> r = {};
    if (SHORT && d < 8) {
        if constexpr (std::is_same<T, F32>::value) {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (col + i < d) r.v[i / 4][i % 4] = ((const uint32_t*)row)[col + i];
        } else {
            r.v[0] = load8((const uint16_t*)row + col, d - col);
        }
        return r;
    }
    const uint8_t* const p = byte_of(row, (uint32_t)min(col, d - 8) * (uint32_t)size_of<T>());
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (std::is_same<T, F32>::value) r.v[i] = *reinterpret_cast<const uint4_a4*>(p + 16 * i);
        else r.v[i] = *reinterpret_cast<const uint4_a2*>(p);
    }
    return r;
}
// The same in their places, zeros from d on, and nothing but zeros in a lane that is not `live`.
template <class T, bool SHORT>
__device__ __forceinline__ Raw<T> settle(Raw<T> r, int col, int d, bool live = true) {
    constexpr int N = size_of<T>() / 2;
    if ((d & 7) && !(SHORT && d < 8)) {
        const int past = min(max(col - (d - 8), 0), 8);
        if (past) {
            if constexpr (std::is_same<T, F32>::value) {
                if (past & 4) r.v[0] = r.v[1], r.v[1] = (uint4_t){0, 0, 0, 0};
                if (past & 2) r.v[0] = (uint4_t){r.v[0][2], r.v[0][3], r.v[1][0], r.v[1][1]}, r.v[1] = (uint4_t){r.v[1][2], r.v[1][3], 0, 0};
                if (past & 1) r.v[0] = (uint4_t){r.v[0][1], r.v[0][2], r.v[0][3], r.v[1][0]}, r.v[1] = (uint4_t){r.v[1][1], r.v[1][2], r.v[1][3], 0};
            } else {
                uint4_t x = r.v[0];
                if (past & 4) x = (uint4_t){x[2], x[3], 0, 0};
                if (past & 2) x = (uint4_t){x[1], x[2], x[3], 0};
                if (past & 1) x = (uint4_t){x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
                r.v[0] = x;
            }
        }
    }
    const bool in = live && col < d;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) r.v[i][w] = in ? r.v[i][w] : 0u;
    return r;
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

// Dropout's random numbers: Philox4x32 of ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011).  Eight elements of a row share a block: 16 bits each, the low half of a word before its high half.  The counter is (place of
// the eight in the row, row, both halves of the offset), the key the seed's halves: an element's bits depend on nothing else, so the
// backward pass draws them again and no mask is stored.  A product of 32 by 32 bits is a multiplication at a quarter of the rate, 20
// of them a block: 16 bits an element keep that below what the memory takes.
struct Random {
    uint32_t k0, k1, c2, c3, share;
    float keep;        // what is kept is multiplied by it: 1 / (1 - share / 65536); with nothing kept 1, which nothing is multiplied by
    __device__ __forceinline__ Random(const rsh_drop_t& d) {
        const uint64_t seed = d.seed_dev && d.share ? *d.seed_dev : d.seed;
        k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32), c2 = (uint32_t)d.offset, c3 = (uint32_t)(d.offset >> 32), share = d.share;
        keep = share < 65536u ? 65536.f / (float)(65536u - share) : 1.f;
    }
    __device__ __forceinline__ uint4_t bits(uint32_t place, uint32_t row) const {
        asm volatile("" : "+v"(place));       // its first product is not kept from row to row
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
    // Whether element i of a block is kept.  share << 16 fits 32 bits but for its last value, so less one; share 0 is nothing to drop.
    __device__ __forceinline__ bool keeps(const uint4_t& r, int i) const { return (i & 1 ? r[i / 2] : r[i / 2] << 16) > (share << 16) - 1u; }
    // Bit i: element col + i is kept.
    __device__ __forceinline__ uint32_t kept(int col, int64_t row) const {
        const uint4_t r = bits((uint32_t)col / 8, (uint32_t)row);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m |= keeps(r, i) ? 1u << i : 0u;
        return m;
    }
    // What is dropped becomes zero, infinities and NaN too; what is kept is multiplied by `factor`.
    __device__ __forceinline__ void drop(Eight& e, int col, int64_t row, float factor) const {
        const uint4_t r = bits((uint32_t)col / 8, (uint32_t)row);
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = keeps(r, i) ? e.v[i] * factor : 0.f;
    }
};

}  // namespace rsh
