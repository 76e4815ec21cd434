// What the kernels of the feed-forward block share: operands, results, the activations and the end of a product.
#pragma once
#include "../../include/rsh_spmm.h"
#include "mx4.hpp"

namespace rsh {

// How an operand lies in memory.
enum Form {
    kAlong,     // k along memory: row i at i * ld
    kAcross,    // k across memory: k at k * ld
    kCodes,     // blocks of codes and their scales, k along memory; turned into 16 bits on the way into LDS
    kFours      // the same, multiplied as it is
};

struct Operand {
    const void* data[2];           // two matrices of equal shape (gate and up), or one
    const uint8_t* scales[2];
    int64_t ld;                    // elements (kAlong, kAcross) or blocks (kCodes, kFours) from row to row
    int64_t ld_scales;             // bytes from row to row of the scales
};

enum Act { kSilu = RSH_ACT_SILU, kGelu = RSH_ACT_GELU, kRelu = RSH_ACT_RELU };

struct Result {
    uint16_t* out[2];              // C, or H; [1]: the second of two results that share P (dWu)
    uint16_t* gate;                // G and U where they are wanted, kept four by four (keep4)
    uint16_t* up;
    int64_t ld, ld_gate;
    int act;
};

// act(g) and its derivative.  silu: g s with s = 1 / (1 + exp(-g)); gelu: g times the normal distribution function.
__device__ __forceinline__ float act_of(int act, float g) {
    if (act == kSilu) return g / (1.f + __expf(-g));
    if (act == kGelu) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    return g * (g > 0.f ? 1.f : 0.f);
}
__device__ __forceinline__ float act_of(int act, float g, float* slope) {
    if (act == kSilu) {
        const float s = 1.f / (1.f + __expf(-g));
        *slope = s * (1.f + g * (1.f - s));
        return g * s;
    }
    if (act == kGelu) {
        const float c = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        *slope = c + g * __expf(-0.5f * g * g) * 0.3989422804014327f;
        return g * c;
    }
    *slope = g > 0.f ? 1.f : 0.f;
    return g * *slope;
}

// G and U as they are kept for the gradients: four numbers in the 8 bytes that four of 16 bits take, 14 bits each and the exponent e
// of the largest.  A number is the middle of one of 8191 steps up to 2^(e - 126), or as many below zero, or zero itself: half a step
// off at most, and never across zero, on which relu's slope hangs.  In bfloat16 G and U alone would bring as much error into the
// gradients as those get by being rounded themselves (on a normal X, Wg and Wu 0.0031 of a gradient's size in all, 0.0023 so kept).
// Four in which one is an infinity or a NaN have exponent 255 and are fp32 without the last 18 bits.
constexpr float kKeptSteps = 8191.f / 8192.f;
constexpr int kKeptZero = -8192;
__device__ __forceinline__ uint2_t keep4(float4_t x) {
    uint32_t m = 0, b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        b[i] = __float_as_uint(x[i]);
        m = max(m, b[i] & 0x7fffffffu);
    }
    uint32_t e = m >> 23, f[4];
    if (e == 255u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[i] != x[i] ? 0x1fffu : b[i] >> 18;
    } else {
        e = max(e, 13u);
        const float scale = __uint_as_float((266u - e) << 23) * kKeptSteps;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (uint32_t)(x[i] == 0.f ? kKeptZero : (int)floorf(x[i] * scale)) & 0x3fffu;
    }
    return (uint2_t){f[0] | f[1] << 14 | f[2] << 28, f[2] >> 4 | f[3] << 10 | e << 24};
}
__device__ __forceinline__ float4_t kept4(uint2_t v) {
    const uint32_t lo = v[0], hi = v[1], e = hi >> 24;
    const uint32_t f[4] = {lo & 0x3fffu, lo >> 14 & 0x3fffu, lo >> 28 | (hi << 4 & 0x3ff0u), hi >> 10 & 0x3fffu};
    const float scale = __uint_as_float((max(e, 13u) - 12u) << 23) * (1.f / kKeptSteps);
    float4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int step = (int)(f[i] << 18) >> 18;
        x[i] = e == 255u ? __uint_as_float(f[i] << 18) : step == kKeptZero ? 0.f : ((float)step + 0.5f) * scale;
    }
    return x;
}

// What becomes of the sums of four columns of a row.
template <class T, bool GATED>
__device__ __forceinline__ void finish(const Result& res, uint16_t* out, int64_t row, int64_t col, int64_t left, float4_t x, float4_t y) {
    if constexpr (GATED) {
        if (res.gate) {        // rows of whole fours
#pragma unroll
            for (int v = 1; v < 4; ++v)
                if (v >= left) x[v] = y[v] = 0.f;
            *reinterpret_cast<uint2_t*>(res.gate + row * res.ld_gate + col) = keep4(x);
            *reinterpret_cast<uint2_t*>(res.up + row * res.ld_gate + col) = keep4(y);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = act_of(res.act, x[v]) * y[v];
    }
    store4(out + row * res.ld + col, (uint2_t){T::pair(x[0], x[1]), T::pair(x[2], x[3])}, left);
}

// Whether the kernel for few rows (few.hip) takes a product, and its launch.  Operands as for the tiles (ffn.hip); P is kAlong,
// kCodes or kFours, Q kAlong or, beside kFours, kFours.
bool takes_few(int64_t rows);
template <class T, Form FP, bool GATED>
void launch_few(const Operand& P, const Operand& Q, const Result& res, int64_t rows, int64_t cols, int64_t k, hipStream_t st);

}  // namespace rsh
