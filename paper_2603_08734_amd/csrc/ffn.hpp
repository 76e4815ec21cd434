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
    // G and U where they are wanted, as they were summed: binary16 does not have the range of a sum, bfloat16 would bring as much error
    // into the gradients as those get by being rounded themselves, and an exponent shared by neighbours loses the small ones.
    float* gate;
    float* up;
    int64_t ld, ld_gate;
    int act;
};

// max(g, 0), of NaN NaN.  (g times a truth value would make NaN of minus infinity.)
__device__ __forceinline__ float relu_of(float g) { return g < 0.f ? 0.f : g; }
// act(g) and its derivative.  silu: g s with s = 1 / (1 + exp(-g)); gelu: g times the normal distribution function.
__device__ __forceinline__ float act_of(int act, float g) {
    if (act == kSilu) return g / (1.f + __expf(-g));
    if (act == kGelu) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    return relu_of(g);
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
    return relu_of(g);
}

// What becomes of the sums of four columns of a row.
template <class T, bool GATED>
__device__ __forceinline__ void finish(const Result& res, uint16_t* out, int64_t row, int64_t col, int64_t left, float4_t x, float4_t y) {
    if constexpr (GATED) {
        if (res.gate) {        // rows of whole fours; nobody looks at what lies past the end
            *reinterpret_cast<float4_t*>(res.gate + row * res.ld_gate + col) = x;
            *reinterpret_cast<float4_t*>(res.up + row * res.ld_gate + col) = y;
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
