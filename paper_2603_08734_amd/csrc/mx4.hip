// Quantisation of matrices to microscaled 4-bit floating point, and back.  Passes over the matrix, bound by memory.
//
// A lane has eight elements, four lanes a block: their largest exponent goes round the four lanes and each turns its eight
// elements into four bytes of codes with the conversions of gfx950, which round to nearest, ties to the even code, and hold 6
// for anything above.  The scale is the power of two that brings the largest element into [4, 8): its exponent field less two,
// and the largest exponent field is the largest bit pattern's, so neither a logarithm nor a sum is taken.  A block of zeros (or
// of numbers below 2^-125) has the smallest scale; one with an infinity or a NaN has scale 255 and codes 0.
// Measured: 28672 x 8192 bfloat16 to 4 bits and back 219 us, 1.19 GB at 5.4 TB/s, above a copy's 5.1; 1999 x 4999 fp32 18.6 us (8.8
// and 10.9 of it in the kernels); one row of 8192 1.7 us each way.
#include "mx4.hpp"

#include <algorithm>

#include "../../include/rsh_spmm.h"

namespace rsh {

namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 4;      // pieces of eight elements that a thread has in flight

// Largest of v over the four lanes of a block.
__device__ __forceinline__ uint32_t max_of_four(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));   // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));   // lanes 2 3 0 1
}

// By value: a bit cast of a vector's element itself takes the first one.
template <class P>
__device__ __forceinline__ P as_pair(uint32_t w) { return __builtin_bit_cast(P, w); }

struct Loaded {
    uint4_t lo, hi;    // hi: the second half of eight fp32 elements
};

template <int TYPE>
__device__ __forceinline__ Loaded load_piece(const void* X, int64_t at, int64_t valid) {
    Loaded r = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if constexpr (TYPE == RSH_F32) {
        const uint32_t* p = (const uint32_t*)X + at;
        if (valid >= 8) {
            r.lo = *reinterpret_cast<const uint4_a4*>(p);
            r.hi = *reinterpret_cast<const uint4_a4*>(p + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < valid) (i < 4 ? r.lo : r.hi)[i & 3] = p[i];
        }
    } else {
        r.lo = load8((const uint16_t*)X + at, valid);
    }
    return r;
}

// The exponent field that the largest magnitude among the eight elements has as an fp32 number.
template <int TYPE>
__device__ __forceinline__ uint32_t top_exponent(const Loaded& x) {
    uint32_t m = 0;
    if constexpr (TYPE == RSH_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(x.lo[i] & 0x7fffffffu, x.hi[i] & 0x7fffffffu));
        return m >> 23;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(x.lo[i] & 0x7fffu, x.lo[i] >> 16 & 0x7fffu));
        if constexpr (TYPE == RSH_BF16) return m >> 7;
        if (m >= 0x7c00u) return 255u;
        return __float_as_uint(F16::widen((uint16_t)m)) >> 23;
    }
}

template <int TYPE>
__device__ __forceinline__ uint32_t to_codes(const Loaded& x, float scale) {
    uint32_t c = 0;
    if constexpr (TYPE == RSH_F32) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.lo[0]), __uint_as_float(x.lo[1]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.lo[2]), __uint_as_float(x.lo[3]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.hi[0]), __uint_as_float(x.hi[1]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.hi[2]), __uint_as_float(x.hi[3]), scale, 3);
    } else if constexpr (TYPE == RSH_F16) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, as_pair<half2_t>(x.lo[0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, as_pair<half2_t>(x.lo[1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, as_pair<half2_t>(x.lo[2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, as_pair<half2_t>(x.lo[3]), scale, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair<bf2_t>(x.lo[0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair<bf2_t>(x.lo[1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair<bf2_t>(x.lo[2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair<bf2_t>(x.lo[3]), scale, 3);
    }
    return c;
}

// Where piece i of the matrix lies: pieces count through the blocks of a row, four a block, then through the rows.  WHOLE: rows
// are whole blocks without gaps, so a piece lies where its number says.
template <bool WHOLE>
struct Place {
    int64_t at;        // element in memory
    int64_t valid;     // elements that exist
    __device__ __forceinline__ Place(int64_t i, int64_t pieces, int64_t k, int64_t ld) {
        if constexpr (WHOLE) {
            at = 8 * i;
            valid = 8;
        } else {
            const int64_t row = (uint64_t)pieces < (1ull << 32) && (uint64_t)i < (1ull << 32) ? (int64_t)((uint32_t)i / (uint32_t)pieces) : i / pieces;
            const int64_t first = 8 * (i - row * pieces);
            at = row * ld + first;
            valid = k - first;
        }
    }
};

}  // namespace

template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rsh_mx4_quantize_kernel(const void* __restrict__ X, uint32_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales, int64_t n, int64_t pieces, int64_t k, int64_t ld) {
    const int64_t first = (int64_t)blockIdx.x * (kThreads * kTurns) + threadIdx.x;
    Loaded x[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t i = first + u * kThreads;
        const Place<WHOLE> p(i, pieces, k, ld);
        x[u] = load_piece<TYPE>(X, p.at, i < n ? p.valid : 0);
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t i = first + u * kThreads;
        const uint32_t e = max_of_four(top_exponent<TYPE>(x[u]));
        const uint32_t s = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
        const uint32_t c = e == 255u ? 0u : to_codes<TYPE>(x[u], scale_of(s));
        if (i < n) {       // n is a multiple of four: a block's lanes are all in or all out
            codes[i] = c;
            if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)s;
        }
    }
}

template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rsh_mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                      void* __restrict__ Y, int64_t n, int64_t pieces, int64_t k, int64_t ld) {
    const int64_t first = (int64_t)blockIdx.x * (kThreads * kTurns) + threadIdx.x;
    uint32_t c[kTurns], s[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t i = min(first + u * kThreads, n - 1);
        c[u] = codes[i];
        s[u] = scales[i >> 2];
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t i = first + u * kThreads;
        if (i >= n) break;
        const Place<WHOLE> p(i, pieces, k, ld);
        const float scale = scale_of(s[u]);
        if constexpr (TYPE == RSH_F32) {
            const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 1);
            const float2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 3);
            float* const y = (float*)Y + p.at;
            if (p.valid >= 8) {
                *reinterpret_cast<float4_a4*>(y) = (float4_t){a[0], a[1], b[0], b[1]};
                *reinterpret_cast<float4_a4*>(y + 4) = (float4_t){d[0], d[1], e[0], e[1]};
            } else {
                const float v[8] = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < p.valid) y[j] = v[j];
            }
        } else {
            using T = std::conditional_t<TYPE == RSH_F16, F16, BF16>;
            const uint4_t v = from_codes8<T>(c[u], scale);
            uint16_t* const y = (uint16_t*)Y + p.at;
            if (p.valid >= 8) {
                *reinterpret_cast<uint4_a2*>(y) = v;
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < p.valid) y[j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
            }
        }
    }
}

namespace {
int launched() { return hipGetLastError() == hipSuccess ? RSH_OK : RSH_ERR_HIP; }

// Pieces of a row, workgroups for all of them, and whether the pieces of the matrix lie one behind the other.
struct Cover {
    int64_t pieces, n;
    unsigned blocks;
    bool whole;
    Cover(int64_t rows, int64_t k, int64_t ld)
        : pieces((k + kBlock - 1) / kBlock * 4), n(rows * pieces), blocks((unsigned)((n + kThreads * kTurns - 1) / (kThreads * kTurns))),
          whole(k % kBlock == 0 && (ld == k || rows == 1)) {}
};

template <class F>
void by_type(int type, bool whole, F f) {
    auto pick = [&](auto w) {
        if (type == RSH_F32) f(std::integral_constant<int, RSH_F32>(), w);
        else if (type == RSH_F16) f(std::integral_constant<int, RSH_F16>(), w);
        else f(std::integral_constant<int, RSH_BF16>(), w);
    };
    if (whole) pick(std::true_type());
    else pick(std::false_type());
}
}  // namespace

int launch_mx4_quantize(const void* X, int type, int64_t rows, int64_t k, int64_t ld, void* codes, void* scales, void* stream) {
    const Cover c(rows, k, ld);
    by_type(type, c.whole, [&](auto t, auto w) {
        hipLaunchKernelGGL((rsh_mx4_quantize_kernel<decltype(t)::value, decltype(w)::value>), dim3(c.blocks), dim3(kThreads), 0, (hipStream_t)stream,
                           X, (uint32_t*)codes, (uint8_t*)scales, c.n, c.pieces, k, ld);
    });
    return launched();
}

int launch_mx4_dequantize(const void* codes, const void* scales, int64_t rows, int64_t k, void* Y, int type, int64_t ld, void* stream) {
    const Cover c(rows, k, ld);
    by_type(type, c.whole, [&](auto t, auto w) {
        hipLaunchKernelGGL((rsh_mx4_dequantize_kernel<decltype(t)::value, decltype(w)::value>), dim3(c.blocks), dim3(kThreads), 0, (hipStream_t)stream,
                           (const uint32_t*)codes, (const uint8_t*)scales, Y, c.n, c.pieces, k, ld);
    });
    return launched();
}

}  // namespace rsh
