// The products of the feed-forward block for few rows (tokens): every weight is read once and multiplied with all of them, so the
// time is that of the weight's bytes.
//
// A wave has groups of 16 weight rows and takes every n-th step of k for them, n the waves of its workgroup; its weights go from
// memory straight into the registers that the matrix unit reads, next to 16 tokens' pieces of the same k.  Which k a lane has is
// free as long as both operands agree: lane (row r, quarter q) of 16 x 4 has 8 elements of 16 bits, or one whole block of 32 codes,
// whose four words then make four operands.  Several groups of rows share the tokens' pieces.  The waves' sums meet in LDS and are
// added in the waves' order.
#include <algorithm>

#include "ffn.hpp"

namespace rsh {

namespace {

constexpr int kWaves = 8;          // most waves of a workgroup

// Words of a lane in a step: U loads of 16 bytes a group of rows.
template <Form FP>
struct Step {
    static constexpr int kLoads = FP == kAlong ? 4 : FP == kCodes ? 2 : 4;
    static constexpr int kLoadK = FP == kAlong ? 32 : 128;       // k of a load of all four quarters
    static constexpr int kK = kLoads * kLoadK;
    static constexpr int kXLoads = FP == kCodes ? 4 * kLoads : kLoads;
};

// Binary16 beside codes: bfloat16 has every value of a code exactly, and two of it make a binary16 number.  A token has two columns
// of the sixteen, eight apart: one with the number rounded to bfloat16, one with what is left.
__device__ __forceinline__ uint4_t part_of(uint4_t x, bool rest) {
    uint4_t v;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t word = x[w];
        const float a = F16::widen((uint16_t)word), b = F16::widen((uint16_t)(word >> 16));
        const uint32_t head = BF16::pair(a, b);
        // the rest of an infinity is not a number: any finite one does
        const float ra = fmaxf(a - BF16::widen((uint16_t)head), -65504.f), rb = fmaxf(b - BF16::widen((uint16_t)(head >> 16)), -65504.f);
        v[w] = rest ? BF16::pair(ra, rb) : head;
    }
    return v;
}

}  // namespace

// T: type of the result, and of the operands of 16 bits.  GROUPS groups of 16 weight rows a wave (GATED: half of them of either
// matrix), TOKENS tiles of 16 columns: 16 tokens, or 8 beside codes in binary16.
template <class T, Form FP, bool GATED, int GROUPS, int TOKENS>
__global__ __launch_bounds__(64 * kWaves) void rsh_few_rows_kernel(Operand P, Operand Q, Result res, int64_t rows, int64_t cols, int64_t k) {
    constexpr bool kSplit = FP == kCodes && std::is_same<T, F16>::value;
    constexpr bool kFour = FP == kFours;
    constexpr int kOut = GATED ? GROUPS / 2 : GROUPS;      // groups of columns of the result
    constexpr int kTile = kSplit ? 8 : 16;                 // tokens of a tile
    using S = Step<FP>;
    using M = std::conditional_t<kSplit, BF16, T>;         // what the matrix unit multiplies
    __shared__ float4_t sums[kWaves][GROUPS * TOKENS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t first = (int64_t)blockIdx.x * (16 * kOut);

    // rows past the end read the last one; nobody keeps their sums
    const uint8_t* w[GROUPS];
    const uint8_t* ws[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int which = GATED ? g / kOut : 0;
        const int64_t row = min(first + 16 * (g % kOut) + r, cols - 1);
        w[g] = (const uint8_t*)P.data[which] + (FP == kAlong ? 2 * (row * P.ld + 8 * q) : (row * P.ld + q) * kBlockBytes);
        ws[g] = FP == kAlong ? nullptr : P.scales[which] + row * P.ld + q;
    }
    const uint8_t* x[TOKENS];
    const uint8_t* xs[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const int64_t row = min((int64_t)kTile * t + (kSplit ? r & 7 : r), rows - 1);
        x[t] = (const uint8_t*)Q.data[0] + (kFour ? (row * Q.ld + q) * kBlockBytes : 2 * (row * Q.ld + (FP == kCodes ? 32 : 8) * q));
        xs[t] = kFour ? Q.scales[0] + row * Q.ld + q : nullptr;
    }

    struct Pieces {
        uint4_t w[GROUPS][S::kLoads], x[TOKENS][S::kXLoads];
        uint32_t ws[GROUPS][FP == kAlong ? 1 : S::kLoads], xs[TOKENS][kFour ? S::kLoads : 1];
    };
    // WHOLE: the step ends within k
    auto load = [&](Pieces& p, int64_t k0, auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            const int64_t kk = k0 + j * S::kLoadK;       // of all quarters
            const bool block = kWhole || kk / kBlock + q < P.ld;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if constexpr (FP == kAlong) {
                    p.w[g][j] = load8((const uint16_t*)w[g] + kk, kWhole ? 8 : k - kk - 8 * q);
                } else {
                    p.w[g][j] = block ? *reinterpret_cast<const uint4_t*>(w[g] + kk / kBlock * kBlockBytes) : (uint4_t){0, 0, 0, 0};
                    p.ws[g][j] = block ? ws[g][kk / kBlock] : 0u;
                }
            }
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                if constexpr (kFour) {
                    p.x[t][j] = block ? *reinterpret_cast<const uint4_t*>(x[t] + kk / kBlock * kBlockBytes) : (uint4_t){0, 0, 0, 0};
                    p.xs[t][j] = block ? xs[t][kk / kBlock] : 0u;
                } else if constexpr (FP == kAlong) {
                    p.x[t][j] = load8((const uint16_t*)x[t] + kk, kWhole ? 8 : k - kk - 8 * q);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p.x[t][4 * j + i] = load8((const uint16_t*)x[t] + kk + 8 * i, kWhole ? 8 : k - kk - 32 * q - 8 * i);
                }
            }
        }
    };
    float4_t acc[GROUPS][TOKENS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) acc[g][t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Pieces& p) {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            if constexpr (kFour) {
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) {
                        const uint4_t a = p.w[g][j], b = p.x[t][j];
                        const int8v_t fa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, fb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
                        acc[g][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, acc[g][t], 4, 4, 0, p.ws[g][j], 0, p.xs[t][j]);
                    }
            } else if constexpr (FP == kAlong) {
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) acc[g][t] = M::mfma16(p.w[g][j], p.x[t][j], acc[g][t]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4_t b[TOKENS];
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) b[t] = kSplit ? part_of(p.x[t][4 * j + i], r >= 8) : p.x[t][4 * j + i];
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const uint4_t a = from_codes8<M>(p.w[g][j][i], scale_of(p.ws[g][j]));
#pragma unroll
                        for (int t = 0; t < TOKENS; ++t) acc[g][t] = M::mfma16(a, b[t], acc[g][t]);
                    }
                }
            }
        }
    };

    // The wave's whole steps, one in flight ahead; the step that ends past k, if there is one, is the workgroup's last.
    const int64_t steps = k / S::kK;
    Pieces now, next;
    if (wave < steps) {
        load(now, wave * S::kK, std::true_type());
        for (int64_t s = wave + waves; s < steps; s += waves) {
            load(next, s * S::kK, std::true_type());
            multiply(now);
            now = next;
        }
        multiply(now);
    }
    if (steps * S::kK < k && steps % waves == wave) {
        load(now, steps * S::kK, std::false_type());
        multiply(now);
    }

#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[wave][g * TOKENS + t][lane] = acc[g][t];
    __syncthreads();
    // A lane has rows 4 q .. 4 q + 3 of the group for token r.
    for (int i = wave; i < kOut * TOKENS; i += waves) {
        const int g = i / TOKENS, t = i % TOKENS;
        float4_t a = {0.f, 0.f, 0.f, 0.f}, b = a;
        for (int v = 0; v < waves; ++v) {
            a += sums[v][g * TOKENS + t][lane];
            if constexpr (GATED) b += sums[v][(g + kOut) * TOKENS + t][lane];
        }
        if constexpr (kSplit) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                a[v] += __int_as_float(swap_lane8(__float_as_int(a[v])));
                if constexpr (GATED) b[v] += __int_as_float(swap_lane8(__float_as_int(b[v])));
            }
        }
        const int64_t row = kTile * t + r, col = first + 16 * g + 4 * q;
        if (r < kTile && row < rows && col < cols) finish<T, GATED>(res, res.out[0], row, col, cols - col, a, b);
    }
}

bool takes_few(int64_t rows, bool) { return rows <= 16; }

template <class T, Form FP, bool GATED>
void launch_few(const Operand& P, const Operand& Q, const Result& res, int64_t rows, int64_t cols, int64_t k, hipStream_t st) {
    constexpr bool kSplit = FP == kCodes && std::is_same<T, F16>::value;
    constexpr int kMost = FP == kAlong ? 2 : 4;      // groups of rows that share the tokens' pieces
    const int64_t steps = std::max<int64_t>(1, (k + Step<FP>::kK - 1) / Step<FP>::kK);
    const int waves = (int)std::min<int64_t>(kWaves, steps);
    auto launch = [&](auto kernel, int groups) {
        const int64_t each = 16 * (GATED ? groups / 2 : groups);
        hipLaunchKernelGGL(kernel, dim3((unsigned)((cols + each - 1) / each)), dim3(64 * waves), 0, st, P, Q, res, rows, cols, k);
    };
    // as many groups as leave two workgroups for every compute unit
    const bool many = cols * (GATED ? 2 : 1) >= 512 * 16 * kMost;
    if constexpr (kSplit) {
        if (rows > 8) {
            many ? launch(rsh_few_rows_kernel<T, FP, GATED, kMost, 2>, kMost) : launch(rsh_few_rows_kernel<T, FP, GATED, 2, 2>, 2);
            return;
        }
    }
    many ? launch(rsh_few_rows_kernel<T, FP, GATED, kMost, 1>, kMost) : launch(rsh_few_rows_kernel<T, FP, GATED, 2, 1>, 2);
}

#define RSH_FEW(T, FP, GATED) \
    template void launch_few<T, FP, GATED>(const Operand&, const Operand&, const Result&, int64_t, int64_t, int64_t, hipStream_t);
RSH_FEW(F16, kAlong, true)
RSH_FEW(BF16, kAlong, true)
RSH_FEW(F16, kCodes, true)
RSH_FEW(BF16, kCodes, true)
RSH_FEW(F16, kCodes, false)
RSH_FEW(BF16, kCodes, false)
RSH_FEW(F16, kFours, false)
RSH_FEW(BF16, kFours, false)
#undef RSH_FEW

}  // namespace rsh
