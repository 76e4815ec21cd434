// The products of the feed-forward block for few rows (tokens): every weight is read once and multiplied with all of them, so the
// time is that of the weight's bytes.
//
// A wave has groups of 16 weight rows and takes every n-th step of k for them, n the waves of its workgroup; its weights go from
// memory straight into the registers that the matrix unit reads, next to 16 tokens' pieces of the same k.  Which k a lane has is
// free as long as both operands agree: lane (row r, quarter q) of 16 x 4 has 8 elements of 16 bits, or one whole block of 32 codes,
// whose four words then make four operands.  Several groups of rows share the tokens' pieces.  The waves' sums meet in LDS and are
// added in the waves' order.
//
// Measured: one token through the gated block of 8192 x 28672 in bfloat16 164 us (940 MB, 5.7 TB/s); through 28672 x 8192 in 4 bits
// 27 us (125 MB, 4.6 TB/s; 39 on the matrix units); 16 tokens through the gated block of 4096 x 16384 in 4 bits 21 us (71 MB), bound
// by the reads of the tokens, 4 KB for every 4 KB of codes.
#include <algorithm>

#include "ffn.hpp"

namespace rsh {

namespace {

constexpr int kWaves = 8;          // most waves of a workgroup

// A step is what a wave has in flight ahead: kLoads loads of 16 bytes a group of rows.  Of codes a step is one load, and four of
// them in a row are the wave's turn, whose scales come as one load of 16 bytes a row.
template <Form FP>
struct Step {
    static constexpr int kLoads = FP == kAlong ? 4 : 1;
    static constexpr int kLoadK = FP == kAlong ? 32 : 128;       // k of a load of all four quarters
    static constexpr int kK = kLoads * kLoadK;
    static constexpr int kTurn = FP == kAlong ? 1 : 4;           // steps of a turn
    static constexpr int kXLoads = FP == kCodes ? 4 : kLoads;
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
__global__ __launch_bounds__(64 * kWaves, FP == kAlong ? 4 : 2) void rsh_few_rows_kernel(Operand P, Operand Q, Result res, int64_t rows, int64_t cols, int64_t k) {
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
        ws[g] = FP == kAlong ? nullptr : P.scales[which] + row * P.ld;
    }
    const uint8_t* x[TOKENS];
    const uint8_t* xs[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const int64_t row = min((int64_t)kTile * t + (kSplit ? r & 7 : r), rows - 1);
        x[t] = (const uint8_t*)Q.data[0] + (kFour ? (row * Q.ld + q) * kBlockBytes : 2 * (row * Q.ld + (FP == kCodes ? 32 : 8) * q));
        xs[t] = kFour ? Q.scales[0] + row * Q.ld : nullptr;
    }

    struct Pieces {
        uint4_t w[GROUPS][S::kLoads], x[TOKENS][S::kXLoads];
    };
    struct Scales {
        uint4_t w[FP == kAlong ? 1 : GROUPS], x[kFour ? TOKENS : 1];     // byte 4 s + q: of the lane in step s of the turn
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
                if constexpr (FP == kAlong) p.w[g][j] = load8((const uint16_t*)w[g] + kk, kWhole ? 8 : k - kk - 8 * q);
                else p.w[g][j] = block ? *reinterpret_cast<const uint4_t*>(w[g] + kk / kBlock * kBlockBytes) : (uint4_t){0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                if constexpr (kFour) {
                    p.x[t][j] = block ? *reinterpret_cast<const uint4_t*>(x[t] + kk / kBlock * kBlockBytes) : (uint4_t){0, 0, 0, 0};
                } else if constexpr (FP == kAlong) {
                    p.x[t][j] = load8((const uint16_t*)x[t] + kk, kWhole ? 8 : k - kk - 8 * q);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p.x[t][4 * j + i] = load8((const uint16_t*)x[t] + kk + 8 * i, kWhole ? 8 : k - kk - 32 * q - 8 * i);
                }
            }
        }
    };
    auto load_scales = [&](Scales& c, int64_t k0) {
        if constexpr (FP != kAlong) {
            const int64_t b = k0 / kBlock;
            auto sixteen = [&](const uint8_t* at) {
                uint4_t v = {0, 0, 0, 0};
                if (b + 16 <= P.ld) {
                    __builtin_memcpy(&v, at + b, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 15; ++i)
                        if (b + i < P.ld) v[i / 4] |= (uint32_t)at[b + i] << (8 * (i & 3));
                }
                return v;
            };
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) c.w[g] = sixteen(ws[g]);
            if constexpr (kFour) {
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) c.x[t] = sixteen(xs[t]);
            }
        }
    };
    float4_t acc[GROUPS][TOKENS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) acc[g][t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Pieces& p, const Scales& c, int step) {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            if constexpr (kFour) {
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) {
                        const uint4_t a = p.w[g][j], b = p.x[t][j];
                        const int8v_t fa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, fb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
                        acc[g][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, acc[g][t], 4, 4, 0, c.w[g][step] >> (8 * q), 0, c.x[t][step] >> (8 * q));
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
                        const uint4_t a = from_codes8<M>(p.w[g][j][i], scale_of(c.w[g][step] >> (8 * q) & 255u));
#pragma unroll
                        for (int t = 0; t < TOKENS; ++t) acc[g][t] = M::mfma16(a, b[t], acc[g][t]);
                    }
                }
            }
        }
    };

    // The wave's whole turns, one step in flight ahead; the turn that ends past k, if there is one, is the last wave's.
    constexpr int64_t kTurnK = S::kTurn * S::kK;
    const int64_t turns = k / kTurnK;
    Pieces f[2];
    Scales now, next;
    if (wave < turns) {
        load_scales(now, wave * kTurnK);
        load(f[0], wave * kTurnK, std::true_type());
        // MORE: another turn follows.  (Loads that might not be there would have the products wait for all.)
        auto turn = [&](int64_t u, auto more) {
            constexpr bool kMore = decltype(more)::value;
#pragma unroll
            for (int s = 0; s < S::kTurn; ++s) {
                if (s + 1 < S::kTurn) {
                    load(f[(s + 1) & 1], u * kTurnK + (s + 1) * S::kK, std::true_type());
                } else if constexpr (kMore) {
                    load_scales(next, (u + waves) * kTurnK);
                    load(f[(s + 1) & 1], (u + waves) * kTurnK, std::true_type());
                }
                multiply(f[s & 1], now, s);
            }
            if constexpr (S::kTurn == 1 && kMore) f[0] = f[1];
            now = next;
        };
        int64_t u = wave;
        for (; u + waves < turns; u += waves) turn(u, std::true_type());
        turn(u, std::false_type());
    }
    if (turns * kTurnK < k && turns % waves == wave) {
        load_scales(now, turns * kTurnK);
#pragma unroll
        for (int s = 0; s < S::kTurn; ++s) {
            if (turns * kTurnK + s * S::kK >= k) break;
            load(f[0], turns * kTurnK + s * S::kK, std::false_type());
            multiply(f[0], now, s);
        }
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

namespace {

constexpr int kLaneK = 32;                     // k of a lane: a block
constexpr int kWaveK = 64 * kLaneK;            // k of a wave's 64 lanes

// Eight codes and their scale as fp32.
__device__ __forceinline__ void widen8(uint32_t codes, float scale, float* v) {
    const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    const float2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

}  // namespace

// One row of activations and weights in 4 bits.  A lane has one block of k, in fp32 registers for the activations, and streams that
// block of one weight row after the other past it, kTurn rows in flight and as many in work: a load is 1 KB of one row, and nothing
// but weights passes through the memory pipeline, where the matrix unit's operands would take four loads of activations for every one
// of codes.  `chunks` waves of a workgroup have its k in turn, the next as many the same for other rows; `rows` of them a wave, whose
// sums wait in LDS and are added in the waves' order at the end.
constexpr int kTurn = 4, kMostRows = 64;

template <class T, Form FP, bool GATED>
__global__ __launch_bounds__(64 * kWaves, 4) void rsh_one_row_kernel(Operand P, Operand Q, Result res, int64_t cols, int64_t k, int chunks, int rows) {
    constexpr int kOut = GATED ? kTurn / 2 : kTurn;        // columns of the result in a turn
    __shared__ float sums[kWaves][kMostRows * (GATED ? 2 : 1)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sets = kWaves / chunks, set = wave / chunks;
    const int64_t first = ((int64_t)blockIdx.x * sets + set) * rows;
    struct Rows {
        uint4_t w[kTurn];
        uint32_t s[kTurn];
    };
    if ((int64_t)(wave % chunks) * kWaveK >= k)       // nothing to add
        for (int i = lane; i < kMostRows * (GATED ? 2 : 1); i += 64) sums[wave][i] = 0.f;
    for (int64_t k0 = (int64_t)(wave % chunks) * kWaveK; k0 < k; k0 += (int64_t)chunks * kWaveK) {
        const bool again = k0 >= (int64_t)chunks * kWaveK;
        const int64_t kk = k0 + kLaneK * lane;
        const bool in = kk < k;
        // lanes past k read the row's last block, which their zeros of x meet
        const int b = (int)(in ? kk / kBlock : P.ld - 1);
        float x[kLaneK];
        if constexpr (FP == kFours) {
            const uint4_t c = reinterpret_cast<const uint4_t*>(Q.data[0])[b];
            const float e = scale_of(Q.scales[0][b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) widen8(c[i], e, x + 8 * i);
        } else {
            uint4_t v[4];
            if (k0 + kWaveK <= k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4_a2*>((const uint16_t*)Q.data[0] + kk + 8 * i);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = load8((const uint16_t*)Q.data[0] + kk + 8 * i, k - kk - 8 * i);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t word = v[i / 4][i % 4];
                x[2 * i] = T::widen((uint16_t)word);
                x[2 * i + 1] = T::widen((uint16_t)(word >> 16));
            }
        }
        auto load = [&](Rows& n, int turn) {
#pragma unroll
            for (int r = 0; r < kTurn; ++r) {
                // rows past the end read the last one; nobody keeps their sums
                const int which = GATED ? r / kOut : 0;
                const int64_t at = min(first + turn + r % kOut, cols - 1) * P.ld;
                n.w[r] = reinterpret_cast<const uint4_t*>((const uint8_t*)P.data[which] + at * kBlockBytes)[b];
                n.s[r] = (P.scales[which] + at)[b];
            }
        };
        auto multiply = [&](const Rows& n, int turn) {
            float acc[kTurn];
#pragma unroll
            for (int r = 0; r < kTurn; ++r) {
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[8];
                    widen8(n.w[r][i], scale_of(n.s[r]), v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j & 1] = fmaf(v[j], x[8 * i + j], sum[j & 1]);
                }
                acc[r] = in ? sum[0] + sum[1] : 0.f;
            }
            // each sixteen lanes take one of the four rows, and add up
            float one[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float keep = lane & 32 ? acc[r + 2] : acc[r], give = lane & 32 ? acc[r] : acc[r + 2];
                one[r] = keep + __shfl_xor(give, 32);
            }
            float v = (lane & 16 ? one[1] : one[0]) + __shfl_xor(lane & 16 ? one[0] : one[1], 16);
            v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
            v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
            v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, false));
            v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, false));
            const int r = lane >> 4;
            float* const to = &sums[wave][GATED ? (r / 2) * kMostRows + turn + r % 2 : turn + r];
            if ((lane & 15) == 0) *to = again ? *to + v : v;
        };
        Rows now, next;
        load(now, 0);
        for (int turn = 0; turn < rows; turn += kOut) {
            if (turn + kOut < rows) load(next, turn + kOut);
            multiply(now, turn);
            now = next;
        }
    }
    __syncthreads();
    for (int i = 4 * threadIdx.x; i < sets * rows; i += 4 * 64 * kWaves) {
        float4_t a = {0.f, 0.f, 0.f, 0.f}, c = a;
        const int from = i / rows * chunks, r = i % rows;
        for (int v = 0; v < chunks; ++v)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] += sums[from + v][r + j];
                if constexpr (GATED) c[j] += sums[from + v][kMostRows + r + j];
            }
        const int64_t col = (int64_t)blockIdx.x * sets * rows + i;
        if (col < cols) finish<T, GATED>(res, res.out[0], 0, col, cols - col, a, c);
    }
}

// Up to one tile of 16 tokens (two of eight beside codes in binary16).  Beyond, tiles of 128 x 64 read the tokens once for 128 weight
// rows, and a second tile of tokens would double the reads here.  Measured with weights from memory, 16 tokens here and 17 there, us:
// 28672 x 8192 in 4 bits beside bfloat16 45 and 62 (to 64 tokens 63), beside binary16 60 and 59, 4 bits on both sides 35 and 34;
// 4096 x 4096 9 and 13, 12 and 13, 7 and 11; gated 8192 x 28672 in bfloat16 186 and 182, in 4 bits 90 and 104, beside binary16 120 and 109.
// Rows of 28672 beside binary16 lose from 9 tokens on (68 to 76 against 58).
bool takes_few(int64_t rows) { return rows <= 16; }

template <class T, Form FP, bool GATED>
void launch_few(const Operand& P, const Operand& Q, const Result& res, int64_t rows, int64_t cols, int64_t k, hipStream_t st) {
    if constexpr (FP != kAlong) {
        if (rows == 1) {
            // As many of the eight waves on k as it has waves' worth, the others on further rows; rows for two workgroups on
            // every compute unit, at least a turn's.
            const int64_t need = (k + kWaveK - 1) / kWaveK;
            const int chunks = need > 4 ? 8 : need > 2 ? 4 : (int)need, sets = kWaves / chunks;
            const int each = (int)std::min<int64_t>(kMostRows, std::max<int64_t>(4, (cols + 512 * sets - 1) / (512 * sets) + 3)) / 4 * 4;
            hipLaunchKernelGGL((rsh_one_row_kernel<T, FP, GATED>), dim3((unsigned)((cols + each * sets - 1) / (each * sets))), dim3(64 * kWaves), 0, st, P, Q,
                               res, cols, k, chunks, each);
            return;
        }
    }
    constexpr bool kSplit = FP == kCodes && std::is_same<T, F16>::value;
    constexpr int kMost = FP == kAlong ? 2 : 4;      // groups of rows that share the tokens' pieces
    constexpr int64_t kTurnK = Step<FP>::kTurn * Step<FP>::kK;
    const int waves = (int)std::min<int64_t>(kWaves, (k + kTurnK - 1) / kTurnK);
    auto launch = [&](auto kernel, int groups) {
        const int64_t each = 16 * (GATED ? groups / 2 : groups);
        hipLaunchKernelGGL(kernel, dim3((unsigned)((cols + each - 1) / each)), dim3(64 * waves), 0, st, P, Q, res, rows, cols, k);
    };
    // as many groups as leave a workgroup for every compute unit
    const bool many = cols * (GATED ? 2 : 1) >= 256 * 16 * kMost;
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
