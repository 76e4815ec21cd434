// The edges of a block: S = X + scale * gate * drop(N1(B)) and Y = N2(S), their gradients, and dropout alone.
#include <algorithm>

#include "rows.hpp"

namespace rsh {

namespace {

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

// Sums over the LANES lanes that share a row; every lane gets them, always added in the same order.  Waves meet in LDS, in two places
// by turns: a wave that writes a place again has passed the barrier that all come to after having read it.
template <int LANES>
struct Team {
    static constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    typedef float2_t Meeting[2][kWaves];
    Meeting& place;
    int turn = 0;
    __device__ __forceinline__ explicit Team(Meeting& p) : place(p) {}
    static __device__ __forceinline__ float in_wave(float v) {
        v = add_dpp<0xb1>(v);       // lanes 1 0 3 2
        v = add_dpp<0x4e>(v);       // lanes 2 3 0 1
        v = add_dpp<0x141>(v);      // eight lanes mirrored
        if constexpr (LANES >= 16) v = add_dpp<0x140>(v);      // sixteen
        const int lane = threadIdx.x & 63;
        if constexpr (LANES >= 32) v += shfl_f32(v, lane ^ 16);
        if constexpr (LANES >= 64) v += shfl_f32(v, lane ^ 32);
        return v;
    }
    __device__ __forceinline__ float2_t sum(float a, float b) {
        a = in_wave(a);
        b = in_wave(b);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6] = (float2_t){a, b};
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float2_t p = place[turn][w];
                a += p[0];
                b += p[1];
            }
            turn ^= 1;
        }
        return (float2_t){a, b};
    }
};

// f(c, column) for the runs of eight columns that a lane has: C of them, kept in registers, or (C = 0) as many as there are.
template <int LANES, int C, class F>
__device__ __forceinline__ void each_run(int d, F f) {
    const int lane = threadIdx.x % LANES;
    if constexpr (C > 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) f(c, 8 * (lane + LANES * c));
    } else {
        for (int col = 8 * lane; col < d; col += 8 * LANES) f(0, col);
    }
}

__device__ __forceinline__ void clear_from(Eight& e, int valid) {
    if (valid < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = i < valid ? e.v[i] : 0.f;
    }
}

// Parameters of a run: ones or zeros where there are none.
__device__ __forceinline__ Eight parameters(const void* p, int type, int col, int valid, float otherwise) {
    if (p) return load_eight(type, p, col, valid);
    Eight e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = otherwise;
    return e;
}

// m and r of a row whose runs are get(c, column), zeros behind the row's end.  Where a sum leaves the range of fp32, once more with the
// row scaled by a power of two.
template <int LANES, int C, class GET>
__device__ __forceinline__ float2_t statistics(const rsh_norm_t& norm, int d, Team<LANES>& team, GET get) {
    float m = 0.f, q = 0.f;
    auto attempt = [&](float c) {
        if (norm.kind == RSH_NORM_LAYER) {
            float a = 0.f;
            each_run<LANES, C>(d, [&](int i, int col) {
                const Eight e = get(i, col);
#pragma unroll
                for (int j = 0; j < 8; ++j) a += e.v[j] * c;
            });
            m = team.sum(a, 0.f)[0] / (float)d;
        }
        q = 0.f;
        each_run<LANES, C>(d, [&](int i, int col) {
            Eight e = get(i, col);
#pragma unroll
            for (int j = 0; j < 8; ++j) e.v[j] = e.v[j] * c - m;
            clear_from(e, d - col);
#pragma unroll
            for (int j = 0; j < 8; ++j) q += e.v[j] * e.v[j];
        });
        q = team.sum(q, 0.f)[0] / (float)d;
    };
    attempt(1.f);
    if (m - m + q < INFINITY) return (float2_t){m, 1.f / sqrtf(q + norm.eps)};
    const float c = 0x1p-70f;
    attempt(c);
    return (float2_t){m / c, c / sqrtf(q + fmaxf(norm.eps * c * c, 0x1p-149f))};
}

__device__ __forceinline__ void normalise(Eight& e, const rsh_norm_t& norm, float2_t s, int col, int valid) {
    const Eight w = parameters(norm.weight, norm.weight_type, col, valid, 1.f), b = parameters(norm.bias, norm.bias_type, col, valid, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = (e.v[i] - s[0]) * s[1] * w.v[i] + b.v[i];
}

template <int LANES> constexpr int kThreadsOf = LANES < 256 && LANES <= 64 ? 256 : LANES;
template <int LANES> constexpr int kRowsOf = kThreadsOf<LANES> / LANES;

}  // namespace

template <class T, int LANES, int C>
__global__ __launch_bounds__(kThreadsOf<LANES>) void rsh_join_forward_kernel(rsh_join_t j) {
    __shared__ typename Team<LANES>::Meeting meeting;
    Team<LANES> team(meeting);
    const Random random(j.drop);
    const int d = (int)j.d;
    for (int64_t first = (int64_t)blockIdx.x * kRowsOf<LANES>; first < j.t; first += (int64_t)gridDim.x * kRowsOf<LANES>) {
        const int64_t mine = first + threadIdx.x / LANES, row = min(mine, j.t - 1);
        const bool live = mine < j.t, leads = live && threadIdx.x % LANES == 0;
        Eight kept[C ? C : 1];       // B, then S
        float2_t after = {0.f, 1.f};
        auto loaded = [&](int c, int col) { return C ? kept[c] : load_eight<T>(j.B, row * j.ld_b + col, d - col); };
        if (j.B && C) each_run<LANES, C>(d, [&](int c, int col) { kept[c] = load_eight<T>(j.B, row * j.ld_b + col, d - col); });
        if (j.B && j.after.kind != RSH_NORM_NONE) {
            after = statistics<LANES, C>(j.after, d, team, loaded);
            if (leads && j.after.stats) *reinterpret_cast<float2_t*>(j.after.stats + 2 * row) = after;
        }
        auto sum = [&](int c, int col) {
            const int valid = d - col;
            Eight s = load_eight<T>(j.X, row * j.ld_x + col, valid);
            if (j.B) {
                Eight n = loaded(c, col);
                if (j.after.kind != RSH_NORM_NONE) normalise(n, j.after, after, col, valid);
                if (j.drop.share) random.drop(n, col, row, random.keep);
                const Eight g = parameters(j.gate, j.gate_type, 0, 0, 1.f);
                const Eight gate = j.gate ? load_eight(j.gate_type, j.gate, row * j.ld_gate + col, valid) : g;
#pragma unroll
                for (int i = 0; i < 8; ++i) s.v[i] += j.scale * gate.v[i] * n.v[i];
                clear_from(s, valid);
            }
            return s;
        };
        each_run<LANES, C>(d, [&](int c, int col) {
            const Eight s = sum(c, col);
            if (C) kept[c] = s;
            if (j.B && live) store_eight<T>(j.S, row * d + col, s, d - col);
        });
        if (j.before.kind == RSH_NORM_NONE) continue;
        auto summed = [&](int c, int col) { return C ? kept[c] : sum(c, col); };
        const float2_t before = statistics<LANES, C>(j.before, d, team, summed);
        if (leads && j.before.stats) *reinterpret_cast<float2_t*>(j.before.stats + 2 * row) = before;
        each_run<LANES, C>(d, [&](int c, int col) {
            Eight y = summed(c, col);
            normalise(y, j.before, before, col, d - col);
            if (live) store_eight<T>(j.Y, row * d + col, y, d - col);
        });
    }
}

namespace {

// The vectors among the gradients, in the order of their sums.
enum Slot { kBeforeWeight, kBeforeBias, kAfterWeight, kAfterBias, kGate, kSlots };
struct Vectors {
    void* out[kSlots];
    int type[kSlots];
    int at[kSlots];        // place among the wanted ones, or -1
    int count;
};

// Gradients of a run of a row.
struct Run {
    Eight g, xh;           // of Y times N2's weight; S without mean and size
    Eight ds;              // of S
    Eight gb, xb;          // of N1's result times its weight; B without mean and size
};

// A run's share of the vectors.
struct Sums {
    Eight before_weight, before_bias, after_weight, after_bias, gate;
    __device__ __forceinline__ const Eight& of(int k) const {
        return k == kBeforeWeight ? before_weight : k == kBeforeBias ? before_bias : k == kAfterWeight ? after_weight : k == kAfterBias ? after_bias : gate;
    }
};

// What a row's gradients need beside its elements.
struct RowState {
    int64_t row;
    bool live;
    float2_t before, after;        // m and r
    float2_t mean;                 // of g and of g xh
};

template <class T>
struct Backward {
    const rsh_join_t& j;
    const rsh_join_gradients_t& g;
    const Random& random;
    int d;
    bool first, second;        // whether N2 and its gradient, and whether N1 are there

    __device__ __forceinline__ Backward(const rsh_join_t& join, const rsh_join_gradients_t& grad, const Random& r)
        : j(join), g(grad), random(r), d((int)join.d), first(join.before.kind != RSH_NORM_NONE && grad.dY),
          second(join.B && join.after.kind != RSH_NORM_NONE) {}
    __device__ __forceinline__ RowState state(int64_t mine) const {
        RowState s = {min(mine, j.t - 1), mine < j.t, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
        if (s.live && first) s.before = *reinterpret_cast<const float2_t*>(j.before.stats + 2 * s.row);
        if (s.live && second) s.after = *reinterpret_cast<const float2_t*>(j.after.stats + 2 * s.row);
        return s;
    }
    __device__ __forceinline__ int valid(const RowState& s, int col) const { return s.live ? d - col : 0; }
    // Gradient of Y and the normalised S.
    template <bool SUM>
    __device__ __forceinline__ void load_before(const RowState& s, int col, Run& x, Sums& sums) const {
        const int v = valid(s, col);
        x.g = load_eight<T>(g.dY, s.row * g.ld_dy + col, v);
        x.xh = j.B ? load_eight<T>(j.S, s.row * d + col, v) : load_eight<T>(j.X, s.row * j.ld_x + col, v);
        const Eight w = parameters(j.before.weight, j.before.weight_type, col, v, 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.xh.v[i] = (x.xh.v[i] - s.before[0]) * s.before[1];
            if (SUM) sums.before_weight.v[i] += x.g.v[i] * x.xh.v[i], sums.before_bias.v[i] += x.g.v[i];
            x.g.v[i] *= w.v[i];
        }
    }
    __device__ __forceinline__ void load_sum(const RowState& s, int col, Run& x) const {
        const int v = valid(s, col);
        if (g.dS) x.ds = load_eight<T>(g.dS, s.row * g.ld_ds + col, v);
        else x.ds = Eight{};
    }
    __device__ __forceinline__ void join_sum(const RowState& s, int col, Run& x) const {
        if (first) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x.ds.v[i] += s.before[1] * (x.g.v[i] - s.mean[0] - x.xh.v[i] * s.mean[1]);
        }
        clear_from(x.ds, valid(s, col));
    }
    // From the gradient of S to that of N1's result; returns what the gate's gradient gets.
    template <bool SUM>
    __device__ __forceinline__ Eight through(const RowState& s, int col, Run& x, Sums& sums) const {
        const int v = valid(s, col);
        Eight b = load_eight<T>(j.B, s.row * j.ld_b + col, v), w, n;
        x.xb = b;
        if (second) {
            w = parameters(j.after.weight, j.after.weight_type, col, v, 1.f);
            n = parameters(j.after.bias, j.after.bias_type, col, v, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x.xb.v[i] = (b.v[i] - s.after[0]) * s.after[1];
                b.v[i] = x.xb.v[i] * w.v[i] + n.v[i];
            }
        }
        Eight factor;
#pragma unroll
        for (int i = 0; i < 8; ++i) factor.v[i] = j.scale;
        if (j.drop.share) {
            random.drop(factor, col, s.row, random.keep);
#pragma unroll
            for (int i = 0; i < 8; ++i) b.v[i] = factor.v[i] == 0.f ? 0.f : b.v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            b.v[i] *= x.ds.v[i] * factor.v[i];
            if (SUM) sums.gate.v[i] += b.v[i];
        }
        if (j.gate) {
            const Eight k = load_eight(j.gate_type, j.gate, s.row * j.ld_gate + col, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) factor.v[i] *= k.v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.gb.v[i] = x.ds.v[i] * factor.v[i];
            if (second) {
                if (SUM) sums.after_weight.v[i] += x.gb.v[i] * x.xb.v[i], sums.after_bias.v[i] += x.gb.v[i];
                x.gb.v[i] *= w.v[i];
            }
        }
        return b;
    }
};

}  // namespace

// One pass over the rows.  C = 1: a row in its lanes' registers, and the vectors' sums with it, a part of them from every workgroup.
// C = 0: rows of any length; the means of g and g xh go to `means` and another kernel adds up the vectors.
template <class T, int LANES, int C>
__global__ __launch_bounds__(kThreadsOf<LANES>) void rsh_join_backward_kernel(rsh_join_t j, rsh_join_gradients_t g, Vectors vectors, float* parts,
                                                                              float* means) {
    constexpr int kThreads = kThreadsOf<LANES>, kRows = kRowsOf<LANES>;
    __shared__ typename Team<LANES>::Meeting meeting;
    __shared__ float joined[C && kRows > 1 ? kThreads * 8 : 1];
    Team<LANES> team(meeting);
    const Random random(j.drop);
    const Backward<T> back(j, g, random);
    const int d = back.d;
    constexpr bool kSum = C > 0;
    Sums sums = {};
    const bool full = g.dgate && j.ld_gate;        // the gate's gradient is a matrix
    for (int64_t head = (int64_t)blockIdx.x * kRows; head < j.t; head += (int64_t)gridDim.x * kRows) {
        RowState s = back.state(head + threadIdx.x / LANES);
        Run kept[C ? C : 1];
        if (back.first) {
            float a = 0.f, b = 0.f;
            each_run<LANES, C>(d, [&](int c, int col) {
                Run& x = kept[c];
                back.template load_before<kSum>(s, col, x, sums);
#pragma unroll
                for (int i = 0; i < 8; ++i) a += x.g.v[i], b += x.g.v[i] * x.xh.v[i];
            });
            s.mean = team.sum(a, b) / (float)d;
            if (j.before.kind != RSH_NORM_LAYER) s.mean[0] = 0.f;
            if (means && s.live && threadIdx.x % LANES == 0) *reinterpret_cast<float2_t*>(means + 2 * s.row) = s.mean;
        }
        // Gradient of S of a run, and that of N1's result.
        auto of_sum = [&](int c, int col) {
            Run& x = kept[c];
            if (!C && back.first) back.template load_before<false>(s, col, x, sums);
            back.load_sum(s, col, x);
            back.join_sum(s, col, x);
        };
        float a = 0.f, b = 0.f;
        each_run<LANES, C>(d, [&](int c, int col) {
            of_sum(c, col);
            Run& x = kept[c];
            const int v = back.valid(s, col);
            if (g.dX) store_eight<T>(g.dX, s.row * d + col, x.ds, v);
            if (!j.B) return;
            const Eight gate = back.template through<kSum>(s, col, x, sums);
            if (full) store_eight(j.gate_type, g.dgate, s.row * d + col, gate, v);
            if (!back.second && g.dB) store_eight<T>(g.dB, s.row * d + col, x.gb, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) a += x.gb.v[i], b += x.gb.v[i] * x.xb.v[i];
        });
        if (!back.second || !g.dB) continue;
        float2_t mean = team.sum(a, b) / (float)d;
        if (j.after.kind != RSH_NORM_LAYER) mean[0] = 0.f;
        each_run<LANES, C>(d, [&](int c, int col) {
            Run& x = kept[c];
            if constexpr (!C) {
                of_sum(c, col);
                back.template through<false>(s, col, x, sums);
            }
            Eight db;
#pragma unroll
            for (int i = 0; i < 8; ++i) db.v[i] = s.after[1] * (x.gb.v[i] - mean[0] - x.xb.v[i] * mean[1]);
            store_eight<T>(g.dB, s.row * d + col, db, back.valid(s, col));
        });
    }
    if constexpr (C > 0) {
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (vectors.at[k] < 0) continue;
            float* const out = parts + ((int64_t)blockIdx.x * vectors.count + vectors.at[k]) * d;
            if constexpr (kRows == 1) {
                store_eight<F32>(out, 8 * threadIdx.x, sums.of(k), d - 8 * (int)threadIdx.x);
            } else {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[threadIdx.x * 8 + i] = sums.of(k).v[i];
                __syncthreads();
                for (int col = threadIdx.x; col < d; col += kThreads) {
                    float a = 0.f;
#pragma unroll
                    for (int r = 0; r < kRows; ++r) a += joined[r * LANES * 8 + col];
                    out[col] = a;
                }
            }
        }
    }
}

// The vectors' sums of rows too long for a team's registers: a thread has eight columns of the rows of a part.
template <class T>
__global__ __launch_bounds__(256) void rsh_join_columns_kernel(rsh_join_t j, rsh_join_gradients_t g, Vectors vectors, float* parts,
                                                               const float* means) {
    const Random random(j.drop);
    const Backward<T> back(j, g, random);
    const int col = 8 * (int)(blockIdx.x * 256 + threadIdx.x);
    if (col >= back.d) return;
    Sums sums = {};
    for (int64_t row = blockIdx.y; row < j.t; row += gridDim.y) {
        RowState s = back.state(row);
        Run x;
        if (back.first) {
            s.mean = *reinterpret_cast<const float2_t*>(means + 2 * row);
            back.template load_before<true>(s, col, x, sums);
        }
        if (!j.B) continue;
        back.load_sum(s, col, x);
        back.join_sum(s, col, x);
        (void)back.template through<true>(s, col, x, sums);
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k)
        if (vectors.at[k] >= 0)
            store_eight<F32>(parts + ((int64_t)blockIdx.y * vectors.count + vectors.at[k]) * back.d, col, sums.of(k), back.d - col);
}

// Sum of the parts, in their order within each of 32 runs of them, then of the runs.
__global__ __launch_bounds__(1024) void rsh_join_vectors_kernel(const float* parts, Vectors vectors, int64_t n, int64_t d) {
    __shared__ float joined[32][33];
    int k = 0;
    while (vectors.at[k] != (int)blockIdx.y) ++k;
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;
    float a = 0.f;
    if (col < d) {
#pragma unroll 4
        for (int64_t p = run; p < n; p += 32) a += parts[(p * vectors.count + blockIdx.y) * d + col];
    }
    joined[run][lane] = a;
    __syncthreads();
    if (run || col >= d) return;
    a = 0.f;
#pragma unroll
    for (int r = 0; r < 32; ++r) a += joined[r][lane];
    if (vectors.type[k] == RSH_F32) ((float*)vectors.out[k])[col] = a;
    else ((uint16_t*)vectors.out[k])[col] = (uint16_t)(vectors.type[k] == RSH_F16 ? F16::pair(a, 0.f) : BF16::pair(a, 0.f));
}

template <class T>
__global__ __launch_bounds__(256) void rsh_dropout_kernel(const void* X, void* Y, rsh_drop_t drop, int64_t n, int64_t runs, int64_t d, int64_t ld) {
    const Random random(drop);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / runs, col = 8 * (i - row * runs);
        const int valid = (int)min(d - col, (int64_t)8);
        Eight e = load_eight<T>(X, row * ld + col, valid);
        random.drop(e, (int)col, row, random.keep);
        store_eight<T>(Y, row * d + col, e, valid);
    }
}

namespace {
int launched() { return hipGetLastError() == hipSuccess ? RSH_OK : RSH_ERR_HIP; }

template <class F>
void by_type(int type, F f) {
    if (type == RSH_F32) f(F32());
    else if (type == RSH_F16) f(F16());
    else f(BF16());
}

// f(lanes of a row, runs of a lane): the fewest lanes that have the row in registers.  most: runs that a lane may have.
template <int MOST, class F>
void by_width(int64_t d, F f) {
    using std::integral_constant;
    const int64_t runs = (d + 7) / 8;
    if (runs <= 8) f(integral_constant<int, 8>(), integral_constant<int, 1>());
    else if (runs <= 16) f(integral_constant<int, 16>(), integral_constant<int, 1>());
    else if (runs <= 32) f(integral_constant<int, 32>(), integral_constant<int, 1>());
    else if (runs <= 64) f(integral_constant<int, 64>(), integral_constant<int, 1>());
    else if (runs <= 128) f(integral_constant<int, 128>(), integral_constant<int, 1>());
    else if (runs <= 256) f(integral_constant<int, 256>(), integral_constant<int, 1>());
    else if (runs <= 512) f(integral_constant<int, 512>(), integral_constant<int, 1>());
    else if (runs <= 1024) f(integral_constant<int, 1024>(), integral_constant<int, 1>());
    else if (MOST >= 4 && runs <= 4096) f(integral_constant<int, 1024>(), integral_constant<int, MOST >= 4 ? 4 : 1>());
    else f(integral_constant<int, 1024>(), integral_constant<int, 0>());
}

// Workgroups of the backward pass, each with a part of the vectors' sums, or parts of the columns' kernel.
constexpr int64_t kRegisterWidth = 8192, kColumnParts = 64;
int64_t backward_parts(int64_t t, int64_t d) {
    if (d > kRegisterWidth) return std::min(t, kColumnParts);
    int64_t parts = 0;
    by_width<1>(d, [&](auto lanes, auto) {
        constexpr int L = decltype(lanes)::value;
        parts = std::min<int64_t>((t + kRowsOf<L> - 1) / kRowsOf<L>, 256 * (1024 / kThreadsOf<L>));
    });
    return parts;
}
int64_t vector_bytes(int64_t t, int64_t d, int vectors) { return (backward_parts(t, d) * vectors * d * 4 + 15) / 16 * 16; }
}  // namespace

int64_t join_backward_work(int64_t t, int64_t d, int vectors) {
    return vector_bytes(t, d, vectors) + (d > kRegisterWidth && vectors ? (8 * t + 15) / 16 * 16 : 0);
}

int launch_join_forward(const rsh_join_t& join, void* stream) {
    by_type(join.type, [&](auto type) {
        by_width<4>(join.d, [&](auto lanes, auto runs) {
            constexpr int L = decltype(lanes)::value, C = decltype(runs)::value;
            const unsigned blocks = (unsigned)std::min<int64_t>((join.t + kRowsOf<L> - 1) / kRowsOf<L>, 1 << 16);
            hipLaunchKernelGGL((rsh_join_forward_kernel<decltype(type), L, C>), dim3(blocks), dim3(kThreadsOf<L>), 0, (hipStream_t)stream, join);
        });
    });
    return launched();
}

int launch_join_backward(const rsh_join_t& join, const rsh_join_gradients_t& g, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    Vectors v = {{g.before_weight, g.before_bias, g.after_weight, g.after_bias, join.ld_gate ? nullptr : g.dgate},
                 {join.before.weight_type, join.before.bias_type, join.after.weight_type, join.after.bias_type, join.gate_type}, {}, 0};
    for (int k = 0; k < kSlots; ++k) v.at[k] = v.out[k] ? v.count++ : -1;
    float* const parts = (float*)g.work;
    const int64_t n = backward_parts(join.t, join.d);
    by_type(join.type, [&](auto type) {
        using T = decltype(type);
        by_width<1>(join.d, [&](auto lanes, auto runs) {
            constexpr int L = decltype(lanes)::value, C = decltype(runs)::value;
            if constexpr (C) {
                hipLaunchKernelGGL((rsh_join_backward_kernel<T, L, C>), dim3((unsigned)n), dim3(kThreadsOf<L>), 0, st, join, g, v, parts, nullptr);
            } else {
                float* const means = v.count ? (float*)((char*)g.work + vector_bytes(join.t, join.d, v.count)) : nullptr;
                hipLaunchKernelGGL((rsh_join_backward_kernel<T, L, 0>), dim3((unsigned)std::min<int64_t>(join.t, 1 << 16)), dim3(L), 0, st, join, g, v,
                                   nullptr, means);
                if (v.count)
                    hipLaunchKernelGGL(rsh_join_columns_kernel<T>, dim3((unsigned)((join.d + 2047) / 2048), (unsigned)n), dim3(256), 0, st, join, g, v,
                                       parts, means);
            }
        });
    });
    if (v.count)
        hipLaunchKernelGGL(rsh_join_vectors_kernel, dim3((unsigned)((join.d + 31) / 32), v.count), dim3(1024), 0, st, parts, v, n, join.d);
    return launched();
}

int launch_dropout(const void* X, int type, int64_t t, int64_t d, int64_t ld, const rsh_drop_t& drop, void* Y, void* stream) {
    const int64_t runs = (d + 7) / 8, n = t * runs;
    by_type(type, [&](auto T) {
        hipLaunchKernelGGL(rsh_dropout_kernel<decltype(T)>, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 14)), dim3(256), 0,
                           (hipStream_t)stream, X, Y, drop, n, runs, d, ld);
    });
    return launched();
}

}  // namespace rsh
