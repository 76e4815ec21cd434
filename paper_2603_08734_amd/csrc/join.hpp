// Kernels of norms and joins, a source file for each type.  For every row
//   n = N1(B),  D = drop(n),  S = X + scale * gate * D,  Y = N2(S),   N(x) = (x - m) r w + b,  r = (mean of (x - m)^2 + eps)^-1/2
// with m the mean (RSH_NORM_LAYER) or zero, and backwards, xh = (S - m) r and g = dY w2:
//   dS' = dS + r (g - mean(g) - xh mean(g xh)),  dX = dS',  dn = dS' scale gate (1 / (1 - p) or zero),  dB as dS' from dn w1 and B's xh,
//   dw = sum of dY xh over the rows, db = sum of dY, dgate = dS' scale D (summed where the gate is a vector)
// (mean(g) without a mean in the forward pass is zero).  Each tensor is read once and written once (gradients of rows beyond 8192 columns read theirs
// twice), a few dozen operations an element: bound by memory, if the work of a row leaves it busy.  So a row is eight columns to a lane, whatever number of lanes that takes (8 to 1024),
// and a workgroup goes through many rows: parameters stay in its registers, the gradients' sums over the rows in LDS, the next row is on
// its way while one is computed, and the only waits within a row are for the sums over its lanes, one a norm (two with a mean).
// Measured (a copy too large for the caches runs at 5.1 TB/s, reading and writing; smaller ones up to 7.2): 2048 x 8192 bfloat16, sum and norm
// 24.0 us (134 MB, 5.6 TB/s); 2^20 x 64 binary16, norm 53.7 and its gradients 78 us (5.0, 5.2); 8192 x 8192 bfloat16 with both norms, gate and
// dropout 126 us forward and 170 to 189 backward (4.3, 4.3 to 4.7), where dropout's random numbers cost 16 us and each wait for sums about 10; 1001 x 500 fp32
// 7.2 and 10.8 us, 16 x 4096 4.8, 1 x 8192 2.7 (the norm alone), where a launch's latency counts.
#pragma once
#include <algorithm>

#include "rows.hpp"

namespace rsh {

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// Sum over groups of N neighbouring lanes, N up to 16, in all of them.
template <int N>
__device__ __forceinline__ float sum_near(float v) {
    if constexpr (N >= 2) v = add_dpp<0xb1>(v);        // lanes 1 0 3 2
    if constexpr (N >= 4) v = add_dpp<0x4e>(v);        // lanes 2 3 0 1
    if constexpr (N >= 8) v = add_dpp<0x141>(v);       // eight lanes mirrored
    if constexpr (N >= 16) v = add_dpp<0x140>(v);      // sixteen
    return v;
}
// Over a wave, alike in all lanes: the last lane of a row of sixteen goes to the next row, that of the second row to the upper half.
__device__ __forceinline__ float sum_wave(float v) {
    v = add_dpp<0x143, 0xc>(add_dpp<0x142, 0xa>(sum_near<16>(v)));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums over the LANES lanes that share a row; every lane gets them, always added in the same order.  Waves meet in LDS, in two places
// by turns: a wave that writes a place again has passed the barrier that all come to after having read it.  A row waits for its sums with
// nothing else to do, so they are formed by moves between lanes alone (with two reads of other lanes by way of LDS and one of every wave's sum
// a norm of 8192 columns more cost 25 us of 110 in 8192 rows).
template <int LANES>
struct Team {
    static constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    typedef float2_t Meeting[2][kWaves];
    Meeting& place;
    int turn = 0;
    __device__ __forceinline__ explicit Team(Meeting& p) : place(p) {}
    static __device__ __forceinline__ float in_wave(float v) {
        if constexpr (LANES >= 64) return sum_wave(v);
        v = sum_near<LANES < 16 ? LANES : 16>(v);
        if constexpr (LANES == 32) v += shfl_f32(v, (threadIdx.x & 63) ^ 16);
        return v;
    }
    __device__ __forceinline__ float2_t sum(float a, float b) {
        a = in_wave(a);
        b = in_wave(b);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6] = (float2_t){a, b};
            __syncthreads();
            const float2_t p = place[turn][threadIdx.x % kWaves];
            a = sum_near<kWaves>(p[0]);
            b = sum_near<kWaves>(p[1]);
            turn ^= 1;
        }
        return (float2_t){a, b};
    }
    __device__ __forceinline__ float sum(float a) {
        a = in_wave(a);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6][0] = a;
            __syncthreads();
            a = sum_near<kWaves>(place[turn][threadIdx.x % kWaves][0]);
            turn ^= 1;
        }
        return a;
    }
};

// What is widened from it before is not kept for after: it is widened again, an instruction an element in place of a register.
template <class T>
__device__ __forceinline__ void renew(Raw<T>& r) {
#pragma unroll
    for (auto& v : r.v) asm volatile("" : "+v"(v));
}

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

// A run of a row of parameters or of the gate, in fp32 or in the rows' type.
template <class T, bool SHORT>
__device__ __forceinline__ Eight load_vector(const void* p, int type, int col, int d) {
    if (std::is_same<T, F32>::value || type == RSH_F32) return widen(settle<F32, SHORT>(load_raw<F32, SHORT>(p, col, d), col, d));
    return widen(settle<T, SHORT>(load_raw<T, SHORT>(p, col, d), col, d));
}
// Parameters of a run: ones or zeros where there are none.
template <class T, bool SHORT>
__device__ __forceinline__ Eight parameters(const void* p, int type, int col, int d, float otherwise) {
    if (p) return load_vector<T, SHORT>(p, type, col, d);
    Eight e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = otherwise;
    return e;
}
// The row of a team: `head`, alike in all lanes of a wave, and the lane's distance from it, which is zero where a team is no smaller than a wave.
// A row's address is then a scalar product and one addition; with teams of a few lanes it was a 64-bit product of vectors for every tensor.
struct Place {
    int64_t head;
    int mine;
    __device__ __forceinline__ int64_t row() const { return head + mine; }
    // What lies row() * ld elements of `size` behind `base`, which may be null; ld * size is below 2^32.
    __device__ __forceinline__ const void* of(const void* base, int64_t ld, int size) const {
        return base ? (const uint8_t*)base + head * ld * size + (uint64_t)(uint32_t)mine * (uint32_t)(ld * size) : nullptr;
    }
};
template <int LANES>
__device__ __forceinline__ Place place_of(int64_t first, int64_t t, bool* live) {
    if constexpr (LANES >= 64) {
        const int64_t r = first + threadIdx.x / LANES;
        const int64_t head = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(r >> 32)) << 32 |
                                       (uint32_t)__builtin_amdgcn_readfirstlane((int)r));
        *live = head < t;
        return {min(head, t - 1), 0};
    }
    const int mine = threadIdx.x / LANES;
    *live = first + mine < t;
    return {first, (int)min((int64_t)mine, t - 1 - first)};
}

// Into a row of d at column col.
template <class T>
__device__ __forceinline__ void store_run(void* base, const Place& row, int col, int d, const Eight& e) {
    store_eight<T>((void*)byte_of(row.of(base, d, size_of<T>()), (uint32_t)col * (uint32_t)size_of<T>()), 0, e, d - col);
}

// m and r of a row whose runs are get(c, column), zeros behind the row's end.  Where a sum leaves the range of fp32, once more with the
// row scaled by a power of two.
template <int LANES, int C, class GET>
__device__ __forceinline__ float2_t statistics(const rsh_norm_t& norm, int d, Team<LANES>& team, GET get) {
    const float share = 1.f / (float)d;
    float m = 0.f, q = 0.f;
    auto attempt = [&](float c) {
        if (norm.kind == RSH_NORM_LAYER) {
            float a = 0.f;
            each_run<LANES, C>(d, [&](int i, int col) {
                const Eight e = get(i, col);
#pragma unroll
                for (int j = 0; j < 8; ++j) a += e.v[j] * c;
            });
            m = team.sum(a) * share;
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
        q = team.sum(q) * share;
    };
    attempt(1.f);
    if (m - m + q < INFINITY) return (float2_t){m, __builtin_amdgcn_rsqf(q + norm.eps)};      // one step of fp32 off at most, a normal number
    const float c = 0x1p-80f;      // 2^21 squares of numbers of 2^128 stay in range
    attempt(c);
    return (float2_t){m / c, c / sqrtf(q + fmaxf(norm.eps * c * c, 0x1p-149f))};
}

template <int LANES> constexpr int kThreadsOf = LANES <= 64 ? 256 : LANES;
template <int LANES> constexpr int kRowsOf = kThreadsOf<LANES> / LANES;

// Parameters of the run of columns that a lane has in every row: kept in fp32 registers while the workgroup goes through its rows.  Loaded anew
// for every row they took as many instructions as the row itself, and their latency showed.
template <class T, bool SHORT>
struct Affine {
    Eight w, b;
    __device__ __forceinline__ Affine(const rsh_norm_t& n, int col, int d)
        : w(parameters<T, SHORT>(n.kind == RSH_NORM_NONE ? nullptr : n.weight, n.weight_type, col, d, 1.f)),
          b(parameters<T, SHORT>(n.kind == RSH_NORM_NONE ? nullptr : n.bias, n.bias_type, col, d, 0.f)) {}
    __device__ __forceinline__ void apply(Eight& e, float2_t s) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (e.v[i] - s[0]) * s[1] * w.v[i] + b.v[i];
    }
};

// Rows of up to 8 LANES columns, a run a lane.  JOIN: whether there is a B.  The next row's loads go out before
// this one is begun: a row takes as long as they do.
template <class T, int LANES, bool JOIN>
__global__ __launch_bounds__(kThreadsOf<LANES>) __attribute__((amdgpu_waves_per_eu(4))) void rsh_join_forward_kernel(rsh_join_t j) {
    constexpr bool kShort = LANES == 8;        // rows may be shorter than a run
    constexpr int kSize = size_of<T>(), kRows = kRowsOf<LANES>;
    __shared__ typename Team<LANES>::Meeting meeting;
    Team<LANES> team(meeting);
    const Random random(j.drop);
    const int d = (int)j.d, col = 8 * (threadIdx.x % LANES);
    const Affine<T, kShort> first(j.after, col, d), second(j.before, col, d);
    const float factor = j.drop.share ? j.scale * random.keep : j.scale;
    Eight gate = parameters<T, kShort>(j.ld_gate ? nullptr : j.gate, j.gate_type, col, d, 1.f);
    const int64_t step = (int64_t)gridDim.x * kRows;
    Raw<T> x, b, next_x, next_b;
    auto load = [&](int64_t head) {
        bool is;
        const Place row = place_of<LANES>(head, j.t, &is);
        if constexpr (JOIN) next_b = load_raw<T, kShort>(row.of(j.B, j.ld_b, kSize), col, d);
        next_x = load_raw<T, kShort>(row.of(j.X, j.ld_x, kSize), col, d);
    };
    load((int64_t)blockIdx.x * kRows);
    for (int64_t head = (int64_t)blockIdx.x * kRows; head < j.t; head += step) {
        bool live;
        const Place row = place_of<LANES>(head, j.t, &live);
        const bool leads = live && threadIdx.x % LANES == 0;
        x = next_x;
        if constexpr (JOIN) b = next_b;
        if (head + step < j.t) load(head + step);
        Eight s;
        if constexpr (JOIN) {
            Eight n = widen(settle<T, kShort>(b, col, d));
            if (j.after.kind != RSH_NORM_NONE) {
                const float2_t at = statistics<LANES, 1>(j.after, d, team, [&](int, int) { return n; });
                if (leads && j.after.stats) *reinterpret_cast<float2_t*>(j.after.stats + 2 * row.row()) = at;
                first.apply(n, at);
            }
            if (j.ld_gate) gate = load_vector<T, kShort>(row.of(j.gate, j.ld_gate, j.gate_type == RSH_F32 ? 4 : 2), j.gate_type, col, d);
            if (j.drop.share) random.drop(n, col, row.row(), factor);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) n.v[i] *= factor;
            s = widen(settle<T, kShort>(x, col, d));
#pragma unroll
            for (int i = 0; i < 8; ++i) s.v[i] += gate.v[i] * n.v[i];
            clear_from(s, d - col);
            if (live) store_run<T>(j.S, row, col, d, s);
        } else {
            s = widen(settle<T, kShort>(x, col, d));
        }
        if (j.before.kind == RSH_NORM_NONE) continue;
        const float2_t at = statistics<LANES, 1>(j.before, d, team, [&](int, int) { return s; });
        if (leads && j.before.stats) *reinterpret_cast<float2_t*>(j.before.stats + 2 * row.row()) = at;
        second.apply(s, at);
        if (live) store_run<T>(j.Y, row, col, d, s);
    }
}

// Longer rows: C runs a lane in registers, or (C = 0) as many as there are, read again at every pass.
template <class T, int LANES, int C, bool JOIN>
__global__ __launch_bounds__(LANES) __attribute__((amdgpu_waves_per_eu(4))) void rsh_join_forward_long_kernel(rsh_join_t j) {
    constexpr int kSize = size_of<T>();
    __shared__ typename Team<LANES>::Meeting meeting;
    Team<LANES> team(meeting);
    const Random random(j.drop);
    const int d = (int)j.d;
    const float factor = j.drop.share ? j.scale * random.keep : j.scale;
    for (int64_t at = blockIdx.x; at < j.t; at += gridDim.x) {
        const Place row = {at, 0};
        const void* const x_row = row.of(j.X, j.ld_x, kSize);
        const void* const b_row = row.of(j.B, j.ld_b, kSize);
        Raw<T> x[C ? C : 1], b[JOIN && C ? C : 1];
        Eight kept[C ? C : 1];
        if constexpr (C > 0) {
            if constexpr (JOIN) each_run<LANES, C>(d, [&](int c, int col) { b[c] = load_raw<T, false>(b_row, col, d); });
            each_run<LANES, C>(d, [&](int c, int col) { x[c] = load_raw<T, false>(x_row, col, d); });
        }
        float2_t after = {0.f, 1.f};
        auto loaded = [&](int c, int col) { return widen(settle<T, false>(C ? b[c] : load_raw<T, false>(b_row, col, d), col, d)); };
        if (JOIN && j.after.kind != RSH_NORM_NONE) {
            after = statistics<LANES, C>(j.after, d, team, loaded);
            if (threadIdx.x == 0 && j.after.stats) *reinterpret_cast<float2_t*>(j.after.stats + 2 * row.row()) = after;
        }
        auto sum = [&](int c, int col) {
            Eight s = widen(settle<T, false>(C ? x[c] : load_raw<T, false>(x_row, col, d), col, d));
            if constexpr (JOIN) {
                Eight n = loaded(c, col);
                if (j.after.kind != RSH_NORM_NONE) Affine<T, false>(j.after, col, d).apply(n, after);
                if (j.drop.share) random.drop(n, col, row.row(), factor);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) n.v[i] *= factor;
                const Eight gate = parameters<T, false>(row.of(j.gate, j.ld_gate, j.gate_type == RSH_F32 ? 4 : 2), j.gate_type, col, d, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) s.v[i] += gate.v[i] * n.v[i];
                clear_from(s, d - col);
            }
            return s;
        };
        if constexpr (JOIN || C > 0) {
            each_run<LANES, C>(d, [&](int c, int col) {
                if constexpr (C > 0 && JOIN) renew(b[c]);
                const Eight s = sum(c, col);
                if (C) kept[c] = s;
                if (JOIN) store_run<T>(j.S, row, col, d, s);
            });
        }
        if (j.before.kind == RSH_NORM_NONE) continue;
        auto summed = [&](int c, int col) { return C ? kept[c] : sum(c, col); };
        const float2_t before = statistics<LANES, C>(j.before, d, team, summed);
        if (threadIdx.x == 0 && j.before.stats) *reinterpret_cast<float2_t*>(j.before.stats + 2 * row.row()) = before;
        each_run<LANES, C>(d, [&](int c, int col) {
            Eight y = summed(c, col);
            Affine<T, false>(j.before, col, d).apply(y, before);
            store_run<T>(j.Y, row, col, d, y);
        });
    }
}

// The vectors among the gradients, in the order of their sums.
enum Slot { kBeforeWeight, kBeforeBias, kAfterWeight, kAfterBias, kGate, kSlots };
struct Vectors {
    void* out[kSlots];
    int type[kSlots];
    int at[kSlots];        // place among the wanted ones, or -1
    int count;
};

// A run's share of the vectors, which add(slot, terms) takes.  In registers, or, where a row's gradients need those, in LDS, 16 bytes a thread
// and turn that it alone reads and writes: weights and gate, or with the biases all but the gate (five would be all of the LDS).
struct NoSums {
    __device__ __forceinline__ void add(Slot, const Eight&) {}
};
struct RegisterSums {
    Eight of[kSlots] = {};
    __device__ __forceinline__ void add(Slot k, const Eight& e) {
#pragma unroll
        for (int i = 0; i < 8; ++i) of[k].v[i] += e.v[i];
    }
    __device__ __forceinline__ Eight get(int k) const { return of[k]; }
};
template <int THREADS, bool BIAS>
struct LdsSums {
    static constexpr int SLOTS = BIAS ? 4 : 3;
    typedef float4_t Place[SLOTS][2][THREADS];
    Place& place;
    const Vectors& vectors;
    Eight gate = {};
    __device__ __forceinline__ LdsSums(Place& p, const Vectors& v) : place(p), vectors(v) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) place[k][0][threadIdx.x] = place[k][1][threadIdx.x] = (float4_t){0.f, 0.f, 0.f, 0.f};
    }
    static __device__ __forceinline__ constexpr int at(int k) {      // SLOTS: not there
        return k == kBeforeWeight ? 0 : k == kAfterWeight ? 1 : k == kGate ? (BIAS ? SLOTS : 2) : BIAS ? (k == kBeforeBias ? 2 : 3) : SLOTS;
    }
    __device__ __forceinline__ void add(Slot k, const Eight& e) {
        if (BIAS && k == kGate) {
#pragma unroll
            for (int i = 0; i < 8; ++i) gate.v[i] += e.v[i];
        } else if (at(k) < SLOTS && vectors.at[k] >= 0) {
            float4_t* const lo = &place[at(k)][0][threadIdx.x];
            float4_t* const hi = &place[at(k)][1][threadIdx.x];
            *lo += (float4_t){e.v[0], e.v[1], e.v[2], e.v[3]};
            *hi += (float4_t){e.v[4], e.v[5], e.v[6], e.v[7]};
        }
    }
    __device__ __forceinline__ Eight get(int k) const {
        if (at(k) >= SLOTS) return gate;
        const float4_t a = place[at(k)][0][threadIdx.x], b = place[at(k)][1][threadIdx.x];
        return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
    }
};

template <class T>
struct Inputs {
    Raw<T> x, b, ds, dy;
    float2_t before, after;        // m and r of S and of B
    bool live;
};

// Gradients of a run of a row.
struct Run {
    Eight g, xh;           // of Y times N2's weight; S without mean and size
    Eight ds;              // of S
    Eight xb;              // B without mean and size
    Eight gb;              // gradient of N1's result times its weight
    uint32_t kept;         // of dropout
};

// The parameters of a run: of every row the same run, so kept, or loaded anew.
template <class T, bool SHORT, bool BIAS>
struct KeptParameters {
    Affine<T, SHORT> after, before;
    Eight gate;
    __device__ __forceinline__ KeptParameters(const rsh_join_t& j, int col, int d)
        : after(j.after, col, d), before(j.before, col, d),
          gate(parameters<T, SHORT>(j.ld_gate ? nullptr : j.gate, j.gate_type, col, d, 1.f)) {}
    __device__ __forceinline__ Eight after_weight(int) const { return after.w; }
    __device__ __forceinline__ Eight after_bias(int) const { return BIAS ? after.b : Eight{}; }
    __device__ __forceinline__ Eight before_weight(int) const { return before.w; }
    __device__ __forceinline__ Eight gate_of(int) const { return gate; }
};
template <class T>
struct LoadedParameters {
    const rsh_join_t& j;
    int d;
    __device__ __forceinline__ Eight after_weight(int col) const { return parameters<T, false>(j.after.weight, j.after.weight_type, col, d, 1.f); }
    __device__ __forceinline__ Eight after_bias(int col) const { return parameters<T, false>(j.after.bias, j.after.bias_type, col, d, 0.f); }
    __device__ __forceinline__ Eight before_weight(int col) const { return parameters<T, false>(j.before.weight, j.before.weight_type, col, d, 1.f); }
    __device__ __forceinline__ Eight gate_of(int col) const { return parameters<T, false>(j.ld_gate ? nullptr : j.gate, j.gate_type, col, d, 1.f); }
};

// JOIN as above; SUMS: where the vectors are added up, PARAMETERS: where the parameters come from.
template <class T, bool JOIN, bool SHORT, class SUMS, class PARAMETERS>
struct Backward {
    static constexpr int kSize = size_of<T>();
    const rsh_join_t& j;
    const rsh_join_gradients_t& g;
    const Random& random;
    const PARAMETERS& given;
    int d;
    bool first, second;        // whether N2 and its gradient, and whether N1 are there

    __device__ __forceinline__ Backward(const rsh_join_t& join, const rsh_join_gradients_t& grad, const Random& r, const PARAMETERS& p)
        : j(join), g(grad), random(r), given(p), d((int)join.d), first(join.before.kind != RSH_NORM_NONE && grad.dY),
          second(JOIN && join.after.kind != RSH_NORM_NONE) {}

    // Of a row.  live: it is one, else all of it counts as zero.
    __device__ __forceinline__ Inputs<T> load(const Place& row, bool live, int col) const {
        Inputs<T> in = {};
        in.live = live;
        auto run = [&](const void* p, int64_t ld) { return load_raw<T, SHORT>(row.of(p, ld, kSize), col, d); };
        if (first) {
            in.dy = run(g.dY, g.ld_dy);
            in.x = run(j.X, j.ld_x);
            in.before = *reinterpret_cast<const float2_t*>(j.before.stats + 2 * row.row());
        }
        if constexpr (JOIN) {
            in.b = run(j.B, j.ld_b);
            if (second) in.after = *reinterpret_cast<const float2_t*>(j.after.stats + 2 * row.row());
            if (g.dS) in.ds = run(g.dS, g.ld_ds);
        }
        return in;
    }
    __device__ __forceinline__ Eight value(const Inputs<T>& in, const Raw<T>& r, int col) const {
        return widen(settle<T, SHORT>(r, col, d, in.live));
    }
    // N1's result, after dropout but for its factor.
    __device__ __forceinline__ Eight inner(const Run& x, int col) const {
        Eight n = x.xb;
        if (second) {
            const Eight w = given.after_weight(col), b = given.after_bias(col);
#pragma unroll
            for (int i = 0; i < 8; ++i) n.v[i] = n.v[i] * w.v[i] + b.v[i];
        }
        drop(n, x);
        return n;
    }
    __device__ __forceinline__ float factor() const { return j.drop.share ? j.scale * random.keep : j.scale; }
    // scale * gate times dropout's factor.
    __device__ __forceinline__ Eight factors(const Place& row, int col) const {
        Eight f;
        if (j.ld_gate) f = load_vector<T, SHORT>(row.of(j.gate, j.ld_gate, j.gate_type == RSH_F32 ? 4 : 2), j.gate_type, col, d);
        else f = given.gate_of(col);
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] *= factor();
        return f;
    }
    // What is dropped becomes zero, infinities and NaN too, in either direction.
    __device__ __forceinline__ void drop(Eight& e, const Run& x) const {
        if (!j.drop.share) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = x.kept >> i & 1 ? e.v[i] : 0.f;
    }
    __device__ __forceinline__ void store_gate(const Place& row, int col, const Eight& gate) const {
        if (std::is_same<T, F32>::value || j.gate_type == RSH_F32) store_run<F32>(g.dgate, row, col, d, gate);
        else store_run<T>(g.dgate, row, col, d, gate);
    }
    // Up to the gradient of N2 and what its two means are of.
    __device__ __forceinline__ void before(const Inputs<T>& in, const Place& row, int col, Run& x, SUMS& sums) const {
        if constexpr (JOIN) {
            x.xb = value(in, in.b, col);
            if (second) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x.xb.v[i] = (x.xb.v[i] - in.after[0]) * in.after[1];
            }
            if (j.drop.share) x.kept = random.kept(col, row.row());
        }
        if (!first) return;
        x.xh = value(in, in.x, col);
        if constexpr (JOIN) {
            const Eight n = inner(x, col), f = factors(row, col);
#pragma unroll
            for (int i = 0; i < 8; ++i) x.xh.v[i] += f.v[i] * n.v[i];
        }
        x.g = value(in, in.dy, col);
        const Eight w = given.before_weight(col);
        Eight term;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.xh.v[i] = (x.xh.v[i] - in.before[0]) * in.before[1];
            term.v[i] = x.g.v[i] * x.xh.v[i];
        }
        sums.add(kBeforeWeight, term);
        sums.add(kBeforeBias, x.g);
#pragma unroll
        for (int i = 0; i < 8; ++i) x.g.v[i] *= w.v[i];
    }
    // The gradient of S, from the means of g and g xh.
    __device__ __forceinline__ void sum(const Inputs<T>& in, float2_t mean, int col, Run& x) const {
        x.ds = g.dS ? value(in, in.ds, col) : Eight{};
        if (first) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x.ds.v[i] += in.before[1] * (x.g.v[i] - mean[0] - x.xh.v[i] * mean[1]);
        }
        clear_from(x.ds, in.live ? d - col : 0);
    }
    // From there to the gradient of N1's result; returns what the gate's gradient gets.
    __device__ __forceinline__ Eight through(const Inputs<T>&, const Place& row, int col, Run& x, SUMS& sums) const {
        const Eight f = factors(row, col);
        Eight gate = {};
        if (g.dgate) {
            gate = inner(x, col);
#pragma unroll
            for (int i = 0; i < 8; ++i) gate.v[i] *= x.ds.v[i] * factor();
            sums.add(kGate, gate);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x.gb.v[i] = x.ds.v[i] * f.v[i];
        drop(x.gb, x);
        if (second) {
            const Eight w = given.after_weight(col);
            Eight term;
#pragma unroll
            for (int i = 0; i < 8; ++i) term.v[i] = x.gb.v[i] * x.xb.v[i];
            sums.add(kAfterWeight, term);
            sums.add(kAfterBias, x.gb);
#pragma unroll
            for (int i = 0; i < 8; ++i) x.gb.v[i] *= w.v[i];
        }
        return gate;
    }
};

// One pass over the rows, each in its lanes' registers, and the vectors' sums with it, a part of them from every workgroup.  The next
// row is on its way while one is computed.  128 registers are all that 1024 lanes have: in 16 bits without biases they do, with biases 48 to 68 bytes
// of a lane go to scratch memory, in fp32 12, with biases 112.  8192 x 8192 with dropout, forward and backward: bfloat16 RMS without biases 293 us, layer norms with biases 429 (a
// copy of the bytes 211); fp32 525 and 757 (421).
template <class T, int LANES, bool JOIN, bool BIAS>
__global__ __launch_bounds__(kThreadsOf<LANES>) __attribute__((amdgpu_waves_per_eu(!JOIN || LANES > 256 ? 4 : LANES > 64 ? 3 : 2))) void rsh_join_backward_kernel(rsh_join_t j, rsh_join_gradients_t g, Vectors vectors, float* parts) {
    constexpr int kThreads = kThreadsOf<LANES>, kRows = kRowsOf<LANES>;
    // Whether the registers hold the next row beside this one: a row takes about as long as its loads.
    constexpr bool kEarly = !JOIN || (size_of<T>() == 2 && !BIAS);
    __shared__ typename Team<LANES>::Meeting meeting;
    using Sums = std::conditional_t<JOIN, LdsSums<kThreads, BIAS>, RegisterSums>;
    __shared__ std::conditional_t<JOIN, typename LdsSums<kThreads, BIAS>::Place, float> place;
    __shared__ float joined[kRows > 1 ? kThreads * 8 : 1];
    Team<LANES> team(meeting);
    const Random random(j.drop);
    const int d = (int)j.d, col = 8 * (threadIdx.x % LANES);
    const KeptParameters<T, LANES == 8, BIAS> given(j, col, d);
    const Backward<T, JOIN, LANES == 8, Sums, KeptParameters<T, LANES == 8, BIAS>> back(j, g, random, given);
    Sums sums = [&] {
        if constexpr (JOIN) return Sums(place, vectors);
        else return Sums();
    }();
    const int64_t step = (int64_t)gridDim.x * kRows;
    auto load = [&](int64_t head) {
        bool live;
        const Place row = place_of<LANES>(head, j.t, &live);
        return back.load(row, live, col);
    };
    Inputs<T> next = load((int64_t)blockIdx.x * kRows);
    for (int64_t head = (int64_t)blockIdx.x * kRows; head < j.t; head += step) {
        bool live;
        const Place row = place_of<LANES>(head, j.t, &live);
        Inputs<T> in = next;
        if (kEarly && head + step < j.t) next = load(head + step);
        Run x;
        float2_t mean = {0.f, 0.f};
        back.before(in, row, col, x, sums);
        if (!kEarly && head + step < j.t) next = load(head + step);
        if (back.first) {
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a += x.g.v[i], b += x.g.v[i] * x.xh.v[i];
            mean = team.sum(a, b) * (1.f / (float)d);
            if (j.before.kind != RSH_NORM_LAYER) mean[0] = 0.f;
        }
        back.sum(in, mean, col, x);
        if (g.dX && live) store_run<T>(g.dX, row, col, d, x.ds);
        if constexpr (JOIN) {
            const Eight gate = back.through(in, row, col, x, sums);
            if (g.dgate && j.ld_gate && live) back.store_gate(row, col, gate);
            if (!g.dB) continue;
            if (back.second) {
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) a += x.gb.v[i], b += x.gb.v[i] * x.xb.v[i];
                mean = team.sum(a, b) * (1.f / (float)d);
                if (j.after.kind != RSH_NORM_LAYER) mean[0] = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x.gb.v[i] = in.after[1] * (x.gb.v[i] - mean[0] - x.xb.v[i] * mean[1]);
            }
            if (live) store_run<T>(g.dB, row, col, d, x.gb);
        }
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        if ((!JOIN && k >= kAfterWeight) || (!BIAS && (k == kBeforeBias || k == kAfterBias))) continue;
        if (vectors.at[k] >= 0) {
            float* const out = parts + ((int64_t)blockIdx.x * vectors.count + vectors.at[k]) * d;
            if constexpr (kRows == 1) {
                store_eight<F32>(out, col, sums.get(k), d - col);
            } else {
                const Eight e = sums.get(k);
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[threadIdx.x * 8 + i] = e.v[i];
                __syncthreads();
                for (int c = threadIdx.x; c < d; c += kThreads) {
                    float a = 0.f;
#pragma unroll
                    for (int r = 0; r < kRows; ++r) a += joined[r * LANES * 8 + c];
                    out[c] = a;
                }
            }
        }
    }
}

// Longer rows: this kernel forms the four means of a row, means[4 row] = those of g and g xh and those of N1's, and the next one goes through the
// columns.  N1's means are of gb = (dS + r g - r mean(g) - r xh mean(g xh)) fw with fw = w1 scale gate drop, so of (dS + r g) fw, fw and xh fw,
// which need no other mean: one pass has them all.  (With three passes over
// the rows, and a fourth for the vectors, a step of 1677 x 20000 bfloat16 took 448 us, with these two 353.)  The price is a difference of sums: where g is
// nearly a constant, 100 times its spread, dB is 3.0e-7 off in fp32 for 1.3e-7 from finished terms (8192 columns); elsewhere both are 0.8e-7.
template <class T, bool JOIN>
__global__ __launch_bounds__(1024) void rsh_join_means_kernel(rsh_join_t j, rsh_join_gradients_t g, float* means) {
    __shared__ Team<1024>::Meeting meeting;
    Team<1024> team(meeting);
    const Random random(j.drop);
    const LoadedParameters<T> given{j, (int)j.d};
    const Backward<T, JOIN, false, NoSums, LoadedParameters<T>> back(j, g, random, given);
    const int d = back.d;
    const float share = 1.f / (float)d;
    NoSums none;
    for (int64_t at = blockIdx.x; at < j.t; at += gridDim.x) {
        const Place row = {at, 0};
        float a1 = 0.f, a2 = 0.f, b1 = 0.f, b2 = 0.f, c1 = 0.f, c2 = 0.f, d1 = 0.f, d2 = 0.f;
        Inputs<T> in;
        each_run<1024, 0>(d, [&](int, int col) {
            in = back.load(row, true, col);
            Run x;
            back.before(in, row, col, x, none);
            if (back.first) {
#pragma unroll
                for (int i = 0; i < 8; ++i) a1 += x.g.v[i], a2 += x.g.v[i] * x.xh.v[i];
            }
            if (JOIN && back.second && g.dB) {
                Eight fw = back.factors(row, col), ds = g.dS ? back.value(in, in.ds, col) : Eight{};
                const Eight w = given.after_weight(col);
#pragma unroll
                for (int i = 0; i < 8; ++i) fw.v[i] *= w.v[i];
                clear_from(fw, d - col);
                back.drop(fw, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) ds.v[i] = (back.first ? ds.v[i] + in.before[1] * x.g.v[i] : ds.v[i]) * fw.v[i];
                back.drop(ds, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = fw.v[i], xb = x.xb.v[i], p = ds.v[i];
                    b1 += p, b2 += p * xb;
                    if (back.first) {
                        const float h = x.xh.v[i] * f;
                        c1 += f, c2 += f * xb, d1 += h, d2 += h * xb;
                    }
                }
            }
        });
        float2_t outer = {0.f, 0.f}, inner = {0.f, 0.f};
        if (back.first) {
            in.before = *reinterpret_cast<const float2_t*>(j.before.stats + 2 * at);
            outer = team.sum(a1, a2) * share;
            if (j.before.kind != RSH_NORM_LAYER) outer[0] = 0.f;
        }
        if (JOIN && back.second && g.dB) {
            inner = team.sum(b1, b2);
            if (back.first) inner -= in.before[1] * (outer[0] * team.sum(c1, c2) + outer[1] * team.sum(d1, d2));
            inner *= share;
            if (j.after.kind != RSH_NORM_LAYER) inner[0] = 0.f;
        }
        if (threadIdx.x == 0) *reinterpret_cast<float4_t*>(means + 4 * at) = (float4_t){outer[0], outer[1], inner[0], inner[1]};
    }
}

// A thread has eight columns of the rows of a part: their gradients, and their share of the vectors.  Nothing is waited for between rows.
template <class T, bool JOIN>
__global__ __launch_bounds__(256) void rsh_join_columns_kernel(rsh_join_t j, rsh_join_gradients_t g, Vectors vectors, float* parts,
                                                               const float* means) {
    const Random random(j.drop);
    const int d = (int)j.d, col = 8 * (int)(blockIdx.x * 256 + threadIdx.x);
    if (col >= d) return;
    const KeptParameters<T, false, true> given(j, col, d);
    const Backward<T, JOIN, false, RegisterSums, KeptParameters<T, false, true>> back(j, g, random, given);
    RegisterSums sums;
    Inputs<T> next = back.load({blockIdx.y, 0}, true, col);
    for (int64_t at = blockIdx.y; at < j.t; at += gridDim.y) {
        const Place row = {at, 0};
        const Inputs<T> in = next;
        if (at + gridDim.y < j.t) next = back.load({at + gridDim.y, 0}, true, col);
        const float4_t mean = *reinterpret_cast<const float4_t*>(means + 4 * at);
        Run x;
        back.before(in, row, col, x, sums);
        back.sum(in, (float2_t){mean[0], mean[1]}, col, x);
        if (g.dX) store_run<T>(g.dX, row, col, d, x.ds);
        if constexpr (JOIN) {
            const Eight gate = back.through(in, row, col, x, sums);
            if (g.dgate && j.ld_gate) back.store_gate(row, col, gate);
            if (!g.dB) continue;
            if (back.second) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x.gb.v[i] = in.after[1] * (x.gb.v[i] - mean[2] - x.xb.v[i] * mean[3]);
            }
            store_run<T>(g.dB, row, col, d, x.gb);
        }
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k)
        if (vectors.at[k] >= 0)
            store_eight<F32>(parts + ((int64_t)blockIdx.y * vectors.count + vectors.at[k]) * d, col, sums.get(k), d - col);
}

// f(lanes) of the kernels that have a row in registers, a run a lane: the fewest that do.
// Workgroups of the columns' kernel: as many as fit the chip at once (a step of 1677 x 20000 353 us, with 256 395, with 1024 358).
constexpr int64_t kRegisterWidth = 8192, kColumnBlocks = 512;
template <class F>
void by_width(int64_t d, F f) {
    using std::integral_constant;
    const int64_t runs = (d + 7) / 8;
    if (runs <= 8) f(integral_constant<int, 8>());
    else if (runs <= 16) f(integral_constant<int, 16>());
    else if (runs <= 32) f(integral_constant<int, 32>());
    else if (runs <= 64) f(integral_constant<int, 64>());
    else if (runs <= 128) f(integral_constant<int, 128>());
    else if (runs <= 256) f(integral_constant<int, 256>());
    else if (runs <= 512) f(integral_constant<int, 512>());
    else if (runs <= 1024) f(integral_constant<int, 1024>());
}
int64_t backward_parts(int64_t t, int64_t d);
int64_t vector_bytes(int64_t t, int64_t d, int vectors);

// Launches of one type, in a source file of its own.
template <class T>
void join_forward_of(const rsh_join_t& j, hipStream_t st);
template <class T>
void join_backward_of(const rsh_join_t& j, const rsh_join_gradients_t& g, const Vectors& v, float* parts, int64_t n, hipStream_t st);

#define RSH_JOIN_OF(T)                                                                                                                              \
    template <>                                                                                                                                     \
    void join_forward_of<T>(const rsh_join_t& j, hipStream_t st) {                                                                                   \
        join_forward_launch<T>(j, st);                                                                                    \
    }                                                                                                                   \
    template <>                                                                                                                                     \
    void join_backward_of<T>(const rsh_join_t& j, const rsh_join_gradients_t& g, const Vectors& v, float* parts, int64_t n, hipStream_t st) {        \
        join_backward_launch<T>(j, g, v, parts, n, st);                                                                                              \
    }

template <class T>
void join_forward_launch(const rsh_join_t& j, hipStream_t st) {
    if (j.d > kRegisterWidth) {
        // Joins keep a row in registers up to 32768 columns, or read it again, from the caches, at every pass.  With both norms and a gate, in us, the former
        // and the latter of 10240, 16384, 20000 and 28672 columns (67 MB a tensor): bfloat16 93 118, 67 96, 107 107, 83 118; fp32, where 108 to 136 bytes
        // of a lane go to scratch memory, 85 85, 73 98, 101 106, 89 110.  A sum and a norm: bfloat16 69 73, 57 65, 81 68, 63 76; fp32 70 60, 66 82, 86 86, 77 91.
        // A norm alone: bfloat16 35 26, 29 26, 42 26, 33 29; fp32 31 26, 26 28, 35 31, 31 33: read again.
        const dim3 rows((unsigned)std::min<int64_t>(j.t, 1 << 16));
        if (!j.B) hipLaunchKernelGGL((rsh_join_forward_long_kernel<T, 1024, 0, false>), rows, dim3(1024), 0, st, j);
        else if (j.d <= 2 * kRegisterWidth) hipLaunchKernelGGL((rsh_join_forward_long_kernel<T, 512, 4, true>), rows, dim3(512), 0, st, j);
        else if (j.d <= 4 * kRegisterWidth) hipLaunchKernelGGL((rsh_join_forward_long_kernel<T, 1024, 4, true>), rows, dim3(1024), 0, st, j);
        else hipLaunchKernelGGL((rsh_join_forward_long_kernel<T, 1024, 0, true>), rows, dim3(1024), 0, st, j);
        return;
    }
    by_width(j.d, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const unsigned blocks = (unsigned)std::min<int64_t>((j.t + kRowsOf<L> - 1) / kRowsOf<L>, 256 * (2048 / kThreadsOf<L>));
        if (j.B) hipLaunchKernelGGL((rsh_join_forward_kernel<T, L, true>), dim3(blocks), dim3(kThreadsOf<L>), 0, st, j);
        else hipLaunchKernelGGL((rsh_join_forward_kernel<T, L, false>), dim3(blocks), dim3(kThreadsOf<L>), 0, st, j);
    });
}

template <class T>
void join_backward_launch(const rsh_join_t& j, const rsh_join_gradients_t& g, const Vectors& v, float* parts, int64_t n, hipStream_t st) {
    if (j.d > kRegisterWidth) {
        float* const means = (float*)((char*)g.work + vector_bytes(j.t, j.d, v.count));
        const dim3 rows((unsigned)std::min<int64_t>(j.t, 1 << 16)), columns((unsigned)((j.d + 2047) / 2048), (unsigned)n);
        if (j.B) hipLaunchKernelGGL((rsh_join_means_kernel<T, true>), rows, dim3(1024), 0, st, j, g, means);
        else hipLaunchKernelGGL((rsh_join_means_kernel<T, false>), rows, dim3(1024), 0, st, j, g, means);
        if (j.B) hipLaunchKernelGGL((rsh_join_columns_kernel<T, true>), columns, dim3(256), 0, st, j, g, v, parts, means);
        else hipLaunchKernelGGL((rsh_join_columns_kernel<T, false>), columns, dim3(256), 0, st, j, g, v, parts, means);
        return;
    }
    const bool bias = v.at[kBeforeBias] >= 0 || v.at[kAfterBias] >= 0 || j.after.bias;
    by_width(j.d, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const dim3 grid((unsigned)n), block(kThreadsOf<L>);
        auto launch = [&](auto b) {
            if (j.B) hipLaunchKernelGGL((rsh_join_backward_kernel<T, L, true, decltype(b)::value>), grid, block, 0, st, j, g, v, parts);
            else hipLaunchKernelGGL((rsh_join_backward_kernel<T, L, false, decltype(b)::value>), grid, block, 0, st, j, g, v, parts);
        };
        if constexpr (L >= 256) {
            if (bias) launch(std::true_type());
            else launch(std::false_type());
        } else {
            launch(std::true_type());
        }
    });
}

}  // namespace rsh
