// The edges of a block: launches of norms and joins, the sums of their vectors' gradients, and dropout alone.
//
// Dropout reads and writes each element once; ten rounds for eight elements are about 20 instructions' time an element, below what memory takes:
// 4096 x 16384 bfloat16 46.4 us, 1999 x 4999 fp32 14.0 us (5.8 and 5.7 TB/s; part of it stays in the last-level cache).
#include "join.hpp"

namespace rsh {

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
        if (drop.share) random.drop(e, (int)col, row, random.keep);
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
}  // namespace

template <> void join_forward_of<F32>(const rsh_join_t&, hipStream_t);
template <> void join_forward_of<F16>(const rsh_join_t&, hipStream_t);
template <> void join_forward_of<BF16>(const rsh_join_t&, hipStream_t);
template <> void join_backward_of<F32>(const rsh_join_t&, const rsh_join_gradients_t&, const Vectors&, float*, int64_t, hipStream_t);
template <> void join_backward_of<F16>(const rsh_join_t&, const rsh_join_gradients_t&, const Vectors&, float*, int64_t, hipStream_t);
template <> void join_backward_of<BF16>(const rsh_join_t&, const rsh_join_gradients_t&, const Vectors&, float*, int64_t, hipStream_t);

// Workgroups of the backward pass, each with a part of the vectors' sums, or parts of the columns' kernel: what fits the chip at once (twice as many
// 310 us for 294 in a step of 8192 x 8192, 155 for 147 of 2^20 x 64; half as many 180 for 177 of 16384 x 2048, 144 for 147 of 2^20 x 64).
int64_t backward_parts(int64_t t, int64_t d) {
    if (d > kRegisterWidth) return std::min<int64_t>(t, std::max<int64_t>(1, kColumnBlocks / ((d + 2047) / 2048)));
    int64_t parts = 0;
    by_width(d, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        parts = std::min<int64_t>((t + kRowsOf<L> - 1) / kRowsOf<L>, 256 * ((L <= 64 ? 2048 : 1024) / kThreadsOf<L>));
    });
    return parts;
}
int64_t vector_bytes(int64_t t, int64_t d, int vectors) { return (backward_parts(t, d) * vectors * d * 4 + 15) / 16 * 16; }

int64_t join_backward_work(int64_t t, int64_t d, int vectors) {
    return vector_bytes(t, d, vectors) + (d > kRegisterWidth ? 16 * t : 0);
}

int launch_join_forward(const rsh_join_t& join, void* stream) {
    by_type(join.type, [&](auto type) { join_forward_of<decltype(type)>(join, (hipStream_t)stream); });
    return launched();
}

int launch_join_backward(const rsh_join_t& join, const rsh_join_gradients_t& g, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    Vectors v = {{g.before_weight, g.before_bias, g.after_weight, g.after_bias, join.ld_gate ? nullptr : g.dgate},
                 {join.before.weight_type, join.before.bias_type, join.after.weight_type, join.after.bias_type, join.gate_type}, {}, 0};
    for (int k = 0; k < kSlots; ++k) v.at[k] = v.out[k] ? v.count++ : -1;
    float* const parts = (float*)g.work;
    const int64_t n = backward_parts(join.t, join.d);
    by_type(join.type, [&](auto type) { join_backward_of<decltype(type)>(join, g, v, parts, n, st); });
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
