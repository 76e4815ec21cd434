// Products of the feed-forward block: activations with weights in 16 or 4 bits, the gated block, and its gradients.
//
// Every product is C[r][c] = sum over k of Q[r][k] P[c][k], rows r of the result (tokens, or hidden features where a weight's
// gradient is formed) by columns c, in fp32 on the matrix units with one rounding at the end:
//   product    Q = X [t][d]             P = W [n][d]                  both with k running along memory
//   gated      Q = X [t][d]             P = Wg and Wu [f][d]          G and U side by side; H = act(G) U before the rounding
//   dX         Q = dG, then dU [t][f]   P = Wg, then Wu [f][d]        k runs along memory in Q, across it in P; two sums in one
//   dWg, dWu   Q = dG / dU [t][f]       P = X [t][d]                  k (tokens) runs across memory in both
// P is the first operand of the matrix instruction, so a lane ends up with runs of four columns of one row.
#include <algorithm>

#include "../../include/rsh_spmm.h"
#include "ffn.hpp"

namespace rsh {

namespace {

struct Shape {
    int64_t rows, cols, k;         // of one product
    int tiles_r, tiles_c;
};

constexpr int kRowBytes = 128;     // of k in one step: 64 elements of 16 bits, 256 of 4

// Sixteen scales of which `valid` exist; the others are 0.
__device__ __forceinline__ uint4_t load_scales16(const uint8_t* p, int64_t valid) {
    uint4_t v = {0, 0, 0, 0};
    if (valid >= 16) {
        __builtin_memcpy(&v, p, 16);
    } else {
        for (int i = 0; i < valid; ++i) {
            const uint32_t byte = (uint32_t)p[i] << (8 * (i & 3));
            v[0] |= i / 4 == 0 ? byte : 0u;
            v[1] |= i / 4 == 1 ? byte : 0u;
            v[2] |= i / 4 == 2 ? byte : 0u;
            v[3] |= i / 4 == 3 ? byte : 0u;
        }
    }
    return v;
}

// Value of the other lane of a pair.
__device__ __forceinline__ int swap_pair(int v) { return __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, false); }

__device__ __forceinline__ half4_t read_transposed(const unsigned char* p) {
    return __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4_t __attribute__((address_space(3)))*)p));
}

// Byte of chunk c (16 bytes) of row r in LDS.  Rows of kRowBytes with k along them are read by 32 lanes at a time, a row each,
// and rows with k across by 16 lanes, four rows each: the chunks of neighbouring rows are dealt to other banks.
__device__ __forceinline__ int along_at(int r, int c) { return r * kRowBytes + ((c ^ (r & 7)) << 4); }
template <int WIDTH>
__device__ __forceinline__ int across_at(int k, int c) {
    return k * (2 * WIDTH) + ((c ^ ((k & 7) << 1 & (WIDTH / 8 - 1))) << 4);
}

// Chunks of one operand's tile on their way through registers into LDS: codes, which are turned into 16 bits, and rows that do not
// lie at 16-byte boundaries.  Offsets are 32 bits from the tile's first element (launches see to it that they fit).  Lines past the
// operand's last are read as that one: only what lies past k has to be zero, in both operands, since rows and columns past the
// result's end are not kept.
template <Form FORM, int WIDTH, int THREADS, bool PAIR>
struct Stage {
    static constexpr int kChunks = FORM == kCodes ? WIDTH * 2 / THREADS : WIDTH * 8 / THREADS;
    static_assert(kChunks > 0);
    uint4_t v[kChunks];
    uint32_t s[FORM == kCodes ? kChunks : 1];
    uint32_t line[kChunks];        // byte of the chunk's line (kCodes: of its scales)
    int64_t first, stride;         // bytes to the tile's first element, from line to line
    int64_t span;                  // from there to the operand's end
    int chunk;                     // in its line; the same for all chunks of a thread

    // Which of two matrices, where they run side by side: 32 lines of one, then 32 of the other.
    static __device__ __forceinline__ int matrix(int j) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return PAIR ? (wave + THREADS / 64 * j) >> (FORM == kCodes ? 0 : 2) & 1 : 0;
    }
    __device__ __forceinline__ void start(const Operand& o, int64_t tile, int64_t extent, int64_t k) {
        const int64_t width = PAIR ? WIDTH / 2 : WIDTH, left = extent - tile * width;
        stride = FORM == kCodes ? o.ld : 2 * o.ld;
        if constexpr (FORM == kAcross) {
            chunk = threadIdx.x % (WIDTH / 8);
            first = 2 * tile * width;
            span = (k - 1) * stride + 2 * left;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) line[j] = (uint32_t)((threadIdx.x + THREADS * j) / (WIDTH / 8) * stride);
        } else {
            constexpr int kIn = FORM == kCodes ? 2 : 8;       // chunks of a line
            chunk = threadIdx.x % kIn;
            first = tile * width * stride;
            span = (left - 1) * stride + 2 * k;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const int i = (threadIdx.x + THREADS * j) / kIn, at = PAIR ? (i >> 6) * 32 + (i & 31) : i;
                line[j] = (uint32_t)(min((int64_t)at, left - 1) * stride);
            }
        }
    }
    __device__ __forceinline__ void load(const Operand& o, int seg, int64_t k0) {
        if constexpr (FORM == kCodes) {
            const uint32_t b = (uint32_t)min(k0 / kBlock + chunk, o.ld - 1);
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                v[j] = *reinterpret_cast<const uint4_t*>((const uint8_t*)o.data[matrix(j)] + first * kBlockBytes + (line[j] + b) * kBlockBytes);
                s[j] = (o.scales[matrix(j)] + first)[line[j] + b];
            }
        } else {
            const int64_t ahead = FORM == kAlong ? 2 * k0 : k0 * stride;
            const int last = (int)min(span - ahead - 16, (int64_t)0x7ffffff0);      // below 0 where less than 16 bytes are left
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const uint8_t* const base = (const uint8_t*)o.data[PAIR ? matrix(j) : seg] + first + ahead;
                if (__builtin_expect(span >= 16, 1)) {      // a chunk that the operand's end cuts is read as its last 16 bytes
                    v[j] = *reinterpret_cast<const uint4_a2*>(base + min((int)line[j] + 16 * chunk, last));
                } else {               // seven elements at most
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t x = *reinterpret_cast<const uint16_t*>(base + min((int64_t)line[j] + 16 * chunk + 2 * e, span - ahead - 2));
                        v[j][e / 2] = e & 1 ? v[j][e / 2] | x << 16 : x;
                    }
                }
            }
        }
    }
    // In the last step: the elements of a cut chunk go to its front, what lies past k becomes zero.
    __device__ __forceinline__ void trim(const Operand& o, int64_t k0, int64_t k) {
        if (k0 + 64 < k) return;
        const int left = (int)(k - k0), end = (int)(span - (FORM == kAlong ? 2 * k0 : k0 * stride)) - 16;     // of k; of the operand's bytes
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            if constexpr (FORM == kCodes) {
                if (k0 / kBlock + chunk >= o.ld) v[j] = (uint4_t){0, 0, 0, 0}, s[j] = 0;
            } else {
                const int past = (int)line[j] + 16 * chunk - end, drop = span >= 16 ? max(0, min(past, 16)) / 2 : 0;
                const int keep = FORM == kAlong ? left - 8 * chunk : (int)(threadIdx.x + THREADS * j) / (WIDTH / 8) < left ? 8 : 0;
                uint4_t x = v[j];
                if (drop & 4) x = (uint4_t){x[2], x[3], 0, 0};
                if (drop & 2) x = (uint4_t){x[1], x[2], x[3], 0};
                if (drop & 1) x = (uint4_t){x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
#pragma unroll
                for (int w = 0; w < 4; ++w) x[w] &= (2 * w < keep ? 0xffffu : 0u) | (2 * w + 1 < keep ? 0xffff0000u : 0u);
                v[j] = x;
            }
        }
    }
    // shift: added to the scale bytes of a thread's rows (kCodes; rows stay a thread's own through all steps)
    template <class T>
    __device__ __forceinline__ void store(unsigned char* lds, const int* shift) const {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int i = threadIdx.x + THREADS * j;
            if constexpr (FORM == kAcross) {
                *reinterpret_cast<uint4_t*>(lds + across_at<WIDTH>(i / (WIDTH / 8), i % (WIDTH / 8))) = v[j];
            } else if constexpr (FORM == kCodes) {
                const float scale = scale_of(s[j] == 255u ? 255u : (uint32_t)max(0, (int)s[j] + shift[j]));
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    *reinterpret_cast<uint4_t*>(lds + along_at(i >> 1, 4 * (i & 1) + c)) = from_codes8<T>(v[j][c], scale);
            } else {
                *reinterpret_cast<uint4_t*>(lds + along_at(i >> 3, i & 7)) = v[j];
            }
        }
    }
};

// 16 bytes a lane from byte `at` of a buffer of `size` bytes to the lane's place behind `lds`; zero past the buffer's end.  (The
// host's pass over this file does not know the type of a buffer's description.)
__device__ __forceinline__ void load_to_lds([[maybe_unused]] const uint8_t* buffer, [[maybe_unused]] uint32_t size, [[maybe_unused]] uint32_t at,
                                            [[maybe_unused]] unsigned char* lds) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)buffer, 0, size, 0x00020000),
                                             (__attribute__((address_space(3))) void*)lds, 16, at, 0, 0, 0);
#endif
}

// The same straight into LDS: 16 bytes a lane, 1 KB a wave and turn, in the order of the lanes, so the chunks are dealt to their
// banks by the lane's choice of source.  Reads past the operand's end come back as zero (the buffer's range check); rows must be
// whole chunks at 16-byte boundaries.
template <Form FORM, int WIDTH, int THREADS, bool PAIR>
struct Direct {
    static constexpr int kChunks = WIDTH * 8 / THREADS;
    static constexpr uint32_t kNowhere = 0x80000000u;      // past every buffer
    uint32_t at[kChunks];          // byte of the lane's chunks from the tile's first, at k = 0
    int64_t first, span, stride;   // byte of the tile's first row (kAcross: column), bytes from there to the operand's end, row to row
    int chunk;                     // chunk of its row that a lane loads (kAlong, kFours); the same in every turn

    __device__ __forceinline__ void start(const Operand& o, int64_t tile, int64_t extent, int64_t k) {
        const int64_t width = PAIR ? WIDTH / 2 : WIDTH;
        stride = FORM == kFours ? o.ld * kBlockBytes : o.ld * 2;
        if constexpr (FORM == kAcross) {
            chunk = 0;
            first = tile * width * 2;
            span = (k - 1) * stride + (extent - tile * width) * 2;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const int i = threadIdx.x + THREADS * j, kk = i / (WIDTH / 8), c = i % (WIDTH / 8) ^ ((kk & 7) << 1 & (WIDTH / 8 - 1));
                at[j] = tile * width + 8 * c < extent ? (uint32_t)(kk * stride + 16 * c) : kNowhere;
            }
        } else {
            chunk = (threadIdx.x & 7) ^ (threadIdx.x >> 3 & 7);
            first = tile * width * stride;
            span = (extent - tile * width - 1) * stride + (FORM == kFours ? stride : 2 * k);
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const int r = (threadIdx.x + THREADS * j) >> 3;
                at[j] = (uint32_t)((PAIR ? (r >> 6) * 32 + (r & 31) : r) * stride + 16 * chunk);
            }
        }
    }
    __device__ __forceinline__ void issue(const Operand& o, int seg, int64_t k0, int64_t k, unsigned char* lds) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t ahead = FORM == kAcross ? k0 * stride : FORM == kFours ? k0 / 2 : k0 * 2;
        const uint32_t left = (uint32_t)min(span - ahead, (int64_t)0x7ffffff0);
        const bool in = FORM == kAcross || k0 + (FORM == kFours ? 32 : 8) * chunk < k;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int which = PAIR ? (wave + THREADS / 64 * j) >> 2 & 1 : seg;
            load_to_lds((const uint8_t*)o.data[which] + first + ahead, left, in ? at[j] : kNowhere, lds + (wave * 64 + THREADS * j) * 16);
        }
    }
};

// All of a wave's loads into LDS have arrived and its reads of LDS are done; then all waves'.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The 16 bytes of an operand that a lane feeds to the matrix unit: row `base` + lane % 32 of the tile, step s.
template <Form FORM, int WIDTH>
__device__ __forceinline__ uint4_t fragment(const unsigned char* lds, int base, int s, int lane) {
    if constexpr (FORM == kAcross) {
        const int k = 16 * s + 8 * (lane >> 5) + (lane >> 2 & 3), col = base + (lane & 16) + 4 * (lane & 3);
        const half4_t a = read_transposed(lds + across_at<WIDTH>(k, col >> 3) + 2 * (col & 7));
        const half4_t b = read_transposed(lds + across_at<WIDTH>(k + 4, col >> 3) + 2 * (col & 7));
        return __builtin_bit_cast(uint4_t, (half8_t){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
    } else {
        return *reinterpret_cast<const uint4_t*>(lds + along_at(base + (lane & 31), 2 * s + (lane >> 5)));
    }
}

constexpr int kSpan = 10;   // binary16: the largest scale of a row of codes is brought to 2^kSpan

}  // namespace

// A part of the steps of k, whose sums go to `partial` as fp32 [part][result][row][columns rounded up to 4, gate before up], where
// there is more than one.
struct Split {
    int parts;
    int64_t steps;         // of one part
    float* partial;
};

// T: F16 or BF16 (results, and operands unless they are kFours).  WP x WQ waves, each TP x TQ tiles of 32 x 32.  DIRECT: operands
// that need no conversion go straight into LDS.
template <class T, Form FP, Form FQ, bool GATED, int SEGS, int WP, int WQ, int TP, int TQ, bool DIRECT>
__global__ __launch_bounds__(64 * WP * WQ) void rsh_product_kernel(Operand P, Operand Q, Result res, Shape sh, Split split) {
    constexpr int kThreads = 64 * WP * WQ, kWidthP = 32 * WP * TP, kWidthQ = 32 * WQ * TQ;
    constexpr int kBytesP = kWidthP * kRowBytes, kBytesQ = kWidthQ * kRowBytes;
    constexpr int kStep = FP == kFours ? 256 : 64;       // k of a step
    constexpr bool kShifted = FP == kCodes && std::is_same<T, F16>::value;
    constexpr bool kScaled = FP == kFours;
    constexpr bool kDirectP = DIRECT && FP != kCodes;
    constexpr int kTurns = kScaled ? (kWidthP + kWidthQ + kThreads - 1) / kThreads : 1;
    using StageP = Stage<FP, kWidthP, kThreads, GATED>;
    using StageQ = Stage<FQ, kWidthQ, kThreads, false>;
    __shared__ __attribute__((aligned(16))) unsigned char lds[2][kBytesP + kBytesQ];
    __shared__ uint2_t scales[kScaled ? 2 : 1][kScaled ? kWidthP + kWidthQ : 1];
    __shared__ int tops[kShifted ? kWidthP : 1];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % WP, wq = wave / WP;
    // Tiles are dealt to the XCDs in runs of their order, which goes through eight tiles of rows before the next column, so that
    // the workgroups of an XCD share rows of both operands in its L2.
    const int64_t tiles = (int64_t)sh.tiles_r * sh.tiles_c, chunk = (tiles + 7) / 8;
    const int64_t tile = (int64_t)(blockIdx.x & 7) * chunk + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= chunk || tile >= tiles) return;
    const int64_t strip = tile / (8 * sh.tiles_c), in_strip = tile % (8 * sh.tiles_c), tall = min((int64_t)8, sh.tiles_r - 8 * strip);
    const int64_t tr = 8 * strip + in_strip % tall, tc = in_strip / tall;
    const int second = SEGS == 1 ? blockIdx.z : 0;       // which of two results that share P

    std::conditional_t<kDirectP, Direct<FP, kWidthP, kThreads, GATED>, StageP> sp;
    std::conditional_t<DIRECT, Direct<FQ, kWidthQ, kThreads, false>, StageQ> sq;
    sp.start(P, tc, sh.cols, sh.k);
    sq.start(Q, tr, sh.rows, sh.k);
    int shift[StageP::kChunks] = {};
    if constexpr (kShifted) {
        // the largest scale of each row within the part's k; two threads share a row, 16 blocks each in turn
        const int64_t b0 = blockIdx.y * split.steps * (kStep / kBlock), b1 = min(P.ld, b0 + split.steps * (kStep / kBlock));
#pragma unroll
        for (int j = 0; j < StageP::kChunks; ++j) {
            const int i = threadIdx.x + kThreads * j;
            const uint8_t* const at = P.scales[sp.matrix(j)] + sp.first + sp.line[j];
            int top = 0;
            for (int64_t b = b0 + 16 * (i & 1); b < b1; b += 32) {
                const uint4_t v = load_scales16(at + b, b1 - b);
#pragma unroll
                for (int w = 0; w < 16; ++w) {
                    const int s = v[w / 4] >> (8 * (w & 3)) & 255;
                    top = max(top, s == 255 ? 0 : s);
                }
            }
            top = max(top, swap_pair(top));
            shift[j] = 127 + kSpan - top;
            if ((i & 1) == 0) tops[i >> 1] = top;
        }
    }

    float16_t acc[TP][TQ];
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TQ; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

    const int64_t steps = (sh.k + kStep - 1) / kStep;
    const int64_t begin = blockIdx.y * split.steps, end = min(SEGS * steps, begin + split.steps);
    uint2_t sc[kTurns];
    auto load = [&](int64_t step, int buf) {
        const int seg = SEGS == 2 ? (int)(step >= steps) : 0;
        const int64_t k0 = (SEGS == 2 ? step - seg * steps : step) * kStep;
        if constexpr (kDirectP) sp.issue(P, seg, k0, sh.k, lds[buf]);
        else sp.load(P, seg, k0);
        if constexpr (DIRECT) sq.issue(Q, SEGS == 2 ? seg : second, k0, sh.k, lds[buf] + kBytesP);
        else sq.load(Q, SEGS == 2 ? seg : second, k0);
        if constexpr (kScaled) {
            // the eight scales of one row of either operand
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int i = threadIdx.x + kThreads * u;
                sc[u] = (uint2_t){0, 0};
                const Operand& o = i < kWidthP ? P : Q;
                const int64_t row = i < kWidthP ? tc * kWidthP + i : tr * kWidthQ + (i - kWidthP), b = k0 / kBlock;
                if (i >= kWidthP + kWidthQ || row >= (i < kWidthP ? sh.cols : sh.rows)) continue;
                const uint8_t* const at = o.scales[0] + row * o.ld + b;
                if (b + 8 <= o.ld) {
                    __builtin_memcpy(&sc[u], at, 8);
                } else {
#pragma unroll
                    for (int j = 0; j < 7; ++j)
                        if (b + j < o.ld) sc[u][j / 4] |= (uint32_t)at[j] << (8 * (j & 3));
                }
            }
        }
    };
    auto store = [&](int64_t step, int buf) {
        const int64_t k0 = (SEGS == 2 && step >= steps ? step - steps : step) * kStep;
        if constexpr (!kDirectP) {
            sp.trim(P, k0, sh.k);
            sp.template store<T>(lds[buf], shift);
        }
        if constexpr (!DIRECT) {
            sq.trim(Q, k0, sh.k);
            sq.template store<T>(lds[buf] + kBytesP, nullptr);
        }
        if constexpr (kScaled) {
#pragma unroll
            for (int u = 0; u < kTurns; ++u)
                if (threadIdx.x + kThreads * u < kWidthP + kWidthQ) scales[buf][threadIdx.x + kThreads * u] = sc[u];
        }
    };

    if (begin < end) {
        load(begin, 0);
        store(begin, 0);
    }
    meet();
    for (int64_t step = begin; step < end; ++step) {
        const int buf = (int)((step - begin) & 1);
        if (step + 1 < end) load(step + 1, buf ^ 1);
        const unsigned char *lp = lds[buf], *lq = lds[buf] + kBytesP;
        uint2_t ea[TP], eb[TQ];     // scales of the lane's rows: lanes from 32 on have every second block
        if constexpr (kScaled) {
#pragma unroll
            for (int i = 0; i < TP; ++i) ea[i] = scales[buf][32 * (wp * TP + i) + (lane & 31)] >> (8 * (lane >> 5));
#pragma unroll
            for (int i = 0; i < TQ; ++i) eb[i] = scales[buf][kWidthP + 32 * (wq * TQ + i) + (lane & 31)] >> (8 * (lane >> 5));
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            uint4_t a[TP], b[TQ];
#pragma unroll
            for (int i = 0; i < TP; ++i) a[i] = fragment<FP == kAcross ? kAcross : kAlong, kWidthP>(lp, 32 * (wp * TP + i), s, lane);
#pragma unroll
            for (int i = 0; i < TQ; ++i) b[i] = fragment<FQ == kAcross ? kAcross : kAlong, kWidthQ>(lq, 32 * (wq * TQ + i), s, lane);
            if constexpr (kScaled) {
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j) {
                        const int8v_t fa = {(int)a[i][0], (int)a[i][1], (int)a[i][2], (int)a[i][3], 0, 0, 0, 0};
                        const int8v_t fb = {(int)b[j][0], (int)b[j][1], (int)b[j][2], (int)b[j][3], 0, 0, 0, 0};
                        // step s takes bytes 0 and 2 of the first word, then of the second
                        if (s & 1) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa, fb, acc[i][j], 4, 4, 2, ea[i][s / 2], 2, eb[j][s / 2]);
                        else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa, fb, acc[i][j], 4, 4, 0, ea[i][s / 2], 0, eb[j][s / 2]);
                    }

            } else {
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j) acc[i][j] = T::mfma32(a[i], b[j], acc[i][j]);
            }
        }
        if (step + 1 < end) store(step + 1, buf ^ 1);
        meet();
    }

    // A lane has columns 8 g + 4 (lane / 32) .. + 3, g = 0 .. 3, of row lane % 32 of every tile of 32 x 32.
    uint16_t* const out = res.out[second];
    const int64_t wide = (sh.cols + 3) / 4 * 4, ld_partial = GATED ? 2 * wide : wide;
    float* const partial = split.parts > 1 ? split.partial + ((int64_t)blockIdx.y * gridDim.z + blockIdx.z) * sh.rows * ld_partial : nullptr;
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
        const int64_t row = tr * kWidthQ + 32 * (wq * TQ + j) + (lane & 31);
        if (row >= sh.rows) continue;
#pragma unroll
        for (int i = 0; i < TP; i += GATED ? 2 : 1) {
            const int at = 32 * (wp * TP + i);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int in_tile = 8 * g + 4 * (lane >> 5);
                const int64_t col = GATED ? tc * (kWidthP / 2) + at / 2 + in_tile : tc * kWidthP + at + in_tile;
                const int64_t left = sh.cols - col;
                if (left <= 0) continue;
                float4_t x, y = {};
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    x[v] = acc[i][j][4 * g + v];
                    if constexpr (kShifted) x[v] = ldexpf(x[v], tops[at + in_tile + v] - (127 + kSpan));
                    if constexpr (GATED) {
                        y[v] = acc[i + 1][j][4 * g + v];
                        if constexpr (kShifted) y[v] = ldexpf(y[v], tops[at + 32 + in_tile + v] - (127 + kSpan));
                    }
                }
                if (partial) {
                    *reinterpret_cast<float4_t*>(partial + row * ld_partial + col) = x;
                    if constexpr (GATED) *reinterpret_cast<float4_t*>(partial + row * ld_partial + wide + col) = y;
                } else {
                    finish<T, GATED>(res, out, row, col, left, x, y);
                }
            }
        }
    }
}

// Sums of the parts in their order, and what a tile does with finished sums.  A thread has four columns.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void rsh_join_parts_kernel(const float* __restrict__ partial, Result res, int64_t rows, int64_t cols, int parts) {
    const int64_t wide = (cols + 3) / 4 * 4, ld = GATED ? 2 * wide : wide, stride = gridDim.z * rows * ld;
    const uint32_t across = (uint32_t)((cols + 1023) / 1024), row = blockIdx.x / across;
    const int64_t col = 4 * ((int64_t)(blockIdx.x % across) * 256 + threadIdx.x);
    if (col >= cols) return;
    const float* at = partial + (blockIdx.z * rows + row) * ld + col;
    float4_t x = {0.f, 0.f, 0.f, 0.f}, y = x;
    for (int p = 0; p < parts; ++p, at += stride) {
        x += *reinterpret_cast<const float4_t*>(at);
        if constexpr (GATED) y += *reinterpret_cast<const float4_t*>(at + wide);
    }
    finish<T, GATED>(res, res.out[blockIdx.z], row, col, cols - col, x, y);
}

// dU = dH act(G) and dG = dH U act'(G), eight elements a thread, rounded to the 16 bits that the matrix units take.
template <class T>
__global__ __launch_bounds__(256) void rsh_gate_backward_kernel(const uint16_t* __restrict__ dH, const uint16_t* __restrict__ G,
                                                                const uint16_t* __restrict__ U, uint16_t* __restrict__ dG,
                                                                uint16_t* __restrict__ dU, int64_t t, int64_t f, int64_t ld, int64_t ld_gate, int act) {
    const uint32_t across = (uint32_t)((ld_gate + 2047) / 2048), slab = blockIdx.x / across;
    const int64_t row = slab, col = 8 * ((int64_t)(blockIdx.x - slab * across) * 256 + threadIdx.x), at = row * ld_gate + col;
    if (row >= t || col >= ld_gate) return;
    const uint4_t h = load8(dH + row * ld + col, f - col);
    const uint4_t g = *reinterpret_cast<const uint4_t*>(G + at), u = *reinterpret_cast<const uint4_t*>(U + at);
    uint4_t a, b;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float dg[2], du[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float hv = T::widen((uint16_t)(h[w] >> 16 * e)), gv = T::widen((uint16_t)(g[w] >> 16 * e)), uv = T::widen((uint16_t)(u[w] >> 16 * e));
            float slope;
            du[e] = hv * act_of(act, gv, &slope);
            dg[e] = hv * uv * slope;
            if (col + 2 * w + e >= f) du[e] = dg[e] = 0.f;
        }
        a[w] = T::pair(dg[0], dg[1]);
        b[w] = T::pair(du[0], du[1]);
    }
    *reinterpret_cast<uint4_t*>(dG + at) = a;
    *reinterpret_cast<uint4_t*>(dU + at) = b;
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
namespace {

int launched() { return hipGetLastError() == hipSuccess ? RSH_OK : RSH_ERR_HIP; }

// Tiles and parts of k for a product.
struct Choice {
    int form;          // 0: 256 x 256 by 8 waves, 1: 128 x 128 by 4, 2: 128 columns x 64 rows by 4
    int parts;
};

constexpr int64_t kTall[3] = {256, 128, 64}, kWide[3] = {256, 128, 128};

// The form and the parts whose rounds of workgroups take the least time, in units of a step of a lone workgroup of 256 x 256:
// `steps` of k in all, `pairs`: columns come in two matrices, `results` products side by side.
Choice choose(int64_t rows, int64_t cols, int64_t steps, bool pairs, int results) {
    constexpr double step[3] = {1.0, 0.33, 0.2};      // a step of one workgroup with its neighbours on the compute unit
    constexpr int room[3] = {1, 2, 3};                 // workgroups of a compute unit
    Choice best = {0, 1};
    double least = 1e300;
    for (int form = 0; form < 3; ++form) {
        const int64_t wide = kWide[form] / (pairs ? 2 : 1);
        const int64_t tiles = ((rows + kTall[form] - 1) / kTall[form]) * ((cols + wide - 1) / wide) * results;
        for (int parts = 1; parts <= 16 && parts <= steps; parts = parts < 4 ? parts + 1 : parts * 2) {
            const int64_t each = (steps + parts - 1) / parts, work = tiles * ((steps + each - 1) / each);
            const int64_t slots = 256 * room[form];
            double t = (double)((work + slots - 1) / slots) * ((double)each * step[form] * room[form] + 4.0);
            // sums through memory: written and read once, and a launch
            if (parts > 1) t += 4.0 + 8e-6 * (double)(parts * rows * cols * results * (pairs ? 2 : 1));
            if (t < least) {
                least = t;
                best = {form, parts};
            }
        }
    }
    return best;
}

int64_t partial_bytes(const Choice& c, int64_t rows, int64_t cols, bool pairs, int results) {
    return c.parts == 1 ? 0 : (int64_t)c.parts * results * rows * ((cols + 3) / 4 * 4) * (pairs ? 2 : 1) * (int64_t)sizeof(float);
}

// Whether an operand's lines are whole chunks at 16-byte boundaries.
bool whole_chunks(const Operand& o, Form form, int64_t along) {
    if (form == kCodes || form == kFours) return true;
    return ((uintptr_t)o.data[0] | (uintptr_t)o.data[1]) % 16 == 0 && o.ld % 8 == 0 && along % 8 == 0;
}

template <class T, Form FP, Form FQ, bool GATED, int SEGS, bool DIRECT>
void launch_tiles(int form, dim3 grid, const Operand& P, const Operand& Q, const Result& res, const Shape& sh, const Split& split, hipStream_t st) {
    if (form == 0)
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, 4, 2, 2, 4, DIRECT>), grid, dim3(512), 0, st, P, Q, res, sh, split);
    else if (form == 1)
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, 2, 2, 2, 2, DIRECT>), grid, dim3(256), 0, st, P, Q, res, sh, split);
    else
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, 2, 2, 2, 1, DIRECT>), grid, dim3(256), 0, st, P, Q, res, sh, split);
}

template <class T, Form FP, Form FQ, bool GATED, int SEGS>
void product(const Operand& P, const Operand& Q, const Result& res, int64_t rows, int64_t cols, int64_t k, int results, void* work, hipStream_t st) {
    constexpr int64_t kStep = FP == kFours ? 256 : 64;
    const int64_t steps = SEGS * ((k + kStep - 1) / kStep);
    const Choice c = choose(rows, cols, steps, GATED, results);
    const int64_t wide = kWide[c.form] / (GATED ? 2 : 1), tall = kTall[c.form], each = (steps + c.parts - 1) / c.parts;
    const Shape sh = {rows, cols, k, (int)((rows + tall - 1) / tall), (int)((cols + wide - 1) / wide)};
    const Split split = {c.parts, each, (float*)work};
    const int64_t tiles = (int64_t)sh.tiles_r * sh.tiles_c;
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8), c.parts, results);
    if constexpr (FP != kFours) {
        if (!whole_chunks(P, FP, FP == kAcross ? cols : k) || !whole_chunks(Q, FQ, FQ == kAcross ? rows : k))
            launch_tiles<T, FP, FQ, GATED, SEGS, false>(c.form, grid, P, Q, res, sh, split, st);
        else launch_tiles<T, FP, FQ, GATED, SEGS, true>(c.form, grid, P, Q, res, sh, split, st);
    } else {
        launch_tiles<T, FP, FQ, GATED, SEGS, true>(c.form, grid, P, Q, res, sh, split, st);
    }
    if (c.parts > 1)
        hipLaunchKernelGGL((rsh_join_parts_kernel<T, GATED>), dim3((unsigned)((cols + 1023) / 1024 * rows), 1, results), dim3(256), 0, st,
                           (const float*)work, res, rows, cols, c.parts);
}

template <class F>
void by_half(int type, F f) {
    if (type == RSH_F16) f(F16());
    else f(BF16());
}

}  // namespace

int64_t mx4_product_work(int x_type, int64_t t, int64_t n, int64_t k) {
    const int64_t step = x_type == RSH_MX4 ? 256 : 64;
    if (takes_few(t, x_type == RSH_MX4)) return 0;
    return partial_bytes(choose(t, n, (k + step - 1) / step, false, 1), t, n, false, 1);
}

int64_t gated_forward_work(int64_t t, int64_t d, int64_t f) {
    if (takes_few(t, false)) return 0;
    return partial_bytes(choose(t, f, (d + 63) / 64, true, 1), t, f, true, 1);
}

// dG and dU, and behind them the larger of the sums of dX and of the weights' gradients (of both, or of one alone).
int64_t gated_backward_work(int64_t t, int64_t d, int64_t f) {
    const int64_t gates = 4 * t * ((f + 7) / 8 * 8);
    int64_t sums = partial_bytes(choose(t, d, 2 * ((f + 63) / 64), false, 1), t, d, false, 1);
    for (int results = 1; results <= 2; ++results)
        sums = std::max(sums, partial_bytes(choose(f, d, (t + 63) / 64, false, results), f, d, false, results));
    return gates + sums;
}

int launch_mx4_product(const void* X, const void* x_scales, int x_type, int64_t ld_x, const void* W, const void* w_scales, void* Y, int y_type,
                       int64_t t, int64_t n, int64_t k, void* work, void* stream) {
    const int64_t blocks = (k + kBlock - 1) / kBlock;
    const Operand p = {{W, nullptr}, {(const uint8_t*)w_scales, nullptr}, blocks};
    const Operand q = {{X, nullptr}, {(const uint8_t*)x_scales, nullptr}, x_type == RSH_MX4 ? blocks : ld_x};
    const Result res = {{(uint16_t*)Y, nullptr}, nullptr, nullptr, n, 0, 0};
    by_half(y_type, [&](auto half) {
        using T = decltype(half);
        if (takes_few(t, x_type == RSH_MX4)) {
            if (x_type == RSH_MX4) launch_few<T, kFours, false>(p, q, res, t, n, k, (hipStream_t)stream);
            else launch_few<T, kCodes, false>(p, q, res, t, n, k, (hipStream_t)stream);
        } else if (x_type == RSH_MX4) product<T, kFours, kFours, false, 1>(p, q, res, t, n, k, 1, work, (hipStream_t)stream);
        else product<T, kCodes, kAlong, false, 1>(p, q, res, t, n, k, 1, work, (hipStream_t)stream);
    });
    return launched();
}

int launch_gated_forward(const void* X, int type, int64_t ld_x, const void* Wg, const void* Wu, int64_t ld_w, const void* g_scales,
                         const void* u_scales, int act, void* H, void* G, void* U, int64_t t, int64_t d, int64_t f, void* work, void* stream) {
    const int64_t blocks = (d + kBlock - 1) / kBlock;
    const Operand p = {{Wg, Wu}, {(const uint8_t*)g_scales, (const uint8_t*)u_scales}, g_scales ? blocks : ld_w};
    const Operand q = {{X, nullptr}, {nullptr, nullptr}, ld_x};
    const Result res = {{(uint16_t*)H, nullptr}, (uint16_t*)G, (uint16_t*)U, f, (f + 7) / 8 * 8, act};
    by_half(type, [&](auto half) {
        using T = decltype(half);
        if (takes_few(t, false)) {
            if (g_scales) launch_few<T, kCodes, true>(p, q, res, t, f, d, (hipStream_t)stream);
            else launch_few<T, kAlong, true>(p, q, res, t, f, d, (hipStream_t)stream);
        } else if (g_scales) product<T, kCodes, kAlong, true, 1>(p, q, res, t, f, d, 1, work, (hipStream_t)stream);
        else product<T, kAlong, kAlong, true, 1>(p, q, res, t, f, d, 1, work, (hipStream_t)stream);
    });
    return launched();
}

int launch_gated_backward(const void* X, int type, int64_t ld_x, const void* Wg, const void* Wu, int64_t ld_w, const void* G, const void* U,
                          const void* dH, int64_t ld_h, int act, void* dX, void* dWg, void* dWu, int64_t t, int64_t d, int64_t f, void* work,
                          void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    const int64_t ld_gate = (f + 7) / 8 * 8, blocks = t * ((ld_gate + 2047) / 2048);
    uint16_t* const dG = (uint16_t*)work;
    uint16_t* const dU = dG + t * ld_gate;
    void* const sums = dU + t * ld_gate;
    const Operand gates = {{dG, dU}, {nullptr, nullptr}, ld_gate};
    by_half(type, [&](auto half) {
        using T = decltype(half);
        hipLaunchKernelGGL(rsh_gate_backward_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, (const uint16_t*)dH, (const uint16_t*)G,
                           (const uint16_t*)U, dG, dU, t, f, ld_h, ld_gate, act);
        if (dX) {
            const Operand w = {{Wg, Wu}, {nullptr, nullptr}, ld_w};
            const Result res = {{(uint16_t*)dX, nullptr}, nullptr, nullptr, d, 0, 0};
            product<T, kAcross, kAlong, false, 2>(w, gates, res, t, d, f, 1, sums, st);
        }
        if (dWg || dWu) {
            const Operand x = {{X, nullptr}, {nullptr, nullptr}, ld_x}, only_u = {{dU, nullptr}, {nullptr, nullptr}, ld_gate};
            const Result res = {{(uint16_t*)(dWg ? dWg : dWu), (uint16_t*)dWu}, nullptr, nullptr, d, 0, 0};
            product<T, kAcross, kAcross, false, 1>(x, dWg ? gates : only_u, res, f, d, t, dWg && dWu ? 2 : 1, sums, st);
        }
    });
    return launched();
}

}  // namespace rsh
