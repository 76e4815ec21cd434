// Products of the feed-forward block: activations with weights in 16 or 4 bits, the gated block, and its gradients.
//
// Every product is C[r][c] = sum over k of Q[r][k] P[c][k], rows r of the result (tokens, or hidden features where a weight's
// gradient is formed) by columns c, in fp32 on the matrix units with one rounding at the end:
//   product    Q = X [t][d]             P = W [n][d]                  both with k running along memory
//   gated      Q = X [t][d]             P = Wg and Wu [f][d]          G and U side by side; H = act(G) U before the rounding
//   dX         Q = dG, then dU [t][f]   P = Wg, then Wu [f][d]        k runs along memory in Q, across it in P; two sums in one
//   dWg, dWu   Q = dG / dU [t][f]       P = X [t][d]                  k (tokens) runs across memory in both
// P is the first operand of the matrix instruction, so a lane ends up with runs of four columns of one row.
//
// Tiles of 256 x 256 need 64 KB of operands for every 64 k, eight waves of 64 x 128 read 96 KB of them out of LDS in 2048 cycles of
// products, and a compute unit holds one such workgroup; smaller products take tiles of 128 x 128 or 128 x 64, and k in parts.  What
// bounds the large ones is power: with X all zeros the same launch runs a quarter faster, since the clock stays up.
// Measured (bfloat16 unless said): 2048 tokens through a gated block of 8192 x 28672 1.49 ms, 1290 TFLOP/s where the library's product
// of the same shape alone runs at 1490; a training step of 4096 tokens on 4096 x 16384 2.85 ms, 1160 TFLOP/s with dX at 1290 and the
// weights' gradients at 1260 (the library's products: 1190 and 1000); 4096 tokens through 28672 x 8192, 4 bits on both sides 0.65 ms,
// 2950 TFLOP/s; 128 tokens through 8192 x 28672 in 4 bits beside binary16 99 us, where four parts of k and a slice's latency count.
#include <algorithm>

#include "../../include/rsh_spmm.h"
#include "ffn.hpp"

namespace rsh {

namespace {

struct Shape {
    int64_t rows, cols, k;         // of one product
    int tiles_r, tiles_c;
};

// A part of the slices of k, whose sums go to `partial` as fp32 [part][result][row][columns rounded up to 4, gate before up], where
// there is more than one.
struct Split {
    int parts, slices;             // slices of a part
    float* partial;
};

constexpr int kSpan = 10;          // binary16: the largest scale of a row of codes is brought to 2^kSpan

__device__ __forceinline__ half4_t read_transposed(const unsigned char* p) {
    return __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4_t __attribute__((address_space(3)))*)p));
}

// Byte of chunk c (16 bytes) of row r of a slice in LDS.  The 64 banks are 256 bytes wide, two or four rows of ROW bytes: 16 lanes
// that read a chunk of as many rows at once shall find the 16 different chunks of that width, and so shall 32 lanes that read halves
// of four chunks in four rows with k across.
template <int ROW>
__device__ __forceinline__ int along_turn(int r) {
    return ROW == 128 ? r >> 1 & 7 : r >> 2 & 3;
}
template <int WIDTH>
__device__ __forceinline__ int across_turn(int k) {
    return WIDTH >= 128 ? (k & 3) << 2 ^ (k >> 3 & 1) << 1 : (k >> 1 & 1) << 2 ^ (k >> 3 & 1) << 1;
}
template <int ROW>
__device__ __forceinline__ int along_at(int r, int c) {
    return r * ROW + ((c ^ along_turn<ROW>(r)) << 4);
}
template <int WIDTH>
__device__ __forceinline__ int across_at(int k, int c) {
    return k * (2 * WIDTH) + ((c ^ across_turn<WIDTH>(k)) << 4);
}
// Place of a row of codes, 16 bytes a slice, where two matrices run side by side: a wave loads 64 rows of one of them.
template <bool PAIR>
__device__ __forceinline__ int codes_place(int r) {
    return PAIR ? (r >> 7) * 128 + (r >> 5 & 1) * 64 + (r >> 6 & 1) * 32 + (r & 31) : r;
}
template <bool PAIR>
__device__ __forceinline__ int codes_row(int place) {
    return PAIR ? (place >> 7) * 128 + (place >> 5 & 1) * 64 + (place >> 6 & 1) * 32 + (place & 31) : place;
}
// Line of its own matrix that row i of a tile is: 32 rows of the one, then 32 of the other.
template <bool PAIR>
__device__ __forceinline__ int line_of(int i) {
    return PAIR ? (i >> 6) * 32 + (i & 31) : i;
}

// Chunks of one operand's slice on their way through registers into LDS, for rows that do not lie at 16-byte boundaries.  Offsets
// are 32 bits from the tile's first element (launches see to it that they fit).  Lines past the operand's last are read as that
// one: only what lies past k has to be zero, in both operands, since rows and columns past the result's end are not kept.
template <Form FORM, int ROW, int WIDTH, int THREADS, bool PAIR>
struct Stage {
    static constexpr int kIn = ROW / 16, kSlice = ROW / 2;      // chunks of a row, k of a slice
    static constexpr int kChunks = WIDTH * kIn / THREADS;
    uint4_t v[2][kChunks];         // slices of even and odd number
    uint32_t line[kChunks];        // byte of the chunk's line
    const uint8_t* base[2];        // the tile's first element of either matrix
    int64_t stride;                // bytes from line to line
    int64_t span;                  // from the first element to the operand's end
    int chunk;                     // in its line; the same for all chunks of a thread

    static __device__ __forceinline__ int matrix(int j) { return PAIR ? __builtin_amdgcn_readfirstlane((threadIdx.x + THREADS * j) / (32 * kIn)) & 1 : 0; }
    __device__ __forceinline__ void start(const Operand& o, int64_t tile, int64_t extent, int64_t k) {
        const int64_t width = PAIR ? WIDTH / 2 : WIDTH, left = extent - tile * width;
        stride = 2 * o.ld;
        const int64_t first = tile * width * (FORM == kAcross ? 2 : stride);
        base[0] = (const uint8_t*)o.data[0] + first;
        base[1] = (const uint8_t*)o.data[1] + first;
        if constexpr (FORM == kAcross) {
            chunk = threadIdx.x % (WIDTH / 8);
            span = (k - 1) * stride + 2 * left;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) line[j] = (uint32_t)((threadIdx.x + THREADS * j) / (WIDTH / 8) * stride);
        } else {
            chunk = threadIdx.x % kIn;
            span = (left - 1) * stride + 2 * k;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) line[j] = (uint32_t)(min((int64_t)line_of<PAIR>((threadIdx.x + THREADS * j) / kIn), left - 1) * stride);
        }
    }
    __device__ __forceinline__ void load(int odd, int seg, int64_t k0) {
        const int64_t ahead = FORM == kAlong ? 2 * k0 : k0 * stride;
        const int last = (int)min(span - ahead - 16, (int64_t)0x7ffffff0);      // below 0 where less than 16 bytes are left
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const uint8_t* const at = ((PAIR ? matrix(j) : seg) ? base[1] : base[0]) + ahead;
            if (__builtin_expect(span >= 16, 1)) {      // a chunk that the operand's end cuts is read as its last 16 bytes
                v[odd][j] = *reinterpret_cast<const uint4_a2*>(at + min((int)line[j] + 16 * chunk, last));
            } else {                                    // seven elements at most
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = *reinterpret_cast<const uint16_t*>(at + min((int64_t)line[j] + 16 * chunk + 2 * e, span - ahead - 2));
                    v[odd][j][e / 2] = e & 1 ? v[odd][j][e / 2] | x << 16 : x;
                }
            }
        }
    }
    // Into LDS.  The elements of a cut chunk go to its front, and what lies past k becomes zero.  Both are of the last slice, but for k
    // across lines of one to three elements: a chunk then runs through lines behind its own, and the operand's end cuts those of the last
    // seven lines, some of which the slice before may have.
    __device__ __forceinline__ void store(int odd, int64_t k0, int64_t k, unsigned char* lds) {
        const int left = (int)min(k - k0, (int64_t)kSlice), end = (int)min(span - (FORM == kAlong ? 2 * k0 : k0 * stride) - 16, (int64_t)0x7ffffff0);
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int i = threadIdx.x + THREADS * j;
            uint4_t x = v[odd][j];
            if (k0 + kSlice + (FORM == kAcross ? 6 : 0) >= k) {
                const int past = (int)line[j] + 16 * chunk - end, drop = span >= 16 ? max(0, min(past, 16)) / 2 : 0;
                const int keep = FORM == kAlong ? left - 8 * chunk : i / (WIDTH / 8) < left ? 8 : 0;
                if (drop & 4) x = (uint4_t){x[2], x[3], 0, 0};
                if (drop & 2) x = (uint4_t){x[1], x[2], x[3], 0};
                if (drop & 1) x = (uint4_t){x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
#pragma unroll
                for (int w = 0; w < 4; ++w) x[w] &= (2 * w < keep ? 0xffffu : 0u) | (2 * w + 1 < keep ? 0xffff0000u : 0u);
            }
            *reinterpret_cast<uint4_t*>(lds + (FORM == kAcross ? across_at<WIDTH>(i / (WIDTH / 8), chunk) : along_at<ROW>(i / kIn, chunk))) = x;
        }
    }
};

// Where a wave reads: a buffer's description, the same in all lanes.
struct Buffer {
    uint64_t at;
    uint32_t size;     // bytes; reads past them come back as zero
};

// BYTES (16 or 4) a lane from byte `at` of a buffer to LDS: lane by lane behind byte `lds` + PLUS of it.
// Written as an instruction because the compiler, which does not see that reads of LDS are of other slices, has them wait for every
// load that it knows to be on its way there.  What a wave has in flight is counted where it meets the others.
template <int BYTES, int PLUS>
__device__ __forceinline__ void load_to_lds([[maybe_unused]] Buffer buffer, [[maybe_unused]] uint32_t at, [[maybe_unused]] uint32_t lds) {
    static_assert(BYTES == 16 || BYTES == 4);
#ifdef __HIP_DEVICE_COMPILE__
    const uint4_t d = {(uint32_t)buffer.at, (uint32_t)(buffer.at >> 32), buffer.size, 0x00020000u};
#define RSH_LOAD(name) asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\t" name " %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(d), "n"(PLUS) : "memory", "scc")
    if constexpr (BYTES == 16) RSH_LOAD("buffer_load_dwordx4");
    else RSH_LOAD("buffer_load_dword");
#undef RSH_LOAD
#endif
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform_address(const void* p) {
    return (uint64_t)uniform((uint32_t)((uint64_t)p >> 32) & 0xffffu) << 32 | uniform((uint32_t)(uint64_t)p);
}
__device__ __forceinline__ uint32_t lds_byte(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)p;
}

// The same straight into LDS: 16 bytes a lane, 1 KB a wave and turn, in the order of the lanes, so the chunks are dealt to their
// banks by the lane's choice of source.  Reads past the operand's end come back as zero (the buffer's range check); rows must be
// whole chunks at 16-byte boundaries, as those of codes always are.
template <Form FORM, int ROW, int WIDTH, int THREADS, bool PAIR>
struct Direct {
    static constexpr int kIn = ROW / 16;                   // chunks of a row
    static constexpr int kChunks = FORM == kCodes ? (WIDTH + THREADS - 1) / THREADS : WIDTH * kIn / THREADS;
    static constexpr int kBytes = kChunks * THREADS * 16;  // of a slice; a workgroup wider than a tile of codes loads zeros behind it
    static constexpr int kSlice = FORM == kFours ? 2 * ROW : ROW / 2;
    static constexpr uint32_t kNowhere = 0x80000000u;      // past every buffer
    uint32_t at[kChunks];          // byte of the lane's chunks from the tile's first, in any slice
    int chunk;                     // chunk of its row that a lane loads; the same in every turn
    Buffer from;                   // of the slice that comes next
    uint64_t other;                // the second segment's first byte
    uint32_t step, whole, cut;     // bytes from slice to slice; sizes of a slice of rows of k, and of the last one
    int left;                      // of k

    // which: the matrix of a wave, or of the first segment
    __device__ __forceinline__ void start(const Operand& o, int64_t tile, int64_t extent, int64_t k, int which, int slice) {
        const int64_t width = PAIR ? WIDTH / 2 : WIDTH, lines = min(extent - tile * width, (int64_t)width);
        const int64_t stride = FORM == kFours || FORM == kCodes ? o.ld * kBlockBytes : o.ld * 2;
        const int64_t first = tile * width * (FORM == kAcross ? 2 : stride);
        step = uniform(FORM == kAcross ? (uint32_t)(kSlice * stride) : FORM == kCodes ? 16 : ROW);
        from.at = uniform_address((const uint8_t*)(which ? o.data[1] : o.data[0]) + first + (int64_t)slice * step);
        other = uniform_address((const uint8_t*)o.data[1] + first);
        left = (int)uniform((uint32_t)min(k - (int64_t)slice * kSlice, (int64_t)0x7fffffff));
        if constexpr (FORM == kAcross) {
            whole = uniform((uint32_t)((kSlice - 1) * stride + 2 * lines));
            cut = uniform((uint32_t)(((k - 1) % kSlice) * stride + 2 * lines));
        } else {
            whole = uniform((uint32_t)((lines - 1) * stride + (FORM == kAlong ? 2 * k : stride)));
            from.size = uniform(whole - (uint32_t)slice * step);
        }
        chunk = FORM == kAlong || FORM == kFours ? (threadIdx.x % kIn) ^ along_turn<ROW>(threadIdx.x / kIn) : 0;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int i = threadIdx.x + THREADS * j;
            if constexpr (FORM == kAcross) {
                const int kk = i / (WIDTH / 8), c = i % (WIDTH / 8) ^ across_turn<WIDTH>(kk);
                at[j] = 8 * c < lines ? (uint32_t)(kk * stride + 16 * c) : kNowhere;
            } else if constexpr (FORM == kCodes) {
                at[j] = i < WIDTH ? (uint32_t)(line_of<PAIR>(codes_row<PAIR>(i)) * stride) : kNowhere;
            } else {
                at[j] = (uint32_t)(line_of<PAIR>(i / kIn) * stride + 16 * chunk);
            }
        }
    }
    // Chunk J of the slice that comes next, to `lds` + PLUS; nothing but zeros where there is none any more.
    template <int J, int PLUS>
    __device__ __forceinline__ void issue(bool live, uint32_t lds) const {
        Buffer b = from;
        if constexpr (FORM == kAcross) b.size = left >= kSlice ? whole : cut;
        b.size = live ? b.size : 0u;
        // a row's chunks past its end would be the next row's
        const bool in = FORM == kAcross || FORM == kCodes || (FORM == kFours ? 32 : 8) * chunk < left;
        load_to_lds<16, PLUS + THREADS * J * 16>(b, in ? at[J] : kNowhere, lds);
    }
    // The slice after that; `turn`: the first of the second segment, whose k is `k`.
    __device__ __forceinline__ void next(bool turn, int k) {
        if (turn) {
            from.at = other;
            left = k;
            if constexpr (FORM != kAcross) from.size = whole;
        } else {
            from.at += step;
            left -= kSlice;
            if constexpr (FORM != kAcross) from.size -= step;
        }
    }
};

// All reads and writes of LDS by a wave are done and all but the last PENDING of its loads have arrived (64: whatever is in
// flight may stay so); then the same of all waves.
template <int PENDING>
__device__ __forceinline__ void meet() {
    if constexpr (PENDING < 64) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PENDING) : "memory");
    else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The 16 bytes of an operand that a lane feeds to the matrix unit: row 32 i + lane % 32 of a wave's rows, piece s of a slice.  What
// depends on the lane is found once; the rest are constants of the instruction.
template <Form FORM, int ROW, int WIDTH, bool PAIR, int N>
struct Reader {
    int off[FORM == kAcross ? N : FORM == kCodes ? 1 : ROW / 32];
    __device__ __forceinline__ void start(int first, int lane) {
        if constexpr (FORM == kAcross) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int k = 8 * (lane >> 5) + (lane >> 2 & 3), col = first + 32 * i + (lane & 16) + 4 * (lane & 3);
                off[i] = across_at<WIDTH>(k, col >> 3) + 2 * (col & 7);
            }
        } else if constexpr (FORM == kCodes) {
            off[0] = codes_place<PAIR>(first + (lane & 31)) * 16 + 4 * (lane >> 5);
        } else {
#pragma unroll
            for (int s = 0; s < ROW / 32; ++s) off[s] = along_at<ROW>(first + (lane & 31), 2 * s + (lane >> 5));
        }
    }
    __device__ __forceinline__ uint4_t get(const unsigned char* lds, int i, int s) const {
        if constexpr (FORM == kAcross) {
            const unsigned char* const at = lds + off[i] + s * 16 * (2 * WIDTH);      // rows four on lie in the same banks
            const half4_t a = read_transposed(at), b = read_transposed(at + 4 * (2 * WIDTH));
            return __builtin_bit_cast(uint4_t, (half8_t){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        } else if constexpr (FORM == kCodes) {
            return (uint4_t){*reinterpret_cast<const uint32_t*>(lds + off[0] + (PAIR ? 64 : 32) * 16 * i + 8 * s), 0, 0, 0};     // eight codes
        } else {
            return *reinterpret_cast<const uint4_t*>(lds + off[s] + i * 32 * ROW);
        }
    }
};

// f(FROM) .. f(TO - 1), each with its own constant.
template <int FROM, int TO, class F>
__device__ __forceinline__ void each_of(F f) {
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>());
        each_of<FROM + 1, TO>(f);
    }
}

constexpr int larger(int a, int b) { return a > b ? a : b; }

}  // namespace

// T: F16 or BF16 (results, and operands unless they are kFours).  WP x WQ waves, each TP x TQ tiles of 32 x 32.  DIRECT: operands
// of 16 bits go straight into LDS.
template <class T, Form FP, Form FQ, bool GATED, int SEGS, int ROW, int WP, int WQ, int TP, int TQ, bool DIRECT>
__global__ __launch_bounds__(64 * WP * WQ) void rsh_product_kernel(Operand P, Operand Q, Result res, Shape sh, Split split) {
    constexpr int kThreads = 64 * WP * WQ, kWidthP = 32 * WP * TP, kWidthQ = 32 * WQ * TQ;
    constexpr bool kShifted = FP == kCodes && std::is_same<T, F16>::value;
    constexpr bool kFour = FP == kFours, kCode = FP == kCodes;
    constexpr bool kDirectP = DIRECT || kCode;
    constexpr int kSlice = kFour ? 2 * ROW : ROW / 2;   // k of a slice
    constexpr int kRing = 256 / ROW, kPieces = ROW / 32;                 // slices in LDS, pieces of a slice
    static_assert(ROW == 64 || (ROW == 128 && !kFour && !kCode));
    using DirectP = Direct<FP, ROW, kWidthP, kThreads, GATED>;
    using DirectQ = Direct<FQ, ROW, kWidthQ, kThreads, false>;
    constexpr int kBytesP = kCode ? DirectP::kBytes : kWidthP * ROW, kBytesSlice = kBytesP + kWidthQ * ROW;
    constexpr int kWide = GATED ? kWidthP / 2 : kWidthP;                 // columns of the tile's result
    constexpr int kScaleRows = kFour ? kWidthP + kWidthQ : kWidthP;      // rows of a slice that have scales
    constexpr int kScaleTurns = (kScaleRows + kThreads - 1) / kThreads;
    __shared__ __attribute__((aligned(16))) unsigned char lds[larger(kRing * kBytesSlice, (GATED ? 4 : 2) * kWide * kWidthQ)];
    // Four scales of a row: those of a slice, or beside codes, at their place, those of a ring of slices (a byte with every slice took as many
    // cycles of the loads' addresses as the codes: 128 rows through 8192 x 28672 113 us against 99).  A workgroup with more threads
    // than rows loads zeros behind them.
    __shared__ uint32_t scales[kFour ? kRing : 1][kFour || kCode ? kScaleTurns * kThreads : 1];
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
    const int slices = (int)((sh.k + kSlice - 1) / kSlice);
    const int begin = blockIdx.y * split.slices, end = min(SEGS * slices, begin + split.slices);

    std::conditional_t<kDirectP, DirectP, Stage<FP, ROW, kWidthP, kThreads, GATED>> sp;
    std::conditional_t<DIRECT, DirectQ, Stage<FQ, ROW, kWidthQ, kThreads, false>> sq;
    const int seg0 = SEGS == 2 && begin >= slices ? 1 : 0;
    if constexpr (kDirectP)
        sp.start(P, tc, sh.cols, sh.k, !GATED ? seg0 : kCode ? wave & 1 : wave * 64 / (32 * DirectP::kIn) & 1, begin - seg0 * slices);
    else sp.start(P, tc, sh.cols, sh.k);
    if constexpr (DIRECT) sq.start(Q, tr, sh.rows, sh.k, SEGS == 2 ? seg0 : second, begin - seg0 * slices);
    else sq.start(Q, tr, sh.rows, sh.k);

    // Scales: a lane loads those of its rows, a wave those of 64 rows of one matrix, four bytes at a time.  kCodes: for four slices, of
    // which a part of k begins with the first; kFours: of a slice, rows of P before those of Q.
    const int wave0 = (int)uniform(wave);
    Buffer scale_from[kScaleTurns];
    uint32_t scale_at[kScaleTurns];
    if constexpr (kFour || kCode) {
#pragma unroll
        for (int u = 0; u < kScaleTurns; ++u) {
            const int first = 64 * wave0 + kThreads * u, i = first + lane;
            const bool of_q = kFour && first >= kWidthP;
            const int which = kCode && GATED ? first >> 6 & 1 : 0;
            const Operand& o = of_q ? Q : P;
            const int64_t row0 = of_q ? tr * kWidthQ : tc * (kCode ? kWide : kWidthP);
            const int64_t rows = min((of_q ? sh.rows : sh.cols) - row0, (int64_t)(of_q ? kWidthQ : kCode ? kWide : kWidthP));
            const int line = of_q ? i - kWidthP : kCode ? line_of<GATED>(codes_row<GATED>(i)) : i;
            const int ahead = kFour ? 4 * begin : begin;
            scale_from[u].at = uniform_address((which ? o.scales[1] : o.scales[0]) + row0 * o.ld_scales + ahead);
            scale_from[u].size = uniform((uint32_t)(rows * o.ld_scales - ahead));
            scale_at[u] = i < kScaleRows ? (uint32_t)(line * o.ld_scales) : 0x80000000u;
        }
    }
    if constexpr (kShifted) {
        // The largest scale of each row within the part's k, and from it the lanes' shifts of their rows' scales.
        for (int i = threadIdx.x; i < kWidthP; i += kThreads) {
            const uint8_t* const row = (GATED && (i >> 5 & 1) ? P.scales[1] : P.scales[0]) +
                                       min(tc * kWide + line_of<GATED>(i), sh.cols - 1) * P.ld_scales;
            int top = 0, b = begin;
            for (; b + 16 <= end; b += 16) {
                uint4_t v;
                __builtin_memcpy(&v, row + b, 16);
#pragma unroll
                for (int w = 0; w < 16; ++w) {
                    const uint32_t word = v[w / 4];
                    const int s = word >> (8 * (w & 3)) & 255;
                    top = max(top, s == 255 ? 0 : s);
                }
            }
            for (; b < end; ++b) top = max(top, row[b] == 255 ? 0 : (int)row[b]);
            tops[i] = top;
        }
    }

    float16_t acc[TP][TQ];
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TQ; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

    // What goes into LDS by way of registers: two slices on the way, of even and odd number.
    auto load = [&](int slice, int odd) {
        slice = min(slice, end - 1);       // past the end: of no use, but the loads in flight are counted
        [[maybe_unused]] const int seg = SEGS == 2 && slice >= slices ? 1 : 0;
        [[maybe_unused]] const int64_t k0 = (int64_t)(slice - seg * slices) * kSlice;
        if constexpr (!kDirectP) sp.load(odd, seg, k0);
        if constexpr (!DIRECT) sq.load(odd, SEGS == 2 ? seg : second, k0);
    };
    auto store = [&](int slice, int odd) {
        if (slice >= end) return;
        [[maybe_unused]] const int at = (slice - begin) & (kRing - 1);
        [[maybe_unused]] const int64_t k0 = (int64_t)(SEGS == 2 && slice >= slices ? slice - slices : slice) * kSlice;
        if constexpr (!kDirectP) sp.store(odd, k0, sh.k, lds + at * kBytesSlice);
        if constexpr (!DIRECT) sq.store(odd, k0, sh.k, lds + at * kBytesSlice + kBytesP);
    };
    // What goes straight into LDS: load j of a slice's kLoads.
    constexpr int kLoadsP = kDirectP ? DirectP::kChunks : 0, kLoadsPQ = kLoadsP + (DIRECT ? DirectQ::kChunks : 0);
    constexpr int kLoads = kLoadsPQ + (kFour || kCode ? kScaleTurns : 0), kSure = kCode ? kLoadsPQ : kLoads;      // at most, at least
    const uint32_t lds0 = uniform(lds_byte(lds)) + wave0 * 1024, scales0 = uniform(lds_byte(scales)) + wave0 * 256;
    // of the slice that comes next, into place PLACE of the ring
    auto issue = [&](bool live, auto place, auto load) {
        constexpr int kPlace = decltype(place)::value, J = decltype(load)::value;
        if constexpr (kDirectP)
            if constexpr (J < kLoadsP) sp.template issue<J, kPlace * kBytesSlice>(live, lds0);
        if constexpr (DIRECT)
            if constexpr (J >= kLoadsP && J < kLoadsPQ) sq.template issue<J - kLoadsP, kPlace * kBytesSlice + kBytesP>(live, lds0);
        if constexpr (J >= kLoadsPQ && (kFour || kPlace == 0))
            load_to_lds<4, (kPlace * kScaleTurns + J - kLoadsPQ) * kThreads * 4>(
                Buffer{scale_from[J - kLoadsPQ].at, live ? scale_from[J - kLoadsPQ].size : 0u}, scale_at[J - kLoadsPQ], scales0);
    };
    auto issued = [&](int slice, auto place) {         // all of `slice`
        const bool turn = SEGS == 2 && slice + 1 == slices;
        if constexpr (kDirectP) sp.next(turn, (int)min(sh.k, (int64_t)0x7fffffff));
        if constexpr (DIRECT) sq.next(turn, (int)min(sh.k, (int64_t)0x7fffffff));
        if constexpr (kFour || (kCode && decltype(place)::value == 0)) {
#pragma unroll
            for (int u = 0; u < kScaleTurns; ++u) {
                scale_from[u].at += 4;
                scale_from[u].size -= 4;
            }
        }
    };

    // Fragment n of the kReads of a piece.
    constexpr int kReads = TP + TQ, kProducts = TP * TQ;
    struct Pieces {
        uint4_t a[TP], b[TQ];      // a[][0] alone: eight codes
    };
    Reader<kCode ? kCodes : FP == kAcross ? kAcross : kAlong, ROW, kWidthP, GATED, TP> rp;
    Reader<FQ == kAcross ? kAcross : kAlong, ROW, kWidthQ, false, TQ> rq;
    rp.start(32 * wp * TP, lane);
    rq.start(32 * wq * TQ, lane);
    static_assert(!kCode || TP == 2);
    auto read = [&](Pieces& f, int at, int s, int n) {
        if (n < TP) f.a[n] = rp.get(lds + at * kBytesSlice, n, s);
        else f.b[n - TP] = rq.get(lds + at * kBytesSlice + kBytesP, n - TP, s);
    };
    // Scales of the lane's rows in a slice: kFours: lanes from 32 on have every second block; kCodes: one block of the four at hand.
    uint32_t ea[TP], eb[TQ];
    int shift[TP];
    uint32_t na[TP], nb[TQ];       // of the next slice, as they lie in LDS
    auto read_scales = [&](auto place) {
        constexpr int at = decltype(place)::value;
        if constexpr (kFour || (kCode && at == 0)) {
#pragma unroll
            for (int i = 0; i < TP; ++i) na[i] = scales[at][codes_place<kCode && GATED>(32 * (wp * TP + i) + (lane & 31))];
        }
        if constexpr (kFour) {
#pragma unroll
            for (int i = 0; i < TQ; ++i) nb[i] = scales[at][kWidthP + 32 * (wq * TQ + i) + (lane & 31)];
        }
    };
    auto take_scales = [&]([[maybe_unused]] auto place) {
        if constexpr (kFour) {
#pragma unroll
            for (int i = 0; i < TP; ++i) ea[i] = na[i] >> (8 * (lane >> 5));
#pragma unroll
            for (int i = 0; i < TQ; ++i) eb[i] = nb[i] >> (8 * (lane >> 5));
        }
        if constexpr (kCode) {
#pragma unroll
            for (int i = 0; i < TP; ++i) {
                const uint32_t e = na[i] >> (8 * decltype(place)::value) & 255u;
                ea[i] = (kShifted && e != 255u ? (uint32_t)max(0, (int)e + shift[i]) : e) << 23;
            }
        }
    };
    // The products of a piece, then(n) behind the n-th.
    auto multiply = [&](const Pieces& f, int s, auto then) {
#pragma unroll
        for (int i = 0; i < TP; ++i) {
            uint4_t a = f.a[i];
            if constexpr (kCode) a = from_codes8<T>(a[0], __uint_as_float(ea[i]));
#pragma unroll
            for (int j = 0; j < TQ; ++j) {
                if constexpr (kFour) {
                    const int8v_t fa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
                    const int8v_t fb = {(int)f.b[j][0], (int)f.b[j][1], (int)f.b[j][2], (int)f.b[j][3], 0, 0, 0, 0};
                    if (s) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa, fb, acc[i][j], 4, 4, 2, ea[i], 2, eb[j]);
                    else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa, fb, acc[i][j], 4, 4, 0, ea[i], 0, eb[j]);
                } else {
                    acc[i][j] = T::mfma32(a, f.b[j], acc[i][j]);
                }
                then(i * TQ + j);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // Of things FROM .. TO - 1, spread over the products, those behind product n.
    auto spread = [&](auto from, auto to, int n, auto thing) {
        constexpr int kFrom = decltype(from)::value, kTo = decltype(to)::value;
        each_of<kFrom, kTo>([&](auto j) {
            if ((j - kFrom) * kProducts / (kTo - kFrom) == n) thing(j);
        });
    };

    // Slice i is multiplied in kPieces pieces of 16 k (64 of 4 bits).  Before the last all waves meet: its fragments are in registers
    // by then, slice i + 1 is in LDS, and the place of slice i is free for slice i + kRing, half of whose loads are issued during the
    // last piece and half during the first of the next slice.  So a load has nearly kRing - 1 slices to arrive, and products, reads and
    // loads alternate, which keeps any of them from holding up the products behind it.  (All loads in the last piece: the same time.)
    constexpr int kEarly = (kLoads + 1) / 2;
    constexpr int kPending = kLoads ? (kRing - 2) * kSure : 64;       // registers that loads go to are waited for where they are used
    each_of<0, kRing>([&](auto place) {
        each_of<0, kLoads>([&](auto j) { issue(begin + place < end, place, j); });
        issued(begin + place, place);
    });
    load(begin, 0);
    store(begin, 0);
    load(begin + 1, 1);
    load(begin + 2, 0);
    meet<kLoads ? (kRing - 1) * kSure : 64>();
    if constexpr (kShifted) {
#pragma unroll
        for (int i = 0; i < TP; ++i) shift[i] = 127 + kSpan - tops[32 * (wp * TP + i) + (lane & 31)];
    }
    Pieces f[2];
    const std::integral_constant<int, 0> none;
    read_scales(none);
    take_scales(none);
#pragma unroll
    for (int n = 0; n < kReads; ++n) read(f[0], 0, 0, n);
    const std::integral_constant<int, kEarly> early;
    const std::integral_constant<int, kLoads> all;
    const std::integral_constant<int, kReads> reads;
    // Slice `slice`, which lies at place PLACE.
    auto turn = [&](int slice, auto place) {
        constexpr int kPlace = decltype(place)::value, kNext = (kPlace + 1) % kRing;
        const auto before = std::integral_constant<int, (kPlace + kRing - 1) % kRing>();
        const auto after = std::integral_constant<int, kNext>();
#pragma unroll
        for (int s = 0; s < kPieces - 1; ++s) {
            multiply(f[s & 1], s, [&](int n) {
                spread(none, reads, n, [&](auto r) { read(f[(s + 1) & 1], kPlace, s + 1, r); });
                if (s == 0 && slice > begin) {
                    spread(early, all, n, [&](auto j) { issue(slice - 1 + kRing < end, before, j); });
                    if (n == kProducts - 1) issued(slice - 1 + kRing, before);
                }
            });
        }
        store(slice + 1, (kPlace + 1) & 1);
        meet<kPending>();
        load(slice + 3, (kPlace + 1) & 1);
        read_scales(after);
        multiply(f[1], kPieces - 1, [&](int n) {
            spread(none, reads, n, [&](auto r) { read(f[0], kNext, 0, r); });
            spread(none, early, n, [&](auto j) { issue(slice + kRing < end, place, j); });
        });
        take_scales(after);
    };
    for (int slice = begin; slice < end; slice += kRing)
        each_of<0, kRing>([&](auto place) {
            if (slice + place < end) turn(slice + place, place);
        });
    meet<0>();

    // A lane has columns 8 g + 4 (lane / 32) .. + 3, g = 0 .. 3, of row lane % 32 of every tile of 32 x 32.
    const int half = 4 * (lane >> 5);
    if constexpr (kShifted) {
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int e = tops[32 * (wp * TP + i) + 8 * (v / 4) + half + v % 4] - (127 + kSpan);
#pragma unroll
                for (int j = 0; j < TQ; ++j) acc[i][j][v] = ldexpf(acc[i][j][v], e);
            }
    }
    const int64_t col0 = tc * kWide, row0 = tr * kWidthQ;
    if (split.parts > 1) {
        const int64_t wide = (sh.cols + 3) / 4 * 4, ld = GATED ? 2 * wide : wide;
        float* const partial = split.partial + ((int64_t)blockIdx.y * gridDim.z + blockIdx.z) * sh.rows * ld;
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int64_t row = row0 + 32 * (wq * TQ + j) + (lane & 31);
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * (wp * TP + i);
                    const int64_t col = col0 + (GATED ? at / 64 * 32 : at) + 8 * g + half;
                    if (row < sh.rows && col < sh.cols)
                        *reinterpret_cast<float4_t*>(partial + row * ld + (GATED && i % 2 ? wide : 0) + col) =
                            (float4_t){acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                }
        }
        return;
    }
    // Rounded, a result goes through LDS (its chunks dealt to the banks by their row) and leaves in whole lines.
    constexpr int kTurn = (kWide < 128 ? kWide : 128) / 8 - 1;
    unsigned char* const turned = lds;
    auto put = [&](int i, int j, int g, uint2_t v) {
        const int row = 32 * (wq * TQ + j) + (lane & 31), at = 32 * (wp * TP + i), col = (GATED ? at / 64 * 32 : at) + 8 * g;
        *reinterpret_cast<uint2_t*>(turned + row * (2 * kWide) + ((col / 8 ^ (row & kTurn)) << 4) + 2 * half) = v;
    };
    auto leave = [&](uint16_t* out, int64_t ld, int64_t cols) {
        __syncthreads();
        constexpr int kIn = kWide / 8;         // chunks of a row
#pragma unroll 4
        for (int n = threadIdx.x; n < kIn * kWidthQ; n += kThreads) {
            const int row = n / kIn, c = n % kIn;
            const int64_t left = cols - col0 - 8 * c;
            const uint4_t v = *reinterpret_cast<const uint4_t*>(turned + row * (2 * kWide) + ((c ^ (row & kTurn)) << 4));
            uint16_t* const at = out + (row0 + row) * ld + col0 + 8 * c;
            if (row0 + row < sh.rows) {
                if (left >= 8) {
                    *reinterpret_cast<uint4_a2*>(at) = v;
                } else {
                    for (int e = 0; e < left; ++e) at[e] = (uint16_t)((e & 4 ? (e & 2 ? v[3] : v[2]) : (e & 2 ? v[1] : v[0])) >> (16 * (e & 1)));
                }
            }
        }
        __syncthreads();
    };
    auto each = [&](auto value) {
#pragma unroll
        for (int i = 0; i < TP; i += GATED ? 2 : 1)
#pragma unroll
            for (int j = 0; j < TQ; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) put(i, j, g, (uint2_t){T::pair(value(i, j, 4 * g), value(i, j, 4 * g + 1)), T::pair(value(i, j, 4 * g + 2), value(i, j, 4 * g + 3))});
    };
    if constexpr (GATED) {
        if (res.gate) {
            auto keep = [&](float* out, int which) {       // the same way, in 32 bits
                constexpr int kIn = kWide / 4;
#pragma unroll
                for (int i = 0; i < TP; i += 2)
#pragma unroll
                    for (int j = 0; j < TQ; ++j)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int row = 32 * (wq * TQ + j) + (lane & 31), c = (32 * (wp * TP + i) / 64 * 32 + 8 * g + half) / 4;
                            *reinterpret_cast<float4_t*>(lds + row * (4 * kWide) + ((c ^ (row & 15)) << 4)) =
                                (float4_t){acc[i + which][j][4 * g], acc[i + which][j][4 * g + 1], acc[i + which][j][4 * g + 2], acc[i + which][j][4 * g + 3]};
                        }
                __syncthreads();
#pragma unroll 4
                for (int n = threadIdx.x; n < kIn * kWidthQ; n += kThreads) {
                    const int row = n / kIn, c = n % kIn;
                    const float4_t v = *reinterpret_cast<const float4_t*>(lds + row * (4 * kWide) + ((c ^ (row & 15)) << 4));
                    if (row0 + row < sh.rows && col0 + 4 * c < res.ld_gate)
                        *reinterpret_cast<float4_t*>(out + (row0 + row) * res.ld_gate + col0 + 4 * c) = v;
                }
                __syncthreads();
            };
            keep(res.gate, 0);
            keep(res.up, 1);
        }
        auto finished = [&](auto act) {
            each([&](int i, int j, int v) { return act_of(decltype(act)::value, acc[i][j][v]) * acc[i + 1][j][v]; });
        };
        if (res.act == kSilu) finished(std::integral_constant<int, kSilu>());
        else if (res.act == kGelu) finished(std::integral_constant<int, kGelu>());
        else finished(std::integral_constant<int, kRelu>());
    } else {
        each([&](int i, int j, int v) { return acc[i][j][v]; });
    }
    leave(res.out[second], res.ld, sh.cols);
}

// Rows of scales at multiples of four bytes, as lanes load them four at a time: those of W, then those of X.
__global__ __launch_bounds__(256) void rsh_align_scales_kernel(const uint8_t* __restrict__ W, const uint8_t* __restrict__ X, uint32_t* __restrict__ out,
                                                               int64_t n, int64_t t, int blocks) {
    const int words = (blocks + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (n + t) * words) return;
    const int64_t row = i / words, b = 4 * (i - row * words);
    const uint8_t* const at = row < n ? W + row * blocks : X + (row - n) * blocks;
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (b + j < blocks) v |= (uint32_t)at[b + j] << (8 * j);
    out[i] = v;
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

// dU = dH act(G) and dG = dH U act'(G), eight elements a thread, rounded to the 16 bits that the matrix units take: the gradients'
// one rounding besides that of their results.  A pass over five arrays: 187 us at 4096 x 16384, 5.0 TB/s.
template <class T>
__global__ __launch_bounds__(256) void rsh_gate_backward_kernel(const uint16_t* __restrict__ dH, const float* __restrict__ G,
                                                                const float* __restrict__ U, uint16_t* __restrict__ dG,
                                                                uint16_t* __restrict__ dU, int64_t t, int64_t f, int64_t ld, int64_t ld_gate, int act) {
    const uint32_t across = (uint32_t)((ld_gate + 2047) / 2048);
    const int64_t col = 8 * ((int64_t)(blockIdx.x % across) * 256 + threadIdx.x);
    if (col >= ld_gate) return;
    for (int64_t row = blockIdx.x / across; row < t; row += gridDim.x / across) {
        const int64_t at = row * ld_gate + col;
        const uint4_t h = load8(dH + row * ld + col, f - col);
        const float4_t g[2] = {*reinterpret_cast<const float4_t*>(G + at), *reinterpret_cast<const float4_t*>(G + at + 4)};
        const float4_t u[2] = {*reinterpret_cast<const float4_t*>(U + at), *reinterpret_cast<const float4_t*>(U + at + 4)};
        uint4_t a, b;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float dg[2], du[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t word = h[w];
                const float hv = T::widen((uint16_t)(word >> 16 * e)), gv = g[w / 2][2 * (w & 1) + e], uv = u[w / 2][2 * (w & 1) + e];
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

// What the operands of a product do on their way: straight into LDS, through registers, or in 4 bits on both sides.
enum Way { kStraight, kStaged, kFourBits };

// The form and the parts of k whose workgroups take the least time by this account, fitted to products of 17 to 4096 rows by 500 to
// 28672 columns, all forms and 1 to 16 parts of each, in microseconds: a slice of k of one workgroup alone on its compute unit, and
// of each of several or where all of them work; what a workgroup takes besides; a join's launch and the bytes that pass through
// memory for it.  (1024 rows of a gated block
// of 2048 x 2048: 25 in form 1, 42 in form 0 and two parts, 32 in form 2.)
Choice choose(int64_t rows, int64_t cols, int64_t slices, bool pairs, int results, Way way) {
    constexpr double alone[3][3] = {{0.56, 0.27, 0.23}, {1.2, 0.8, 0.62}, {0.75, 0.38, 0.3}};
    constexpr double shared[3][3] = {{0.56, 0.29, 0.2}, {1.2, 0.5, 0.37}, {1.1, 0.5, 0.32}};
    constexpr double besides[3] = {8, 1.5, 0.7};
    constexpr int room[3] = {1, 2, 3};                 // workgroups of a compute unit
    Choice best = {0, 1};
    double least = 1e300;
    for (int form = 0; form < 3; ++form) {
        const int64_t wide = kWide[form] / (pairs ? 2 : 1);
        const int64_t tiles = ((rows + kTall[form] - 1) / kTall[form]) * ((cols + wide - 1) / wide) * results;
        for (int tried = 1; tried <= 16 && tried <= slices; tried += tried < 4 ? 1 : tried < 8 ? 2 : 4) {
            const int64_t each = (slices + tried - 1) / tried, parts = (slices + each - 1) / each;
            const double n = (double)((tiles * parts + 255) / 256), rounds = (double)(((int64_t)n + room[form] - 1) / room[form]);
            double t = (double)each * std::max(alone[way][form] * rounds, n * shared[way][form]) + n * besides[form];
            if (parts > 1) t += 5.0 + 8.0 / 5.1e6 * (double)(parts * rows * cols * results * (pairs ? 2 : 1));
            if (t < least) {
                least = t;
                best = {form, (int)parts};
            }
        }
    }
    return best;
}

// Of a product whose operands may go either way.
int64_t partial_bytes(int64_t rows, int64_t cols, int64_t slices, bool pairs, int results, bool four) {
    int parts = 1;
    for (const Way way : {kStraight, kStaged, kFourBits})
        if (four == (way == kFourBits)) {
            const int p = choose(rows, cols, slices, pairs, results, way).parts;
            parts = std::max(parts, p);
        }
    return parts == 1 ? 0 : (int64_t)parts * results * rows * ((cols + 3) / 4 * 4) * (pairs ? 2 : 1) * (int64_t)sizeof(float);
}

// Whether an operand's lines are whole chunks at 16-byte boundaries.
bool whole_chunks(const Operand& o, Form form, int64_t along) {
    if (form == kCodes || form == kFours) return true;
    return ((uintptr_t)o.data[0] | (uintptr_t)o.data[1]) % 16 == 0 && o.ld % 8 == 0 && along % 8 == 0;
}

// Bytes of a row of a slice in tiles of 256 x 256.  Whole lines of 128 bytes halve the requests that L2 serves (2048 tokens through
// 8192 x 28672: 1.62 ms against 1.71 in rows of 64), where both operands are of 16 bits.
// 4-bit ones have four slices on the way, and rows that pass through registers would not fit those.
constexpr int row_bytes(Form p, bool direct) { return direct && (p == kAlong || p == kAcross) ? 128 : 64; }

template <class T, Form FP, Form FQ, bool GATED, int SEGS, bool DIRECT>
void launch_tiles(int form, dim3 grid, const Operand& P, const Operand& Q, const Result& res, const Shape& sh, const Split& split, hipStream_t st) {
    if (form == 0)
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, row_bytes(FP, DIRECT), 4, 2, 2, 4, DIRECT>), grid, dim3(512), 0, st, P, Q, res, sh, split);
    else if (form == 1)
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, 64, 2, 2, 2, 2, DIRECT>), grid, dim3(256), 0, st, P, Q, res, sh, split);
    else
        hipLaunchKernelGGL((rsh_product_kernel<T, FP, FQ, GATED, SEGS, 64, 2, 2, 2, 1, DIRECT>), grid, dim3(256), 0, st, P, Q, res, sh, split);
}

// Of a product: the form, rows and columns of a tile's result, parts of k and the slices of each.
struct Tiling {
    int form;
    int64_t tall, wide;
    int parts, each;
};
Tiling tiling(Form p, int segs, bool pairs, int results, bool direct, int64_t rows, int64_t cols, int64_t k) {
    const int64_t least = p == kFours ? 128 : 32;
    const Choice c = choose(rows, cols, segs * ((k + least - 1) / least), pairs, results, p == kFours ? kFourBits : direct ? kStraight : kStaged);
    const int64_t slice = c.form == 0 ? least * row_bytes(p, direct) / 64 : least, slices = segs * ((k + slice - 1) / slice);
    const int64_t share = (slices + c.parts - 1) / c.parts, each = p == kCodes ? (share + 3) / 4 * 4 : share;      // parts begin where a word of scales does
    return {c.form, kTall[c.form], kWide[c.form] / (pairs ? 2 : 1), (int)((slices + each - 1) / each), (int)each};
}

template <class T, Form FP, Form FQ, bool GATED, int SEGS>
void product(const Operand& P, const Operand& Q, const Result& res, int64_t rows, int64_t cols, int64_t k, int results, void* work, hipStream_t st) {
    const bool direct = FP == kFours || (whole_chunks(P, FP, FP == kAcross ? cols : k) && whole_chunks(Q, FQ, FQ == kAcross ? rows : k));
    const Tiling c = tiling(FP, SEGS, GATED, results, direct, rows, cols, k);
    const int parts = c.parts;
    const Shape sh = {rows, cols, k, (int)((rows + c.tall - 1) / c.tall), (int)((cols + c.wide - 1) / c.wide)};
    const Split split = {parts, c.each, (float*)work};
    const int64_t tiles = (int64_t)sh.tiles_r * sh.tiles_c;
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8), parts, results);
    if constexpr (FP != kFours)
        if (!direct) launch_tiles<T, FP, FQ, GATED, SEGS, false>(c.form, grid, P, Q, res, sh, split, st);
    if (direct) launch_tiles<T, FP, FQ, GATED, SEGS, true>(c.form, grid, P, Q, res, sh, split, st);
    if (parts > 1)
        hipLaunchKernelGGL((rsh_join_parts_kernel<T, GATED>), dim3((unsigned)((cols + 1023) / 1024 * rows), 1, results), dim3(256), 0, st,
                           (const float*)work, res, rows, cols, parts);
}

template <class F>
void by_half(int type, F f) {
    if (type == RSH_F16) f(F16());
    else f(BF16());
}

}  // namespace

// Bytes of `rows` rows of scales in whole words, where theirs are not.
int64_t aligned_scales(int64_t rows, int64_t k) {
    const int64_t blocks = (k + kBlock - 1) / kBlock;
    return blocks % 4 == 0 ? 0 : (rows * ((blocks + 3) / 4) * 4 + 15) / 16 * 16;
}

// Puts them there: those of `a`'s n rows (second: of its second matrix too) and of b's t.  Returns what of `work` lies behind them.
uint8_t* align_scales(Operand& a, int64_t n, bool second, Operand& b, int64_t t, int64_t k, void* work, hipStream_t st) {
    const int64_t bytes = aligned_scales(second ? 2 * n : n + t, k), blocks = (k + kBlock - 1) / kBlock;
    if (bytes) {
        const uint8_t* const next = second ? a.scales[1] : b.scales[0];
        const int64_t rest = second ? n : t;
        a.ld_scales = b.ld_scales = (blocks + 3) / 4 * 4;
        const int64_t words = (n + rest) * (a.ld_scales / 4);
        hipLaunchKernelGGL(rsh_align_scales_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, st, a.scales[0], next, (uint32_t*)work, n, rest,
                           (int)blocks);
        a.scales[0] = (const uint8_t*)work;
        (second ? a.scales[1] : b.scales[0]) = a.scales[0] + n * a.ld_scales;
    }
    return (uint8_t*)work + bytes;
}

int64_t mx4_product_work(int x_type, int64_t t, int64_t n, int64_t k) {
    const int64_t step = x_type == RSH_MX4 ? 128 : 32;
    if (takes_few(t)) return 0;
    return aligned_scales(x_type == RSH_MX4 ? n + t : n, k) + partial_bytes(t, n, (k + step - 1) / step, false, 1, x_type == RSH_MX4);
}

int64_t gated_forward_work(bool codes, int64_t t, int64_t d, int64_t f) {
    if (takes_few(t)) return 0;
    return (codes ? aligned_scales(2 * f, d) : 0) + partial_bytes(t, f, (d + 31) / 32, true, 1, false);
}

// tile: rows and columns of the result, parts of k; zeros for the kernels of few rows.  The same choice as the launches'.
void ffn_tiles(int which, bool aligned, int64_t t, int64_t a, int64_t b, int32_t* tile) {
    Tiling c = {0, 0, 0, 0, 0};
    const bool backward = which == RSH_TILES_DX || which == RSH_TILES_DW || which == RSH_TILES_DW_ONE;
    if (which == RSH_TILES_DX) c = tiling(kAcross, 2, false, 1, aligned, t, a, b);
    else if (backward) c = tiling(kAcross, 1, false, which == RSH_TILES_DW ? 2 : 1, aligned, b, a, t);
    else if (!takes_few(t) && which == RSH_TILES_PRODUCT) c = tiling(kCodes, 1, false, 1, aligned, t, a, b);
    else if (!takes_few(t) && which == RSH_TILES_PRODUCT4) c = tiling(kFours, 1, false, 1, true, t, a, b);
    else if (!takes_few(t)) c = tiling(which == RSH_TILES_GATED4 ? kCodes : kAlong, 1, true, 1, aligned, t, b, a);
    tile[0] = (int32_t)c.tall;
    tile[1] = (int32_t)c.wide;
    tile[2] = c.parts;
}

// dG and dU, and behind them the larger of the sums of dX and of the weights' gradients (of both, or of one alone).
int64_t gated_backward_work(int64_t t, int64_t d, int64_t f) {
    const int64_t gates = 4 * t * ((f + 7) / 8 * 8);
    int64_t sums = partial_bytes(t, d, 2 * ((f + 31) / 32), false, 1, false);
    for (int results = 1; results <= 2; ++results)
        sums = std::max(sums, partial_bytes(f, d, (t + 31) / 32, false, results, false));
    return gates + sums;
}

int launch_mx4_product(const void* X, const void* x_scales, int x_type, int64_t ld_x, const void* W, const void* w_scales, void* Y, int y_type,
                       int64_t t, int64_t n, int64_t k, void* work, void* stream) {
    const int64_t blocks = (k + kBlock - 1) / kBlock;
    const Operand p = {{W, nullptr}, {(const uint8_t*)w_scales, nullptr}, blocks, blocks};
    const Operand q = {{X, nullptr}, {(const uint8_t*)x_scales, nullptr}, x_type == RSH_MX4 ? blocks : ld_x, blocks};
    const Result res = {{(uint16_t*)Y, nullptr}, nullptr, nullptr, n, 0, 0};
    by_half(y_type, [&](auto half) {
        using T = decltype(half);
        if (takes_few(t)) {
            if (x_type == RSH_MX4) launch_few<T, kFours, false>(p, q, res, t, n, k, (hipStream_t)stream);
            else launch_few<T, kCodes, false>(p, q, res, t, n, k, (hipStream_t)stream);
        } else {
            const bool four = x_type == RSH_MX4;
            Operand w = p, x = q;
            void* const rest = align_scales(w, n, false, x, four ? t : 0, k, work, (hipStream_t)stream);
            if (four) product<T, kFours, kFours, false, 1>(w, x, res, t, n, k, 1, rest, (hipStream_t)stream);
            else product<T, kCodes, kAlong, false, 1>(w, x, res, t, n, k, 1, rest, (hipStream_t)stream);
        }
    });
    return launched();
}

int launch_gated_forward(const void* X, int type, int64_t ld_x, const void* Wg, const void* Wu, int64_t ld_w, const void* g_scales,
                         const void* u_scales, int act, void* H, void* G, void* U, int64_t t, int64_t d, int64_t f, void* work, void* stream) {
    const int64_t blocks = (d + kBlock - 1) / kBlock;
    const Operand p = {{Wg, Wu}, {(const uint8_t*)g_scales, (const uint8_t*)u_scales}, g_scales ? blocks : ld_w, blocks};
    const Operand q = {{X, nullptr}, {nullptr, nullptr}, ld_x, 0};
    const Result res = {{(uint16_t*)H, nullptr}, (float*)G, (float*)U, f, (f + 7) / 8 * 8, act};
    by_half(type, [&](auto half) {
        using T = decltype(half);
        if (takes_few(t)) {
            if (g_scales) launch_few<T, kCodes, true>(p, q, res, t, f, d, (hipStream_t)stream);
            else launch_few<T, kAlong, true>(p, q, res, t, f, d, (hipStream_t)stream);
        } else if (g_scales) {
            Operand w = p, x = q;
            void* const rest = align_scales(w, f, true, x, 0, d, work, (hipStream_t)stream);
            product<T, kCodes, kAlong, true, 1>(w, x, res, t, f, d, 1, rest, (hipStream_t)stream);
        } else product<T, kAlong, kAlong, true, 1>(p, q, res, t, f, d, 1, work, (hipStream_t)stream);
    });
    return launched();
}

int launch_gated_backward(const void* X, int type, int64_t ld_x, const void* Wg, const void* Wu, int64_t ld_w, const void* G, const void* U,
                          const void* dH, int64_t ld_h, int act, void* dX, void* dWg, void* dWu, int64_t t, int64_t d, int64_t f, void* work,
                          void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    const int64_t ld_gate = (f + 7) / 8 * 8, across = (ld_gate + 2047) / 2048, blocks = std::min<int64_t>(t, std::max<int64_t>(1, (1 << 20) / across)) * across;
    uint16_t* const dG = (uint16_t*)work;
    uint16_t* const dU = dG + t * ld_gate;
    void* const sums = dU + t * ld_gate;
    const Operand gates = {{dG, dU}, {nullptr, nullptr}, ld_gate, 0};
    by_half(type, [&](auto half) {
        using T = decltype(half);
        hipLaunchKernelGGL(rsh_gate_backward_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, (const uint16_t*)dH, (const float*)G,
                           (const float*)U, dG, dU, t, f, ld_h, ld_gate, act);
        if (dX) {
            const Operand w = {{Wg, Wu}, {nullptr, nullptr}, ld_w, 0};
            const Result res = {{(uint16_t*)dX, nullptr}, nullptr, nullptr, d, 0, 0};
            product<T, kAcross, kAlong, false, 2>(w, gates, res, t, d, f, 1, sums, st);
        }
        if (dWg || dWu) {
            const Operand x = {{X, nullptr}, {nullptr, nullptr}, ld_x, 0}, only_u = {{dU, nullptr}, {nullptr, nullptr}, ld_gate, 0};
            const Result res = {{(uint16_t*)(dWg ? dWg : dWu), (uint16_t*)dWu}, nullptr, nullptr, d, 0, 0};
            product<T, kAcross, kAcross, false, 1>(x, dWg ? gates : only_u, res, f, d, t, dWg && dWu ? 2 : 1, sums, st);
        }
    });
    return launched();
}

}  // namespace rsh
