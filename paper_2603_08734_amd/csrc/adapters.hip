// Low-rank adapters of many requests beside a shared projection: out = Y + s_i (X A_i^T) B_i, and its gradients.
//
// With both factors rank first, A_i [r][k] and B_i [r][m], three products make up both directions:
//   shrink   H = X A_i^T, and dH = dout B_i^T      long rows against r short ones: matrix instructions of 16 bits
//   expand   out = Y + s H B_i, and dX = s dH A_i   r terms for every element: H is fp32, and enters as three numbers of bfloat16
//   outer    dA_i = s dH^T X, and dB_i = s H^T dout    the tokens of an adapter summed up, H in the same way
// Tokens are taken in tiles that share an adapter.  A kernel of one workgroup deals them out (8 to 9 us for 4096 tokens, all of it latency; it is
// kept for the gradients); a few tokens are dealt out by every workgroup for itself, which saves a launch.
//
// Ranks are small, so all three are passes over X, Y and dout, bound by memory; operands go from memory to the matrix unit through registers
// alone, a step ahead of their use.  Measured (bfloat16): 4096 tokens of 28672 features at rank 16, shrink 57 us (235 MB, 4.1 TB/s),
// expand to 8192 columns 33 us (134 MB, 4.1); 4096 tokens at rank 64 between 4096 and 16384 features: shrink 17 and 48 us, expand 23
// and 86, outer 26 and 55 (a copy of the bytes would take 7, 26, 7, 53, 7 and 26): what counts there is the time until a workgroup's first
// loads have come, since all of them fit the chip at once or nearly so.  One token at rank 16 between 8192 and 28672 features 13.9 us in one
// launch, 7.0 at 1024 features: one compute unit's reading of A, 35 KB a us; 77 tokens of 61 adapters at 4100 by 1003 11.2 us.
#include <algorithm>

#include "rows.hpp"

namespace rsh {

namespace {

constexpr int kFewTokens = 256, kFewTile = 16, kFewParts = 8, kFewColumns = 1024, kTile = 64, kShares = 2;     // kShares: workgroups of the second product that share a tile
constexpr int kSortThreads = 1024, kSortWords = 7 * (RSH_ADAPTERS_MAX + 1);     // counters in LDS

struct Tile {
    int adapter, first, count, pad;        // adapter: n for none; first: in the order
};

// Of the tokens: int32 or int64, anything but 0 .. n - 1 for none.
struct Index {
    const void* data;
    int wide, n;
    __device__ __forceinline__ int at(int64_t i) const {      // n: none
        const int64_t a = wide ? ((const int64_t*)data)[i] : ((const int32_t*)data)[i];
        return a >= 0 && a < n ? (int)a : n;
    }
};

// Where the tokens' order is.
struct Order {
    const int32_t* token;      // by adapter, those without one behind the others
    const int32_t* starts;     // of every adapter, n + 2
    const Tile* tiles;
    const int32_t* n_tiles;
};

typedef int FewPlace[kFewTokens + 4 + kFewTile];

// The tile of a workgroup whose tokens are few: its own token is the first of sixteen with the same adapter, or there is nothing to do.
// Returns the adapter, n for none, or -1; the tokens are behind place[kFewTokens + 4].
__device__ __forceinline__ int few_tile(const Index& index, int t, int mine, FewPlace& place, int* count) {
    const int i = threadIdx.x, wave = threadIdx.x >> 6;
    int a = -1;
    if (i < t) a = index.at(i);
    if (i < kFewTokens) place[i] = a;
    __syncthreads();
    const int own = place[mine];
    const uint64_t same = __ballot(i < t && a == own);
    if (i < kFewTokens && (i & 63) == 0) place[kFewTokens + wave] = __popcll(same);
    __syncthreads();
    int before = 0, all = 0, rank = 0;
#pragma unroll
    for (int w = 0; w < kFewTokens / 64; ++w) {
        const int c = place[kFewTokens + w];
        before += w < wave ? c : 0;
        all += c;
    }
    before += (int)bits_below_lane(same);
    if (i < t && a == own) place[i] = before;      // place in its adapter's order
    __syncthreads();
    rank = place[mine];
    if (rank % kFewTile) return -1;
    if (i < t && a == own && before >= rank && before < rank + kFewTile) place[kFewTokens + 4 + before - rank] = i;
    __syncthreads();
    *count = min(all - rank, kFewTile);
    return own;
}

// Eight elements of a row of d, zeros behind its end and in a lane that is not `in`.
__device__ __forceinline__ uint4_t run_of(const uint16_t* row, int64_t col, int64_t d, bool in = true) {
    return settle<F16, true>(load_raw<F16, true>(row, (int)col, (int)d), (int)col, (int)d, in).v[0];
}

// Tokens of a tile.
template <bool FEW>
struct Members {
    const int32_t* token;
    int adapter, count;        // adapter: n for none
    __device__ __forceinline__ int at(int i) const { return token[min(i, count - 1)]; }
};
template <bool FEW>
__device__ __forceinline__ bool members(const Index& index, const Order& order, int64_t t, int at, int* place, Members<FEW>* m) {
    if constexpr (FEW) {
        m->adapter = few_tile(index, (int)t, at, *reinterpret_cast<FewPlace*>(place), &m->count);
        m->token = place + kFewTokens + 4;
        return m->adapter >= 0;
    } else {
        if (at >= *order.n_tiles) return false;
        const Tile tile = order.tiles[at];
        m->adapter = tile.adapter;
        m->count = tile.count;
        m->token = order.token + tile.first;
        return true;
    }
}

}  // namespace

// Tokens by adapter, in their own order, the tiles, and where every adapter's tokens begin.  A wave has a run of the tokens and its own
// counters for all adapters.
__global__ __launch_bounds__(kSortThreads) void rsh_adapters_sort_kernel(Index index, int64_t t, int waves, int tile, int32_t* token, int32_t* starts,
                                                                         Tile* tiles, int32_t* n_tiles) {
    __shared__ int32_t counts[kSortWords];     // [adapter][wave]
    __shared__ int32_t tile_start[RSH_ADAPTERS_MAX + 2], token_start[RSH_ADAPTERS_MAX + 2];
    __shared__ int32_t sums[2][kSortThreads / 64];
    __shared__ int32_t total[2];
    const int n = index.n, groups = n + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < groups * waves; i += kSortThreads) counts[i] = 0;
    if (threadIdx.x < 2) total[threadIdx.x] = 0;
    __syncthreads();
    const int64_t share = ((t + waves - 1) / waves + 63) / 64 * 64, begin = wave * share, end = min(t, begin + share);
    int bits = 0;
    while (n >> bits) ++bits;
    // Lanes whose token has the same adapter as this one's; a run of tokens of one request needs no look at the bits.
    auto peers = [&](int a, bool in) {
        uint64_t same = __ballot(in);
        if (same == __ballot(in && a == __builtin_amdgcn_readfirstlane(a))) return same;      // lane 0 is always in
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot(a >> b & 1);
            same &= a >> b & 1 ? set : ~set;
        }
        return same;
    };
    // The adapters of the wave's first tokens stay in registers for the second look.
    constexpr int kHeld = 8;
    int held[kHeld];
    volatile int32_t* const count = counts;
    if (wave < waves) {
#pragma unroll
        for (int c = 0; c < kHeld; ++c) held[c] = begin + 64 * c + lane < end ? index.at(begin + 64 * c + lane) : 0;
        auto add = [&](int64_t i0, int a) {
            const bool in = i0 + lane < end;
            const uint64_t same = peers(a, in);
            if (in && bits_below_lane(same) == 0) count[a * waves + wave] = count[a * waves + wave] + __popcll(same);
        };
#pragma unroll
        for (int c = 0; c < kHeld; ++c)
            if (begin + 64 * c < end) add(begin + 64 * c, held[c]);
        for (int64_t i0 = begin + 64 * kHeld; i0 < end; i0 += 64) add(i0, i0 + lane < end ? index.at(i0 + lane) : 0);
    }
    __syncthreads();
    // Of every adapter: its tokens and tiles, added up over the adapters before it.
    for (int a0 = 0; a0 < groups; a0 += kSortThreads) {
        const int a = a0 + threadIdx.x;
        int c = 0;
        if (a < groups)
            for (int w = 0; w < waves; ++w) c += counts[a * waves + w];
        int before[2] = {c, (c + tile - 1) / tile};
        const int own[2] = {before[0], before[1]};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int up = shfl_i32(before[s], lane - d < 0 ? lane : lane - d);
                before[s] += lane >= d ? up : 0;
            }
            if (lane == 63) sums[s][wave] = before[s];
        }
        __syncthreads();
        int start = total[0] + before[0] - own[0], first = total[1] + before[1] - own[1];
        for (int w = 0; w < wave; ++w) start += sums[0][w], first += sums[1][w];
        if (a < groups) {
            starts[a] = token_start[a] = start;
            tile_start[a] = first;
            for (int w = 0; w < waves; ++w) {
                const int x = counts[a * waves + w];
                counts[a * waves + w] = start;
                start += x;
            }
        }
        __syncthreads();
        if (threadIdx.x == kSortThreads - 1) total[0] = start, total[1] = first + own[1];
        __syncthreads();
    }
    const int all = total[1];
    if (threadIdx.x == 0) {
        starts[groups] = token_start[groups] = (int32_t)t;
        *n_tiles = all;
    }
    if (wave < waves) {
        auto place = [&](int64_t i0, int a) {
            const bool in = i0 + lane < end;
            const uint64_t same = peers(a, in);
            const int rank = (int)bits_below_lane(same);
            if (in) {
                const int at = count[a * waves + wave];
                token[at + rank] = (int32_t)(i0 + lane);
                if (rank == 0) count[a * waves + wave] = at + __popcll(same);
            }
        };
#pragma unroll
        for (int c = 0; c < kHeld; ++c)
            if (begin + 64 * c < end) place(begin + 64 * c, held[c]);
        for (int64_t i0 = begin + 64 * kHeld; i0 < end; i0 += 64) place(i0, i0 + lane < end ? index.at(i0 + lane) : 0);
    }
    // A tile's adapter: the last that begins at or before it (those without tiles share theirs with the next).
    __syncthreads();
    for (int b = threadIdx.x; b < all; b += kSortThreads) {
        int lo = 0, hi = groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (tile_start[mid] <= b) lo = mid;
            else hi = mid - 1;
        }
        const int start = token_start[lo] + (b - tile_start[lo]) * tile;
        tiles[b] = {lo, start, min(tile, token_start[lo + 1] - start), 0};
    }
}

// H of a tile's tokens and 16 RT ranks, over a part of k.  WAVES waves share the part.
template <class T, int RT, int TT, bool FEW, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(RT == 1 ? 4 : RT == 2 ? 3 : 2))) void rsh_adapters_shrink_kernel(const uint16_t* X, int64_t ld_x, const uint16_t* A, Index index, Order order,
                                                                         float* H, int64_t t, int64_t k, int r, int steps) {
    __shared__ int place[FEW ? sizeof(FewPlace) / sizeof(int) : 1];
    __shared__ float4_t joined[WAVES][TT][64];
    Members<FEW> tile;
    if (!members<FEW>(index, order, t, (int)blockIdx.x, place, &tile) || tile.adapter == index.n) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    const int r0 = 16 * RT * (int)blockIdx.y, r16 = (r + 15) / 16 * 16, tiles = (tile.count + 15) / 16;
    const uint16_t* a[RT];
    const uint16_t* x[TT];
#pragma unroll
    for (int i = 0; i < RT; ++i) a[i] = A + ((int64_t)tile.adapter * r + min(r0 + 16 * i + c, r - 1)) * k;
#pragma unroll
    for (int i = 0; i < TT; ++i) x[i] = X + (int64_t)tile.at(16 * i + c) * ld_x;
    float4_t acc[RT][TT] = {};
    const int64_t begin = (int64_t)blockIdx.z * steps, end = min((k + 63) / 64, begin + steps);
    struct Slab {
        uint4_t a[RT][2], x[TT][2];
    };
    auto load = [&](int64_t step) {        // a whole one
        Slab v;
        const int64_t at = 64 * step + 8 * g;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < RT; ++i) v.a[i][h] = *reinterpret_cast<const uint4_a2*>(a[i] + at + 32 * h);
#pragma unroll
            for (int i = 0; i < TT; ++i) v.x[i][h] = *reinterpret_cast<const uint4_a2*>(x[i] + at + 32 * h);
        }
        return v;
    };
    auto multiply = [&](const Slab& v) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < RT; ++i) acc[i][j] = T::mfma16(v.a[i][h], v.x[j][h], acc[i][j]);
    };
    const int64_t whole = min(end, k / 64);
    if (begin + wave < whole) {
        Slab next = load(begin + wave);
        for (int64_t step = begin + wave; step < whole; step += WAVES) {
            const Slab v = next;
            if (step + WAVES < whole) next = load(step + WAVES);
            multiply(v);
        }
    }
    if (whole < end && (whole - begin) % WAVES == wave) {      // what is left of k
        const int64_t at = 64 * whole + 8 * g;
        Slab v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < RT; ++i) v.a[i][h] = run_of(a[i], at + 32 * h, k);
#pragma unroll
            for (int i = 0; i < TT; ++i) v.x[i][h] = run_of(x[i], at + 32 * h, k);
        }
        multiply(v);
    }
    // The waves' sums, in their order.
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < TT; ++j) joined[wave][j][lane] = acc[i][j];
        __syncthreads();
        const int rank = r0 + 16 * i + 4 * g;
        for (int j = wave; j < tiles; j += WAVES) {
            float4_t s = joined[0][j][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += joined[w][j][lane];
#pragma unroll
            for (int v = 0; v < 4; ++v) s[v] = rank + v < r ? s[v] : 0.f;
            if (rank < r16 && 16 * j + c < tile.count)
                *reinterpret_cast<float4_t*>(H + ((int64_t)blockIdx.z * t + tile.at(16 * j + c)) * r16 + rank) = s;
        }
    }
}

// Four fp32 numbers as three of bfloat16 each, hi + mid + lo: cut into eight bits at a time, so the three are the number itself (its last bits
// may be lost below 2^-110, where lo is subnormal); of an infinity or a NaN mid and lo are zero.  Sums of r or t products of one of them with 16-bit
// numbers are formed by the matrix unit's 16-bit instructions, whose products and sums are fp32: 16 terms take two of them for bfloat16, three for binary16.
// Its fp32 form takes four times as long as two and was 55 of the 100 us of 4096 tokens at rank 64 by 16384 columns.  (Two numbers of bfloat16, 2^-17
// off, make that step 80 us, three 86.)
struct Thirds {
    uint2_t hi, mid, lo;
};
__device__ __forceinline__ uint2_t upper(const uint32_t* v) {
    return {__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
}
__device__ __forceinline__ Thirds thirds(const float* h) {
    uint32_t hi[4], mid[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = __float_as_uint(h[i]) & 0xffff0000u;
        const float rest = h[i] - __uint_as_float(hi[i]);
        mid[i] = rest - rest == 0.f ? __float_as_uint(rest) & 0xffff0000u : 0u;
        lo[i] = rest - rest == 0.f ? __float_as_uint(rest - __uint_as_float(mid[i])) : 0u;
    }
    return {upper(hi), upper(mid), upper(lo)};
}
// 16 by 16 results of 16 terms in two forms at once, a0 b0 + a1 b1: lane l has terms 4 (l / 16) .. + 3 of row l % 16 of either operand.  Every sum is
// made of this instruction alone: one of 16 terms that takes up its result at once, as the compiler orders them, finds it unfinished.
__device__ __forceinline__ float4_t multiply(uint2_t a0, uint2_t a1, uint2_t b0, uint2_t b1, float4_t c) {
    return BF16::mfma16((uint4_t){a0[0], a0[1], a1[0], a1[1]}, (uint4_t){b0[0], b0[1], b1[0], b1[1]}, c);
}

// Column q of four rows of eight 16-bit numbers, as an operand.  bfloat16 goes as it is; a number of binary16 is two of bfloat16 exactly, of which
// `rest` is the second.
template <class T>
struct Column {
    uint2_t main, rest;
    __device__ __forceinline__ Column(const uint4_t* rows, int q) : rest{0, 0} {
        auto pick = [](uint32_t a, uint32_t b, int odd) { return __builtin_amdgcn_perm(b, a, odd ? 0x07060302u : 0x05040100u); };
        if constexpr (std::is_same<T, BF16>::value) {
            main = (uint2_t){pick(rows[0][q / 2], rows[1][q / 2], q & 1), pick(rows[2][q / 2], rows[3][q / 2], q & 1)};
        } else {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = F16::widen((uint16_t)(rows[i][q / 2] >> (16 * (q & 1))));
                hi[i] = __float_as_uint(x);
                const float r = x - __uint_as_float(hi[i] & 0xffff0000u);
                lo[i] = __float_as_uint(r - r == 0.f ? r : 0.f);
            }
            main = upper(hi), rest = upper(lo);
        }
    }
    // c and the products with H, whose numbers are the rows' terms.  FIRST: the column is the first operand, its place the results' row.
    template <bool FIRST>
    __device__ __forceinline__ float4_t times(const Thirds& h, float4_t c) const {
        if constexpr (std::is_same<T, BF16>::value) {
            const uint2_t none = {0, 0};
            c = FIRST ? multiply(main, main, h.hi, h.mid, c) : multiply(h.hi, h.mid, main, main, c);
            return FIRST ? multiply(main, main, h.lo, none, c) : multiply(h.lo, none, main, main, c);
        } else {
            c = FIRST ? multiply(main, rest, h.hi, h.hi, c) : multiply(h.hi, h.hi, main, rest, c);
            c = FIRST ? multiply(main, rest, h.mid, h.mid, c) : multiply(h.mid, h.mid, main, rest, c);
            return FIRST ? multiply(main, rest, h.lo, h.lo, c) : multiply(h.lo, h.lo, main, rest, c);
        }
    }
};
// The pieces' products make NaN of an infinity, which a piece that is zero multiplies too.  So where a sum has come out as NaN, it is
// formed again from the numbers themselves, and is NaN where the formula is.  That way is taken whole, in a loop behind the other: between its steps it
// cost one token 0.8 us, since every jump over it went to instructions that were not there yet.
__device__ __forceinline__ bool is_nan(const Eight& e) {
    bool is = false;
#pragma unroll
    for (int q = 0; q < 8; ++q) is |= e.v[q] != e.v[q];
    return is;
}
// All of it: nothing that is added changes it.  Steps whose gradients are NaN, as of a loss scaled too far, would take twenty times as long without a
// look at that (4096 tokens at rank 64 between 4096 and 16384 features 5.4 ms).
__device__ __forceinline__ bool stays_nan(const Eight& e) {
    bool is = true;
#pragma unroll
    for (int q = 0; q < 8; ++q) is &= e.v[q] != e.v[q];
    return is;
}
__device__ __forceinline__ void add_products(Eight& e, float h, const Eight& v) {
#pragma unroll
    for (int q = 0; q < 8; ++q) e.v[q] += h * v.v[q];
}
// A lane's four pieces of 128 columns of a token's row: Y, and sum(u) where the token has an adapter, or again(u) where one of those is NaN.
template <class T, class SUM, class AGAIN>
__device__ __forceinline__ void store_token(const uint16_t* Y, const uint4_t* y, uint16_t* out, int64_t col, int64_t m, bool some, SUM sum, AGAIN again) {
    bool is = false;
#pragma unroll
    for (int u = 0; u < 4; ++u) is |= is_nan(sum(u));      // zeros where the token has no adapter
    auto store = [&](int u, Eight e, const Eight& s) {
        if (some) {
#pragma unroll
            for (int q = 0; q < 8; ++q) e.v[q] += s.v[q];
        }
        store_eight<T>(out, col + 32 * u, e, (int)min(m - col - 32 * u, (int64_t)8));
    };
    if (__builtin_expect(!is, 1)) {
#pragma unroll
        for (int u = 0; u < 4; ++u) store(u, widen8<T>(y[u]), sum(u));
        return;
    }
#pragma unroll 1
    for (int u = 0; u < 4; ++u) store(u, Y ? widen8<T>(run_of(Y, col + 32 * u, m)) : Eight{}, again(col + 32 * u));
}

// out = Y + s H B_i of a tile's tokens and 128 columns a wave.  A lane's loads of B are eight columns of four rows, four for each of eight
// results of 16 columns by 16 tokens; which eight is chosen so that lanes store pieces of a row that lie side by side.  The sums of all tokens
// of a tile stay in registers while B goes by once, 16 rows at a time and the next 16 on their way.
template <class T, bool FEW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void rsh_adapters_expand_kernel(const uint16_t* Y, int64_t ld_y, const float* H,
                                                                                                         int parts, const uint16_t* B, const float* scales,
                                                                                                         Index index, Order order, uint16_t* out, int64_t t,
                                                                                                         int64_t m, int r) {
    constexpr int kGroups = (FEW ? kFewTile : kTile / kShares) / 16;
    constexpr int kBlocks = FEW ? 1 : 8;       // of 16 ranks, whose H is in LDS at once
    __shared__ int place[FEW ? sizeof(FewPlace) / sizeof(int) : 1];
    // H of the tile as the matrix unit takes it, which the four waves share: read by each for itself it was as many requests as Y.
    __shared__ __attribute__((aligned(16))) uint4_t shared_upper[FEW ? 1 : kBlocks][FEW ? 1 : kGroups][64];
    __shared__ __attribute__((aligned(8))) uint2_t shared_lo[FEW ? 1 : kBlocks][FEW ? 1 : kGroups][64];
    Members<FEW> tile;
    if (!members<FEW>(index, order, t, (int)(FEW ? blockIdx.x : blockIdx.x / kShares), place, &tile)) return;
    if constexpr (!FEW) {
        const int first = 16 * kGroups * ((int)blockIdx.x % kShares);
        if (first >= tile.count) return;
        tile.token += first;
        tile.count = min(tile.count - first, 16 * kGroups);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15, r16 = (r + 15) / 16 * 16;
    const int64_t col0 = 512 * (int64_t)blockIdx.y + 128 * wave;
    if (FEW && col0 >= m) return;
    const bool active = col0 < m;
    const bool some = tile.adapter < index.n;
    const int64_t col = col0 + 8 * (4 * (c & 3) + (c >> 2));
    // Whole pieces of eight columns where m has them: a load under a condition of its own would have to arrive before the next goes out.
    const bool whole = col0 + 128 <= m;
    int64_t token[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) token[i] = tile.at(16 * i + c);
    struct Four {
        uint4_t y[4];
    };
    auto read = [&](int64_t row) {
        Four v;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t to = col0 + 32 * u + 8 * g;
            if (!Y) v.y[u] = (uint4_t){0, 0, 0, 0};
            else if (whole) v.y[u] = *reinterpret_cast<const uint4_a2*>(Y + row * ld_y + to);
            else v.y[u] = run_of(Y + row * ld_y, to, m);
        }
        return v;
    };
    Four head = {};
    if (active) head = read(token[0]);
    float4_t acc[kGroups][8] = {};
    if (some) {
        const float scale = scales ? scales[tile.adapter] : 1.f;
        const uint16_t* const b = B + (int64_t)tile.adapter * r * m;
        struct Slab {
            uint4_t rows[4];
        };
        auto load = [&](int rank) {
            Slab v;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int row = rank + 4 * g + s;
                if (whole) v.rows[s] = *reinterpret_cast<const uint4_a2*>(b + (int64_t)min(row, r - 1) * m + col);
                else v.rows[s] = run_of(b + (int64_t)min(row, r - 1) * m, col, m);
            }
            return v;
        };
        // H of four ranks of a token, from its parts where there are any.
        auto thirds_of = [&](int64_t row, int rank) {
            const float* const p = H + row * r16 + rank + 4 * g;
            float4_t h = *reinterpret_cast<const float4_t*>(p);
            if constexpr (FEW) {
                float4_t part[kFewParts];
#pragma unroll
                for (int q = 1; q < kFewParts; ++q) part[q] = *reinterpret_cast<const float4_t*>(p + (int64_t)min(q, parts - 1) * t * r16);
#pragma unroll
                for (int q = 1; q < kFewParts; ++q)
                    if (q < parts) h += part[q];
            }
            const float hv[4] = {h[0] * scale, h[1] * scale, h[2] * scale, h[3] * scale};
            return thirds(hv);
        };
        Slab next = {};
        if (active) next = load(0);
        for (int rank0 = 0; rank0 < r16; rank0 += 16 * kBlocks) {
            const int last = min(r16, rank0 + 16 * kBlocks);
            if constexpr (!FEW) {
                if (rank0) __syncthreads();
                const int group = wave % kGroups;
                const int64_t row = tile.at(16 * group + c);
                for (int rank = rank0 + 16 * (wave / kGroups); rank < last; rank += 16 * (4 / kGroups)) {
                    const Thirds h = thirds_of(row, rank);
                    shared_upper[(rank - rank0) / 16][group][lane] = (uint4_t){h.hi[0], h.hi[1], h.mid[0], h.mid[1]};
                    shared_lo[(rank - rank0) / 16][group][lane] = h.lo;
                }
                __syncthreads();
            }
            if (!active) continue;
            for (int rank = rank0; rank < last; rank += 16) {
                Slab v = next;
                if (rank + 16 < r16) next = load(rank + 16);
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int w = 0; w < 4; ++w) v.rows[s][w] = rank + 4 * g + s < r ? v.rows[s][w] : 0u;
                Thirds h[kGroups];
#pragma unroll
                for (int i = 0; i < kGroups; ++i) {
                    if constexpr (FEW) {
                        h[i] = thirds_of(token[i], rank);
                    } else {
                        const uint4_t u = shared_upper[(rank - rank0) / 16][i][lane];
                        h[i] = {{u[0], u[1]}, {u[2], u[3]}, shared_lo[(rank - rank0) / 16][i][lane]};
                    }
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const Column<T> column(v.rows, q);
#pragma unroll
                    for (int i = 0; i < kGroups; ++i) acc[i][q] = column.template times<true>(h[i], acc[i][q]);
                }
            }
        }
    }
    if (!active) return;
    // the others all at once, in registers that B no longer needs
    Four y[kGroups];
    y[0] = head;
#pragma unroll
    for (int i = 1; i < kGroups; ++i)
        if (16 * i < tile.count) y[i] = read(token[i]);
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        if (16 * i >= tile.count) break;
        if (16 * i + c >= tile.count) continue;
        store_token<T>(
            Y ? Y + token[i] * ld_y : nullptr, y[i].y, out + token[i] * m, col0 + 8 * g, m, some,
            [&](int u) {
                Eight e;
#pragma unroll
                for (int q = 0; q < 8; ++q) e.v[q] = acc[i][q][u];
                return e;
            },
            [&](int64_t to) {
                Eight e = {};
#pragma unroll 1
                for (int rank = 0; rank < r && !stays_nan(e); ++rank) {
                    float h = H[token[i] * r16 + rank];
                    for (int p = 1; p < (FEW ? parts : 1); ++p) h += H[((int64_t)p * t + token[i]) * r16 + rank];
                    add_products(e, h * (scales ? scales[tile.adapter] : 1.f), widen8<T>(run_of(B + ((int64_t)tile.adapter * r + rank) * m, to, m)));
                }
                return e;
            });
    }
}

// A few tokens in one launch: every workgroup forms H of its tile for itself, sixteen waves over k, and eight of them go on to 128 columns each.
template <class T, int RT>
__global__ __launch_bounds__(1024) void rsh_adapters_few_kernel(const uint16_t* X, int64_t ld_x, const uint16_t* A, const uint16_t* Y, int64_t ld_y,
                                                                const uint16_t* B, const float* scales, Index index, uint16_t* out, int64_t t, int64_t k,
                                                                int64_t m, int r) {
    constexpr int kWaves = 16, kAhead = RT == 1 ? 4 : 2;
    __shared__ int place[sizeof(FewPlace) / sizeof(int)];
    __shared__ float4_t joined[RT][kWaves][64];
    __shared__ float4_t sums[RT][64];      // as a lane of the matrix unit has them: token lane % 16, ranks 4 (lane / 16) .. + 3
    Members<true> tile;
    if (!members<true>(index, Order{}, t, (int)blockIdx.x, place, &tile)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    const bool some = tile.adapter < index.n;
    const int64_t col0 = kFewColumns * (int64_t)blockIdx.y + 128 * wave, col = col0 + 8 * (4 * (c & 3) + (c >> 2)), token = tile.at(c);
    const bool columns = 128 * wave < kFewColumns && col0 < m, all = col0 + 128 <= m;
    uint4_t rows[RT][4], y[4];
    if (columns) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t to = col0 + 32 * u + 8 * g;
            if (!Y) y[u] = (uint4_t){0, 0, 0, 0};
            else if (all) y[u] = *reinterpret_cast<const uint4_a2*>(Y + token * ld_y + to);
            else y[u] = run_of(Y + token * ld_y, to, m);
        }
        if (some) {
            const uint16_t* const b = B + (int64_t)tile.adapter * r * m;
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int row = 16 * i + 4 * g + s;
                    if (all) rows[i][s] = *reinterpret_cast<const uint4_a2*>(b + (int64_t)min(row, r - 1) * m + col);
                    else rows[i][s] = run_of(b + (int64_t)min(row, r - 1) * m, col, m);
                }
        }
    }
    if (some) {
        const uint16_t* a[RT];
        const uint16_t* const x = X + token * ld_x;
#pragma unroll
        for (int i = 0; i < RT; ++i) a[i] = A + ((int64_t)tile.adapter * r + min(16 * i + c, r - 1)) * k;
        float4_t acc[RT] = {};
        const int64_t whole = k / 64;
        for (int64_t step = wave; step < whole; step += kWaves * kAhead) {
            uint4_t av[kAhead][RT][2], xv[kAhead][2];
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                const int64_t at = 64 * min(step + kWaves * s, whole - 1) + 8 * g;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    xv[s][h] = *reinterpret_cast<const uint4_a2*>(x + at + 32 * h);
#pragma unroll
                    for (int i = 0; i < RT; ++i) av[s][i][h] = *reinterpret_cast<const uint4_a2*>(a[i] + at + 32 * h);
                }
            }
#pragma unroll
            for (int s = 0; s < kAhead; ++s)
                if (step + kWaves * s < whole)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < RT; ++i) acc[i] = T::mfma16(av[s][i][h], xv[s][h], acc[i]);
        }
        if (k % 64 && whole % kWaves == wave) {
            const int64_t at = 64 * whole + 8 * g;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4_t xv = run_of(x, at + 32 * h, k);
#pragma unroll
                for (int i = 0; i < RT; ++i) acc[i] = T::mfma16(run_of(a[i], at + 32 * h, k), xv, acc[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) joined[i][wave][lane] = acc[i];
        __syncthreads();
        if (wave < RT) {
            float4_t s = joined[wave][0][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) s += joined[wave][w][lane];
            const float scale = scales ? scales[tile.adapter] : 1.f;
#pragma unroll
            for (int v = 0; v < 4; ++v) s[v] = 16 * wave + 4 * g + v < r ? s[v] * scale : 0.f;
            sums[wave][lane] = s;
        }
        __syncthreads();
    }
    if (!columns) return;
    float4_t acc[8] = {};
    if (some) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const float4_t h = sums[i][lane];
            const float hv[4] = {h[0], h[1], h[2], h[3]};
            const Thirds three = thirds(hv);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int w = 0; w < 4; ++w) rows[i][s][w] = 16 * i + 4 * g + s < r ? rows[i][s][w] : 0u;
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[q] = Column<T>(rows[i], q).template times<true>(three, acc[q]);
        }
    }
    if (c >= tile.count) return;
    store_token<T>(
        Y ? Y + token * ld_y : nullptr, y, out + token * m, col0 + 8 * g, m, some,
        [&](int u) {
            Eight e;
#pragma unroll
            for (int q = 0; q < 8; ++q) e.v[q] = acc[q][u];
            return e;
        },
        [&](int64_t to) {
            Eight e = {};
#pragma unroll 1
            for (int rank = 0; rank < r && !stays_nan(e); ++rank)
                add_products(e, sums[rank / 16][16 * (rank % 16 / 4) + c][rank % 4],
                             widen8<T>(run_of(B + ((int64_t)tile.adapter * r + rank) * m, to, m)));
            return e;
        });
}

// H of all tokens from its parts.
__global__ __launch_bounds__(256) void rsh_adapters_join_kernel(const float4_t* from, float4_t* to, int64_t n, int parts) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        float4_t s = from[i];
        for (int p = 1; p < parts; ++p) s += from[p * n + i];
        to[i] = s;
    }
}

// s H^T X over a part of the tokens of adapter blockIdx.y, 16 RT ranks by 128 columns: into `out` where there is one part, into `sums`
// ([part][adapter][rank][column], fp32) where there are more.
template <class T, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void rsh_adapters_outer_kernel(const uint16_t* X, int64_t ld_x, const float* H, const float* scales, Order order,
                                                                        uint16_t* out, float* sums, int parts, int64_t k, int n, int r) {
    __shared__ float4_t joined[WAVES][8][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15, r16 = (r + 15) / 16 * 16;
    const int adapter = blockIdx.y, part = blockIdx.z % parts, r0 = 16 * RT * ((int)blockIdx.z / parts);
    const int start = order.starts[adapter], tokens = order.starts[adapter + 1] - start, share = (tokens + parts - 1) / parts;
    const int begin = start + (int)min((int64_t)tokens, (int64_t)part * share), end = start + (int)min((int64_t)tokens, (int64_t)(part + 1) * share);
    const int64_t col = 128 * (int64_t)blockIdx.x + 8 * c;
    float4_t acc[RT][8] = {};
    // 16 tokens a turn and wave, four of them a lane's.
    struct Slab {
        uint4_t x[4];
        float h[RT][4];
    };
    const int valid = (int)min(k - col, (int64_t)8);
    const bool whole = 128 * (int64_t)blockIdx.x + 128 <= k;
    struct Four {
        int token[4];
    };
    auto find = [&](int i0) {
        Four f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f.token[i] = order.token[min(i0 + 4 * g + i, end - 1)];
        return f;
    };
    auto load = [&](const Four& f) {       // of tokens behind the last: the last, which counts as zeros when it is used
        Slab s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t token = f.token[i];
            if (whole) s.x[i] = *reinterpret_cast<const uint4_a2*>(X + token * ld_x + col);
            else s.x[i] = run_of(X + token * ld_x, col, k);
#pragma unroll
            for (int j = 0; j < RT; ++j) s.h[j][i] = H[token * r16 + min(r0 + 16 * j, r16 - 16) + c];
        }
        return s;
    };
    const int first = begin + 16 * wave;
    if (first < end) {
        Slab next = load(find(first));
        Four after = find(first + 16 * WAVES);
        for (int i0 = first; i0 < end; i0 += 16 * WAVES) {
            Slab s = next;
            if (i0 + 16 * WAVES < end) {
                next = load(after);
                after = find(i0 + 32 * WAVES);
            }
            if (i0 + 16 > end) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = i0 + 4 * g + i < end;
#pragma unroll
                    for (int w = 0; w < 4; ++w) s.x[i][w] = in ? s.x[i][w] : 0u;
#pragma unroll
                    for (int j = 0; j < RT; ++j) s.h[j][i] = in ? s.h[j][i] : 0.f;
                }
            }
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                const Thirds h = thirds(s.h[j]);
#pragma unroll
                for (int q = 0; q < 8; ++q) acc[j][q] = Column<T>(s.x, q).template times<false>(h, acc[j][q]);
            }
        }
    }
    // No tokens, no product: the scale of an adapter that nothing uses may be anything, and an infinite one leaves an empty part out.
    const float scale = scales && begin < end ? scales[adapter] : 1.f;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; ++q) joined[wave][q][lane] = acc[i][q];
        __syncthreads();
        for (int v = wave; v < 4; v += WAVES) {
            const int rank = r0 + 16 * i + 4 * g + v;
            Eight e;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float s = joined[0][q][lane][v];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) s += joined[w][q][lane][v];
                e.v[q] = s;
            }
            if (rank >= r || col >= k) continue;
            if (__builtin_expect(is_nan(e), 0)) {
                e = {};
#pragma unroll 1
                for (int n = begin; n < end && !stays_nan(e); ++n) {
                    const int64_t token = order.token[n];
                    add_products(e, H[token * r16 + rank], widen8<T>(run_of(X + token * ld_x, col, k)));
                }
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) e.v[q] *= scale;
            const int64_t at = ((int64_t)adapter * r + rank) * k + col;
            if (parts == 1) store_eight<T>(out, at, e, valid);
            else store_eight<F32>(sums, (int64_t)part * n * r * k + at, e, valid);
        }
    }
}

// The parts of a factor's gradient, added up in their order.
template <class T>
__global__ __launch_bounds__(256) void rsh_adapters_sum_kernel(const float* sums, uint16_t* out, int64_t n, int parts) {
    for (int64_t i = 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < n; i += 8 * (int64_t)gridDim.x * 256) {
        const int valid = (int)min(n - i, (int64_t)8);
        Eight s = load_eight<F32>(sums, i, valid);
        for (int p = 1; p < parts; ++p) {
            const Eight e = load_eight<F32>(sums, p * n + i, valid);
#pragma unroll
            for (int q = 0; q < 8; ++q) s.v[q] += e.v[q];
        }
        store_eight<T>(out, i, s, valid);
    }
}

namespace {
int launched() { return hipGetLastError() == hipSuccess ? RSH_OK : RSH_ERR_HIP; }
int64_t rounded(int64_t bytes) { return (bytes + 15) / 16 * 16; }
int64_t wide_rank(int r) { return (r + 15) / 16 * 16; }

template <class F>
void by_half(int type, F f) {
    if (type == RSH_F16) f(F16());
    else f(BF16());
}
template <class F>
void by_rank(int r, F f) {
    if (r <= 16) f(std::integral_constant<int, 1>());
    else if (r <= 32) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

int64_t most_tiles(int64_t t, int n) { return t / kTile + std::min<int64_t>(t, n + 1); }

// The order's place in the work memory.
struct Sorted {
    int64_t token, starts, tiles, n_tiles, bytes;
    Sorted(int64_t t, int n) {
        token = 0;
        starts = rounded(4 * t);
        tiles = starts + rounded(4 * (n + 2));
        n_tiles = tiles + (int64_t)sizeof(Tile) * most_tiles(t, n);
        bytes = n_tiles + 16;
    }
    Order at(void* work) const {
        char* const w = (char*)work;
        return {(const int32_t*)(w + token), (const int32_t*)(w + starts), (const Tile*)(w + tiles), (const int32_t*)(w + n_tiles)};
    }
};

// Whether a few tokens go in one launch, in which every workgroup reads its A for itself.  It takes 4.4 us and 1 us for every 30 KB of A (7.0 us at
// k = 1024 and rank 16, 13.9 at 8192).  Called one by one two launches cost the host 3 to 4 us more (16.4 for 12.6 us at 1024, 16.7 for 13.7 at
// 8192): so one up to 256 KB, and while what all workgroups read together stays below 64 MB.  Inside a graph of many calls the host does not count, and
// two would be as good at 1024 (8.1 for 7.5 us) and better at 8192 (8.9 for 13.6).
bool in_one(int64_t t, int64_t k, int64_t m, int r) {
    const int64_t factor = 2 * k * wide_rank(r), columns = (m + kFewColumns - 1) / kFewColumns;
    return t <= kFewTokens && r <= 32 && factor <= (1 << 18) && factor * columns * t <= (1 << 26);
}

// Parts of the long axis of a shrinking product, and the steps of 64 in each: as many as bring all compute units their fill of workgroups at
// once, since a second round costs as much as the first (4096 tokens at rank 64 by 16384 columns in 16 parts and four rounds 63 us; the training
// step between 4096 and 16384 columns with half as many 273 us, with twice as many 291, for 267).  Tiles are counted as if every adapter had some: 512
// tokens of four adapters at 28672 features take 31 us with 4 of them loaded, 40 with 64 and 147 with 512.
constexpr int kFewWaves = 8, kOuterWaves = 4;
constexpr int shrink_waves(int r) { return r <= 16 ? 8 : 4; }      // fewer parts to add up where the registers leave room (63 -> 60 us)
int slots_of(int r) { return r <= 16 ? 1024 : r <= 32 ? 768 : 512; }     // workgroups of four waves that fit the chip, by their registers
struct Split {
    int parts, steps;
    Split(int64_t t, int64_t k, int n, int r, bool few) {
        const int64_t all = (k + 63) / 64, waves = few ? kFewWaves : shrink_waves(r);
        const int64_t blocks = (few ? t : most_tiles(t, n)) * ((r + 63) / 64), slots = few ? 512 : slots_of(r) * 4 / shrink_waves(r);
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>(few ? kFewParts : 16, slots / blocks));
        const int64_t each = (all + want * waves - 1) / (want * waves) * waves;
        steps = (int)each;
        parts = (int)((all + each - 1) / each);
    }
};

// Parts of the tokens in a factor's gradient: as many as fill the chip if all adapters have tokens alike (8 or 32 in place of 16 take the same time).  With
// 4096 tokens of one adapter at 4096 features and rank 64 a step takes 163 us if it is the only one loaded, 184 of 4, 343 of 64 and 443 of
// 256, whose gradients are 268 MB of zeros.
int outer_parts(int64_t t, int64_t k, int n, int r) {
    const int64_t blocks = (k + 127) / 128 * n * ((r + 63) / 64);
    return (int)std::max<int64_t>(1, std::min<int64_t>({16, slots_of(r) / blocks, t / 64}));
}

void sort(const rsh_adapters_t& a, void* work, hipStream_t st) {
    const Sorted s(a.t, a.n);
    const int waves = std::min(kSortThreads / 64, kSortWords / (a.n + 1));
    char* const w = (char*)work;
    hipLaunchKernelGGL(rsh_adapters_sort_kernel, dim3(1), dim3(kSortThreads), 0, st, Index{a.index, a.index_size == 8, a.n}, a.t, waves, kTile,
                       (int32_t*)(w + s.token), (int32_t*)(w + s.starts), (Tile*)(w + s.tiles), (int32_t*)(w + s.n_tiles));
}

template <class T>
void shrink(const rsh_adapters_t& a, bool few, const void* X, int64_t ld, int64_t k, const void* A, const Order& order, const Split& split, float* H,
            hipStream_t st) {
    const Index index = {a.index, a.index_size == 8, a.n};
    by_rank(a.r, [&](auto rt) {
        constexpr int RT = decltype(rt)::value;
        const dim3 grid((unsigned)(few ? a.t : most_tiles(a.t, a.n)), (a.r + 16 * RT - 1) / (16 * RT), split.parts);
        if (few)
            hipLaunchKernelGGL((rsh_adapters_shrink_kernel<T, RT, 1, true, kFewWaves>), grid, dim3(64 * kFewWaves), 0, st, (const uint16_t*)X, ld,
                               (const uint16_t*)A, index, order, H, a.t, k, a.r, split.steps);
        else
            hipLaunchKernelGGL((rsh_adapters_shrink_kernel<T, RT, 4, false, shrink_waves(16 * RT)>), grid, dim3(64 * shrink_waves(16 * RT)), 0, st, (const uint16_t*)X, ld,
                               (const uint16_t*)A, index, order, H, a.t, k, a.r, split.steps);
    });
}

template <class T>
void expand(const rsh_adapters_t& a, bool few, const void* Y, int64_t ld, const float* H, int parts, const void* B, const Order& order, void* out,
            int64_t m, hipStream_t st) {
    const Index index = {a.index, a.index_size == 8, a.n};
    const dim3 grid((unsigned)(few ? a.t : kShares * most_tiles(a.t, a.n)), (unsigned)((m + 511) / 512));
    if (few)
        hipLaunchKernelGGL((rsh_adapters_expand_kernel<T, true>), grid, dim3(256), 0, st, (const uint16_t*)Y, ld, H, parts, (const uint16_t*)B, a.scales,
                           index, order, (uint16_t*)out, a.t, m, a.r);
    else
        hipLaunchKernelGGL((rsh_adapters_expand_kernel<T, false>), grid, dim3(256), 0, st, (const uint16_t*)Y, ld, H, 1, (const uint16_t*)B, a.scales, index,
                           order, (uint16_t*)out, a.t, m, a.r);
}

void join(const float* from, float* to, int64_t t, int r, int parts, hipStream_t st) {
    const int64_t n = t * wide_rank(r) / 4;
    hipLaunchKernelGGL(rsh_adapters_join_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, st, (const float4_t*)from,
                       (float4_t*)to, n, parts);
}

template <class T>
void outer(const rsh_adapters_t& a, const void* X, int64_t ld, int64_t k, const float* H, const Order& order, void* out, float* sums, hipStream_t st) {
    const int parts = outer_parts(a.t, k, a.n, a.r);
    by_rank(a.r, [&](auto rt) {
        constexpr int RT = decltype(rt)::value;
        const dim3 grid((unsigned)((k + 127) / 128), a.n, (a.r + 16 * RT - 1) / (16 * RT) * parts);
        hipLaunchKernelGGL((rsh_adapters_outer_kernel<T, RT, kOuterWaves>), grid, dim3(64 * kOuterWaves), 0, st, (const uint16_t*)X, ld, H, a.scales, order, (uint16_t*)out, sums,
                           parts, k, a.n, a.r);
    });
    if (parts > 1) {
        const int64_t n = (int64_t)a.n * a.r * k;
        hipLaunchKernelGGL(rsh_adapters_sum_kernel<T>, dim3((unsigned)std::min<int64_t>((n + 2047) / 2048, 4096)), dim3(256), 0, st, sums, (uint16_t*)out, n,
                           parts);
    }
}
}  // namespace

// What a forward pass leaves for the gradients: H, and behind it the order of the tokens where it has made one.
int64_t adapters_kept(int64_t t, int n, int r) { return t * wide_rank(r) * 4 + (t <= kFewTokens ? 0 : Sorted(t, n).bytes); }

int64_t adapters_forward_work(int64_t t, int64_t k, int64_t m, int n, int r, bool keep) {
    if (!keep && in_one(t, k, m, r)) return 0;
    const bool few = t <= kFewTokens;
    return (few ? 0 : Sorted(t, n).bytes) + (Split(t, k, n, r, few).parts + 1) * t * wide_rank(r) * 4;
}

int64_t adapters_backward_work(int64_t t, int64_t k, int64_t m, int n, int r) {
    int64_t sums = 0;
    for (int64_t w : {k, m}) {
        const int parts = outer_parts(t, w, n, r);
        if (parts > 1) sums = std::max(sums, parts * w * n * r * 4);
    }
    return Sorted(t, n).bytes + (Split(t, m, n, r, false).parts + 1) * t * wide_rank(r) * 4 + sums;
}

int launch_adapters_forward(const rsh_adapters_t& a, void* work, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    const bool few = a.t <= kFewTokens;
    if (!a.kept && in_one(a.t, a.k, a.m, a.r)) {
        const dim3 grid((unsigned)a.t, (unsigned)((a.m + kFewColumns - 1) / kFewColumns));
        by_half(a.type, [&](auto half) {
            using T = decltype(half);
            auto launch = [&](auto rt) {
                hipLaunchKernelGGL((rsh_adapters_few_kernel<T, decltype(rt)::value>), grid, dim3(1024), 0, st, (const uint16_t*)a.X, a.ld_x,
                                   (const uint16_t*)a.A, (const uint16_t*)a.Y, a.ld_y, (const uint16_t*)a.B, a.scales,
                                   Index{a.index, a.index_size == 8, a.n}, (uint16_t*)a.out, a.t, a.k, a.m, a.r);
            };
            if (a.r <= 16) launch(std::integral_constant<int, 1>());
            else launch(std::integral_constant<int, 2>());
        });
        return launched();
    }
    const Split split(a.t, a.k, a.n, a.r, few);
    const Sorted s(a.t, a.n);
    float* const H = (float*)((char*)work + (few ? 0 : s.bytes));
    void* const order = a.kept ? (char*)a.kept + a.t * wide_rank(a.r) * 4 : work;
    if (!few) sort(a, order, st);
    by_half(a.type, [&](auto half) {
        using T = decltype(half);
        float* const direct = split.parts == 1 && a.kept ? (float*)a.kept : H;
        shrink<T>(a, few, a.X, a.ld_x, a.k, a.A, s.at(order), split, direct, st);
        int parts = split.parts;
        const float* all = direct;
        if (parts > 1 && (a.kept || !few)) {
            float* const to = a.kept ? (float*)a.kept : H + parts * a.t * wide_rank(a.r);
            join(H, to, a.t, a.r, parts, st);
            all = to;
            parts = 1;
        }
        expand<T>(a, few, a.Y, a.ld_y, all, parts, a.B, s.at(order), a.out, a.m, st);
    });
    return launched();
}

int launch_adapters_backward(const rsh_adapters_t& a, const void* dout, int64_t ld_dout, void* dX, void* dA, void* dB, void* work, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    const Split split(a.t, a.m, a.n, a.r, false);
    const Sorted s(a.t, a.n);
    float* const parts = (float*)((char*)work + s.bytes);
    float* const dH = parts + (split.parts > 1 ? split.parts * a.t * wide_rank(a.r) : 0);
    float* const sums = parts + (split.parts + 1) * a.t * wide_rank(a.r);
    const bool sorted = a.t > kFewTokens;
    const Order order = s.at(sorted ? (char*)a.kept + a.t * wide_rank(a.r) * 4 : work);
    if (!sorted) sort(a, work, st);
    by_half(a.type, [&](auto half) {
        using T = decltype(half);
        if (dX || dA) {
            shrink<T>(a, false, dout, ld_dout, a.m, a.B, order, split, parts, st);
            if (split.parts > 1) join(parts, dH, a.t, a.r, split.parts, st);
        }
        if (dX) expand<T>(a, false, nullptr, 0, dH, 1, a.A, order, dX, a.k, st);
        if (dA) outer<T>(a, a.X, a.ld_x, a.k, dH, order, dA, sums, st);
        if (dB) outer<T>(a, dout, ld_dout, a.m, (const float*)a.kept, order, dB, sums, st);
    });
    return launched();
}

}  // namespace rsh
