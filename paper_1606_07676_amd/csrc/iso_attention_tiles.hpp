// gfx950 matrix kernels for attention over an isomorphic neighbourhood, 16-bit types.
//
// A workgroup takes a tile of the torus: 64 columns (rank, head), 16 for each of its four wavefronts, against the rows
// (keys) that any of its ranks reads.  The tile's box plus the neighbourhood's reach holds far fewer rows than ranks times
// neighbours (8 x 8 ranks, 13 x 13 neighbours: 400 rows in place of 10816), each is read once and staged in LDS, and the
// scores of 16 rows against 16 columns are one matrix product of which the pairs that are no neighbours are masked away
// (there: a third).  The table of who is whose neighbour is the same for all tiles: see iso_tiles.hpp.
//
// Scores are computed transposed, S^T = K Q^T, so that a lane holds one column and four rows of each 16 x 16 block, and the
// weights of two blocks are, in registers, the right-hand operand of out^T += V^T P^T: the order of rows inside a product
// of 32 is free as long as both operands keep it.  V^T comes out of the row-major LDS tile through the transposing read.
//
// Vector arithmetic on the scores bounds these kernels, and waiting for LDS and for each other, not the matrix products
// (vector units busy for 62 % of the time, matrix units for 17 %, memory for a third; 256 x 256 ranks, 169 neighbours), so a
// score costs as few instructions as it can: the table holds the byte offset of the pair's bias in LDS, and for pairs that
// are no neighbours that of a -inf.  Rows go from memory to LDS without passing through registers, one chunk ahead of the
// one in use.
//
// Rounding: the weights P and, backward, da are rounded to the tensors' type for the second product (a relative 2^-9 in
// bfloat16, as large as that of the output); scores, sums, maxima, lse and all accumulators stay in 32 bits.
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_fastdiv.hpp"
#include "iso_tiles.hpp"

namespace iso {

struct TileDim {                           // of the torus, the last dimension first
    FastDiv tiles;
    int32_t tile, size, inner, wraps;
};

struct TileArgs {
    AttentionArgs a;
    TileDim dim[ISO_MAX_DIMS];
    FastDiv n_tiles, parts, biases;        // parts: sets of `heads` q heads that share a key head; biases: s + 1
    uint32_t items, per_xcd;               // (key head, tile, part), and how many of them one XCD takes
    int32_t heads;                         // columns of one rank
    int32_t chunks;                        // of TileLds<DP>::kRows rows
    int32_t words;                         // of a position
    const uint2 *column_at, *row_at;       // [][words]: positions relative to the tile's first rank, four dimensions in a word
    const uint32_t *active;
    const uint16_t *index;
    const uint32_t *slots;                 // the bias's gradient, or null: see TilePlan
    int32_t slot_rounds, slot_words;
    const void *zeros;                     // a row of zeros
};

// What is read from LDS while rows are on their way there has to be of these types: the compiler takes a read of a struct for
// one of those rows, and waits for all of them first.
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int32_t i4 __attribute__((ext_vector_type(4)));

template <typename T> struct Matrix;
template <> struct Matrix<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    typedef float f4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f4 multiply(x8 a, x8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Matrix<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    typedef float f4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f4 multiply(x8 a, x8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Maximum and sum over the four lanes that hold the rows of one column.
__device__ __forceinline__ float column_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// LDS of a tile kernel: chunks of rows of two tensors, then per row of the tile its rank and segment, then the biases.
//
// Loads into LDS write a wavefront's 64 pieces of 16 bytes one after the other, so rows are dense; which piece of its row a
// lane fetches is permuted by the row, so that the 16 rows of a product's operand lie in 16 different groups of banks.
template <int DP> struct TileLds {
    static constexpr int kRows = DP > 32 ? 32 : 64;                 // of a chunk
    static constexpr int kGroups = kRows / 16;
    static constexpr int kRowBytes = DP * 2, kPieces = DP / 8, kTensor = kRows * kRowBytes;
    static constexpr int kLoads = (kRows * kPieces + 255) / 256;
    // The table of a chunk goes to LDS with its rows, or to registers where LDS is what limits the workgroups of a CU (rows of
    // 128: 53 us in place of 59 for 32 x 32 x 32, 27 neighbours; rows of 64 the other way round: 121 in place of 131 us for
    // 256 x 256, 169 neighbours).
    static constexpr bool kIndexInLds = DP <= 96;
    static constexpr int kIndex = kIndexInLds ? kGroups * 4 * 512 : 0;
    static constexpr int kStage = 2 * kTensor + kIndex;
    unsigned char *chunk;                  // [2]: rows of the first tensor, of the second, table
    int32_t *rank, *segment;
    uint32_t *active;                      // [chunks]: bit 4 * wave + g: group g holds a neighbour of one of the wavefront's columns
    float *bias;

    static __host__ __device__ int words(int chunks) { return (chunks + 3) / 4 * 4; }
    static __host__ __device__ size_t bytes(int chunks, size_t floats) {
        return 2 * (size_t)kStage + (size_t)chunks * kRows * 8 + words(chunks) * 4 + floats * 4;
    }
    __device__ TileLds(unsigned char *at, int chunks) {
        chunk = at;
        rank = (int32_t *)(at + 2 * kStage);
        segment = rank + chunks * kRows;
        active = (uint32_t *)(segment + chunks * kRows);
        bias = (float *)(active + words(chunks));
    }
    static __device__ __forceinline__ int place(int row, int piece) {
        return DP == 32 ? piece ^ (row >> 2 & 3) : DP == 64 ? piece ^ (row >> 1 & 7) : DP == 128 ? piece ^ (row & 15)
                                                                                              : (piece + (row >> 2 & 3)) % 12;
    }
    static __device__ __forceinline__ int piece_at(int row, int place) {
        return DP == 32 ? place ^ (row >> 2 & 3) : DP == 64 ? place ^ (row >> 1 & 7) : DP == 128 ? place ^ (row & 15)
                                                                                              : (place + 12 - (row >> 2 & 3)) % 12;
    }
};

constexpr int32_t kNoToken = INT32_MIN;    // segment of a row that is outside the mesh or holds no token
constexpr int32_t kNoColumn = INT32_MIN + 1;

// Rank at a position relative to the tile's first rank, -1 outside the mesh (and for positions that only columns outside the
// torus, of a ragged tile, refer to).  The tile's own position is scalar work.
template <bool COLUMN>
__device__ __forceinline__ void add_dim(const TileDim &d, uint32_t &tile, int32_t at, int32_t &rank, bool &there) {
    uint32_t rest, place;
    fast_divmod(tile, d.tiles, rest, place);
    tile = rest;
    int32_t x = (int32_t)place * d.tile + at;
    if (!COLUMN && d.wraps) {
        x += x < 0 ? d.size : 0;
        x -= x >= d.size ? d.size : 0;
    }
    there = there && (uint32_t)x < (uint32_t)d.size;
    rank += x * d.inner;
}
template <bool COLUMN> __device__ __forceinline__ int32_t rank_at(const TileArgs &t, uint32_t tile, const uint2 *at, uint2 word) {
    int32_t rank = 0;
    bool there = true;
    const int d = t.a.torus.d;
    add_dim<COLUMN>(t.dim[0], tile, (int16_t)(word.x & 0xFFFF), rank, there);
    if (d > 1) add_dim<COLUMN>(t.dim[1], tile, (int32_t)word.x >> 16, rank, there);
    if (d > 2) add_dim<COLUMN>(t.dim[2], tile, (int16_t)(word.y & 0xFFFF), rank, there);
    if (d > 3) add_dim<COLUMN>(t.dim[3], tile, (int32_t)word.y >> 16, rank, there);
    for (int j = 4; j < d; ++j) {
        const uint2 more = at[j / 4];
        const uint32_t two = j % 4 < 2 ? more.x : more.y;
        add_dim<COLUMN>(t.dim[j], tile, j % 2 ? (int32_t)two >> 16 : (int16_t)(two & 0xFFFF), rank, there);
    }
    return there ? rank : -1;
}
template <bool COLUMN> __device__ __forceinline__ int32_t rank_at(const TileArgs &t, uint32_t tile, const uint2 *at) {
    return rank_at<COLUMN>(t, tile, at, at[0]);
}

// What a workgroup works on: workgroups are handed to the 8 XCDs in turn, and each XCD takes a run of consecutive tiles of
// one head, whose rows its L2 then holds for all tiles that share them.
struct TileWork {
    uint32_t tile;
    int key_head, part;
    bool any;
};
__device__ __forceinline__ TileWork tile_work(const TileArgs &t) {
    TileWork w;
    const uint32_t block = t.a.first_block + blockIdx.x, item = (block & 7) * t.per_xcd + (block >> 3);
    uint32_t pair, part, head, tile;
    fast_divmod(item, t.parts, pair, part);
    fast_divmod(pair, t.n_tiles, head, tile);
    w.part = part;
    w.tile = tile;
    w.key_head = head;
    w.any = item < t.items;
    return w;
}

// Ranks and segments of the tile's rows.  A row that is not there keeps rank -1 where segments are compared, and is then
// staged as zeros; on a torus without segments only columns outside the torus refer to such rows, and any rank serves.
template <int DP, bool SEGMENTS> __device__ __forceinline__ void tile_rows(const TileArgs &t, uint32_t tile, TileLds<DP> &lds) {
    const int rows = t.chunks * TileLds<DP>::kRows;
    const auto one = [&](int u, uint2 word) {
        const int32_t rank = rank_at<false>(t, tile, t.row_at + (int64_t)u * t.words, word);
        if (SEGMENTS) {
            int32_t segment = rank < 0 ? kNoToken : t.a.segments ? t.a.segments[rank] : 0;
            if (segment < 0) segment = kNoToken;
            lds.rank[u] = segment < 0 ? -1 : rank;
            lds.segment[u] = segment;
        } else {
            lds.rank[u] = max(rank, 0);
        }
    };
    for (int c = threadIdx.x; c < t.chunks; c += 256)
        lds.active[c] = TileLds<DP>::kGroups == 4 ? t.active[c] : t.active[c / 2] >> (c % 2 * 2) & 0x3333;
    for (int u = threadIdx.x; u < rows; u += 512) {                 // two trips to memory under way at a time
        const bool second = u + 256 < rows;
        const uint2 a = t.row_at[(int64_t)u * t.words], b = t.row_at[(int64_t)(second ? u + 256 : u) * t.words];
        one(u, a);
        if (second) one(u + 256, b);
    }
}

__device__ __forceinline__ int32_t column_segment(const AttentionArgs &a, int64_t rank) {
    const int32_t own = rank < 0 ? kNoColumn : a.segments ? a.segments[rank] : 0;
    return own < 0 ? kNoColumn : own;
}

// Biases of `heads` q heads times log2 e in LDS, a -inf behind each; zeros where there are none.
template <typename T>
__device__ __forceinline__ void tile_biases(const TileArgs &t, int first_head, int heads, float *at) {
    const AttentionArgs &a = t.a;
    const int s = a.torus.s;
    for (int i = threadIdx.x; i < heads * (s + 1); i += 256) {
        uint32_t h, j;
        fast_divmod(i, t.biases, h, j);
        float b = (int)j == s ? -INFINITY : a.bias ? (float)((const T *)a.bias)[(int64_t)(first_head + h) * s + j] : 0.f;
        // the product must not make an infinity of a bias near the type's lowest value
        if (fabsf(b) < INFINITY) b = fminf(fmaxf(b * kLog2e, -3.4e38f), 3.4e38f);
        at[i] = b;
    }
}

// One chunk of rows of two tensors on its way into LDS.  Tensors are given by the address of rank 0's row and the bytes
// between ranks, below 2^32; a lane whose piece lies behind the row's end reads zeros for every rank.
template <int DP, bool SEGMENTS> struct RowLoads {
    typedef TileLds<DP> Lds;
    const unsigned char *first[Lds::kLoads], *second[Lds::kLoads], *zeros, *index;
    uint32_t first_stride[Lds::kLoads], second_stride[Lds::kLoads];

    __device__ __forceinline__ RowLoads(const TileArgs &t, const Heads &a, const Heads &b, int head) : zeros((const unsigned char *)t.zeros), index((const unsigned char *)t.index + threadIdx.x * 16) {
#pragma unroll
        for (int i = 0; i < Lds::kLoads; ++i) {
            const int unit = threadIdx.x + 256 * i, piece = Lds::piece_at(unit / Lds::kPieces, unit % Lds::kPieces);
            const bool inside = piece * 8 < t.a.head_dim;
            first[i] = inside ? (const unsigned char *)a.data + head * a.head_stride * 2 + piece * 16 : zeros;
            second[i] = inside ? (const unsigned char *)b.data + head * b.head_stride * 2 + piece * 16 : zeros;
            first_stride[i] = inside ? (uint32_t)(a.rank_stride * 2) : 0;
            second_stride[i] = inside ? (uint32_t)(b.rank_stride * 2) : 0;
        }
    }
    __device__ __forceinline__ void start(const TileLds<DP> &lds, int chunk_number, int stage) const {
        const int32_t *rank = lds.rank + chunk_number * Lds::kRows;
        unsigned char *chunk = lds.chunk + stage * Lds::kStage;
#pragma unroll
        for (int i = 0; i < Lds::kLoads; ++i) {
            const int unit = threadIdx.x + 256 * i, row = unit / Lds::kPieces;
            if (Lds::kRows * Lds::kPieces % 256 && unit >= Lds::kRows * Lds::kPieces) break;      // whole wavefronts
            const int32_t r = rank[row];
            const unsigned char *a = first[i] + (uint64_t)(uint32_t)r * first_stride[i];
            const unsigned char *b = second[i] + (uint64_t)(uint32_t)r * second_stride[i];
            if (SEGMENTS && r < 0) a = b = zeros;
            unsigned char *to = chunk + __builtin_amdgcn_readfirstlane((threadIdx.x & ~63u) * 16 + 4096 * i);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)a,
                                             (__attribute__((address_space(3))) void *)to, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)b,
                                             (__attribute__((address_space(3))) void *)(to + Lds::kTensor), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < Lds::kIndex / 4096; ++i) {
            unsigned char *to = chunk + 2 * Lds::kTensor + __builtin_amdgcn_readfirstlane((threadIdx.x & ~63u) * 16 + 4096 * i);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(index + (int64_t)chunk_number * Lds::kIndex + 4096 * i),
                                             (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        }
    }
};
// The chunk that was started is in LDS, and all wavefronts have done with the one before.
__device__ __forceinline__ void wait_for_rows() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The table's entries of a chunk: byte offsets of the biases of this lane's column and rows 4 (lane / 16) + 0..3 of each group.
template <int DP> struct Pairs {
    static constexpr int kPairs = TileLds<DP>::kGroups / 2;
    u4 of[kPairs];
    uint32_t active;

    __device__ __forceinline__ void read(const u4 *at) {
        at += (threadIdx.x >> 6) * 64 + (threadIdx.x & 63);
#pragma unroll
        for (int n = 0; n < kPairs; ++n) of[n] = at[n * kTileWaves * 64];
    }
    // before a chunk's rows are started
    __device__ __forceinline__ void prefetch(const TileArgs &t, int chunk) {
        if constexpr (!TileLds<DP>::kIndexInLds) read((const u4 *)t.index + (int64_t)chunk * kPairs * kTileWaves * 64);
    }
    // once they are there; next: what was prefetched
    __device__ __forceinline__ Pairs(const TileLds<DP> &lds, const Pairs &next, int chunk, int stage) {
        active = __builtin_amdgcn_readfirstlane(lds.active[chunk] >> ((threadIdx.x >> 6) * 4)) & 15;
        if constexpr (TileLds<DP>::kIndexInLds) {
            read((const u4 *)(lds.chunk + stage * TileLds<DP>::kStage + 2 * TileLds<DP>::kTensor));
        } else {
#pragma unroll
            for (int n = 0; n < kPairs; ++n) of[n] = next.of[n];
        }
    }
    __device__ Pairs() {}
    __device__ __forceinline__ uint32_t at(int g, int r) const {
        const u4 &eight = of[g / 2];
        const uint32_t two = g % 2 ? (r < 2 ? eight.z : eight.w) : (r < 2 ? eight.x : eight.y);
        return r % 2 ? two >> 16 : two & 0xFFFF;
    }
    __device__ __forceinline__ float bias(const unsigned char *base, int g, int r) const { return *(const float *)(base + at(g, r)); }
};

// A column's row as right-hand operand: lane holds column lane % 16, elements 32 k + 8 (lane / 16) + 0..7.
template <typename T, int DP>
__device__ __forceinline__ void load_column(const Heads &h, int64_t rank, int head, int head_dim, typename Matrix<T>::x8 (&x)[DP / 32]) {
    const int at = (threadIdx.x & 63) / 16 * 8;
    const T *row = (const T *)h.data + rank * h.rank_stride + head * h.head_stride;
#pragma unroll
    for (int k = 0; k < DP / 32; ++k) {
        x[k] = {};
        if (rank >= 0 && 32 * k + at < head_dim) x[k] = *(const typename Matrix<T>::x8 *)(row + 32 * k + at);
    }
}

// Transposing reads: lane i of 16 gets column i of four rows whose 16 columns the lanes' addresses name, four columns each.
// The compiler takes the builtin for a read of whatever is on its way into LDS and waits for the next chunk's rows before
// it; here the reads are waited for where they are issued.
struct Turned {
    u4 first, second;
};
template <int HALF> __device__ __forceinline__ Turned read_transposed(uint32_t first, uint32_t second) {
    uint2 a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %2, %5\n\tds_read_b64_tr_b16 %3, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d)
                 : "v"(first), "v"(second), "n"(HALF));
    return {u4{a.x, a.y, b.x, b.y}, u4{c.x, c.y, d.x, d.y}};
}

// Where a lane finds its pieces of staged rows: the same for every group of 16.
template <typename T, int DP> struct LanePieces {
    uint32_t plain[DP / 32], turned[DP / 16];
    __device__ LanePieces() {
        const int lane = threadIdx.x & 63, quarter = lane / 16, within = lane % 16, row = quarter * 4 + within / 4;
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) plain[k] = within * TileLds<DP>::kRowBytes + TileLds<DP>::place(within, 4 * k + quarter) * 16;
#pragma unroll
        for (int e = 0; e < DP / 16; ++e)
            turned[e] = row * TileLds<DP>::kRowBytes + TileLds<DP>::place(row, 2 * e + within % 4 / 2) * 16 + within % 2 * 8;
    }
    // 16 staged rows times the columns, on top of s: lane holds column lane % 16, rows 4 (lane / 16) + 0..3.
    __device__ __forceinline__ typename Matrix<T>::f4 rows_times_columns(const unsigned char *rows, const typename Matrix<T>::x8 (&column)[DP / 32],
                                                                         typename Matrix<T>::f4 s) const {
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) s = Matrix<T>::multiply(*(const typename Matrix<T>::x8 *)(rows + plain[k]), column[k], s);
        return s;
    }
    // acc^T += rows^T w for 32 rows: w holds, for each lane's column, its weights of 4 rows of either half.
    __device__ __forceinline__ void add_weighted_rows(const unsigned char *rows, typename Matrix<T>::x8 w, typename Matrix<T>::f4 (&acc)[DP / 16]) const {
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)rows;
#pragma unroll
        for (int e = 0; e < DP / 16; e += 2) {
            const Turned x = read_transposed<16 * TileLds<DP>::kRowBytes>(base + turned[e], base + turned[e + 1]);
            acc[e] = Matrix<T>::multiply(__builtin_bit_cast(typename Matrix<T>::x8, x.first), w, acc[e]);
            acc[e + 1] = Matrix<T>::multiply(__builtin_bit_cast(typename Matrix<T>::x8, x.second), w, acc[e + 1]);
        }
    }
};

template <typename T>
__device__ __forceinline__ typename Matrix<T>::x8 as_weights(const typename Matrix<T>::f4 &a, const typename Matrix<T>::f4 &b) {
    // weights are rounded to the tensors' type, as the matrix units take them: at most half a unit in their last place each,
    // of weights whose sum, for the output's denominator, is kept in 32 bits
    typename Matrix<T>::x8 w;
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = (T)a[r], w[4 + r] = (T)b[r];
    return w;
}

// A column's result: lane holds elements 16 e + 4 (lane / 16) + 0..3 of column lane % 16.  Whether all are finite.
template <typename T, int DP>
__device__ __forceinline__ bool store_column(const Heads &h, int64_t rank, int head, int head_dim, const typename Matrix<T>::f4 (&acc)[DP / 16],
                                             float factor) {
    const int at = (threadIdx.x & 63) / 16 * 4;
    T *row = (T *)h.data + rank * h.rank_stride + head * h.head_stride;
    float worst = 0.f;
#pragma unroll
    for (int e = 0; e < DP / 16; ++e) {
        typename Matrix<T>::x4 y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = acc[e][r] * factor;
            worst = fmaf(0.f, x, worst);                            // NaN once an element is not finite
            y[r] = (T)x;
        }
        if (rank >= 0 && 16 * e + at < head_dim) *(typename Matrix<T>::x4 *)(row + 16 * e + at) = y;
    }
    return worst == 0.f;
}

// A column is made again row by row where it is not finite: an infinity or NaN in a row that is a neighbour of another column
// of the wavefront, and has weight 0 here, makes 0 * inf in the matrix product.
template <typename F> __device__ __forceinline__ void redo_columns(bool bad, F &&redo) {
    uint64_t columns = __ballot(bad);
    columns = (columns | columns >> 16 | columns >> 32 | columns >> 48) & 0xFFFF;
    while (columns) {
        const int column = __builtin_ctzll(columns);
        columns &= columns - 1;
        redo(column);
    }
}

// Measured: 256 x 256 ranks, 169 neighbours, 8 heads of 64: 120 us of 41 for the bytes once (the row kernel 2.7 ms);
// 32 x 32 x 32, 27 neighbours, 8 query and 2 key heads of 128: 52 us of 26 (533).  What is left is waiting: finding the tile's
// rows and storing the result take 40 us of the 120, in which no product can run.
template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256, DP > 64 ? 3 : SEGMENTS ? 4 : 5) void attention_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    typedef TileLds<DP> Lds;
    constexpr int G = Lds::kGroups;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t coords[kTileWaves][ISO_MAX_DIMS];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t);
    if (!work.any) return;
    Lds lds(lds_bytes, t.chunks);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group + work.part * t.heads, head = first_head + column % t.heads;
    const int64_t rank = rank_at<true>(t, work.tile, t.column_at + column / t.heads * t.words);
    const int32_t own = SEGMENTS ? column_segment(a, rank) : 0;
    typename Matrix<T>::x8 q[DP / 32];
    load_column<T, DP>(a.q, rank, head, a.head_dim, q);
    tile_rows<DP, SEGMENTS>(t, work.tile, lds);
    tile_biases<T>(t, first_head, t.heads, lds.bias);
    const LanePieces<T, DP> pieces;
    const RowLoads<DP, SEGMENTS> loads(t, a.k, a.v, work.key_head);
    // Scores times log2 e and less the column's base, so that the weights are powers of two.  The base comes into the
    // products' start value (the cap's constant); it is raised, and what was added up before scaled, only when a score exceeds
    // it by more than 8: weights of up to 256 lose nothing, and most chunks need no maximum over the lanes of a column.
    // Scores made on top of a base far from theirs lose bits to it, all of them after a first chunk of neighbours that a bias
    // of -1e9 masks.  So the first base lies at most kBelow under the head's highest bias: 2^-24 of that is lost.
    constexpr float kBelow = 128.f, kLowestBase = -1e16f;           // the latter keeps the start value finite
    const float scale = a.scale * kLog2e, per_scale = 1.f / scale, cap = a.cap * kLog2e, to_cap = a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : 0.f;
    __syncthreads();

    f4 acc[DP / 16] = {}, from = {0.f, 0.f, 0.f, 0.f};              // from: - base / scale
    float base = 0.f, limit = -INFINITY, l = 0.f;                   // l: of this lane's rows; limit: 8 once the column has a base
    float cap_less_base = cap;
    Pairs<DP> next;
    next.prefetch(t, 0);
    loads.start(lds, 0, 0);
    for (int chunk = 0; chunk < t.chunks; ++chunk) {
        wait_for_rows();
        const Pairs<DP> pairs(lds, next, chunk, chunk % 2);
        if (chunk + 1 < t.chunks) {
            next.prefetch(t, chunk + 1);
            loads.start(lds, chunk + 1, 1 - chunk % 2);
        }
        const unsigned char *rows = lds.chunk + chunk % 2 * Lds::kStage;
        const uint32_t active = pairs.active;
        if (!active) continue;
        f4 x[G];
        float top = -INFINITY;
        // 32 rows at a time, so that the reads of one product are under way while the other waits
#pragma unroll
        for (int pair = 0; pair < G / 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
            f4 dot[2], bias[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
#pragma unroll
                for (int r = 0; r < 4; ++r) bias[half][r] = pairs.bias((const unsigned char *)lds.bias, g, r);
                dot[half] = pieces.rows_times_columns(rows + g * 16 * Lds::kRowBytes, q, from);
            }
            if (a.cap > 0.f) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float e = __builtin_amdgcn_exp2f(dot[half][r] * to_cap);
                        x[2 * pair + half][r] = fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + e), cap_less_base) + bias[half][r];
                    }
            } else {
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[2 * pair + half][r] = fmaf(dot[half][r], scale, bias[half][r]);
            }
#pragma unroll
            for (int g = 2 * pair; g < 2 * pair + 2; ++g) {
                if (SEGMENTS) {
                    const i4 seg = *(const i4 *)(lds.segment + chunk * Lds::kRows + g * 16 + lane / 16 * 4);
                    x[g][0] = seg.x == own ? x[g][0] : -INFINITY;
                    x[g][1] = seg.y == own ? x[g][1] : -INFINITY;
                    x[g][2] = seg.z == own ? x[g][2] : -INFINITY;
                    x[g][3] = seg.w == own ? x[g][3] : -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, x[g][r]);
            }
        }
        if (__any(top > limit)) {
            top = column_max(top);
            const bool based = limit > 0.f;
            float raise = based ? fmaxf(top, 0.f) : finite_floor(top);
            if (__any(raise < -kBelow)) {                           // first bases only
                const float *biases = lds.bias + column % t.heads * (a.torus.s + 1);
                float highest = -INFINITY;
#pragma nounroll
                for (int i = lane / 16; i < a.torus.s; i += 4) highest = fmaxf(highest, biases[i]);
                highest = column_max(highest);
                if (raise < -kBelow) raise = fmaxf(raise, fmaxf(highest - kBelow, kLowestBase));
            }
            const float keep = based ? __builtin_amdgcn_exp2f(-raise) : 1.f;
            if (top > -INFINITY) limit = 8.f;
            base += raise;
            from = a.cap > 0.f ? from : f4{1.f, 1.f, 1.f, 1.f} * (-base * per_scale);
            cap_less_base = cap - base;
            l *= keep;
#pragma unroll
            for (int e = 0; e < DP / 16; ++e) acc[e] *= keep;
#pragma unroll
            for (int g = 0; g < G; ++g) x[g] -= raise;
        }
#pragma unroll
        for (int pair = 0; pair < G / 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
#pragma unroll
            for (int g = 2 * pair; g < 2 * pair + 2; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[g][r] = __builtin_amdgcn_exp2f(x[g][r]);
                    l += x[g][r];
                }
            pieces.add_weighted_rows(rows + Lds::kTensor + pair * 32 * Lds::kRowBytes, as_weights<T>(x[2 * pair], x[2 * pair + 1]), acc);
        }
    }
    l = column_sum(l);
    bool fine = store_column<T, DP>(a.out, rank, head, a.head_dim, acc, l == 0.f ? 0.f : 1.f / l);
    // again: NaN or infinities among the scores; biases near the type's highest value, whose products with log2 e and 1 / scale
    // leave the range; no score as high as the base, by whose highest biases the column has no neighbour, or whose biases are
    // all the type's lowest value (the highest weight of any other column with a neighbour is 1 or more)
    const bool again = !(l < INFINITY) || !(fabsf(base) < 1e30f) || (limit > 0.f && l < 0.5f);
    if (a.lse && rank >= 0 && lane < 16 && !again)
        a.lse[rank * a.q_heads + head] = l == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * kLn2;
    redo_columns(rank >= 0 && !(fine && !again), [&](int c) {
        const uint32_t r = (uint32_t)__shfl((int)rank, c);
        const int h = __shfl(head, c);
        const bool lse = __shfl((int)again, c);
        store_coordinates(a.torus, r, lane, coords[wave]);
        __builtin_amdgcn_wave_barrier();
        RowState<8> st;
        attend_row<T, true>(a, r, r, h, 0, 1, coords[wave], st);
        write_row<T, true>(a, r, h, st, lse);                      // lse stays where it does not depend on what was wrong
        __builtin_amdgcn_wave_barrier();
    });
}

// ---- backward ------------------------------------------------------------------------
//
// Weights are made again from lse.  grad_q takes the forward pass's tiles: S and dP = V grad_out^T from the staged keys and
// values, grad_q^T += K^T da.  grad_k and grad_v take tiles of keys against the ranks that read them, with queries and
// grad_out staged: S and dP with the roles changed, grad_k^T += Q^T da, grad_v^T += grad_out^T P, head by head of the group.
// Both gather: a tile's results are written once, by one workgroup, in one order.

// P, dx and da of a pair, the bias times log2 e: -inf, and P 0, for pairs that are no neighbours.  Without a cap `dot` started
// at -lse / scale, with one `lse` (times log2 e) is taken off here; dp started at -delta.
struct GradientFactors {
    float scale, cap, to_cap;
    __device__ explicit GradientFactors(const AttentionArgs &a)
        : scale(a.scale * kLog2e), cap(a.cap * kLog2e), to_cap(a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : 0.f) {}
    // what dot starts at for an lse (natural, finite), and what operator() is given for it
    __device__ __forceinline__ float start(const AttentionArgs &a, float lse) const { return a.cap > 0.f ? 0.f : -lse / a.scale; }
    template <bool SEGMENTS> __device__ __forceinline__ PairGradient operator()(float dot, float bias, float lse, float dp, bool counts) const {
        PairGradient g;
        if (cap > 0.f) {
            const float y = fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(dot * to_cap)), 1.f);      // tanh
            g.p = __builtin_amdgcn_exp2f(fmaf(cap, y, bias) - lse);
            g.dx = g.p * dp;
            g.da = g.dx * fmaf(-y, y, 1.f);
        } else {
            g.p = __builtin_amdgcn_exp2f(fmaf(dot, scale, bias));
            g.dx = g.p * dp;
            g.da = g.dx;
        }
        if (SEGMENTS) {                    // what a pair that does not count holds must not reach its slot of the bias's gradient
            g.p = counts ? g.p : 0.f;
            g.dx = counts ? g.dx : 0.f;
            g.da = counts ? g.da : 0.f;
        }
        return g;
    }
};

// A lane's part of the bias's gradient: the places of up to 16 pairs of one slot among a wavefront's dx of 32 rows, in which
// every lane has written four rows of its column, 16 bytes at once.
constexpr int kDxFloats = 516;
struct SlotRound {
    uint32_t slot;
    u4 first, second;
    __device__ __forceinline__ void load(const TileArgs &t, int pair, int round, int wave, int lane) {
        const uint32_t *at = t.slots + (((int64_t)pair * kTileWaves + wave) * t.slot_rounds + round) * (64 + 256 * t.slot_words);
        slot = at[lane];
        first = *(const u4 *)(at + 64 + lane * 4);
        if (t.slot_words > 1) second = *(const u4 *)(at + 64 + 256 + lane * 4);
    }
    static __device__ __forceinline__ float eight(const float *dx, const u4 &w) {
        const float a = dx[w.x & 0xFFFF] + dx[w.x >> 16], b = dx[w.y & 0xFFFF] + dx[w.y >> 16];
        const float c = dx[w.z & 0xFFFF] + dx[w.z >> 16], d = dx[w.w & 0xFFFF] + dx[w.w >> 16];
        return (a + b) + (c + d);
    }
    __device__ __forceinline__ float sum(const float *dx, int words) const {
        float x = eight(dx, first);
        if (words > 1) x += eight(dx, second);
        return x;
    }
};

// Two products for the scores and their gradients, one for grad_q, and the bias's gradient summed by slots, as a score's dx has
// to be added to the others of its neighbour and no matrix product does that.  256 x 256 ranks, 49 neighbours, 8 heads of 64:
// 213 us, vector units busy for 46 % of them; 32 x 32 x 32, 27 neighbours, 8 and 2 heads of 128: 105 us.
template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256, 3) void attention_grad_q_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    typedef TileLds<DP> Lds;
    constexpr int G = Lds::kGroups;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t coords[kTileWaves][ISO_MAX_DIMS];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t);
    if (!work.any) return;
    Lds lds(lds_bytes, t.chunks);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group + work.part * t.heads, head = first_head + column % t.heads;
    const int s = a.torus.s, slots = t.heads * s;
    // behind the biases: dx of 32 rows and the wavefront's columns, a zero, and the sums of its slots over the tile's rows
    float *behind = lds.bias + (t.heads * (s + 1) + 3) / 4 * 4, *dx_at = behind + wave * kDxFloats;
    float *sums = behind + kTileWaves * kDxFloats + wave * (slots + 1);
    if (t.slots) {
        for (int i = lane; i <= slots; i += 64) sums[i] = 0.f;
        if (lane == 0) dx_at[512] = 0.f;
    }
    const int64_t rank = rank_at<true>(t, work.tile, t.column_at + column / t.heads * t.words);
    const int32_t own = SEGMENTS ? column_segment(a, rank) : 0;
    typename Matrix<T>::x8 q[DP / 32], g_out[DP / 32];
    load_column<T, DP>(a.q, rank, head, a.head_dim, q);
    load_column<T, DP>(a.grad_out, rank, head, a.head_dim, g_out);
    float delta = 0.f, lse = rank >= 0 ? a.lse[rank * a.q_heads + head] : 0.f;
    {
        typename Matrix<T>::x8 out[DP / 32];
        load_column<T, DP>(a.out, rank, head, a.head_dim, out);
        tile_rows<DP, SEGMENTS>(t, work.tile, lds);                 // while these are on their way
        tile_biases<T>(t, first_head, t.heads, lds.bias);
#pragma unroll
        for (int k = 0; k < DP / 32; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)g_out[k][e], (float)out[k][e], delta);
        delta = column_sum(delta);
    }
    lse = finite_floor(lse);
    if (rank >= 0 && lane < 16) {
        // what the other pass starts its products at; a large lse is a NaN there, and whoever reads the row is made again
        const int64_t at = rank * a.q_heads + head;
        const GradientFactors f(a);
        a.delta[at] = delta;
        a.starts[at] = fabsf(lse) > kLargeLse ? NAN : a.cap > 0.f ? lse * kLog2e : f.start(a, lse);
        a.starts[(int64_t)a.n * a.q_heads + at] = -delta;
    }
    const LanePieces<T, DP> pieces;
    const RowLoads<DP, SEGMENTS> loads(t, a.k, a.v, work.key_head);
    const GradientFactors factors(a);
    // A column with a large lse is made again below, its part of the bias's gradient with it.
    const bool large = fabsf(lse) > kLargeLse;
    const f4 from = f4{1.f, 1.f, 1.f, 1.f} * (large ? NAN : factors.start(a, lse)), from_dp = f4{-1.f, -1.f, -1.f, -1.f} * delta;
    const float lse2 = large ? NAN : lse * kLog2e;
    __syncthreads();

    f4 acc[DP / 16] = {};
    Pairs<DP> next;
    next.prefetch(t, 0);
    loads.start(lds, 0, 0);
    for (int chunk = 0; chunk < t.chunks; ++chunk) {
        wait_for_rows();
        const Pairs<DP> pairs(lds, next, chunk, chunk % 2);
        SlotRound round;
        if (t.slots) round.load(t, chunk * (G / 2), 0, wave, lane);
        if (chunk + 1 < t.chunks) {
            next.prefetch(t, chunk + 1);
            loads.start(lds, chunk + 1, 1 - chunk % 2);
        }
        const unsigned char *rows = lds.chunk + chunk % 2 * Lds::kStage;
        const uint32_t active = pairs.active;
#pragma unroll
        for (int pair = 0; pair < G / 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
            f4 da[2], dot[2], dp[2], bias[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
#pragma unroll
                for (int r = 0; r < 4; ++r) bias[half][r] = pairs.bias((const unsigned char *)lds.bias, g, r);
                dot[half] = pieces.rows_times_columns(rows + g * 16 * Lds::kRowBytes, q, from);
                dp[half] = pieces.rows_times_columns(rows + Lds::kTensor + g * 16 * Lds::kRowBytes, g_out, from_dp);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
                const i4 seg = SEGMENTS ? *(const i4 *)(lds.segment + chunk * Lds::kRows + g * 16 + lane / 16 * 4) : i4{};
                f4 dx;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const PairGradient pg = factors.template operator()<SEGMENTS>(
                        dot[half][r], bias[half][r], lse2, dp[half][r], (r == 0 ? seg.x : r == 1 ? seg.y : r == 2 ? seg.z : seg.w) == own);
                    dx[r] = pg.dx;
                    da[half][r] = pg.da;
                }
                if (t.slots) *(f4 *)(dx_at + (half * 64 + lane) * 4) = rank >= 0 && !large ? dx : f4{0.f, 0.f, 0.f, 0.f};
            }
            pieces.add_weighted_rows(rows + pair * 32 * Lds::kRowBytes, as_weights<T>(da[0], da[1]), acc);
            if (t.slots)                                            // every lane adds up the pairs of one slot in 32 rows
                for (int n = 0; n < t.slot_rounds; ++n) {
                    if (n || pair) round.load(t, chunk * (G / 2) + pair, n, wave, lane);
                    sums[round.slot] += round.sum(dx_at, t.slot_words);
                }
        }
    }
    const bool fine = store_column<T, DP>(a.grad_q, rank, head, a.head_dim, acc, a.scale);
    redo_columns(rank >= 0 && !fine, [&](int c) {
        const uint32_t r = (uint32_t)__shfl((int)rank, c);
        const int h = __shfl(head, c);
        const float row_delta = __shfl(delta, c);
        store_coordinates(a.torus, r, lane, coords[wave]);
        __builtin_amdgcn_wave_barrier();
        const bool bias_too = t.slots && __shfl((int)large, c);
        grad_q_row<T, true>(a, r, h, row_delta, coords[wave], bias_too ? sums + (h - first_head) * s : nullptr);
        __builtin_amdgcn_wave_barrier();
    });
    if (t.slots) {
        __syncthreads();
        const float *all = behind + kTileWaves * kDxFloats;
        float *out = a.partials + (uint64_t)work.tile * a.q_heads * s + (int64_t)first_head * s;
        for (int i = threadIdx.x; i < slots; i += 256)
            out[i] = all[i] + all[slots + 1 + i] + all[2 * (slots + 1) + i] + all[3 * (slots + 1) + i];
    }
}

// Four products, with accumulators for two results: 200 registers at 128 elements, so that two workgroups share a CU, and the
// wavefronts wait for 56 % of the time.  179 us and 130 us in the places of the above.
template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256, 2) void attention_grad_kv_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    typedef TileLds<DP> Lds;
    constexpr int G = Lds::kGroups;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t coords[kTileWaves][ISO_MAX_DIMS];
    __shared__ __align__(16) float row_starts[2][2 * Lds::kRows];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t);
    if (!work.any) return;
    Lds lds(lds_bytes, t.chunks);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group, s = a.torus.s;
    const int64_t rank = rank_at<true>(t, work.tile, t.column_at + column * t.words);
    const int32_t own = SEGMENTS ? column_segment(a, rank) : 0;
    typename Matrix<T>::x8 k[DP / 32], v[DP / 32];
    load_column<T, DP>(a.k, rank, work.key_head, a.head_dim, k);
    load_column<T, DP>(a.v, rank, work.key_head, a.head_dim, v);
    tile_rows<DP, SEGMENTS>(t, work.tile, lds);
    tile_biases<T>(t, first_head, a.bias ? a.group : 1, lds.bias);
    const LanePieces<T, DP> pieces;
    const GradientFactors factors(a);
    __syncthreads();

    f4 dk[DP / 16] = {}, dv[DP / 16] = {};
    // the rows of all chunks for the first head of the group, then for the next, and what products with them start at
    Pairs<DP> next;
    const auto start = [&](int h, int chunk, int stage) {
        next.prefetch(t, chunk);
        const RowLoads<DP, SEGMENTS> loads(t, a.q, a.grad_out, first_head + h);
        loads.start(lds, chunk, stage);
        const float *from = a.starts + first_head + h;
#pragma unroll
        for (int i = 0; i < Lds::kRows / 32; ++i) {                 // every wavefront the same: -lse / scale, then -delta
            const int n = lane + 64 * i;
            const int64_t r = max(lds.rank[chunk * Lds::kRows + n % Lds::kRows], 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + (n / Lds::kRows * (int64_t)a.n + r) * a.q_heads),
                                             (__attribute__((address_space(3))) void *)(row_starts[stage] + 64 * i), 4, 0, 0);
        }
    };
    start(0, 0, 0);
    int chunk = 0, h = 0;
    for (int stage = 0; h < a.group; stage = 1 - stage) {
        wait_for_rows();
        const Pairs<DP> pairs(lds, next, chunk, stage);
        const int now = chunk, now_h = h;
        if (++chunk == t.chunks) chunk = 0, ++h;
        if (h < a.group) start(h, chunk, 1 - stage);
        const unsigned char *rows = lds.chunk + stage * Lds::kStage;
        const unsigned char *biases = (const unsigned char *)(lds.bias + (a.bias ? now_h * (s + 1) : 0));
        const uint32_t active = pairs.active;
#pragma unroll
        for (int pair = 0; pair < G / 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
            f4 p[2], da[2], dot[2], dp[2], bias[2], lse[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
#pragma unroll
                for (int r = 0; r < 4; ++r) bias[half][r] = pairs.bias(biases, g, r);
                lse[half] = *(const f4 *)(row_starts[stage] + g * 16 + lane / 16 * 4);
                dot[half] = pieces.rows_times_columns(rows + g * 16 * Lds::kRowBytes, k, a.cap > 0.f ? f4{0.f, 0.f, 0.f, 0.f} : lse[half]);
                dp[half] = pieces.rows_times_columns(rows + Lds::kTensor + g * 16 * Lds::kRowBytes, v,
                                                     *(const f4 *)(row_starts[stage] + Lds::kRows + g * 16 + lane / 16 * 4));
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
                const i4 seg = SEGMENTS ? *(const i4 *)(lds.segment + now * Lds::kRows + g * 16 + lane / 16 * 4) : i4{};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const PairGradient pg = factors.template operator()<SEGMENTS>(
                        dot[half][r], bias[half][r], lse[half][r], dp[half][r], (r == 0 ? seg.x : r == 1 ? seg.y : r == 2 ? seg.z : seg.w) == own);
                    p[half][r] = pg.p;
                    da[half][r] = pg.da;
                }
            }
            pieces.add_weighted_rows(rows + Lds::kTensor + pair * 32 * Lds::kRowBytes, as_weights<T>(p[0], p[1]), dv);
            pieces.add_weighted_rows(rows + pair * 32 * Lds::kRowBytes, as_weights<T>(da[0], da[1]), dk);
        }
    }
    const bool fine_v = store_column<T, DP>(a.grad_v, rank, work.key_head, a.head_dim, dv, 1.f);
    const bool fine_k = store_column<T, DP>(a.grad_k, rank, work.key_head, a.head_dim, dk, a.scale);
    redo_columns(rank >= 0 && !(fine_v && fine_k), [&](int c) {
        const uint32_t r = (uint32_t)__shfl((int)rank, c);
        store_coordinates(a.torus, r, lane, coords[wave]);
        __builtin_amdgcn_wave_barrier();
        grad_kv_row<T, true>(a, r, work.key_head, coords[wave]);
        __builtin_amdgcn_wave_barrier();
    });
}

}  // namespace iso
