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
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_tiles.hpp"

namespace iso {

struct TileArgs {
    AttentionArgs a;
    int32_t tile[ISO_MAX_DIMS], tiles[ISO_MAX_DIMS];
    uint32_t n_tiles, per_xcd;             // workgroups of one XCD
    int32_t heads, parts;                  // columns of one rank; sets of `heads` q heads that share a key head
    int32_t chunks;
    const int32_t *column_at, *row_at;
    const uint32_t *active;
    const uint16_t *index;
    const uint32_t *slots_of;              // the bias's gradient, or null: see TilePlan
    const TilePlan::Slot *slots;
    const uint16_t *pairs;
};

template <typename T> struct Matrix;
template <> struct Matrix<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    typedef float f4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f4 multiply(x8 a, x8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ x4 read_transposed(const __bf16 *at) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) x4 *)at);
    }
};
template <> struct Matrix<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    typedef float f4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f4 multiply(x8 a, x8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ x4 read_transposed(const _Float16 *at) {
        typedef __fp16 h4 __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4 *)at));
    }
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

// LDS of a tile kernel: two staged tensors of kChunkRows rows, padded by 16 bytes so that the 16 rows of a product start in
// 16 different groups of banks, then per row of the tile its rank and segment, then the biases.
template <typename T, int DP> struct TileLds {
    static constexpr int kStride = DP + 8;
    T *first, *second;
    int32_t *rank, *segment;
    float *bias;
    static __host__ __device__ size_t bytes(int chunks, size_t biases) {
        return 2 * sizeof(T) * kChunkRows * kStride + (size_t)chunks * kChunkRows * 8 + biases * 4;
    }
    __device__ TileLds(unsigned char *at, int chunks) {
        first = (T *)at;
        second = first + kChunkRows * kStride;
        rank = (int32_t *)(second + kChunkRows * kStride);
        segment = rank + chunks * kChunkRows;
        bias = (float *)(segment + chunks * kChunkRows);
    }
};

constexpr int32_t kNoToken = INT32_MIN;    // segment of a row that is outside the mesh or holds no token
constexpr int32_t kNoColumn = INT32_MIN + 1;

// Rank at a position relative to the tile's first rank, -1 outside the mesh (and for positions that only columns outside the
// torus, of a ragged tile, refer to).
__device__ __forceinline__ int32_t rank_at(const TileArgs &t, const int32_t *origin, const int32_t *at, bool column) {
    int32_t rank = 0;
    bool there = true;
    for (int j = 0; j < t.a.torus.d; ++j) {
        const int32_t n = t.a.torus.dims[j];
        int32_t x = origin[j] + at[j];
        if (!column && !(t.a.torus.open >> j & 1)) {
            x += x < 0 ? n : 0;
            x -= x >= n ? n : 0;
        }
        there = there && (uint32_t)x < (uint32_t)n;
        rank += x * t.a.torus.inner[j];
    }
    return there ? rank : -1;
}

// What a workgroup works on: workgroups are handed to the 8 XCDs in turn, and each XCD takes a run of consecutive tiles of
// one head, whose rows its L2 then holds for all tiles that share them.
struct TileWork {
    uint32_t tile;
    int key_head, part;
    bool any;
};
__device__ __forceinline__ TileWork tile_work(const TileArgs &t, int key_heads) {
    TileWork w;
    const uint32_t item = (blockIdx.x & 7) * t.per_xcd + (blockIdx.x >> 3), pairs = item / t.parts;
    w.part = item % t.parts;
    w.tile = pairs % t.n_tiles;
    w.key_head = pairs / t.n_tiles;
    w.any = w.key_head < key_heads;
    return w;
}

template <typename T, int DP>
__device__ __forceinline__ void tile_rows(const TileArgs &t, uint32_t tile, int32_t *origin, TileLds<T, DP> &lds) {
    const int d = t.a.torus.d;
    if ((int)threadIdx.x < d) {
        uint32_t rest = tile;
        for (int j = d - 1; j > (int)threadIdx.x; --j) rest /= (uint32_t)t.tiles[j];
        origin[threadIdx.x] = (int32_t)(rest % (uint32_t)t.tiles[threadIdx.x]) * t.tile[threadIdx.x];
    }
    __syncthreads();
    for (int u = threadIdx.x; u < t.chunks * kChunkRows; u += 256) {
        const int32_t rank = rank_at(t, origin, t.row_at + (int64_t)u * d, false);
        int32_t segment = rank < 0 ? kNoToken : t.a.segments ? t.a.segments[rank] : 0;
        if (segment < 0) segment = kNoToken;
        lds.rank[u] = segment < 0 ? -1 : rank;                      // rows without a token are staged as zeros
        lds.segment[u] = segment;
    }
}

// One chunk of rows of two tensors: into registers, 16 bytes a lane, and from there into LDS.
template <typename T, int DP> struct Staged {
    static constexpr int kUnits = DP / 8, kPerThread = kChunkRows * kUnits / 256;
    typename Matrix<T>::x8 first[kPerThread], second[kPerThread];

    __device__ __forceinline__ void load(const T *a, int64_t a_stride, const T *b, int64_t b_stride, const int32_t *rank, int head_dim) {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int unit = threadIdx.x + 256 * i, row = unit / kUnits, at = unit % kUnits * 8;
            const int32_t r = rank[row];
            first[i] = {};
            second[i] = {};
            if (r >= 0 && at < head_dim) {
                first[i] = *(const typename Matrix<T>::x8 *)(a + r * a_stride + at);
                second[i] = *(const typename Matrix<T>::x8 *)(b + r * b_stride + at);
            }
        }
    }
    __device__ __forceinline__ void store(TileLds<T, DP> &lds) const {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int unit = threadIdx.x + 256 * i, row = unit / kUnits, at = unit % kUnits * 8;
            *(typename Matrix<T>::x8 *)(lds.first + row * lds.kStride + at) = first[i];
            *(typename Matrix<T>::x8 *)(lds.second + row * lds.kStride + at) = second[i];
        }
    }
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

// 16 staged rows times the columns: lane holds column lane % 16, rows 4 (lane / 16) + 0..3.
template <typename T, int DP>
__device__ __forceinline__ typename Matrix<T>::f4 rows_times_columns(const T *rows, const typename Matrix<T>::x8 (&column)[DP / 32]) {
    const int lane = threadIdx.x & 63;
    const T *at = rows + lane % 16 * TileLds<T, DP>::kStride + lane / 16 * 8;
    typename Matrix<T>::f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < DP / 32; ++k) s = Matrix<T>::multiply(*(const typename Matrix<T>::x8 *)(at + 32 * k), column[k], s);
    return s;
}

// acc^T += rows^T w for 32 rows: w holds, for each lane's column, its weights of 4 rows of either half.
template <typename T, int DP>
__device__ __forceinline__ void add_weighted_rows(const T *rows, typename Matrix<T>::x8 w, typename Matrix<T>::f4 (&acc)[DP / 16]) {
    const int lane = threadIdx.x & 63, quarter = lane / 16, within = lane % 16;
    const T *at = rows + (quarter * 4 + within / 4) * TileLds<T, DP>::kStride + within % 4 * 4;
#pragma unroll
    for (int e = 0; e < DP / 16; ++e) {
        const typename Matrix<T>::x4 low = Matrix<T>::read_transposed(at + 16 * e);
        const typename Matrix<T>::x4 high = Matrix<T>::read_transposed(at + 16 * e + 16 * TileLds<T, DP>::kStride);
        acc[e] = Matrix<T>::multiply(__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7), w, acc[e]);
    }
}

template <typename T>
__device__ __forceinline__ typename Matrix<T>::x8 as_weights(const typename Matrix<T>::f4 &a, const typename Matrix<T>::f4 &b) {
    // weights are rounded to the tensors' type, as the matrix units take them: at most half a unit in their last place each,
    // of weights whose sum, for the output's denominator, is kept in 32 bits
    typename Matrix<T>::x8 w;
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = (T)a[r], w[4 + r] = (T)b[r];
    return w;
}

// A column's result: lane holds elements 16 e + 4 (lane / 16) + 0..3 of column lane % 16.
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

template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256) void attention_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t origin[ISO_MAX_DIMS], coords[kTileWaves][ISO_MAX_DIMS];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t, a.kv_heads);
    if (!work.any) return;
    TileLds<T, DP> lds(lds_bytes, t.chunks);
    tile_rows<T, DP>(t, work.tile, origin, lds);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group + work.part * t.heads, head = first_head + column % t.heads;
    const int s = a.torus.s;
    if (a.bias)
        for (int i = threadIdx.x; i < t.heads * s; i += 256)
            lds.bias[i / s * (s + 1) + i % s] = (float)((const T *)a.bias)[(int64_t)first_head * s + i];
    const int64_t rank = rank_at(t, origin, t.column_at + column / t.heads * a.torus.d, true);
    int32_t own = kNoColumn;
    if (rank >= 0) own = a.segments ? a.segments[rank] : 0;
    if (own < 0) own = kNoColumn;
    typename Matrix<T>::x8 q[DP / 32];
    load_column<T, DP>(a.q, rank, head, a.head_dim, q);
    __syncthreads();

    const T *k0 = (const T *)a.k.data + work.key_head * a.k.head_stride, *v0 = (const T *)a.v.data + work.key_head * a.v.head_stride;
    const float *bias = lds.bias + column % t.heads * (s + 1);
    f4 acc[DP / 16] = {};
    float m = -INFINITY, l = 0.f;                                   // l: of this lane's rows
    Staged<T, DP> next;
    next.load(k0, a.k.rank_stride, v0, a.v.rank_stride, lds.rank, a.head_dim);
    for (int chunk = 0; chunk < t.chunks; ++chunk) {
        __syncthreads();
        next.store(lds);
        __syncthreads();
        if (chunk + 1 < t.chunks)
            next.load(k0, a.k.rank_stride, v0, a.v.rank_stride, lds.rank + (chunk + 1) * kChunkRows, a.head_dim);
        const uint32_t active = __builtin_amdgcn_readfirstlane(t.active[chunk] >> (4 * wave) & 15);
        if (!active) continue;
        f4 x[4];
        float top = m;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            x[g] = f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (!(active >> g & 1)) continue;
            const uint2 who = *(const uint2 *)(t.index + (((int64_t)(chunk * 4 + g) * kTileWaves + wave) * 64 + lane) * 4);
            const f4 dot = rows_times_columns<T, DP>(lds.first + g * 16 * lds.kStride, q);
            const int4 seg = SEGMENTS ? *(const int4 *)(lds.segment + chunk * kChunkRows + g * 16 + lane / 16 * 4) : int4{};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = (r < 2 ? who.x : who.y) >> (r % 2 * 16) & 0xFFFF;
                float y = dot[r] * a.scale;
                if (a.cap > 0.f) y = capped(y, a.cap);
                if (a.bias) y += bias[i];
                const bool counts = i != s && (!SEGMENTS || (r == 0 ? seg.x : r == 1 ? seg.y : r == 2 ? seg.z : seg.w) == own);
                x[g][r] = counts ? y : -INFINITY;
                top = fmaxf(top, x[g][r]);
            }
        }
        top = column_max(top);
        const float base = finite_floor(top);
        if (__any(top > m)) {
            const float keep = exp_above(m, base);
            l *= keep;
#pragma unroll
            for (int e = 0; e < DP / 16; ++e) acc[e] *= keep;
            m = top;
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[g][r] = exp_above(x[g][r], base);
                l += x[g][r];
            }
#pragma unroll
        for (int pair = 0; pair < 2; ++pair)
            if (active >> (2 * pair) & 3)
                add_weighted_rows<T, DP>(lds.second + pair * 32 * lds.kStride, as_weights<T>(x[2 * pair], x[2 * pair + 1]), acc);
    }
    l = column_sum(l);
    const bool fine = store_column<T, DP>(a.out, rank, head, a.head_dim, acc, l == 0.f ? 0.f : 1.f / l);
    if (a.lse && rank >= 0 && lane < 16) a.lse[rank * a.q_heads + head] = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l) * kLn2;
    redo_columns(rank >= 0 && !fine, [&](int c) {
        const uint32_t r = (uint32_t)__shfl((int)rank, c);
        const int h = __shfl(head, c);
        store_coordinates(a.torus, r, lane, coords[wave]);
        __builtin_amdgcn_wave_barrier();
        RowState<8> st;
        attend_row<T, true>(a, r, r, h, 0, 1, coords[wave], st);
        write_row<T, true, false>(a, r, h, st);       // lse does not depend on the values
        __builtin_amdgcn_wave_barrier();
    });
}

// ---- backward ------------------------------------------------------------------------
//
// Weights are made again from lse.  grad_q takes the forward pass's tiles: S and dP = V grad_out^T from the staged keys and
// values, grad_q^T += K^T da.  grad_k and grad_v take tiles of keys against the ranks that read them, with queries and
// grad_out staged: S and dP with the roles changed, grad_k^T += Q^T da, grad_v^T += grad_out^T P, head by head of the group.
// Both gather: a tile's results are written once, by one workgroup, in one order.

template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256) void attention_grad_q_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t origin[ISO_MAX_DIMS], coords[kTileWaves][ISO_MAX_DIMS];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t, a.kv_heads);
    if (!work.any) return;
    TileLds<T, DP> lds(lds_bytes, t.chunks);
    tile_rows<T, DP>(t, work.tile, origin, lds);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group + work.part * t.heads, head = first_head + column % t.heads;
    const int s = a.torus.s, slots = t.heads * s;
    if (a.bias)
        for (int i = threadIdx.x; i < slots; i += 256)
            lds.bias[i / s * (s + 1) + i % s] = (float)((const T *)a.bias)[(int64_t)first_head * s + i];
    // behind the biases: dx of the wavefront's blocks of a chunk, and the sums of its slots over the chunks
    float *dx_at = lds.bias + (t.heads * (s + 1) + 3) / 4 * 4 + wave * 1024;
    float *sums = lds.bias + (t.heads * (s + 1) + 3) / 4 * 4 + kTileWaves * 1024 + wave * slots;
    if (t.slots_of)
        for (int i = lane; i < slots; i += 64) sums[i] = 0.f;
    const int64_t rank = rank_at(t, origin, t.column_at + column / t.heads * a.torus.d, true);
    int32_t own = kNoColumn;
    if (rank >= 0) own = a.segments ? a.segments[rank] : 0;
    if (own < 0) own = kNoColumn;
    typename Matrix<T>::x8 q[DP / 32], g_out[DP / 32];
    load_column<T, DP>(a.q, rank, head, a.head_dim, q);
    load_column<T, DP>(a.grad_out, rank, head, a.head_dim, g_out);
    float delta = 0.f;
    {
        typename Matrix<T>::x8 out[DP / 32];
        load_column<T, DP>(a.out, rank, head, a.head_dim, out);
#pragma unroll
        for (int k = 0; k < DP / 32; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)g_out[k][e], (float)out[k][e], delta);
        delta = column_sum(delta);
    }
    const float lse = rank >= 0 ? finite_floor(a.lse[rank * a.q_heads + head]) : 0.f;
    if (rank >= 0 && lane < 16) a.delta[rank * a.q_heads + head] = delta;
    __syncthreads();

    const T *k0 = (const T *)a.k.data + work.key_head * a.k.head_stride, *v0 = (const T *)a.v.data + work.key_head * a.v.head_stride;
    const float *bias = lds.bias + column % t.heads * (s + 1);
    f4 acc[DP / 16] = {};
    Staged<T, DP> next;
    next.load(k0, a.k.rank_stride, v0, a.v.rank_stride, lds.rank, a.head_dim);
    for (int chunk = 0; chunk < t.chunks; ++chunk) {
        __syncthreads();
        next.store(lds);
        __syncthreads();
        if (chunk + 1 < t.chunks)
            next.load(k0, a.k.rank_stride, v0, a.v.rank_stride, lds.rank + (chunk + 1) * kChunkRows, a.head_dim);
        const uint32_t active = __builtin_amdgcn_readfirstlane(t.active[chunk] >> (4 * wave) & 15);
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
            f4 da[2] = {};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
                if (!(active >> g & 1)) continue;
                const uint2 who = *(const uint2 *)(t.index + (((int64_t)(chunk * 4 + g) * kTileWaves + wave) * 64 + lane) * 4);
                const f4 dot = rows_times_columns<T, DP>(lds.first + g * 16 * lds.kStride, q);
                const f4 dp = rows_times_columns<T, DP>(lds.second + g * 16 * lds.kStride, g_out);
                const int4 seg = SEGMENTS ? *(const int4 *)(lds.segment + chunk * kChunkRows + g * 16 + lane / 16 * 4) : int4{};
                f4 dx;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = (r < 2 ? who.x : who.y) >> (r % 2 * 16) & 0xFFFF;
                    const bool counts = i != s && (!SEGMENTS || (r == 0 ? seg.x : r == 1 ? seg.y : r == 2 ? seg.z : seg.w) == own);
                    const PairGradient pg = pair_gradient(dot[r], a.bias ? bias[i] : 0.f, lse, dp[r], delta, a.scale, a.cap);
                    dx[r] = counts ? pg.dx : 0.f;
                    da[half][r] = counts ? pg.da : 0.f;
                }
                if (t.slots_of) *(f4 *)(dx_at + (g * 64 + lane) * 4) = rank >= 0 ? dx : f4{0.f, 0.f, 0.f, 0.f};
            }
            add_weighted_rows<T, DP>(lds.first + pair * 32 * lds.kStride, as_weights<T>(da[0], da[1]), acc);
        }
        if (t.slots_of) {
            // every lane adds up the pairs of one slot: blocks that hold none of its pairs are not read
            __builtin_amdgcn_wave_barrier();
            const uint32_t begin = t.slots_of[chunk * kTileWaves + wave], end = t.slots_of[chunk * kTileWaves + wave + 1];
            for (uint32_t j = begin + lane; j < end; j += 64) {
                const TilePlan::Slot slot = t.slots[j];
                float sum = 0.f;
                for (uint32_t n = 0; n < slot.count; ++n) sum += dx_at[t.pairs[slot.first + n]];
                sums[slot.slot] += sum;
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    const bool fine = store_column<T, DP>(a.grad_q, rank, head, a.head_dim, acc, a.scale);
    redo_columns(rank >= 0 && !fine, [&](int c) {
        const uint32_t r = (uint32_t)__shfl((int)rank, c);
        const int h = __shfl(head, c);
        const float row_delta = __shfl(delta, c);
        store_coordinates(a.torus, r, lane, coords[wave]);
        __builtin_amdgcn_wave_barrier();
        grad_q_row<T, true>(a, r, h, row_delta, coords[wave]);
        __builtin_amdgcn_wave_barrier();
    });
    if (t.slots_of) {
        __syncthreads();
        const float *all = lds.bias + (t.heads * (s + 1) + 3) / 4 * 4 + kTileWaves * 1024;
        float *out = a.partials + (uint64_t)work.tile * a.q_heads * s + (int64_t)first_head * s;
        for (int i = threadIdx.x; i < slots; i += 256) out[i] = all[i] + all[slots + i] + all[2 * slots + i] + all[3 * slots + i];
    }
}

template <typename T, int DP, bool SEGMENTS>
__global__ __launch_bounds__(256) void attention_grad_kv_tile_kernel(const TileArgs t) {
    typedef typename Matrix<T>::f4 f4;
    extern __shared__ __align__(16) unsigned char lds_bytes[];
    __shared__ int32_t origin[ISO_MAX_DIMS], coords[kTileWaves][ISO_MAX_DIMS];
    __shared__ __align__(16) float row_lse[kChunkRows], row_delta[kChunkRows];
    const AttentionArgs &a = t.a;
    const TileWork work = tile_work(t, a.kv_heads);
    if (!work.any) return;
    TileLds<T, DP> lds(lds_bytes, t.chunks);
    tile_rows<T, DP>(t, work.tile, origin, lds);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, column = 16 * wave + lane % 16;
    const int first_head = work.key_head * a.group, s = a.torus.s;
    if (a.bias)
        for (int i = threadIdx.x; i < a.group * s; i += 256)
            lds.bias[i / s * (s + 1) + i % s] = (float)((const T *)a.bias)[(int64_t)first_head * s + i];
    const int64_t rank = rank_at(t, origin, t.column_at + column * a.torus.d, true);
    int32_t own = kNoColumn;
    if (rank >= 0) own = a.segments ? a.segments[rank] : 0;
    if (own < 0) own = kNoColumn;
    typename Matrix<T>::x8 k[DP / 32], v[DP / 32];
    load_column<T, DP>(a.k, rank, work.key_head, a.head_dim, k);
    load_column<T, DP>(a.v, rank, work.key_head, a.head_dim, v);
    __syncthreads();

    f4 dk[DP / 16] = {}, dv[DP / 16] = {};
    Staged<T, DP> next;
    float next_lse = 0.f, next_delta = 0.f;
    const auto fetch = [&](int step) {
        const int h = first_head + step / t.chunks, chunk = step % t.chunks;
        next.load((const T *)a.q.data + h * a.q.head_stride, a.q.rank_stride, (const T *)a.grad_out.data + h * a.grad_out.head_stride,
                  a.grad_out.rank_stride, lds.rank + chunk * kChunkRows, a.head_dim);
        if (threadIdx.x < kChunkRows) {
            const int32_t r = lds.rank[chunk * kChunkRows + threadIdx.x];
            next_lse = r >= 0 ? finite_floor(a.lse[(int64_t)r * a.q_heads + h]) : 0.f;
            next_delta = r >= 0 ? a.delta[(int64_t)r * a.q_heads + h] : 0.f;
        }
    };
    const int steps = a.group * t.chunks;
    fetch(0);
    for (int step = 0; step < steps; ++step) {
        const int chunk = step % t.chunks;
        const float *bias = lds.bias + step / t.chunks * (s + 1);
        __syncthreads();
        next.store(lds);
        if (threadIdx.x < kChunkRows) row_lse[threadIdx.x] = next_lse, row_delta[threadIdx.x] = next_delta;
        __syncthreads();
        if (step + 1 < steps) fetch(step + 1);
        const uint32_t active = __builtin_amdgcn_readfirstlane(t.active[chunk] >> (4 * wave) & 15);
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            if (!(active >> (2 * pair) & 3)) continue;
            f4 p[2] = {}, da[2] = {};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int g = 2 * pair + half;
                if (!(active >> g & 1)) continue;
                const uint2 who = *(const uint2 *)(t.index + (((int64_t)(chunk * 4 + g) * kTileWaves + wave) * 64 + lane) * 4);
                const f4 dot = rows_times_columns<T, DP>(lds.first + g * 16 * lds.kStride, k);
                const f4 dp = rows_times_columns<T, DP>(lds.second + g * 16 * lds.kStride, v);
                const f4 lse = *(const f4 *)(row_lse + g * 16 + lane / 16 * 4), delta = *(const f4 *)(row_delta + g * 16 + lane / 16 * 4);
                const int4 seg = SEGMENTS ? *(const int4 *)(lds.segment + chunk * kChunkRows + g * 16 + lane / 16 * 4) : int4{};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = (r < 2 ? who.x : who.y) >> (r % 2 * 16) & 0xFFFF;
                    const bool counts = i != s && (!SEGMENTS || (r == 0 ? seg.x : r == 1 ? seg.y : r == 2 ? seg.z : seg.w) == own);
                    const PairGradient pg = pair_gradient(dot[r], a.bias ? bias[i] : 0.f, lse[r], dp[r], delta[r], a.scale, a.cap);
                    p[half][r] = counts ? pg.p : 0.f;
                    da[half][r] = counts ? pg.da : 0.f;
                }
            }
            add_weighted_rows<T, DP>(lds.second + pair * 32 * lds.kStride, as_weights<T>(p[0], p[1]), dv);
            add_weighted_rows<T, DP>(lds.first + pair * 32 * lds.kStride, as_weights<T>(da[0], da[1]), dk);
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
