// gfx950 kernels for attention over an isomorphic neighbourhood.
//
// Every rank R of the torus holds a query row per q head and a key and a value row per kv head.  Its keys are those of the
// ranks S_i = R (-) C^i, the sources of the allgather's blocks, read where they lie: no copy per neighbour exists.
//
//     a_i = scale q_R . k_i      t_i = cap tanh(a_i / cap)      x_i = t_i + bias[h][i]
//     lse = log sum_i exp x_i    out = sum_i exp(x_i - lse) v_i
//
// Neighbours without a source (mesh) or of another segment do not count; with none left out = 0 and lse = -inf.
//
// This file holds the row kernels: one wavefront (or several, over parts of the neighbours) for one row, in vector
// arithmetic, for every type, head size, stride and alignment.  Every row reads its neighbours' keys and values from the
// caches (32 x 32 x 32 ranks, 27 neighbours, 8 query and 2 key heads of 128, bfloat16: 27 times the tensors' bytes, 533 us
// forward and 2.2 ms backward), so vector arithmetic and the caches bound them where rows are many, and the chain of loads
// of one row where they are few: one row of 16 heads, 64 neighbours, 8 us with the launch; 37 rows, 169 neighbours 10.6 us.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "iso.h"

namespace iso {

constexpr int kAttentionMaxHeadDim = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// The torus for kernels that go from a rank to its neighbours.
struct NeighbourTorus {
    int32_t d, s;
    uint32_t p;
    uint32_t open;                         // bit j: dimension j does not wrap
    int32_t dims[ISO_MAX_DIMS];
    int32_t inner[ISO_MAX_DIMS];           // rank stride of dimension j
    const int32_t *offsets;                // device [s][d]: residues where the dimension wraps, else in [-p_j, p_j]
};

struct Heads {                             // element strides
    const void *data;
    int64_t rank_stride, head_stride;
};

struct AttentionArgs {
    NeighbourTorus torus;
    Heads q, k, v, out;                    // out: written by the forward pass, read by the backward pass
    Heads grad_out, grad_q, grad_k, grad_v;
    float *lse;                            // [n][q_heads]
    float *delta;                          // [p][q_heads]: grad_out . out of every row, for the gradients of k and v
    float *starts;                         // [2][p][q_heads]: -lse / scale (cap: lse log2 e) and -delta, or null: for the tile kernels
    float *norms;                          // [p][q_heads]: 1 / (sum of the weights), of rows with a large lse
    float *partials;                       // [parts][q_heads * s] of the bias's gradient
    const void *bias;                      // [q_heads][s] of the tensors' type, or null
    const int32_t *segments;               // [p] or null
    const int64_t *rows;                   // device [n] ranks, or null: row n is rank n
    uint32_t n;                            // rows
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t lanes_log2;                    // lanes that share one neighbour's row
    int32_t waves;                         // wavefronts that share one row (1: four rows in a workgroup)
    int32_t parts;                         // of the bias's gradient
    float scale, cap;
    uint32_t first_block;                  // workgroups of the launches before, where one launch cannot hold all
};

// ---- elements ---------------------------------------------------------------

template <typename T> struct ElementTraits;
template <> struct ElementTraits<float> { static constexpr int kPerLane = 4; };
template <> struct ElementTraits<__bf16> { static constexpr int kPerLane = 8; };
template <> struct ElementTraits<_Float16> { static constexpr int kPerLane = 8; };

// kPerLane elements of a row from element `at` on; zeros from `end` on.  WIDE: rows are 16-byte aligned and hold whole groups.
template <typename T, bool WIDE>
__device__ __forceinline__ void load_elements(const T *row, int at, int end, float (&x)[ElementTraits<T>::kPerLane]) {
    constexpr int E = ElementTraits<T>::kPerLane;
    if constexpr (WIDE) {
        typedef T vec_t __attribute__((ext_vector_type(E)));
        vec_t v = {};
        if (at < end) v = *(const vec_t *)(row + at);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = at + e < end ? (float)row[at + e] : 0.f;
    }
}

template <typename T, bool WIDE>
__device__ __forceinline__ void store_elements(T *row, int at, int end, const float (&x)[ElementTraits<T>::kPerLane]) {
    constexpr int E = ElementTraits<T>::kPerLane;
    if constexpr (WIDE) {
        typedef T vec_t __attribute__((ext_vector_type(E)));
        vec_t v;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (T)x[e];
        if (at < end) *(vec_t *)(row + at) = v;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at + e < end) row[at + e] = (T)x[e];
    }
}

// cap * tanh(a / cap).  For 16-bit tensors tanh y = 1 - 2 / (1 + e^2y), whose error is about 2^-22 of the cap whatever the
// score.  Above kPlainCap (2^-15 of a weight there)
// small scores go by tanh y / y as a series to y^8, whose rest is 2^-26, and the tile kernels, whose registers have no room
// for it, are not taken: 32 x 32 x 32 ranks, 27 neighbours, 8 and 2 heads of 128, 46 us at a cap of 128, 466 above.
constexpr float kPlainCap = 128.f, kSmallTanh = 0.25f;
template <typename T> __device__ __forceinline__ float capped(float a, float cap) {
    if constexpr (sizeof(T) == 4) return cap * tanhf(a / cap);
    if (__builtin_expect(cap > kPlainCap, 0)) {
        const float y = a * (1.f / cap), y2 = y * y;
        const float ratio = fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
        if (fabsf(y) < kSmallTanh) return a * ratio;
    }
    const float e = __builtin_amdgcn_exp2f(a * (2.f * kLog2e / cap));
    return cap - 2.f * cap * __builtin_amdgcn_rcpf(1.f + e);
}

// exp(x - of): the difference first, so that scores near the type's lowest value stay finite; -inf gives 0.
__device__ __forceinline__ float exp_above(float x, float of) { return __builtin_amdgcn_exp2f((x - of) * kLog2e); }

// A maximum or lse to subtract: -inf (no neighbour counts, or every bias is -inf) becomes 0, and the weights exp(-inf) = 0.
__device__ __forceinline__ float finite_floor(float m) { return m == -INFINITY ? 0.f : m; }

// ---- neighbours --------------------------------------------------------------

// Coordinates of a rank, one per dimension, into LDS (read back below with one broadcast read per dimension).
__device__ __forceinline__ void store_coordinates(const NeighbourTorus &t, uint32_t rank, int lane, int32_t *coords) {
    if (lane < t.d) coords[lane] = (int32_t)(rank / (uint32_t)t.inner[lane] % (uint32_t)t.dims[lane]);
}

// Neighbour i of the rank with these coordinates: R (-) C^i, or R (+) C^i where TARGET.  -1: none.  Sizes go to 2^31 - 1, so
// what wraps takes one difference that stays inside 32 bits, and what does not is compared without a sign.
template <bool TARGET>
__device__ __forceinline__ int32_t neighbour_rank(const NeighbourTorus &t, const int32_t *coords, int i) {
    uint32_t rank = 0;
    bool there = true;
    const int32_t *c = t.offsets + (int64_t)i * t.d;
    for (int first = 0; first < t.d; first += 4) {                  // four offsets under way at a time
        int32_t step[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) step[q] = first + q < t.d ? c[first + q] : 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = first + q;
            if (j >= t.d) break;
            const uint32_t at = (uint32_t)coords[j], n = (uint32_t)t.dims[j], by = (uint32_t)step[q];
            uint32_t x;
            if (t.open >> j & 1) {
                x = TARGET ? at + by : at - by;
                there = there && x < n;
            } else {
                x = TARGET ? at - (n - by) : at - by;
                x += (int32_t)x < 0 ? n : 0;
            }
            rank += x * (uint32_t)t.inner[j];
        }
    }
    return there ? (int32_t)rank : -1;
}

__device__ __forceinline__ float sum_over_lanes(float x, int lanes_log2) {
    for (int l = 0; l < lanes_log2; ++l) x += __shfl_xor(x, 1 << l);
    return x;
}

// Sums over the lanes that share a row and over all neighbours' lanes: a whole wavefront.
__device__ __forceinline__ float sum_across_groups(float x, int lanes_log2) {
    for (int l = lanes_log2; l < 6; ++l) x += __shfl_xor(x, 1 << l);
    return x;
}

// ---- forward: one row -----------------------------------------------------------

// Softmax state of one lane's share: elements [at, at + E) of the weighted sum of values.
template <int E> struct RowState {
    float m = -INFINITY, l = 0.f;
    float acc[E] = {};

    __device__ void merge(float om, float ol, const float (&oacc)[E]) {
        const float top = fmaxf(m, om), base = finite_floor(top);
        const float a = exp_above(m, base), b = exp_above(om, base);
        l = l * a + ol * b;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * a + oacc[e] * b;
        m = top;
    }
};

// The neighbours first, first + step, ... of one (rank, q head); lanes of one wavefront, 64 >> lanes_log2 neighbours at a time.
// `first` and `step` count such sets of neighbours.  All lanes leave with the state of all sets that this call took.
template <typename T, bool WIDE>
__device__ __forceinline__ void attend_row(const AttentionArgs &a, uint32_t row, uint32_t rank, int h, int first, int step,
                                           const int32_t *coords, RowState<ElementTraits<T>::kPerLane> &st) {
    constexpr int E = ElementTraits<T>::kPerLane;
    const NeighbourTorus &t = a.torus;
    const int lane = threadIdx.x & 63, L = a.lanes_log2, sets = 64 >> L;
    const int at = (lane & ((1 << L) - 1)) * E, hk = h / a.group;
    const int32_t own = a.segments ? a.segments[rank] : 0;
    float q[E];
    load_elements<T, WIDE>((const T *)a.q.data + row * a.q.rank_stride + h * a.q.head_stride, at, a.head_dim, q);
    const T *k0 = (const T *)a.k.data + hk * a.k.head_stride, *v0 = (const T *)a.v.data + hk * a.v.head_stride;
    const T *bias = a.bias ? (const T *)a.bias + (int64_t)h * t.s : nullptr;
    if (own < 0) return;                                            // the row's rank holds no token
    for (int i0 = first * sets; i0 < t.s; i0 += step * sets) {
        const int i = i0 + (lane >> L);
        int32_t src = i < t.s ? neighbour_rank<false>(t, coords, i) : -1;
        if (src >= 0 && a.segments && a.segments[src] != own) src = -1;
        float k[E], v[E];
        load_elements<T, WIDE>(k0 + (src < 0 ? 0 : src) * a.k.rank_stride, at, src < 0 ? 0 : a.head_dim, k);
        load_elements<T, WIDE>(v0 + (src < 0 ? 0 : src) * a.v.rank_stride, at, src < 0 ? 0 : a.head_dim, v);
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x);
        x = sum_over_lanes(x, L) * a.scale;
        if (a.cap > 0.f) x = capped<T>(x, a.cap);
        if (bias && src >= 0) x += (float)bias[i];
        if (src < 0) x = -INFINITY;
        const float top = fmaxf(st.m, x), base = finite_floor(top);
        const float keep = exp_above(st.m, base), w = exp_above(x, base);
        st.l = st.l * keep + w;
#pragma unroll
        for (int e = 0; e < E; ++e) st.acc[e] = st.acc[e] * keep + w * v[e];
        st.m = top;
    }
    for (int b = L; b < 6; ++b) {                                   // join the sets of lanes
        const float om = __shfl_xor(st.m, 1 << b), ol = __shfl_xor(st.l, 1 << b);
        float oacc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) oacc[e] = __shfl_xor(st.acc[e], 1 << b);
        st.merge(om, ol, oacc);
    }
}

template <typename T, bool WIDE>
__device__ __forceinline__ void write_row(const AttentionArgs &a, uint32_t row, int h, const RowState<ElementTraits<T>::kPerLane> &st,
                                          bool lse = true) {
    constexpr int E = ElementTraits<T>::kPerLane;
    const int lane = threadIdx.x & 63;
    if (lane >> a.lanes_log2) return;
    float y[E];
    const float inv = st.l == 0.f ? 0.f : 1.f / st.l;               // nothing counted: acc is 0 as well
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = st.acc[e] * inv;
    store_elements<T, WIDE>((T *)a.out.data + row * a.out.rank_stride + h * a.out.head_stride, lane * E, a.head_dim, y);
    if (lse && a.lse && lane == 0) a.lse[(int64_t)row * a.q_heads + h] = st.l == 0.f ? -INFINITY : st.m + __builtin_amdgcn_logf(st.l) * kLn2;
}

// A row outside the torus, given in `rows`: treated as one without neighbours.
__device__ __forceinline__ int64_t rank_of_row(const AttentionArgs &a, uint32_t row) { return a.rows ? a.rows[row] : (int64_t)row; }

// Four (row, q head) in a workgroup, one wavefront each.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void attention_row_kernel(const AttentionArgs a) {
    __shared__ int32_t coords[4][ISO_MAX_DIMS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint64_t item = ((uint64_t)a.first_block + blockIdx.x) * 4 + wave;
    const uint32_t row = (uint32_t)(item / a.q_heads);
    const int h = (int)(item % a.q_heads);
    const int64_t rank = row < a.n ? rank_of_row(a, row) : -1;
    const bool inside = rank >= 0 && rank < a.torus.p;
    if (inside) store_coordinates(a.torus, (uint32_t)rank, lane, coords[wave]);
    __syncthreads();
    if (row >= a.n) return;
    RowState<ElementTraits<T>::kPerLane> st;
    if (inside) attend_row<T, WIDE>(a, row, (uint32_t)rank, h, 0, 1, coords[wave], st);
    write_row<T, WIDE>(a, row, h, st);
}

// One (row, q head) in a workgroup of `waves` wavefronts, each over its share of the neighbours, joined in LDS.
template <typename T, bool WIDE>
__global__ __launch_bounds__(1024) void attention_split_row_kernel(const AttentionArgs a) {
    constexpr int E = ElementTraits<T>::kPerLane;
    __shared__ int32_t coords[ISO_MAX_DIMS];
    __shared__ float part_m[16], part_l[16];
    __shared__ float part_acc[16][kAttentionMaxHeadDim];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t row = blockIdx.x / a.q_heads;
    const int h = (int)(blockIdx.x % a.q_heads);
    const int64_t rank = rank_of_row(a, row);
    const bool inside = rank >= 0 && rank < a.torus.p;
    if (inside && wave == 0) store_coordinates(a.torus, (uint32_t)rank, lane, coords);
    __syncthreads();
    RowState<E> st;
    if (inside) attend_row<T, WIDE>(a, row, (uint32_t)rank, h, wave, a.waves, coords, st);
    const bool holds = lane >> a.lanes_log2 == 0 && lane * E < kAttentionMaxHeadDim;
    if (lane == 0) part_m[wave] = st.m, part_l[wave] = st.l;
    if (holds)
#pragma unroll
        for (int e = 0; e < E; ++e) part_acc[wave][lane * E + e] = st.acc[e];
    __syncthreads();
    if (wave > 0) return;
    // lane w weighs part w; then every lane adds up its elements of all parts, whose reads do not wait for each other
    const float m = lane < a.waves ? part_m[lane] : -INFINITY;
    float top = m;
#pragma unroll
    for (int b = 0; b < 4; ++b) top = fmaxf(top, __shfl_xor(top, 1 << b));
    top = __shfl(top, 0);
    const float weight = exp_above(m, finite_floor(top));
    float l = lane < a.waves ? part_l[lane] * weight : 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) l += __shfl_xor(l, 1 << b);
    st.m = top;
    st.l = __shfl(l, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) st.acc[e] = 0.f;
    for (int w = 0; w < a.waves; ++w) {
        const float by = __shfl(weight, w);
        if (holds)
#pragma unroll
            for (int e = 0; e < E; ++e) st.acc[e] = fmaf(part_acc[w][lane * E + e], by, st.acc[e]);
    }
    write_row<T, WIDE>(a, row, h, st);
}

// ---- backward: rows ------------------------------------------------------------------
//
//     dP_i = grad_out . v_i     delta = grad_out . out     dx_i = P_i (dP_i - delta)     da_i = dx_i (1 - (t_i / cap)^2)
//     grad_q = scale sum_i da_i k_i       grad_bias[h][i] = sum over ranks of dx_i
//     grad_k and grad_v of rank S: sums over the pairs (R, i) with R = S (+) C^i, and over the q heads that share the key
//
// Every gradient is gathered by the row that it belongs to: no atomics, and the same sum in the same order every time.

// Beyond this lse its own rounding shows in the weights (by 2^-11 and more; where every bias of a row is the type's lowest
// value, the logarithm of their sum is lost whole): weights are then divided by what they add up to.
constexpr float kLargeLse = 8192.f;

// P_i and da_i of one neighbour whose dot products are given; norm: 1, or what corrects the weights of a large lse.
struct PairGradient {
    float p, dx, da;
};
template <typename T>
__device__ __forceinline__ PairGradient pair_gradient(float dot, float bias, float lse, float norm, float dp, float delta, float scale, float cap) {
    float t = dot * scale, slope = 1.f;
    if (cap > 0.f) {
        t = capped<T>(t, cap);
        const float y = t / cap;
        slope = 1.f - y * y;
    }
    PairGradient g;
    g.p = exp_above(t + bias, finite_floor(lse)) * norm;
    g.dx = g.p * (dp - delta);
    g.da = g.dx * slope;
    return g;
}

template <typename T, bool WIDE>
__device__ __forceinline__ float row_delta(const AttentionArgs &a, uint32_t rank, int h, int at) {
    constexpr int E = ElementTraits<T>::kPerLane;
    float g[E], o[E], x = 0.f;
    load_elements<T, WIDE>((const T *)a.grad_out.data + rank * a.grad_out.rank_stride + h * a.grad_out.head_stride, at, a.head_dim, g);
    load_elements<T, WIDE>((const T *)a.out.data + rank * a.out.rank_stride + h * a.out.head_stride, at, a.head_dim, o);
#pragma unroll
    for (int e = 0; e < E; ++e) x = fmaf(g[e], o[e], x);
    return sum_over_lanes(x, a.lanes_log2);
}

// bias_sums: of the row's head, to which dx is added, or null.
template <typename T, bool WIDE>
__device__ __forceinline__ void grad_q_row(const AttentionArgs &a, uint32_t rank, int h, float delta, const int32_t *coords,
                                           float *bias_sums = nullptr) {
    constexpr int E = ElementTraits<T>::kPerLane;
    const NeighbourTorus &t = a.torus;
    const int lane = threadIdx.x & 63, L = a.lanes_log2, sets = 64 >> L;
    const int at = (lane & ((1 << L) - 1)) * E, hk = h / a.group;
    const int32_t own = a.segments ? a.segments[rank] : 0;
    const float lse = a.lse[(int64_t)rank * a.q_heads + h];
    float q[E], g[E], acc[E] = {};
    load_elements<T, WIDE>((const T *)a.q.data + rank * a.q.rank_stride + h * a.q.head_stride, at, a.head_dim, q);
    load_elements<T, WIDE>((const T *)a.grad_out.data + rank * a.grad_out.rank_stride + h * a.grad_out.head_stride, at, a.head_dim, g);
    const T *k0 = (const T *)a.k.data + hk * a.k.head_stride, *v0 = (const T *)a.v.data + hk * a.v.head_stride;
    const T *bias = a.bias ? (const T *)a.bias + (int64_t)h * t.s : nullptr;
    float norm = 1.f, sum = 0.f;
    const bool large = fabsf(lse) > kLargeLse && fabsf(lse) < INFINITY;
    if (large) {                                                    // what the weights add up to
        for (int i0 = 0; i0 < (own < 0 ? 0 : t.s); i0 += sets) {
            const int i = i0 + (lane >> L);
            int32_t src = i < t.s ? neighbour_rank<false>(t, coords, i) : -1;
            if (src >= 0 && a.segments && a.segments[src] != own) src = -1;
            float k[E], x = 0.f;
            load_elements<T, WIDE>(k0 + (src < 0 ? 0 : src) * a.k.rank_stride, at, src < 0 ? 0 : a.head_dim, k);
#pragma unroll
            for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x);
            x = sum_over_lanes(x, L);
            if (src >= 0) sum += pair_gradient<T>(x, bias ? (float)bias[i] : 0.f, lse, 1.f, 0.f, 0.f, a.scale, a.cap).p;
        }
        sum = sum_across_groups(sum, L);
        norm = sum > 0.f ? 1.f / sum : 1.f;
        if (lane == 0) a.norms[(int64_t)rank * a.q_heads + h] = norm;
    }
    for (int i0 = 0; i0 < (own < 0 ? 0 : t.s); i0 += sets) {
        const int i = i0 + (lane >> L);
        int32_t src = i < t.s ? neighbour_rank<false>(t, coords, i) : -1;
        if (src >= 0 && a.segments && a.segments[src] != own) src = -1;
        float k[E], v[E], x = 0.f, dp = 0.f;
        load_elements<T, WIDE>(k0 + (src < 0 ? 0 : src) * a.k.rank_stride, at, src < 0 ? 0 : a.head_dim, k);
        load_elements<T, WIDE>(v0 + (src < 0 ? 0 : src) * a.v.rank_stride, at, src < 0 ? 0 : a.head_dim, v);
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x), dp = fmaf(g[e], v[e], dp);
        x = sum_over_lanes(x, L);
        dp = sum_over_lanes(dp, L);
        if (src >= 0) {
            const PairGradient pg = pair_gradient<T>(x, bias ? (float)bias[i] : 0.f, lse, norm, dp, delta, a.scale, a.cap);
            if (bias_sums && at == 0) bias_sums[i] += pg.dx;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(pg.da, k[e], acc[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = sum_across_groups(acc[e], L) * a.scale;
    if (lane >> L == 0)
        store_elements<T, WIDE>((T *)a.grad_q.data + rank * a.grad_q.rank_stride + h * a.grad_q.head_stride, at, a.head_dim, acc);
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void attention_grad_q_row_kernel(const AttentionArgs a) {
    constexpr int E = ElementTraits<T>::kPerLane;
    __shared__ int32_t coords[4][ISO_MAX_DIMS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint64_t item = ((uint64_t)a.first_block + blockIdx.x) * 4 + wave;
    const uint32_t rank = (uint32_t)(item / a.q_heads);
    const int h = (int)(item % a.q_heads);
    if (rank < a.n) store_coordinates(a.torus, rank, lane, coords[wave]);
    __syncthreads();
    if (rank >= a.n) return;
    const float delta = row_delta<T, WIDE>(a, rank, h, (lane & ((1 << a.lanes_log2) - 1)) * E);
    if (lane == 0) {
        const int64_t at = (int64_t)rank * a.q_heads + h;
        a.delta[at] = delta;
        if constexpr (sizeof(T) == 2) {
            if (a.starts) {
                const float lse = finite_floor(a.lse[at]);
                a.starts[at] = fabsf(lse) > kLargeLse ? NAN : a.cap > 0.f ? lse * kLog2e : -lse / a.scale;
                a.starts[(int64_t)a.n * a.q_heads + at] = -delta;
            }
        }
    }
    grad_q_row<T, WIDE>(a, rank, h, delta, coords[wave]);
}

// The grad_q kernels, which run first, have left it for rows with a large lse.
__device__ __forceinline__ float norm_of(const AttentionArgs &a, int64_t rank, int h, float lse) {
    return fabsf(lse) > kLargeLse && fabsf(lse) < INFINITY ? a.norms[rank * a.q_heads + h] : 1.f;
}

// grad_k and grad_v of one (rank, kv head): all ranks R (+) C^i and all q heads of the group.
template <typename T, bool WIDE>
__device__ __forceinline__ void grad_kv_row(const AttentionArgs &a, uint32_t rank, int hk, const int32_t *coords) {
    constexpr int E = ElementTraits<T>::kPerLane;
    const NeighbourTorus &t = a.torus;
    const int lane = threadIdx.x & 63, L = a.lanes_log2, sets = 64 >> L;
    const int at = (lane & ((1 << L) - 1)) * E;
    const int32_t own = a.segments ? a.segments[rank] : 0;
    float k[E], v[E], dk[E] = {}, dv[E] = {};
    load_elements<T, WIDE>((const T *)a.k.data + rank * a.k.rank_stride + hk * a.k.head_stride, at, a.head_dim, k);
    load_elements<T, WIDE>((const T *)a.v.data + rank * a.v.rank_stride + hk * a.v.head_stride, at, a.head_dim, v);
    for (int i0 = 0; i0 < (own < 0 ? 0 : t.s); i0 += sets) {
        const int i = i0 + (lane >> L);
        int32_t dst = i < t.s ? neighbour_rank<true>(t, coords, i) : -1;
        if (dst >= 0 && a.segments && a.segments[dst] != own) dst = -1;
        const int64_t r = dst < 0 ? 0 : dst;
        for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
            float q[E], g[E], x = 0.f, dp = 0.f;
            load_elements<T, WIDE>((const T *)a.q.data + r * a.q.rank_stride + h * a.q.head_stride, at, dst < 0 ? 0 : a.head_dim, q);
            load_elements<T, WIDE>((const T *)a.grad_out.data + r * a.grad_out.rank_stride + h * a.grad_out.head_stride, at,
                                   dst < 0 ? 0 : a.head_dim, g);
#pragma unroll
            for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x), dp = fmaf(g[e], v[e], dp);
            x = sum_over_lanes(x, L);
            dp = sum_over_lanes(dp, L);
            if (dst >= 0) {
                const float b = a.bias ? (float)((const T *)a.bias)[(int64_t)h * t.s + i] : 0.f;
                const float lse = a.lse[r * a.q_heads + h], norm = norm_of(a, r, h, lse);
                const PairGradient pg = pair_gradient<T>(x, b, lse, norm, dp, a.delta[r * a.q_heads + h], a.scale, a.cap);
#pragma unroll
                for (int e = 0; e < E; ++e) dk[e] = fmaf(pg.da, q[e], dk[e]), dv[e] = fmaf(pg.p, g[e], dv[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        dk[e] = sum_across_groups(dk[e], L) * a.scale;
        dv[e] = sum_across_groups(dv[e], L);
    }
    if (lane >> L == 0) {
        store_elements<T, WIDE>((T *)a.grad_k.data + rank * a.grad_k.rank_stride + hk * a.grad_k.head_stride, at, a.head_dim, dk);
        store_elements<T, WIDE>((T *)a.grad_v.data + rank * a.grad_v.rank_stride + hk * a.grad_v.head_stride, at, a.head_dim, dv);
    }
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void attention_grad_kv_row_kernel(const AttentionArgs a) {
    __shared__ int32_t coords[4][ISO_MAX_DIMS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint64_t item = ((uint64_t)a.first_block + blockIdx.x) * 4 + wave;
    const uint32_t rank = (uint32_t)(item / a.kv_heads);
    if (rank < a.n) store_coordinates(a.torus, rank, lane, coords[wave]);
    __syncthreads();
    if (rank < a.n) grad_kv_row<T, WIDE>(a, rank, (int)(item % a.kv_heads), coords[wave]);
}

// dx of one neighbour summed over a part of the ranks: one wavefront per (part, q head, neighbour).  grad_q's kernel has
// run before, for delta.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void attention_grad_bias_row_kernel(const AttentionArgs a) {
    constexpr int E = ElementTraits<T>::kPerLane;
    const NeighbourTorus &t = a.torus;
    const int lane = threadIdx.x & 63, L = a.lanes_log2, sets = 64 >> L;
    const uint64_t item = ((uint64_t)a.first_block + blockIdx.x) * 4 + (threadIdx.x >> 6), slots = (uint64_t)a.q_heads * t.s;
    const int part = (int)(item / slots);
    if (part >= a.parts) return;
    const int slot = (int)(item % slots), h = slot / t.s, i = slot % t.s, hk = h / a.group;
    const int at = (lane & ((1 << L) - 1)) * E;
    const uint32_t per = (a.n + a.parts - 1) / a.parts, begin = min(a.n, part * per), end = min(a.n, begin + per);
    const float bias = (float)((const T *)a.bias)[slot];
    const int32_t *c = t.offsets + (int64_t)i * t.d;
    float sum = 0.f;
    for (uint32_t r0 = begin; r0 < end; r0 += sets) {
        const uint32_t rank = r0 + (lane >> L);
        int32_t src = -1;
        if (rank < end) {
            uint32_t from = 0;
            bool there = true;
            for (int j = 0; j < t.d; ++j) {
                const uint32_t n = (uint32_t)t.dims[j];
                uint32_t x = rank / (uint32_t)t.inner[j] % n - (uint32_t)c[j];
                if (t.open >> j & 1) there = there && x < n;
                else x += (int32_t)x < 0 ? n : 0;
                from += x * (uint32_t)t.inner[j];
            }
            src = (int32_t)from;
            if (!there || (a.segments && (a.segments[rank] < 0 || a.segments[src] != a.segments[rank]))) src = -1;
        }
        const int64_t r = src < 0 ? 0 : rank, u = src < 0 ? 0 : src;
        const int end_at = src < 0 ? 0 : a.head_dim;
        float q[E], g[E], k[E], v[E], x = 0.f, dp = 0.f;
        load_elements<T, WIDE>((const T *)a.q.data + r * a.q.rank_stride + h * a.q.head_stride, at, end_at, q);
        load_elements<T, WIDE>((const T *)a.grad_out.data + r * a.grad_out.rank_stride + h * a.grad_out.head_stride, at, end_at, g);
        load_elements<T, WIDE>((const T *)a.k.data + u * a.k.rank_stride + hk * a.k.head_stride, at, end_at, k);
        load_elements<T, WIDE>((const T *)a.v.data + u * a.v.rank_stride + hk * a.v.head_stride, at, end_at, v);
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x), dp = fmaf(g[e], v[e], dp);
        x = sum_over_lanes(x, L);
        dp = sum_over_lanes(dp, L);
        if (src >= 0) {
            const float lse = a.lse[r * a.q_heads + h];
            sum += pair_gradient<T>(x, bias, lse, norm_of(a, r, h, lse), dp, a.delta[r * a.q_heads + h], a.scale, a.cap).dx;
        }
    }
    sum = sum_across_groups(sum, L);
    if (lane == 0) a.partials[(uint64_t)part * slots + slot] = sum;
}

// The parts of the bias's gradient added up, always in the same order: 16 slots of a workgroup, 64 lanes over the parts of each.
struct SumPartsArgs {
    const float *partials;
    void *out;
    uint32_t slots, parts, first_block;
};
template <typename T>
__global__ __launch_bounds__(1024) void sum_parts_kernel(const SumPartsArgs a) {
    __shared__ float sums[64][17];
    const uint32_t col = threadIdx.x & 15, row = threadIdx.x >> 4, slot = (a.first_block + blockIdx.x) * 16 + col;
    float sum = 0.f;
    if (slot < a.slots) {
#pragma unroll 4
        for (uint32_t part = row; part < a.parts; part += 64) sum += a.partials[(uint64_t)part * a.slots + slot];
    }
    sums[row][col] = sum;
    for (uint32_t half = 32; half; half /= 2) {
        __syncthreads();
        if (row < half) sums[row][col] += sums[row + half][col];
    }
    if (row == 0 && slot < a.slots) ((T *)a.out)[slot] = (T)sums[0][col];
}

}  // namespace iso
