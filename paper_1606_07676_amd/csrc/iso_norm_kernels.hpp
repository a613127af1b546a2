// gfx950 kernels for layer norm over the rows of the ranks' tokens, and its gradients.
//
//     h = (x - mean) rstd        out = weight h + bias        rstd = 1 / sqrt(var + eps)
//     grad_x = rstd (g - mean(g) - h mean(g h)),  g = weight grad_out
//     grad_weight = sum grad_out h,  grad_bias = sum grad_out  over all rows
//
// A row is held in the registers of the lanes that share it, at most 16 elements each: up to 64 lanes of a wavefront, or all
// lanes of a workgroup.  So each tensor is gone through once, and its bytes bound the kernels.  Lanes keep their places in the
// row from row to row, weights stay in registers, and so do the sums over rows of the weight's and the bias's gradient.
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_fastdiv.hpp"

namespace iso {

constexpr int kNormLaneElements = 16;
constexpr int kNormMaxChannels = 1024 * kNormLaneElements;

struct NormArgs {
    Heads x, out;                          // out: of the forward pass; the gradient of x in the backward pass
    Heads grad_out;
    const void *weight, *bias;             // [channels] or null
    float *mean, *rstd;                    // [n][heads]; may be null in the forward pass
    float *partials;                       // [workgroups][2][channels]: sums for the weight's and the bias's gradient
    uint64_t rows;
    FastDiv heads;
    int32_t channels, units;               // units: of 16 bytes in a row, the last one perhaps not whole
    int32_t lanes;                         // that share a row: a power of two
    float eps, inverse;                    // inverse: 1 / channels
    uint32_t first_block;
};

// x + (x of the lane whose number differs in one bit), for the sums over neighbouring lanes: each step doubles the lanes that
// hold the same sum, so mirrored lanes serve as well as exchanged ones.  Same bits in all lanes.
template <int CONTROL> __device__ __forceinline__ float add_moved(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float add_other_16(float x) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float add_other_32(float x) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
// Sums over groups of `lanes` lanes, a power of two up to 64.
template <int N> __device__ __forceinline__ void sum_over_lanes(float (&x)[N], int lanes) {
    const auto all = [&](auto &&step) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = step(x[i]);
    };
    if (lanes > 1) all([](float v) { return add_moved<0xB1>(v); });       // quads: 1 0 3 2
    if (lanes > 2) all([](float v) { return add_moved<0x4E>(v); });       // quads: 2 3 0 1
    if (lanes > 4) all([](float v) { return add_moved<0x141>(v); });      // 8 lanes mirrored
    if (lanes > 8) all([](float v) { return add_moved<0x140>(v); });      // 16 lanes mirrored
    if (lanes > 16) all(add_other_16);
    if (lanes > 32) all(add_other_32);
}
// Sums over the lanes of a row.  WHOLE: the row has all of the workgroup's wavefronts.
template <bool WHOLE, int N> __device__ __forceinline__ void sum_over_row(float (&x)[N], int lanes, float (*shared)[16]) {
    sum_over_lanes(x, WHOLE ? 64 : lanes);
    if constexpr (WHOLE) {
        const int waves = blockDim.x >> 6;
        __syncthreads();                                               // the sums before these have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) shared[i][threadIdx.x >> 6] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = 0.f;
            for (int w = 0; w < waves; ++w) x[i] += shared[i][w];
        }
    }
}

// A lane's units of a row: units lane, lane + lanes, ...  WIDE: rows on 16-byte boundaries in whole units; otherwise units are
// read and written at any alignment and the elements of the last one singly.
template <typename T, bool WIDE, int U> struct NormRow {
    static constexpr int E = ElementTraits<T>::kPerLane;
    typedef T vec_t __attribute__((ext_vector_type(E)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    vec_t v[U];

    __device__ __forceinline__ void load(const T *row, int lane, const NormArgs &a) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * a.lanes, at = unit * E;
            v[u] = {};
            if (WIDE || at + E <= a.channels) {
                if (unit < a.units) v[u] = WIDE ? *(const vec_t *)(row + at) : *(const loose_t *)(row + at);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at + e < a.channels) v[u][e] = row[at + e];
            }
        }
    }
    __device__ __forceinline__ void store(T *row, int lane, const NormArgs &a) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * a.lanes, at = unit * E;
            if (WIDE || at + E <= a.channels) {
                if (unit >= a.units) continue;
                if (WIDE) *(vec_t *)(row + at) = v[u];
                else *(loose_t *)(row + at) = v[u];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at + e < a.channels) row[at + e] = v[u][e];
            }
        }
    }
    __device__ __forceinline__ bool there(int u, int e, int lane, const NormArgs &a) const {
        const int unit = lane + u * a.lanes;
        return WIDE ? unit < a.units : unit * E + e < a.channels;
    }
};

template <typename T> __device__ __forceinline__ T *norm_row(const Heads &h, uint64_t row, const NormArgs &a) {
    uint32_t token, head;
    fast_divmod((uint32_t)row, a.heads, token, head);
    return (T *)h.data + token * h.rank_stride + head * h.head_stride;
}

// Rows of this lane's group: first, first + step, ...
struct NormRows {
    int lane;
    uint64_t first, step;
};
template <bool WHOLE> __device__ __forceinline__ NormRows norm_rows(const NormArgs &a) {
    if (WHOLE) return {(int)threadIdx.x, a.first_block + blockIdx.x, gridDim.x};
    const uint32_t groups = blockDim.x / a.lanes;
    return {(int)(threadIdx.x & (a.lanes - 1)), (uint64_t)(a.first_block + blockIdx.x) * groups + threadIdx.x / a.lanes,
            (uint64_t)gridDim.x * groups};
}

// The mean is made in two steps: the elements' distances from a first one give what that is off by, so that a row far from zero
// loses nothing to the rounding of its sum; the variance is that of the distances.
template <typename T, bool WIDE, int U, bool WHOLE>
__global__ __launch_bounds__(WHOLE ? 1024 : 256) void layer_norm_kernel(const NormArgs a) {
    typedef NormRow<T, WIDE, U> Row;
    constexpr int E = Row::E;
    __shared__ float shared[2][16];
    const NormRows rows = norm_rows<WHOLE>(a);
    Row weight, bias, x, next;
    if (a.weight) weight.load((const T *)a.weight, rows.lane, a);
    if (a.bias) bias.load((const T *)a.bias, rows.lane, a);
    if (rows.first < a.rows) next.load(norm_row<T>(a.x, rows.first, a), rows.lane, a);
    for (uint64_t row = rows.first; row < a.rows; row += rows.step) {
        x = next;
        if (row + rows.step < a.rows) next.load(norm_row<T>(a.x, row + rows.step, a), rows.lane, a);
        float sum[1] = {0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += (float)x.v[u][e];
        sum_over_row<WHOLE>(sum, a.lanes, shared);
        const float start = sum[0] * a.inverse;
        float d[U][E], moments[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                d[u][e] = x.there(u, e, rows.lane, a) ? (float)x.v[u][e] - start : 0.f;
                moments[0] += d[u][e];
                moments[1] = fmaf(d[u][e], d[u][e], moments[1]);
            }
        sum_over_row<WHOLE>(moments, a.lanes, shared);
        const float off = moments[0] * a.inverse, var = fmaxf(fmaf(-off, off, moments[1] * a.inverse), 0.f);
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (rows.lane == 0) {
            if (a.mean) a.mean[row] = start + off;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float y = (d[u][e] - off) * rstd;
                if (a.weight) y *= (float)weight.v[u][e];
                if (a.bias) y += (float)bias.v[u][e];
                x.v[u][e] = (T)y;
            }
        x.store(norm_row<T>(a.out, row, a), rows.lane, a);
    }
}

// SUMS: the weight's and the bias's gradient are asked for.  mean is one rounding off the row's mean; what that is off by is
// found again, from the same distances, so that rows far from zero give exact products.
template <typename T, bool WIDE, int U, bool WHOLE, bool SUMS>
__global__ __launch_bounds__(WHOLE ? 1024 : 256) void layer_norm_backward_kernel(const NormArgs a) {
    typedef NormRow<T, WIDE, U> Row;
    constexpr int E = Row::E;
    __shared__ float shared[3][16];
    extern __shared__ __align__(16) float wave_sums[];                 // [wavefronts][2][channels] where rows have less than a workgroup
    const NormRows rows = norm_rows<WHOLE>(a);
    Row weight, x, dy;
    float weight_sum[SUMS ? U : 1][SUMS ? E : 1] = {}, bias_sum[SUMS ? U : 1][SUMS ? E : 1] = {};
    if (a.weight) weight.load((const T *)a.weight, rows.lane, a);
    for (uint64_t row = rows.first; row < a.rows; row += rows.step) {
        x.load(norm_row<T>(a.x, row, a), rows.lane, a);
        dy.load(norm_row<T>(a.grad_out, row, a), rows.lane, a);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sums[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = x.there(u, e, rows.lane, a) ? (float)x.v[u][e] - mean : 0.f;
                const float g = (float)dy.v[u][e] * (a.weight ? (float)weight.v[u][e] : 1.f);
                sums[0] += d;
                sums[1] += g;
                sums[2] = fmaf(g, d, sums[2]);
            }
        sum_over_row<WHOLE>(sums, a.lanes, shared);
        const float off = sums[0] * a.inverse, mean_g = sums[1] * a.inverse;
        const float mean_gh = (sums[2] - off * sums[1]) * a.inverse * rstd;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float h = ((float)x.v[u][e] - mean - off) * rstd;
                const float g = (float)dy.v[u][e] * (a.weight ? (float)weight.v[u][e] : 1.f);
                if constexpr (SUMS) {
                    weight_sum[u][e] = fmaf((float)dy.v[u][e], h, weight_sum[u][e]);
                    bias_sum[u][e] += (float)dy.v[u][e];
                }
                x.v[u][e] = (T)(rstd * (g - mean_g - h * mean_gh));
            }
        x.store(norm_row<T>(a.out, row, a), rows.lane, a);
    }
    if constexpr (SUMS) {
        float *partial = a.partials + (uint64_t)(a.first_block + blockIdx.x) * 2 * a.channels;
        const auto put = [&](float *to) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x.there(u, e, rows.lane, a)) {
                        const int at = (rows.lane + u * a.lanes) * E + e;
                        to[at] = weight_sum[u][e];
                        to[a.channels + at] = bias_sum[u][e];
                    }
        };
        if constexpr (WHOLE) {
            put(partial);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    for (int m = a.lanes; m < 64; m *= 2) {            // the wavefront's rows
                        weight_sum[u][e] += __shfl_xor(weight_sum[u][e], m);
                        bias_sum[u][e] += __shfl_xor(bias_sum[u][e], m);
                    }
            if ((int)(threadIdx.x & 63) < a.lanes) put(wave_sums + (threadIdx.x >> 6) * 2 * a.channels);
            __syncthreads();
            for (int i = threadIdx.x; i < 2 * a.channels; i += 256) {
                float s = 0.f;
                for (int w = 0; w < 4; ++w) s += wave_sums[w * 2 * a.channels + i];
                partial[i] = s;
            }
        }
    }
}

struct NormSumArgs {
    const float *partials;                 // [parts][2][channels]
    void *out[2];                          // of the weight and of the bias, either may be null
    int32_t parts, channels;
    uint32_t first_block;
};

// 16 of the 2 * channels sums to a workgroup, its 64 groups of 16 lanes taking the parts in turn.
template <typename T> __global__ __launch_bounds__(1024) void layer_norm_sum_kernel(const NormSumArgs a) {
    __shared__ float shared[16][17];
    const int slot = (a.first_block + blockIdx.x) * 16 + threadIdx.x % 16, slots = 2 * a.channels;
    float sum = 0.f;
    if (slot < slots)
        for (int part = threadIdx.x / 16; part < a.parts; part += 64) sum += a.partials[(uint64_t)part * slots + slot];
    sum = add_other_32(add_other_16(sum));
    if (threadIdx.x % 64 < 16) shared[threadIdx.x / 64][threadIdx.x % 16] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || slot >= slots) return;
    sum = 0.f;
    for (int w = 0; w < 16; ++w) sum += shared[w][threadIdx.x];
    T *out = (T *)a.out[slot >= a.channels];
    if (out) out[slot % a.channels] = (T)sum;
}

}  // namespace iso
