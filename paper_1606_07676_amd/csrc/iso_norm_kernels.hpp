// gfx950 kernels for layer norm over the rows of the ranks' tokens, and its gradients.
//
//     h = (x - mean) rstd        out = weight h + bias        rstd = 1 / sqrt(var + eps)
//     grad_x = rstd (g - mean(g) - h mean(g h)),  g = weight grad_out
//     grad_weight = sum grad_out h,  grad_bias = sum grad_out  over all rows
//
// A row is held in the registers of the lanes that share it, at most 16 elements each: 8 to 64 lanes of a wavefront, or all lanes
// of a workgroup.  So each tensor is gone through once, and its bytes bound the kernels.  Lanes keep their places in the row, and
// their head, from row to row, the next row is under way while one is worked on, weights stay in registers, and so do the sums
// over rows of the weight's and the bias's gradient.  Rows of whole 128-byte lines are stored past the caches, which then hold
// more of what is read: 32768 x 1024 in bfloat16 134 MB in 25.6 us (26.2 otherwise), 70000 x 512 in float32 287 MB in 49.9 (52.6),
// gradients of the former 201 MB in 43.5 (44.2); queries and keys of 64 x 64 x 64 ranks, 10 heads of 128 in bfloat16, 1.34 GB in
// 251 (263), where vector arithmetic takes part.  Loads past the caches as well: 27.6, 49.9, 42.3 and 243.  Times here and below are
// of passes whose inputs take turns, 1.6 GB of them, so that they come from memory.
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
    uint64_t rows, step;                   // step: rows that all workgroups have at a time, a multiple of the heads but where noted
    uint64_t token_step;                   // step / heads
    FastDiv heads;
    int32_t channels, units;               // units: of 16 bytes in a row, the last one perhaps not whole
    float eps, inverse;                    // inverse: 1 / channels
    int32_t past_caches;                   // results are stored past the caches
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
// Sums over the lanes of a row, LANES of them; 0: all of the workgroup's.
template <int LANES, int N> __device__ __forceinline__ void sum_over_row(float (&x)[N], float (*shared)[16]) {
    const auto all = [&](auto &&step) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = step(x[i]);
    };
    all([](float v) { return add_moved<0xB1>(v); });                      // quads: 1 0 3 2
    all([](float v) { return add_moved<0x4E>(v); });                      // quads: 2 3 0 1
    all([](float v) { return add_moved<0x141>(v); });                     // 8 lanes mirrored
    if (!LANES || LANES > 8) all([](float v) { return add_moved<0x140>(v); });       // 16 lanes mirrored
    if (!LANES || LANES > 16) all(add_other_16);
    if (!LANES || LANES > 32) all(add_other_32);
    if constexpr (!LANES) {
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

// The lane's place, the row that it begins with, and its units of a row: units place, place + lanes, ...  WIDE: rows on 16-byte
// boundaries in whole units; otherwise units are read and written at any alignment.
template <typename T, bool WIDE, int U, int LANES> struct NormLane {
    static constexpr int E = ElementTraits<T>::kPerLane;
    typedef T vec_t __attribute__((ext_vector_type(E)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    struct Units {
        vec_t v[U];
    };
    int place, lanes, channels, units;
    uint64_t row;

    __device__ __forceinline__ explicit NormLane(const NormArgs &a) : channels(a.channels), units(a.units) {
        lanes = LANES ? LANES : blockDim.x;
        place = threadIdx.x % lanes;
        row = (uint64_t)(a.first_block + blockIdx.x) * (LANES ? 256 / LANES : 1) + (LANES ? threadIdx.x / LANES : 0);
    }
    __device__ __forceinline__ T *first(const Heads &h, const NormArgs &a) const { return at_row(h, a, row); }
    static __device__ __forceinline__ T *at_row(const Heads &h, const NormArgs &a, uint64_t row) {
        uint32_t token, head;
        fast_divmod((uint32_t)row, a.heads, token, head);
        return (T *)h.data + (int64_t)token * h.rank_stride + (int64_t)head * h.head_stride;
    }
    __device__ __forceinline__ bool unit_there(int u) const { return place + u * lanes < units; }
    // Where unit u of this lane begins in the row.  A last unit that is not whole ends with the row and begins inside the one before:
    // both hold, and store, the same values there, and sums take them once.  No load waits for the elements of a broken unit then
    // (gradients of 37271 x 483 in float16 30.6 us, with single elements 47.7).
    __device__ __forceinline__ int begin(int u) const {
        const int at = (place + u * lanes) * E;
        return WIDE ? at : max(0, min(at, channels - E));
    }
    // f(u, e) for all elements of the units that are there
    template <typename F> __device__ __forceinline__ void each(F &&f) const {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (unit_there(u)) {
#pragma unroll
                for (int e = 0; e < E; ++e) f(u, e);
            }
    }
    // Whether element e of unit u is in the row and the lane's own.
    __device__ __forceinline__ bool own(int u, int e) const {
        return WIDE || (begin(u) + e >= (place + u * lanes) * E && begin(u) + e < channels);
    }
    __device__ __forceinline__ float if_own(int u, int e, float v) const { return own(u, e) ? v : 0.f; }
    __device__ __forceinline__ void load(Units &x, const T *from) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x.v[u] = {};
            if (!unit_there(u)) continue;
            if (WIDE) {
                x.v[u] = *(const vec_t *)(from + begin(u));
            } else if (channels >= E) {
                x.v[u] = *(const loose_t *)(from + begin(u));
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < channels) x.v[u][e] = from[e];
            }
        }
    }
    __device__ __forceinline__ void store(const Units &x, T *to, bool past_caches) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!unit_there(u)) continue;
            if (WIDE && past_caches) {
                asm volatile("");                                      // or the compiler makes one plain store of both
                __builtin_nontemporal_store(x.v[u], (vec_t *)(to + begin(u)));
                asm volatile("");
            } else if (WIDE) {
                *(vec_t *)(to + begin(u)) = x.v[u];
            } else if (channels >= E) {
                *(loose_t *)(to + begin(u)) = x.v[u];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < channels) to[e] = x.v[u][e];
            }
        }
    }
    // weight or bias, `otherwise` where there is none
    __device__ __forceinline__ void load_or(Units &x, const void *from, float otherwise) const {
        if (from) {
            load(x, (const T *)from);
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) x.v[u][e] = (T)otherwise;
    }
};

// The mean is made in two steps: the elements' distances from a first one give what that is off by, so that a row far from zero
// loses nothing to the rounding of its sum; the variance is that of the distances.
template <typename T, bool WIDE, int U, int LANES>
__global__ __launch_bounds__(LANES ? 256 : 1024) void layer_norm_kernel(const NormArgs a) {
    typedef NormLane<T, WIDE, U, LANES> Lane;
    __shared__ float shared[2][16];
    const Lane lane(a);
    typename Lane::Units weight, bias, x, next;
    if (lane.row >= a.rows) return;                        // all lanes of the row
    const T *in = lane.first(a.x, a);
    T *out = lane.first(a.out, a);
    lane.load_or(weight, a.weight, 1.f);
    lane.load_or(bias, a.bias, 0.f);
    lane.load(next, in);
    for (uint64_t row = lane.row; row < a.rows; row += a.step) {
        x = next;
        in += a.token_step * a.x.rank_stride;
        if (row + a.step < a.rows) lane.load(next, in);
        float sum[1] = {0.f}, moments[2] = {0.f, 0.f};
        lane.each([&](int u, int e) { sum[0] += lane.if_own(u, e, (float)x.v[u][e]); });
        sum_over_row<LANES>(sum, shared);
        const float start = sum[0] * a.inverse;
        lane.each([&](int u, int e) {
            const float d = lane.if_own(u, e, (float)x.v[u][e] - start);
            moments[0] += d;
            moments[1] = fmaf(d, d, moments[1]);
        });
        sum_over_row<LANES>(moments, shared);
        const float off = moments[0] * a.inverse, var = fmaf(-off, off, moments[1] * a.inverse);
        const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);       // NaN stays
        if (lane.place == 0) {
            if (a.mean) a.mean[row] = start + off;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < Lane::E; ++e)
                x.v[u][e] = (T)fmaf(((float)x.v[u][e] - start - off) * rstd, (float)weight.v[u][e], (float)bias.v[u][e]);
        lane.store(x, out, a.past_caches);
        out += a.token_step * a.out.rank_stride;
    }
}

// SUMS: the weight's and the bias's gradient are asked for.  mean is one rounding off the row's mean; what that is off by is
// found again, from the same distances, so that rows far from zero give exact products.  MOVES: the step is no multiple of the
// heads, so that lanes come to other heads from row to row (at the price of registers; each workgroup leaves a partial sum, of which
// there should be no more for more heads).
template <typename T, bool WIDE, int U, int LANES, bool SUMS, bool MOVES>
__global__ __launch_bounds__(LANES ? 256 : 1024, LANES ? MOVES ? 2 : 3 : 4) void layer_norm_backward_kernel(const NormArgs a) {
    typedef NormLane<T, WIDE, U, LANES> Lane;
    constexpr int E = Lane::E;
    constexpr bool kAhead = LANES != 0;                                // 16 wavefronts have no registers for another row, nor for weights
    __shared__ float shared[3][16];
    extern __shared__ __align__(16) float wave_sums[];                 // [wavefronts][2][channels] where rows have less than a workgroup
    const Lane lane(a);
    typename Lane::Units weight, x, dy, next_x, next_dy;
    float weight_sum[SUMS ? U : 1][SUMS ? E : 1] = {}, bias_sum[SUMS ? U : 1][SUMS ? E : 1] = {};
    if (kAhead) lane.load_or(weight, a.weight, 1.f);
    const T *in = lane.first(a.x, a), *in_dy = lane.first(a.grad_out, a);
    T *out = lane.first(a.out, a);
    float next_mean = 0.f, next_rstd = 0.f;
    const auto advance = [&](auto *&now, const Heads &h, uint64_t row) {       // to `row`, which may be behind the last one
        if (MOVES) now = Lane::at_row(h, a, row);
        else now += a.token_step * h.rank_stride;
    };
    const auto load_next = [&](uint64_t row) {
        lane.load(next_x, in);
        lane.load(next_dy, in_dy);
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
    };
    if (kAhead && lane.row < a.rows) load_next(lane.row);
    for (uint64_t row = lane.row; row < a.rows; row += a.step) {
        if (!kAhead) {
            load_next(row);
            lane.load_or(weight, a.weight, 1.f);
        }
        x = next_x;
        dy = next_dy;
        const float mean = next_mean, rstd = next_rstd;
        advance(in, a.x, row + a.step);
        advance(in_dy, a.grad_out, row + a.step);
        if (kAhead && row + a.step < a.rows) load_next(row + a.step);
        float sums[3] = {0.f, 0.f, 0.f};
        lane.each([&](int u, int e) {
            const float d = lane.if_own(u, e, (float)x.v[u][e] - mean);
            const float g = lane.if_own(u, e, (float)dy.v[u][e] * (float)weight.v[u][e]);
            sums[0] += d;
            sums[1] += g;
            sums[2] = fmaf(g, d, sums[2]);
        });
        sum_over_row<LANES>(sums, shared);
        const float off = sums[0] * a.inverse, mean_g = sums[1] * a.inverse;
        const float mean_gh = (sums[2] - off * sums[1]) * a.inverse * rstd;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float h = ((float)x.v[u][e] - mean - off) * rstd;
                const float g = (float)dy.v[u][e] * (float)weight.v[u][e];
                if constexpr (SUMS) {
                    weight_sum[u][e] = fmaf((float)dy.v[u][e], h, weight_sum[u][e]);
                    bias_sum[u][e] += (float)dy.v[u][e];
                }
                x.v[u][e] = (T)(rstd * (fmaf(-h, mean_gh, g) - mean_g));
            }
        lane.store(x, out, a.past_caches);
        advance(out, a.out, row + a.step);
    }
    if constexpr (SUMS) {
        float *partial = a.partials + (uint64_t)(a.first_block + blockIdx.x) * 2 * a.channels;
        const auto put = [&](float *to) {
            lane.each([&](int u, int e) {
                const int at = lane.begin(u) + e;
                if (lane.own(u, e)) {
                    to[at] = weight_sum[u][e];
                    to[a.channels + at] = bias_sum[u][e];
                }
            });
        };
        if constexpr (!LANES) {
            put(partial);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int m = LANES; m < 64; m *= 2) {              // the wavefront's rows
                        weight_sum[u][e] += __shfl_xor(weight_sum[u][e], m);
                        bias_sum[u][e] += __shfl_xor(bias_sum[u][e], m);
                    }
            if ((threadIdx.x & 63) < LANES) put(wave_sums + (threadIdx.x >> 6) * 2 * a.channels);
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
