// gfx950 kernel for rotary positions with several axes: pair j of a row's channels is turned by
// position[axis_j] * frequency_j, all heads of a rank by the same angles; channels beyond the pairs are copied.
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_fastdiv.hpp"

namespace iso {

constexpr int kRotaryAngles = 256;         // angles that a workgroup holds in LDS: about one per lane

struct RotaryArgs {
    Heads x, out;
    const int32_t *positions;              // device [n][n_axes], or null: the coordinates of rank n
    const double *turns;                   // device [pairs]: frequency_j / 2 pi
    const int32_t *axes;                   // device [pairs]
    uint32_t n, first_block;               // first_block: workgroups of the launches before, where one cannot hold all
    int32_t n_axes, head_dim, pairs, ranks;    // ranks: of one workgroup
    int32_t interleaved;                   // pairs (2j, 2j + 1) instead of (j, j + pairs)
    float sign;                            // -1 turns back
    FastDiv by_pairs, by_units, by_heads;  // units: work items of one head's row
    int32_t dims[ISO_MAX_DIMS], inner[ISO_MAX_DIMS];
};

// The bytes of x and out bound it, so each is touched once, 16 bytes a lane, and the angles, which all heads share, are
// made once per rank: by the first part of the workgroup into LDS.  The angle is reduced in turns in 64 bits (position *
// turns is exact to 2^-53 of its size), so that positions of any size turn by the right angle; sine and cosine in 32.
// 10 heads of 128 in bfloat16 at 64 x 64 x 64 ranks: 1.34 GB in 224 us, 6.0 TB/s (a copy of that size 6.6); five tokens:
// 3.2 us, one launch.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
    constexpr int E = WIDE ? ElementTraits<T>::kPerLane : 1;
    __shared__ float2 turn[kRotaryAngles];                          // count * pairs
    const uint32_t first = (a.first_block + blockIdx.x) * (uint32_t)a.ranks, count = min((uint32_t)a.ranks, a.n - first);
    for (uint32_t item = threadIdx.x; item < count * (uint32_t)a.pairs; item += 256) {
        uint32_t r, j;
        fast_divmod(item, a.by_pairs, r, j);
        const int axis = a.axes[j];
        const uint32_t rank = first + r;
        const int32_t at = a.positions ? a.positions[(uint64_t)rank * a.n_axes + axis]
                                       : (int32_t)(rank / (uint32_t)a.inner[axis] % (uint32_t)a.dims[axis]);
        double w = (double)at * a.turns[j];
        w -= rint(w);
        float s, c;
        sincospif(2.f * (float)w, &s, &c);
        turn[item] = make_float2(c, s * a.sign);
    }
    __syncthreads();
    typedef T vec_t __attribute__((ext_vector_type(E)));
    const int paired = a.interleaved ? 0 : a.pairs / E;                // units that hold first channels, their partners with them
    const uint32_t units = count * a.by_heads.div * a.by_units.div;
    for (uint32_t item = threadIdx.x; item < units; item += 256) {
        uint32_t head_row, unit, r, h;
        fast_divmod(item, a.by_units, head_row, unit);
        fast_divmod(head_row, a.by_heads, r, h);
        const int64_t rank = first + r;
        const T *x = (const T *)a.x.data + rank * a.x.rank_stride + h * a.x.head_stride;
        T *y = (T *)a.out.data + rank * a.out.rank_stride + h * a.out.head_stride;
        const float2 *cs = turn + r * a.pairs;
        if ((int)unit < paired) {                                      // channels j and j + pairs
            const int j = unit * E;
            const vec_t u = *(const vec_t *)(x + j), v = *(const vec_t *)(x + j + a.pairs);
            vec_t p, q;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float2 t = cs[j + e];
                p[e] = (T)((float)u[e] * t.x - (float)v[e] * t.y);
                q[e] = (T)((float)u[e] * t.y + (float)v[e] * t.x);
            }
            *(vec_t *)(y + j) = p;
            *(vec_t *)(y + j + a.pairs) = q;
            continue;
        }
        if constexpr (WIDE) {
            const int j = a.interleaved ? unit * E : 2 * a.pairs + (unit - paired) * E;
            vec_t u = *(const vec_t *)(x + j);
            if (j < 2 * a.pairs) {                                     // channels 2j and 2j + 1
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 t = cs[(j + e) / 2];
                    const float p = (float)u[e], q = (float)u[e + 1];
                    u[e] = (T)(p * t.x - q * t.y);
                    u[e + 1] = (T)(p * t.y + q * t.x);
                }
            }
            *(vec_t *)(y + j) = u;
        } else if (a.interleaved && (int)unit < a.pairs) {
            const float2 t = cs[unit];
            const float p = (float)x[2 * unit], q = (float)x[2 * unit + 1];
            y[2 * unit] = (T)(p * t.x - q * t.y);
            y[2 * unit + 1] = (T)(p * t.y + q * t.x);
        } else {
            y[a.pairs + unit] = x[a.pairs + unit];                     // units from `pairs` on: channels from 2 * pairs on
        }
    }
}

}  // namespace iso
