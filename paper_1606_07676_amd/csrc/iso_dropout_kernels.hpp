// gfx950 kernel for dropout from a counter-based generator: whether an element is kept follows from its number and the seed, so
// no mask is stored and the gradient's pass makes the same decisions again.
//
// Generator: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011), one block of 128
// bits for 8 elements, 16 bits each.  16 bits, because 32 would make the generator's multiplications as dear as the tensors'
// bytes; a rate is rounded to a multiple of 2^-16, and what is kept is scaled by the rounded rate's factor.
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_fastdiv.hpp"

namespace iso {

struct DropoutArgs {
    const void *x, *residual;              // residual: or null
    void *out;
    int64_t x_stride, residual_stride, out_stride;      // elements between rows
    const uint64_t *seed;                  // device [2]: key, and the upper half of the counter
    uint64_t elements;
    uint32_t blocks;                       // of 8 elements
    uint32_t channels;
    FastDiv row_blocks;                    // blocks of a row, where rows hold whole blocks
    int32_t flat;                          // the tensors are dense: one row
    uint32_t threshold;                    // of 65536: numbers below are dropped
    float scale;
    uint32_t first_block;
};

__device__ __forceinline__ uint4 philox_block(uint64_t counter, uint64_t more, uint64_t key) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)more, c3 = (uint32_t)(more >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}

// WIDE: blocks of 8 elements lie on 16-byte boundaries in all tensors, in dense tensors (the last one may not be whole) or in
// rows of whole blocks.  A lane makes one block of numbers; two 16-byte units of float32 are those of a block, and the wavefront
// hands the numbers round so that its loads and stores stay dense.
//
// The tensors' bytes bound it: 32768 x 1024 in bfloat16 with a residual 201 MB in 34.5 us, 5.8 TB/s, without 134 MB in 23.2, inputs
// from memory (1.6 GB of them take turns).  Stores that stay in the caches take 36.3 and 24.2 us, loads past them as well 33.1 and
// 22.8.  Tensors that are not WIDE go element by element: 65535 rows of 333 inside rows of 336 in bfloat16 50 us, dense rows of 336 15.8.
template <typename T, bool WIDE, bool RESIDUAL> __global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a) {
    constexpr int E = ElementTraits<T>::kPerLane, kUnits = 8 / E;
    typedef T vec_t __attribute__((ext_vector_type(E)));
    const uint32_t block = (a.first_block + blockIdx.x) * 256u + threadIdx.x;
    const uint64_t key = a.seed[0], more = a.seed[1];
    const T *x = (const T *)a.x, *residual = (const T *)a.residual;
    T *out = (T *)a.out;
    const auto dropped_or = [&](float value, uint32_t number) { return number >= a.threshold ? value * a.scale : 0.f; };
    const uint32_t whole = (uint32_t)(a.elements / 8);
    if constexpr (WIDE) {
        // unit i of this lane: the same block, or of the wavefront's 128 units the lane's and the one 64 behind
        vec_t v[kUnits], r[kUnits];
        const uint32_t lane = threadIdx.x & 63, first = block - lane;
        uint32_t row[kUnits];
        int64_t at[kUnits];
        bool there[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const uint32_t of = kUnits == 1 ? block : first + 32 * i + lane / 2;
            uint32_t rest = of;
            row[i] = 0;
            if (!a.flat) fast_divmod(of, a.row_blocks, row[i], rest);
            at[i] = rest * 8ll + (kUnits == 1 ? 0 : lane % 2 * 4);
            there[i] = of < whole;
            if (there[i]) {
                v[i] = *(const vec_t *)(x + row[i] * a.x_stride + at[i]);
                if (RESIDUAL) r[i] = *(const vec_t *)(residual + row[i] * a.residual_stride + at[i]);
            }
        }
        const uint4 bits = philox_block(block, more, key);
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            uint32_t words[E / 2];
            if constexpr (kUnits == 1) {
                words[0] = bits.x, words[1] = bits.y, words[2] = bits.z, words[3] = bits.w;
            } else {
                const int from = 32 * i + lane / 2;
                const uint32_t low[2] = {(uint32_t)__shfl(bits.x, from), (uint32_t)__shfl(bits.y, from)};
                const uint32_t high[2] = {(uint32_t)__shfl(bits.z, from), (uint32_t)__shfl(bits.w, from)};
                words[0] = lane % 2 ? high[0] : low[0];
                words[1] = lane % 2 ? high[1] : low[1];
            }
            if (!there[i]) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float y = dropped_or((float)v[i][e], e % 2 ? words[e / 2] >> 16 : words[e / 2] & 0xFFFF);
                v[i][e] = (T)(RESIDUAL ? (float)r[i][e] + y : y);
            }
            __builtin_nontemporal_store(v[i], (vec_t *)(out + row[i] * a.out_stride + at[i]));
        }
        if (block != whole) return;                        // what is left of a dense tensor
    }
    if (block >= a.blocks) return;
    const uint4 bits = philox_block(block, more, key);
    const uint32_t words[4] = {bits.x, bits.y, bits.z, bits.w};
    const uint64_t begin = (uint64_t)block * 8;
    uint64_t row = 0, at = begin;
    if (!a.flat) {
        row = begin / a.channels;
        at = begin - row * a.channels;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (begin + e >= a.elements) return;
        const float y = dropped_or((float)x[row * a.x_stride + at], e % 2 ? words[e / 2] >> 16 : words[e / 2] & 0xFFFF);
        out[row * a.out_stride + at] = (T)(RESIDUAL ? (float)residual[row * a.residual_stride + at] + y : y);
        if (++at == a.channels && !a.flat) {
            at = 0;
            ++row;
        }
    }
}

}  // namespace iso
