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
// rows of whole blocks.
template <typename T, bool WIDE> __global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a) {
    const uint32_t block = (a.first_block + blockIdx.x) * 256u + threadIdx.x;
    if (block >= a.blocks) return;
    const uint64_t first = (uint64_t)block * 8;
    const uint64_t key = a.seed[0], more = a.seed[1];
    const T *x = (const T *)a.x, *residual = (const T *)a.residual;
    T *out = (T *)a.out;
    typedef T vec_t __attribute__((ext_vector_type(8)));
    typedef vec_t half_aligned_t __attribute__((aligned(16)));
    const bool whole = WIDE && first + 8 <= a.elements;
    uint64_t row = 0, at = first;
    half_aligned_t v = {}, r = {};
    if (whole) {
        if (!a.flat) {
            uint32_t q, rest;
            fast_divmod(block, a.row_blocks, q, rest);
            row = q;
            at = rest * 8ull;
        }
        v = *(const half_aligned_t *)(x + row * a.x_stride + at);
        if (residual) r = *(const half_aligned_t *)(residual + row * a.residual_stride + at);
    }
    const uint4 bits = philox_block(block, more, key);
    const uint32_t words[4] = {bits.x, bits.y, bits.z, bits.w};
    const auto kept = [&](float value, int e) {
        const uint32_t number = e % 2 ? words[e / 2] >> 16 : words[e / 2] & 0xFFFF;
        return number >= a.threshold ? value * a.scale : 0.f;
    };
    if (whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = kept((float)v[e], e);
            v[e] = (T)(residual ? (float)r[e] + y : y);
        }
        *(half_aligned_t *)(out + row * a.out_stride + at) = v;
        return;
    }
    if (!a.flat) {
        row = first / a.channels;
        at = first - row * a.channels;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (first + e >= a.elements) return;
        const float y = kept((float)x[row * a.x_stride + at], e);
        out[row * a.out_stride + at] = (T)(residual ? (float)residual[row * a.residual_stride + at] + y : y);
        if (++at == a.channels && !a.flat) {
            at = 0;
            ++row;
        }
    }
}

}  // namespace iso
