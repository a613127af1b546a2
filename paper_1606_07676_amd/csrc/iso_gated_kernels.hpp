// gfx950 kernels for the gated projections of a feed-forward block, and their gradients.
//
//     g = x . gate,  u = x . up,  out = f(g) u                          (rows of x: tokens; rows of gate and up: hidden units)
//     d_up = grad_out f(g),  d_gate = grad_out u f'(g)
//     grad_x = d_gate gate + d_up up,  grad_gate = d_gate^T x,  grad_up = d_up^T x
//
// All of it is matrix products, four kinds of them over one main loop (ProductKind); the activation, the product and its
// derivatives happen on the accumulators of the first, so g and u are never stored: the backward pass makes them again (a third
// of its products) and keeps d_gate and d_up in the tensors' type in its workspace.  All sums are 32-bit.
//
// float16 has too few exponents for d_gate and d_up as they are: below 2^-14 it rounds by up to 2^-25, whatever the value.  So what
// is below kLarge is kept times kScale as well, in a second row behind each token's, and marks tell the later products where none
// of a result's values is larger (Marks below): grad_x by token, the weights' gradients by block of hidden units.  They take
// such rows and blocks from the copy, and undo the scale, a power of two, on their 32-bit sums.  No value is off by more than half a
// unit in its last place, or 2^-25 where the row or block holds values of kLarge and more, 2^-41 where it does not.  32768 tokens,
// 1024 channels, 2816 hidden units: 1158 us, 1216 where all are small, 1130 without copies; 200000 tokens, 128 channels, 384 hidden
// units 363, 412 and 335.
//
// The main loop: a workgroup takes a tile of the result, TileP elements along a row by TileQ rows.  Operands come in steps of
// 128 bytes of the summed axis, 64 elements of 16 bits or 32 of 32, into one of two stages in LDS, one step ahead.  An operand
// whose summed axis is its rows' (DOWN below) is read back transposed, so none is ever laid out anew in memory.
//
// The matrix units bound it for large products, up to the tiles' ends and what loads take from them: 32768 tokens, 1024 channels,
// 4096 hidden units, bfloat16, 468 us forward with inputs from memory, 1.17 PFLOP/s (a library product of these sizes 1.26); 8192 of
// each 1.41.  The gradients at 2816 hidden units 1.09 ms: 404, 311 and 362 us for the three products, 25 for the sums of the last
// one's parts.  float32 reaches 135 TFLOP/s of a library product's 153.
#pragma once

#include "iso_attention_kernels.hpp"
#include "iso_attention_tiles.hpp"
#include "iso_fastdiv.hpp"

#include <type_traits>

namespace iso {

enum Activation { kSilu = ISO_ACTIVATION_SILU, kGelu = ISO_ACTIVATION_GELU };

struct Rows {                              // element stride
    const void *data;
    int64_t stride;
};

enum class ProductKind {
    kForward,                              // P: gate and up, half a tile each   Q: x             sum over channels
    kGates,                                // the same, up to d_gate and d_up
    kGradX,                                // P: gate, then up, down their rows  Q: d_gate, d_up  sum over hidden units, twice
    kGradWeights                           // P: x, down its rows                Q: d_gate or d_up, down its rows    sum over tokens
};

struct ProductArgs {
    Rows p[2], q[2], out[2];
    Rows grad_out;                         // kGates
    float *partials;                       // [splits][halves][rows of the result][elements of a row], where splits > 1
    int32_t np, nq, nk;                    // elements of a result's row, its rows, length of the summed axis
    int32_t p_units;                       // elements of a row of P in whole units of 16 bytes, where P is gone through down its rows
    int32_t d_width;                       // elements of a row of d_gate and d_up in whole units
    uint32_t *marks;                       // float16 gradients: [groups of 16 tokens][blocks of hidden units]
    int32_t marks_row, marks_block;        // blocks of a group, hidden units of a block
    int32_t steps, split_steps;            // of the whole summed axis, and of one split of it
    int32_t splits;
    uint32_t p_tiles, q_tiles;
    FastDiv tiles, band_items;             // tiles of all halves; of a full band of kBand rows of tiles
    uint32_t halves;                       // results of a kind: 2 for kGradWeights
    uint32_t items, per_xcd, first_block;
    int32_t activation;
    int32_t past_caches;                   // kForward: whole tiles of `out` are stored past the caches
};

constexpr int kBand = 8;
constexpr int kStepBytes = 128;

// A mark: of 16 tokens and a block of hidden units, bit t whether token t has a finite d_gate of kLarge or more there, bit 16 + t the
// same of d_up.  What is smaller fits in float16 times kScale.  With kLarge at 1/2 a row that has a value as large as that loses
// nothing that could be seen in its sums to those below 2^-14: 2^-25 is 2^-24 of that value.
constexpr float kLarge = 0.5f, kScale = 65536.f;
template <typename T, ProductKind KIND> constexpr bool kScaled = std::is_same<T, _Float16>::value && KIND != ProductKind::kForward;

static __device__ const u4 kZeroUnit = {0, 0, 0, 0};

// ---- activations -------------------------------------------------------------

// f(g) = g s and f'(g).  In 16 bits exponentials and reciprocals are the hardware's, off by 2^-22 or so, and the error function's
// share is 0.5 erfc(|g| / sqrt 2) = t P(t) exp(-g^2 / 2), t = 1 / (1 + 0.26 |g|), P of degree 8 fitted to the smallest largest
// relative error: with the constants below 7.9e-8 for |g| < 14.5, beyond which the share is 0 in 32 bits.  Made in 32 bits it is off
// by less than 2^-24 (8 + 2 g^2) of itself, most of it from the exponential's argument.  The exponential serves the derivative too.
template <typename T> __device__ __forceinline__ void activate(int activation, float g, float &f, float &slope) {
    if (activation == kSilu) {
        float s;
        if constexpr (sizeof(T) == 4) s = 1.f / (1.f + expf(-g));
        else s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * g));
        f = g * s;
        slope = fmaf(f, 1.f - s, s);
    } else {
        float c, e;
        if constexpr (sizeof(T) == 4) {
            c = 0.5f * erfcf(-0.70710678118654752440f * g);
            e = expf(-0.5f * g * g);
        } else {
            const float t = __builtin_amdgcn_rcpf(fmaf(0.26f, fabsf(g), 1.f));
            e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * (g * g));
            constexpr float kTerms[9] = {0.103757021f, 0.103050987f, 0.102788585f, 0.0519652266f, 0.158757743f,
                                         -0.147787768f, 0.248731736f, -0.151493681f, 0.0302301365f};
            float rest = kTerms[8];
#pragma unroll
            for (int i = 7; i >= 0; --i) rest = fmaf(t, rest, kTerms[i]);
            rest *= t * e;
            c = g < 0.f ? rest : 1.f - rest;
        }
        f = g * c;
        slope = fmaf(g * 0.39894228040143267794f, e, c);
    }
}

// ---- operands in LDS -----------------------------------------------------------

// An operand's tile for one step.  !DOWN: N rows of 128 bytes, the summed axis along the row.  DOWN: one row of N elements for
// each of the step's places on the summed axis.  16-byte units of a row are permuted by the row (turn), so that lanes that read
// together find different banks.  PAIR: the rows are those of two tensors, half a tile each.  RUN: of how many groups of 16 a
// product's lanes take four rows each in turn, so that a lane's results are 4 RUN neighbours (!DOWN).
template <typename T, int N, bool DOWN, bool PAIR, int RUN, int THREADS> struct Operand {
    static constexpr int E = 16 / sizeof(T), kStep = kStepBytes / sizeof(T), kBytes = N * kStepBytes;
    static constexpr int kLoads = N * 8 / THREADS, kUnits = DOWN ? N / E : 8;       // loads of a lane, units of a row
    static constexpr int kThreads = THREADS, kTensors = PAIR ? 2 : 1, kRows = PAIR ? N / 2 : N;
    static_assert(N * 8 % THREADS == 0 && (!PAIR || kLoads % 2 == 0));

    static __device__ __forceinline__ int turn(int row) {
        if (!DOWN) return RUN == 2 ? (row & 3) | (row >> 3 & 1) << 2 : row & 7;
        if (sizeof(T) == 2) return ((row & 3) << 1 | (row >> 3 & 1) << 3) & (kUnits - 1);
        return (row >> 2 & 3) << 2;
    }
    static __device__ __forceinline__ int row_of(int i) { return (threadIdx.x + THREADS * i) / kUnits; }
    static __device__ __forceinline__ int unit_of(int i) { return (threadIdx.x + THREADS * i) % kUnits ^ turn(row_of(i)); }
    static constexpr __device__ int tensor_of(int i) { return PAIR && i >= kLoads / 2; }

    const unsigned char *base[kTensors];   // of the tile's first row at the step, the same for all lanes
    uint32_t offset[kLoads];               // of the lane's units from there: rows of fewer than 2^24 bytes

    __device__ __forceinline__ void begin_at(const Rows *x, int k, int first) {
#pragma unroll
        for (int t = 0; t < kTensors; ++t) base[t] = (const unsigned char *)((const T *)x[t].data + first * x[t].stride + k);
    }
    // Rows first, first + 1, ..., of which there are `rows` (the last stands for those behind it), the summed axis from k on.
    __device__ __forceinline__ void begin_rows(const Rows *x, int k, int first, int rows) {
        begin_at(x, k, first);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            offset[i] = min(row_of(i) % kRows, rows - 1 - first) * (uint32_t)(x[tensor_of(i)].stride * sizeof(T)) + unit_of(i) * 16;
    }
    // Elements from `first` on of rows k, k + 1, ..., which hold `end`, a multiple of E.
    __device__ __forceinline__ void begin_down(const Rows &x, int k, int first, int end) {
        base[0] = (const unsigned char *)((const T *)x.data + k * x.stride + first);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            offset[i] = row_of(i) * (uint32_t)(x.stride * sizeof(T)) + min(unit_of(i) * E, end - E - first) * (uint32_t)sizeof(T);
    }
    __device__ __forceinline__ void advance(int64_t stride) {
#pragma unroll
        for (int t = 0; t < kTensors; ++t) base[t] += DOWN ? kStep * stride * (int64_t)sizeof(T) : kStepBytes;
    }
    // Straight into LDS, 16 bytes a lane, one lane's after the other's; waited for by wait_for_stage.  In assembly, as the compiler
    // would wait for the whole stage before each transposing read of the other one.  places: how many of the step's places on the
    // summed axis there are; the others become zeros.
    __device__ __forceinline__ void start(unsigned char *stage, int places) const {
        const uint32_t first = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)stage +
                               __builtin_amdgcn_readfirstlane((threadIdx.x & ~63u) * 16);
        uint32_t m0;
        if (places >= kStep) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                             : "=&s"(m0) : "s"(first + THREADS * 16 * i), "v"(offset[i]), "s"(base[tensor_of(i)]) : "memory");
            return;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const void *from = base[tensor_of(i)] + offset[i];
            if ((DOWN ? row_of(i) : unit_of(i) * E) >= places) from = &kZeroUnit;
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                         : "=&s"(m0) : "s"(first + THREADS * 16 * i), "v"(from) : "memory");
        }
    }

    // Where a lane reads: row or element lane % 16 of a group of 16, a quarter of the step's places by lane / 16.
    static __device__ __forceinline__ uint32_t lane_base() {
        const int lane = threadIdx.x & 63, quarter = lane / 16, within = lane % 16;
        if (!DOWN) {
            const int row = within / 4 * 4 * RUN + within % 4;
            return row * kStepBytes + (quarter ^ turn(row)) * 16;
        }
        if (sizeof(T) == 2) {
            const int row = 8 * quarter + within / 4;
            return row * N * 2 + (turn(row) ^ (within % 4 / 2)) * 16 + within % 2 * 8;
        }
        return 4 * quarter * N * 4 + ((quarter << 2) ^ (within / 4)) * 16 + within % 4 * 4;
    }
    // The group of 16 rows or elements that begins at `first`, half `h` of the step: 8 elements of 16 bits, or 4 of 32, of the
    // summed axis.
    static __device__ __forceinline__ u4 read(const unsigned char *stage, uint32_t base, int first, int h) {
        const int g = first / 16;
        if constexpr (!DOWN) {
            return *(const u4 *)(stage + ((base + first * kStepBytes) ^ (h * 64)));
        } else if constexpr (sizeof(T) == 2) {
            constexpr int kGroups = kUnits / 2 < 8 ? kUnits / 2 : 8;       // groups of 16 that the permutation mixes
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 *lds_t;
            const unsigned char *from = stage + (base ^ (g % kGroups * 32)) + g / kGroups * kGroups * 32 + h * 32 * N * 2;
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)from));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(from + 4 * N * 2)));
            return u4{a.x, a.y, b.x, b.y};
        } else {
            const unsigned char *from = stage + (base ^ (g % 4 * 64)) + g / 4 * 256 + h * 16 * N * 4;
            u4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *(const uint32_t *)(from + i * N * 4);
            return v;
        }
    }
};

// Rows at any alignment, of any length and any distance: through registers into the same places.
template <typename Operand, typename T> struct LooseRows {
    static constexpr int kLoads = Operand::kLoads;
    const T *at[kLoads];
    u4 held[kLoads];

    __device__ __forceinline__ void begin_rows(const Rows *x, int k, int first, int rows) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const Rows &y = x[Operand::tensor_of(i)];
            at[i] = (const T *)y.data + min(first + Operand::row_of(i) % Operand::kRows, rows - 1) * y.stride + k + Operand::unit_of(i) * Operand::E;
        }
    }
    __device__ __forceinline__ void advance() {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) at[i] += Operand::kStep;
    }
    __device__ __forceinline__ void fetch(int places) {
        constexpr int E = Operand::E;
        typedef T vec_t __attribute__((ext_vector_type(E)));
        typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int left = places - Operand::unit_of(i) * E;
            vec_t v = {};
            if (left >= E) {
                v = *(const loose_t *)at[i];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < left) v[e] = at[i][e];
            }
            held[i] = __builtin_bit_cast(u4, v);
        }
    }
    __device__ __forceinline__ void keep(unsigned char *stage) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) *(u4 *)(stage + (threadIdx.x + Operand::kThreads * i) * 16) = held[i];
    }
};

typedef float f4 __attribute__((ext_vector_type(4)));
template <typename T> __device__ __forceinline__ f4 multiply_units(u4 p, u4 q, f4 acc) {
    if constexpr (sizeof(T) == 2) {
        typedef typename Matrix<T>::x8 x8;
        return Matrix<T>::multiply(__builtin_bit_cast(x8, p), __builtin_bit_cast(x8, q), acc);
    } else {
        const f4 x = __builtin_bit_cast(f4, p), y = __builtin_bit_cast(f4, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], acc, 0, 0, 0);
        return acc;
    }
}

// ---- tiles ---------------------------------------------------------------------

// WP x WQ wavefronts, each GP x GQ groups of 16 x 16.
template <int WP_, int WQ_, int GP_, int GQ_> struct ProductTile {
    static constexpr int WP = WP_, WQ = WQ_, GP = GP_, GQ = GQ_;
    static constexpr int P = WP * GP * 16, Q = WQ * GQ * 16, kThreads = WP * WQ * 64;
    static constexpr int kLds = 2 * (P + Q) * kStepBytes;
};

// Which tile a workgroup takes.  Workgroups go to the 8 XCDs in turn; each XCD takes a run of tiles, in bands of kBand rows of
// tiles, so that those it has at a time share their operands in its L2.
struct ProductWork {
    int p, q, half, split;
    bool any;
};
__device__ __forceinline__ ProductWork product_work(const ProductArgs &a) {
    const uint32_t block = a.first_block + blockIdx.x, item = (block & 7) * a.per_xcd + (block >> 3);
    ProductWork w{};
    w.any = item < a.items;
    uint32_t tile, split, half, band, within;
    fast_divmod(item, a.tiles, split, tile);
    half = tile >= a.p_tiles * a.q_tiles;
    tile -= half ? a.p_tiles * a.q_tiles : 0;
    fast_divmod(tile, a.band_items, band, within);
    const uint32_t left = min(a.q_tiles - band * kBand, (uint32_t)kBand);         // rows of tiles of this band
    w.p = left == kBand ? within / kBand : within / left;
    w.q = band * kBand + (left == kBand ? within % kBand : within % left);
    w.half = half;
    w.split = split;
    return w;
}

// What was started is in LDS, and all wavefronts have done with the stage before.
__device__ __forceinline__ void wait_for_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// N consecutive elements of a row, of which `left` are there, at any alignment.
template <typename T, int N> struct Run {
    typedef T vec_t __attribute__((ext_vector_type(N)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    vec_t v;

    __device__ __forceinline__ void load(const T *from, int left) {
        v = {};
        if (left >= N) {
            v = *(const loose_t *)from;
        } else {
#pragma unroll
            for (int r = 0; r < N - 1; ++r)
                if (r < left) v[r] = from[r];
        }
    }
    __device__ __forceinline__ void store(T *to, int left) const {
        if (left >= N) {
            *(loose_t *)to = v;
        } else {
#pragma unroll
            for (int r = 0; r < N - 1; ++r)
                if (r < left) to[r] = v[r];
        }
    }
};
template <typename T> __device__ __forceinline__ void store_four(T *to, f4 x, int left) {
    Run<T, 4> y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y.v[r] = (T)x[r];
    y.store(to, left);
}

// What becomes of neighbouring hidden units of a token, from h on, from their g and u, N / 4 groups of four.  d_gate and d_up are
// rounded to the tensors' type, as the matrix units take them in the products that follow: at most half a unit in the last place
// each (float16: see above), which leaves the gradients' error at about 1.4 times that of their own rounding.
template <typename T, bool BACKWARD, int N> struct GatedEnd {
    static constexpr bool kTwice = BACKWARD && std::is_same<T, _Float16>::value;
    Run<T, N> dy;

    __device__ __forceinline__ void load(const ProductArgs &a, int token, int h, int left) {
        if (BACKWARD) dy.load((const T *)a.grad_out.data + (int64_t)token * a.grad_out.stride + h, left);
    }
    static __device__ __forceinline__ bool large(float d) { return fabsf(d) >= kLarge && fabsf(d) <= 3.402823466e38f; }
    // For each of 16 tokens, whether one of its four lanes says so.
    static __device__ __forceinline__ uint32_t tokens_of(bool lane_has) {
        const uint64_t lanes = __ballot(lane_has);
        const uint32_t halves = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        return (halves | halves >> 16) & 0xFFFF;
    }
    // left: hidden units from h on; there: whether the token is (kTwice: all lanes of the wavefront come here, for 16 tokens)
    template <bool PAST_CACHES = false>
    __device__ __forceinline__ void finish(const ProductArgs &a, int token, bool there, int h, int left, const f4 (&g)[N / 4],
                                           const f4 (&u)[N / 4]) const {
        Run<T, N> first, second, first_scaled, second_scaled;
        bool large_first = false, large_second = false;
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float f, slope;
            activate<T>(a.activation, g[r / 4][r % 4], f, slope);
            if constexpr (BACKWARD) {
                // rows of the workspace are whole units of 16 bytes; what is behind the last hidden unit stays out of all sums
                const bool inside = r < left && (!kTwice || there);
                const float d_gate = inside ? (float)dy.v[r] * u[r / 4][r % 4] * slope : 0.f, d_up = inside ? (float)dy.v[r] * f : 0.f;
                first.v[r] = (T)d_gate;
                second.v[r] = (T)d_up;
                if constexpr (kTwice) {
                    first_scaled.v[r] = (T)(d_gate * kScale);
                    second_scaled.v[r] = (T)(d_up * kScale);
                    large_first |= large(d_gate);
                    large_second |= large(d_up);
                }
            } else {
                first.v[r] = (T)(f * u[r / 4][r % 4]);
            }
        }
        if (!BACKWARD && PAST_CACHES) {
            __builtin_nontemporal_store(first.v, (typename Run<T, N>::loose_t *)((T *)a.out[0].data + (int64_t)token * a.out[0].stride + h));
            return;
        }
        if (BACKWARD) left += a.d_width - a.np;
        T *const to = (T *)a.out[0].data + (int64_t)token * a.out[0].stride + h;
        if constexpr (!kTwice) {
            first.store(to, left);
            if (BACKWARD) second.store((T *)a.out[1].data + (int64_t)token * a.out[1].stride + h, left);
        } else {
            const uint32_t lane = threadIdx.x & 63, firsts = tokens_of(large_first), seconds = tokens_of(large_second);
            if (there) {
                T *const to_up = (T *)a.out[1].data + (int64_t)token * a.out[1].stride + h;
                first.store(to, left);
                second.store(to_up, left);
                if (!(firsts >> lane % 16 & 1)) first_scaled.store(to + a.d_width, left);
                if (!(seconds >> lane % 16 & 1)) second_scaled.store(to_up + a.d_width, left);
                if (lane == 0 && h < a.np) a.marks[(int64_t)(token / 16) * a.marks_row + h / (4 * N)] = firsts | seconds << 16;
            }
        }
    }
};

// Of a tile's rows of d_gate or d_up, which are taken as they are and which from their scaled copies.
//
// grad_x: results are tokens, each with all its hidden units, first d_gate's and then d_up's.  Weights' gradients: results are hidden
// units, taken by groups of 16 over the tokens that are summed here, of one of the two.
template <int Q, int THREADS> struct Marks {
    static constexpr int kGroups = Q / 16;
    const uint32_t *groups;                // in LDS: bit r: row r of the group as it is (r + 16: in d_up)

    template <bool TOKENS>
    __device__ __forceinline__ Marks(const ProductArgs &a, std::integral_constant<bool, TOKENS>, int q0, int half, int first_token,
                                     int end_token, uint32_t *shared) : groups(shared) {
        if (threadIdx.x < kGroups) shared[threadIdx.x] = 0;
        __syncthreads();
        const int group = threadIdx.x % kGroups, at = q0 + group * 16, part = threadIdx.x / kGroups, parts = THREADS / kGroups;
        if (at < a.nq) {
            uint32_t found = 0;
            if (TOKENS) {
                const uint32_t *marks = a.marks + (int64_t)(at / 16) * a.marks_row;
                for (int i = part; i < a.marks_row; i += parts) found |= marks[i];
            } else {
                const uint32_t *marks = a.marks + at / a.marks_block;
                for (int i = first_token / 16 + part; i < (end_token + 15) / 16; i += parts) found |= marks[(int64_t)i * a.marks_row];
                found = found >> 16 * half & 0xFFFF ? 0xFFFF : 0;
            }
            if (found) atomicOr(shared + group, found);
        }
        __syncthreads();
    }
    __device__ __forceinline__ bool as_it_is(int row, int part) const { return groups[row / 16] >> (row % 16 + 16 * part) & 1; }
};

// DIRECT: operands lie on 16-byte boundaries in whole units and go straight to LDS.  The backward pass sees to that, with copies
// in its workspace where need be; the forward pass, which has none, takes other rows through registers.
template <typename T, ProductKind KIND, typename Tile, bool DIRECT>
__global__ __launch_bounds__(Tile::kThreads) void product_kernel(const ProductArgs a) {
    constexpr bool kPair = KIND == ProductKind::kForward || KIND == ProductKind::kGates;
    static_assert(DIRECT || KIND == ProductKind::kForward);
    constexpr int GP = Tile::GP, GQ = Tile::GQ;
    constexpr int kRun = kPair ? GP / 2 : 1;
    typedef Operand<T, Tile::P, !kPair, kPair, kRun, Tile::kThreads> OperandP;
    typedef Operand<T, Tile::Q, KIND == ProductKind::kGradWeights, false, 1, Tile::kThreads> OperandQ;
    constexpr int kStep = OperandP::kStep, kStage = OperandP::kBytes + OperandQ::kBytes;
    __shared__ __align__(256) unsigned char stages[Tile::kLds];
    const ProductWork work = product_work(a);
    if (!work.any) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wp = wave % Tile::WP, wq = wave / Tile::WP;
    // a pair's tile holds P / 2 units of either weight
    const int p0 = work.p * (kPair ? Tile::P / 2 : Tile::P), q0 = work.q * Tile::Q;
    const int first = work.split * a.split_steps, last = min(first + a.split_steps, a.steps);
    const int part_steps = KIND == ProductKind::kGradX ? a.steps / 2 : a.steps;      // kGradX goes through both halves
    const auto places_of = [&](int step) {
        return a.nk - (KIND == ProductKind::kGradX && step >= part_steps ? step - part_steps : step) * kStep;
    };

    // Which of the lane's loads of Q, i, and of its results' rows, j, are as they are: bits i + 4 part and 8 + j + 8 part; the others are
    // times kScale.
    uint32_t unscaled = 0;
    static_assert(OperandQ::kLoads <= 4 && GQ <= 8);
    constexpr bool kUndo = kScaled<T, KIND> && !kPair;
    if constexpr (kUndo) {
        constexpr bool kTokens = KIND == ProductKind::kGradX;
        const Marks<Tile::Q, Tile::kThreads> marks(a, std::integral_constant<bool, kTokens>{}, q0, work.half, first * kStep,
                                                   min(last * kStep, a.nk), (uint32_t *)stages);
#pragma unroll
        for (int part = 0; part < (kTokens ? 2 : 1); ++part) {
            for (int i = 0; i < OperandQ::kLoads; ++i)
                unscaled |= (uint32_t)marks.as_it_is(kTokens ? OperandQ::row_of(i) : OperandQ::unit_of(i) * OperandQ::E, part) << (i + 4 * part);
            for (int j = 0; j < GQ; ++j) unscaled |= (uint32_t)marks.as_it_is((wq * GQ + j) * 16 + lane % 16, part) << (8 + j + 8 * part);
        }
        __syncthreads();                                   // the first stage comes to the marks' place
    }
    const auto scale_of = [&](int j, int part) { return unscaled >> (8 + j + 8 * part) & 1 ? 1.f : kScale; };
    // Before use, or the compiler keeps all that follows from the bits in registers, through the main loop.
    const auto use_bits = [&] { asm volatile("" : "+v"(unscaled)); };

    f4 acc[GP][GQ] = {};
    const uint32_t base_p = OperandP::lane_base(), base_q = OperandQ::lane_base();
    // Half h of a step of P, and a half of its rows of Q, in registers.
    u4 ps[2][GP], qs[2][GQ / 2];
    const auto read_p = [&](u4 (&x)[GP], const unsigned char *stage, int h) {
#pragma unroll
        for (int i = 0; i < GP; ++i) {
            // a pair's wavefront takes the same units of either weight
            const int at = kPair ? wp * kRun * 16 + i % kRun * 4 + i / kRun * (Tile::P / 2) : (wp * GP + i) * 16;
            x[i] = OperandP::read(stage, base_p, at, h);
        }
    };
    const auto read_q = [&](u4 (&x)[GQ / 2], const unsigned char *stage, int h, int part) {
#pragma unroll
        for (int j = 0; j < GQ / 2; ++j) x[j] = OperandQ::read(stage + OperandP::kBytes, base_q, (wq * GQ + part * (GQ / 2) + j) * 16, h);
    };
    const auto multiply = [&](const u4 (&p)[GP], const u4 (&q)[GQ / 2], int part) {
#pragma unroll
        for (int i = 0; i < GP; ++i)
#pragma unroll
            for (int j = 0; j < GQ / 2; ++j) acc[i][part * (GQ / 2) + j] = multiply_units<T>(p[i], q[j], acc[i][part * (GQ / 2) + j]);
    };

    if constexpr (DIRECT) {
        OperandP p;
        OperandQ q;
        const auto copy_offset = [&](int i, int part) { return unscaled >> (i + 4 * part) & 1 ? 0u : a.d_width * (uint32_t)sizeof(T); };
        const auto begin = [&](int step) {
            const int part = KIND == ProductKind::kGradX && step >= part_steps, k = (step - part * part_steps) * kStep;
            if constexpr (kPair) p.begin_rows(a.p, k, p0, a.np);
            else p.begin_down(a.p[part], k, p0, a.p_units);
            const Rows &y = a.q[KIND == ProductKind::kGradX ? part : work.half];
            if constexpr (KIND == ProductKind::kGradWeights) q.begin_down(y, k, q0, a.d_width);
            else q.begin_rows(&y, k, q0, a.nq);
            if constexpr (kUndo) {
#pragma unroll
                for (int i = 0; i < OperandQ::kLoads; ++i) q.offset[i] += copy_offset(i, part);
            }
        };
        const auto start = [&](int step) {                 // begin(step - 1) or start(step - 1) was before
            if (KIND == ProductKind::kGradX && step == part_steps && step > first) {
                p.begin_down(a.p[1], 0, p0, a.p_units);
                q.begin_at(a.q + 1, 0, q0);                // d_up's rows are as far apart as d_gate's
                if constexpr (kUndo) {
                    use_bits();
#pragma unroll
                    for (int i = 0; i < OperandQ::kLoads; ++i) q.offset[i] += copy_offset(i, 1) - copy_offset(i, 0);
                }
            } else if (step > first) {
                p.advance(KIND == ProductKind::kGradX && step > part_steps ? a.p[1].stride : a.p[0].stride);
                q.advance(a.q[0].stride);
            }
            unsigned char *stage = stages + ((step - first) & 1) * kStage;
            p.start(stage, places_of(step));
            q.start(stage + OperandP::kBytes, places_of(step));
        };
        // A quarter of a step is read while the one before is multiplied.  The barrier lies before the last quarter, all of whose
        // operands are in registers by then, so that the next step's first reads have products to run under.  A CU takes loads at
        // 64 bytes a cycle, and wavefronts that start theirs stand still until they are taken: where a workgroup has two wavefronts
        // on each SIMD, one starts them before its last quarter and the other behind it, so that one of them multiplies (8192
        // tokens, 8192 channels, 2048 hidden units, bfloat16: 1253 us for the gradients, 1309 with both before, 1284 with both
        // behind, 1378 with the loads one by one between the products).
        const bool starts_late = Tile::kThreads == 512 && __builtin_amdgcn_readfirstlane((int)threadIdx.x) >= 256;
        if (first < last) {
            begin(first);
            start(first);
            wait_for_stage();
            if (first + 1 < last) start(first + 1);
            read_p(ps[0], stages, 0);
            read_q(qs[0], stages, 0, 0);
            for (int step = first; step < last; ++step) {
                const unsigned char *now = stages + ((step - first) & 1) * kStage, *next = stages + ((step - first + 1) & 1) * kStage;
                if constexpr (kUndo && KIND == ProductKind::kGradX)
                    if (step == part_steps) {              // sums over d_gate go on with d_up, which may have another scale
                        use_bits();
#pragma unroll
                        for (int j = 0; j < GQ; ++j) {
                            const float change = scale_of(j, 1) / scale_of(j, 0);
#pragma unroll
                            for (int i = 0; i < GP; ++i) acc[i][j] *= change;
                        }
                    }
                read_q(qs[1], now, 0, 1);
                multiply(ps[0], qs[0], 0);
                read_p(ps[1], now, 1);
                read_q(qs[0], now, 1, 0);
                multiply(ps[0], qs[1], 1);
                read_q(qs[1], now, 1, 1);
                multiply(ps[1], qs[0], 0);
                if (step + 1 < last) {
                    wait_for_stage();
                    read_p(ps[0], next, 0);
                    read_q(qs[0], next, 0, 0);
                    if (step + 2 < last && !starts_late) start(step + 2);
                }
                multiply(ps[1], qs[1], 1);
                if (step + 2 < last && starts_late) {
                    __builtin_amdgcn_sched_barrier(0);
                    start(step + 2);
                }
            }
        }
    } else {
        LooseRows<OperandP, T> p;
        LooseRows<OperandQ, T> q;
        p.begin_rows(a.p, 0, p0, a.np);
        q.begin_rows(a.q, 0, q0, a.nq);
        p.fetch(places_of(0));
        q.fetch(places_of(0));
        for (int step = 0; step < last; ++step) {
            unsigned char *stage = stages + (step & 1) * kStage;
            p.keep(stage);
            q.keep(stage + OperandP::kBytes);
            __syncthreads();
            if (step + 1 < last) {
                p.advance();
                q.advance();
                p.fetch(places_of(step + 1));
                q.fetch(places_of(step + 1));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_p(ps[0], stage, h);
                read_q(qs[0], stage, h, 0);
                read_q(qs[1], stage, h, 1);
                multiply(ps[0], qs[0], 0);
                multiply(ps[0], qs[1], 1);
            }
        }
    }

    if constexpr (kPair) {
        // lane: row lane % 16 and hidden units 4 kRun (lane / 16) + 0, 1, ... of what the wavefront has; whole tiles without branches,
        // so that all of grad_out is on its way at once
        constexpr bool kBackward = KIND == ProductKind::kGates;
        const int h = p0 + wp * kRun * 16 + lane / 16 * 4 * kRun, row0 = q0 + wq * GQ * 16 + lane % 16;
        const auto finish = [&](auto whole, auto past_caches) {
            constexpr bool kWhole = decltype(whole)::value;
            const int left = kWhole ? 4 * kRun : a.np - h;
            GatedEnd<T, kBackward, 4 * kRun> end[GQ];
#pragma unroll
            for (int j = 0; j < GQ; ++j)
                if (kWhole || row0 + j * 16 < a.nq) end[j].load(a, row0 + j * 16, h, left);
#pragma unroll
            for (int j = 0; j < GQ; ++j) {
                f4 g[kRun], u[kRun];
#pragma unroll
                for (int i = 0; i < kRun; ++i) g[i] = acc[i][j], u[i] = acc[i + kRun][j];
                const bool there = kWhole || row0 + j * 16 < a.nq;
                if (there || kScaled<T, KIND>) end[j].template finish<decltype(past_caches)::value>(a, row0 + j * 16, there, h, left, g, u);
            }
        };
        if (p0 + Tile::P / 2 > a.np || q0 + Tile::Q > a.nq) finish(std::false_type{}, std::false_type{});
        else if (!kBackward && a.past_caches) finish(std::true_type{}, std::true_type{});
        else finish(std::true_type{}, std::false_type{});
    } else {
        // lane: row lane % 16 and elements 4 (lane / 16) + 0..3 of each group
        if constexpr (kUndo) use_bits();
#pragma unroll
        for (int j = 0; j < GQ; ++j) {
            const int row = q0 + (wq * GQ + j) * 16 + lane % 16;
            if (row >= a.nq) continue;
            if constexpr (kUndo) {
                const float undo = 1.f / scale_of(j, KIND == ProductKind::kGradX && last > part_steps);
#pragma unroll
                for (int i = 0; i < GP; ++i) acc[i][j] *= undo;
            }
#pragma unroll
            for (int i = 0; i < GP; ++i) {
                const int e = p0 + (wp * GP + i) * 16 + lane / 16 * 4;
                if (a.splits > 1) {
                    float *to = a.partials + (((uint64_t)work.split * a.halves + work.half) * a.nq + row) * a.np + e;
                    store_four(to, acc[i][j], a.np - e);
                } else {
                    const Rows &y = a.out[work.half];
                    store_four((T *)y.data + (int64_t)row * y.stride + e, acc[i][j], a.np - e);
                }
            }
        }
    }
}

struct AlignArgs {
    Rows from[3], to[3];                   // to: rows of whole units
    uint64_t rows[3], first_unit[4];       // first_unit: units of the tensors before
    int32_t channels, units;               // units of a row
    uint32_t first_block;
};

// Rows at any alignment and of any length into rows of whole 16-byte units, zeros behind their end.
template <typename T> __global__ __launch_bounds__(256) void align_rows_kernel(const AlignArgs a) {
    constexpr int E = 16 / sizeof(T);
    typedef T vec_t __attribute__((ext_vector_type(E)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    uint64_t unit = ((uint64_t)a.first_block + blockIdx.x) * 256 + threadIdx.x;
    if (unit >= a.first_unit[3]) return;
    const int which = unit >= a.first_unit[2] ? 2 : unit >= a.first_unit[1] ? 1 : 0;
    unit -= a.first_unit[which];
    const uint64_t row = unit / a.units;
    const int at = (int)(unit - row * a.units) * E;
    const Rows &x = a.from[which], &y = a.to[which];
    const T *from = (const T *)x.data + (int64_t)row * x.stride;
    vec_t v = {};
    if (at + E <= a.channels) {
        v = *(const loose_t *)(from + at);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at + e < a.channels) v[e] = from[at + e];
    }
    *(vec_t *)((T *)y.data + (int64_t)row * y.stride + at) = v;
}

struct ProductSumArgs {
    const float *partials;                 // [splits][halves][rows][channels]
    Rows out[2];
    uint64_t slots;                        // halves * rows * channels
    uint32_t rows, channels, splits;
    uint32_t first_block;
};

// The splits of a sum, in their order.
template <typename T> __global__ __launch_bounds__(256) void product_sum_kernel(const ProductSumArgs a) {
    const uint64_t slot = ((uint64_t)a.first_block + blockIdx.x) * 1024 + threadIdx.x * 4;
    if (slot >= a.slots) return;
    const int there = (int)min(a.slots - slot, (uint64_t)4);
    f4 sum = {};
    for (uint32_t s = 0; s < a.splits; ++s) {
        Run<float, 4> part;
        part.load(a.partials + s * a.slots + slot, there);
        sum += part.v;
    }
    uint64_t row = slot / a.channels;
    uint32_t e = (uint32_t)(slot - row * a.channels);
    for (int i = 0; i < there; ++i) {
        const Rows &y = a.out[row >= a.rows];
        ((T *)y.data)[(int64_t)(row >= a.rows ? row - a.rows : row) * y.stride + e] = (T)sum[i];
        if (++e == a.channels) {
            e = 0;
            ++row;
        }
    }
}

// ---- few tokens ------------------------------------------------------------------

// 16 hidden units of both weights to a workgroup, for up to 16 NT tokens: the weights' bytes bound it, so they go from memory to
// the matrix units' registers once, with no stage between, and the wavefronts share the channels and join their sums in LDS.
// 1 token, 2048 channels, 5632 hidden units: 46 MB in bfloat16 in 15.6 us from memory, in 14.0 where the last-level cache holds them, 92 MB
// in float32 in 28.1; 4 or 16 wavefronts, and twice as many products at once, change that by less than 5 %.
template <typename T, int NT, bool BACKWARD, bool DIRECT>
__global__ __launch_bounds__(512) void gated_few_kernel(const ProductArgs a) {
    constexpr int E = 16 / sizeof(T), kStep = 4 * E;       // channels of one product: 32 of 16 bits, 16 of 32
    extern __shared__ __align__(16) unsigned char lds[];
    typedef T vec_t __attribute__((ext_vector_type(E)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int h0 = (int)(a.first_block + blockIdx.x) * 16, h = min(h0 + lane % 16, a.np - 1);
    const T *gate = (const T *)a.p[0].data + h * a.p[0].stride, *up = (const T *)a.p[1].data + h * a.p[1].stride;
    const T *x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = (const T *)a.q[0].data + (int64_t)min(t * 16 + lane % 16, a.nq - 1) * a.q[0].stride;
    const auto load = [&](const T *row, int k) -> u4 {
        vec_t v = {};
        if (k + E <= a.nk) {
            if (DIRECT) v = *(const vec_t *)(row + k);
            else v = *(const loose_t *)(row + k);
        } else if (!DIRECT) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k + e < a.nk) v[e] = row[k + e];
        }
        return __builtin_bit_cast(u4, v);
    };
    f4 g[NT] = {}, u[NT] = {};
    constexpr int kAtOnce = NT > 2 ? 2 : 4;                // products whose loads are under way together
    for (int k0 = wave * kAtOnce * kStep; k0 < a.nk; k0 += waves * kAtOnce * kStep) {
        u4 gs[kAtOnce], us[kAtOnce], xs[kAtOnce][NT];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int k = k0 + i * kStep + lane / 16 * E;
            gs[i] = load(gate, k);
            us[i] = load(up, k);
#pragma unroll
            for (int t = 0; t < NT; ++t) xs[i][t] = load(x[t], k);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                g[t] = multiply_units<T>(gs[i], xs[i][t], g[t]);
                u[t] = multiply_units<T>(us[i], xs[i][t], u[t]);
            }
    }
    f4 *sums = (f4 *)lds;                                  // [wavefronts][NT][2][64]
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        sums[((wave * NT + t) * 2 + 0) * 64 + lane] = g[t];
        sums[((wave * NT + t) * 2 + 1) * 64 + lane] = u[t];
    }
    __syncthreads();
    for (int t = wave; t < NT; t += waves) {
        f4 gs = {}, us = {};
        for (int w = 0; w < waves; ++w) {
            gs += sums[((w * NT + t) * 2 + 0) * 64 + lane];
            us += sums[((w * NT + t) * 2 + 1) * 64 + lane];
        }
        const int token = t * 16 + lane % 16, at = h0 + lane / 16 * 4;
        GatedEnd<T, BACKWARD, 4> end;
        const bool there = token < a.nq;
        if (there) end.load(a, token, at, a.np - at);
        if (there || end.kTwice) end.finish(a, token, there, at, a.np - at, {gs}, {us});
    }
}

}  // namespace iso
