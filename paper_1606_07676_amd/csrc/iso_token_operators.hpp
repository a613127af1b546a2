// Host side of the operators on each token by itself (layer norm, dropout, gated projections): argument checks, the choice of
// kernels and the launches of a request.
#pragma once

#include "iso_dropout_kernels.hpp"
#include "iso_gated_kernels.hpp"
#include "iso_norm_kernels.hpp"
#include "iso_operators.hpp"

#include <numeric>

namespace iso {

inline int check_dtype(int dtype) {
    return dtype == ISO_DTYPE_F32 || dtype == ISO_DTYPE_BF16 || dtype == ISO_DTYPE_F16 ? ISO_SUCCESS : ISO_ERR_ARG;
}
inline bool same_rows(const iso_heads_t &a, const iso_heads_t &b) {
    return a.data == b.data && a.rank_stride == b.rank_stride && a.head_stride == b.head_stride;
}
inline bool same_rows(const iso_rows_t &a, const iso_rows_t &b) { return a.data == b.data && a.stride == b.stride; }
inline iso_heads_t one_head(const iso_rows_t &t) { return iso_heads_t{t.data, t.stride, 0}; }
inline bool wide(const iso_rows_t &t, int elements, int dtype) { return wide(one_head(t), elements, dtype); }
// Rows of whole 128-byte lines: they may be stored past the caches, where others would be written to memory in pieces (norm of
// 100000 x 3 heads of 72 in bfloat16, 22.9 us in place of 21.2; 100000 x 232 21.1 and 20.9).
inline bool whole_lines(const iso_heads_t &t, int elements, int dtype) {
    const uint64_t size = dtype_size(dtype);
    return (((uintptr_t)t.data | (uint64_t)t.rank_stride * size | (uint64_t)t.head_stride * size | (uint64_t)elements * size) & 127) == 0;
}

// ---- layer norm --------------------------------------------------------------------

// How lanes share a row: 8 lanes or more, with as many units each as a lane may hold where that leaves 8.
struct NormShape {
    int units, per_lane, lanes;            // units of a row, of a lane (1, 2 or 4), lanes of a row
    bool whole;                            // a row takes a workgroup
    uint64_t groups() const { return whole ? 1 : 256 / lanes; }        // rows of a workgroup at a time
    uint32_t threads() const { return whole ? (uint32_t)lanes : 256u; }
};
inline NormShape norm_shape(int channels, int dtype) {
    const int E = dtype == ISO_DTYPE_F32 ? 4 : 8, most = kNormLaneElements / E;
    NormShape s{(channels + E - 1) / E, 1, 8, false};
    while (s.per_lane < most && s.lanes * s.per_lane < s.units) s.per_lane *= 2;
    while (s.lanes * s.per_lane < s.units) s.lanes *= 2;
    s.whole = s.lanes > 64;
    return s;
}
// Workgroups that together take whole tokens' rows at a time, so that a lane keeps its head: as many as have the threads of `most`
// of 256 at most, but those of one token's rows at least.
inline uint64_t norm_unit(const NormShape &s, uint64_t heads) { return heads / std::gcd(heads, s.groups()); }
inline uint64_t norm_need(const NormShape &s, uint64_t rows) { return std::max<uint64_t>(1, (rows + s.groups() - 1) / s.groups()); }
inline uint64_t norm_limit(const NormShape &s, uint64_t most) { return std::max<uint64_t>(1, most * 256 / s.threads()); }
inline uint64_t norm_workgroups(const NormShape &s, uint64_t rows, uint64_t heads, uint64_t most) {
    const uint64_t unit = norm_unit(s, heads);
    return std::min((norm_need(s, rows) + unit - 1) / unit, std::max<uint64_t>(1, norm_limit(s, most) / unit)) * unit;
}
// Of 256 threads.  Norms with 3, 6, 8 and 12 for each CU, inputs from memory, us: 32768 x 1024 in bfloat16 26.1, 25.9, 25.8, 25.6;
// 70000 x 512 in float32 50.8, 51.0, 51.3, 49.9; 262144 x 10 heads of 128 265, 254, 261, 251.  Gradients with 256, 512, 768, 1024 parts:
// 32768 x 1024 in bfloat16 42.7, 43.5, 44.6, 50.3 (a CU holds 3 workgroups); 37271 x 483 in float16 31.7, 30.6, 31.0, 36.3; 70000 x 512
// in float32 78.7, 81.6, 83.1, 83.5; 100000 x 16 heads of 64 160, 113, 118, 122.
constexpr uint64_t kNormWorkgroups = 12 * 256, kNormParts = 512;
// Workgroups of a gradient that sums over rows, each of which leaves a part of the sums.  Where one token's rows take more than the
// limit, lanes move from head to head instead: 64 x 4099 heads of 128 in bfloat16 39.0 us with 512 parts, with 4099 59.7.
inline bool norm_moves(const NormShape &s, uint64_t heads) { return norm_unit(s, heads) > norm_limit(s, kNormParts); }
inline uint64_t norm_parts(const NormShape &s, uint64_t rows, uint64_t heads) {
    return norm_moves(s, heads) ? std::min(norm_need(s, rows), norm_limit(s, kNormParts)) : norm_workgroups(s, rows, heads, kNormParts);
}

inline int check_norm(int64_t n, int heads, int channels, int dtype) {
    ISO_TRY(check_dtype(dtype));
    if (n < 0 || heads < 1 || channels < 1) return ISO_ERR_ARG;
    if (channels > kNormMaxChannels || heads > 65536 || n > 0xFFFFFFFFll / heads) return ISO_ERR_TOO_LARGE;
    return ISO_SUCCESS;
}
inline uint64_t norm_workspace(int64_t n, int heads, int channels, int dtype) {
    return norm_parts(norm_shape(channels, dtype), (uint64_t)n * heads, heads) * 2 * channels * 4;
}

enum class NormPass { kForward, kBackward, kSums, kMovingSums };
template <typename T, bool WIDE, int U, int LANES> const void *norm_kernel(NormPass pass) {
    switch (pass) {
        case NormPass::kForward: return (const void *)(layer_norm_kernel<T, WIDE, U, LANES>);
        case NormPass::kBackward: return (const void *)(layer_norm_backward_kernel<T, WIDE, U, LANES, false, false>);
        case NormPass::kSums: return (const void *)(layer_norm_backward_kernel<T, WIDE, U, LANES, true, false>);
        default: return (const void *)(layer_norm_backward_kernel<T, WIDE, U, LANES, true, true>);
    }
}
template <typename T, bool WIDE> const void *norm_kernel(const NormShape &s, NormPass pass) {
    constexpr int kMost = kNormLaneElements * (int)sizeof(T) / 16;
    if (s.whole) return norm_kernel<T, WIDE, kMost, 0>(pass);
    switch (s.lanes) {
        case 64: return norm_kernel<T, WIDE, kMost, 64>(pass);
        case 32: return norm_kernel<T, WIDE, kMost, 32>(pass);
        case 16: return norm_kernel<T, WIDE, kMost, 16>(pass);
    }
    if (s.per_lane == 1) return norm_kernel<T, WIDE, 1, 8>(pass);
    if constexpr (kMost == 4)
        if (s.per_lane == 4) return norm_kernel<T, WIDE, 4, 8>(pass);
    return norm_kernel<T, WIDE, 2, 8>(pass);
}
inline const void *norm_kernel(int dtype, bool is_wide, const NormShape &s, NormPass pass) {
    switch (dtype) {
        case ISO_DTYPE_F32: return is_wide ? norm_kernel<float, true>(s, pass) : norm_kernel<float, false>(s, pass);
        case ISO_DTYPE_BF16: return is_wide ? norm_kernel<__bf16, true>(s, pass) : norm_kernel<__bf16, false>(s, pass);
        default: return is_wide ? norm_kernel<_Float16, true>(s, pass) : norm_kernel<_Float16, false>(s, pass);
    }
}

inline int bind_layer_norm(BoundOperator &b, const iso_layer_norm_t &t, const iso_layer_norm_grads_t *g, void *workspace,
                           size_t workspace_bytes) {
    ISO_TRY(check_norm(t.n, t.heads, t.channels, t.dtype));
    if (!g && !(t.eps >= 0.f && t.eps <= 3.4e38f)) return ISO_ERR_ARG;
    if (g && t.n && (!t.mean || !t.rstd)) return ISO_ERR_ARG;
    if (g && g->grad_weight && !t.weight) return ISO_ERR_ARG;
    const uint64_t n = (uint64_t)t.n, rows = n * t.heads, size = dtype_size(t.dtype), row_bytes = t.channels * size;
    const bool sums = g && (g->grad_weight || g->grad_bias);
    const uint64_t work = sums ? norm_workspace(t.n, t.heads, t.channels, t.dtype) : 0;
    const iso_heads_t &in = g ? g->grad_out : t.x, &out = g ? g->grad_x : t.out;       // may be the same rows
    Regions r;
    ISO_TRY(r.heads(out, n, t.heads, t.channels, t.dtype, true));
    if (g || !same_rows(in, out)) ISO_TRY(r.heads(t.x, n, t.heads, t.channels, t.dtype, false));
    if (g && !same_rows(in, out)) ISO_TRY(r.heads(in, n, t.heads, t.channels, t.dtype, false));
    if (t.weight) ISO_TRY(r.array(t.weight, row_bytes, size, false));
    if (t.bias && !g) ISO_TRY(r.array(t.bias, row_bytes, size, false));
    if (t.mean) ISO_TRY(r.array(t.mean, rows * 4, 4, !g));
    if (t.rstd) ISO_TRY(r.array(t.rstd, rows * 4, 4, !g));
    if (sums) {
        if (g->grad_weight) ISO_TRY(r.array(g->grad_weight, row_bytes, size, true));
        if (g->grad_bias) ISO_TRY(r.array(g->grad_bias, row_bytes, size, true));
        if (!workspace || workspace_bytes < work) return ISO_ERR_WORKSPACE;
        ISO_TRY(r.array(workspace, work, 4, true));
    }
    ISO_TRY(r.disjoint());
    if (!rows && !sums) return ISO_SUCCESS;

    const NormShape s = norm_shape(t.channels, t.dtype);
    NormArgs a{};
    a.x = device_heads(t.x);
    a.out = device_heads(out);
    if (g) a.grad_out = device_heads(in);
    a.weight = t.weight;
    a.bias = t.bias;
    a.mean = t.mean;
    a.rstd = t.rstd;
    a.partials = (float *)workspace;
    a.rows = rows;
    a.heads = make_fastdiv((uint32_t)t.heads);
    a.channels = t.channels;
    a.units = s.units;
    a.eps = t.eps;
    a.inverse = 1.f / (float)t.channels;
    const auto at_16 = [](const void *p) { return ((uintptr_t)p & 15) == 0; };
    const bool is_wide = wide(t.x, t.channels, t.dtype) && wide(out, t.channels, t.dtype) && wide(in, t.channels, t.dtype) && at_16(t.weight) &&
                         (g || at_16(t.bias));
    a.past_caches = whole_lines(out, t.channels, t.dtype);
    const NormPass pass = !g ? NormPass::kForward : !sums ? NormPass::kBackward : norm_moves(s, t.heads) ? NormPass::kMovingSums : NormPass::kSums;
    const void *func = norm_kernel(t.dtype, is_wide, s, pass);
    const uint64_t workgroups = sums ? norm_parts(s, rows, t.heads) : norm_workgroups(s, rows, t.heads, kNormWorkgroups);
    a.step = workgroups * s.groups();
    a.token_step = a.step / t.heads;
    ISO_TRY(add_launch(b, func, workgroups, s.threads(), a, sums && !s.whole ? 4 * 2 * (size_t)t.channels * 4 : 0));
    if (!sums) return ISO_SUCCESS;
    NormSumArgs sum{};
    sum.partials = a.partials;
    sum.out[0] = g->grad_weight;
    sum.out[1] = g->grad_bias;
    sum.parts = (int32_t)workgroups;
    sum.channels = t.channels;
    const void *sum_func = t.dtype == ISO_DTYPE_F32 ? (const void *)(layer_norm_sum_kernel<float>)
                           : t.dtype == ISO_DTYPE_BF16 ? (const void *)(layer_norm_sum_kernel<__bf16>)
                                                       : (const void *)(layer_norm_sum_kernel<_Float16>);
    return add_launch(b, sum_func, (2 * (uint64_t)t.channels + 15) / 16, 1024, sum);
}

// ---- dropout -----------------------------------------------------------------------

template <bool RESIDUAL> struct Dropout {
    template <typename T, bool WIDE> struct Kernel {
        static const void *func() { return (const void *)(dropout_kernel<T, WIDE, RESIDUAL>); }
    };
};

inline int bind_dropout(BoundOperator &b, const iso_dropout_t &t) {
    ISO_TRY(check_dtype(t.dtype));
    if (t.n < 0 || t.channels < 1 || !(t.rate >= 0.f && t.rate <= 1.f)) return ISO_ERR_ARG;
    if (t.n > ((int64_t(1) << 34) - 1) / t.channels) return ISO_ERR_TOO_LARGE;
    const uint64_t n = (uint64_t)t.n, elements = n * t.channels;
    const bool residual = t.residual.data != nullptr;
    Regions r;
    ISO_TRY(r.heads(one_head(t.out), n, 1, t.channels, t.dtype, true));
    if (!same_rows(t.x, t.out)) ISO_TRY(r.heads(one_head(t.x), n, 1, t.channels, t.dtype, false));
    if (residual && !same_rows(t.residual, t.out)) ISO_TRY(r.heads(one_head(t.residual), n, 1, t.channels, t.dtype, false));
    if (n) ISO_TRY(r.array(t.seed, 16, 8, false));
    ISO_TRY(r.disjoint());
    if (!n) return ISO_SUCCESS;

    DropoutArgs a{};
    a.x = t.x.data;
    a.out = t.out.data;
    a.residual = t.residual.data;
    a.x_stride = t.x.stride;
    a.out_stride = t.out.stride;
    a.residual_stride = t.residual.stride;
    a.seed = t.seed;
    a.elements = elements;
    a.blocks = (uint32_t)((elements + 7) / 8);
    a.channels = (uint32_t)t.channels;
    a.row_blocks = make_fastdiv((uint32_t)std::max(1, t.channels / 8));
    const auto all = [&](auto &&ok) { return ok(t.x) && ok(t.out) && (!residual || ok(t.residual)); };
    a.flat = n == 1 || all([&](const iso_rows_t &x) { return x.stride == t.channels; });
    const bool is_wide = a.flat ? all([](const iso_rows_t &x) { return ((uintptr_t)x.data & 15) == 0; })
                                : t.channels % 8 == 0 && all([&](const iso_rows_t &x) { return wide(x, t.channels, t.dtype); });
    a.threshold = (uint32_t)std::floor((double)t.rate * 65536 + 0.5);
    a.scale = a.threshold < 65536 ? 65536.f / (float)(65536 - a.threshold) : 0.f;
    const void *func = residual ? by_type<Dropout<true>::Kernel>(t.dtype, is_wide) : by_type<Dropout<false>::Kernel>(t.dtype, is_wide);
    return add_launch(b, func, ((uint64_t)a.blocks + 255) / 256, 256, a);
}

// ---- gated projections ----------------------------------------------------------------

constexpr int kGatedMaxWidth = 1 << 20;
constexpr int kFewTokens = 64;

typedef ProductTile<4, 2, 4, 8> LargeTile;         // 256 x 256, 8 wavefronts
typedef ProductTile<2, 2, 4, 4> MiddleTile;        // 128 x 128, 4
typedef ProductTile<2, 2, 2, 2> SmallTile;         // 64 x 64, 4

// How a product is cut up.
struct ProductPlan {
    int tile;                              // 0 large, 1 middle, 2 small
    uint64_t p_tiles, q_tiles;
    int steps, splits, split_steps;
};

// Times in us, of a step of a tile that has its CU for itself, of one among as many as fit beside it, and of a tile's end.
struct TileTimes {
    double alone, among, end;
    int beside;
};

// np: elements of a result's row (of a pair: hidden units of one weight), nq: its rows, nk: the summed axis.
//
// The tile and the parts of the summed axis by the time that they would take: a CU works on its share of the tiles, step by step
// in the time of one alone or, side by side, of all; the sums of parts are written and read again at 5 TB/s.  Constants are those
// of 16 and 32 bits on the GPU.  Weights' gradients of 32768 tokens, 1024 channels, 2816 hidden units, bfloat16: large tiles in 2
// parts 370 and 11 us, in 5 389 together, in 1 715, middle ones in 1 524, small ones in 2 658 and 11; of 200000 tokens, 128
// channels, 384 hidden units small ones in 1 2300, in 6 384 and 4; grad_x of 300 tokens, 1024 channels, 2816 hidden units large ones
// in 1 117, small ones in 1 51, in 4 15 and 4.
inline ProductPlan plan_product(ProductKind kind, int dtype, uint64_t np, uint64_t nq, uint64_t nk) {
    static constexpr int kSize[3] = {LargeTile::P, MiddleTile::P, SmallTile::P};
    static constexpr TileTimes kTimes[2][3] = {{{1.40, 1.50, 7.0, 1}, {0.85, 0.51, 2.2, 2}, {0.70, 0.27, 0.7, 5}},
                                               {{0, 0, 0, 0}, {2.10, 1.88, 3.0, 2}, {0.74, 0.50, 1.0, 5}}};
    const bool pair = kind == ProductKind::kForward || kind == ProductKind::kGates, single = dtype == ISO_DTYPE_F32;
    const uint64_t halves = kind == ProductKind::kGradWeights ? 2 : 1;
    const int step = kStepBytes / (int)dtype_size(dtype);
    const int steps = (int)((nk + step - 1) / step) * (kind == ProductKind::kGradX ? 2 : 1);
    ProductPlan best{};
    double best_time = 0;
    for (int tile = single ? 1 : 0; tile < 3; ++tile) {
        const uint64_t width = pair ? kSize[tile] / 2 : kSize[tile];
        ProductPlan plan{tile, (np + width - 1) / width, (nq + kSize[tile] - 1) / kSize[tile], steps, 1, steps};
        const TileTimes &t = kTimes[single][tile];
        for (int splits = 1; splits == 1 || (!pair && splits <= std::min(256, steps / 8)); splits += 1 + splits / 8) {
            plan.split_steps = std::max(1, (steps + splits - 1) / splits);
            plan.splits = std::max(1, (steps + plan.split_steps - 1) / plan.split_steps);
            const uint64_t items = plan.p_tiles * plan.q_tiles * halves * plan.splits, share = (items + 255) / 256;
            double time = plan.split_steps * std::max(t.alone * (double)((share + t.beside - 1) / t.beside), t.among * (double)share) +
                          t.end * (double)share * (kind == ProductKind::kGates ? 2 : 1);
            if (plan.splits > 1) time += 5 + 2 * 4e-6 / 5 * (double)plan.splits * (double)(halves * np * nq);
            if (!best.p_tiles || time < best_time) {
                best = plan;
                best_time = time;
            }
        }
    }
    return best;
}

template <typename T, ProductKind KIND> const void *product_func(int tile, bool direct) {
    if constexpr (KIND == ProductKind::kForward)
        if (!direct) {
            if constexpr (sizeof(T) == 2)
                if (tile == 0) return (const void *)(product_kernel<T, KIND, LargeTile, false>);
            return tile <= 1 ? (const void *)(product_kernel<T, KIND, MiddleTile, false>) : (const void *)(product_kernel<T, KIND, SmallTile, false>);
        }
    if constexpr (sizeof(T) == 2)
        if (tile == 0) return (const void *)(product_kernel<T, KIND, LargeTile, true>);
    return tile <= 1 ? (const void *)(product_kernel<T, KIND, MiddleTile, true>) : (const void *)(product_kernel<T, KIND, SmallTile, true>);
}
template <ProductKind KIND> const void *product_func(int dtype, int tile, bool direct) {
    switch (dtype) {
        case ISO_DTYPE_F32: return product_func<float, KIND>(tile, direct);
        case ISO_DTYPE_BF16: return product_func<__bf16, KIND>(tile, direct);
        default: return product_func<_Float16, KIND>(tile, direct);
    }
}
template <typename T, bool BACKWARD> const void *few_func(int groups, bool direct) {
    if (groups == 1) return direct ? (const void *)(gated_few_kernel<T, 1, BACKWARD, true>) : (const void *)(gated_few_kernel<T, 1, BACKWARD, false>);
    if (groups == 2) return direct ? (const void *)(gated_few_kernel<T, 2, BACKWARD, true>) : (const void *)(gated_few_kernel<T, 2, BACKWARD, false>);
    return direct ? (const void *)(gated_few_kernel<T, 4, BACKWARD, true>) : (const void *)(gated_few_kernel<T, 4, BACKWARD, false>);
}
template <bool BACKWARD> const void *few_func(int dtype, int groups, bool direct) {
    switch (dtype) {
        case ISO_DTYPE_F32: return few_func<float, BACKWARD>(groups, direct);
        case ISO_DTYPE_BF16: return few_func<__bf16, BACKWARD>(groups, direct);
        default: return few_func<_Float16, BACKWARD>(groups, direct);
    }
}

inline int64_t whole_units(int elements) { return (elements + 7) / 8 * 8; }

// Offsets, each a multiple of 256 bytes: d_gate and d_up of all tokens, in float16 each row followed by its scaled copy, and the marks
// of which to take; copies of x, gate and up with aligned rows where theirs are not, the sums of splits.
struct GatedWorkspace {
    uint64_t d_gate = 0, d_up = 0, marks = 0, copies[3] = {}, partials = 0, bytes = 0;
};
constexpr int kMarkUnits = 16;             // hidden units of a mark at least
inline GatedWorkspace gated_workspace(int64_t n, int channels, int hidden, int dtype) {
    GatedWorkspace w;
    const auto take = [&](uint64_t rows, int width) {
        const uint64_t at = w.bytes;
        w.bytes += (rows * whole_units(width) * dtype_size(dtype) + 255) / 256 * 256;
        return at;
    };
    const uint64_t kept = dtype == ISO_DTYPE_F16 ? 2 : 1;
    w.d_gate = take(kept * n, hidden);
    w.d_up = take(kept * n, hidden);
    w.marks = w.bytes;
    if (dtype == ISO_DTYPE_F16) w.bytes += ((uint64_t)(n + 15) / 16 * ((hidden + kMarkUnits - 1) / kMarkUnits) * 4 + 255) / 256 * 256;
    w.copies[0] = take(n, channels);
    w.copies[1] = take(n ? hidden : 0, channels);
    w.copies[2] = take(n ? hidden : 0, channels);
    w.partials = w.bytes;
    const ProductPlan x = plan_product(ProductKind::kGradX, dtype, channels, n, hidden);
    const ProductPlan weights = plan_product(ProductKind::kGradWeights, dtype, channels, hidden, n);
    if (x.splits > 1) w.bytes += (uint64_t)x.splits * n * channels * 4;
    if (weights.splits > 1) w.bytes = std::max(w.bytes, w.partials + (uint64_t)weights.splits * 2 * hidden * channels * 4);
    return w;
}
inline int check_gated(int64_t n, int channels, int hidden, int dtype) {
    ISO_TRY(check_dtype(dtype));
    if (n < 0 || channels < 1 || hidden < 1) return ISO_ERR_ARG;
    if (channels > kGatedMaxWidth || hidden > kGatedMaxWidth || n >= 1 << 30) return ISO_ERR_TOO_LARGE;
    return ISO_SUCCESS;
}

class GatedBinder {
  public:
    GatedBinder(BoundOperator &out, const iso_gated_t &gated, const iso_gated_grads_t *grads) : b(out), t(gated), g(grads) {}

    int bind(void *workspace, size_t workspace_bytes) {
        ISO_TRY(check_gated(t.n, t.channels, t.hidden, t.dtype));
        if (t.activation != ISO_ACTIVATION_SILU && t.activation != ISO_ACTIVATION_GELU) return ISO_ERR_ARG;
        ISO_TRY(check_buffers(workspace, workspace_bytes));
        return g ? backward((char *)workspace) : forward();
    }

  private:
    int check_buffers(void *workspace, size_t workspace_bytes) {
        Regions r;
        const uint64_t n = (uint64_t)t.n, hidden = (uint64_t)t.hidden;
        const auto rows = [&](const iso_rows_t &x, uint64_t count, int width, bool written) {
            return r.heads(one_head(x), count, 1, width, t.dtype, written);
        };
        ISO_TRY(rows(t.x, n, t.channels, false));
        ISO_TRY(rows(t.gate, n ? hidden : 0, t.channels, false));
        ISO_TRY(rows(t.up, n ? hidden : 0, t.channels, false));
        if (!g) {
            ISO_TRY(rows(t.out, n, t.hidden, true));
            return r.disjoint();
        }
        ISO_TRY(rows(g->grad_out, n, t.hidden, false));
        ISO_TRY(rows(g->grad_x, n, t.channels, true));
        ISO_TRY(rows(g->grad_gate, hidden, t.channels, true));
        ISO_TRY(rows(g->grad_up, hidden, t.channels, true));
        work = gated_workspace(t.n, t.channels, t.hidden, t.dtype);
        if (work.bytes && (!workspace || workspace_bytes < work.bytes)) return ISO_ERR_WORKSPACE;
        ISO_TRY(r.array(workspace, work.bytes, 16, true));
        return r.disjoint();
    }

    static Rows device_rows(const iso_rows_t &x) { return Rows{x.data, x.stride}; }

    int add_product(ProductKind kind, const void *func(int, int, bool), bool direct, ProductArgs a, void *partials) {
        const ProductPlan plan = plan_product(kind, t.dtype, a.np, a.nq, a.nk);
        a.halves = kind == ProductKind::kGradWeights ? 2 : 1;
        a.steps = plan.steps;
        a.splits = plan.splits;
        a.split_steps = plan.split_steps;
        a.p_tiles = (uint32_t)plan.p_tiles;
        a.q_tiles = (uint32_t)plan.q_tiles;
        const uint64_t tiles = plan.p_tiles * plan.q_tiles * a.halves, items = tiles * plan.splits;
        if (items > 0x7FFFFFF0ull) return ISO_ERR_TOO_LARGE;
        a.tiles = make_fastdiv((uint32_t)tiles);
        a.band_items = make_fastdiv((uint32_t)plan.p_tiles * kBand);
        a.items = (uint32_t)items;
        a.per_xcd = (uint32_t)((items + 7) / 8);
        a.partials = (float *)partials;
        a.activation = t.activation;
        ISO_TRY(add_launch(b, func(t.dtype, plan.tile, direct), (uint64_t)a.per_xcd * 8, plan.tile == 0 ? LargeTile::kThreads : 256, a));
        if (plan.splits == 1) return ISO_SUCCESS;
        ProductSumArgs s{};
        s.partials = a.partials;
        s.out[0] = a.out[0];
        s.out[1] = a.out[1];
        s.slots = (uint64_t)a.halves * a.nq * a.np;
        s.rows = (uint32_t)a.nq;
        s.channels = (uint32_t)a.np;
        s.splits = (uint32_t)plan.splits;
        const void *sum_func = t.dtype == ISO_DTYPE_F32 ? (const void *)(product_sum_kernel<float>)
                               : t.dtype == ISO_DTYPE_BF16 ? (const void *)(product_sum_kernel<__bf16>)
                                                           : (const void *)(product_sum_kernel<_Float16>);
        return add_launch(b, sum_func, (s.slots + 1023) / 1024, 256, s);
    }

    int32_t units_end() const {                // of a row's elements, in whole units
        const int E = 16 / (int)dtype_size(t.dtype);
        return (t.channels + E - 1) / E * E;
    }
    // Rows that the products take straight from memory: on 16-byte boundaries, in whole units, fewer than 2^24 bytes apart.
    bool direct(const iso_rows_t &x) const {
        return wide(x, t.channels, t.dtype) && x.stride * (int64_t)dtype_size(t.dtype) < (1 << 24);
    }

    // g and u of all tokens, up to out or to d_gate and d_up.
    template <bool BACKWARD> int add_projections(ProductArgs a) {
        a.np = t.hidden;
        a.nq = (int32_t)t.n;
        a.nk = t.channels;
        if (t.n <= kFewTokens) {
            const bool aligned = direct(t.gate) && direct(t.up) && direct(t.x);
            const int groups = t.n <= 16 ? 1 : t.n <= 32 ? 2 : 4;
            a.p[0] = device_rows(t.gate);
            a.p[1] = device_rows(t.up);
            a.q[0] = device_rows(t.x);
            a.activation = t.activation;
            return add_launch(b, few_func<BACKWARD>(t.dtype, groups, aligned), ((uint64_t)t.hidden + 15) / 16, 512, a, (size_t)groups << 14);
        }
        a.p[0] = gate;
        a.p[1] = up;
        a.q[0] = x;
        constexpr ProductKind kind = BACKWARD ? ProductKind::kGates : ProductKind::kForward;
        return add_product(kind, product_func<kind>, BACKWARD || (direct(t.gate) && direct(t.up) && direct(t.x)), a, nullptr);
    }

    int forward() {
        if (!t.n) return ISO_SUCCESS;
        ProductArgs a{};
        x = device_rows(t.x);
        gate = device_rows(t.gate);
        up = device_rows(t.up);
        a.out[0] = device_rows(t.out);
        // What is stored past the caches leaves them to the operands: 32768 tokens, 1024 channels, 4096 hidden units, bfloat16, 468 us
        // in place of 492.  Not where a wavefront's 64 bytes of a row are parts of more lines: 117 became 122 us for 232 channels and
        // 2044 hidden units, though 499 became 488 for 1024 and 4092.
        a.past_caches = (((uintptr_t)t.out.data | (uint64_t)t.out.stride * dtype_size(t.dtype)) & 63) == 0;
        return add_projections<false>(a);
    }

    // The backward pass's products need rows on 16-byte boundaries in whole units: others are copied first.  2000 tokens, 2685
    // channels, 8192 hidden units, bfloat16: 0.60 ms in place of 2.2 with products that take such rows through registers.
    int align_rows(char *workspace) {
        AlignArgs a{};
        a.channels = t.channels;
        const int width = (int)whole_units(t.channels);
        a.units = width / (16 / (int)dtype_size(t.dtype));
        const iso_rows_t *const from[3] = {&t.x, &t.gate, &t.up};
        Rows *const to[3] = {&x, &gate, &up};
        for (int i = 0; i < 3; ++i) {
            *to[i] = device_rows(*from[i]);
            if (!direct(*from[i])) {
                a.from[i] = *to[i];
                a.to[i] = *to[i] = Rows{workspace + work.copies[i], width};
                a.rows[i] = i ? (uint64_t)t.hidden : (uint64_t)t.n;
            }
            a.first_unit[i + 1] = a.first_unit[i] + a.rows[i] * a.units;
        }
        if (!a.first_unit[3]) return ISO_SUCCESS;
        const void *func = t.dtype == ISO_DTYPE_F32 ? (const void *)(align_rows_kernel<float>)
                           : t.dtype == ISO_DTYPE_BF16 ? (const void *)(align_rows_kernel<__bf16>)
                                                       : (const void *)(align_rows_kernel<_Float16>);
        return add_launch(b, func, (a.first_unit[3] + 255) / 256, 256, a);
    }

    int backward(char *workspace) {
        const int64_t padded = whole_units(t.hidden), stride = t.dtype == ISO_DTYPE_F16 ? 2 * padded : padded;
        const Rows d_gate{workspace + work.d_gate, stride}, d_up{workspace + work.d_up, stride};
        void *partials = workspace + work.partials;
        ProductArgs kept{};
        kept.d_width = (int32_t)padded;
        kept.marks = (uint32_t *)(workspace + work.marks);
        // the hidden units that a wavefront of the kernel up to d_gate and d_up has, one set of 16 or two
        kept.marks_block = t.n <= kFewTokens || plan_product(ProductKind::kGates, t.dtype, t.hidden, t.n, t.channels).tile == 2 ? 16 : 32;
        kept.marks_row = (t.hidden + kept.marks_block - 1) / kept.marks_block;
        if (t.n) {
            ISO_TRY(align_rows(workspace));
            ProductArgs a = kept;
            a.out[0] = d_gate;
            a.out[1] = d_up;
            a.grad_out = device_rows(g->grad_out);
            ISO_TRY(add_projections<true>(a));
            a = kept;
            a.p[0] = gate;
            a.p[1] = up;
            a.q[0] = d_gate;
            a.q[1] = d_up;
            a.out[0] = device_rows(g->grad_x);
            a.np = t.channels;
            a.p_units = units_end();
            a.nq = (int32_t)t.n;
            a.nk = t.hidden;
            ISO_TRY(add_product(ProductKind::kGradX, product_func<ProductKind::kGradX>, true, a, partials));
        }
        ProductArgs a = kept;
        a.p[0] = x;
        a.q[0] = d_gate;
        a.q[1] = d_up;
        a.out[0] = device_rows(g->grad_gate);
        a.out[1] = device_rows(g->grad_up);
        a.np = t.channels;
        a.p_units = units_end();
        a.nq = t.hidden;
        a.nk = (int32_t)t.n;
        return add_product(ProductKind::kGradWeights, product_func<ProductKind::kGradWeights>, true, a, partials);
    }

    BoundOperator &b;
    const iso_gated_t &t;
    const iso_gated_grads_t *g;
    GatedWorkspace work;
    Rows x{}, gate{}, up{};                // as the products read them
};

}  // namespace iso
