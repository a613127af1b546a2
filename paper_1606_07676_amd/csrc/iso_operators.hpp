// Host side of the operators on the ranks' tokens (attention over the neighbourhood, rotary positions): argument checks,
// the choice of kernels and the launches of a request.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <vector>

#include "iso_attention_kernels.hpp"
#include "iso_attention_tiles.hpp"
#include "iso_bind.hpp"
#include "iso_rotary_kernels.hpp"
#include "iso_tiles.hpp"

namespace iso {

// One kernel launch of an operator: its arguments are one struct, kept with it.
struct OperatorLaunch {
    const void *func = nullptr;
    uint32_t grid = 0, threads = 0, lds = 0;
    std::shared_ptr<void> args;
};

struct BoundOperator {
    std::vector<OperatorLaunch> launches;
    void *dev_table = nullptr;             // owned by the request
};

inline void set_first_block(TileArgs &args, uint32_t first) { args.a.first_block = first; }
template <typename Args> void set_first_block(Args &args, uint32_t first) { args.first_block = first; }

// A launch holds fewer than 2^32 work-items: more workgroups than that go in several, each a multiple of 8 but the last, so
// that a workgroup's XCD stays the one that its number names.
template <typename Args>
int add_launch(BoundOperator &b, const void *func, uint64_t grid, uint32_t threads, Args args, size_t lds = 0) {
    if (grid > 0xFFFFFFFFull) return ISO_ERR_TOO_LARGE;
    const uint64_t most = 0xFFFFFFFFull / threads / 8 * 8;
    for (uint64_t first = 0; first < grid; first += most) {
        set_first_block(args, (uint32_t)first);
        b.launches.push_back({func, (uint32_t)std::min(most, grid - first), threads, (uint32_t)lds, std::make_shared<Args>(args)});
    }
    return ISO_SUCCESS;
}

inline int enqueue_operator(const OperatorLaunch &l, hipStream_t stream) {
    void *args[1] = {l.args.get()};
    ISO_HIP_TRY(hipLaunchKernel(l.func, dim3(l.grid), dim3(l.threads), args, l.lds, stream));
    return ISO_SUCCESS;
}

inline size_t dtype_size(int dtype) { return dtype == ISO_DTYPE_F32 ? 4 : 2; }

// ---- buffers -------------------------------------------------------------------

// n ranks with `heads` rows of `bytes` each, strides in bytes; a plain array is one head.
struct Region {
    uintptr_t at;
    uint64_t n, heads, rank_stride, head_stride, bytes;
    bool written;

    bool empty() const { return !n || !heads || !bytes; }
    uint64_t footprint() const { return (heads - 1) * head_stride + bytes; }     // of one rank
    uint64_t span() const { return (n - 1) * rank_stride + footprint(); }
};

constexpr uint64_t kMaxSpan = uint64_t(1) << 60;

// Rows of tensors that share their strides (slices of one buffer) are told apart rank by rank, or head by head where the heads
// lie further apart than the ranks; anything else by the ranges that they span.
//
// lattice_apart: two sets of cells, `outer` bytes from one to the next, with rows `inner` bytes apart in each.  They share no
// byte where the rows of b's cell lie behind all of a's, or between them.
struct Cells {
    uint64_t outer, inner, rows, bytes;
    uint64_t footprint() const { return (rows - 1) * inner + bytes; }
};
inline bool lattice_apart(const Cells &a, const Cells &b, uint64_t distance) {
    if (!a.outer || a.outer != b.outer || a.footprint() > a.outer) return false;
    const uint64_t delta = distance % a.outer;
    const bool inside = delta + b.footprint() <= a.outer;          // b's cell ends before a's next one
    if (inside && delta >= a.footprint()) return true;
    if (!a.inner || a.inner != b.inner || !(inside || a.outer % a.inner == 0)) return false;
    return delta % a.inner >= a.bytes && delta % a.inner + b.bytes <= a.inner;
}
inline bool regions_meet(const Region &a, const Region &b) {
    if (a.empty() || b.empty()) return false;
    if (a.at + a.span() <= b.at || b.at + b.span() <= a.at) return false;
    // b - a, and a - b, up to whole cells
    const auto apart = [&](const Cells &x, const Cells &y) {
        if (!x.outer) return false;
        const uint64_t ahead = b.at >= a.at ? (b.at - a.at) % x.outer : x.outer - (a.at - b.at) % x.outer;
        return lattice_apart(x, y, ahead) || lattice_apart(y, x, x.outer - ahead % x.outer);
    };
    return !apart({a.rank_stride, a.head_stride, a.heads, a.bytes}, {b.rank_stride, b.head_stride, b.heads, b.bytes}) &&
           !apart({a.head_stride, a.rank_stride, a.n, a.bytes}, {b.head_stride, b.rank_stride, b.n, b.bytes});
}

// Two rows of one written tensor must not share bytes.
inline bool region_meets_itself(const Region &r) {
    if (r.empty()) return false;
    const bool by_rank = (r.heads == 1 || r.head_stride >= r.bytes) && (r.n == 1 || r.rank_stride >= r.footprint());
    const bool by_head = (r.n == 1 || r.rank_stride >= r.bytes) &&
                         (r.heads == 1 || r.head_stride >= (r.n - 1) * r.rank_stride + r.bytes);
    return !by_rank && !by_head;
}

// The buffers of one request.
class Regions {
  public:
    int heads(const iso_heads_t &t, uint64_t n, int heads, int head_dim, int dtype, bool written) {
        const uint64_t size = dtype_size(dtype);
        if (!n || !heads || !head_dim) return ISO_SUCCESS;
        if (!t.data || t.rank_stride < 0 || t.head_stride < 0 || (uintptr_t)t.data % size) return ISO_ERR_ARG;
        if ((uint64_t)t.rank_stride > kMaxSpan / size / n || (uint64_t)t.head_stride > kMaxSpan / size / (uint64_t)heads)
            return ISO_ERR_TOO_LARGE;
        return add({(uintptr_t)t.data, n, (uint64_t)heads, (uint64_t)t.rank_stride * size, (uint64_t)t.head_stride * size,
                    (uint64_t)head_dim * size, written});
    }
    int array(const void *data, uint64_t bytes, uint64_t alignment, bool written) {
        if (!bytes) return ISO_SUCCESS;
        if (!data || (uintptr_t)data % alignment) return ISO_ERR_ARG;
        return add({(uintptr_t)data, 1, 1, 0, 0, bytes, written});
    }
    // except: this pair of regions may be the same rows (an operator in place)
    int disjoint(int except_a = -1, int except_b = -1) const {
        for (size_t i = 0; i < list.size(); ++i) {
            if (list[i].written && region_meets_itself(list[i])) return ISO_ERR_OVERLAP;
            for (size_t j = 0; j < i; ++j) {
                if ((int)j == except_a && (int)i == except_b) continue;
                if ((list[i].written || list[j].written) && regions_meet(list[i], list[j])) return ISO_ERR_OVERLAP;
            }
        }
        return ISO_SUCCESS;
    }

  private:
    int add(const Region &r) {
        list.push_back(r);
        return check_device_range((const void *)r.at, r.span());
    }
    std::vector<Region> list;
};

inline Heads device_heads(const iso_heads_t &t) { return Heads{t.data, t.rank_stride, t.head_stride}; }

// Rows start on 16-byte boundaries and hold whole groups of 16 bytes.
inline bool wide(const iso_heads_t &t, int head_dim, int dtype) {
    const uint64_t size = dtype_size(dtype);
    return (((uintptr_t)t.data | (uint64_t)t.rank_stride * size | (uint64_t)t.head_stride * size | (uint64_t)head_dim * size) & 15) == 0;
}

// Offsets as the kernels add them: residues where the dimension wraps; where it does not, a coordinate beyond the mesh's
// size has no source from anywhere, as the size itself has none.
inline std::vector<int32_t> kernel_offsets(const Comm &c) {
    std::vector<int32_t> out((size_t)c.s * c.d);
    for (int i = 0; i < c.s; ++i)
        for (int j = 0; j < c.d; ++j) {
            const int32_t n = c.dims[j], x = c.c(i, j);
            out[(size_t)i * c.d + j] = c.periodic[j] ? x : std::clamp(x, -n, n);
        }
    return out;
}

inline NeighbourTorus neighbour_torus(const Comm &c, const void *offsets) {
    NeighbourTorus t{};
    t.d = c.d;
    t.s = c.s;
    t.p = (uint32_t)c.p;
    for (int j = 0; j < c.d; ++j) {
        t.dims[j] = c.dims[j];
        t.inner[j] = (int32_t)c.inner[j];
        if (!c.periodic[j]) t.open |= 1u << j;
    }
    t.offsets = (const int32_t *)offsets;
    return t;
}

// The parts of a request's device table, each on a 16-byte boundary.
class Table {
  public:
    template <typename V> size_t add(const std::vector<V> &part) {
        const size_t at = (bytes.size() + 15) / 16 * 16;
        bytes.resize(at + part.size() * sizeof(V));
        if (!part.empty()) std::memcpy(bytes.data() + at, part.data(), part.size() * sizeof(V));
        return at;
    }
    std::vector<unsigned char> bytes;
};

inline int upload_table(BoundOperator &b, const void *host, size_t bytes) {
    if (!bytes) return ISO_SUCCESS;
    ISO_HIP_TRY(hipMalloc(&b.dev_table, bytes));
    ISO_HIP_TRY(hipMemcpy(b.dev_table, host, bytes, hipMemcpyHostToDevice));
    return ISO_SUCCESS;
}

#define ISO_TRY(expr)                              \
    do {                                           \
        const int st_ = (expr);                    \
        if (st_ != ISO_SUCCESS) return st_;        \
    } while (0)

// ---- attention --------------------------------------------------------------------

template <template <typename, bool> class Kernel>
const void *by_type(int dtype, bool wide) {
    switch (dtype) {
        case ISO_DTYPE_F32: return wide ? Kernel<float, true>::func() : Kernel<float, false>::func();
        case ISO_DTYPE_BF16: return wide ? Kernel<__bf16, true>::func() : Kernel<__bf16, false>::func();
        default: return wide ? Kernel<_Float16, true>::func() : Kernel<_Float16, false>::func();
    }
}
#define ISO_KERNEL_BY_TYPE(name, kernel)                                            \
    template <typename T, bool WIDE> struct name {                                  \
        static const void *func() { return (const void *)(kernel<T, WIDE>); }       \
    };
ISO_KERNEL_BY_TYPE(RowKernel, attention_row_kernel)
ISO_KERNEL_BY_TYPE(SplitRowKernel, attention_split_row_kernel)
ISO_KERNEL_BY_TYPE(GradQRowKernel, attention_grad_q_row_kernel)
ISO_KERNEL_BY_TYPE(GradKVRowKernel, attention_grad_kv_row_kernel)
ISO_KERNEL_BY_TYPE(GradBiasRowKernel, attention_grad_bias_row_kernel)
ISO_KERNEL_BY_TYPE(RotaryKernel, rotary_kernel)
#undef ISO_KERNEL_BY_TYPE

template <template <typename, int, bool> class Kernel, typename T>
const void *tile_by_size(int head_dim, bool segments) {
    if (head_dim <= 32) return segments ? Kernel<T, 32, true>::func() : Kernel<T, 32, false>::func();
    if (head_dim <= 64) return segments ? Kernel<T, 64, true>::func() : Kernel<T, 64, false>::func();
    if (head_dim <= 96) return segments ? Kernel<T, 96, true>::func() : Kernel<T, 96, false>::func();
    return segments ? Kernel<T, 128, true>::func() : Kernel<T, 128, false>::func();
}
template <template <typename, int, bool> class Kernel>
const void *tile_by_type(int dtype, int head_dim, bool segments) {
    return dtype == ISO_DTYPE_BF16 ? tile_by_size<Kernel, __bf16>(head_dim, segments) : tile_by_size<Kernel, _Float16>(head_dim, segments);
}
#define ISO_TILE_KERNEL(name, kernel)                                                           \
    template <typename T, int DP, bool SEGMENTS> struct name {                                  \
        static const void *func() { return (const void *)(kernel<T, DP, SEGMENTS>); }           \
    };
ISO_TILE_KERNEL(TileKernel, attention_tile_kernel)
ISO_TILE_KERNEL(GradQTileKernel, attention_grad_q_tile_kernel)
ISO_TILE_KERNEL(GradKVTileKernel, attention_grad_kv_tile_kernel)
#undef ISO_TILE_KERNEL

constexpr int kTileMaxHeadDim = 128;
constexpr size_t kTileMaxLds = 64 << 10;
constexpr uint64_t kSplitWaves = 4096;     // wavefronts up to which a row's neighbours are shared out
inline int tile_head_dim(int head_dim) { return (head_dim + 31) / 32 * 32; }
inline int tile_chunk_rows(int head_dim) { return tile_head_dim(head_dim) > 32 ? TileLds<64>::kRows : TileLds<32>::kRows; }
inline size_t tile_lds_bytes(int head_dim, int chunks, size_t biases) {
    switch (tile_head_dim(head_dim)) {
        case 32: return TileLds<32>::bytes(chunks, biases);
        case 64: return TileLds<64>::bytes(chunks, biases);
        case 96: return TileLds<96>::bytes(chunks, biases);
        default: return TileLds<128>::bytes(chunks, biases);
    }
}

// Lanes that share one neighbour's row in the row kernels.
inline int row_lanes(int dtype, int head_dim) {
    int lanes = 1;
    while (lanes * (dtype == ISO_DTYPE_F32 ? 4 : 8) < head_dim) lanes *= 2;
    return lanes;
}

inline const void *sum_parts_by_type(int dtype) {
    switch (dtype) {
        case ISO_DTYPE_F32: return (const void *)(sum_parts_kernel<float>);
        case ISO_DTYPE_BF16: return (const void *)(sum_parts_kernel<__bf16>);
        default: return (const void *)(sum_parts_kernel<_Float16>);
    }
}

// Parts of the ranks that the bias's gradient is summed over: enough wavefronts for the GPU, 16 ranks or more in each.  Float32
// backward of 4 heads of 64, with 1024 wavefronts to 8192 to 65536, in us: 12 x 11 x 10 ranks, 27 neighbours, 115, 68, 69; 64 x 64
// ranks, 25 neighbours, 279, 136, 137.
inline uint64_t bias_parts(const Comm &c, int q_heads) {
    const uint64_t slots = std::max<uint64_t>(1, (uint64_t)q_heads * c.s);
    return std::clamp<uint64_t>(8192 / slots, 1, ((uint64_t)c.p + 15) / 16);
}

struct BackwardWorkspace {
    uint64_t delta = 0, starts = 0, norms = 0, partials = 0, bytes = 0;     // offsets
};
inline int tile_heads(int group) {             // q heads of a rank that one tile of columns takes together
    int heads = 1;
    while (heads < 8 && group % (2 * heads) == 0) heads *= 2;
    return heads;
}
// Tensors that the tile kernels may take, whatever their strides.
inline bool tile_tensors(int dtype, int head_dim) {
    return dtype != ISO_DTYPE_F32 && head_dim <= kTileMaxHeadDim && head_dim * dtype_size(dtype) % 16 == 0;
}
inline int backward_workspace(const Comm &c, int dtype, int q_heads, int kv_heads, int head_dim, bool bias, BackwardWorkspace &w) {
    const uint64_t rows = (uint64_t)c.p * q_heads;               // below 2^47
    const bool tiles = tile_tensors(dtype, head_dim);
    w.starts = (rows * 4 + 255) / 256 * 256;
    w.norms = w.starts + (tiles ? (rows * 8 + 255) / 256 * 256 : 0);
    w.partials = w.norms + (rows * 4 + 255) / 256 * 256;
    w.bytes = w.partials;
    if (bias) {
        if ((uint64_t)q_heads * c.s > 0x7FFFFFFFull) return ISO_ERR_TOO_LARGE;
        uint64_t parts = bias_parts(c, q_heads);
        for (int heads = tiles ? tile_heads(q_heads / kv_heads) : 0; heads; heads /= 2)
            if (tile_table_holds(heads, c.s)) parts = std::max<uint64_t>(parts, (uint64_t)tile_shape(c, heads).n_tiles);
        w.bytes += parts * q_heads * c.s * 4;
    }
    return ISO_SUCCESS;
}

inline int check_shape(int dtype, int q_heads, int kv_heads, int head_dim) {
    if (dtype != ISO_DTYPE_F32 && dtype != ISO_DTYPE_BF16 && dtype != ISO_DTYPE_F16) return ISO_ERR_ARG;
    if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || head_dim < 1) return ISO_ERR_ARG;
    if (q_heads > 65536 || head_dim > kAttentionMaxHeadDim) return ISO_ERR_TOO_LARGE;
    return ISO_SUCCESS;
}

class AttentionBinder {
  public:
    AttentionBinder(BoundOperator &out, const Comm &comm, const iso_attention_t &attention, const iso_attention_grads_t *grads)
        : b(out), c(comm), t(attention), g(grads) {}

    int bind(void *workspace, size_t workspace_bytes) {
        ISO_TRY(check_shape(t.dtype, t.q_heads, t.kv_heads, t.head_dim));
        if (!(t.cap >= 0.f) || std::isinf(t.cap) || !std::isfinite(t.scale)) return ISO_ERR_ARG;
        if (t.n_rows < 0 || (t.n_rows && !t.rows) || (g && t.rows)) return ISO_ERR_ARG;
        if (t.n_rows > 0x7FFFFFFF) return ISO_ERR_TOO_LARGE;
        n = t.rows ? (uint64_t)t.n_rows : (uint64_t)c.p;
        ISO_TRY(check_buffers(workspace, workspace_bytes));
        if (!n) return ISO_SUCCESS;
        Table table;
        table.add(kernel_offsets(c));
        choose_width();
        const int group = t.q_heads / t.kv_heads;
        const bool sums = g && g->grad_bias && c.s;                // dx of 32 rows and the slots, of every wavefront
        // fewer heads together where what they need does not fit in LDS
        for (int heads = tile_heads(group); heads && !forward_side.tiles; heads /= 2)
            forward_side.take(*this, table, heads, false, sums,
                              (size_t)heads * (c.s + 1) + (sums ? 3 + kTileWaves * (kDxFloats + (size_t)heads * c.s + 1) : 0));
        if (g) backward_side.take(*this, table, 1, true, false, (t.bias ? (size_t)group : 1) * (c.s + 1));
        ISO_TRY(upload_table(b, table.bytes.data(), table.bytes.size()));
        fill_args(workspace);
        return g ? backward() : forward();
    }

  private:
    int check_buffers(void *workspace, size_t workspace_bytes) {
        Regions r;
        const int nq = t.q_heads, nk = t.kv_heads, D = t.head_dim, dt = t.dtype;
        const uint64_t p = (uint64_t)c.p, slots = (uint64_t)nq * c.s, size = dtype_size(dt);
        ISO_TRY(r.heads(t.q, n, nq, D, dt, false));
        ISO_TRY(r.heads(t.k, n ? p : 0, nk, D, dt, false));
        ISO_TRY(r.heads(t.v, n ? p : 0, nk, D, dt, false));
        ISO_TRY(r.heads(t.out, n, nq, D, dt, !g));
        if (g && !t.lse) return ISO_ERR_ARG;
        if (t.lse) ISO_TRY(r.array(t.lse, n * nq * 4, 4, !g));
        if (t.bias && n) ISO_TRY(r.array(t.bias, slots * size, size, false));
        if (t.segments && n) ISO_TRY(r.array(t.segments, p * 4, 4, false));
        if (t.rows) ISO_TRY(r.array(t.rows, n * 8, 8, false));
        if (g) {
            ISO_TRY(r.heads(g->grad_out, n, nq, D, dt, false));
            ISO_TRY(r.heads(g->grad_q, n, nq, D, dt, true));
            ISO_TRY(r.heads(g->grad_k, n, nk, D, dt, true));
            ISO_TRY(r.heads(g->grad_v, n, nk, D, dt, true));
            if (g->grad_bias && !t.bias && c.s) return ISO_ERR_ARG;
            if (g->grad_bias) ISO_TRY(r.array(g->grad_bias, slots * size, size, true));
            ISO_TRY(backward_workspace(c, dt, nq, nk, D, g->grad_bias != nullptr, work));
            if (!workspace || workspace_bytes < work.bytes) return ISO_ERR_WORKSPACE;
            ISO_TRY(r.array(workspace, work.bytes, 4, true));
        }
        return r.disjoint();
    }

    void fill_args(void *workspace) {
        a = AttentionArgs{};
        a.torus = neighbour_torus(c, b.dev_table);
        a.q = device_heads(t.q);
        a.k = device_heads(t.k);
        a.v = device_heads(t.v);
        a.out = device_heads(t.out);
        a.lse = t.lse;
        a.bias = c.s ? t.bias : nullptr;
        a.segments = t.segments;
        a.rows = t.rows;
        a.n = (uint32_t)n;
        a.q_heads = t.q_heads;
        a.kv_heads = t.kv_heads;
        a.group = t.q_heads / t.kv_heads;
        a.head_dim = t.head_dim;
        a.scale = t.scale;
        a.cap = t.cap;
        a.lanes_log2 = __builtin_ctz(row_lanes(t.dtype, t.head_dim));
        if (g) {
            a.grad_out = device_heads(g->grad_out);
            a.grad_q = device_heads(g->grad_q);
            a.grad_k = device_heads(g->grad_k);
            a.grad_v = device_heads(g->grad_v);
            a.delta = (float *)((char *)workspace + work.delta);
            a.starts = work.norms > work.starts ? (float *)((char *)workspace + work.starts) : nullptr;
            a.norms = (float *)((char *)workspace + work.norms);
            a.partials = (float *)((char *)workspace + work.partials);
        }
    }

    void choose_width() {
        is_wide = true;
        for (const iso_heads_t *x : {&t.q, &t.k, &t.v, &t.out}) is_wide = is_wide && wide(*x, t.head_dim, t.dtype);
        if (!g) return;
        for (const iso_heads_t *x : {&g->grad_out, &g->grad_q, &g->grad_k, &g->grad_v})
            is_wide = is_wide && wide(*x, t.head_dim, t.dtype);
    }

    // The tiles of one direction, where there are any.
    struct Side {
        bool tiles = false;
        TilePlan plan;
        size_t lds = 0, columns = 0, rows = 0, active = 0, index = 0, slots = 0, zeros = 0;
        int chunks = 0;

        // Tiles or rows, by what either would take, in us.  A tile takes 32 of its rows after the other, as fast as one does alone
        // or as all side by side do together; a row takes its neighbours in sets, as many as lanes have room for, and something
        // to begin and end with, likewise.  Constants by kernel (forward; grad_q with the bias's gradient; grad_kv), fitted to
        // 681 times of either: heads of 32, 64, 80 and 128, 8 / 8, 8 / 2 and 2 / 2 of them, 64 to 38416 ranks, 5 to 169 neighbours in
        // 1 to 4 dimensions; tiles a tenth under their fit, as a wrong choice of rows costs more.  What is taken is 1 % over
        // the better of the two in the mean, 70 % at worst; for 693 others (heads of 32 to 128, 3 to 81 neighbours, to 200000
        // ranks) 0.3 % and 65 %.  Tiles to rows: 128 x 128, 169 neighbours, 8 / 8 heads, forward, 29 to 338 at 32 elements, 54 to
        // 1294 at 128; 8 x 8, the same, 15.9 to 8.3 and 28.8 to 12.9; grad_kv of 10 x 10 x 10, 27 neighbours, 8 / 2 heads of 32,
        // 25.9 to 16.3; 40 neighbours scattered over 4 dimensions, 8 / 8 heads of 128, forward, 1296 ranks 58 to 38, 14641 ranks
        // 279 to 364.
        struct Estimate {
            double tile, rows32, rows32_element, beside, beside_element;
            double row, set, row_beside, row_sets;
        };
        static bool tiles_pay(const AttentionBinder &o, int heads, bool back, int rows, int64_t n_tiles) {
            static constexpr Estimate kForward{4.6, 0.177, 0.0045, 4.35e-4, 1.31e-5, 5.9, 0.18, 2.28e-4, 1.5};
            static constexpr Estimate kGradQ{7.6, 0.61, 0.0071, 1.5e-3, 2.35e-5, 13.8, 1.85, 7.6e-4, 0.6};
            static constexpr Estimate kGradKV{5.3, 0.416, 0.0065, 4.7e-4, 2.8e-5, 7.8, 1.25, 3.87e-4, 1.8};
            const Estimate &e = back ? kGradKV : o.g ? kGradQ : kForward;
            const int chunk = tile_chunk_rows(o.t.head_dim), elements = tile_head_dim(o.t.head_dim), group = o.t.q_heads / o.t.kv_heads;
            const double turns = back ? group : 1, side_by_side = (double)n_tiles * o.t.kv_heads * (back ? 1 : group / heads);
            const double chunks = (double)((rows + chunk - 1) / chunk) * (chunk / 32) * turns;
            const double tile = e.tile + chunks * std::max(e.rows32 + e.rows32_element * elements,
                                                           side_by_side * (e.beside + e.beside_element * elements));
            const double lanes = row_lanes(o.t.dtype, o.t.head_dim), sets = std::ceil(o.c.s * lanes / 64);
            return tile <= e.row + std::max(sets * turns * e.set, (double)o.c.p * o.t.q_heads * (sets + e.row_sets) * e.row_beside);
        }

        void take(const AttentionBinder &o, Table &table, int heads, bool back, bool sums, size_t floats) {
            if (o.t.rows || !o.is_wide || !tile_tensors(o.t.dtype, o.t.head_dim)) return;
            if (!(std::fabs(o.t.scale) > 1e-20f && std::fabs(o.t.scale) < 1e20f)) return;      // the kernels divide by it
            if (o.t.cap > kPlainCap) return;                       // scores would be off by more than the weights' rounding
            for (const iso_heads_t *x : {&o.t.q, &o.t.k, &o.t.v, o.g ? &o.g->grad_out : &o.t.q})
                if (x->rank_stride >> 31) return;                  // strides in bytes: 32 bits
            const int chunk = tile_chunk_rows(o.t.head_dim);
            const auto lds_of = [&](int rows) { return tile_lds_bytes(o.t.head_dim, (rows + chunk - 1) / chunk, floats); };
            if (!build_tile_plan(o.c, heads, back, sums, plan, [&](int rows, int64_t n_tiles) {
                    return lds_of(rows) <= kTileMaxLds && tiles_pay(o, heads, back, rows, n_tiles);
                }))
                return;
            chunks = (plan.rows + chunk - 1) / chunk;
            lds = lds_of(plan.rows);
            columns = table.add(plan.column_at);
            rows = table.add(plan.row_at);
            active = table.add(plan.active);
            index = table.add(plan.index);
            zeros = table.add(std::vector<uint16_t>(kTileMaxHeadDim));
            if (sums) slots = table.add(plan.slots);
            tiles = true;
        }
    };

    int add_tiles(const Side &side, const void *func, int parts) {
        const TilePlan &p = side.plan;
        TileArgs ta{};
        ta.a = a;
        const uint64_t work = (uint64_t)p.n_tiles * t.kv_heads * parts;
        if (work > 0x7FFFFFF0ull) return ISO_ERR_TOO_LARGE;
        for (int i = 0; i < c.d; ++i) {
            const int j = c.d - 1 - i;
            ta.dim[i] = {make_fastdiv((uint32_t)p.tiles[j]), p.tile[j], c.dims[j], (int32_t)c.inner[j], c.periodic[j]};
        }
        ta.n_tiles = make_fastdiv((uint32_t)p.n_tiles);
        ta.parts = make_fastdiv((uint32_t)parts);
        ta.biases = make_fastdiv((uint32_t)c.s + 1);
        ta.items = (uint32_t)work;
        ta.heads = p.heads;
        ta.words = (c.d + 3) / 4;
        ta.chunks = side.chunks;
        const char *base = (const char *)b.dev_table;
        ta.column_at = (const uint2 *)(base + side.columns);
        ta.row_at = (const uint2 *)(base + side.rows);
        ta.active = (const uint32_t *)(base + side.active);
        ta.index = (const uint16_t *)(base + side.index);
        ta.zeros = base + side.zeros;
        if (!p.slots.empty()) {
            ta.slots = (const uint32_t *)(base + side.slots);
            ta.slot_rounds = p.slot_rounds;
            ta.slot_words = p.slot_words;
        }
        ta.per_xcd = (uint32_t)((work + 7) / 8);
        return add_launch(b, func, (uint64_t)ta.per_xcd * 8, 256, ta, side.lds);
    }

    int forward() {
        const bool segments = t.segments || c.mesh;
        if (forward_side.tiles)
            return add_tiles(forward_side, tile_by_type<TileKernel>(t.dtype, t.head_dim, segments), a.group / forward_side.plan.heads);
        const uint64_t items = n * t.q_heads;
        // Few rows: the wavefronts of a workgroup share the neighbours of one, so that the GPU has work, up to 4 wavefronts for
        // each of its 1024 SIMDs.  One wavefront a row to this, in us: 8 heads of 64, 49 neighbours, 100 rows 12.0 to 8.9, 250
        // rows 12.5 to 10.7; 169 neighbours, 37 rows 27.3 to 10.6.  Twice as many wavefronts: 250 rows 11.2, 500 rows 20.0 for
        // 15.1; sixteen a row, 250 rows 16.0.
        const uint64_t sets = 64 >> a.lanes_log2, takes = ((uint64_t)c.s + sets - 1) / sets;
        a.waves = (int)std::clamp<uint64_t>(std::min(takes, kSplitWaves / items), 1, 16);
        if (a.waves > 1) return add_launch(b, by_type<SplitRowKernel>(t.dtype, is_wide), items, 64u * a.waves, a);
        return add_launch(b, by_type<RowKernel>(t.dtype, is_wide), (items + 3) / 4, 256, a);
    }

    int backward() {
        const bool segments = t.segments || c.mesh, bias = g->grad_bias && c.s;
        if (forward_side.tiles)
            ISO_TRY(add_tiles(forward_side, tile_by_type<GradQTileKernel>(t.dtype, t.head_dim, segments), a.group / forward_side.plan.heads));
        else
            ISO_TRY(add_launch(b, by_type<GradQRowKernel>(t.dtype, is_wide), (n * t.q_heads + 3) / 4, 256, a));
        if (backward_side.tiles)
            ISO_TRY(add_tiles(backward_side, tile_by_type<GradKVTileKernel>(t.dtype, t.head_dim, segments), 1));
        else
            ISO_TRY(add_launch(b, by_type<GradKVRowKernel>(t.dtype, is_wide), (n * t.kv_heads + 3) / 4, 256, a));
        if (!bias) return ISO_SUCCESS;
        const uint64_t slots = (uint64_t)t.q_heads * c.s;
        a.parts = forward_side.tiles ? (int)forward_side.plan.n_tiles : (int)bias_parts(c, t.q_heads);
        if (!forward_side.tiles)
            ISO_TRY(add_launch(b, by_type<GradBiasRowKernel>(t.dtype, is_wide), (slots * a.parts + 3) / 4, 256, a));
        return add_launch(b, sum_parts_by_type(t.dtype), (slots + 15) / 16, 1024,
                          SumPartsArgs{a.partials, g->grad_bias, (uint32_t)slots, (uint32_t)a.parts, 0});
    }

    BoundOperator &b;
    const Comm &c;
    const iso_attention_t &t;
    const iso_attention_grads_t *g;
    uint64_t n = 0;
    BackwardWorkspace work;
    AttentionArgs a{};
    bool is_wide = false;
    Side forward_side, backward_side;          // columns are ranks; columns are keys
};

// ---- rotary positions --------------------------------------------------------------

inline int bind_rotary(BoundOperator &b, const Comm *c, const iso_rotary_t &t) {
    ISO_TRY(check_shape(t.dtype, t.heads, t.heads, t.head_dim));
    if (t.pairs < 0 || 2 * (int64_t)t.pairs > t.head_dim || (t.pairs && (!t.freqs || !t.axes)) || t.n < 0) return ISO_ERR_ARG;
    if (t.n > 0x7FFFFFFF) return ISO_ERR_TOO_LARGE;
    if (!t.n) return ISO_SUCCESS;
    if (!t.positions && (!c || t.n != c->p)) return ISO_ERR_ARG;
    const int n_axes = t.positions ? t.n_axes : c->d;
    for (int j = 0; j < t.pairs; ++j)
        if (t.axes[j] < 0 || t.axes[j] >= n_axes || !std::isfinite(t.freqs[j])) return ISO_ERR_ARG;
    Regions r;
    const bool in_place = t.x.data == t.out.data && t.x.rank_stride == t.out.rank_stride && t.x.head_stride == t.out.head_stride;
    ISO_TRY(r.heads(t.x, (uint64_t)t.n, t.heads, t.head_dim, t.dtype, false));
    ISO_TRY(r.heads(t.out, (uint64_t)t.n, t.heads, t.head_dim, t.dtype, true));
    if (t.positions) ISO_TRY(r.array(t.positions, (uint64_t)t.n * n_axes * 4, 4, false));
    ISO_TRY(in_place ? r.disjoint(0, 1) : r.disjoint());

    std::vector<unsigned char> table((size_t)t.pairs * 12);
    for (int j = 0; j < t.pairs; ++j) {
        const double turns = t.freqs[j] / 6.283185307179586476925286766559;
        std::memcpy(table.data() + (size_t)j * 8, &turns, 8);
        std::memcpy(table.data() + (size_t)t.pairs * 8 + (size_t)j * 4, &t.axes[j], 4);
    }
    ISO_TRY(upload_table(b, table.data(), table.size()));
    RotaryArgs a{};
    a.x = device_heads(t.x);
    a.out = device_heads(t.out);
    a.positions = t.positions;
    a.turns = (const double *)b.dev_table;
    a.axes = (const int32_t *)((const char *)b.dev_table + (size_t)t.pairs * 8);
    a.n = (uint32_t)t.n;
    a.n_axes = n_axes;
    a.head_dim = t.head_dim;
    a.pairs = t.pairs;
    a.interleaved = t.interleaved != 0;
    a.sign = t.inverse ? -1.f : 1.f;
    for (int j = 0; c && j < c->d; ++j) {
        a.dims[j] = c->dims[j];
        a.inner[j] = (int32_t)c->inner[j];
    }
    // As many ranks as a workgroup holds angles of, at most 8: 16 heads of 80 at 255 x 257 ranks take 129 us, with one rank a
    // workgroup 136, with four times as many 140; 10 heads of 128 at 64 x 64 x 64 ranks 226, 349 and 243.
    static_assert(kRotaryAngles >= kAttentionMaxHeadDim / 2);
    a.ranks = std::clamp(kRotaryAngles / std::max(1, t.pairs), 1, 8);
    const int per_lane = t.dtype == ISO_DTYPE_F32 ? 4 : 8;
    const bool whole = (t.interleaved ? 2 * t.pairs : t.pairs) % per_lane == 0;      // no unit of 16 bytes mixes both kinds
    const bool is_wide = whole && wide(t.x, t.head_dim, t.dtype) && wide(t.out, t.head_dim, t.dtype);
    const int E = is_wide ? per_lane : 1;
    const int units = t.interleaved && is_wide ? t.head_dim / E : (t.head_dim - t.pairs) / E;
    a.by_pairs = make_fastdiv((uint32_t)std::max(1, t.pairs));
    a.by_units = make_fastdiv((uint32_t)units);
    a.by_heads = make_fastdiv((uint32_t)t.heads);
    return add_launch(b, by_type<RotaryKernel>(t.dtype, is_wide), ((uint64_t)t.n + a.ranks - 1) / a.ranks, 256, a);
}

}  // namespace iso
