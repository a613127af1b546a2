"""Which kernels a start of an operator on the ranks' tokens enqueues, on the CPU (see stub_library.py)."""
import math
import re

import pytest

import iso_inputs as gen
import paper_1606_07676_amd as iso
from tile_shapes import TILED

SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TYPE = {"f32": iso.ISO_DTYPE_F32, "bf16": iso.ISO_DTYPE_BF16, "f16": iso.ISO_DTYPE_F16}


def plain_name(name):
    """Of a demangled name, or of one with a type that c++filt does not know: tile<64> for attention_tile_kernel<__bf16, 64, false>."""
    found = re.match(r"_ZN3iso\d+(\w+?)_kernelI\w+?Li(\d+)E", name) or re.match(r"(\w+)_kernel<[^,]+, (\d+)", name)
    if found:
        return f"{found[1]}<{found[2]}>".replace("attention_", "")
    return re.match(r"(?:_ZN3iso\d+)?(\w+?)_kernel", name)[1].replace("attention_", "")


class Kernels:
    """Requests over dense stand-in buffers."""

    def __init__(self, stub):
        import sys
        self.stub, self.b, self.owned = stub, sys.modules["iso_on_stub.binding"], []

    def alloc(self, n):
        self.owned.append(self.stub.lib.stub_device_alloc(max(1, n)))
        return self.owned[-1]

    def start(self, dims, offsets, q_heads, kv_heads, D, dtype="bf16", periodic=None, backward=False, bias=False, segments=False, rows=0,
              cap=0.0, scale=None, shift=0):
        """The kernels of one start, those over tiles as name<elements of a row>."""
        import ctypes
        lib, p, s, e = self.stub.iso.load_library(), math.prod(dims), len(offsets), SIZE[dtype]
        comm = self.stub.comm(dims, offsets, periodic)
        heads = lambda n, h: self.b.iso_heads_t(self.alloc(n * h * D * e + shift * e) + shift * e, h * D, D)       # noqa: E731
        n = rows or p
        t = self.b.iso_attention_t(dtype=TYPE[dtype], q_heads=q_heads, kv_heads=kv_heads, head_dim=D, cap=cap,
                                   scale=D ** -0.5 if scale is None else scale, n_rows=rows)
        t.q, t.out, t.k, t.v = heads(n, q_heads), heads(n, q_heads), heads(p, kv_heads), heads(p, kv_heads)
        t.lse = self.alloc(n * q_heads * 4)
        t.bias = self.alloc(q_heads * s * e) if bias else None
        t.segments = self.alloc(p * 4) if segments else None
        t.rows = self.alloc(rows * 8) if rows else None
        h = ctypes.c_void_p()
        if backward:
            g = self.b.iso_attention_grads_t(grad_bias=self.alloc(q_heads * s * e) if bias else None)
            g.grad_out, g.grad_q, g.grad_k, g.grad_v = heads(n, q_heads), heads(n, q_heads), heads(p, kv_heads), heads(p, kv_heads)
            size = ctypes.c_size_t()
            assert lib.iso_neighbor_attention_backward_workspace_bytes(comm.handle, TYPE[dtype], q_heads, kv_heads, D, int(bias), ctypes.byref(size)) == 0
            st = lib.iso_neighbor_attention_backward_init(ctypes.byref(t), ctypes.byref(g), self.alloc(size.value), size.value, comm.handle, ctypes.byref(h))
        else:
            st = lib.iso_neighbor_attention_init(ctypes.byref(t), comm.handle, ctypes.byref(h))
        assert st == 0
        names = self.stub.launched(lambda: lib.iso_start(h, None))
        assert lib.iso_request_free(ctypes.byref(h)) == 0
        return [plain_name(n) for n in names]

    def free(self):
        for q in self.owned:
            self.stub.lib.stub_device_free(q)


@pytest.fixture
def kernels(stub_library):
    k = Kernels(stub_library)
    yield k
    k.free()


def short(names):
    return [n.split("<")[0] for n in names]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dims,offsets", [((8, 8), [(9, 0), (0, -8)]), ((4, 6), [(4, 0), (0, -6)]), ((1, 40), [(1, 0), (-1, 3)]),
                                          ((64, 64), [(64, 0)])])
def test_a_mesh_without_any_source_has_no_tiles(kernels, dims, offsets, dtype):
    """No key of any rank: nothing to stage, and the row kernels write what is left."""
    mesh = (0,) * len(dims)
    assert short(kernels.start(dims, offsets, 2, 2, 64, dtype, mesh)) in (["row"], ["split_row"])
    assert short(kernels.start(dims, offsets, 4, 2, 64, dtype, mesh, backward=True, bias=True)) == ["grad_q_row", "grad_kv_row", "grad_bias_row", "sum_parts"]
    # with one source it is tiles again, where they pay
    assert short(kernels.start((64, 64), gen.moore(2, 2) + [(64, 0)], 2, 2, 64, dtype, mesh)) == ["tile"]


def test_large_caps_go_by_rows(kernels):
    """The tiles' form of the cap is off by about 2^-22 of it."""
    volume = ((32, 32, 32), gen.moore(3, 1), 4, 2, 64)
    assert short(kernels.start(*volume, cap=128.0)) == ["tile"] and short(kernels.start(*volume, cap=129.0)) == ["row"]
    assert short(kernels.start(*volume, cap=30.0, backward=True)) == ["grad_q_tile", "grad_kv_tile"]
    assert short(kernels.start(*volume, cap=1e4, backward=True)) == ["grad_q_row", "grad_kv_row"]


MOST = (1 << 32) // 256 - 8                    # workgroups of 256 that a launch holds, in eights


@pytest.mark.parametrize("dims,heads,kv_heads,D,dtype", [((2048, 1024), 32, 1, 4, "f32"), ((1 << 24, 1), 5, 5, 1, "bf16")])
def test_more_rows_than_a_launch_holds(kernels, dims, heads, kv_heads, D, dtype):
    """2^32 work-items and more: several launches, which together have a wavefront for every row."""
    rows = math.prod(dims) * heads
    names = kernels.start(dims, [(1, 0)], heads, kv_heads, D, dtype)
    grids = list(kernels.stub.grids)
    assert short(names) == ["row"] * -(-rows // 4 // MOST) and len(grids) > 1
    assert sum(grids) == rows // 4 and all(n == MOST for n in grids[:-1])
    names = kernels.start(dims, [(1, 0)], heads, kv_heads, D, dtype, backward=True)
    of = lambda name: sum(n for n, k in zip(kernels.stub.grids, short(names)) if k == name)          # noqa: E731
    assert of("grad_q_row") == rows // 4 and of("grad_kv_row") == rows // heads * kv_heads // 4


def test_more_tiles_than_a_launch_holds(kernels):
    assert short(kernels.start((8192, 8192), gen.moore(2, 1), 16, 16, 8)) == ["tile"] * 2
    assert kernels.stub.grids == [MOST, 8192 * 8192 // 64 * 16 - MOST]


def test_more_tokens_than_a_launch_holds(kernels):
    """A workgroup of the rotary kernel takes 8 tokens of one pair of channels."""
    import ctypes
    import numpy as np
    n, lib = (1 << 27) + 3, kernels.stub.iso.load_library()
    freqs, axes, h = np.ones(1), np.zeros(1, np.int32), ctypes.c_void_p()
    t = kernels.b.iso_rotary_t(dtype=TYPE["f16"], heads=1, head_dim=2, pairs=1, n=n, freqs=freqs.ctypes.data, axes=axes.ctypes.data,
                               positions=kernels.alloc(4 * n), n_axes=1)
    t.x = t.out = kernels.b.iso_heads_t(kernels.alloc(4 * n), 2, 2)
    assert lib.iso_rotary_init(ctypes.byref(t), None, ctypes.byref(h)) == 0
    assert len(kernels.stub.launched(lambda: lib.iso_start(h, None))) == 2 and sum(kernels.stub.grids) == -(-n // 8)
    for form in (iso.ISO_GRAPH_CHAIN, iso.ISO_GRAPH_OFF):
        assert lib.iso_request_set_graph(h, form) == 0 and lib.iso_start(h, None) == 0
    assert lib.iso_request_free(ctypes.byref(h)) == 0


def test_rings_longer_than_half_the_32_bits_have_no_tiles(kernels):
    """A tile's place and a position in it add up in 32 bits."""
    for n, want in (((1 << 20), "tile"), ((1 << 30) + 64, "row")):
        assert set(short(kernels.start((n,), [(c,) for c in range(-20, 21)], 1, 1, 8))) == {want}, n


@pytest.mark.parametrize("dims,offsets,heads,forward,grad_q,grad_kv", [
    ((128, 128), gen.moore(2, 6), (8, 8, 32), "tile<32>", "grad_q_tile<32>", "grad_kv_tile<32>"),
    ((128, 128), gen.moore(2, 6), (8, 8, 128), "tile<128>", "grad_q_tile<128>", "grad_kv_tile<128>"),
    ((8, 8), gen.moore(2, 6), (8, 8, 32), "split_row", None, None),
    ((8, 8), gen.moore(2, 6), (8, 8, 128), "split_row", "grad_q_tile<128>", "grad_kv_tile<128>"),
    ((10, 10, 10), gen.moore(3, 1), (8, 2, 32), "tile<32>", "grad_q_tile<32>", "grad_kv_row"),
    ((8, 8, 8, 8), gen.random_distinct(4, -3, 3, 40, 7), (8, 2, 128), "tile<128>", "grad_q_tile<128>", "grad_kv_row"),
    ((6, 6, 6, 6), gen.random_distinct(4, -3, 3, 40, 7), (8, 8, 128), "row", None, "grad_kv_row")])
def test_tiles_or_rows_by_what_was_faster(kernels, dims, offsets, heads, forward, grad_q, grad_kv):
    """Places where one of the two was 1.3 to 25 times as fast (None: either)."""
    names = kernels.start(dims, offsets, *heads) + kernels.start(dims, offsets, *heads, backward=True, bias=True)
    assert all(want in (None, got) for want, got in zip((forward, grad_q, grad_kv), names)), names


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", TILED)
def test_shapes_of_the_tile_tests_take_tiles(kernels, shape, dtype):
    dims, periodic, offsets, q_heads, kv_heads, D = TILED[shape]
    assert short(kernels.start(dims, offsets, q_heads, kv_heads, D, dtype, periodic)) == ["tile"]
    for bias in (False, True):
        names = short(kernels.start(dims, offsets, q_heads, kv_heads, D, dtype, periodic, backward=True, bias=bias))
        assert names == ["grad_q_tile", "grad_kv_tile"] + ["sum_parts"] * bias


def test_the_workspace_holds_what_the_kernels_use(kernels):
    """Partial sums by the tile only where tiles are possible: not for float32, odd rows, or more neighbours than their tables hold."""
    import ctypes
    lib = kernels.stub.iso.load_library()

    def size(dims, offsets, q_heads, kv_heads, D, dtype, bias=True):
        out = ctypes.c_size_t()
        assert lib.iso_neighbor_attention_backward_workspace_bytes(kernels.stub.comm(dims, offsets).handle, TYPE[dtype], q_heads, kv_heads, D,
                                                                   int(bias), ctypes.byref(out)) == 0
        return out.value
    window, rows = gen.moore(2, 6), 256 * 256 * 8
    for dtype, D, by_row in (("f32", 64, 8), ("bf16", 63, 8), ("f16", 136, 8), ("bf16", 64, 16)):
        assert size((256, 256), window, 8, 8, D, dtype, False) == by_row * rows
        parts = (size((256, 256), window, 8, 8, D, dtype) - by_row * rows) / (8 * len(window) * 4)
        assert parts == (1024 if by_row == 16 else 8192 // (8 * len(window)))
    many = gen.moore(2, 64)                                        # 16640 neighbours
    assert size((1000, 1000), many, 8, 8, 64, "bf16") == 16 * 8 * 10 ** 6 + 8 * len(many) * 4
