"""What the operators on each token by itself refuse, which kernels they take, and what they ask of their workspaces, without a
GPU (see stub_library.py)."""
import ctypes
import math
import re
import sys

import numpy as np
import pytest

from token_shapes import FEW, LARGE, MANY_HEADS, NORMS, TILED

N, C, F, H = 40, 24, 32, 3                # tokens, channels, hidden units, heads
SIZE = {0: 4, 1: 2, 2: 2}


class Operands:
    """Descriptors over dense stand-in device buffers, float32."""

    def __init__(self, stub):
        self.stub, self.iso, self.lib = stub, stub.iso, stub.iso.load_library()
        self.b, self.owned = sys.modules["iso_on_stub.binding"], []

    def alloc(self, n):
        self.owned.append(self.stub.lib.stub_device_alloc(max(1, n)))
        return self.owned[-1]

    def free(self):
        for q in self.owned:
            self.stub.lib.stub_device_free(q)

    def rows(self, n, width, size=4, shift=0):
        return self.b.iso_rows_t(self.alloc(n * width * size + shift * size) + shift * size, width)

    def heads(self, n=N, heads=H, width=C):
        return self.b.iso_heads_t(self.alloc(n * heads * width * 4), heads * width, width)

    def norm(self, **change):
        t = self.b.iso_layer_norm_t(dtype=0, heads=H, channels=C, n=N, eps=1e-5)
        t.x, t.out, t.weight, t.bias = self.heads(), self.heads(), self.alloc(C * 4), self.alloc(C * 4)
        t.mean, t.rstd = self.alloc(N * H * 4), self.alloc(N * H * 4)
        return self.changed(t, change)

    def norm_grads(self, **change):
        return self.changed(self.b.iso_layer_norm_grads_t(self.heads(), self.heads(), self.alloc(C * 4), self.alloc(C * 4)), change)

    def dropout(self, **change):
        t = self.b.iso_dropout_t(dtype=0, channels=C, n=N, seed=self.alloc(16), rate=0.1)
        t.x, t.out, t.residual = self.rows(N, C), self.rows(N, C), self.rows(N, C)
        return self.changed(t, change)

    def gated(self, n=N, channels=C, hidden=F, dtype=0, shift=0, **change):
        t = self.b.iso_gated_t(dtype=dtype, activation=0, channels=channels, hidden=hidden, n=n)
        rows = lambda count, width: self.rows(count, width, SIZE[dtype], shift)       # noqa: E731
        t.x, t.gate, t.up, t.out = rows(n, channels), rows(hidden, channels), rows(hidden, channels), rows(n, hidden)
        return self.changed(t, change)

    def gated_grads(self, n=N, channels=C, hidden=F, dtype=0, **change):
        rows = lambda count, width: self.rows(count, width, SIZE[dtype])              # noqa: E731
        return self.changed(self.b.iso_gated_grads_t(rows(n, hidden), rows(n, channels), rows(hidden, channels), rows(hidden, channels)), change)

    @staticmethod
    def changed(t, change):
        for name, value in change.items():
            setattr(t, name, value)
        return t

    def init(self, call, *args, started=False):
        """Status of the call; with `started`, the names of the kernels of one start."""
        h = ctypes.c_void_p(1)
        st = getattr(self.lib, call)(*args, ctypes.byref(h))
        names = []
        if st == 0:
            names = self.stub.launched(lambda: self.lib.iso_start(h, None))
            assert self.lib.iso_request_free(ctypes.byref(h)) == 0
        assert not h.value
        return [re.search(r"([a-z_]+)_kernel", n)[1] for n in names] if started else st

    def bytes_of(self, call, *args):
        size = ctypes.c_size_t()
        assert getattr(self.lib, call)(*args, ctypes.byref(size)) == 0
        return size.value

    def forward(self, t, **kw):
        return self.init("iso_layer_norm_init", ctypes.byref(t), **kw)

    def backward(self, t, g, work="own", size=None, **kw):
        need = self.bytes_of("iso_layer_norm_backward_workspace_bytes", N, H, C, 0)
        return self.init("iso_layer_norm_backward_init", ctypes.byref(t), ctypes.byref(g), self.alloc(need) if work == "own" else work,
                         need if size is None else size, **kw)

    def drop(self, t, **kw):
        return self.init("iso_dropout_init", ctypes.byref(t), **kw)

    def project(self, t, **kw):
        return self.init("iso_gated_init", ctypes.byref(t), **kw)

    def project_back(self, t, g, work="own", size=None, **kw):
        need = self.bytes_of("iso_gated_backward_workspace_bytes", t.n, t.channels, t.hidden, t.dtype) if t.n >= 0 and size is None else 1 << 20
        return self.init("iso_gated_backward_init", ctypes.byref(t), ctypes.byref(g), self.alloc(need) if work == "own" else work,
                         need if size is None else size, **kw)


@pytest.fixture
def ops(stub_library):
    o = Operands(stub_library)
    yield o
    o.free()


def test_what_is_taken(ops):
    assert ops.forward(ops.norm()) == 0
    assert ops.forward(ops.norm(weight=None, bias=None, mean=None, rstd=None, eps=0.0)) == 0
    assert ops.backward(ops.norm(), ops.norm_grads()) == 0
    assert ops.backward(ops.norm(weight=None), ops.norm_grads(grad_weight=None, grad_bias=None), work=None, size=0) == 0
    assert ops.drop(ops.dropout()) == 0
    assert ops.drop(ops.dropout(rate=0.0)) == 0 and ops.drop(ops.dropout(rate=1.0, residual=ops.b.iso_rows_t())) == 0
    assert ops.project(ops.gated()) == 0 and ops.project(ops.gated(activation=1)) == 0
    assert ops.project_back(ops.gated(), ops.gated_grads()) == 0


def test_nothing_for_no_tokens(ops):
    empty = ops.b.iso_heads_t(), ops.b.iso_rows_t()
    assert ops.forward(ops.norm(n=0, x=empty[0], out=empty[0], mean=None, rstd=None), started=True) == []
    assert ops.drop(ops.dropout(n=0, x=empty[1], out=empty[1], residual=empty[1], seed=None), started=True) == []
    assert ops.project(ops.gated(n=0, x=empty[1], out=empty[1]), started=True) == []
    # gradients that sum over tokens are zeros
    grads = ops.norm_grads(grad_out=empty[0], grad_x=empty[0])
    assert ops.backward(ops.norm(n=0, x=empty[0], mean=None, rstd=None), grads, started=True) == ["layer_norm_backward", "layer_norm_sum"]
    grads = ops.gated_grads(grad_out=empty[1], grad_x=empty[1])
    assert ops.project_back(ops.gated(n=0, x=empty[1], out=empty[1]), grads, started=True) == ["product"]


@pytest.mark.parametrize("change", [dict(dtype=3), dict(dtype=-1), dict(heads=0), dict(channels=0), dict(n=-1), dict(eps=-1.0), dict(eps=math.nan),
                                    dict(eps=math.inf)], ids=str)
def test_bad_values_of_norms(ops, change):
    assert ops.forward(ops.norm(**change)) == ops.iso.ISO_ERR_ARG
    if "eps" not in change:
        assert ops.backward(ops.norm(**change), ops.norm_grads()) == ops.iso.ISO_ERR_ARG


@pytest.mark.parametrize("change", [dict(dtype=3), dict(channels=0), dict(n=-1), dict(rate=-0.1), dict(rate=1.5), dict(rate=math.nan), dict(seed=None)], ids=str)
def test_bad_values_of_dropout(ops, change):
    assert ops.drop(ops.dropout(**change)) == ops.iso.ISO_ERR_ARG


@pytest.mark.parametrize("change", [dict(dtype=3), dict(activation=2), dict(activation=-1)], ids=str)
def test_bad_values_of_projections(ops, change):
    t = ops.gated()
    for k, v in change.items():
        setattr(t, k, v)
    assert ops.project(t) == ops.iso.ISO_ERR_ARG
    assert ops.project_back(t, ops.gated_grads(), size=1 << 20) == ops.iso.ISO_ERR_ARG


def test_bad_counts_of_projections(ops):
    for change in (dict(channels=0), dict(hidden=0), dict(n=-1)):
        t = ops.gated()
        for k, v in change.items():
            setattr(t, k, v)
        assert ops.project(t) == ops.iso.ISO_ERR_ARG, change


def test_sizes_that_are_too_large(ops):
    large = ops.iso.ISO_ERR_TOO_LARGE
    assert ops.forward(ops.norm(channels=16385)) == large and ops.forward(ops.norm(heads=65537)) == large
    assert ops.forward(ops.norm(n=2 ** 32)) == large
    assert ops.drop(ops.dropout(n=2 ** 30)) == large and ops.drop(ops.dropout(n=2 ** 60)) == large
    for change in (dict(channels=2 ** 20 + 1), dict(hidden=2 ** 20 + 1), dict(n=2 ** 30)):
        t = ops.gated()
        for k, v in change.items():
            setattr(t, k, v)
        assert ops.project(t) == large, change
    size = ctypes.c_size_t()
    assert ops.lib.iso_gated_backward_workspace_bytes(2 ** 30, C, F, 0, ctypes.byref(size)) == large
    assert ops.lib.iso_layer_norm_backward_workspace_bytes(1, 1, 16385, 0, ctypes.byref(size)) == large
    t = ops.gated()
    t.gate.stride = 1 << 59
    assert ops.project(t) == large


def test_bad_tensors(ops):
    iso = ops.iso
    host = np.zeros(N * H * C, np.float32)
    calls = [(ops.norm, ops.forward, ("x", "out"), "rank_stride"), (ops.dropout, ops.drop, ("x", "out", "residual"), "stride"),
             (ops.gated, ops.project, ("x", "gate", "up", "out"), "stride"),
             (ops.gated, lambda t: ops.project_back(t, ops.gated_grads()), ("x", "gate", "up"), "stride"),
             (ops.norm, lambda t: ops.backward(t, ops.norm_grads()), ("x",), "rank_stride")]
    for make, call, names, stride in calls:
        for name in names:
            changes = [({stride: -1}, iso.ISO_ERR_ARG), ({stride: 100 * H * C}, iso.ISO_ERR_POINTER), (dict(data=host.ctypes.data), iso.ISO_ERR_POINTER)]
            if name != "residual":
                changes.append((dict(data=None), iso.ISO_ERR_ARG))
            for change, want in changes:
                t = make()
                for k, v in change.items():
                    setattr(getattr(t, name), k, v)
                assert call(t) == want, (name, change)
            t = make()
            getattr(t, name).data += 2                             # half an element
            assert call(t) == iso.ISO_ERR_ARG, name
    for name in ("grad_out", "grad_x", "grad_gate", "grad_up"):
        g = ops.gated_grads()
        getattr(g, name).data = None
        assert ops.project_back(ops.gated(), g) == iso.ISO_ERR_ARG, name
    for name in ("mean", "rstd"):
        assert ops.backward(ops.norm(**{name: None}), ops.norm_grads()) == iso.ISO_ERR_ARG
    assert ops.backward(ops.norm(weight=None), ops.norm_grads()) == iso.ISO_ERR_ARG       # a gradient of what is not there


def test_null_handles(ops):
    arg, h = ops.iso.ISO_ERR_ARG, ctypes.byref(ctypes.c_void_p())
    assert ops.lib.iso_layer_norm_init(None, h) == arg and ops.lib.iso_dropout_init(None, h) == arg and ops.lib.iso_gated_init(None, h) == arg
    assert ops.lib.iso_layer_norm_backward_init(ctypes.byref(ops.norm()), None, None, 0, h) == arg
    assert ops.lib.iso_gated_backward_init(ctypes.byref(ops.gated()), None, None, 0, h) == arg
    assert ops.lib.iso_layer_norm_init(ctypes.byref(ops.norm()), None) == arg
    assert ops.lib.iso_dropout_init(ctypes.byref(ops.dropout()), None) == arg
    assert ops.lib.iso_gated_init(ctypes.byref(ops.gated()), None) == arg
    assert ops.lib.iso_layer_norm_backward_workspace_bytes(N, H, C, 0, None) == arg
    assert ops.lib.iso_gated_backward_workspace_bytes(N, C, F, 0, None) == arg


def test_overlaps_and_what_may_be_in_place(ops):
    meet = ops.iso.ISO_ERR_OVERLAP
    t = ops.norm()
    t.out = t.x
    assert ops.forward(t) == 0
    t.out = ops.b.iso_heads_t(t.x.data + 4, t.x.rank_stride, t.x.head_stride)
    assert ops.forward(t) in (meet, ops.iso.ISO_ERR_POINTER)
    t = ops.norm()
    t.mean = t.rstd
    assert ops.forward(t) == meet
    t = ops.norm()
    t.out.head_stride = C - 1                                      # rows of the result share elements
    assert ops.forward(t) == meet
    t, g = ops.norm(), ops.norm_grads()
    g.grad_x = g.grad_out
    assert ops.backward(t, g) == 0
    g.grad_x = t.x
    assert ops.backward(t, g) == meet
    g = ops.norm_grads()
    g.grad_bias = g.grad_weight
    assert ops.backward(ops.norm(), g) == meet
    for name in ("x", "residual"):
        t = ops.dropout()
        t.out = getattr(t, name)
        assert ops.drop(t) == 0
    t = ops.dropout()
    t.x = t.residual = t.out
    assert ops.drop(t) == 0
    t = ops.dropout(n=N - 1)
    t.out = ops.b.iso_rows_t(t.x.data + 4 * C, C)                  # one row on
    assert ops.drop(t) == meet
    t = ops.dropout()
    t.seed = t.out.data
    assert ops.drop(t) == meet
    t = ops.dropout()
    t.out.stride = 0
    assert ops.drop(t) == meet
    t = ops.gated()
    t.up = t.gate
    assert ops.project(t) == 0
    t.out = t.x
    assert ops.project(t) in (meet, ops.iso.ISO_ERR_POINTER)
    t, g = ops.gated(), ops.gated_grads()
    g.grad_x = t.x
    assert ops.project_back(t, g) == meet
    g = ops.gated_grads()
    g.grad_up = g.grad_gate
    assert ops.project_back(ops.gated(), g) == meet
    t = ops.gated()
    t.x.stride = 0                                                 # an input's row repeated
    assert ops.project(t) == 0


def test_partial_overlaps(ops):
    """Inside one buffer that holds both, so that nothing but the overlap is wrong."""
    meet, rows, heads = ops.iso.ISO_ERR_OVERLAP, ops.b.iso_rows_t, ops.b.iso_heads_t
    size = N * H * C * 4
    for on, want in ((4, meet), (C * 4, meet), (H * C * 4, meet), (size - 4, meet), (size, 0)):
        both = ops.alloc(2 * size)
        for x, out in ((both, both + on), (both + on, both)):
            assert ops.forward(ops.norm(x=heads(x, H * C, C), out=heads(out, H * C, C))) == want, on
            assert ops.backward(ops.norm(x=heads(x, H * C, C)), ops.norm_grads(grad_x=heads(out, H * C, C))) == want, on
            assert ops.backward(ops.norm(), ops.norm_grads(grad_out=heads(x, H * C, C), grad_x=heads(out, H * C, C))) == want, on
    size = N * C * 4
    for on, want in ((4, meet), (C * 4, meet), (size - 4, meet), (size, 0)):
        both = ops.alloc(2 * size)
        for name in ("x", "residual"):
            for x, out in ((both, both + on), (both + on, both)):
                assert ops.drop(ops.dropout(**{name: rows(x, C), "out": rows(out, C)})) == want, (name, on)
    length = {"x": N * C * 4, "gate": F * C * 4, "up": F * C * 4, "out": N * F * 4, "grad_out": N * F * 4, "grad_x": N * C * 4,
              "grad_gate": F * C * 4, "grad_up": F * C * 4}
    width = {"out": F, "grad_out": F}
    for name in ("x", "gate", "up"):
        for on, want in ((-4, meet), (4 - length["out"], meet), (-length["out"], 0), (4, meet), (length[name] - 4, meet), (length[name], 0)):
            at = ops.alloc(3 * length["out"]) + length["out"]
            assert ops.project(ops.gated(**{name: rows(at, C), "out": rows(at + on, F)})) == want, (name, on)
    # a gradient over an operand, or over another gradient
    for name in ("grad_x", "grad_gate", "grad_up"):
        for other in ("x", "gate", "up", "grad_out", "grad_x", "grad_gate", "grad_up"):
            if other == name:
                continue
            for on, want in ((4, meet), (length[other] - 4, meet), (length[other], 0)):
                at = ops.alloc(length[other] + length[name])
                t, g = ops.gated(), ops.gated_grads()
                setattr(g if other.startswith("grad") else t, other, rows(at, width.get(other, C)))
                setattr(g, name, rows(at + on, C))
                assert ops.project_back(t, g) == want, (name, other, on)
    # a workspace over an operand's end, and behind it
    need = ops.bytes_of("iso_gated_backward_workspace_bytes", N, C, F, 0)
    for name in ("x", "gate", "up", "grad_out", "grad_x", "grad_gate", "grad_up"):
        at, t, g = ops.alloc(length[name] + need), ops.gated(), ops.gated_grads()
        setattr(g if name.startswith("grad") else t, name, rows(at, width.get(name, C)))
        assert ops.project_back(t, g, work=at + length[name] - 16) == meet and ops.project_back(t, g, work=at + length[name]) == 0, name
    need, size = ops.bytes_of("iso_layer_norm_backward_workspace_bytes", N, H, C, 0), N * H * C * 4
    for name in ("x", "grad_out", "grad_x"):
        at, t, g = ops.alloc(size + need), ops.norm(), ops.norm_grads()
        setattr(g if name.startswith("grad") else t, name, heads(at, H * C, C))
        assert ops.backward(t, g, work=at + size - 4) == meet and ops.backward(t, g, work=at + size) == 0, name


def test_slices_of_one_buffer(ops):
    """Weights and their gradients side by side in rows of one buffer."""
    both, grads = ops.alloc(F * 2 * C * 4), ops.alloc(F * 2 * C * 4)
    t, g = ops.gated(), ops.gated_grads()
    t.gate, t.up = ops.b.iso_rows_t(both, 2 * C), ops.b.iso_rows_t(both + C * 4, 2 * C)
    g.grad_gate, g.grad_up = ops.b.iso_rows_t(grads, 2 * C), ops.b.iso_rows_t(grads + C * 4, 2 * C)
    assert ops.project_back(t, g) == 0
    g.grad_up.data -= 4
    assert ops.project_back(t, g) == ops.iso.ISO_ERR_OVERLAP


def test_workspaces(ops):
    iso = ops.iso
    assert ops.backward(ops.norm(), ops.norm_grads(), size=16) == iso.ISO_ERR_WORKSPACE
    assert ops.backward(ops.norm(), ops.norm_grads(), work=None) == iso.ISO_ERR_WORKSPACE
    assert ops.project_back(ops.gated(), ops.gated_grads(), size=16) == iso.ISO_ERR_WORKSPACE
    assert ops.project_back(ops.gated(), ops.gated_grads(), work=None) == iso.ISO_ERR_WORKSPACE
    need = ops.bytes_of("iso_gated_backward_workspace_bytes", N, C, F, 0)
    assert ops.project_back(ops.gated(), ops.gated_grads(), work=ops.alloc(need + 8) + 8) == iso.ISO_ERR_ARG       # not on 16 bytes
    t = ops.gated()
    assert ops.project_back(t, ops.gated_grads(), work=t.x.data) in (iso.ISO_ERR_OVERLAP, iso.ISO_ERR_POINTER)
    size = ctypes.c_size_t()
    for bad in ((-1, H, C, 0), (N, 0, C, 0), (N, H, 0, 0), (N, H, C, 5)):
        assert ops.lib.iso_layer_norm_backward_workspace_bytes(*bad, ctypes.byref(size)) == iso.ISO_ERR_ARG
    for bad in ((-1, C, F, 0), (N, 0, F, 0), (N, C, 0, 0), (N, C, F, 5)):
        assert ops.lib.iso_gated_backward_workspace_bytes(*bad, ctypes.byref(size)) == iso.ISO_ERR_ARG


@pytest.mark.parametrize("heads", [1, 3, 31, 300, 509, 4099, 4100, 65521, 65536])
def test_workspaces_of_norms_do_not_grow_with_the_heads(ops, heads):
    """One part of the sums for every 256 threads at most, 512 of them, or 1024 of 128."""
    for dtype in (0, 1, 2):
        for channels in (1, 24, 128, 1000, 1500, 3000, 16384):
            for n in (0, 1, 2, 50, 60000):
                need = ops.bytes_of("iso_layer_norm_backward_workspace_bytes", n, heads, channels, dtype)
                assert need <= 1024 * 2 * channels * 4, (dtype, channels, n, need)


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_kernels_of_projections(ops, dtype):
    few = ops.gated(n=64, dtype=dtype)
    assert ops.project(few, started=True) == ["gated_few"]
    assert ops.project(ops.gated(n=65, dtype=dtype), started=True) == ["product"]
    assert ops.project(ops.gated(n=65, channels=23, dtype=dtype), started=True) == ["product"]
    back = lambda started=True, **kw: ops.project_back(ops.gated(dtype=dtype, **kw), ops.gated_grads(dtype=dtype, **{k: v for k, v in kw.items() if k != "shift"}),  # noqa: E731
                                                       started=started)
    assert back(n=1) == ["gated_few", "product", "product"]
    assert back(n=90) == ["product"] * 3
    assert back(n=90, channels=23) == ["align_rows"] + ["product"] * 3
    assert back(n=90, shift=1) == ["align_rows"] + ["product"] * 3
    assert back(n=20, channels=23) == ["align_rows", "gated_few", "product", "product"]
    # a long axis and few tiles: parts, and their sum
    assert back(n=20000) == ["product"] * 3 + ["product_sum"]


def test_rows_far_apart_are_copied_first(ops):
    t, stride = ops.gated(n=90), 1 << 22                           # 2^24 bytes
    t.gate = ops.b.iso_rows_t(ops.alloc(((F - 1) * stride + C) * 4), stride)
    assert ops.project_back(t, ops.gated_grads(n=90), started=True) == ["align_rows"] + ["product"] * 3
    assert ops.project(t, started=True) == ["product"]


def test_binding_refuses(ops):
    torch = pytest.importorskip("torch")
    iso = ops.iso
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    for bad in (lambda: iso.iso_layer_norm_init(torch.zeros(3), torch.zeros(3)), lambda: iso.iso_layer_norm_init(x, torch.zeros(4, 9)),
                lambda: iso.iso_layer_norm_init(x, x.double()), lambda: iso.iso_layer_norm_init(x, x, weight=torch.zeros(7)),
                lambda: iso.iso_layer_norm_init(x.t(), x.t()), lambda: iso.iso_layer_norm_init(x, x, mean=torch.zeros(5)),
                lambda: iso.iso_dropout_init(x, x, torch.zeros(2), 0.1), lambda: iso.iso_dropout_init(x, x, torch.zeros(3, dtype=torch.int64), 0.1),
                lambda: iso.iso_dropout_init(torch.zeros(4), x, torch.zeros(2, dtype=torch.int64), 0.1),
                lambda: iso.iso_gated_init(x, w, torch.zeros(5, 8), torch.zeros(4, 6)), lambda: iso.iso_gated_init(x, w, w, torch.zeros(4, 7)),
                lambda: iso.iso_gated_init(x, w, w, torch.zeros(4, 6), activation="tanh"), lambda: iso.iso_gated_init(x, w.half(), w, torch.zeros(4, 6)),
                lambda: iso.iso_gated_init(x, w.t().contiguous().t(), w, torch.zeros(4, 6))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        iso.iso_dropout_init(x.double(), x.double(), torch.zeros(2, dtype=torch.int64), 0.1)


def test_gpu_tests_take_every_kernel_of_the_projections(ops):
    taken = set()
    for shape in FEW + TILED + LARGE:
        for dtype in (0, 1, 2):
            o = Operands(ops.stub)
            t, g, h = o.gated(*shape, dtype), o.gated_grads(*shape, dtype), ctypes.c_void_p()
            need = o.bytes_of("iso_gated_backward_workspace_bytes", *shape, dtype)
            work = o.alloc(need)
            for call, args in (("iso_gated_init", (ctypes.byref(t),)), ("iso_gated_backward_init", (ctypes.byref(t), ctypes.byref(g), work, need))):
                assert getattr(o.lib, call)(*args, ctypes.byref(h)) == 0
                ops.stub.lib.stub_log_clear()
                assert o.lib.iso_start(h, None) == 0
                for i in range(ops.stub.lib.stub_log_size()):
                    name = ops.stub.lib.stub_log_name(i).decode()
                    m = re.search(r"\d(product|gated_few|align_rows|product_sum)_kernelI(f|DF16b|DF16_)", name)
                    numbers = re.search(r"ProductKindE(\d)ENS_\d+ProductTileILi(\d)ELi\dELi(\d)ELi\dEEELb(\d)", name)
                    few = re.search(r"Li(\d)ELb(\d)ELb(\d)", name)
                    taken.add((m[1], m[2], *(numbers.groups() if m[1] == "product" else few.groups() if m[1] == "gated_few" else ())))
                assert o.lib.iso_request_free(ctypes.byref(h)) == 0
            o.free()
    large, middle, small = ("4", "4"), ("2", "4"), ("2", "2")
    want = set()
    for dtype, tiles in (("f", (middle, small)), ("DF16b", (large, middle, small)), ("DF16_", (large, middle, small))):
        want |= {("align_rows", dtype), ("product_sum", dtype)}
        want |= {("product", dtype, kind, *tile, "1") for kind in "0123" for tile in tiles}
        want |= {("product", dtype, "0", *tile, "0") for tile in tiles}
        want |= {("gated_few", dtype, groups, backward, direct) for groups in "124" for backward in "01" for direct in "01"}
    assert taken == want, (want - taken, taken - want)


def test_gpu_tests_take_every_kernel_of_the_norm(ops):
    taken = set()
    for n, heads, channels in NORMS:
        for dtype in (0, 1, 2):
            o, h = Operands(ops.stub), ctypes.c_void_p()
            rows = lambda: o.b.iso_heads_t(o.alloc(n * heads * channels * SIZE[dtype]), heads * channels, channels)       # noqa: E731
            t = o.b.iso_layer_norm_t(dtype=dtype, heads=heads, channels=channels, n=n, eps=1e-5, x=rows(), out=rows())
            t.weight, t.bias = o.alloc(channels * 4), o.alloc(channels * 4)
            t.mean, t.rstd = o.alloc(n * heads * 4), o.alloc(n * heads * 4)
            need = o.bytes_of("iso_layer_norm_backward_workspace_bytes", n, heads, channels, dtype)
            g = [o.b.iso_layer_norm_grads_t(rows(), rows(), *sums) for sums in ((o.alloc(channels * 4), o.alloc(channels * 4)), (None, None))]
            work = o.alloc(need)
            for call, args in (("iso_layer_norm_init", (ctypes.byref(t),)),
                               ("iso_layer_norm_backward_init", (ctypes.byref(t), ctypes.byref(g[0]), work, need)),
                               ("iso_layer_norm_backward_init", (ctypes.byref(t), ctypes.byref(g[1]), None, 0))):
                assert getattr(o.lib, call)(*args, ctypes.byref(h)) == 0
                ops.stub.lib.stub_log_clear()
                assert o.lib.iso_start(h, None) == 0
                for i in range(ops.stub.lib.stub_log_size()):
                    m = re.search(r"\d(layer_norm\w*?)_kernelI(f|DF16b|DF16_)(?:Lb(\d)ELi(\d)ELi(\d+)E(?:Lb(\d))?)?", ops.stub.lib.stub_log_name(i).decode())
                    taken.add(tuple(v for v in m.groups() if v is not None))
                assert o.lib.iso_request_free(ctypes.byref(h)) == 0
            o.free()
    want = set()
    for dtype, most in (("f", "4"), ("DF16b", "2"), ("DF16_", "2")):
        want.add(("layer_norm_sum", dtype))
        for wide in "01":
            for units, lanes in {("1", "8"), ("2", "8"), (most, "8"), (most, "16"), (most, "32"), (most, "64"), (most, "0")}:
                want.add(("layer_norm", dtype, wide, units, lanes))
                want |= {("layer_norm_backward", dtype, wide, units, lanes, sums) for sums in "01"}
    assert taken == want, (want - taken, taken - want)


def test_gpu_tests_take_every_kernel_of_the_norm_that_moves_from_head_to_head(ops):
    taken = set()
    for n, heads, channels in MANY_HEADS:
        for dtype in (0, 1, 2):
            o, h = Operands(ops.stub), ctypes.c_void_p()
            rows = lambda: o.b.iso_heads_t(o.alloc(n * heads * channels * SIZE[dtype]), heads * channels, channels)       # noqa: E731
            t = o.b.iso_layer_norm_t(dtype=dtype, heads=heads, channels=channels, n=n, x=rows(), weight=o.alloc(channels * 4))
            t.mean, t.rstd = o.alloc(n * heads * 4), o.alloc(n * heads * 4)
            g = o.b.iso_layer_norm_grads_t(rows(), rows(), o.alloc(channels * 4), o.alloc(channels * 4))
            need = o.bytes_of("iso_layer_norm_backward_workspace_bytes", n, heads, channels, dtype)
            assert o.lib.iso_layer_norm_backward_init(ctypes.byref(t), ctypes.byref(g), o.alloc(need), need, ctypes.byref(h)) == 0
            ops.stub.lib.stub_log_clear()
            assert o.lib.iso_start(h, None) == 0
            name = ops.stub.lib.stub_log_name(0).decode()
            m = re.search(r"layer_norm_backward_kernelI(f|DF16b|DF16_)Lb(\d)ELi(\d)ELi(\d+)ELb1ELb1E", name)
            assert m, name
            taken.add(m.groups())
            assert o.lib.iso_request_free(ctypes.byref(h)) == 0
            o.free()
    want = {(dtype, wide, *of) for dtype, most in (("f", "4"), ("DF16b", "2"), ("DF16_", "2")) for wide in "01"
            for of in {("1", "8"), ("2", "8"), (most, "8"), (most, "16"), (most, "32"), (most, "64"), (most, "0")}}
    assert taken == want, (want - taken, taken - want)
