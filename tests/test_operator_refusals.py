"""What the operators on the ranks' tokens refuse, and what their requests are, without a GPU (see stub_library.py)."""
import ctypes
import math

import numpy as np
import pytest

import iso_inputs as gen

DIMS, NQ, NK, D = (4, 6), 4, 2, 16
P = math.prod(DIMS)
OFFSETS = gen.moore(2, 1)
S = len(OFFSETS)


class Operands:
    """Descriptors over stand-in device buffers, float32, dense."""

    def __init__(self, lib):
        self.b = lib.iso.binding if hasattr(lib.iso, "binding") else __import__("sys").modules["iso_on_stub.binding"]
        self.iso, self.lib = lib.iso, lib.lib
        self.owned = []

    def alloc(self, n):
        q = self.lib.stub_device_alloc(n)
        self.owned.append(q)
        return q

    def heads(self, heads, n=P, at=None):
        return self.b.iso_heads_t(self.alloc(n * heads * D * 4) if at is None else at, heads * D, D)

    def attention(self, **change):
        t = self.b.iso_attention_t(dtype=self.iso.ISO_DTYPE_F32, q_heads=NQ, kv_heads=NK, head_dim=D, scale=0.25, cap=0.0)
        t.q, t.out, t.k, t.v = self.heads(NQ), self.heads(NQ), self.heads(NK), self.heads(NK)
        t.lse, t.bias, t.segments = self.alloc(P * NQ * 4), self.alloc(NQ * S * 4), self.alloc(P * 4)
        for k, v in change.items():
            setattr(t, k, v)
        return t

    def grads(self, **change):
        g = self.b.iso_attention_grads_t(grad_bias=self.alloc(NQ * S * 4))
        g.grad_out, g.grad_q, g.grad_k, g.grad_v = self.heads(NQ), self.heads(NQ), self.heads(NK), self.heads(NK)
        for k, v in change.items():
            setattr(g, k, v)
        return g

    def free(self):
        for q in self.owned:
            self.lib.stub_device_free(q)


@pytest.fixture
def ops(stub_library):
    o = Operands(stub_library)
    o.comm = stub_library.comm(DIMS, OFFSETS)
    o.raw = stub_library.iso.load_library()
    yield o
    o.free()


def forward(ops, t, comm=True):
    h = ctypes.c_void_p(1)
    st = ops.raw.iso_neighbor_attention_init(ctypes.byref(t), ops.comm.handle if comm else None, ctypes.byref(h))
    if st == ops.iso.ISO_SUCCESS:
        assert ops.raw.iso_request_free(ctypes.byref(h)) == 0
    assert not h.value
    return st


def backward(ops, t, g, size=None, work=None):
    need = ctypes.c_size_t()
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(ops.comm.handle, 0, NQ, NK, D, 1, ctypes.byref(need)) == 0
    size = need.value if size is None else size
    work = ops.alloc(need.value) if work is None else work
    h = ctypes.c_void_p(1)
    st = ops.raw.iso_neighbor_attention_backward_init(ctypes.byref(t), ctypes.byref(g), work, size, ops.comm.handle, ctypes.byref(h))
    if st == ops.iso.ISO_SUCCESS:
        assert ops.raw.iso_request_free(ctypes.byref(h)) == 0
    assert not h.value
    return st


def test_what_is_taken(ops):
    iso = ops.iso
    assert forward(ops, ops.attention()) == iso.ISO_SUCCESS
    assert forward(ops, ops.attention(lse=None, bias=None, segments=None, cap=2.0)) == iso.ISO_SUCCESS
    assert backward(ops, ops.attention(), ops.grads()) == iso.ISO_SUCCESS
    assert backward(ops, ops.attention(bias=None), ops.grads(grad_bias=None)) == iso.ISO_SUCCESS
    t = ops.attention(rows=ops.alloc(3 * 8), n_rows=3)
    t.q, t.out, t.lse = ops.heads(NQ, 3), ops.heads(NQ, 3), ops.alloc(3 * NQ * 4)
    assert forward(ops, t) == iso.ISO_SUCCESS


@pytest.mark.parametrize("change", [dict(dtype=3), dict(dtype=-1), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0),
                                    dict(cap=-1.0), dict(cap=math.inf), dict(cap=math.nan), dict(scale=math.nan), dict(scale=math.inf),
                                    dict(n_rows=-1), dict(n_rows=2)], ids=str)
def test_bad_values(ops, change):
    assert forward(ops, ops.attention(**change)) == ops.iso.ISO_ERR_ARG


def test_sizes_that_are_too_large(ops):
    iso = ops.iso
    assert forward(ops, ops.attention(head_dim=257)) == iso.ISO_ERR_TOO_LARGE
    assert forward(ops, ops.attention(q_heads=65538)) == iso.ISO_ERR_TOO_LARGE
    t = ops.attention()
    t.k.rank_stride = 1 << 59
    assert forward(ops, t) == iso.ISO_ERR_TOO_LARGE
    t = ops.attention(rows=ops.alloc(64), n_rows=1 << 31)
    assert forward(ops, t) == iso.ISO_ERR_TOO_LARGE


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_bad_tensors(ops, name):
    iso = ops.iso
    for change, want in ((dict(data=None), iso.ISO_ERR_ARG), (dict(rank_stride=-1), iso.ISO_ERR_ARG), (dict(head_stride=-16), iso.ISO_ERR_ARG),
                         (dict(rank_stride=10 * NQ * D), iso.ISO_ERR_POINTER)):
        t = ops.attention()
        for k, v in change.items():
            setattr(getattr(t, name), k, v)
        assert forward(ops, t) == want, change
    t = ops.attention()
    getattr(t, name).data += 2                                     # half an element
    assert forward(ops, t) == iso.ISO_ERR_ARG
    t = ops.attention()
    host = np.zeros(P * NQ * D, np.float32)
    getattr(t, name).data = host.ctypes.data
    assert forward(ops, t) == iso.ISO_ERR_POINTER


def test_null_handles(ops):
    iso = ops.iso
    assert forward(ops, ops.attention(), comm=False) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_init(None, ops.comm.handle, ctypes.byref(ctypes.c_void_p())) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_init(ctypes.byref(ops.attention()), ops.comm.handle, None) == iso.ISO_ERR_ARG
    assert ops.raw.iso_rotary_init(None, ops.comm.handle, ctypes.byref(ctypes.c_void_p())) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(ops.comm.handle, 0, NQ, NK, D, 1, None) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(None, 0, NQ, NK, D, 1, ctypes.byref(ctypes.c_size_t())) == iso.ISO_ERR_ARG
    assert backward(ops, ops.attention(lse=None), ops.grads()) == iso.ISO_ERR_ARG
    assert backward(ops, ops.attention(bias=None), ops.grads()) == iso.ISO_ERR_ARG      # a gradient of what is not there
    assert backward(ops, ops.attention(rows=ops.alloc(8), n_rows=1), ops.grads()) == iso.ISO_ERR_ARG


def test_overlaps(ops):
    iso = ops.iso
    t = ops.attention()
    t.out = t.q
    assert forward(ops, t) == iso.ISO_ERR_OVERLAP
    t = ops.attention()
    t.lse = t.k.data
    assert forward(ops, t) == iso.ISO_ERR_OVERLAP
    t = ops.attention()
    t.out.head_stride = D - 1                                      # rows of the result share elements
    assert forward(ops, t) == iso.ISO_ERR_OVERLAP
    g = ops.grads()
    g.grad_k = g.grad_v
    assert backward(ops, ops.attention(), g) == iso.ISO_ERR_OVERLAP
    t, g = ops.attention(), ops.grads()
    g.grad_q = t.out
    assert backward(ops, t, g) == iso.ISO_ERR_OVERLAP
    assert backward(ops, t, ops.grads(), work=t.q.data, size=1 << 20) in (iso.ISO_ERR_OVERLAP, iso.ISO_ERR_POINTER)


@pytest.mark.parametrize("head_major", [False, True])
def test_slices_of_one_buffer_do_not_overlap(ops, head_major):
    heads, iso = NQ + 2 * NK, ops.iso
    def cut(base, first):
        return (ops.b.iso_heads_t(base + first * P * D * 4, D, P * D) if head_major else
                ops.b.iso_heads_t(base + first * D * 4, heads * D, D))
    t, g = ops.attention(), ops.grads()
    base, into = ops.alloc(P * heads * D * 4), ops.alloc(P * heads * D * 4)
    t.q, t.k, t.v = cut(base, 0), cut(base, NQ), cut(base, NQ + NK)
    g.grad_q, g.grad_k, g.grad_v = cut(into, 0), cut(into, NQ), cut(into, NQ + NK)
    assert forward(ops, t) == iso.ISO_SUCCESS and backward(ops, t, g) == iso.ISO_SUCCESS
    g.grad_v = cut(into, NQ + NK - 1)                              # one head of another tensor
    assert backward(ops, t, g) == iso.ISO_ERR_OVERLAP
    # heads of q, k and v side by side: [p][heads][3 D]
    t, g = ops.attention(kv_heads=NQ), ops.grads()
    wide, into = ops.alloc(P * NQ * 3 * D * 4), ops.alloc(P * NQ * 3 * D * 4)
    part = lambda base, i: ops.b.iso_heads_t(base + i * D * 4, NQ * 3 * D, 3 * D)      # noqa: E731
    t.q, t.k, t.v = (part(wide, i) for i in range(3))
    g.grad_q, g.grad_k, g.grad_v = (part(into, i) for i in range(3))
    assert backward(ops, t, g) == iso.ISO_SUCCESS
    g.grad_v = part(into, 1)
    assert backward(ops, t, g) == iso.ISO_ERR_OVERLAP


def test_workspace(ops):
    iso = ops.iso
    assert backward(ops, ops.attention(), ops.grads(), size=16) == iso.ISO_ERR_WORKSPACE
    need = ctypes.c_size_t()
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(ops.comm.handle, 7, NQ, NK, D, 1, ctypes.byref(need)) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(ops.comm.handle, 0, NQ, 3, D, 1, ctypes.byref(need)) == iso.ISO_ERR_ARG
    assert ops.raw.iso_neighbor_attention_backward_workspace_bytes(ops.comm.handle, 0, NQ, NK, 300, 1, ctypes.byref(need)) == iso.ISO_ERR_TOO_LARGE


def test_rotary(ops):
    iso, b = ops.iso, ops.b
    freqs, axes = np.ones(D // 2), np.zeros(D // 2, np.int32)

    def call(comm=True, in_place=False, **change):
        t = b.iso_rotary_t(dtype=0, heads=NQ, head_dim=D, pairs=D // 2, n=P, freqs=freqs.ctypes.data, axes=axes.ctypes.data)
        t.x = ops.heads(NQ)
        t.out = t.x if in_place else ops.heads(NQ)
        for k, v in change.items():
            setattr(t, k, v)
        h = ctypes.c_void_p(1)
        st = ops.raw.iso_rotary_init(ctypes.byref(t), ops.comm.handle if comm else None, ctypes.byref(h))
        if st == 0:
            assert ops.raw.iso_request_free(ctypes.byref(h)) == 0
        assert not h.value
        return st

    assert call() == call(in_place=True) == call(pairs=0) == call(comm=False, positions=ops.alloc(P * 4), n_axes=1) == iso.ISO_SUCCESS
    assert call(comm=False, n=0) == iso.ISO_SUCCESS
    for change in (dict(pairs=D // 2 + 1), dict(pairs=-1), dict(n=P - 1), dict(n=-1), dict(dtype=5), dict(heads=0), dict(freqs=None), dict(axes=None),
                   dict(comm=False), dict(positions=ops.alloc(P * 4), n_axes=0)):
        assert call(**change) == iso.ISO_ERR_ARG, change
    assert call(head_dim=258) == iso.ISO_ERR_TOO_LARGE
    bad = np.full(D // 2, np.inf)
    assert call(freqs=bad.ctypes.data) == iso.ISO_ERR_ARG
    far = np.full(D // 2, 2, np.int32)
    assert call(axes=far.ctypes.data) == iso.ISO_ERR_ARG
    x = ops.heads(NQ)
    shifted = b.iso_heads_t(x.data + 4, x.rank_stride, x.head_stride)
    assert call(x=x, out=shifted) in (iso.ISO_ERR_OVERLAP, iso.ISO_ERR_POINTER)


def test_requests_of_operators(ops, stub_library):
    iso = ops.iso
    t, h = ops.attention(), ctypes.c_void_p()
    assert ops.raw.iso_neighbor_attention_init(ctypes.byref(t), ops.comm.handle, ctypes.byref(h)) == 0
    info, start, plan = ops.b.iso_request_info_t(), ops.b.iso_start_info_t(), ctypes.c_void_p()
    assert ops.raw.iso_request_info(h, ctypes.byref(info)) == 0 and info.op == iso.ISO_OP_ATTENTION and info.p == P and info.s == S
    assert ops.raw.iso_request_start_info(h, ctypes.byref(start)) == 0 and start.kernels == info.launches == 1
    assert ops.raw.iso_request_plan(h, ctypes.byref(plan)) == iso.ISO_ERR_ARG
    assert ops.raw.iso_start_range(h, 0, 2, None) == iso.ISO_ERR_ARG and ops.raw.iso_start_range(h, 0, 1, None) == 0
    for form in (iso.ISO_GRAPH_CHAIN, iso.ISO_GRAPH_BRANCHES, iso.ISO_GRAPH_OFF):
        assert ops.raw.iso_request_set_graph(h, form) == 0 and ops.raw.iso_start(h, None) == 0 and ops.raw.iso_wait(h) == 0
    assert ops.raw.iso_request_free(ctypes.byref(h)) == 0
    assert ops.raw.iso_plan_create(ops.comm.handle, iso.ISO_OP_ATTENTION, 0, ctypes.byref(plan)) == iso.ISO_ERR_ARG


def test_rows_without_elements_are_refused_from_python_too(ops):
    """head_dim 0 has no default scale; the library says what is wrong."""
    import torch
    x = torch.empty(P, 2, 0)
    with pytest.raises(ops.iso.IsoError) as e:
        ops.iso.iso_neighbor_attention_init(x, x, x, torch.empty_like(x), ops.comm)
    assert e.value.status == ops.iso.ISO_ERR_ARG
