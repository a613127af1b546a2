"""Which tensors of an operator's call share bytes, on the CPU: every arrangement of slices against the bytes themselves."""
import ctypes
import itertools

import numpy as np
import pytest

import paper_1606_07676_amd as iso


@pytest.fixture
def overlap(stub_library):
    """(n, heads, D, x's place, out's place) -> status; a place is (first byte, rank stride, head stride), strides in elements."""
    import sys
    b, lib, owned = sys.modules["iso_on_stub.binding"], stub_library.iso.load_library(), []
    base = stub_library.lib.stub_device_alloc(1 << 20)

    def call(n, heads, D, x, out):
        t = b.iso_rotary_t(dtype=iso.ISO_DTYPE_F32, heads=heads, head_dim=D, n=n, positions=base, n_axes=0)
        t.x, t.out = (b.iso_heads_t(base + 4 * at, rank, head) for at, rank, head in (x, out))
        h = ctypes.c_void_p()
        st = lib.iso_rotary_init(ctypes.byref(t), None, ctypes.byref(h))
        if st == 0:
            lib.iso_request_free(ctypes.byref(h))
        return st
    yield call
    stub_library.lib.stub_device_free(base)


def elements(n, heads, D, place):
    at, rank, head = place
    return (at + rank * np.arange(n)[:, None, None] + head * np.arange(heads)[None, :, None] + np.arange(D)).ravel()


def test_slices_with_the_same_strides(overlap):
    """[p][heads][parts][D] and [heads][p][parts][D], and slices of ranks or heads of either."""
    n, heads, D = 5, 3, 4
    for parts, pad in itertools.product((1, 2, 3), (0, 4)):
        wide = parts * D + pad
        for rank, head in ((heads * wide, wide), (wide, n * wide), (heads * wide + 8, wide), (wide, n * wide + 12)):
            x = (0, rank, head)
            for at in range(0, 3 * max(rank, head), 2):
                out = (at, rank, head)
                if at == 0:
                    continue                                       # in place
                meet = np.intersect1d(elements(n, heads, D, x), elements(n, heads, D, out)).size > 0
                st = overlap(n, heads, D, x, out)
                if meet:
                    assert st == iso.ISO_ERR_OVERLAP, (x, out)
                elif at < wide:
                    assert st == iso.ISO_SUCCESS, (x, out)         # beside each other in what a rank's head has
                assert overlap(n, heads, D, out, x) == st          # either way round


def test_random_places(overlap):
    rng = np.random.default_rng(5)
    told_apart = 0
    for _ in range(4000):
        n, heads, D = rng.integers(1, 6, 3).tolist()
        rank, head = rng.integers(0, 40, 2).tolist()
        at = int(rng.integers(0, 120))
        x, out = (0, rank, head), (at, rank, head)
        mine = elements(n, heads, D, out)
        meet = np.intersect1d(elements(n, heads, D, x), mine).size > 0 and at > 0
        st = overlap(n, heads, D, x, out)
        if meet or np.unique(mine).size < mine.size:
            assert st == iso.ISO_ERR_OVERLAP, (n, heads, D, x, out)
        told_apart += st == iso.ISO_SUCCESS
    assert told_apart > 1000
