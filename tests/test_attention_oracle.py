"""The oracle of attention and rotary positions against cases whose result is known, and its gradients against differences."""
import numpy as np
import pytest

import iso_inputs as gen
from oracle import attention_oracle as orc
from oracle import iso_oracle


@pytest.mark.parametrize("dims,periodic", [((5, 4, 3), None), ((4, 6), None), ((7,), None)])
def test_neighbours_are_the_allgather_sources(dims, periodic):
    offsets = gen.moore(len(dims), 1) + [(0,) * len(dims), (2,) * len(dims), (1,) * len(dims)]
    p = int(np.prod(dims))
    want = iso_oracle.source_ranks(dims, offsets, np.arange(p))
    assert np.array_equal(orc.neighbours(dims, offsets, periodic), want)


def test_neighbours_of_a_mesh():
    assert orc.neighbours((4,), [(1,), (0,), (-9,)], [False]).tolist() == [[-1, 0, -1], [0, 1, -1], [1, 2, -1], [2, 3, -1]]


def test_one_neighbour_is_copied_and_none_gives_zero():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((6, 2, 5)) for _ in range(3))
    a = orc.Attention((6,), [(1,)], q, k, v)
    assert np.allclose(a.out, np.roll(v, 1, axis=0)) and np.allclose(a.lse, a.scale * (q * np.roll(k, 1, axis=0)).sum(-1))
    a = orc.Attention((6,), [(1,)], q, k, v, segments=np.array([0, 1, 2, 3, -1, -1]))
    assert not a.out.any() and np.all(np.isneginf(a.lse))
    a = orc.Attention((6,), [(1,), (2,)], q, k, v, bias=np.full((2, 2), -np.inf))
    assert not a.out.any() and np.all(np.isneginf(a.lse)) and not a.backward(np.ones_like(q))["grad_v"][0].any()


@pytest.mark.parametrize("cap", [0.0, 1.5])
@pytest.mark.parametrize("periodic", [None, [False, True]])
def test_gradients_against_differences(cap, periodic):
    rng = np.random.default_rng(2)
    dims, offsets = (3, 4), gen.moore(2, 1) + [(0, 0), (0, 1)]
    q, k, v = rng.standard_normal((12, 4, 6)), rng.standard_normal((12, 2, 6)), rng.standard_normal((12, 2, 6))
    bias, g = rng.standard_normal((4, len(offsets))), rng.standard_normal((12, 4, 6))
    seg = np.array([0, 0, 0, 0, 0, 1, 1, 1, -1, 0, 1, 0])
    loss = lambda q, k, v, b: (orc.Attention(dims, offsets, q, k, v, periodic=periodic, bias=b, segments=seg, cap=cap).out * g).sum()  # noqa: E731
    grads = orc.Attention(dims, offsets, q, k, v, periodic=periodic, bias=bias, segments=seg, cap=cap).backward(g)
    at = [q, k, v, bias]
    for i, name in enumerate(("grad_q", "grad_k", "grad_v", "grad_bias")):
        step = rng.standard_normal(at[i].shape)
        h = 1e-5
        hi, lo = (loss(*[x + sign * h * step if j == i else x for j, x in enumerate(at)]) for sign in (1, -1))
        want = (grads[name][0] * step).sum()
        assert abs((hi - lo) / (2 * h) - want) < 1e-7 * max(1, abs(want)), name


def test_rotary_keeps_lengths_and_its_inverse_is_its_transpose():
    rng = np.random.default_rng(3)
    x, y = rng.standard_normal((7, 2, 14)), rng.standard_normal((7, 2, 14))
    at = rng.integers(-50, 50, (7, 3))
    freqs, axes = orc.ladder(6, 3)
    for interleaved in (False, True):
        turned = orc.rotary(x, at, freqs, axes, interleaved=interleaved)
        assert np.allclose((turned ** 2).sum(), (x ** 2).sum()) and np.array_equal(turned[..., 12:], x[..., 12:])
        back = orc.rotary(y, at, freqs, axes, interleaved=interleaved, inverse=True)
        assert np.allclose((turned * y).sum(), (x * back).sum())
        assert np.allclose(orc.rotary(turned, at, freqs, axes, interleaved=interleaved, inverse=True), x)
