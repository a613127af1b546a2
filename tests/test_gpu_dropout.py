"""Dropout against the definition: which elements are kept, exactly; their values inside the error that rounding allows."""
import numpy as np
import pytest
import torch

import paper_1606_07676_amd as iso
from oracle import token_oracle as orc
from token_rows import DEV, TYPES, U, host, inside_rows, untouched_around, within

pytestmark = pytest.mark.gpu

SEED = (0x0123456789ABCDEF, -5)


def seed_of(pair):
    return torch.tensor(pair, dtype=torch.int64, device=DEV)


def tensors(n, C, dtype, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    return [torch.randn(n, C, device=DEV, generator=g).to(TYPES[dtype]) for _ in range(2)]


def drop(x, rate, residual=None, out=None, seed=SEED, stream=None):
    out = torch.full_like(x, 7) if out is None else out
    req = iso.iso_dropout_init(x, out, seed_of(seed), rate, residual=residual)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    iso.iso_start(req, stream)
    iso.iso_wait(req)
    return out


def check(x, out, rate, dtype, residual=None, seed=SEED):
    n, C = x.shape
    keep, factor = orc.kept(n, C, seed, rate)
    x, out = host(x), host(out)
    base = np.zeros_like(x) if residual is None else host(residual)
    assert np.array_equal(out[~keep], base[~keep]), "what is dropped"
    y = x * factor
    # the factor's rounding, the product's and the sum's, in 32 bits
    bound = orc.rounded(base + y, orc.EPS * (3 * np.abs(y) + np.abs(base + y)), U[dtype])
    within(out[keep], (base + y)[keep], bound[keep], "what is kept")


@pytest.mark.parametrize("residual", [False, True], ids=["alone", "residual"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,C", [(1, 1), (1, 7), (1, 8), (2, 9), (3, 5), (40, 64), (63, 333), (700, 128), (5, 4097), (2000, 24)])
def test_dropout(n, C, dtype, residual):
    x, r = tensors(n, C, dtype)
    r = r if residual else None
    check(x, drop(x, 0.3, r), 0.3, dtype, r)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,gap,shift", [(64, 8, 0), (64, 3, 0), (61, 3, 0), (128, 0, 1), (13, 0, 5), (3, 2, 0)])
def test_rows_inside_larger_buffers(C, gap, shift, dtype):
    """The same elements are kept whatever the strides."""
    x, r = tensors(57, C, dtype, seed=1)
    dense = drop(x, 0.1, r)
    views = [inside_rows((57, C), x.dtype, gap, shift) for _ in range(3)]
    views[0].copy_(x)
    views[1].copy_(r)
    out = drop(views[0], 0.1, views[1], views[2])
    check(x, out, 0.1, dtype, r)
    check(x, dense, 0.1, dtype, r)
    untouched_around(out)


@pytest.mark.parametrize("rate", [0.0, 1e-6, 2.0 ** -16, 0.1, 0.5, 0.9, 1 - 2.0 ** -16, 1 - 1e-6, 1.0])
def test_rates(rate):
    x, r = tensors(300, 72, "f32", seed=2)
    check(x, drop(x, rate), rate, "f32")
    check(x, drop(x, rate, r), rate, "f32", r)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype):
    x, r = tensors(90, 100, dtype, seed=3)
    want, alone = drop(x, 0.2, r), drop(x, 0.2)
    over_x, over_r, over = x.clone(), r.clone(), x.clone()
    assert torch.equal(drop(over_x, 0.2, r, over_x), want)
    assert torch.equal(drop(x, 0.2, over_r, over_r), want)
    assert torch.equal(drop(over, 0.2, None, over), alone)
    both = x.clone()
    check(x, drop(both, 0.2, both, both), 0.2, dtype, x)


def test_what_is_dropped_may_hold_anything():
    x, r = tensors(64, 64, "f16", seed=4)
    keep = torch.from_numpy(orc.kept(64, 64, SEED, 0.5)[0]).to(DEV)
    clean = drop(x, 0.5, r)
    x[~keep] = float("nan")
    assert torch.equal(drop(x, 0.5, r), clean)


def test_seeds():
    x, _ = tensors(100, 64, "f32", seed=5)
    for seed in ((0, 0), (0, 1), (1, 0), (-1, -1), (2 ** 63 - 1, -2 ** 63), (2 ** 32, 5), (5, 2 ** 32)):
        check(x, drop(x, 0.5, seed=seed), 0.5, "f32", seed=seed)


def test_gradient_is_the_same_call():
    x, dy = tensors(50, 96, "f32", seed=6)
    keep, factor = orc.kept(50, 96, SEED, 0.25)
    within(host(drop(dy, 0.25)), host(dy) * keep * factor, 4 * orc.EPS * np.abs(host(dy)) * factor + 1e-30, "grad_x")


def test_no_tokens_and_another_stream():
    x, r = tensors(0, 24, "bf16")
    assert drop(x, 0.3, r).shape == (0, 24)
    x, r = tensors(500, 24, "bf16", seed=7)
    assert torch.equal(drop(x, 0.3, r, stream=torch.cuda.Stream()), drop(x, 0.3, r))


def test_the_seed_is_read_at_every_start():
    """One request, and one captured graph of it, draw anew when the program writes another seed."""
    x, r = tensors(200, 40, "f32", seed=8)
    seed, out = seed_of((7, 0)), torch.empty_like(x)
    req = iso.iso_dropout_init(x, out, seed, 0.4, residual=r)
    for step in range(3):
        seed[1] = step
        iso.iso_start(req)
        check(x, out, 0.4, "f32", r, (7, step))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iso.iso_start(req)
    for step in range(3, 7):
        seed[1] = step
        out.fill_(7)
        graph.replay()
        check(x, out, 0.4, "f32", r, (7, step))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counters_beyond_32_bits_of_elements(dtype):
    """Rows that are one row repeated: the last of 2^32 and more elements."""
    n, C = 2 ** 19 + 3, 8200
    x = torch.ones(1, C, device=DEV, dtype=TYPES[dtype]).expand(n, C)
    out = torch.empty(n, C, device=DEV, dtype=TYPES[dtype])
    drop(x, 0.5, out=out)
    words = orc.philox(np.arange((n - 1) * C // 8, n * C // 8), SEED[1] % 2 ** 64, SEED[0] % 2 ** 64)
    numbers = np.stack([words & 0xFFFF, words >> 16], -1).reshape(-1)
    assert (n - 1) * C % 8 == 0 and np.array_equal(host(out[-1]), np.where(numbers >= 32768, 2.0, 0.0))
