"""Layer norm and its gradients against the 64-bit oracle, element by element inside the error that rounding allows."""
import numpy as np
import pytest
import torch

import paper_1606_07676_amd as iso
from oracle import token_oracle as orc
from token_rows import DEV, TYPES, U, host, inside_rows, untouched_around, within
from token_shapes import MANY_HEADS, NORMS

pytestmark = pytest.mark.gpu


def tensors(shape, dtype, seed=0, offset=0.0, affine=True):
    n, heads, C = shape
    g = torch.Generator(DEV).manual_seed(seed)
    normal = lambda *size: torch.randn(*size, device=DEV, generator=g)  # noqa: E731
    t = {"x": (normal(n, heads, C) * 2 + offset).to(TYPES[dtype]), "dy": normal(n, heads, C).to(TYPES[dtype]), "weight": None, "bias": None}
    if affine:
        t |= {"weight": (1 + 0.3 * normal(C)).to(TYPES[dtype]), "bias": normal(C).to(TYPES[dtype])}
    return t


def flat(x):
    return None if x is None else host(x).reshape(-1, x.shape[-1])


def forward(t, out=None, eps=1e-5, stream=None):
    out = torch.full_like(t["x"], 7) if out is None else out
    mean, rstd = (torch.full(t["x"].shape[:-1], 7.0, device=DEV) for _ in range(2))
    req = iso.iso_layer_norm_init(t["x"], out, weight=t["weight"], bias=t["bias"], eps=eps, mean=mean, rstd=rstd)
    iso.iso_start(req, stream)
    iso.iso_wait(req)
    return out, mean, rstd


def backward(t, mean, rstd, sums=True, into=None, dy=None):
    x, dy = t["x"], t["dy"] if dy is None else dy
    n, heads, C = x.shape if x.dim() == 3 else (x.shape[0], 1, x.shape[1])
    grads = {"x": torch.full_like(dy, 7) if into is None else into, "weight": None, "bias": None}
    work = size = None
    if sums:
        grads["bias"] = torch.full((C,), 7.0, device=DEV, dtype=x.dtype)
        grads["weight"] = None if t["weight"] is None else torch.full_like(grads["bias"], 7)
        size = iso.iso_layer_norm_backward_workspace_bytes(n, heads, C, x.dtype)
        work = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    req = iso.iso_layer_norm_backward_init(x, mean, rstd, dy, grads["x"], work, weight=t["weight"], grad_weight=grads["weight"],
                                           grad_bias=grads["bias"], workspace_bytes=size)
    iso.iso_start(req)
    iso.iso_wait(req)
    assert work is None or bool((work[size:] == 0xA5).all()), "written behind the workspace"
    return grads


def check(t, dtype, out, mean, rstd, grads=None, eps=1e-5):
    u = U[dtype]
    weight, bias = (None if t[k] is None else host(t[k]) for k in ("weight", "bias"))
    o = orc.LayerNorm(flat(t["x"]), weight, bias, eps)
    within(flat(out), o.out, o.out_bound(u), "out")
    within(host(mean).reshape(-1), o.mean, o.mean_bound(), "mean")
    within(host(rstd).reshape(-1), o.rstd, o.rstd_bound(), "rstd")
    if grads is None:
        return
    o.backward(flat(t["dy"]))
    within(flat(grads["x"]), o.grad_x, orc.rounded(o.grad_x, o.grad_x_error, u), "grad_x")
    if grads["weight"] is not None:
        within(host(grads["weight"]), o.grad_weight, orc.rounded(o.grad_weight, o.grad_weight_error, u), "grad_weight")
    if grads["bias"] is not None:
        within(host(grads["bias"]), o.grad_bias, orc.rounded(o.grad_bias, o.grad_bias_error, u), "grad_bias")


@pytest.mark.parametrize("affine", [True, False], ids=["affine", "plain"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_norm_and_gradients(shape, dtype, affine):
    t = tensors(shape, dtype, affine=affine)
    out, mean, rstd = forward(t)
    check(t, dtype, out, mean, rstd, backward(t, mean, rstd, sums=affine))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,gap,shift", [((37, 3, 64), 16, 0), ((37, 3, 64), 1, 0), ((20, 1, 1024), 8, 3), ((21, 1, 100), 5, 1)], ids=str)
def test_rows_inside_larger_buffers(shape, gap, shift, dtype):
    """Any strides and addresses; what lies around the rows stays as it was."""
    t = tensors(shape, dtype, seed=1)
    for k in ("x", "dy"):
        rows = inside_rows(shape, t[k].dtype, gap, shift)
        rows.copy_(t[k])
        t[k] = rows
    out, into = inside_rows(shape, t["x"].dtype, gap, shift), inside_rows(shape, t["x"].dtype, gap, shift)
    out, mean, rstd = forward(t, out)
    check(t, dtype, out, mean, rstd, backward(t, mean, rstd, into=into))
    untouched_around(out)
    untouched_around(into)


@pytest.mark.parametrize("dtype", TYPES)
def test_heads_far_apart(dtype):
    """[heads][tokens][channels], as a permuted view."""
    t = tensors((19, 4, 72), dtype, seed=2)
    for k in ("x", "dy"):
        t[k] = t[k].permute(1, 0, 2).contiguous().permute(1, 0, 2)
    out, mean, rstd = forward(t, torch.empty_like(t["x"]))
    check(t, dtype, out, mean, rstd, backward(t, mean, rstd, into=torch.empty_like(t["x"])))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(33, 2, 72), (11, 1, 2048), (900, 1, 483), (40, 3, 9), (50, 2, 3), (700, 1, 5001)], ids=str)
def test_in_place(shape, dtype):
    t = tensors(shape, dtype, seed=3)
    out, mean, rstd = forward(t)
    grads = backward(t, mean, rstd)
    again = dict(t, x=t["x"].clone())
    over, mean2, _ = forward(again, again["x"])
    assert torch.equal(over, out) and torch.equal(mean2, mean)
    dy = t["dy"].clone()
    for name, value in backward(t, mean, rstd, into=dy, dy=dy).items():
        assert torch.equal(value, grads[name]), name


@pytest.mark.parametrize("shape", [(50, 1, 64), (9, 1, 1024), (4, 1, 3000)], ids=str)
def test_rows_far_from_zero(shape):
    """The mean is thousands of deviations away: what rounding of a plain sum would take from the distances."""
    t = tensors(shape, "f32", seed=4, offset=10000.0)
    out, mean, rstd = forward(t)
    check(t, "f32", out, mean, rstd, backward(t, mean, rstd))


def test_rows_that_are_constant_and_rows_that_are_not_numbers():
    t = tensors((12, 1, 96), "f32", seed=5)
    t["x"][3] = 2.5
    t["x"][7, 0, 5] = float("nan")
    t["x"][9, 0, 1] = float("inf")
    out, mean, rstd = forward(t)
    rows = [i for i in range(12) if i not in (7, 9)]
    part = {k: v[rows] if v.shape[0] == 12 else v for k, v in t.items()}
    check(part, "f32", out[rows], mean[rows], rstd[rows])
    assert torch.equal(out[3, 0], t["bias"]) and out[7].isnan().all() and out[9].isnan().all()
    assert rstd[7].isnan().all() and rstd[9].isnan().all()


def test_no_rows():
    t = tensors((0, 2, 24), "bf16")
    out, mean, rstd = forward(t)
    grads = backward(t, mean, rstd)
    assert not grads["weight"].any() and not grads["bias"].any()


def test_a_row_that_is_repeated():
    t = tensors((1, 1, 200), "f16", seed=6)
    t["x"] = t["x"].expand(30, 1, 200)
    t["dy"] = tensors((30, 1, 200), "f16", seed=7)["dy"]
    out, mean, rstd = forward(t, torch.empty(30, 1, 200, device=DEV, dtype=torch.float16))
    check(t, "f16", out, mean, rstd, backward(t, mean, rstd))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(dtype):
    """More rows than lanes take at once, to the same bits every time and on another stream."""
    t = tensors((70000, 1, 64), dtype, seed=8)
    out, mean, rstd = forward(t)
    grads = backward(t, mean, rstd)
    check(t, dtype, out, mean, rstd, grads)
    for name, value in backward(t, mean, rstd).items():
        assert torch.equal(value, grads[name]), name
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        assert torch.equal(forward(t, stream=other)[0], out)


def test_two_dimensions_stand_for_one_head():
    t = tensors((31, 1, 88), "bf16", seed=9)
    out, mean, rstd = forward(t)
    two = {k: v[:, 0] if v.dim() == 3 else v for k, v in t.items()}
    out2, mean2, rstd2 = forward(two)
    assert torch.equal(out2, out[:, 0]) and mean2.shape == (31,) and torch.equal(mean2, mean[:, 0]) and torch.equal(rstd2, rstd[:, 0])


def test_rows_beyond_32_bits_of_elements():
    """One row repeated, and all rows of the result: the last of 2^32 and more elements."""
    n, C = 2 ** 19 + 3, 8200
    x = tensors((1, 1, C), "bf16", seed=13)["x"][0].expand(n, C)
    out = torch.empty(n, C, device=DEV, dtype=torch.bfloat16)
    iso.iso_start(iso.iso_layer_norm_init(x, out))
    o = orc.LayerNorm(host(x[:1]))
    within(host(out[-1:]), o.out, o.out_bound(U["bf16"]), "last row")
    assert torch.equal(out[-1], out[0])


def test_without_statistics():
    t = tensors((31, 2, 88), "bf16", seed=10)
    out, _, _ = forward(t)
    alone = torch.empty_like(out)
    iso.iso_start(iso.iso_layer_norm_init(t["x"], alone, weight=t["weight"], bias=t["bias"]))
    torch.cuda.synchronize()
    assert torch.equal(alone, out)
    only = torch.empty_like(out)
    req = iso.iso_layer_norm_init(t["x"], only, weight=t["weight"])
    iso.iso_start(req)
    iso.iso_wait(req)
    o = orc.LayerNorm(flat(t["x"]), host(t["weight"]))
    within(flat(only), o.out, o.out_bound(U["bf16"]), "without a bias")


def test_gradient_against_differences():
    t = tensors((4, 1, 24), "f32", seed=11)
    out, mean, rstd = forward(t)
    grads = backward(t, mean, rstd)
    w, b, dy = host(t["weight"]), host(t["bias"]), flat(t["dy"])
    for name in ("x", "weight", "bias"):
        direction = np.random.default_rng(12).normal(size=t[name].shape)
        value = lambda s: float((orc.LayerNorm(flat(t["x"]) + (s * direction.reshape(-1, 24) if name == "x" else 0),  # noqa: E731
                                               w + (s * direction if name == "weight" else 0),
                                               b + (s * direction if name == "bias" else 0)).out * dy).sum())
        change = (value(1e-6) - value(-1e-6)) / 2e-6
        assert abs(change - float((host(grads[name]) * direction).sum())) < 1e-5 * np.abs(host(grads[name]) * direction).sum() + 1e-6, name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", MANY_HEADS, ids=str)
def test_many_heads_with_no_common_factor(shape, dtype):
    """More heads than workgroups that sum: a lane comes to other heads from row to row."""
    t = tensors(shape, dtype, seed=14)
    out, mean, rstd = forward(t)
    grads = backward(t, mean, rstd)
    check(t, dtype, out, mean, rstd, grads)
    dy, again = t["dy"].clone(), t["x"].clone()
    assert torch.equal(backward(t, mean, rstd, into=dy, dy=dy)["x"], grads["x"])
    assert torch.equal(forward(dict(t, x=again), again)[0], out)
    rows = inside_rows(shape, t["x"].dtype, 5, 1)
    assert torch.equal(forward(t, rows)[0], out)
    untouched_around(rows)
