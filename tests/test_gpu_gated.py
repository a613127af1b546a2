"""Gated projections and their gradients against the 64-bit oracle, element by element inside the error that rounding allows."""
import numpy as np
import pytest
import torch

import paper_1606_07676_amd as iso
from oracle import token_oracle as orc
from token_rows import DEV, TYPES, U, host, inside_rows, untouched_around, within
from token_shapes import FEW, LARGE, TILED

pytestmark = pytest.mark.gpu


def tensors(n, C, F, dtype, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    normal = lambda *size: torch.randn(*size, device=DEV, generator=g)  # noqa: E731
    return {"x": normal(n, C).to(TYPES[dtype]), "gate": (2 * normal(F, C) * C ** -0.5).to(TYPES[dtype]),
            "up": (normal(F, C) * C ** -0.5).to(TYPES[dtype]), "dy": normal(n, F).to(TYPES[dtype])}


def forward(t, activation, out=None, stream=None):
    out = torch.full_like(t["dy"], 7) if out is None else out
    req = iso.iso_gated_init(t["x"], t["gate"], t["up"], out, activation=activation)
    iso.iso_start(req, stream)
    iso.iso_wait(req)
    return out


def backward(t, activation, into=None):
    (n, C), F = t["x"].shape, t["gate"].shape[0]
    grads = into or {k: torch.full_like(t[k], 7) for k in ("x", "gate", "up")}
    size = iso.iso_gated_backward_workspace_bytes(n, C, F, t["x"].dtype)
    work = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    req = iso.iso_gated_backward_init(t["x"], t["gate"], t["up"], t["dy"], grads["x"], grads["gate"], grads["up"], work,
                                      activation=activation, workspace_bytes=size)
    iso.iso_start(req)
    iso.iso_wait(req)
    assert bool((work[size:] == 0xA5).all()), "written behind the workspace"
    return grads


def near(got, want, error, u, what):
    """Inside the bound element by element; and, as roundings are independent, far inside it together: the roundings of a result
    and of what it is a sum of are each at most u of a value, u / sqrt 3 on average, together u sqrt(2 / 3) of the values' size;
    three times that, and what is off in 32 bits."""
    within(host(got), want, orc.rounded(want, error, u), what)
    size = np.sqrt(np.mean(want ** 2))
    if got.numel() >= 256 and size:
        assert np.sqrt(np.mean((host(got) - want) ** 2)) <= (3 * u * (2 / 3) ** 0.5 + 64 * orc.EPS) * size, what


def check(t, dtype, activation, out, grads=None):
    u = U[dtype]
    o = orc.Gated(*(host(t[k]) for k in ("x", "gate", "up")), activation, dtype != "f32")
    within(host(out), o.out, o.out_bound(u), "out")
    if grads is None:
        return
    o.backward(host(t["dy"]), u)
    near(grads["x"], o.grad_x, o.grad_x_error, u, "grad_x")
    near(grads["gate"], o.grad_gate, o.grad_gate_error, u, "grad_gate")
    near(grads["up"], o.grad_up, o.grad_up_error, u, "grad_up")


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", FEW + TILED, ids=str)
def test_projections_and_gradients(shape, dtype, activation):
    t = tensors(*shape, dtype)
    check(t, dtype, activation, forward(t, activation), backward(t, activation))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_many_tiles(shape, dtype):
    t = tensors(*shape, dtype, seed=1)
    out, grads = forward(t, "silu"), backward(t, "silu")
    check(t, dtype, "silu", out, grads)
    assert torch.equal(forward(t, "silu"), out)
    for name, value in backward(t, "silu").items():
        assert torch.equal(value, grads[name]), name


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tokens_in_the_sum(dtype):
    """The weights' gradient sums over tokens in parts."""
    t = tensors(20000, 40, 56, dtype, seed=2)
    check(t, dtype, "gelu", forward(t, "gelu"), backward(t, "gelu"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(9, 64, 48), (150, 64, 72)], ids=str)
@pytest.mark.parametrize("gap,shift", [(8, 0), (1, 0), (8, 3)])
def test_rows_inside_larger_buffers(gap, shift, shape, dtype):
    """Any strides and addresses; what lies around the rows stays as it was."""
    t = tensors(*shape, dtype, seed=3)
    views = {k: inside_rows(tuple(v.shape), v.dtype, gap, shift) for k, v in t.items()}
    for k, v in t.items():
        views[k].copy_(v)
    out = inside_rows(tuple(t["dy"].shape), t["dy"].dtype, gap, shift)
    into = {k: inside_rows(tuple(t[k].shape), t[k].dtype, gap, shift) for k in ("x", "gate", "up")}
    check(t, dtype, "silu", forward(views, "silu", out), backward(views, "silu", into))
    for view in [out, *into.values()]:
        untouched_around(view)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [30, 100])
def test_weights_in_one_buffer_and_one_row_for_all(n, dtype):
    t = tensors(n, 48, 40, dtype, seed=4)
    both = torch.cat([t["gate"], t["up"]])
    t["gate"], t["up"] = both[:40], both[40:]
    t["x"] = t["x"][:1].expand(n, 48)
    grads = {k: torch.empty(t[k].shape, device=DEV, dtype=t[k].dtype) for k in ("x", "gate", "up")}
    check(t, dtype, "silu", forward(t, "silu"), backward(t, "silu", grads))
    t["up"] = t["gate"]
    check(t, dtype, "gelu", forward(t, "gelu"), backward(t, "gelu", grads))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("n", [4, 90])
def test_far_ends_of_the_activations(n, activation, dtype):
    """Hidden units far below and above zero give 0 and g itself, with slopes 0 and 1, and no infinity on the way."""
    t = tensors(n, 16, 32, dtype, seed=5)
    t["x"][:, 0] = 1
    t["gate"][:, 1:] = 0
    t["gate"][:, 0] = torch.linspace(-300, 300, 32, device=DEV).to(TYPES[dtype])
    check(t, dtype, activation, forward(t, activation), backward(t, activation))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [20, 200])
def test_a_token_that_is_not_a_number_stays_by_itself(n, dtype):
    """Also at the ends of tiles, next to rows and elements that are not there."""
    t = tensors(n, 72, 41, dtype, seed=6)
    clean, grads = forward(t, "silu"), backward(t, "silu")
    bad = [0, 7, n - 1]
    good = torch.ones(n, dtype=torch.bool, device=DEV)
    good[bad] = False
    t["x"][0], t["x"][7, 3], t["x"][n - 1, 71] = float("nan"), float("inf"), float("-inf")
    out, again = forward(t, "silu"), backward(t, "silu")
    assert torch.equal(out[good], clean[good]) and torch.equal(again["x"][good], grads["x"][good])
    assert out[0].isnan().all() and again["gate"].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_no_tokens(dtype):
    t = tensors(0, 40, 24, dtype)
    assert forward(t, "silu").shape == (0, 24)
    grads = backward(t, "silu")
    assert not grads["gate"].any() and not grads["up"].any()


def test_results_beyond_32_bits_of_bytes():
    """The last tokens of many, against themselves alone."""
    n, C, F = 70000, 8, 32776
    g = torch.Generator(DEV).manual_seed(10)
    normal = lambda *size: torch.randn(*size, device=DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    t = {"x": normal(n, C), "gate": normal(F, C), "up": normal(F, C), "dy": torch.empty(n, F, device=DEV, dtype=torch.bfloat16)}
    out, alone = forward(t, "silu"), dict(t, x=t["x"][-40:], dy=t["dy"][-40:])
    o = orc.Gated(*(host(alone[k]) for k in ("x", "gate", "up")), "silu", True)
    within(host(out[-40:]), o.out, o.out_bound(U["bf16"]), "last rows")
    t["dy"].normal_(generator=g)
    grads, last = backward(t, "silu"), backward(dict(t, x=t["x"][-40:], dy=t["dy"][-40:]), "silu")
    o.backward(host(t["dy"][-40:]), U["bf16"])
    for got in (grads["x"][-40:], last["x"]):
        near(got, o.grad_x, o.grad_x_error, U["bf16"], "grad_x")


def test_another_stream():
    t = tensors(300, 128, 256, "bf16", seed=7)
    want, other = forward(t, "gelu"), torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        assert torch.equal(forward(t, "gelu", stream=other), want)


@pytest.mark.parametrize("n", [6, 80])
def test_gradient_against_differences(n):
    t = tensors(n, 20, 24, "f32", seed=8)
    grads, dy = backward(t, "gelu"), host(t["dy"])
    for name in ("x", "gate", "up"):
        direction = np.random.default_rng(9).normal(size=t[name].shape)
        value = lambda s: float((orc.Gated(*(host(t[k]) + (s * direction if k == name else 0) for k in ("x", "gate", "up")),  # noqa: E731
                                           "gelu", False).out * dy).sum())
        change = (value(1e-6) - value(-1e-6)) / 2e-6
        assert abs(change - float((host(grads[name]) * direction).sum())) < 1e-5 * np.abs(host(grads[name]) * direction).sum() + 1e-6, name


# Gradients of x . gate and x . up that float16 holds with fewer bits, or not at all, unscaled.  Of those below 1/2 the products
# take copies times 2^16, which are rounded by at most 2^-25 / 2^16.
SCALED = 2.0 ** -41
SMALL = [(1, 64, 40), (30, 64, 48), (61, 72, 130), (65, 8, 8), (333, 65, 127), (2048, 64, 64), (1320, 120, 343), (5000, 200, 1500), (4096, 2040, 100),
         (12000, 1048, 264)]


def rms(x, axis=None):
    return np.sqrt(np.mean(x ** 2, axis))


def small_bound(want, axis=None):
    """Of a gradient's error, together: the roundings of the result and of what it is a sum of as in `near`, and the result's own
    absolute rounding, at most 2^-25 an element."""
    return (3 * U["f16"] * (2 / 3) ** 0.5 + 64 * orc.EPS) * rms(want, axis) + 2.0 ** -25


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("scale", [1e-3, 1e-5, 1e-6])
@pytest.mark.parametrize("shape", SMALL, ids=str)
def test_small_gradients_in_float16(shape, scale, activation):
    t = tensors(*shape, "f16", seed=11)
    t["dy"] = (t["dy"].float() * scale).to(torch.float16)
    o = orc.Gated(*(host(t[k]) for k in ("x", "gate", "up")), activation, True)
    o.backward(host(t["dy"]), U["f16"], SCALED)
    assert max(np.abs(o.d_gate).max(), np.abs(o.d_up).max()) < 0.49
    grads = backward(t, activation)
    for got, want, error, what in ((grads["x"], o.grad_x, o.grad_x_error, "grad_x"), (grads["gate"], o.grad_gate, o.grad_gate_error, "grad_gate"),
                                   (grads["up"], o.grad_up, o.grad_up_error, "grad_up")):
        within(host(got), want, orc.rounded(want, error, U["f16"]), what)
        assert rms(host(got) - want) <= small_bound(want), what


@pytest.mark.parametrize("shape", [(48, 16, 1024), (700, 16, 1024), (3000, 72, 2048)], ids=str)
def test_tokens_with_small_gradients_beside_others_in_float16(shape):
    """A token's grad_x is as exact as its own gradients allow, whatever the tokens beside it hold."""
    t = tensors(*shape, "f16", seed=12)
    t["gate"], t["up"] = t["gate"] * 4, t["up"] * 4
    small = torch.arange(shape[0], device=DEV) % 3 != 0
    t["dy"][small] = (t["dy"][small].float() * 1e-6).to(torch.float16)
    o = orc.Gated(*(host(t[k]) for k in ("x", "gate", "up")), "silu", True)
    o.backward(host(t["dy"]), U["f16"], SCALED)
    small = small.cpu().numpy()
    assert max(np.abs(o.d_gate[small]).max(), np.abs(o.d_up[small]).max()) < 0.49 < np.abs(o.d_gate[~small]).max()
    grads = backward(t, "silu")
    got, error = host(grads["x"]), orc.rounded(o.grad_x, o.grad_x_error, U["f16"])
    within(got[small], o.grad_x[small], error[small], "small tokens")
    assert rms(got[small] - o.grad_x[small]) <= small_bound(o.grad_x[small])
    # the others, and the sums over all tokens, with whole numbers' rounding below 2^-14
    o.backward(host(t["dy"]), U["f16"])
    check(t, "f16", "silu", forward(t, "silu"), grads)


@pytest.mark.parametrize("shape", [(48, 64, 96), (700, 64, 192), (5000, 200, 1024)], ids=str)
def test_hidden_units_with_small_gradients_beside_others_in_float16(shape):
    """Rows of grad_gate are as exact as their own block of hidden units allows, whatever other blocks hold; grad_up likewise."""
    t = tensors(*shape, "f16", seed=13)
    F = shape[2]
    t["up"][:F // 3] *= 1e-4                               # small d_gate
    t["gate"][2 * F // 3:] *= 1e-4                         # small d_up
    t["dy"] = (t["dy"].float() * 0.01).to(torch.float16)
    t["dy"][0] *= 1000                                     # one token whose gradients are not
    o = orc.Gated(*(host(t[k]) for k in ("x", "gate", "up")), "gelu", True)
    o.backward(host(t["dy"]), U["f16"], SCALED)
    grads = backward(t, "gelu")
    a, b = F // 96 * 32, (2 * F // 3 + 31) // 32 * 32      # whole blocks of 32
    assert np.abs(o.d_gate[:, :a]).max() < 0.49 < np.abs(o.d_gate[:, a:]).max() and np.abs(o.d_up[:, b:]).max() < 0.49 < np.abs(o.d_up[:, :b]).max()
    for got, want, error, rows in ((grads["gate"], o.grad_gate, o.grad_gate_error, slice(0, a)), (grads["up"], o.grad_up, o.grad_up_error, slice(b, F))):
        within(host(got)[rows], want[rows], orc.rounded(want, error, U["f16"])[rows], "small rows")
        assert rms(host(got)[rows] - want[rows]) <= small_bound(want[rows])
    check(t, "f16", "gelu", forward(t, "gelu"), grads)


def test_weights_gradients_beyond_32_bits_of_bytes():
    """Rows of grad_gate and grad_up that sum over all of 70000 tokens, the last of which lie behind 2^32 bytes of grad_out, d_gate and
    d_up: the oracle's, for the first and the last hidden units."""
    n, C, F, some = 70000, 8, 32776, 24
    g = torch.Generator(DEV).manual_seed(15)
    normal = lambda *size: torch.randn(*size, device=DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    t = {"x": normal(n, C), "gate": normal(F, C), "up": normal(F, C), "dy": torch.empty(n, F, device=DEV, dtype=torch.bfloat16)}
    t["dy"].normal_(generator=g)
    t["dy"][-40:] *= 100                                   # the last tokens weigh as much as a tenth of all others
    grads = backward(t, "silu")
    for rows in (slice(0, some), slice(F - some, F)):
        o = orc.Gated(host(t["x"]), host(t["gate"][rows]), host(t["up"][rows]), "silu", True)
        o.backward(host(t["dy"][:, rows]), U["bf16"])
        near(grads["gate"][rows], o.grad_gate, o.grad_gate_error, U["bf16"], "grad_gate")
        near(grads["up"][rows], o.grad_up, o.grad_up_error, U["bf16"], "grad_up")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_many_tiles_of_gelu(shape, dtype):
    """The larger tiles' ends, whole and cut off, with the other activation."""
    t = tensors(*shape, dtype, seed=16)
    check(t, dtype, "gelu", forward(t, "gelu"), backward(t, "gelu"))


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(2048, 72, 2048), (1024, 136, 512), (1100, 136, 1100)], ids=str)
def test_far_ends_of_the_activations_in_larger_tiles(shape, dtype, activation):
    n, C, F = shape
    t = tensors(n, C, F, dtype, seed=17)
    t["x"][:, 0] = 1
    t["gate"][:, 1:] = 0
    t["gate"][:, 0] = torch.linspace(-300, 300, F, device=DEV).to(TYPES[dtype])
    check(t, dtype, activation, forward(t, activation), backward(t, activation))


@pytest.mark.parametrize("shape", [(40, 72, 130), (700, 72, 130), (2100, 136, 1100)], ids=str)
def test_which_gradients_are_small_is_found_at_every_start(shape):
    """One request, started eagerly and replayed, over gradients of changing size, in a workspace that holds what was before."""
    (n, C, F), half = shape, torch.float16
    t = tensors(*shape, "f16", seed=18)
    sizes = [t["dy"].clone(), (t["dy"].float() * 1e-5).to(half), torch.zeros_like(t["dy"]), t["dy"].clone(), (t["dy"].float() * 1e-6).to(half)]
    sizes[3][::3] *= 1e-5
    wants = [{k: v.clone() for k, v in backward(dict(t, dy=dy), "silu").items()} for dy in sizes]
    grads = {k: torch.empty_like(t[k]) for k in ("x", "gate", "up")}
    work = torch.empty(iso.iso_gated_backward_workspace_bytes(n, C, F, half), dtype=torch.uint8, device=DEV)
    req = iso.iso_gated_backward_init(t["x"], t["gate"], t["up"], t["dy"], grads["x"], grads["gate"], grads["up"], work)
    iso.iso_start(req)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iso.iso_start(req)
    for turn in range(2):
        for i, dy in enumerate(sizes):
            for start in (lambda: iso.iso_start(req), graph.replay):
                t["dy"].copy_(dy)
                for v in grads.values():
                    v.fill_(7)
                start()
                torch.cuda.synchronize()
                for name, want in wants[i].items():
                    assert torch.equal(grads[name], want), (turn, i, name)


@pytest.mark.parametrize("n", [30, 300])
def test_gradients_that_are_not_numbers_stay_by_themselves_in_float16(n):
    """Beside small ones, which stay as exact as they were."""
    t = tensors(n, 72, 70, "f16", seed=19)
    t["dy"] = (t["dy"].float() * 1e-5).to(torch.float16)
    clean = backward(t, "silu")
    t["dy"][3, 5], t["dy"][n - 1, 69], t["dy"][17, 33] = float("nan"), float("inf"), float("-inf")
    grads = backward(t, "silu")
    good, rows = torch.ones(n, dtype=torch.bool, device=DEV), torch.ones(70, dtype=torch.bool, device=DEV)
    good[[3, 17, n - 1]], rows[[5, 33, 69]] = False, False
    assert torch.equal(grads["x"][good], clean["x"][good]) and not grads["x"][~good].isfinite().any()
    for name in ("gate", "up"):
        assert torch.equal(grads[name][rows], clean[name][rows]) and not grads[name][~rows].isfinite().any()
