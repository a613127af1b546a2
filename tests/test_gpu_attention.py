"""Attention over neighbourhoods against the 64-bit oracle, element by element inside the error that rounding allows."""
import numpy as np
import pytest
import torch

import iso_inputs as gen
import paper_1606_07676_amd as iso
from oracle import attention_oracle as orc

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def here(d):
    return [(0,) * d]


# dims, periodic, offsets, q heads, kv heads, head_dim
SHAPES = {
    "one_rank": ((1,), None, here(1), 1, 1, 8),
    "line": ((37,), None, [(c,) for c in range(-4, 5)], 2, 2, 32),
    "picture": ((19, 23), None, gen.moore(2, 3) + here(2), 4, 2, 64),
    "mesh": ((19, 23), [False, False], gen.moore(2, 3) + here(2), 4, 1, 64),
    "half_mesh": ((9, 40), [True, False], gen.moore(2, 2), 2, 2, 40),
    "volume": ((9, 11, 10), None, gen.moore(3, 1) + here(3), 6, 2, 128),
    "volume_mesh": ((6, 5, 17), [False, True, False], gen.moore(3, 2) + here(3), 3, 3, 80),
    "wraps_onto_itself": ((3, 4), None, gen.moore(2, 3) + here(2), 2, 1, 64),
    "repeats": ((8, 8), None, [(0, 1), (0, 1), (0, 0), (0, 9), (8, 0), (-3, 2)], 2, 2, 96),
    "far_and_few": ((40, 33), None, [(17, -11), (-20, 3), (5, 16)], 2, 2, 64),
    "far_mesh": ((12, 13), [False, False], [(11, 12), (-11, 0), (2000000000, 1), (-2000000000, -2), (0, 0)], 2, 2, 64),
    "five_dimensions": ((4, 3, 4, 3, 4), None, gen.random_distinct(5, -3, 3, 40, 7), 2, 2, 128),
    "odd_rows": ((14, 15), None, gen.moore(2, 2) + here(2), 3, 1, 33),
    "tiny_rows": ((14, 15), None, gen.von_neumann(2, 2), 2, 2, 1),
    "long_rows": ((6, 7), None, gen.moore(2, 1) + here(2), 2, 1, 256),
    "window": ((33, 30), None, gen.moore(2, 6) + here(2), 2, 2, 64),
    "behind": ((12, 11, 10), [False] * 3, gen.positive_octant(3, 3) + here(3), 4, 2, 64),
    "many_heads": ((5, 6), None, gen.moore(2, 1), 24, 4, 72),
}


def tensors(seed, shape, dtype, bias=False, segments=False, rows=None):
    dims, periodic, offsets, nq, nk, D = SHAPES[shape]
    g = torch.Generator(DEV).manual_seed(seed)
    p = int(np.prod(dims))
    normal = lambda *size: torch.randn(*size, device=DEV, generator=g).to(TYPES[dtype])   # noqa: E731
    t = {"q": normal(p if rows is None else len(rows), nq, D), "k": normal(p, nk, D), "v": normal(p, nk, D)}
    t["bias"] = normal(nq, len(offsets)) if bias else None
    t["segments"] = None
    if segments:                                       # runs of ranks, some of them without a token
        run = torch.randint(1, 9, (p,), device=DEV, generator=g).repeat_interleave(torch.full((p,), 5, device=DEV))[:p]
        t["segments"] = torch.where(run > 7, -1, run % 3).to(torch.int32)
    return t


def comm_of(shape):
    dims, periodic, offsets = SHAPES[shape][:3]
    return iso.iso_neighborhood_create(dims, offsets) if periodic is None else iso.iso_neighborhood_create_mesh(dims, periodic, offsets)


def host(x):
    return None if x is None else x.detach().cpu().to(torch.float64).numpy() if x.is_floating_point() else x.cpu().numpy()


def oracle(shape, t, cap=0.0, rows=None, scale=None):
    dims, periodic, offsets = SHAPES[shape][:3]
    return orc.Attention(dims, offsets, host(t["q"]), host(t["k"]), host(t["v"]), periodic=periodic, bias=host(t["bias"]),
                         segments=host(t["segments"]), cap=cap, rows=rows, scale=scale)


def within(got, want, bound, what):
    got = host(got)
    assert got.shape == want.shape, what
    finite = np.isfinite(want)
    assert np.array_equal(got[~finite], want[~finite]), what
    off = np.abs(got[finite] - want[finite]) / np.broadcast_to(bound, want.shape)[finite]
    assert not off.size or off.max() <= 1, (what, float(off.max()), int((off > 1).sum()), off.size)


def forward(shape, t, cap=0.0, rows=None, out=None, scale=None, stream=None):
    out = torch.full_like(t["q"], 7) if out is None else out
    lse = torch.full(t["q"].shape[:2], 7.0, device=DEV)
    req = iso.iso_neighbor_attention_init(t["q"], t["k"], t["v"], out, comm_of(shape), lse=lse, bias=t["bias"], segments=t["segments"],
                                          cap=cap, scale=scale, rows=None if rows is None else torch.tensor(rows, dtype=torch.int64, device=DEV))
    iso.iso_start(req, stream)
    iso.iso_wait(req)
    return out, lse


def backward(shape, t, out, lse, grad_out, cap=0.0, into=None, scale=None):
    comm = comm_of(shape)
    _, nq, D = t["q"].shape
    g = into or {"grad_q": torch.full_like(t["q"], 7), "grad_k": torch.full_like(t["k"], 7), "grad_v": torch.full_like(t["v"], 7)}
    g["grad_bias"] = None if t["bias"] is None else torch.full_like(t["bias"], 7)
    size = iso.iso_neighbor_attention_backward_workspace_bytes(comm, nq, t["k"].shape[1], D, t["q"].dtype, bias=t["bias"] is not None)
    work = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    req = iso.iso_neighbor_attention_backward_init(t["q"], t["k"], t["v"], out, lse, grad_out, g["grad_q"], g["grad_k"], g["grad_v"], work,
                                                   comm, bias=t["bias"], grad_bias=g["grad_bias"], segments=t["segments"], cap=cap,
                                                   workspace_bytes=size, scale=scale)
    iso.iso_start(req)
    iso.iso_wait(req)
    assert bool((work[size:] == 0xA5).all()), "written behind the workspace"
    return g


OPTIONS = [dict(), dict(bias=True), dict(cap=3.0), dict(segments=True), dict(bias=True, cap=20.0, segments=True)]


@pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype, options):
    cap = options.get("cap", 0.0)
    t = tensors(1, shape, dtype, options.get("bias", False), options.get("segments", False))
    out, lse = forward(shape, t, cap)
    want = oracle(shape, t, cap)
    within(lse, want.lse, want.lse_bound(), "lse")
    within(out, want.out, want.out_bound(out.dtype), "out")


@pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype, options):
    cap = options.get("cap", 0.0)
    t = tensors(2, shape, dtype, options.get("bias", False), options.get("segments", False))
    out, lse = forward(shape, t, cap)
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9)).to(out.dtype)
    got = backward(shape, t, out, lse, grad_out, cap)
    for name, parts in oracle(shape, t, cap).backward(host(grad_out), host(out)).items():
        if got[name] is not None:
            within(got[name], parts[0], orc.gradient_bound(*parts, out.dtype), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ["picture", "mesh", "five_dimensions", "behind", "odd_rows", "volume"])
@pytest.mark.parametrize("n", [1, 2, 37, 700])
def test_rows(shape, dtype, n):
    p = int(np.prod(SHAPES[shape][0]))
    rows = np.random.default_rng(n).integers(0, p, n)
    rows[n // 2:n // 2 + 1] = [p + 5] if n > 2 else rows[n // 2:n // 2 + 1]            # a rank that does not exist
    rows[n // 3:n // 3 + 1] = [-1] if n > 2 else rows[n // 3:n // 3 + 1]
    t = tensors(3, shape, dtype, True, True, rows)
    out, lse = forward(shape, t, 10.0, rows.tolist())
    want = oracle(shape, t, 10.0, rows)
    within(lse, want.lse, want.lse_bound(), "lse")
    within(out, want.out, want.out_bound(out.dtype), "out")


def test_no_rows_and_no_neighbours():
    t = tensors(3, "picture", "bf16", rows=[])
    out, lse = forward("picture", t, rows=[])
    assert out.shape[0] == 0
    x = torch.ones(6, 2, 16, device=DEV, dtype=torch.bfloat16)
    out, lse = torch.full_like(x, 7), torch.zeros(6, 2, device=DEV)
    comm = iso.iso_neighborhood_create((6,), np.zeros((0, 1), dtype=np.int32))
    req = iso.iso_neighbor_attention_init(x, x, x, out, comm, lse=lse)
    iso.iso_start(req)
    iso.iso_wait(req)
    assert not out.any() and bool(torch.isneginf(lse).all())


def fused(shape, dtype, seed, head_major=False, shift=0):
    """q, k, v and gradients as slices of one buffer each, head-major or with an odd start."""
    dims, _, offsets, nq, nk, D = SHAPES[shape]
    p = int(np.prod(dims))
    heads = nq + 2 * nk
    flat = torch.randn(p * heads * D + shift, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(TYPES[dtype])[shift:]
    x = flat.view(heads, p, D).transpose(0, 1) if head_major else flat.view(p, heads, D)
    return x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:]


# neighbourhoods whose tables are large for the heads of one rank together, and whose neighbours have few rows in common
WIDE = {
    "shared_heads_of_many_neighbours": ((9, 8, 10), None, gen.moore(3, 3) + here(3), 4, 1, 128),
    "pairs_of_heads_of_many_neighbours": ((9, 8, 10), [False, True, False], gen.moore(3, 3) + here(3), 4, 2, 64),
    "scattered": ((7, 6, 5, 4), None, gen.random_distinct(4, -3, 3, 60, 11), 2, 1, 128),
    "scattered_mesh": ((7, 6, 9, 4), [False, False, True, True], gen.random_distinct(4, -3, 3, 60, 12), 2, 2, 64),
}


@pytest.mark.parametrize("options", [dict(), dict(bias=True, segments=True)], ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", WIDE)
def test_wide_neighbourhoods(shape, dtype, options, monkeypatch):
    monkeypatch.setitem(SHAPES, shape, WIDE[shape])
    t = tensors(16, shape, dtype, options.get("bias", False), options.get("segments", False))
    out, lse = forward(shape, t)
    want = oracle(shape, t)
    within(lse, want.lse, want.lse_bound(), "lse")
    within(out, want.out, want.out_bound(out.dtype), "out")
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(17)).to(out.dtype)
    got = backward(shape, t, out, lse, grad_out)
    for name, parts in want.backward(host(grad_out), host(out)).items():
        if got[name] is not None:
            within(got[name], parts[0], orc.gradient_bound(*parts, out.dtype), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ["picture", "volume", "half_mesh"])
@pytest.mark.parametrize("head_major,shift", [(False, 0), (True, 0), (False, 3), (False, 8), (True, 1)])
def test_strides_and_alignment(shape, dtype, head_major, shift):
    t = tensors(4, shape, dtype, bias=True)
    t["q"], t["k"], t["v"] = fused(shape, dtype, 5, head_major, shift)
    out, lse = forward(shape, t)
    want = oracle(shape, t)
    within(out, want.out, want.out_bound(out.dtype), "out")
    g = dict(zip(("grad_q", "grad_k", "grad_v"), fused(shape, dtype, 6, head_major, shift)))
    grad_out = fused(shape, dtype, 7, not head_major, shift)[0]
    got = backward(shape, t, out, lse, grad_out, into=g)
    for name, parts in want.backward(host(grad_out), host(out)).items():
        within(got[name], parts[0], orc.gradient_bound(*parts, out.dtype), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ["picture", "volume_mesh", "window", "odd_rows"])
def test_nothing_that_does_not_count_is_seen(shape, dtype):
    """Infinities and NaN in the tokens and biases of places that do not count, in every tensor that has such rows."""
    t = tensors(8, shape, dtype, bias=True, segments=True)
    out, lse = forward(shape, t)
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9)).to(out.dtype)
    clean = backward(shape, t, out, lse, grad_out)
    absent = t["segments"] < 0
    assert bool(absent.any()) and not bool(absent.all())
    bad = {k: v.clone() if v is not None else None for k, v in t.items()}
    for i, name in enumerate("qkv"):
        bad[name][absent] = (float("nan"), float("inf"), float("-inf"))[i]
    out2, lse2 = forward(shape, bad)
    assert torch.equal(lse2, lse)
    want = oracle(shape, t)
    within(out2, want.out, want.out_bound(out.dtype), "out")
    grad_bad = grad_out.clone()
    grad_bad[absent] = float("inf")
    got = backward(shape, bad, out2, lse2, grad_bad)
    for name, parts in want.backward(host(grad_out) * ~host(absent)[:, None, None], host(out)).items():
        within(got[name], parts[0], orc.gradient_bound(*parts, out.dtype), name)
        within(clean[name], parts[0], orc.gradient_bound(*parts, out.dtype), name + " of clean inputs")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_bad_value_reaches_the_ranks_that_see_it_and_no_others(dtype, value):
    shape = "picture"
    t = tensors(8, shape, dtype)
    out, lse = forward(shape, t)
    t2 = {k: v.clone() if v is not None else None for k, v in t.items()}
    t2["v"][100, 1, 3] = value
    out2, lse2 = forward(shape, t2)
    dims, periodic, offsets, nq, nk, _ = SHAPES[shape]
    sees = torch.from_numpy((orc.neighbours(dims, offsets, periodic) == 100).any(1)).to(DEV)
    heads = torch.arange(nq, device=DEV) // (nq // nk) == 1
    touched = sees[:, None] & heads[None, :]
    assert torch.equal(lse2, lse)
    want = oracle(shape, t)
    keep = ~touched
    assert not torch.isfinite(out2[touched][:, 3]).any()
    within(out2[keep], want.out[host(keep)], want.out_bound(out.dtype)[host(keep)], "rows that do not see it")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ["picture", "volume", "odd_rows"])
def test_biases_that_mask(shape, dtype):
    """-inf takes a neighbour out; all biases of a head at the type's lowest value leave its scores equal."""
    t = tensors(10, shape, dtype, bias=True)
    t["bias"][0, ::2] = float("-inf")
    t["bias"][1, :] = float("-inf")
    out, lse = forward(shape, t)
    want = oracle(shape, t)
    within(lse, want.lse, want.lse_bound(), "lse")
    within(out, want.out, want.out_bound(out.dtype), "out")
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9)).to(out.dtype)
    got = backward(shape, t, out, lse, grad_out)
    for name, parts in want.backward(host(grad_out), host(out)).items():
        within(got[name], parts[0], orc.gradient_bound(*parts, out.dtype), name)
    if dtype == "f16":
        return                                                     # its lowest value, -65504, does not swallow a score
    t["bias"][0, :] = torch.finfo(TYPES[dtype]).min
    out, lse = forward(shape, t)
    flat = {k: v.clone() if v is not None else None for k, v in t.items()}
    flat["q"][:, 0], flat["bias"][0] = 0, 0                        # equal scores
    want = oracle(shape, flat)
    within(out[:, 0], want.out[:, 0], want.out_bound(out.dtype)[:, 0], "equal weights")
    assert bool(torch.isfinite(lse[:, 0]).all()) and bool((lse[:, 0] < -3e38).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("shape", ["picture", "volume", "volume_mesh"])
def test_gradients_of_rows_whose_biases_are_all_lowest(shape, cap, dtype):
    """Equal weights, whatever the scores, in every gradient that depends on the weights alone."""
    t = tensors(10, shape, dtype, bias=True)
    t["bias"][0, :] = torch.finfo(TYPES[dtype]).min
    out, lse = forward(shape, t, cap)
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9)).to(out.dtype)
    got = backward(shape, t, out, lse, grad_out, cap)
    flat = {k: v.clone() if v is not None else None for k, v in t.items()}
    flat["q"][:, 0], flat["bias"][0] = 0, 0
    want = oracle(shape, flat, cap).backward(host(grad_out), host(out))
    for name in ("grad_v", "grad_bias"):
        within(got[name], want[name][0], orc.gradient_bound(*want[name], out.dtype), name)
    assert all(bool(torch.isfinite(g).all()) for g in got.values())


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(dtype):
    t = tensors(11, "picture", dtype, bias=True)
    t["q"] *= 60
    for cap in (0.0, 50.0):
        out, lse = forward("picture", t, cap)
        want = oracle("picture", t, cap)
        within(lse, want.lse, want.lse_bound(), "lse")
        within(out, want.out, want.out_bound(out.dtype), "out")


@pytest.mark.parametrize("dtype", TYPES)
def test_scale_and_repeated_rows(dtype):
    """A scale of one's own, and inputs whose rows are one row repeated (strides of 0)."""
    t = tensors(12, "picture", dtype)
    t["k"] = t["k"][:1].expand_as(t["k"])
    out, lse = forward("picture", t, scale=0.3)
    want = oracle("picture", t, scale=0.3)
    within(lse, want.lse, want.lse_bound(), "lse")
    within(out, want.out, want.out_bound(out.dtype), "out")
    with pytest.raises(iso.IsoError) as e:
        forward("picture", t, out=torch.zeros_like(t["q"])[:1].expand_as(t["q"]))
    assert e.value.status == iso.ISO_ERR_OVERLAP


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ["picture", "five_dimensions", "volume_mesh"])
def test_the_same_bits_every_time_on_any_stream_and_in_graphs(shape, dtype):
    t = tensors(13, shape, dtype, bias=True, segments=True)
    out, lse = forward(shape, t, 8.0)
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9)).to(out.dtype)
    first = backward(shape, t, out, lse, grad_out, 8.0)
    for _ in range(2):
        again = backward(shape, t, out, lse, grad_out, 8.0)
        assert all(torch.equal(first[n].view(torch.uint8), again[n].view(torch.uint8)) for n in first)
    out2 = torch.zeros_like(out)
    req = iso.iso_neighbor_attention_init(t["q"], t["k"], t["v"], out2, comm_of(shape), bias=t["bias"], segments=t["segments"], cap=8.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    iso.iso_start(req, side)
    iso.iso_wait(req)
    assert torch.equal(out, out2)
    for form in (iso.ISO_GRAPH_CHAIN, iso.ISO_GRAPH_BRANCHES, iso.ISO_GRAPH_OFF):
        iso.iso_request_set_graph(req, form)
        for _ in range(3):
            out2.zero_()
            iso.iso_start(req)
            iso.iso_wait(req)
            assert torch.equal(out, out2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iso.iso_start(req)
    for seed in (1, 2, 3):
        t["q"].copy_(torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(out.dtype))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, forward(shape, t, 8.0)[0])


def test_gradients_against_differences():
    """In 32 bits, along one direction: the forward kernel's own differences."""
    t = tensors(14, "picture", "f32", bias=True, segments=True)
    out, lse = forward("picture", t, 4.0)
    grad_out = torch.randn(t["q"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(9))
    got = backward("picture", t, out, lse, grad_out, 4.0)
    h = 2.0 ** -7
    for name in ("q", "k", "v", "bias"):
        step = torch.randn(t[name].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(5))
        side = []
        for sign in (2, 1, -1, -2):
            moved = dict(t)
            moved[name] = t[name] + sign * h * step
            side.append(float((forward("picture", moved, 4.0)[0].double() * grad_out).sum()))
        slope = (8 * (side[1] - side[2]) - (side[0] - side[3])) / (12 * h)      # error h^4 / 30 of the fifth derivative
        want = float((got["grad_" + name].double() * step).sum())
        scale = float((got["grad_" + name].double() * step).norm())
        assert abs(slope - want) < 2e-3 * scale + 1e-3 * abs(want), (name, slope, want, scale)


def test_offsets_beyond_32_bits():
    """Keys whose rows lie more than 2^31 elements (and 2^32 bytes) apart."""
    dims, offsets, D = (6, 7), gen.moore(2, 1) + here(2), 64
    stride = (1 << 31) // 20
    big = torch.zeros(42 * stride + 2 * D, dtype=torch.bfloat16, device=DEV)
    k, v = (big.as_strided((42, 1, D), (stride, D, 1), at) for at in (0, D))
    g = torch.Generator(DEV).manual_seed(3)
    for x in (k, v):
        x.copy_(torch.randn(x.shape, device=DEV, generator=g))
    q = torch.randn(42, 1, D, device=DEV, generator=g).to(torch.bfloat16)
    out = torch.empty_like(q)
    for periodic in ([True, True], [False, False]):
        req = iso.iso_neighbor_attention_init(q, k, v, out, iso.iso_neighborhood_create_mesh(dims, periodic, offsets))
        iso.iso_start(req)
        iso.iso_wait(req)
        want = orc.Attention(dims, offsets, host(q), host(k), host(v), periodic=periodic)
        within(out, want.out, want.out_bound(out.dtype), "out")
