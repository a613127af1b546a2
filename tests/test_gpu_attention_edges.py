"""Attention over neighbourhoods at the edges of what the calls take, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import iso_inputs as gen
import paper_1606_07676_amd as iso
from oracle import attention_oracle as orc
from test_gpu_attention import DEV, SHAPES, TYPES, backward, forward, host, oracle, tensors, within

pytestmark = pytest.mark.gpu


def here(d):
    return [(0,) * d]


def normal_like(x, seed):
    return torch.randn(x.shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(x.dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dims,offsets", [((8, 8), [(9, 0), (0, -8)]), ((1, 40), [(1, 0), (-1, 3)])])
def test_a_mesh_without_any_source(dims, offsets, dtype, monkeypatch):
    """Every row is one without neighbours: out 0, lse -inf, gradients 0."""
    monkeypatch.setitem(SHAPES, "outside", (dims, [False] * len(dims), offsets, 4, 2, 64))
    t = tensors(20, "outside", dtype, bias=True)
    out, lse = forward("outside", t)
    assert not out.any() and bool(torch.isneginf(lse).all())
    got = backward("outside", t, out, lse, normal_like(t["q"], 9))
    assert all(not g.any() for g in got.values())
