"""The 64-bit definitions of layer norm, gated projections and dropout: their gradients against differences, and the generator
against the known answers that its authors published."""
import os
import re

import numpy as np
import pytest
from scipy.special import erfcx

from conftest import ROOT
from oracle import token_oracle as orc


def differences(value, x, step=1e-6):
    grad = np.empty_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        above = value()
        x[i] = keep - step
        grad[i] = (above - value()) / (2 * step)
        x[i] = keep
    return grad


def test_layer_norm_gradients():
    r = np.random.default_rng(1)
    x, w, b, dy = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    value = lambda: float((orc.LayerNorm(x, w, b).out * dy).sum())  # noqa: E731
    norm = orc.LayerNorm(x, w, b)
    norm.backward(dy)
    for grad, of in ((norm.grad_x, x), (norm.grad_weight, w), (norm.grad_bias, b)):
        np.testing.assert_allclose(grad, differences(value, of), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_gated_gradients(activation):
    r = np.random.default_rng(2)
    x, gate, up, dy = r.normal(size=(3, 5)), r.normal(size=(4, 5)), r.normal(size=(4, 5)), r.normal(size=(3, 4))
    value = lambda: float((orc.Gated(x, gate, up, activation, False).out * dy).sum())  # noqa: E731
    block = orc.Gated(x, gate, up, activation, False)
    block.backward(dy, 2.0 ** -24)
    for grad, of in ((block.grad_x, x), (block.grad_gate, gate), (block.grad_up, up)):
        np.testing.assert_allclose(grad, differences(value, of), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("counter,more,key,words", [
    (0, 0, 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    (0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822, (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_known_answers_of_the_generator(counter, more, key, words):
    assert tuple(int(w) for w in orc.philox([counter], more, key)[0]) == words


def test_kept_elements():
    keep, factor = orc.kept(3, 5, (12, 34), 0.25)
    words = orc.philox([0, 1], 34, 12).reshape(-1)
    numbers = [int(w) >> s & 0xFFFF for w in words for s in (0, 16)][:15]
    assert keep.reshape(-1).tolist() == [n >= 16384 for n in numbers] and factor == 4 / 3
    assert orc.kept(40, 50, (-1, 2), 0.0)[0].all() and not orc.kept(40, 50, (1, -2), 1.0)[0].any()
    assert abs(orc.kept(400, 500, (5, 6), 0.1)[0].mean() - 0.9) < 5 * (0.09 / 2e5) ** 0.5


def test_the_fit_of_the_error_function():
    """0.5 erfc(|g| / sqrt 2) = t P(t) exp(-g^2 / 2) with the kernel's own constants: in exact arithmetic as near as its comment says;
    in 32 bits off by the argument's three roundings, together 1.5 g^2 units of 2^-24, one unit each for the exponential and the
    last two products, 1.4 for the fit, and what is left of 8 for t and the terms."""
    text = open(os.path.join(ROOT, "paper_1606_07676_amd", "csrc", "iso_gated_kernels.hpp")).read()
    terms = np.array([float(x.rstrip("f")) for x in re.search(r"kTerms\[9\] = \{([^}]*)\}", text)[1].replace("\n", " ").split(",")], dtype=np.float32)
    assert len(terms) == 9 and "fmaf(0.26f, fabsf(g), 1.f)" in text
    f32, wide = np.float32, np.longdouble
    g = np.linspace(0, 14.5, 200001).astype(f32)
    scaled = 0.5 * erfcx(g.astype(float) / np.sqrt(2))                   # without the exponential
    t = 1 / (1 + wide(f32(0.26)) * g.astype(wide))
    rest = np.full(g.shape, terms[8], dtype=wide)
    for term in terms[7::-1]:
        rest = wide(term) + t * rest
    assert float(np.abs(rest * t / scaled - 1).max()) < 7.9e-8
    fma = lambda a, b, c: (a.astype(float) * b.astype(float) + c.astype(float)).astype(f32)       # noqa: E731
    t = (1 / fma(f32(0.26), g, f32(1)).astype(float)).astype(f32)
    e = np.exp2((f32(-0.5 * 1.44269504088896340736) * (g * g)).astype(float)).astype(f32)
    rest = np.full(g.shape, terms[8])
    for term in terms[7::-1]:
        rest = fma(t, rest, term)
    rest = rest * (t * e)
    there = g < 12.5                                                    # above, 32 bits hold the share with fewer bits
    want = scaled * np.exp(-0.5 * g.astype(float) ** 2)
    assert np.all(np.abs(rest / want - 1)[there] < 2.0 ** -24 * (8 + 2 * g[there].astype(float) ** 2))
