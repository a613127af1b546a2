"""The 64-bit definitions of layer norm, gated projections and dropout: their gradients against differences, and the generator
against the known answers that its authors published."""
import numpy as np
import pytest

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
