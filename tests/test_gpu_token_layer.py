"""The example's layer (rotary positions, attention, and both backward) as a whole against the 64-bit oracle."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import iso_inputs as gen
from conftest import ROOT
from oracle import attention_oracle as orc

pytestmark = pytest.mark.gpu


def load_example():
    spec = importlib.util.spec_from_file_location("token_layer", os.path.join(ROOT, "examples", "token_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_step_and_single_token(dtype):
    dims, offsets, nq, nk, D = (6, 5, 4), gen.moore(3, 1) + [(0, 0, 0)], 4, 2, 32
    layer = load_example().TokenLayer(dims, offsets, nq, nk, D, dtype=dtype, cap=10.0)
    g = torch.Generator("cuda").manual_seed(1)
    normal = lambda x: torch.randn(x.shape, device="cuda", generator=g).to(dtype)      # noqa: E731
    qkv = normal(layer.qkv)
    layer.qkv.copy_(qkv)
    layer.bias.copy_(normal(layer.bias))
    layer.grad_out.copy_(normal(layer.grad_out))
    layer.forward()
    layer.backward()
    torch.cuda.synchronize()
    host = lambda x: x.cpu().double().numpy()                                          # noqa: E731
    at = orc.coordinates(dims, np.arange(120))
    # what was turned is rounded to the tensors' type, so the second half is checked from there
    turned = orc.rotary(host(qkv)[:, :nq + nk], at, layer.freqs, layer.axes)
    u = orc.roundoff(dtype)[0]
    assert (np.abs(host(layer.qkv)[:, :nq + nk] - turned) <= u * np.abs(turned) + 2.0 ** -20 * (1 + np.abs(turned))).all()
    a = orc.Attention(dims, offsets, host(layer.q), host(layer.k), host(layer.v), bias=host(layer.bias), cap=10.0)
    assert (np.abs(host(layer.out) - a.out) <= a.out_bound(dtype)).all()
    grads = a.backward(host(layer.grad_out), host(layer.out))
    assert (np.abs(host(layer.grad_bias) - grads["grad_bias"][0]) <= orc.gradient_bound(*grads["grad_bias"], dtype)).all()
    both = np.concatenate([grads["grad_q"][0], grads["grad_k"][0]], axis=1)
    bound = np.concatenate([orc.gradient_bound(*grads[n], dtype) for n in ("grad_q", "grad_k")], axis=1)
    back = orc.rotary(both, at, layer.freqs, layer.axes, inverse=True)
    pairs = D // 2                                 # a pair's error turns with it, and is rounded once more
    size = np.concatenate([bound[..., :pairs] + bound[..., pairs:]] * 2, axis=-1)
    assert (np.abs(host(layer.grad_qkv)[:, :nq + nk] - back) <= size + u * (np.abs(back) + size) + 2.0 ** -20 * (1 + np.abs(back))).all()
    assert (np.abs(host(layer.grad_qkv)[:, nq + nk:] - grads["grad_v"][0]) <= orc.gradient_bound(*grads["grad_v"], dtype)).all()
    rank = 67
    again = layer.one_token(rank, tuple(at[rank]), qkv[rank:rank + 1, :nq])
    assert (np.abs(host(again)[0] - a.out[rank]) <= a.out_bound(dtype)[rank]).all()


def test_the_example_runs(capsys):
    load_example().main()
    text = capsys.readouterr().out
    losses = [float(line.split("loss")[1]) for line in text.splitlines() if "loss" in line]
    assert len(losses) == 3 and losses[2] < losses[0]
    assert float(text.split("at most")[1]) < 0.05
