"""Shared by the tests of the operators on each token by itself."""
import numpy as np
import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {name: torch.finfo(t).eps / 2 for name, t in TYPES.items()}


def host(x):
    return x.detach().cpu().to(torch.float64).numpy()


def within(got, want, bound, what):
    assert got.shape == want.shape, what
    off = np.abs(got - want) / bound
    assert not off.size or off.max() <= 1, (what, float(off.max()), int((~(off <= 1)).sum()), off.size)


def inside_rows(shape, dtype, gap, shift, fill=9.0):
    """A view of the shape with `gap` more elements behind the last dimension, `shift` elements into its buffer."""
    wide = shape[:-1] + (shape[-1] + gap,)
    buffer = torch.full((int(np.prod(wide)) + shift,), fill, device=DEV, dtype=dtype)
    view = buffer[shift:].view(wide)[..., :shape[-1]]
    view.around = (buffer, shift, wide, shape[-1], fill)
    return view


def untouched_around(view):
    buffer, shift, wide, used, fill = view.around
    assert bool((buffer[:shift] == fill).all()) and bool((buffer[shift:].view(wide)[..., used:] == fill).all()), "written outside its rows"
