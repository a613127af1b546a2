"""What the speed of the rest of a layer over the ranks' tokens is judged on: layer norm, the gated projections of the
feed-forward block, and dropout.

A program that keeps one token at every rank of a torus or mesh has, besides the attention over the neighbours, work on
each token by itself: its row is normalised before the attention and before the feed-forward block (and queries and keys head
by head), two projections of the row are joined to the block's hidden units, and what either block gives is added to the
token with dropout.  Cases are single passes of these: forward, backward, and for the few tokens of one serving step.

Definitions.
    layer norm     h = (x - mean) * rstd      out = weight * h + bias       rstd = 1 / sqrt(var + eps), var over the row's elements
                   grad_x = rstd * (g - mean(g) - h * mean(g * h)), g = weight * grad_out
                   grad_weight = sum grad_out * h      grad_bias = sum grad_out      over all rows
    gated          out = f(x . gate) * (x . up)        f(g) = g / (1 + exp(-g)), or g * (1 + erf(g / sqrt 2)) / 2
    dropout        out = residual + x * 65536 / (65536 - t) where the element's number r >= t, residual elsewhere;
                   t = rate * 65536, rounded.  Its gradient is the same call on the gradient, without the residual.
The numbers r come from Philox4x32-10 (Salmon, Moraes, Dror, Shaw, 2011), 16 bits an element: element e of the tensor in
row-major order takes the (e % 8)th half word, low halves first, of the block with the counter (e / 8, second number of the
seed) and the key (first number of the seed), each 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_ELEMENTS = 64 ** 3 * 10 * 128                  # of the largest listed tensor that is gone through once
MAX_PRODUCTS = 32 ** 3 * 1024 * 4096               # tokens * channels * hidden of the largest listed projection
EPS = 1e-5


def _norm(name, op, tokens, heads, channels, dtype, *, affine=True):
    """op: "norm" or "norm_backward".  heads > 1: queries or keys, a part of the buffer of all projections."""
    return {"name": name, "op": op, "tokens": tokens, "heads": heads, "channels": channels, "dtype": dtype, "affine": affine}


def _gated(name, op, tokens, channels, hidden, dtype, *, activation="silu"):
    """op: "gated" or "gated_backward"."""
    return {"name": name, "op": op, "tokens": tokens, "channels": channels, "hidden": hidden, "dtype": dtype, "activation": activation}


def _dropout(name, tokens, channels, rate, dtype, *, residual=True):
    return {"name": name, "op": "dropout", "tokens": tokens, "channels": channels, "rate": rate, "dtype": dtype, "residual": residual}


def listed():
    return [
        # one layer's norm on the smallest torus in use, in full precision: latency
        _norm("norm_8x8_f32", "norm", 8 * 8, 1, 64, "f32"),
        # a volume's norm before its attention or its feed-forward block
        _norm("norm_32x32x32", "norm", 32 ** 3, 1, 1024, "bf16"),
        # queries and keys of a volume, head by head, out of the buffer of all projections; no bias, no weight
        _norm("norm_heads_64x64x64", "norm", 64 ** 3, 10, 128, "bf16", affine=False),
        # training: gradients of the volume's norm
        _norm("norm_backward_32x32x32", "norm_backward", 32 ** 3, 1, 1024, "bf16"),
        # training on packed video clips of odd size, an odd number of channels
        _norm("norm_backward_13x47x61", "norm_backward", 13 * 47 * 61, 1, 483, "f16"),
        # a block's result joins the volume's tokens
        _dropout("dropout_32x32x32", 32 ** 3, 1024, 0.1, "bf16"),
        # the gradient of a picture's dropout in full precision, an odd number of channels
        _dropout("dropout_255x257_f32", 255 * 257, 333, 0.25, "f32", residual=False),
        # the feed-forward block of the next token of a volume that is generated cell by cell
        _gated("gated_1_token", "gated", 1, 2048, 5632, "bf16"),
        # the same for 37 cells that are drawn at the same time
        _gated("gated_37_tokens", "gated", 37, 512, 1408, "f16", activation="gelu"),
        # a volume's feed-forward block
        _gated("gated_32x32x32", "gated", 32 ** 3, 1024, 4096, "bf16"),
        # training: its gradients
        _gated("gated_backward_32x32x32", "gated_backward", 32 ** 3, 1024, 2816, "bf16"),
        # training in full precision on a small mesh of odd sizes
        _gated("gated_backward_12x11x10_f32", "gated_backward", 12 * 11 * 10, 120, 343, "f32", activation="gelu"),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 262144 tokens, 16 to 4096 channels, 16 to 8192 hidden units."""
    return {key: value for key, value in _drawn(rng).items() if key != "name"}


def _drawn(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    dtype = rng.choice(("bf16", "bf16", "bf16", "f16", "f16", "f32"))
    op = rng.choice(("norm", "norm_backward", "dropout", "gated", "gated", "gated_backward", "gated_backward"))
    tokens = log(1, 262144)
    channels = log(16, 4096)
    if rng.random() < 0.7:                         # mostly whole groups of 8
        channels = max(16, channels // 8 * 8)
    if op in ("norm", "norm_backward"):
        heads = 1
        if rng.random() < 0.3:
            heads, channels = rng.randint(2, 32), rng.choice((32, 40, 64, 80, 96, 128))
        share = (2 if op == "norm_backward" else 1) * (2 if dtype == "f32" else 1)
        tokens = max(1, min(tokens, MAX_ELEMENTS // (share * heads * channels)))
        return _norm("drawn", op, tokens, heads, channels, dtype, affine=rng.random() < 0.7)
    if op == "dropout":
        tokens = max(1, min(tokens, MAX_ELEMENTS // 4 // channels))
        return _dropout("drawn", tokens, channels, rng.choice((0.05, 0.1, 0.2, 0.3, 0.5)), dtype, residual=rng.random() < 0.5)
    if rng.random() < 0.3:
        tokens = log(1, 64)                        # a serving step
    hidden = max(16, min(8192, int(channels * rng.uniform(1.5, 4.5))))
    if rng.random() < 0.7:
        hidden = max(16, hidden // 8 * 8)
    cost = channels * hidden * (3 if op == "gated_backward" else 1) * (8 if dtype == "f32" else 1)
    tokens = max(1, min(tokens, MAX_PRODUCTS // cost))
    return _gated("drawn", op, tokens, channels, hidden, dtype, activation=rng.choice(("silu", "silu", "gelu")))


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, op, n, C = DTYPES[case["dtype"]], case["op"], case["tokens"], case["channels"]
    normal = lambda *size: torch.randn(*size, device=DEVICE, generator=g)  # noqa: E731
    empty = lambda *size, of=dtype: torch.empty(*size, device=DEVICE, dtype=of)  # noqa: E731
    state = {}
    if op in ("norm", "norm_backward"):
        heads = case["heads"]
        if heads > 1:                              # the first heads of rows that hold values as well
            x, out, grad_out = (normal(n, heads + 2, C)[:, :heads] for _ in range(3))
        else:                                      # a token's row: some channels are far larger than the others
            x, out, grad_out = normal(n, 1, C), normal(n, 1, C), normal(n, 1, C)
            x = x * torch.exp(0.7 * normal(C)) + 0.5 * normal(C)
        state = {"x": x.to(dtype), "weight": None, "bias": None,
                 "mean": empty(n, heads, of=torch.float32), "rstd": empty(n, heads, of=torch.float32)}
        if case["affine"]:
            state |= {"weight": (1 + 0.2 * normal(C)).to(dtype), "bias": (0.2 * normal(C)).to(dtype)}
        if op == "norm":
            state["out"] = out.to(dtype)
        else:
            state |= {"grad_out": grad_out.to(dtype), "grad_x": torch.empty_like(out.to(dtype)),
                      "grad_weight": empty(C) if case["affine"] else None, "grad_bias": empty(C) if case["affine"] else None}
            h = _plain_norm(state)                 # the forward pass left these behind
            state["mean"].copy_(h["mean"])
            state["rstd"].copy_(h["rstd"])
    elif op == "dropout":
        state = {"x": normal(n, C).to(dtype), "residual": normal(n, C).to(dtype) if case["residual"] else None, "out": empty(n, C),
                 "seed": torch.randint(-2 ** 63, 2 ** 63 - 1, (2,), device=DEVICE, generator=g, dtype=torch.int64)}
    else:
        F = case["hidden"]
        state = {"x": normal(n, C).to(dtype), "gate": (normal(F, C) * C ** -0.5).to(dtype), "up": (normal(F, C) * C ** -0.5).to(dtype)}
        if op == "gated":
            state["out"] = empty(n, F)
        else:
            state |= {"grad_out": normal(n, F).to(dtype), "grad_x": empty(n, C), "grad_gate": empty(F, C), "grad_up": empty(F, C)}
    if own:                                        # the persistent request, bound to the buffers, that a program keeps
        state["request"] = _bind(case, state)
    return state | {"case": case}


def _bind(case, state):
    import paper_1606_07676_amd as iso
    op, dtype, s = case["op"], DTYPES[case["dtype"]], state
    scratch = lambda size: torch.empty(size, dtype=torch.uint8, device=DEVICE)  # noqa: E731
    if op == "norm":
        return iso.iso_layer_norm_init(s["x"], s["out"], weight=s["weight"], bias=s["bias"], eps=EPS, mean=s["mean"], rstd=s["rstd"])
    if op == "norm_backward":
        work = scratch(iso.iso_layer_norm_backward_workspace_bytes(case["tokens"], case["heads"], case["channels"], dtype))
        return iso.iso_layer_norm_backward_init(s["x"], s["mean"], s["rstd"], s["grad_out"], s["grad_x"], work, weight=s["weight"],
                                                grad_weight=s["grad_weight"], grad_bias=s["grad_bias"])
    if op == "dropout":
        return iso.iso_dropout_init(s["x"], s["out"], s["seed"], case["rate"], residual=s["residual"])
    if op == "gated":
        return iso.iso_gated_init(s["x"], s["gate"], s["up"], s["out"], activation=case["activation"])
    work = scratch(iso.iso_gated_backward_workspace_bytes(case["tokens"], case["channels"], case["hidden"], dtype))
    return iso.iso_gated_backward_init(s["x"], s["gate"], s["up"], s["grad_out"], s["grad_x"], s["grad_gate"], s["grad_up"], work,
                                       activation=case["activation"])


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_1606_07676_amd as iso
        iso.iso_start(state["request"])
        names = {"norm": ("out", "mean", "rstd"), "norm_backward": ("grad_x", "grad_weight", "grad_bias"), "dropout": ("out",),
                 "gated": ("out",), "gated_backward": ("grad_x", "grad_gate", "grad_up")}[op]
        return {name: state[name] for name in names if state[name] is not None}
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "dropout": _plain_dropout, "gated": _plain_gated,
            "gated_backward": _plain_gated_backward}[op](state)


def _plain_norm(state):
    x = state["x"].float()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + EPS)
    out = (x - mean) * rstd
    if state["weight"] is not None:
        out = out * state["weight"].float() + state["bias"].float()
    return {"out": out.to(state["x"].dtype), "mean": mean[..., 0], "rstd": rstd[..., 0]}


def _plain_norm_backward(state):
    dtype, dy = state["x"].dtype, state["grad_out"].float()
    rstd = state["rstd"][..., None]
    h = (state["x"].float() - state["mean"][..., None]) * rstd
    g = dy if state["weight"] is None else dy * state["weight"].float()
    grads = {"grad_x": (rstd * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))).to(dtype)}
    if state["weight"] is not None:
        grads |= {"grad_weight": (dy * h).sum((0, 1)).to(dtype), "grad_bias": dy.sum((0, 1)).to(dtype)}
    return grads


def _plain_dropout(state):
    case, x = state["case"], state["x"]
    low = 0xFFFFFFFF
    block = torch.arange((x.numel() + 7) // 8, device=DEVICE)
    key, more = state["seed"][0], state["seed"][1]
    c0, c1, c2, c3 = block & low, block >> 32, (more & low).expand_as(block), (more >> 32 & low).expand_as(block)
    k0, k1 = key & low, key >> 32 & low
    for _ in range(10):                            # products modulo 2^64: both halves come out right
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    r = torch.stack([words & 0xFFFF, words >> 16], 2).flatten()[:x.numel()].reshape(x.shape)
    t = int(math.floor(case["rate"] * 65536 + 0.5))
    y = torch.where(r >= t, x.float() * (65536 / (65536 - t)), 0.0)
    if state["residual"] is not None:
        y = state["residual"].float() + y
    return {"out": y.to(x.dtype)}


def _activation(case, g):
    """f(g) and its derivative."""
    if case["activation"] == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_gated(state):
    x = state["x"].float()
    g, u = x @ state["gate"].float().t(), x @ state["up"].float().t()
    return {"out": (_activation(state["case"], g)[0] * u).to(state["x"].dtype)}


def _plain_gated_backward(state):
    dtype = state["x"].dtype
    x, gate, up, dy = (state[name].float() for name in ("x", "gate", "up", "grad_out"))
    f, slope = _activation(state["case"], x @ gate.t())
    dg, du = dy * (x @ up.t()) * slope, dy * f
    del f, slope
    return {"grad_x": (dg @ gate + du @ up).to(dtype), "grad_gate": (dg.t() @ x).to(dtype), "grad_up": (du.t() @ x).to(dtype)}


def work(case):
    size, n, C = DTYPES[case["dtype"]].itemsize, case["tokens"], case["channels"]
    if case["op"] == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * n * C * size + 16, "flops": (2 if case["residual"] else 1) * n * C}
    if case["op"] in ("norm", "norm_backward"):
        rows, affine = n * case["heads"], 2 * C * size if case["affine"] else 0
        if case["op"] == "norm":
            return {"bytes": 2 * rows * C * size + 8 * rows + affine, "flops": (7 if case["affine"] else 5) * rows * C}
        return {"bytes": 3 * rows * C * size + 8 * rows + affine * 3 // 2, "flops": (12 if case["affine"] else 8) * rows * C}
    F = case["hidden"]
    if case["op"] == "gated":
        return {"bytes": (n * C + 2 * F * C + n * F) * size, "flops": 4 * n * C * F}
    return {"bytes": (2 * n * C + 4 * F * C + n * F) * size, "flops": 12 * n * C * F}


def exact(case, seed):
    """The definitions above in 64 bits: row norms and projections in slices of the tokens, the generator in numpy on the host."""
    state = prepare(case, seed)
    op, n = case["op"], case["tokens"]
    wide = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in state.items()
            if k in ("weight", "bias", "gate", "up")}
    if op == "dropout":
        return {"out": _exact_dropout(case, state)}
    step = max(1, 2 ** 25 // (case["channels"] * case.get("heads", 1) + 4 * case.get("hidden", 0)))
    slices = [slice(i, min(n, i + step)) for i in range(0, n, step)]
    parts, sums = [], {}
    for rows in slices:
        x = state["x"][rows].double()
        if op in ("norm", "norm_backward"):
            mean = x.sum(-1, keepdim=True) / case["channels"]
            var = ((x - mean) ** 2).sum(-1, keepdim=True) / case["channels"]
            h = (x - mean) / (var + EPS) ** 0.5
            if op == "norm":
                y = h if wide["weight"] is None else torch.addcmul(wide["bias"], h, wide["weight"])
                parts.append({"out": y, "mean": mean.squeeze(-1), "rstd": (var + EPS).squeeze(-1) ** -0.5})
                continue
            dy = state["grad_out"][rows].double()
            dh = dy if wide["weight"] is None else dy * wide["weight"]
            # the normalised row does not change along the row of ones and, up to eps, along itself
            dx = dh - dh.mean(-1, keepdim=True) - h * (dh * h).mean(-1, keepdim=True)
            parts.append({"grad_x": dx / (var + EPS) ** 0.5})
            if case["affine"]:
                _add(sums, "grad_weight", torch.einsum("thc,thc->c", dy, h))
                _add(sums, "grad_bias", torch.einsum("thc->c", dy))
            continue
        gate, up = torch.mm(x, wide["gate"].T), torch.mm(x, wide["up"].T)
        if case["activation"] == "silu":
            share = torch.sigmoid(gate)
            slope = share + gate * share * torch.sigmoid(-gate)
        else:
            share = torch.erfc(-gate / 2 ** 0.5) / 2
            slope = share + gate * torch.exp(-gate ** 2 / 2) / (2 * math.pi) ** 0.5
        if op == "gated":
            parts.append({"out": gate * share * up})
            continue
        dy = state["grad_out"][rows].double()
        d_gate, d_up = dy * up * slope, dy * gate * share
        parts.append({"grad_x": torch.mm(d_gate, wide["gate"]) + torch.mm(d_up, wide["up"])})
        _add(sums, "grad_gate", torch.mm(d_gate.T, x))
        _add(sums, "grad_up", torch.mm(d_up.T, x))
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]} | sums


def _add(sums, name, value):
    sums[name] = sums[name] + value if name in sums else value


def _exact_dropout(case, state):
    n = state["x"].numel()
    seed = state["seed"].cpu().numpy().view(np.uint64)
    half, mask = np.uint64(32), np.uint64(0xFFFFFFFF)
    x = [np.arange((n + 7) // 8, dtype=np.uint64), np.uint64(0), np.full(1, seed[1] & mask), np.full(1, seed[1] >> half)]
    x[1] = x[0] >> half
    x[0] = x[0] & mask
    key = [seed[0] & mask, seed[0] >> half]
    for turn in range(10):
        p = np.uint64(0xD2511F53) * x[0]
        q = np.uint64(0xCD9E8D57) * x[2]
        x = [(q >> half) ^ x[1] ^ key[0], q & mask, (p >> half) ^ x[3] ^ key[1], p & mask]
        key = [np.uint64((int(key[0]) + 0x9E3779B9) % 2 ** 32), np.uint64((int(key[1]) + 0xBB67AE85) % 2 ** 32)]
    block = np.empty(((n + 7) // 8, 4), dtype="<u4")
    for i in range(4):
        block[:, i] = x[i]
    r = torch.from_numpy(block.view("<u2").reshape(-1)[:n].astype(np.int32)).to(DEVICE).reshape(state["x"].shape)
    dropped = int(case["rate"] * 65536 + 0.5)
    y = state["x"].double() * (65536.0 / (65536.0 - dropped))
    y[r < dropped] = 0
    return y if state["residual"] is None else y + state["residual"].double()
