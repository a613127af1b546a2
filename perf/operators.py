"""What the speed of the attention over neighbourhoods, and of the rotary positions before it, is judged on.

A program that keeps one token (a cell of a picture, of a video or of a volume) at every rank of a torus or mesh
has its projections in one buffer [p][q heads + 2 kv heads][head_dim].  It turns queries and keys by the ranks'
coordinates, and every rank then attends to the tokens of its neighbours, those that the allgather over the same
neighbourhood would deliver.  Cases are single passes of these: the forward pass over all ranks, the same for
single new tokens, the backward pass, and the rotation with its inverse, which is its gradient.

Definitions.  Neighbour i of rank R is rank R - C_i, coordinate by coordinate: modulo the size where the dimension
wraps, no neighbour where it does not and the source lies outside.  With documents, only neighbours of the rank's
own document count, and a rank of document -1 has none.
    x_i = cap * tanh(scale * q . k_i / cap) + bias[head][i]        (no cap: scale * q . k_i + bias)
    lse = log(sum_i exp(x_i))        out = sum_i exp(x_i - lse) v_i        (no neighbour: lse = -inf, out = 0)
A rotation turns pairs of channels by position[axis of the pair] * frequency of the pair.
"""
import itertools
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
THETA = 10000.0
MAX_PRODUCTS = 256 * 256 * 169 * 8 * 64            # ranks * neighbours * q heads * head_dim of the largest listed attention
MAX_CHANNELS = 64 ** 3 * 10 * 128                  # of the largest listed rotation


def _attention(name, op, torus, shape, radius, q_heads, kv_heads, head_dim, dtype, *, wrap=True, bias=True, cap=0.0,
               documents=False, rows=0):
    """op: "forward", "backward" or "rows" (single tokens: `rows` ranks).  torus: "32x32x32".  shape: see offsets()."""
    return {"name": name, "op": op, "torus": torus, "wrap": wrap, "shape": shape, "radius": radius, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "bias": bias, "cap": cap, "documents": documents,
            "rows": rows}


def _rotary(name, torus, heads, head_dim, turned, dtype, *, interleaved=False, inverse=False, tokens=0):
    """tokens: 0 turns all ranks by their coordinates; n > 0 turns n tokens by positions that are handed over."""
    return {"name": name, "op": "rotary", "torus": torus, "heads": heads, "head_dim": head_dim, "turned": turned,
            "dtype": dtype, "interleaved": interleaved, "inverse": inverse, "tokens": tokens}


def listed():
    return [
        # one layer's attention on the smallest torus in use, in full precision: latency
        _attention("forward_8x8_f32", "forward", "8x8", "moore", 1, 4, 4, 16, "f32"),
        # a volume, 27 neighbours with the rank itself; heads share keys, scores are capped
        _attention("forward_32x32x32", "forward", "32x32x32", "moore", 1, 8, 2, 128, "bf16", cap=30.0),
        # a picture with windows of 13 x 13 and a learned bias for each offset
        _attention("forward_256x256_window13", "forward", "256x256", "moore", 6, 8, 8, 64, "bf16"),
        # packed video clips of odd size on a mesh, windows of 5 x 5 x 5, no bias; some cells hold no token
        _attention("forward_13x47x61_documents", "forward", "13x47x61", "moore", 2, 6, 3, 80, "f16", wrap=False, bias=False,
                   documents=True),
        # the next token of a volume that is generated cell by cell: 64 cells that came before
        _attention("rows_1_of_64x64x64", "rows", "64x64x64", "octant", 3, 16, 4, 128, "bf16", rows=1),
        # one step of 37 pictures' worth of cells that are drawn at the same time
        _attention("rows_37_of_256x256", "rows", "256x256", "moore", 6, 8, 8, 64, "f16", documents=True, rows=37),
        # training: gradients of the volume's layer
        _attention("backward_32x32x32", "backward", "32x32x32", "moore", 1, 8, 2, 128, "bf16", cap=30.0),
        # training: gradients of a picture's layer with windows of 7 x 7, pictures packed side by side
        _attention("backward_256x256_window7", "backward", "256x256", "moore", 3, 8, 8, 64, "bf16", documents=True),
        # training in full precision on a small mesh of odd sizes
        _attention("backward_12x11x10_f32", "backward", "12x11x10", "von_neumann", 1, 3, 1, 40, "f32", wrap=False),
        # serving: q and k of 5 new tokens at the positions that the request gives
        _rotary("rotary_5_tokens", "64x64x64", 20, 128, 128, "bf16", tokens=5),
        # q and k of a volume, three axes
        _rotary("rotary_64x64x64", "64x64x64", 10, 128, 128, "bf16"),
        # the gradient of a picture's rotation in full precision, part of the channels, neighbouring channels as pairs
        _rotary("rotary_inverse_255x257_f32", "255x257", 16, 80, 64, "f32", interleaved=True, inverse=True),
    ]


def draw(rng):
    """A case of the same ranges: tori of 1 to 4 dimensions and 16 to 262144 ranks, 2 to 400 neighbours."""
    return {key: value for key, value in _drawn(rng).items() if key != "name"}


def _drawn(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    d = rng.choice((1, 2, 2, 2, 3, 3, 3, 4))
    p = math.exp(rng.uniform(math.log(16), math.log(262144)))
    dims = [max(2, int(round(p ** (1 / d) * math.exp(rng.uniform(-0.5, 0.5))))) for _ in range(d)]
    torus = "x".join(str(n) for n in dims)
    p = math.prod(dims)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f16", "f16", "f32"))
    op = rng.choice(("forward", "forward", "rows", "backward", "backward", "rotary"))
    if op == "rotary":
        head_dim = 8 * rng.randint(2, 20)
        turned = 2 * rng.randint(max(1, d), head_dim // 2)
        heads = max(1, min(rng.randint(1, 40), MAX_CHANNELS // (p * head_dim)))
        tokens = 0 if dtype == "f32" or rng.random() < 0.5 else log(1, 20000)
        return _rotary("drawn", torus, heads, head_dim, turned, dtype, interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5,
                       tokens=tokens)
    shape, radius = rng.choice((("moore", 1), ("moore", 2), ("moore", 3), ("moore", 6), ("von_neumann", 1), ("von_neumann", 2),
                                ("octant", 1), ("octant", 3), ("random", 4)))
    while len(offsets(shape, d, radius)) > 400:
        radius -= 1
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    q_heads = kv_heads * rng.choice((1, 1, 2, 4))
    head_dim = rng.choice((32, 40, 64, 64, 80, 96, 128, 128)) if dtype != "f32" else 8 * rng.randint(2, 12)
    rows = log(1, min(p, 1000)) if op == "rows" else 0
    pairs = (rows or p) * len(offsets(shape, d, radius)) * (4 if dtype == "f32" else 1) * (2 if op == "backward" else 1)
    while pairs * q_heads * head_dim > MAX_PRODUCTS and (kv_heads > 1 or q_heads > 1 or head_dim > 32):
        if q_heads > kv_heads:
            q_heads //= 2
        elif kv_heads > 1:
            q_heads = kv_heads = kv_heads // 2
        else:
            head_dim = max(32, head_dim // 2 // 8 * 8)
    return _attention("drawn", op, torus, shape, radius, q_heads, kv_heads, head_dim, dtype, wrap=rng.random() < 0.6,
                      bias=rng.random() < 0.7, cap=rng.choice((0.0, 0.0, 20.0, 50.0)), documents=rng.random() < 0.4, rows=rows)


def dims_of(case):
    return [int(n) for n in case["torus"].split("x")]


def offsets(shape, d, radius):
    """The relative coordinates C_i in lexicographic order, the rank itself among them; random: 40 in drawn order."""
    if shape == "random":
        g = torch.Generator().manual_seed(d)
        box = torch.randint(-radius, radius + 1, (400, d), generator=g).tolist()
        return [list(c) for c in dict.fromkeys(tuple(c) for c in box)][:40]
    low = 0 if shape == "octant" else -radius
    box = itertools.product(range(low, radius + 1), repeat=d)
    return [list(c) for c in box if shape != "von_neumann" or sum(abs(x) for x in c) <= radius]


def axes_and_frequencies(case):
    """Which axis turns each pair of channels, and its frequency: the pairs shared out over the axes, a ladder for each."""
    pairs, d = case["turned"] // 2, len(dims_of(case))
    count = [pairs // d + (a < pairs % d) for a in range(d)]
    return ([a for a in range(d) for _ in range(count[a])],
            [THETA ** (-j / count[a]) for a in range(d) for j in range(count[a])])


def _coordinates(dims, ranks):
    """[n][d]: ranks are row-major, the last dimension fastest."""
    inner = [math.prod(dims[j + 1:]) for j in range(len(dims))]
    return torch.stack([ranks // inner[j] % dims[j] for j in range(len(dims))], 1)


def _documents(dims, generator):
    """Bands along the last dimension of uneven widths, one document each; the end of every line holds no token."""
    n = dims[-1]
    cuts = torch.rand(n, device=DEVICE, generator=generator) < 4.0 / n
    band = torch.cumsum(cuts, 0).to(torch.int32)
    band[-max(1, n // 20):] = -1
    return band.expand(*dims).reshape(-1).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dims, dtype = dims_of(case), DTYPES[case["dtype"]]
    p, d = math.prod(dims), len(dims)
    normal = lambda *size: torch.randn(*size, device=DEVICE, generator=g).to(dtype)  # noqa: E731
    if case["op"] == "rotary":
        axes, freqs = axes_and_frequencies(case)
        n = case["tokens"] or p
        state = {"x": normal(n, case["heads"], case["head_dim"]), "positions": None, "axes": axes, "freqs": freqs}
        state["out"] = torch.empty_like(state["x"])
        if case["tokens"]:                         # anywhere in a volume much larger than the torus
            state["positions"] = torch.randint(0, 4096, (n, d), device=DEVICE, generator=g, dtype=torch.int32)
        else:
            state["coordinates"] = _coordinates(dims, torch.arange(p, device=DEVICE))
    else:
        nq, nk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
        rel = offsets(case["shape"], d, case["radius"])
        qkv = normal(p, nq + 2 * nk, D)
        state = {"q": qkv[:, :nq], "k": qkv[:, nq:nq + nk], "v": qkv[:, nq + nk:], "rows": None, "bias": None,
                 "documents": _documents(dims, g) if case["documents"] else None}
        if case["bias"]:
            state["bias"] = normal(nq, len(rel))
        ranks = torch.arange(p, device=DEVICE)
        if case["rows"]:
            ranks = state["rows"] = torch.randperm(p, device=DEVICE, generator=g)[:case["rows"]].contiguous()
            state["q"] = normal(case["rows"], nq, D)
        state["source"] = _sources(dims, rel, ranks, case["wrap"])       # what a program without the library keeps in its place
        state["out"] = torch.empty(len(ranks), nq, D, device=DEVICE, dtype=dtype)
        state["lse"] = torch.empty(len(ranks), nq, device=DEVICE)
        if case["op"] == "backward":
            state["grad_out"] = normal(p, nq, D)
            _plain_forward(case, state, into=state)                      # the forward pass left these behind
            state["target"] = _sources(dims, [[-x for x in c] for c in rel], ranks, case["wrap"])
            grads = torch.empty_like(qkv)
            state |= {"grad_q": grads[:, :nq], "grad_k": grads[:, nq:nq + nk], "grad_v": grads[:, nq + nk:],
                      "grad_bias": None if state["bias"] is None else torch.empty_like(state["bias"])}
    if own:                                        # the persistent request, bound to the buffers, that a program keeps
        state["request"] = _bind(case, state, dims)
    return state | {"case": case}


def _sources(dims, rel, ranks, wrap):
    """[n][s] source ranks, -1 where there is none."""
    size = torch.tensor(dims, device=DEVICE)
    at = _coordinates(dims, ranks)[:, None, :] - torch.tensor(rel, device=DEVICE)[None]
    inside = (at >= 0).logical_and(at < size).all(-1)
    inner = torch.tensor([math.prod(dims[j + 1:]) for j in range(len(dims))], device=DEVICE)
    rank = ((at % size) * inner).sum(-1)
    return rank if wrap else torch.where(inside, rank, -1)


def _bind(case, state, dims):
    import paper_1606_07676_amd as iso
    if case["op"] == "rotary":
        comm = None if case["tokens"] else iso.iso_neighborhood_create(dims, [[0] * len(dims)])
        return iso.iso_rotary_init(state["x"], state["out"], state["freqs"], state["axes"], comm, positions=state["positions"],
                                   interleaved=case["interleaved"], inverse=case["inverse"])
    rel = offsets(case["shape"], len(dims), case["radius"])
    comm = iso.iso_neighborhood_create(dims, rel) if case["wrap"] else iso.iso_neighborhood_create_mesh(dims, [0] * len(dims), rel)
    more = {"bias": state["bias"], "segments": state["documents"], "cap": case["cap"]}
    if case["op"] != "backward":
        return iso.iso_neighbor_attention_init(state["q"], state["k"], state["v"], state["out"], comm, lse=state["lse"],
                                               rows=state["rows"], **more)
    work = torch.empty(iso.iso_neighbor_attention_backward_workspace_bytes(
        comm, case["q_heads"], case["kv_heads"], case["head_dim"], state["q"].dtype, bias=case["bias"]), dtype=torch.uint8, device=DEVICE)
    return iso.iso_neighbor_attention_backward_init(
        state["q"], state["k"], state["v"], state["out"], state["lse"], state["grad_out"], state["grad_q"], state["grad_k"],
        state["grad_v"], work, comm, grad_bias=state["grad_bias"], **more)


def run(state):
    case = state["case"]
    if own:
        import paper_1606_07676_amd as iso
        iso.iso_start(state["request"])
        if case["op"] == "rotary":
            return state["out"]
        if case["op"] != "backward":
            return {"out": state["out"], "lse": state["lse"]}
        return {k: state[k] for k in ("grad_q", "grad_k", "grad_v", "grad_bias") if state[k] is not None}
    if case["op"] == "rotary":
        return _plain_rotary(case, state)
    if case["op"] != "backward":
        return _plain_forward(case, state)
    return _plain_backward(case, state)


def _plain_rotary(case, state):
    x, pairs = state["x"].float(), case["turned"] // 2
    at = state["positions"] if case["tokens"] else state["coordinates"]
    axes, freqs = torch.tensor(state["axes"], device=DEVICE), torch.tensor(state["freqs"], device=DEVICE)
    angle = at.float()[:, axes] * freqs * (-1.0 if case["inverse"] else 1.0)
    cos, sin = angle.cos()[:, None, :], angle.sin()[:, None, :]
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if case["interleaved"] else (slice(0, pairs), slice(pairs, 2 * pairs))
    out = x.clone()
    out[..., first] = x[..., first] * cos - x[..., second] * sin
    out[..., second] = x[..., first] * sin + x[..., second] * cos
    return out.to(state["x"].dtype)


def _plain_scores(case, state):
    """x [n][kv heads][heads of a group][s], -inf where there is no neighbour, and the capped scores without the bias."""
    q, k, source = state["q"].float(), state["k"].float(), state["source"]
    n, s, nk = source.shape[0], source.shape[1], case["kv_heads"]
    keys = k[source.clamp(min=0)].permute(0, 2, 3, 1)                    # [n][kv heads][head_dim][s]
    t = torch.matmul(q.reshape(n, nk, -1, case["head_dim"]), keys) * case["head_dim"] ** -0.5
    if case["cap"]:
        t = case["cap"] * torch.tanh(t / case["cap"])
    x = t if state["bias"] is None else t + state["bias"].float().reshape(nk, -1, s)
    there = source >= 0
    if state["documents"] is not None:
        mine = state["documents"] if state["rows"] is None else state["documents"][state["rows"]]
        there = there & (state["documents"][source.clamp(min=0)] == mine[:, None]) & (mine >= 0)[:, None]
    return torch.where(there[:, None, None, :], x, -math.inf), t


def _plain_forward(case, state, into=None):
    x, _ = _plain_scores(case, state)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).flatten(1)
    values = state["v"].float()[state["source"].clamp(min=0)].permute(0, 2, 1, 3)          # [n][kv heads][s][head_dim]
    out = torch.matmul(e / total.clamp(min=1e-38), values).flatten(1, 2).to(state["v"].dtype)
    if into is not None:
        into["out"].copy_(out)
        into["lse"].copy_(lse)
    return {"out": out, "lse": lse}


def _plain_backward(case, state):
    nk, D, source, target = case["kv_heads"], case["head_dim"], state["source"], state["target"]
    p, s = source.shape
    grouped = lambda y: y.float().reshape(p, nk, -1, D)                  # noqa: E731
    x, t = _plain_scores(case, state)
    P = torch.exp(x - state["lse"].reshape(p, nk, -1, 1).clamp(min=-3e38))
    values = state["v"].float()[source.clamp(min=0)].permute(0, 2, 3, 1)
    dP = torch.matmul(grouped(state["grad_out"]), values)
    dX = P * (dP - (grouped(state["grad_out"]) * grouped(state["out"])).sum(-1, keepdim=True))
    del values, dP, x
    dA = dX * D ** -0.5
    if case["cap"]:
        dA = dA * (1 - (t / case["cap"]) ** 2)
    keys = state["k"].float()[source.clamp(min=0)].permute(0, 2, 1, 3)
    grad_q = torch.matmul(dA, keys).flatten(1, 2)
    del keys, t
    # the key at rank S is neighbour i of rank S + C_i: sums over these ranks, and over the heads that share the key
    there = (target >= 0)[:, None, :, None]
    number = torch.arange(s, device=DEVICE).expand(p, s)

    def back(weights, rows):
        w = weights.permute(0, 3, 1, 2)[target.clamp(min=0), number].permute(0, 2, 1, 3) * there       # [p][kv heads][s][group]
        y = grouped(rows)[target.clamp(min=0)].permute(0, 2, 1, 3, 4).reshape(p, nk, -1, D)
        return torch.matmul(w.reshape(p, nk, 1, -1), y).flatten(1, 2)

    dtype = state["q"].dtype
    grads = {"grad_q": grad_q.to(dtype), "grad_k": back(dA, state["q"]).to(dtype), "grad_v": back(P, state["grad_out"]).to(dtype)}
    if state["bias"] is not None:
        grads["grad_bias"] = dX.sum(0).flatten(0, 1).to(dtype)
    return grads


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    dims = dims_of(case)
    p, d = math.prod(dims), len(dims)
    if case["op"] == "rotary":
        n = case["tokens"] or p
        channels = n * case["heads"] * case["head_dim"]
        return {"bytes": 2 * channels * size + (4 * n * d if case["tokens"] else 0), "flops": 3 * n * case["heads"] * case["turned"]}
    rel = offsets(case["shape"], d, case["radius"])
    nq, nk, D, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["rows"] or p
    pairs = sum(math.prod(max(0, m - (0 if case["wrap"] else abs(x))) for m, x in zip(dims, c)) for c in rel) * n // p
    bias, documents = (nq * len(rel) * size if case["bias"] else 0), (4 * p if case["documents"] else 0)
    kv = 2 * nk * D * size * min(p, n * len(rel))
    row = nq * D * size
    if case["op"] == "backward":                   # q, out, grad_out, k, v, lse in; grad_q, grad_k, grad_v out
        return {"bytes": 4 * p * row + 2 * kv + 4 * p * nq + 2 * bias + documents, "flops": 10 * pairs * nq * D}
    return {"bytes": 2 * n * row + kv + 4 * n * nq + bias + (documents if not case["rows"] else 0), "flops": 4 * pairs * nq * D}


def exact(case, seed):
    """The definitions above in 64 bits, neighbour by neighbour over the grid of coordinates."""
    state = prepare(case, seed)
    dims = dims_of(case)
    p, d = math.prod(dims), len(dims)
    strides = [1] * d
    for j in range(d - 2, -1, -1):
        strides[j] = strides[j + 1] * dims[j + 1]
    ranks = torch.arange(p, device=DEVICE)
    where = [torch.div(ranks, strides[j], rounding_mode="floor") % dims[j] for j in range(d)]
    if case["op"] == "rotary":
        x, half = state["x"].double(), case["turned"] // 2
        y = x.clone()
        for j, (axis, f) in enumerate(zip(state["axes"], state["freqs"])):
            w = (where[axis] if state["positions"] is None else state["positions"][:, axis]).double() * f
            w = (-w if case["inverse"] else w)[:, None]
            a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, half + j)
            y[..., a] = x[..., a] * w.cos() - x[..., b] * w.sin()
            y[..., b] = x[..., b] * w.cos() + x[..., a] * w.sin()
        return y
    rel = offsets(case["shape"], d, case["radius"])
    nq, group = case["q_heads"], case["q_heads"] // case["kv_heads"]
    me = ranks if state["rows"] is None else state["rows"]
    q, k, v = (state[n].double() for n in "qkv")
    bias = state["bias"].double() if state["bias"] is not None else torch.zeros(nq, len(rel), device=DEVICE, dtype=torch.float64)
    scale = 1 / math.sqrt(case["head_dim"])

    def neighbour(i):
        """Its rank, whether it counts, and its score with and without the bias, for all of `me`."""
        src, ok = torch.zeros_like(me), torch.ones_like(me, dtype=torch.bool)
        for j in range(d):
            c = where[j][me] - rel[i][j]
            if not case["wrap"]:
                ok &= (c >= 0) & (c < dims[j])
            src += torch.remainder(c, dims[j]) * strides[j]
        if state["documents"] is not None:
            ok &= (state["documents"][src] == state["documents"][me]) & (state["documents"][me] != -1)
        a = scale * (q * k[src].repeat_interleave(group, 1)).sum(-1)
        t = case["cap"] * torch.tanh(a / case["cap"]) if case["cap"] else a
        x = t + bias[:, i]
        x[~ok] = -math.inf
        return src, x, t

    scores = torch.stack([neighbour(i)[1] for i in range(len(rel))])     # [s][n][q heads]
    lse = torch.logsumexp(scores, 0)
    safe = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
    out = torch.zeros(len(me), nq, case["head_dim"], device=DEVICE, dtype=torch.float64)
    for i in range(len(rel)):
        out += torch.exp(scores[i] - safe)[..., None] * v[neighbour(i)[0]].repeat_interleave(group, 1)
    if case["op"] != "backward":
        return {"out": out, "lse": lse}
    do = state["grad_out"].double()
    delta = (do * out).sum(-1)
    grads = {"grad_q": torch.zeros_like(q), "grad_k": torch.zeros_like(k), "grad_v": torch.zeros_like(v), "grad_bias": torch.zeros_like(bias)}
    shared = lambda y: y.reshape(p, -1, group, y.shape[-1]).sum(2)       # noqa: E731
    for i in range(len(rel)):
        src, x, t = neighbour(i)
        e = torch.exp(x - safe)
        dx = e * ((do * v[src].repeat_interleave(group, 1)).sum(-1) - delta)
        da = scale * dx * ((1 - (t / case["cap"]) ** 2) if case["cap"] else 1)
        grads["grad_bias"][:, i] = dx.sum(0)
        grads["grad_q"] += da[..., None] * k[src].repeat_interleave(group, 1)
        grads["grad_k"].index_add_(0, src, shared(da[..., None] * q))
        grads["grad_v"].index_add_(0, src, shared(e[..., None] * do))
    if state["bias"] is None:
        del grads["grad_bias"]
    return grads
