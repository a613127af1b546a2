"""Plain definitions, in numpy and 64 bits, of the operators on the ranks' tokens: attention over an isomorphic
neighbourhood with its gradients, and rotary positions.  Every sum is written out over gathered copies; nothing is
shared with the library.  The bounds say how far a result of 32-bit arithmetic on elements with the unit roundoff u may
be off, element by element."""


import numpy as np


def coordinates(dims, ranks):
    return np.stack(np.unravel_index(np.asarray(ranks, dtype=np.int64), dims), axis=-1)


def neighbours(dims, offsets, periodic=None, ranks=None):
    """[n][s] source ranks R (-) C^i, -1 where a mesh has none."""
    dims = np.asarray(dims, dtype=np.int64)
    periodic = np.ones(len(dims), bool) if periodic is None else np.asarray(periodic, bool)
    ranks = np.arange(int(np.prod(dims))) if ranks is None else np.asarray(ranks)
    rel = np.asarray(offsets, dtype=np.int64).reshape(len(offsets), len(dims))
    at = coordinates(dims, ranks)[:, None, :] - rel[None, :, :]
    there = np.all(periodic | ((at >= 0) & (at < dims)), axis=-1)
    at = np.mod(at, dims)
    return np.where(there, np.ravel_multi_index(tuple(np.moveaxis(at, -1, 0)), dims), -1)


class Attention:
    """q: [n][q heads][D] (n = p, or len(rows)); k, v: [p][kv heads][D]; all float64.  Attributes: out, lse, and the
    bounds' ingredients."""

    def __init__(self, dims, offsets, q, k, v, *, periodic=None, bias=None, segments=None, scale=None, cap=0.0, rows=None):
        self.scale = q.shape[-1] ** -0.5 if scale is None else scale
        self.cap, self.q, self.k, self.v = cap, q, k, v
        n, self.group, self.s = q.shape[0], q.shape[1] // k.shape[1], len(offsets)
        p = k.shape[0]
        ranks = np.arange(p) if rows is None else np.asarray(rows)
        inside = (ranks >= 0) & (ranks < p)
        src = neighbours(dims, offsets, periodic, np.where(inside, ranks, 0))
        ok = (src >= 0) & inside[:, None]
        if segments is not None:
            own = segments[np.where(inside, ranks, 0)]
            ok &= (segments[src] == own[:, None]) & (own >= 0)[:, None]
        self.src, self.ok = np.where(ok, src, 0), ok
        clean = lambda x: np.where(ok[:, :, None, None], np.repeat(x, self.group, axis=1)[self.src], 0.0)  # noqa: E731
        self.ks, self.vs = clean(k), clean(v)                                  # [n][s][q heads][D]
        a = self.scale * np.einsum("nhd,nshd->nsh", q, self.ks)
        self.t = cap * np.tanh(a / cap) if cap else a
        x = self.t + (0.0 if bias is None else bias.T[None])
        x = np.where(ok[:, :, None], x, -np.inf)
        top = np.where(np.isneginf(x.max(axis=1, initial=-np.inf)), 0.0, x.max(axis=1, initial=-np.inf))
        with np.errstate(divide="ignore"):
            self.lse = top + np.log(np.exp(x - top[:, None]).sum(axis=1))
        self.P = np.exp(x - np.where(np.isneginf(self.lse), 0.0, self.lse)[:, None])
        self.out = np.einsum("nsh,nshd->nhd", self.P, self.vs)
        size = (self.scale * np.einsum("nhd,nshd->nsh", np.abs(q), np.abs(self.ks))).max(initial=0.0)
        big = np.abs(x[np.isfinite(x)]).max(initial=0.0)
        big = min(big, 1e4)                       # scores near the type's lowest value are equal after rounding, or count nothing
        # a dot of D terms in 32 bits (both in q . k and in dO . v, dO . out), the cap's tanh, the exponential and the sums
        self.e = 2.0 ** -24 * (2 * q.shape[-1] * (size + 2) + 16 * big + 32 * cap + 64 + 2 * self.s ** 0.5)

    def out_bound(self, dtype):
        """The weights may be rounded to the tensors' type once, and the result once."""
        u, tiny = roundoff(dtype)
        return (u * np.abs(self.out) + (u + self.e) * np.einsum("nsh,nshd->nhd", self.P, np.abs(self.vs))
                + tiny * (1 + np.abs(self.vs).sum(1)) + 1e-30)

    def lse_bound(self):
        return self.e * np.maximum(1.0, np.where(np.isfinite(self.lse), np.abs(self.lse), 0.0))

    def backward(self, grad_out, out=None):
        """{name: (value, sum of |weight| |row|, error in 32 bits, sum of |row|)}, for gradient_bound.  out: the forward result
        that delta is made from (the rounded one that the kernel was given)."""
        g, out = grad_out, self.out if out is None else out
        delta = (g * out).sum(-1)
        dP = np.einsum("nhd,nshd->nsh", g, self.vs)
        dX = self.P * (dP - delta[:, None])
        size = self.P * (np.einsum("nhd,nshd->nsh", np.abs(g), np.abs(self.vs)) + (np.abs(g) * np.abs(out)).sum(-1)[:, None])
        dA = dX * (1 - (self.t / self.cap) ** 2) if self.cap else dX
        n, kv = g.shape[0], self.k.shape[1]

        def to_keys(w, rows):
            full = np.einsum("nsh,nhd->nshd", w, rows).reshape(n, self.s, kv, self.group, -1).sum(3)
            res = np.zeros(self.k.shape)
            np.add.at(res, self.src[self.ok], full[self.ok])
            return res

        to_q = lambda w, ks: self.scale * np.einsum("nsh,nshd->nhd", w, ks)   # noqa: E731
        e = self.e * (16 if self.cap else 4)
        return {
            "grad_q": (to_q(dA, self.ks), to_q(np.abs(dA), np.abs(self.ks)), e * to_q(size, np.abs(self.ks)),
                       to_q(1.0 * (dA != 0), np.abs(self.ks))),
            "grad_k": (self.scale * to_keys(dA, self.q), self.scale * to_keys(np.abs(dA), np.abs(self.q)),
                       e * self.scale * to_keys(size, np.abs(self.q)), self.scale * to_keys(1.0 * (dA != 0), np.abs(self.q))),
            "grad_v": (to_keys(self.P, g), to_keys(self.P, np.abs(g)), e * to_keys(self.P, np.abs(g)),
                       to_keys(1.0 * (self.P != 0), np.abs(g))),
            "grad_bias": (dX.sum(0).T, 0 * dX.sum(0).T, e * size.sum(0).T, 0 * dX.sum(0).T),
        }


def gradient_bound(value, weighted, small, rows, dtype):
    """Weights rounded once to the tensors' type, the result once, all else in 32 bits."""
    u, tiny = roundoff(dtype)
    return u * np.abs(value) + u * weighted + small + tiny * (1 + rows) + 1e-30


def rotary(x, positions, freqs, axes, *, interleaved=False, inverse=False):
    """x: [n][heads][D]; positions: [n][axes]."""
    y, pairs = x.copy(), len(freqs)
    for j in range(pairs):
        w = positions[:, axes[j]].astype(np.float64) * freqs[j] * (-1 if inverse else 1)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
        cos, sin = np.cos(w)[:, None], np.sin(w)[:, None]
        y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., a] * sin + x[..., b] * cos
    return y


def ladder(pairs, n_axes, theta=10000.0):
    """Pairs shared out over the axes, frequencies theta^(-j / count) for each."""
    count = [pairs // n_axes + (a < pairs % n_axes) for a in range(n_axes)]
    axes = [a for a in range(n_axes) for _ in range(count[a])]
    return [theta ** (-j / count[a]) for a in range(n_axes) for j in range(count[a])], axes


def roundoff(dtype):
    """(u, tiny): a value rounds by at most u of it, or by tiny where it is subnormal."""
    return {"float32": (2.0 ** -24, 0.0), "bfloat16": (2.0 ** -8, 0.0), "float16": (2.0 ** -11, 2.0 ** -25)}[str(dtype).replace("torch.", "")]
