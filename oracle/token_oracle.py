"""Plain definitions, in numpy and 64 bits, of the operators on each token by itself: layer norm and the gated projections
with their gradients, and dropout.  Nothing is shared with the library.  The bounds say how far a result of 32-bit
arithmetic, rounded once to elements with the unit roundoff u, may be off, element by element."""
import math

import numpy as np

EPS = 2.0 ** -24
TINY = {2.0 ** -24: 2.0 ** -126, 2.0 ** -9: 2.0 ** -126, 2.0 ** -8: 2.0 ** -126, 2.0 ** -11: 2.0 ** -25}


def rounded(value, error, u, tiny=None):
    """Bound after rounding value +- error to elements with unit roundoff u; f16 rounds what is below 2^-14 by up to 2^-25.
    tiny: by how much instead, for elements that are kept scaled."""
    return error + u * (np.abs(value) + error) + (TINY[u] if tiny is None else tiny)


class LayerNorm:
    """x: [rows][channels] float64; weight, bias: [channels] or None."""

    def __init__(self, x, weight=None, bias=None, eps=1e-5):
        self.x = x
        self.w = np.ones(x.shape[1]) if weight is None else weight
        self.b = np.zeros(x.shape[1]) if bias is None else bias
        self.mean = x.mean(1)
        d = x - self.mean[:, None]
        self.rstd = (np.mean(d * d, 1) + eps) ** -0.5
        self.h = d * self.rstd[:, None]
        self.out = self.h * self.w + self.b

    # A sum over a row takes at most 16 additions in a lane, 6 over a wavefront's lanes and 16 over the wavefronts, 38 in all,
    # each off by EPS of at most the sum of the absolute values, which for the distances from the mean is one standard
    # deviation an element or less.  Twice: the mean, and what it is off by.  The distances are exact to EPS of themselves.
    def h_error(self):
        return EPS * 64 * (1 + np.abs(self.h))

    def mean_bound(self):
        return EPS * (2 * np.abs(self.mean) + 64 / self.rstd) + 2.0 ** -126

    def rstd_bound(self):
        return EPS * 64 * self.rstd

    def out_bound(self, u):
        return rounded(self.out, self.h_error() * np.abs(self.w) + 4 * EPS * (np.abs(self.h * self.w) + np.abs(self.b)), u)

    def backward(self, dy):
        g = dy * self.w
        one = lambda v: v.mean(1, keepdims=True)  # noqa: E731
        r = self.rstd[:, None]
        self.grad_x = r * (g - one(g) - self.h * one(g * self.h))
        self.grad_weight, self.grad_bias = (dy * self.h).sum(0), dy.sum(0)
        # each of the three terms: its products, the errors of h and rstd, and the two means' sums as above
        self.grad_x_error = EPS * 160 * r * (np.abs(g) + one(np.abs(g)) + (1 + np.abs(self.h)) * one(np.abs(g) * (1 + np.abs(self.h))))
        # rows go to at least 128 sums, or one row each where there are fewer, which are then added up
        n = 64 + 160 + dy.shape[0] / 128
        self.grad_weight_error = EPS * n * (np.abs(dy) * (1 + np.abs(self.h))).sum(0)
        self.grad_bias_error = EPS * n * np.abs(dy).sum(0)


def philox(counter, more, key, rounds=10):
    """Blocks of four 32-bit words: counter an array of 64-bit numbers, more and key 64-bit numbers."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    counter = np.asarray(counter, dtype=np.uint64)
    c = [counter & low, counter >> half, np.full_like(counter, more & 0xFFFFFFFF), np.full_like(counter, more >> 32)]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(rounds):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


def kept(n, channels, seed, rate):
    """[n][channels] whether an element is kept, and the factor of what is."""
    count = n * channels
    words = philox(np.arange((count + 7) // 8), seed[1] % 2 ** 64, seed[0] % 2 ** 64)
    numbers = np.stack([words & 0xFFFF, words >> 16], -1).reshape(-1)[:count].reshape(n, channels)
    t = math.floor(float(np.float32(rate)) * 65536 + 0.5)
    return numbers >= t, 65536 / (65536 - t) if t < 65536 else 0.0


class Gated:
    """x: [n][channels], gate, up: [hidden][channels], float64; fast: the 16-bit kernels' exponential and reciprocal."""

    def __init__(self, x, gate, up, activation, fast):
        self.x, self.gate, self.up = x, gate, up
        self.g, self.u = x @ gate.T, x @ up.T
        if activation == "silu":
            s = np.where(self.g >= 0, 1, np.exp(np.minimum(self.g, 0))) / (1 + np.exp(-np.abs(self.g)))
            rest = np.where(self.g >= 0, np.exp(-np.maximum(self.g, 0)), 1) / (1 + np.exp(-np.abs(self.g)))
            self.f, self.slope = self.g * s, s + self.g * s * rest
        else:
            s = 0.5 * np.vectorize(math.erfc, otypes=[float])(-self.g * math.sqrt(0.5))
            self.f, self.slope = self.g * s, s + self.g * np.exp(-0.5 * self.g ** 2) / math.sqrt(2 * math.pi)
        self.out = self.f * self.u
        # a dot of K terms in 32 bits, in any order
        K = x.shape[1]
        self.g_error, self.u_error = EPS * (K + 2) * (np.abs(x) @ np.abs(gate).T), EPS * (K + 2) * (np.abs(x) @ np.abs(up).T)
        # exp(-g) and exp(-g^2 / 2) are off by the rounding of their argument and a few units more, and so is what they give
        e = EPS * (8 + (4 if fast else 2) * np.minimum(np.abs(self.g), 100) ** (1 if activation == "silu" else 2))
        self.f_error = 1.2 * self.g_error + e * np.abs(self.f) + 2.0 ** -126     # |f'| is below 1.13
        self.slope_error = self.g_error + 2 * e                                  # |f''| is below 0.8

    def out_bound(self, u):
        return rounded(self.out, self.f_error * (np.abs(self.u) + self.u_error) + np.abs(self.f) * self.u_error + 2 * EPS * np.abs(self.out), u)

    def backward(self, dy, u, tiny=None):
        """u: of the tensors' type, to which the gradients of g and u are rounded on the way; tiny: as for rounded."""
        self.d_gate, self.d_up = dy * self.u * self.slope, dy * self.f
        e_gate = rounded(self.d_gate, np.abs(dy) * (self.u_error * (np.abs(self.slope) + self.slope_error) + np.abs(self.u) * self.slope_error) + 2 * EPS * np.abs(self.d_gate), u, tiny)
        e_up = rounded(self.d_up, np.abs(dy) * self.f_error + EPS * np.abs(self.d_up), u, tiny)
        a, b = np.abs(self.d_gate) + e_gate, np.abs(self.d_up) + e_up
        sums = lambda n: EPS * (n + 18)  # noqa: E731  terms, and the splits of a sum
        F, n = self.gate.shape[0], self.x.shape[0]
        self.grad_x = self.d_gate @ self.gate + self.d_up @ self.up
        self.grad_x_error = (e_gate + sums(2 * F) * a) @ np.abs(self.gate) + (e_up + sums(2 * F) * b) @ np.abs(self.up)
        self.grad_gate, self.grad_up = self.d_gate.T @ self.x, self.d_up.T @ self.x
        self.grad_gate_error = (e_gate + sums(n) * a).T @ np.abs(self.x)
        self.grad_up_error = (e_up + sums(n) * b).T @ np.abs(self.x)
