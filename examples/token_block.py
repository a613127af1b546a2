"""One block of a model over the tokens of a torus: a training step, then a few tokens by themselves.

Every rank of a 12 x 10 x 8 volume holds one token.  Its row is normalised and projected; queries and keys are normalised head
by head and turned by the rank's coordinates; every rank attends to its 27 neighbours; what comes out joins the token with
dropout.  The feed-forward block does the same with its two gated projections and the one back.  Plain projections are
torch's; all requests are bound once and started in every step, and a step's masks follow from the step's number.

    python examples/token_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import iso_inputs as gen
import paper_1606_07676_amd as iso


class TokenBlock:
    def __init__(self, dims, offsets, channels, q_heads, kv_heads, head_dim, hidden, rate=0.1, activation="silu", dtype=torch.bfloat16,
                 device="cuda"):
        n = 1
        for size in dims:
            n *= size
        self.comm = iso.iso_neighborhood_create(dims, offsets)
        empty = lambda *size, of=dtype: torch.empty(*size, dtype=of, device=device)          # noqa: E731
        bytes_ = lambda size: empty(max(1, size), of=torch.uint8)                            # noqa: E731
        heads, turned, D = q_heads + 2 * kv_heads, q_heads + kv_heads, head_dim
        shapes = {"norm1": (channels,), "bias1": (channels,), "qkv": (heads * D, channels), "norm_qk": (D,), "out": (channels, q_heads * D),
                  "norm2": (channels,), "bias2": (channels,), "gate": (hidden, channels), "up": (hidden, channels), "down": (channels, hidden)}
        self.weights = {name: empty(*shape) for name, shape in shapes.items()}
        self.grads = {name: empty(*shape) for name, shape in shapes.items()}
        w, g = self.weights, self.grads
        with torch.no_grad():
            for name, x in w.items():
                x.fill_(0.0 if name.startswith("bias") else 1.0) if x.dim() == 1 else x.normal_(std=x.shape[1] ** -0.5)
        rows = lambda width: empty(n, width)                                                 # noqa: E731
        self.x, self.a, self.qkv, self.qk, self.o, self.p = rows(channels), rows(channels), empty(n, heads, D), empty(n, turned, D), empty(n, q_heads, D), rows(channels)
        self.h, self.b, self.f, self.d, self.y = rows(channels), rows(channels), rows(hidden), rows(channels), rows(channels)
        self.dy, self.dd, self.df, self.db, self.dh, self.dp = rows(channels), rows(channels), rows(hidden), rows(channels), rows(channels), rows(channels)
        self.do, self.dqk, self.dqkv, self.da, self.dx = empty(n, q_heads, D), empty(n, turned, D), empty(n, heads, D), rows(channels), rows(channels)
        self.lse = empty(n, q_heads, of=torch.float32)
        self.seeds = torch.tensor([[1, 0], [2, 0]], dtype=torch.int64, device=device)        # one for each dropout
        stat = lambda *size: (empty(*size, of=torch.float32), empty(*size, of=torch.float32))  # noqa: E731
        (m1, r1), (mq, rq), (m2, r2) = stat(n), stat(n, turned), stat(n)
        pairs = D // 2
        count = [pairs // len(dims) + (i < pairs % len(dims)) for i in range(len(dims))]
        axes = [i for i in range(len(dims)) for _ in range(count[i])]
        freqs = [100.0 ** (-j / count[i]) for i in range(len(dims)) for j in range(count[i])]
        cut = lambda x: (x[:, :q_heads], x[:, q_heads:])                                     # noqa: E731
        (q, k), v, dv = cut(self.qk), self.qkv[:, turned:], self.dqkv[:, turned:]
        norm_work = [bytes_(iso.iso_layer_norm_backward_workspace_bytes(n, h, c, dtype)) for h, c in ((1, channels), (turned, D))]
        attention_work = bytes_(iso.iso_neighbor_attention_backward_workspace_bytes(self.comm, q_heads, kv_heads, D, dtype))
        gated_work = bytes_(iso.iso_gated_backward_workspace_bytes(n, channels, hidden, dtype))
        self.steps = {
            "norm1": iso.iso_layer_norm_init(self.x, self.a, weight=w["norm1"], bias=w["bias1"], mean=m1, rstd=r1),
            "norm_qk": iso.iso_layer_norm_init(self.qkv[:, :turned], self.qk, weight=w["norm_qk"], mean=mq, rstd=rq),
            "turn": iso.iso_rotary_init(self.qk, self.qk, freqs, axes, self.comm),
            "attend": iso.iso_neighbor_attention_init(q, k, v, self.o, self.comm, lse=self.lse),
            "join1": iso.iso_dropout_init(self.p, self.h, self.seeds[0], rate, residual=self.x),
            "norm2": iso.iso_layer_norm_init(self.h, self.b, weight=w["norm2"], bias=w["bias2"], mean=m2, rstd=r2),
            "gated": iso.iso_gated_init(self.b, w["gate"], w["up"], self.f, activation=activation),
            "join2": iso.iso_dropout_init(self.d, self.y, self.seeds[1], rate, residual=self.h),
            "join2_back": iso.iso_dropout_init(self.dy, self.dd, self.seeds[1], rate),
            "gated_back": iso.iso_gated_backward_init(self.b, w["gate"], w["up"], self.df, self.db, g["gate"], g["up"], gated_work,
                                                      activation=activation),
            "norm2_back": iso.iso_layer_norm_backward_init(self.h, m2, r2, self.db, self.dh, norm_work[0], weight=w["norm2"],
                                                           grad_weight=g["norm2"], grad_bias=g["bias2"]),
            "join1_back": iso.iso_dropout_init(self.dh, self.dp, self.seeds[0], rate),
            "attend_back": iso.iso_neighbor_attention_backward_init(q, k, v, self.o, self.lse, self.do, *cut(self.dqk), dv, attention_work, self.comm),
            "turn_back": iso.iso_rotary_init(self.dqk, self.dqk, freqs, axes, self.comm, inverse=True),
            "norm_qk_back": iso.iso_layer_norm_backward_init(self.qkv[:, :turned], mq, rq, self.dqk, self.dqkv[:, :turned], norm_work[1],
                                                             weight=w["norm_qk"], grad_weight=g["norm_qk"]),
            "norm1_back": iso.iso_layer_norm_backward_init(self.x, m1, r1, self.da, self.dx, norm_work[0], weight=w["norm1"],
                                                           grad_weight=g["norm1"], grad_bias=g["bias1"]),
        }
        # a few tokens by themselves: the feed-forward half on rows of their own
        self.few_h, self.few_b, self.few_f = empty(4, channels), empty(4, channels), empty(4, hidden)
        self.few = (iso.iso_layer_norm_init(self.few_h, self.few_b, weight=w["norm2"], bias=w["bias2"]),
                    iso.iso_gated_init(self.few_b, w["gate"], w["up"], self.few_f, activation=activation))

    def run(self, *names):
        for name in names:
            iso.iso_start(self.steps[name])

    def forward(self, step):
        """x -> y, with the masks of this step."""
        w = self.weights
        self.seeds[:, 1] = step
        self.run("norm1")
        torch.mm(self.a, w["qkv"].t(), out=self.qkv.flatten(1))
        self.run("norm_qk", "turn", "attend")
        torch.mm(self.o.flatten(1), w["out"].t(), out=self.p)
        self.run("join1", "norm2", "gated")
        torch.mm(self.f, w["down"].t(), out=self.d)
        self.run("join2")
        return self.y

    def backward(self):
        """dy -> dx and the weights' gradients; the masks are those of the last step."""
        w, g = self.weights, self.grads
        self.run("join2_back")
        torch.mm(self.dd.t(), self.f, out=g["down"])
        torch.mm(self.dd, w["down"], out=self.df)
        self.run("gated_back", "norm2_back")
        self.dh += self.dy
        self.run("join1_back")
        torch.mm(self.dp.t(), self.o.flatten(1), out=g["out"])
        torch.mm(self.dp, w["out"], out=self.do.flatten(1))
        self.run("attend_back", "turn_back", "norm_qk_back")
        torch.mm(self.dqkv.flatten(1).t(), self.a, out=g["qkv"])
        torch.mm(self.dqkv.flatten(1), w["qkv"], out=self.da)
        self.run("norm1_back")
        self.dx += self.dh
        return self.dx

    def feed_forward_of(self, rows):
        """The feed-forward half, without dropout, of four rows."""
        self.few_h.copy_(rows)
        for request in self.few:
            iso.iso_start(request)
        return self.few_h + self.few_f @ self.weights["down"].t()


def main():
    torch.manual_seed(0)
    block = TokenBlock((12, 10, 8), gen.moore(3, 1) + [(0, 0, 0)], channels=256, q_heads=4, kv_heads=2, head_dim=64, hidden=704)
    x, target = torch.randn_like(block.x), torch.randn_like(block.x)
    for step in range(3):
        block.x.copy_(x)
        y = block.forward(step)
        loss = (y.float() - target.float()).square().mean()
        block.dy.copy_(2 * (y.float() - target.float()) / y.shape[1])
        block.backward()
        for name, weight in block.weights.items():
            weight -= (0.001 * block.grads[name].float()).to(weight.dtype)
        print(f"step {step}: loss {float(loss):.6f}")
    again = block.feed_forward_of(block.h[5:9])
    print("rows by themselves:", tuple(again.shape), "finite:", bool(again.isfinite().all()))


if __name__ == "__main__":
    main()
