"""One attention layer over the tokens of a torus: a training step, then the same rank drawn again as a single new token.

Every rank of a 24 x 20 x 16 volume holds one token, its projections in one buffer [p][q heads + 2 kv heads][head_dim].
Queries and keys are turned by the ranks' coordinates where they lie, every rank attends to its 27 neighbours (and itself)
with a learned bias for each offset, and the gradients come back through both.  All requests are bound once and started
in every step.

    python examples/token_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import iso_inputs as gen
import paper_1606_07676_amd as iso


class TokenLayer:
    def __init__(self, dims, offsets, q_heads, kv_heads, head_dim, dtype=torch.bfloat16, cap=0.0, device="cuda"):
        p = 1
        for n in dims:
            p *= n
        self.comm = iso.iso_neighborhood_create(dims, offsets)
        empty = lambda *size, of=dtype: torch.empty(*size, dtype=of, device=device)          # noqa: E731
        heads = q_heads + 2 * kv_heads
        self.qkv, self.grad_qkv = empty(p, heads, head_dim), empty(p, heads, head_dim)
        self.out, self.grad_out, self.lse = empty(p, q_heads, head_dim), empty(p, q_heads, head_dim), empty(p, q_heads, of=torch.float32)
        self.bias, self.grad_bias = torch.zeros(q_heads, len(offsets), dtype=dtype, device=device), empty(q_heads, len(offsets))
        cut = lambda x: (x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:])       # noqa: E731
        self.q, self.k, self.v = cut(self.qkv)
        grads = cut(self.grad_qkv)
        # the channels' pairs shared out over the three axes
        pairs = head_dim // 2
        count = [pairs // len(dims) + (a < pairs % len(dims)) for a in range(len(dims))]
        self.axes = [a for a in range(len(dims)) for _ in range(count[a])]
        self.freqs = [10000.0 ** (-j / count[a]) for a in range(len(dims)) for j in range(count[a])]
        turn = slice(0, q_heads + kv_heads)
        work = empty(iso.iso_neighbor_attention_backward_workspace_bytes(self.comm, q_heads, kv_heads, head_dim, dtype, bias=True),
                     of=torch.uint8)
        self.turn = iso.iso_rotary_init(self.qkv[:, turn], self.qkv[:, turn], self.freqs, self.axes, self.comm)
        self.attend = iso.iso_neighbor_attention_init(self.q, self.k, self.v, self.out, self.comm, lse=self.lse, bias=self.bias, cap=cap)
        self.attend_back = iso.iso_neighbor_attention_backward_init(
            self.q, self.k, self.v, self.out, self.lse, self.grad_out, *grads, work, self.comm, bias=self.bias,
            grad_bias=self.grad_bias, cap=cap)
        self.turn_back = iso.iso_rotary_init(self.grad_qkv[:, turn], self.grad_qkv[:, turn], self.freqs, self.axes, self.comm,
                                             inverse=True)
        # a single token: which rank, and where it is
        self.row, self.position = torch.zeros(1, dtype=torch.int64, device=device), torch.zeros(1, len(dims), dtype=torch.int32, device=device)
        self.new_q, self.new_out = empty(1, q_heads, head_dim), empty(1, q_heads, head_dim)
        self.turn_one = iso.iso_rotary_init(self.new_q, self.new_q, self.freqs, self.axes, positions=self.position)
        self.attend_one = iso.iso_neighbor_attention_init(self.new_q, self.k, self.v, self.new_out, self.comm, rows=self.row,
                                                          bias=self.bias, cap=cap)

    def forward(self):
        """qkv holds the projections -> out; qkv's queries and keys are turned."""
        iso.iso_start(self.turn)
        iso.iso_start(self.attend)
        return self.out

    def backward(self):
        """grad_out -> grad_qkv (of the projections) and grad_bias."""
        iso.iso_start(self.attend_back)
        iso.iso_start(self.turn_back)
        return self.grad_qkv, self.grad_bias

    def one_token(self, rank, coordinates, q):
        """The attention of one rank whose query is new, over the keys and values that are there."""
        self.row.fill_(rank)
        self.position.copy_(torch.tensor([coordinates], dtype=torch.int32))
        self.new_q.copy_(q)
        iso.iso_start(self.turn_one)
        iso.iso_start(self.attend_one)
        return self.new_out


def main():
    dims, offsets = (24, 20, 16), gen.moore(3, 1) + [(0, 0, 0)]
    layer = TokenLayer(dims, offsets, q_heads=8, kv_heads=2, head_dim=64, cap=30.0)
    torch.manual_seed(0)
    projections = torch.randn_like(layer.qkv)
    target = torch.randn_like(layer.out)
    for step in range(3):                          # the biases learn, the projections stay
        layer.qkv.copy_(projections)
        out = layer.forward()
        loss = (out.float() - target.float()).square().mean()
        layer.grad_out.copy_((2.0 / out.numel() * out.numel() ** 0.5) * (out.float() - target.float()))
        _, grad_bias = layer.backward()
        layer.bias -= (0.02 * grad_bias.float()).to(layer.bias.dtype)
        print(f"step {step}: loss {float(loss):.6f}")
    rank = 5 * 20 * 16 + 7 * 16 + 3
    layer.qkv.copy_(projections)
    out = layer.forward().clone()
    again = layer.one_token(rank, (5, 7, 3), projections[rank:rank + 1, :8])
    print("one token differs from the whole volume's by at most", float((again[0].float() - out[rank].float()).abs().max()))


if __name__ == "__main__":
    main()
