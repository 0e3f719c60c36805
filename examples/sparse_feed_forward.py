"""A sparse feed-forward block in microscaled 4 bits, as a serving program would hold and run it.

An output projection (rotated, swap vector from a calibration batch) is followed by a router and
gated experts.  Prints how far the block is from the same block in full precision (same 16-bit
inputs, same experts chosen), and the time of a prompt and of a single token.

    python examples/sparse_feed_forward.py [--tokens 2048 --hidden 1152 --ffn 1152 --experts 16 --k 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_24416_gb300 import clq, mx  # noqa: E402


def gated_rows(gate, up):
    """Rows of a gated up projection as MXExperts takes them: 8 of the gate, 8 of the up half, .."""
    E, F, K = gate.shape
    return torch.stack((gate.view(E, F // 8, 8, K), up.view(E, F // 8, 8, K)), 2).view(E, 2 * F, K)


class Block:
    def __init__(self, tokens, hidden, ffn, experts, k, fmt, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        def normal(*shape, std):
            return (std * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
        self.k = k
        scale = torch.ones(hidden, device="cuda")
        scale[torch.randperm(hidden, generator=g, device="cuda")[:max(1, hidden // 100)]] = 30.0
        self.X = (torch.randn((tokens, hidden), generator=g, device="cuda") * scale).to(torch.bfloat16)
        calib = (torch.randn((4, 64, hidden), generator=g, device="cuda") * scale).to(torch.bfloat16)
        self.b = max(b for b in (16, 32, 64) if hidden % b == 0)
        perm, _ = clq.build_permutation_device(clq.outlier_scores(calib))
        self.W = normal(hidden, hidden, std=hidden ** -0.5 / 4)
        self.proj = mx.MXLinear.from_weight(self.W, fmt, perm, self.b)
        self.router = normal(experts, hidden, std=hidden ** -0.5)
        self.gate, self.up = (normal(experts, ffn, hidden, std=hidden ** -0.5) for _ in range(2))
        self.down = normal(experts, hidden, ffn, std=ffn ** -0.5)
        self.experts = mx.MXExperts.from_weights(gated_rows(self.gate, self.up), self.down, fmt)

    def __call__(self, X):
        h = self.proj(X)
        r = mx.route(h @ self.router.t(), self.k)
        return self.experts(h, r), r

    def full_precision(self, X, at):
        h = (X.double() @ self.W.double().t()).to(X.dtype).double()
        p = torch.softmax(h @ self.router.double().t(), 1).gather(1, at.long())
        p = p / p.sum(1, keepdim=True)
        y = torch.zeros_like(h)
        for e in range(self.router.shape[0]):
            t, j = torch.nonzero(at == e, as_tuple=True)
            a = torch.nn.functional.silu(h[t] @ self.gate[e].double().t()) * (h[t] @ self.up[e].double().t())
            y[t] += p[t, j][:, None] * (a @ self.down[e].double().t())
        return y


def micros(fn, n=20):
    fn()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        fn()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) * 1e3 / n


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--hidden", type=int, default=1152)
    p.add_argument("--ffn", type=int, default=1152)
    p.add_argument("--experts", type=int, default=16)
    p.add_argument("--k", type=int, default=2)
    p.add_argument("--format", choices=sorted(mx.FORMATS), default="block32")
    a = p.parse_args(argv)
    block = Block(a.tokens, a.hidden, a.ffn, a.experts, a.k, a.format)
    y, r = block(block.X)
    want = block.full_precision(block.X, r.experts)
    error = float((y.double() - want).norm() / want.norm())
    assert clq.device_status() == 0
    print("%d tokens, %s: relative error %.3f against full precision" % (a.tokens, a.format, error))
    print("prompt %.1f us, one token %.1f us"
          % (micros(lambda: block(block.X)), micros(lambda: block(block.X[:1]))))
    return error


if __name__ == "__main__":
    main()
