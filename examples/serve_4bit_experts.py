"""One mixture-of-experts layer with 4-bit experts, as a server would run it: the experts are packed once, a prompt goes through the
grouped products, then single tokens (or a small batch of them) through the layer for few tokens, from a graph.

    python examples/serve_4bit_experts.py [--experts 64 --topk 6 --hidden 2048 --inter 1408 --prompt 512 --batch 1 --steps 64]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2501_16103_amd import binding as mb  # noqa: E402


class Experts:
    """The layer's weights: the router's in bf16, the experts' in 4 bits."""

    def __init__(self, E, hidden, inter, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape, scale: (torch.randn(*shape, generator=g, device=device) * scale).to(torch.bfloat16)
        self.E, self.hidden, self.inter = E, hidden, inter
        self.router = normal(hidden, E, scale=hidden ** -0.5)
        self.up = mb.Mx4Weights(E, hidden, 2 * inter, gated=True, device=device)
        self.down = mb.Mx4Weights(E, inter, hidden, device=device)
        for e in range(E):          # one expert at a time: the bf16 weights of a whole layer need not be there at once
            self.up.pack_expert(e, normal(hidden, 2 * inter, scale=hidden ** -0.5))
            self.down.pack_expert(e, normal(inter, hidden, scale=inter ** -0.5))


class Prompt:
    """A layer's step for T tokens: router, gate+up product with the activation, down product, weighted sum."""

    def __init__(self, T, k, w, device="cuda:0"):
        self.T, self.k, self.w = T, k, w
        self.ids = torch.empty(T, k, dtype=torch.int32, device=device)
        self.weights = torch.empty(T, k, device=device)
        self.up = mb.MoeMx4ProductPlan(T, k, w.E, w.hidden, 2 * w.inter, gated=True, device=device)
        self.down = mb.MoeMx4ProductPlan(T * k, 1, w.E, w.inter, w.hidden, device=device)   # every activated row is a token of one expert
        self.out = torch.empty(T, w.hidden, dtype=torch.bfloat16, device=device)

    def forward(self, X):
        w, T, k = self.w, self.T, self.k
        mb.moe_route(X @ w.router, k, self.ids, self.weights)
        h = self.up.forward(X, w.up, self.ids)
        y = self.down.forward(h.view(T * k, w.inter), w.down, self.ids.view(T * k, 1))
        mb.moe_combine(y, self.weights, T, k, w.hidden, self.out)
        return self.out


class Step:
    """The same for at most 16 tokens: two launches, and with the router's product one graph."""

    def __init__(self, T, k, w, device="cuda:0"):
        self.w = w
        self.x = torch.zeros(T, w.hidden, dtype=torch.bfloat16, device=device)
        self.logits = torch.empty(T, w.E, dtype=torch.bfloat16, device=device)
        self.plan = mb.MoeFewTokensPlan(T, k, w.E, w.hidden, w.inter, device=device)
        self._run()                                  # (libraries set themselves up outside the capture)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._run()

    def _run(self):
        torch.matmul(self.x, self.w.router, out=self.logits)
        self.plan.forward(self.x, self.logits, self.w.up, self.w.down)

    def forward(self, X):
        self.x.copy_(X)
        self.graph.replay()
        return self.plan.out


def timed(f, n):
    f()
    torch.cuda.synchronize()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(n):
        f()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) * 1e3 / n


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("experts", 64), ("topk", 6), ("hidden", 2048), ("inter", 1408), ("prompt", 512), ("batch", 1), ("steps", 64)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    w = Experts(a.experts, a.hidden, a.inter)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    X = torch.randn(a.prompt, a.hidden, generator=g, device="cuda:0").to(torch.bfloat16)
    prompt, step = Prompt(a.prompt, a.topk, w), Step(a.batch, a.topk, w)
    out = prompt.forward(X).float()
    # the prompt's first tokens again, as a step: the products round their tokens to 4 bits, the step does not
    n = min(a.batch, a.prompt)
    x = torch.zeros(a.batch, a.hidden, dtype=torch.bfloat16, device="cuda:0")
    x[:n] = X[:n]
    again = step.forward(x)[:n].float()
    apart = float((again - out[:n]).norm() / again.norm())
    weights = w.up.codes.numel() + w.up.scales.numel() + w.down.codes.numel() + w.down.scales.numel()
    print(f"{a.experts} experts, {a.hidden} / {a.inter}, {weights / 1e6:.0f} MB in 4 bits")
    print(f"prompt of {a.prompt}: {timed(lambda: prompt.forward(X), 20):.1f} us;  step of {a.batch}: {timed(lambda: step.forward(x), a.steps):.1f} us;  "
          f"the two apart by {apart:.3f} of the output's norm (the prompt's tokens in 4 bits)")
    return apart


if __name__ == "__main__":
    main()
