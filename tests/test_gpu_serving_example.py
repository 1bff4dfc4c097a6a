"""The example runs the operators together; a prompt and a step of the same tokens, against the layer in 64 bits."""
import pytest
import torch

from examples import serve_4bit_experts as example
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu


def _layer(X, logits, up, down, k, quantised):
    """out in 64 bits from the weights' 4-bit values; quantised: tokens and activations in 4 bits too."""
    four = (lambda v: ref.quantize(v)[2]) if quantised else (lambda v: v.double())
    ids, p = ref.route(logits, k, False, True, 1.0)
    out = torch.zeros(X.shape, dtype=torch.float64)
    x = four(X)
    inter = down.shape[1]
    for t in range(X.shape[0]):
        for j in range(k):
            y = x[t] @ up[int(ids[t, j])]
            h = (ref.silu(y[:inter]) * y[inter:]).to(torch.bfloat16)
            out[t] += float(p[t, j]) * (four(h[None])[0] @ down[int(ids[t, j])])
    return out


@pytest.mark.parametrize("T,k,E,hidden,inter", [(5, 2, 8, 256, 96), (16, 4, 16, 136, 72)])
def test_prompt_and_step(T, k, E, hidden, inter, monkeypatch):
    packed = []
    pack = example.mb.Mx4Weights.pack_expert
    monkeypatch.setattr(example.mb.Mx4Weights, "pack_expert", lambda self, e, W, *a: (packed.append(W.cpu()), pack(self, e, W, *a))[1])
    w = example.Experts(E, hidden, inter, seed=T)
    values = [ref.quantize(W.T.contiguous())[2].T for W in packed]       # blocks of 32 along K
    up, down = torch.stack(values[0::2]), torch.stack(values[1::2])
    X = torch.randn(T, hidden, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
    logits = (X.to("cuda:0") @ w.router).cpu()
    prompt, step = example.Prompt(T, k, w), example.Step(T, k, w)
    for out, quantised in ((prompt.forward(X.to("cuda:0")), True), (step.forward(X.to("cuda:0")), False), (step.forward(X.to("cuda:0")), False)):
        want = _layer(X, logits, up, down, k, quantised)
        apart = float((out.cpu().double() - want).norm() / want.norm())
        # bf16 rounds outputs (and a quantised layer's products): 2^-9 on average of each, four times that allowed; where an activation's bf16
        # value turns on a sum's last bits its 4-bit value moves by a step, up to a third of it, which few of them do: 1 % of the norm
        assert apart <= (2.0 ** -7 + 0.01 if quantised else 2.0 ** -7), apart


def test_command_line(capsys):
    assert example.main(["--experts", "8", "--topk", "2", "--hidden", "256", "--inter", "128", "--prompt", "40", "--batch", "4", "--steps", "3"]) < 0.6
    assert "prompt of 40" in capsys.readouterr().out
