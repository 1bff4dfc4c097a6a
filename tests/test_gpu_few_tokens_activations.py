"""The layer for few tokens over bf16 weights: activations between its two products are not rounded to the 8 bits of bf16."""
import pytest
import torch

from tests import helpers as H
from tests import mx4_reference as ref
from tests.test_gpu_few_tokens import _inputs, _run

pytestmark = pytest.mark.gpu


def _expected(X, logits, up, down, k):
    """Output in 64 bits and a bound: fp32 sums of hidden (inter, twice: two halves) exact products in any order, an activation as two bf16 halves,
    the router's weights and the sum over the experts in fp32, the output rounded to bf16 once.  bf16 has 8 significant bits: rounding to nearest is off by
    half a unit, 2^-8 of the value at most; an activation's second half has 2^-8 of it to hold and is off by 2^-8 of that."""
    ids, w = ref.route(logits, k, False, True, 1.0)
    U, D, x = up.double(), down.double(), X.double()
    T, hidden, inter = X.shape[0], X.shape[1], down.shape[1]
    out, tol, mag = (torch.zeros(T, hidden, dtype=torch.float64) for _ in range(3))
    c1, c2 = H.sum_err_coeff(hidden + 64, False), H.sum_err_coeff(2 * inter + 64, False)
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            y, err = x[t] @ U[e], c1 * (x[t].abs() @ U[e].abs())
            g, u, eg, eu = y[:inter], y[inter:], err[:inter], err[inter:]
            h = ref.silu(g) * u
            eh = 1.1 * eg * (u.abs() + eu) + ref.silu(g).abs() * eu + 32 * 2.0 ** -24 * h.abs()
            eh = eh + 2.0 ** -16 * (h.abs() + eh) + 2.0 ** -130
            z, A = h @ D[e], h.abs() @ D[e].abs()
            ez = eh @ D[e].abs() + 1.01 * c2 * (A + eh @ D[e].abs())
            p = float(w[t, j])
            out[t] += p * z
            mag[t] += p * (z.abs() + ez)
            tol[t] += p * ez
    tol += mag * (k + 64) * 2.0 ** -24 + 2.0 ** -8 * out.abs() + 2.0 ** -130
    return out, tol


@pytest.mark.parametrize("T,k,E,hidden,inter", [(1, 1, 1, 8, 8), (1, 6, 64, 256, 176), (3, 3, 5, 264, 40), (5, 2, 8, 512, 384), (8, 1, 2, 1024, 128), (15, 2, 8, 640, 1000),
                                                (16, 8, 300, 64, 64), (16, 2, 3, 2048, 520), (8, 2, 16, 72, 2048)])
def test_bound_without_the_rounding(T, k, E, hidden, inter):
    X, logits, up, down = _inputs(T, E, hidden, inter, T + inter)
    got = _run(X, logits, up, down, k, False)[0].double()
    want, tol = _expected(X, logits, up, down, k)
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((got - want).abs() / tol).max()))
    # of many outputs, the rounding itself: uniform over a unit 2^(e - 7) on the mean square a twelfth of its square, values of a binade m 2^e with log m
    # uniform 3 / (2 log 2) 2^(2 e): 1.5e-3 of the norm, up to 1.7e-3 by the values' distribution
    if got.numel() >= 1024:
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -9


def test_infinite_activations_stay_infinite():
    """gate 8, up beyond fp32: h is infinite, and so is what finite weights make of it; its low half must not turn it into NaN."""
    T, hidden, inter = 2, 8, 8
    X = torch.full((T, hidden), 1.0).to(torch.bfloat16)
    up = torch.ones(1, hidden, 2 * inter)
    up[:, :, inter] = 1e38                        # sums to 8e38
    up[:, :, inter + 1] = 4.2e37                  # sums to 3.36e38, times silu(8) beyond fp32
    up[:, :, inter + 2] = 5.2e36                  # sums to 4.2e37, times silu(8) 3.3e38: a number in fp32
    down = torch.zeros(1, inter, hidden)
    down[:, 2:] = 1.0
    down[:, :2] = 2.0
    down[:, :, 4:] = 1e-6
    got = _run(X, torch.zeros(T, 1), up.to(torch.bfloat16), down.to(torch.bfloat16), 1, False)[0]
    assert bool((got == float("inf")).all()), got
    up[:, :, inter: inter + 2] = 1.0
    got = _run(X, torch.zeros(T, 1), up.to(torch.bfloat16), down.to(torch.bfloat16), 1, False)[0]
    assert bool(torch.isfinite(got[:, 4:]).all()), got
    want = float(ref.silu(torch.tensor(8.0, dtype=torch.float64))) * 8 * float(up[0, 0, inter + 2].to(torch.bfloat16)) * float(torch.tensor(1e-6).to(torch.bfloat16))
    assert bool(((got[:, 4:].double() - want).abs() <= 2.0 ** -8 * want).all()), (got, want)
