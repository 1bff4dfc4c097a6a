"""The router's choice: ids exactly, weights against 64 bits."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _logits(T, E, seed, dtype, kind):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, E, generator=g) * 3
    if kind == "ties":            # few different values, zeros of both signs
        x = torch.round(x)
        x[::2] *= -1.0
    elif kind == "masked":
        x[torch.rand(T, E, generator=g) < 0.6] = -float("inf")
        x[T // 2] = -float("inf")
        x[0, : E - 1] = -float("inf")
    elif kind == "lowest":        # masks of the type's lowest value; a row of nothing else is an even choice
        x[torch.rand(T, E, generator=g) < 0.6] = torch.finfo(dtype).min
        x[T // 2] = torch.finfo(dtype).min
    elif kind == "large":
        x *= 1e4
    return x.to(dtype)


def _run(x_gpu, T, E, k, sigmoid, renormalize, scale):
    ids = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((T, k), 7.0, device=DEV)
    mb.moe_route(x_gpu, k, ids, w, score=mb.MOE_SCORE_SIGMOID if sigmoid else mb.MOE_SCORE_SOFTMAX, renormalize=renormalize, scale=scale)
    return ids.cpu(), w.cpu().double()


def _check(x_gpu, x_cpu, k, sigmoid, renormalize, scale):
    T, E = x_cpu.shape
    ids, w = _run(x_gpu, T, E, k, sigmoid, renormalize, scale)
    want_ids, want = ref.route(x_cpu, k, sigmoid, renormalize, scale)
    assert torch.equal(ids, want_ids)
    assert torch.equal(torch.isnan(w), torch.isnan(want))
    # fp32: exponentials, quotients and the products with the scale a few units in the last place each; sums of E terms in a
    # tree, at most log2(1024) + 4 roundings; an exponent's own rounding (2^-24 relative of up to 88) is inside expf.  Results below
    # 2^-126 may be flushed or rounded in absolute terms.
    tol = 40 * 2.0 ** -24 * want.abs() + 2.0 ** -125
    ok = ~torch.isnan(want)
    assert bool(((w - want).abs() <= tol)[ok].all()), float(((w - want).abs() / tol)[ok].max())


@pytest.mark.parametrize("kind", ["normal", "ties", "masked", "lowest", "large"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 6), (2, 8, 8), (5, 20, 3), (33, 60, 6), (17, 65, 8), (40, 256, 8), (9, 257, 16), (3, 1024, 1), (4, 100, 100),
                                   (2, 1000, 1000)])
def test_route(T, E, k, dtype, kind):
    x = _logits(T, E, T * 1000 + E + k, dtype, kind)
    for sigmoid in (False, True):
        for renormalize in (False, True):
            _check(x.to(DEV), x, k, sigmoid, renormalize, 2.5 if renormalize else 1.0)


def test_many_tokens():
    x = _logits(3001, 160, 4, torch.float32, "ties")
    _check(x.to(DEV), x, 6, False, True, 1.0)


def test_rows_apart():
    wide = _logits(30, 200, 9, torch.float32, "normal")
    _check(wide.to(DEV)[:, 7:135], wide[:, 7:135], 8, False, True, 1.0)
    _check(wide.to(DEV)[::3, :64], wide[::3, :64], 4, True, False, 1.0)
    half = _logits(30, 131, 10, torch.bfloat16, "ties")
    _check(half.to(DEV)[:, 1:], half[:, 1:], 8, False, True, 1.0)


def test_not_a_number():
    """A NaN comes first and makes a softmax row NaN; with a sigmoid it stays with its expert until the weights are renormalised."""
    x = _logits(4, 70, 3, torch.float32, "normal")
    x[0, 68] = float("nan")
    x[1, 3] = float("inf")
    x[2, 3], x[2, 5] = float("nan"), float("nan")
    for sigmoid, renormalize in ((False, True), (False, False), (True, False), (True, True)):
        if sigmoid:
            _check(x.to(DEV), x, 5, True, renormalize, 1.0)
        else:
            ids, w = _run(x.to(DEV), 4, 70, 5, False, renormalize, 1.0)
            want, ww = ref.route(x, 5, False, renormalize, 1.0)
            assert torch.equal(ids, want)
            assert bool(torch.isnan(w[:3]).all()) and not bool(torch.isnan(w[3]).any())


def test_no_tokens():
    assert mb.moe_route(torch.empty(0, 8, device=DEV), 2, torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV)) == mb.MOE_OK
