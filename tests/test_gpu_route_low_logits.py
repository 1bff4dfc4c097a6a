"""Sigmoid scores of rows whose logits are all far below zero: their ratios are what renormalised weights are, long after the scores
themselves leave fp32."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("top", [-10.0, -31.0, -33.0, -60.0, -80.0, -87.0, -89.0, -100.0, -300.0, -650.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,k", [(1, 1), (8, 8), (64, 6), (256, 8), (1000, 70)])
def test_renormalised(E, k, dtype, top):
    g = torch.Generator().manual_seed(E + k)
    T = 5
    x = (top - 20.0 * torch.rand(T, E, generator=g)).to(dtype)
    x[1, E // 2] = -float("inf")
    x[2] = x[2, 0]
    ids, w = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    mb.moe_route(x.to(DEV), k, ids, w, score=mb.MOE_SCORE_SIGMOID, renormalize=True, scale=2.5)
    want_ids, want = ref.route(x, k, True, True, 2.5)
    assert torch.equal(ids.cpu(), want_ids)
    # logits differ by at most 24 (a rounding to bf16 included, 4 at -650), so a difference is rounded by at most 2^-20, 16 * 2^-24 of the
    # exponential; exponential, sum of k <= 70 terms in a tree, quotient and scale: a few units in the last place each, 24 together.  Weights
    # are above 2^-50 of the largest, and the largest at least 2.5 / 70, or 0 (an expert that is masked).
    tol = 40 * 2.0 ** -24 * want + 2.0 ** -100
    assert bool(((w.cpu().double() - want).abs() <= tol).all()), (w.cpu()[:2], want[:2])


def test_scores_that_are_not_renormalised():
    x = torch.tensor([[-20.0, -60.0, -85.0, -100.0, -300.0, -float("inf")]])
    ids, w = torch.empty(1, 6, dtype=torch.int32, device=DEV), torch.empty(1, 6, device=DEV)
    mb.moe_route(x.to(DEV), 6, ids, w, score=mb.MOE_SCORE_SIGMOID, renormalize=False)
    want = torch.sigmoid(x.double())
    assert bool(((w.cpu().double() - want).abs() <= 40 * 2.0 ** -24 * want + 2.0 ** -125).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks(dtype):
    """-inf and the type's lowest value are masks: weight 0 beside others, and rows of nothing else are 0."""
    low = torch.finfo(dtype).min
    x = torch.tensor([[-100.0, low, -101.0, -float("inf")], [low, low, -float("inf"), low], [-200.0, low, low, low]]).to(dtype)
    ids, w = torch.empty(3, 4, dtype=torch.int32, device=DEV), torch.empty(3, 4, device=DEV)
    mb.moe_route(x.to(DEV), 4, ids, w, score=mb.MOE_SCORE_SIGMOID, renormalize=True)
    r = float(torch.exp(x[0, 2].double() - x[0, 0].double()))
    want = torch.tensor([[1 / (1 + r), r / (1 + r), 0, 0], [0, 0, 0, 0], [1, 0, 0, 0]], dtype=torch.float64)
    assert bool(((w.cpu().double() - want).abs() <= 16 * 2.0 ** -24 * want).all()), w
